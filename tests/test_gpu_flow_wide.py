"""The flow decoder's chunk calls over the 4-bit carry in the attention's wide
blocks (a CPU test holds the calls to them), against the fp64 oracle: the paper's
call at 16 streams with few blocks and steps, and keys that are split.

Bound.  Values off by d of themselves are held as a neighbouring code in a share
f = 24 d of the elements; against the rounding that every element has, 0.29
steps, that is sqrt(f) / 0.29 of the change E that the 4-bit carry makes in the
oracle.  In the first block of the first step d is the arithmetic's, 1e-5 (fp32) or
2^-8 (bf16).  Each later one's values are off by what the flips before it make of
them too: d' = d + sqrt(24 d) / 0.29 E (E as an RMS).  So one block and step, where
nothing follows a flip, is held to the first share, more to the last of theirs."""
import numpy as np
import pytest

from paper_2609_35115_amd import synth
from tests.carry4_plan import plan
from tests.gpu_common import TOL, err_stats, say
from tests.test_gpu_flow import _prompts, _run_gpu, _run_oracle
from tests.test_gpu_flow_options import QK, _audit

pytestmark = pytest.mark.gpu

B = 16
SPLIT = dict(synth.TINY_FLOW_ARCH, f_chunk=70, f_call=75, f_retained=420, f_prompt=500, carry_bits=4, **QK)
# architecture; the plan of a chunk call and of a prompt pass of all its frames
ARCHS = {
    "paper": (dict(synth.REAL_FLOW_ARCH, depth=2, n_steps=2, carry_bits=4, **QK), (64, 1), (64, 2)),
    "paper_once": (dict(synth.REAL_FLOW_ARCH, depth=1, n_steps=1, carry_bits=4, **QK), (64, 1), (64, 2)),
    "split": (dict(SPLIT, depth=2, n_steps=2), (64, 3), (16, 2)),
    "split_once": (dict(SPLIT, depth=1, n_steps=1), (64, 3), (16, 2)),
}
STEP = {"f32": 1e-5, "bf16": 2.0 ** -8}


def _bound(dtype, blocks, worst, rms):
    d = STEP[dtype]
    for _ in range(blocks - 1):
        d = STEP[dtype] + (24 * d) ** 0.5 / 0.29 * rms
    return TOL[dtype] + (24 * d) ** 0.5 / 0.29 * worst


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", list(ARCHS))
def test_chunk_calls_match_oracle(name, dtype):
    a = ARCHS[name][0]
    blob = synth.make_flow_weights(a, 7)
    calls = [a["f_call"]] * (8 if a["f_retained"] == 420 else 4)   # past the retained chunks
    prompts = _prompts(a, B, a["f_prompt"])
    prompts[3] = synth.make_flow_prompt(a, a["f_prompt"] // 3, seed=2, stream=3)
    dec, outs, mu, _ = _run_gpu(a, dtype, blob, B, a["f_prompt"], calls, prompts=prompts)
    for b in (0, 3, B - 1):
        s, ref = _run_oracle(a, dtype, blob, b, prompts[b], mu[b], calls)
        _, wide = _run_oracle(dict(a, carry_bits=0), dtype, blob, b, prompts[b], mu[b], calls)
        for k, (g, r, w) in enumerate(zip(outs, ref, wide)):
            e, rms = err_stats(g[b], r)
            tol = _bound(dtype, a["depth"] * a["n_steps"], *err_stats(w, r))
            say(f"  {name} {dtype} stream {b} call {k}: max-abs/RMS {e:.3e} of {tol:.3e}, RMS {rms:.3e}")
            assert np.isfinite(g[b]).all() and e <= tol
        _audit(dec, s, a, dtype, b, [(0, 0, 0, 0), (0, 0, 1, 1)])
    dec.close()


@pytest.mark.parametrize("B", [1, 2, 16])
def test_every_length_has_its_workspace(B):
    """Prompt passes and chunk calls of lengths whose keys are split differently:
    none needs more than the state has placed (such a call is refused), and a split
    result is finite."""
    a = dict(SPLIT, depth=1, n_steps=1)
    plans = {plan(e, n, 2, 2, 64, 500, 420, 495, "bf16") for e, most in ((2 * B, 75), (2, 500)) for n in range(1, most + 1)}
    assert len(plans) > 1 and max(s for _, s in plans) > 1
    dec, _, mu, _ = _run_gpu(a, "bf16", synth.make_flow_weights(a, 1), B, a["f_prompt"], [])
    for n in list(range(1, 76)):
        assert np.isfinite(dec.decode(mu[:, :n]).cpu().numpy()).all(), n
    for frames in (1, 2, 15, 16, 17, 31, 33, 64, 65, 100, 128, 129, 250, 499, 500):
        dec.prompt(B - 1, *synth.make_flow_prompt(a, frames, seed=frames))
        assert np.isfinite(dec.decode(mu[:, :75]).cpu().numpy()).all(), frames
    dec.close()
