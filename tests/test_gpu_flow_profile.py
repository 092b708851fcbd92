"""dc_flow_profile's launches, with each option and with a split attention."""
import pytest

from paper_2609_35115_amd import flow, synth
from tests.test_gpu_flow import _run_gpu

pytestmark = pytest.mark.gpu

QK = dict(qk_norm=1, rope_dims=64, rope_base=10000.0, qk_eps=1e-6)
LONG = dict(f_chunk=70, f_call=75, f_retained=140, f_prompt=500, depth=1, n_steps=2)   # the attention's keys are split


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("options", [{}, QK, dict(carry_bits=4), dict(QK, carry_bits=4)], ids=["plain", "qk", "carry4", "qk_carry4"])
@pytest.mark.parametrize("shape", [{}, LONG], ids=["tiny", "long"])
def test_launches_add_up(shape, options, dtype):
    """The roles' launches are a call's kernels but for the state's advance, which
    a profile leaves out; the attention's join is one of its own."""
    a = dict(synth.TINY_FLOW_ARCH, **options, **shape)
    dec, _, _, _ = _run_gpu(a, dtype, synth.make_flow_weights(a, 0), 1, a["f_prompt"], [a["f_call"]])
    prof = {r["name"]: r for r in dec.profile(2)}
    assert sum(r["launches"] for r in prof.values()) == dec.stats()["kernels_per_call"] - 1
    blocks = a["depth"] * a["n_steps"]
    split = bool(a.get("carry_bits")) and shape is LONG
    assert prof["attn"]["launches"] == blocks * (2 if split else 1)
    assert all(r["us"] > 0 for r in prof.values())
    dec.close()
