"""The flow decoder with options on the GPU against the fp64 oracle: per-head
norms and rotation, the carry in 4 bits, both.

Bounds.  Without the 4-bit carry, those of the plain decoder.  With it, an
element whose value lies next to a border between two codes may be held as the
neighbouring one: with values off by d of themselves that is at most a fraction
f = 2 d 12 of them (a value is at most 12 half steps), each one step off, whose
RMS against the rounding error that every element has (0.29 steps) is
sqrt(f) / 0.29.  So a call's mel may be that share of what the 4-bit carry
itself changes in the oracle, E, further off: d = 1e-5 in fp32 (0.05 E) and
2^-8 in bf16 (1.06 E).
"""
import numpy as np
import pytest

import oracle
from paper_2609_35115_amd import synth
from tests.gpu_common import TOL, bits_equal, err_stats, say
from tests.test_gpu_flow import SEED, _carry_ok, _flow, _prompts, _run_gpu, _run_oracle

pytestmark = pytest.mark.gpu

TINY = synth.TINY_FLOW_ARCH
QK = dict(qk_norm=1, rope_dims=64, rope_base=10000.0, qk_eps=1e-6)
SHARE = {"f32": (2 * 1e-5 * 12) ** 0.5 / 0.29, "bf16": (2 * 2.0 ** -8 * 12) ** 0.5 / 0.29}
OPTIONS = {"qk": QK, "qk16": dict(QK, rope_dims=16, rope_base=100.0), "norm": dict(QK, rope_dims=0), "carry4": dict(carry_bits=4),
           "qk_carry4": dict(QK, carry_bits=4)}


def _check(arch, dtype, blob, b, outs, mu, prompt, calls):
    """Every call of stream b against the oracle; returns the oracle's stream."""
    s, ref = _run_oracle(arch, dtype, blob, b, prompt, mu, calls)
    wide = [None] * len(ref)
    if arch.get("carry_bits"):
        _, wide = _run_oracle(dict(arch, carry_bits=0), dtype, blob, b, prompt, mu, calls)
    for k, (g, r, w) in enumerate(zip(outs, ref, wide)):
        e, er = err_stats(g[b], r)
        tol = TOL[dtype] + (SHARE[dtype] * err_stats(w, r)[0] if w is not None else 0.0)
        say(f"  stream {b} call {k}: max-abs/RMS {e:.3e} of {tol:.3e}, RMS {er:.3e}")
        assert e <= tol, f"stream {b} call {k}: {e:.3e} > {tol:.3e}"
    return s


def _audit(dec, s, arch, dtype, b, at):
    """The carry read back: the operand type within the plain decoder's bound;
    4 bits equal but for elements next to a border (first step and block, which
    no attention reaches) and each at most a step and a half of its group off."""
    for (i, l, c, kv) in at:
        got, want = dec.carry(b, i, l, c, kv), s.carry(i, l, c, kv)
        assert got.shape == want.shape
        if not arch.get("carry_bits"):
            ok, e = _carry_ok(got, want, dtype)
            assert ok, f"carry {(b, i, l, c, kv)}: {e:.3e}"
        elif i == 0 and l == 0:
            off = got != want
            say(f"  carry {(b, i, l, c, kv)}: {off.mean():.2e} of the elements differ")
            assert off.mean() <= SHARE[dtype] ** 2 * 0.29 ** 2
            top = np.abs(want).reshape(-1, 32).max(1, keepdims=True)
            assert (np.abs(got - want).reshape(-1, 32) <= top).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", list(OPTIONS))
def test_tiny_chunks_match_oracle(name, dtype):
    a = dict(TINY, **OPTIONS[name])
    blob = synth.make_flow_weights(a, 0)
    calls = [a["f_call"]] * 5
    say(f"flow tiny {name} {dtype}")
    dec, outs, mu, prompts = _run_gpu(a, dtype, blob, 2, a["f_prompt"], calls)
    st = dec.stats()
    assert st["replays"] == 5 and st["direct"] == 0, st
    for b in range(2):
        s = _check(a, dtype, blob, b, outs, mu[b], prompts[b], calls)
        _audit(dec, s, a, dtype, b, [(0, 0, 0, 0), (0, 0, 1, 1), (0, 0, 1, 0), (a["n_steps"] - 1, a["depth"] - 1, 1, 1)])
    dec.close()


@pytest.mark.parametrize("name", ["qk", "qk_carry4"])
def test_partial_calls_flush_and_new_turn(name):
    """Calls of other sizes, flushes that change no state, prompts of different
    lengths, and a new turn over what an earlier one left."""
    a = dict(TINY, **OPTIONS[name])
    blob = synth.make_flow_weights(a, 0)
    fc = a["f_chunk"]
    calls = [a["f_call"], fc, 3, fc + 1, 1, a["f_call"], 2, fc, fc]
    prompts = [synth.make_flow_prompt(a, P, seed=1, stream=b) for b, P in enumerate((13, 20))]
    dec, outs, mu, _ = _run_gpu(a, "f32", blob, 2, 13, calls, prompts=prompts)
    for b in range(2):
        _check(a, "f32", blob, b, outs, mu[b], prompts[b], calls)
    dec.prompt(0, *synth.make_flow_prompt(a, 7, seed=4))
    again = dec.decode(mu[:, :a["f_call"]]).cpu().numpy()
    flow = _flow()
    fresh = flow.FlowDecoder(a, "f32", blob, 2, rng_seed=SEED)
    fresh.prompt(0, *synth.make_flow_prompt(a, 7, seed=4))
    fresh.prompt(1, *prompts[1])
    assert bits_equal(again[0], fresh.decode(mu[:, :a["f_call"]]).cpu().numpy()[0])
    dec.close()


@pytest.mark.parametrize("shape", [
    dict(f_retained=0),                                            # the ring holds a call's own frames only
    dict(f_chunk=1, f_call=1, f_retained=3, f_prompt=1),           # single frames
    dict(f_chunk=7, f_call=40, f_retained=42, f_prompt=37, heads=1, dim=64),   # a long lookahead, six slots
    dict(f_chunk=70, f_call=75, f_retained=140, f_prompt=500, depth=1, n_steps=2),   # wide blocks, a prompt longer than the ring
], ids=["no_history", "single", "lookahead", "long"])
def test_clock_shapes_match_oracle(shape):
    a = dict(TINY, **OPTIONS["qk_carry4"], **shape)
    blob = synth.make_flow_weights(a, 3)
    calls = [a["f_call"]] * 4 + [max(1, a["f_chunk"] - 1), a["f_chunk"]]
    dec, outs, mu, prompts = _run_gpu(a, "f32", blob, 2, a["f_prompt"], calls)
    for b in range(2):
        s = _check(a, "f32", blob, b, outs, mu[b], prompts[b], calls)
        _audit(dec, s, a, "f32", b, [(0, 0, 0, 0), (0, 0, 1, 1)])
    dec.close()


@pytest.mark.parametrize("name", ["qk", "carry4", "qk_carry4"])
def test_replay_equals_direct_and_batch(name):
    flow = _flow()
    a = dict(TINY, **OPTIONS[name])
    blob = synth.make_flow_weights(a, 2)
    calls = [a["f_call"]] * 4
    prompts = _prompts(a, 5, a["f_prompt"])
    d, o, mu, _ = _run_gpu(a, "bf16", blob, 5, a["f_prompt"], calls, prompts=prompts)
    _, o1, _, _ = _run_gpu(a, "bf16", blob, 5, a["f_prompt"], calls, flags=flow.DC_NO_GRAPH, prompts=prompts, mu=mu)
    _, o2, _, _ = _run_gpu(a, "bf16", blob, 1, a["f_prompt"], calls, prompts=prompts[:1], mu=mu[:1])
    for x, y, z in zip(o, o1, o2):
        assert bits_equal(x, y) and bits_equal(x[0], z[0])
    assert d.stats()["kernels_per_call"] == len_launches(a)


def len_launches(a):
    """Kernels of a call: assemble, per step (in, per block qkv, heads, attention, o, fc1, fc2, then out, Euler), advance."""
    return 1 + a["n_steps"] * (3 + a["depth"] * 6) + 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_match_oracle(dtype):
    """24 streams: the many-row GEMM, and attention in its other shapes."""
    a = dict(TINY, **OPTIONS["qk_carry4"])
    blob = synth.make_flow_weights(a, 5)
    calls = [a["f_call"]] * 3
    dec, outs, mu, prompts = _run_gpu(a, dtype, blob, 24, a["f_prompt"], calls)
    for b in (0, 11, 23):
        _check(a, dtype, blob, b, outs, mu[b], prompts[b], calls)
    dec.close()


@pytest.mark.parametrize("name", ["qk", "qk_carry4"])
def test_real_shape_matches_oracle(name):
    """The paper-shaped decoder in bf16 with a 302-frame prompt: three calls, the
    last past the first cut of the carry; the 4-bit carry's size."""
    a = dict(synth.REAL_FLOW_ARCH, **OPTIONS[name])
    blob = synth.make_flow_weights(a, 0)
    calls = [a["f_call"]] * 3
    say(f"flow real {name} bf16")
    dec, outs, mu, prompts = _run_gpu(a, "bf16", blob, 1, a["f_prompt"], calls)
    s = _check(a, "bf16", blob, 0, outs, mu[0], prompts[0], calls)
    assert s.extent == 402
    _audit(dec, s, a, "bf16", 0, [(0, 0, 0, 0), (0, 0, 1, 1)] + ([] if a.get("carry_bits") else [(9, 15, 0, 1)]))
    if a.get("carry_bits"):
        st = dec.stats()
        assert st["carry_live_bytes"] == 10 * 16 * 4 * 402 * 8 * 34 and st["carry_bytes"] < 1.15 * st["carry_live_bytes"]
    dec.close()
