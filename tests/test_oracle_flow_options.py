"""The flow oracle's options on the CPU: per-head norm and rotation and the
4-bit values against independent arithmetic, what a carry holds, and the
refusals of dc_flow_init_opt before any device call."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import paper_2609_35115_amd as dc
from paper_2609_35115_amd import flow, synth

TINY = synth.TINY_FLOW_ARCH
QK = dict(qk_norm=1, rope_dims=64, rope_base=10000.0, qk_eps=1e-6)


@pytest.mark.parametrize("rope_dims,position", [(64, 0), (64, 1), (64, 12345), (16, 77), (0, 5)])
def test_norm_and_rotation(rope_dims, position):
    rng = np.random.default_rng(1)
    x, gain = rng.standard_normal(64), rng.standard_normal(64)
    got = oracle.qk(x, gain, 1e-6, rope_dims, 10000.0, position)
    t = torch.tensor(x)
    y = torch.nn.functional.rms_norm(t, (64,), torch.tensor(gain), 1e-6).numpy().copy()
    h = rope_dims // 2
    if h:   # as complex numbers of the pairs
        f = (10000.0 ** (-np.arange(h) / h)).astype(np.float32).astype(np.float64)
        z = (y[:h] + 1j * y[h:2 * h]) * np.exp(1j * position * f)
        y[:h], y[h:2 * h] = z.real, z.imag
    assert np.abs(got - y).max() < 1e-11


def test_rotation_depends_on_distance_only():
    rng = np.random.default_rng(2)
    q, k, one = rng.standard_normal(64), rng.standard_normal(64), np.ones(64)
    s = [oracle.qk(q, one, 0.0, 64, 10000.0, p + 9) @ oracle.qk(k, one, 0.0, 64, 10000.0, p) for p in (0, 3, 1000)]
    assert np.ptp(s) < 1e-10


def test_held_values():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((300, 32)) * 10.0 ** rng.uniform(-30, 30, (300, 1))
    x[0], x[1, 1:] = 0.0, 0.0
    x[2] = np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], 4)   # ties, to the even code
    got = oracle.hold4(x.ravel()).reshape(x.shape)
    assert np.array_equal(got[2][:8], [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]) and not got[0].any()
    top = np.abs(x).max(1, keepdims=True)
    with np.errstate(divide="ignore"):
        e = np.where(top > 0, np.ceil(np.log2(top / 6)), -126)
    a = np.abs(x) / 2.0 ** e
    assert a.max() <= 6 and (a.max(1)[3:] > 3).all()
    grid = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    near = np.abs(a[..., None] - grid).min(-1)
    assert np.allclose(np.abs(np.abs(got) / 2.0 ** e - a), near, atol=1e-12)
    assert np.array_equal(oracle.hold4(got.ravel()), got.ravel())   # held values are held as they are


def _first_carry(a):
    s = oracle.FlowStream(a, "f32", synth.make_flow_weights(a, 0), seed=5, key=0)
    s.prompt(*synth.make_flow_prompt(a, a["f_prompt"]))
    s.chunk(synth.make_flow_mu(a, 1, a["f_call"])[0])
    return [s.carry(0, 0, c, kv) for c in (0, 1) for kv in (0, 1)]   # before any attention has been read


def test_what_the_carry_holds():
    """The first block's keys and values at the first step depend on no
    attention: with options they are the plain ones, normalised, rotated by
    their frame's position, and held in 4 bits."""
    plain = _first_carry(TINY)
    a = dict(TINY, **QK)
    gains = synth.split_flow_weights(a, synth.make_flow_weights(a, 0))["qk.gain"]
    assert np.array_equal(synth.make_flow_weights(a, 0)[:synth.flow_blob_floats(TINY)], synth.make_flow_weights(TINY, 0))
    P, fc = a["f_prompt"], a["f_chunk"]
    frames = list(range(P, P + fc)) + list(range(P))   # the newest chunk in front of the prompt
    want = [x.copy() for x in plain]
    for x in want[::2]:
        for r, p in enumerate(frames):
            for h in range(a["heads"]):
                x[r, 64 * h:64 * h + 64] = oracle.qk(x[r, 64 * h:64 * h + 64], gains[0, 1], 1e-6, 64, 10000.0, p)
    for got, w in zip(_first_carry(a), want):
        assert np.array_equal(got, w)
    for arch, ref in ((dict(TINY, carry_bits=4), plain), (dict(a, carry_bits=4), want)):
        for got, w in zip(_first_carry(arch), ref):
            assert np.array_equal(got, oracle.hold4(w.ravel()).reshape(w.shape))


def test_without_rotation_and_with_no_effect():
    """Equal gains scale both sides alike, and a decoder whose options are all off is the plain one."""
    for off in (dict(carry_bits=0), dict(qk_norm=0, rope_dims=0)):
        for x, y in zip(_first_carry(TINY), _first_carry(dict(TINY, **off))):
            assert np.array_equal(x, y)


def _status(arch, blob, **bad):
    opt = flow.make_flow_opt(arch)
    for k, v in bad.items():
        setattr(opt, k, v)
    cfg, h = flow.make_flow_cfg(arch, "f32", 2), ctypes.c_void_p()
    st = flow.flib().dc_flow_init_opt(blob.ctypes.data, blob.nbytes, ctypes.byref(cfg), ctypes.byref(opt), ctypes.byref(h))
    return st, flow.dc_flow_last_error(None), flow.dc_flow_blob_floats(cfg, opt)


def test_init_refuses_bad_options_before_any_device_call():
    a = dict(TINY, **QK)
    blob = synth.make_flow_weights(a, 0)
    assert flow.dc_flow_blob_floats(flow.make_flow_cfg(a, "f32", 2), flow.make_flow_opt(a)) == blob.size
    assert flow.dc_flow_blob_floats(flow.make_flow_cfg(a, "f32", 2)) == synth.flow_blob_floats(TINY)
    assert _status(a, blob, abi_version=0)[0] == dc.DC_EVERSION
    for k, v, word in [("carry_bits", 8, "carry_bits"), ("qk_norm", 2, "qk_norm"), ("rope_dims", 8, "rope_dims"),
                       ("rope_dims", 80, "rope_dims"), ("rope_dims", -16, "rope_dims"), ("qk_norm", 0, "qk_norm"),
                       ("rope_base", 0.0, "rope_base"), ("rope_base", float("inf"), "rope_base"), ("qk_eps", -1.0, "qk_eps"),
                       ("qk_eps", float("nan"), "qk_eps")]:
        st, msg, floats = _status(a, blob, **{k: v})
        assert st == dc.DC_EINVAL and word in msg and floats == 0, (k, v, st, msg)
    st, msg, _ = _status(a, blob[:-1])
    assert st == dc.DC_EINVAL and "blob size" in msg
    st, msg, _ = _status(dict(TINY, carry_bits=4), blob)   # gains that no option asks for
    assert st == dc.DC_EINVAL and "blob size" in msg
    with pytest.raises(ValueError):
        oracle.FlowStream(TINY, "f32", blob)


def test_carry_sizes():
    """What a stream's carry takes on the host's own account: 34 bytes per head,
    frame and key or value against 128 (bf16), slots padded."""
    a = synth.REAL_FLOW_ARCH
    regions = 2 * 2 * a["heads"] * a["depth"] * a["n_steps"] // 2   # (step, block, branch, head)
    slots = a["f_prompt"] + a["f_retained"] + a["f_call"]
    four = regions * ((slots * 68 + 255) // 256 * 256)
    bf16 = 2 * regions * (304 + 3 * 56) * 128
    assert bf16 == 309_329_920 and 3.7 < bf16 / four < 3.9
