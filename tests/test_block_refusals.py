"""The transformer-block operators without a GPU: what the entry points refuse on the host, and the rotary frequencies."""
import ctypes
import math

import pytest

from paper_2602_00608_b200 import binding as vd
from paper_2602_00608_b200 import build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


P = ctypes.c_void_p(4096)                        # an address that is checked and never followed


def xattn(**kw):
    d = dict(struct_size=ctypes.sizeof(vd.VdXattnDesc), dtype=vd.VD_BF16, batch=2, q_len=3, kv_len=5, heads=4, kv_heads=2, head_dim=64, impl=0, scale=0.125,
             q_batch=768, q_token=256, q_head=64, k_batch=640, k_token=128, k_head=64, v_batch=640, v_token=128, v_head=64,
             o_batch=768, o_token=256, o_head=64)
    d.update(kw)
    return vd.VdXattnDesc(**d)


def test_struct_sizes_match_the_header_layout():
    assert ctypes.sizeof(vd.VdXattnDesc) == 40 + 12 * 8
    assert ctypes.sizeof(vd.VdRotaryDesc) == 56 + 9 * 8
    assert ctypes.sizeof(vd.VdRotaryFreqDesc) == 32 + 5 * 8
    assert ctypes.sizeof(vd.VdGateNormDesc) == 56 + 14 * 8


@pytest.mark.parametrize("change", [
    dict(struct_size=8), dict(dtype=2), dict(batch=-1), dict(q_len=-1), dict(kv_len=-1), dict(heads=0), dict(kv_heads=0), dict(heads=5),
    dict(head_dim=0), dict(head_dim=257), dict(impl=9), dict(impl=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan),
    dict(q_token=-1), dict(o_batch=-5), dict(o_token=0), dict(o_head=63), dict(o_batch=0), dict(o_batch=767),
    dict(batch=1 << 20, q_len=1 << 20), dict(batch=1 << 15, heads=1 << 14, kv_heads=1, q_len=4),
    dict(kv_len=(1 << 25) + 1), dict(batch=1, heads=2, kv_heads=2, q_len=(1 << 29) + 1),
])
def test_cross_attention_refuses(change):
    assert vd.lib().vd_op_cross_attention(ctypes.byref(xattn(**change)), P, P, P, None, P, None) == vd.VD_ERR_INVALID_ARG
    assert vd.lib().vd_last_error(None)


def test_cross_attention_refuses_pointers():
    l, d = vd.lib(), ctypes.byref(xattn())
    odd = ctypes.c_void_p(4097)
    assert l.vd_op_cross_attention(None, P, P, P, None, P, None) == vd.VD_ERR_INVALID_ARG
    for args in ((None, P, P, None, P), (P, None, P, None, P), (P, P, None, None, P), (P, P, P, None, None), (odd, P, P, None, P),
                 (P, odd, P, None, P), (P, P, odd, None, P), (P, P, P, ctypes.c_void_p(4098), P), (P, P, P, None, odd)):
        assert l.vd_op_cross_attention(d, *args, None) == vd.VD_ERR_INVALID_ARG


@pytest.mark.parametrize("change", [dict(batch=0), dict(q_len=0)])
def test_cross_attention_of_nothing_is_done(change):
    assert vd.lib().vd_op_cross_attention(ctypes.byref(xattn(**change)), None, None, None, None, None, None) == vd.VD_OK


def rotary(**kw):
    pairs = (ctypes.c_int32 * 4)(*kw.pop("axis_pairs", (32, 0, 0, 0)))
    d = dict(struct_size=ctypes.sizeof(vd.VdRotaryDesc), dtype=vd.VD_BF16, batch=2, tokens=3, heads=4, head_dim=80, rotary_dim=64, layout=0, axes=1,
             axis_pairs=pairs, amplitude=1.0, x_batch=960, x_token=320, x_head=80, y_batch=960, y_token=320, y_head=80, pos_batch=3, pos_token=1,
             first_position=0)
    d.update(kw)
    return vd.VdRotaryDesc(**d)


@pytest.mark.parametrize("change", [
    dict(struct_size=0), dict(dtype=-1), dict(batch=-1), dict(tokens=-1), dict(heads=-1), dict(head_dim=0), dict(head_dim=1025), dict(rotary_dim=63),
    dict(rotary_dim=82, axis_pairs=(41, 0, 0, 0)), dict(rotary_dim=-2), dict(layout=2), dict(axes=0), dict(axes=5), dict(axis_pairs=(31, 0, 0, 0)),
    dict(axes=2, axis_pairs=(33, -1, 0, 0)), dict(amplitude=math.nan), dict(amplitude=math.inf), dict(y_head=79), dict(x_token=-1), dict(pos_batch=-1),
    dict(batch=1 << 16, tokens=1 << 16),
])
def test_rotary_refuses(change):
    assert vd.lib().vd_op_rotary(ctypes.byref(rotary(**change)), P, P, P, ctypes.c_void_p(1 << 20), None) == vd.VD_ERR_INVALID_ARG
    assert vd.lib().vd_last_error(None)


def test_rotary_refuses_pointers():
    l, y = vd.lib(), ctypes.c_void_p(1 << 20)
    d = rotary()
    for args in ((None, P, P, y), (P, P, None, y), (P, P, P, None), (ctypes.c_void_p(4097), P, P, y), (P, ctypes.c_void_p(4098), P, y), (P, P, ctypes.c_void_p(4100), y)):
        assert l.vd_op_rotary(ctypes.byref(d), *args, None) == vd.VD_ERR_INVALID_ARG
    assert l.vd_op_rotary(None, P, P, P, y, None) == vd.VD_ERR_INVALID_ARG
    assert l.vd_op_rotary(ctypes.byref(rotary(x_token=640, x_batch=1920)), P, P, P, P, None) == vd.VD_ERR_INVALID_ARG            # in place, other strides
    assert l.vd_op_rotary(ctypes.byref(rotary(axes=2, axis_pairs=(16, 16, 0, 0))), P, None, P, y, None) == vd.VD_ERR_INVALID_ARG  # axes without positions
    assert l.vd_op_rotary(ctypes.byref(rotary(first_position=1 << 50)), P, None, P, y, None) == vd.VD_ERR_INVALID_ARG
    assert l.vd_op_rotary(ctypes.byref(rotary(batch=0)), None, None, None, None, None) == vd.VD_OK


def gate_norm(**kw):
    d = dict(struct_size=ctypes.sizeof(vd.VdGateNormDesc), batch=2, tokens=6, channels=64, x_dtype=0, h_dtype=1, y_dtype=1, mod_dtype=1, norm=0, post_norm=0,
             mod_tokens=3, eps=1e-6, residual_scale=1.0, x_batch=384, x_token=64, h_batch=384, h_token=64, xo_batch=384, xo_token=64, y_batch=384, y_token=64,
             gate_batch=128, gate_group=64, scale_batch=128, scale_group=64, shift_batch=128, shift_group=64)
    d.update(kw)
    return vd.VdGateNormDesc(**d)


X, H, XO, Y = (ctypes.c_void_p(1 << 20 | i << 12) for i in range(4))


@pytest.mark.parametrize("change", [
    dict(struct_size=4), dict(batch=-1), dict(tokens=-1), dict(channels=0), dict(channels=16385), dict(x_dtype=2), dict(h_dtype=2), dict(y_dtype=-1),
    dict(mod_dtype=7), dict(norm=2), dict(post_norm=2), dict(mod_tokens=0), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(residual_scale=math.inf),
    dict(x_token=-64), dict(xo_token=63), dict(y_batch=0), dict(batch=1 << 16, tokens=1 << 16),
])
def test_gate_norm_refuses(change):
    assert vd.lib().vd_op_gate_norm(ctypes.byref(gate_norm(**change)), X, H, None, P, XO, P, P, P, P, Y, None) == vd.VD_ERR_INVALID_ARG
    assert vd.lib().vd_last_error(None)


def test_gate_norm_refuses_what_does_not_go_together():
    l = vd.lib()
    call = lambda d, x=X, h=H, post=None, gate=P, xo=XO, w=P, b=P, sc=P, sh=P, y=Y: l.vd_op_gate_norm(ctypes.byref(d), x, h, post, gate, xo, w, b, sc, sh, y, None)
    bad = vd.VD_ERR_INVALID_ARG
    d = gate_norm()
    assert l.vd_op_gate_norm(None, X, H, None, P, XO, P, P, P, P, Y, None) == bad
    assert call(d, x=None) == bad
    assert call(d, h=None) == bad and call(gate_norm(post_norm=1), h=None, gate=None) == bad                      # gate, norm of h without h
    assert call(d, post=P) == bad                                                                                 # its weight without the norm
    assert call(d, y=None) == bad and call(d, y=None, w=None, b=None, sc=None, sh=None, xo=None) == bad
    assert call(d, xo=H) == bad and call(d, xo=Y) == bad and call(d, y=X) == bad
    assert call(gate_norm(xo_token=128, xo_batch=768), xo=X) == bad                                               # in place, other strides
    assert call(gate_norm(y_dtype=0), y=H) == bad                                                                 # over h in another type
    for name in ("x", "h", "xo", "w", "b", "sc", "sh", "y", "gate"):
        assert call(d, **{name: ctypes.c_void_p((1 << 24) + 1)}) == bad, name
    assert l.vd_op_gate_norm(ctypes.byref(gate_norm(tokens=0)), None, None, None, None, XO, None, None, None, None, None, None) == vd.VD_OK


# ---- frequencies (host-only)
def test_rotary_frequencies_are_the_formula():
    f = vd.rotary_frequencies(64, 10000.0)
    assert f.shape == (32,) and all(abs(float(f[i]) * 2 * math.pi / 10000.0 ** (-i / 32) - 1) < 1e-14 for i in range(32))
    f = vd.rotary_frequencies(20, 500.0, axis_pairs=(4, 3, 3))
    want = [500.0 ** (-i / n) / (2 * math.pi) for n in (4, 3, 3) for i in range(n)]
    assert all(abs(float(a) / b - 1) < 1e-14 for a, b in zip(f, want))
    assert vd.rotary_frequencies(0).shape == (0,)


def test_rotary_frequencies_scaled_for_long_contexts():
    plain = vd.rotary_frequencies(128, 10000.0)
    lin = vd.rotary_frequencies(128, 10000.0, scaling=vd.VD_ROTARY_SCALE_LINEAR, factor=4.0)
    assert (lin * 4 / plain - 1).abs().max() < 1e-14
    base = vd.rotary_frequencies(128, 10000.0, scaling=vd.VD_ROTARY_SCALE_BASE, factor=8.0)
    assert abs(float(base[0] / plain[0]) - 1) < 1e-14 and abs(float(base[-1] / plain[-1]) * 8 - 1) < 1e-12 and (base[1:-1] < plain[1:-1]).all()
    parts = vd.rotary_frequencies(128, 10000.0, scaling=vd.VD_ROTARY_SCALE_PARTS, factor=8.0, original_len=8192, fast=32.0, slow=1.0)
    for i in range(64):
        turns, ratio = 8192 * float(plain[i]), float(parts[i] / plain[i])
        w = min(max((turns - 1) / 31, 0), 1)
        assert abs(ratio - (w + (1 - w) / 8)) < 1e-13
    assert float(parts[0] / plain[0]) == 1.0 and abs(float(parts[-1] / plain[-1]) - 0.125) < 1e-15
    one = vd.rotary_frequencies(2, 10000.0, scaling=vd.VD_ROTARY_SCALE_BASE, factor=8.0)       # one pair: nothing to move
    assert abs(float(one[0]) * 2 * math.pi - 1) < 1e-15


@pytest.mark.parametrize("kw", [dict(rotary_dim=63), dict(rotary_dim=-2), dict(base=1.0), dict(base=math.inf), dict(scaling=4), dict(axis_pairs=(16, 15)),
                                dict(axis_pairs=(33, -1)), dict(axis_pairs=(8,) * 5), dict(scaling=1, factor=0.5), dict(scaling=2, factor=math.inf),
                                dict(scaling=3, factor=2.0), dict(scaling=3, factor=2.0, original_len=100.0, fast=1.0, slow=1.0)])
def test_rotary_frequencies_refuse(kw):
    args = dict(rotary_dim=64)
    args.update(kw)
    with pytest.raises(vd.VdError) as e:
        vd.rotary_frequencies(args.pop("rotary_dim"), args.pop("base", 10000.0), **args)
    assert e.value.status == vd.VD_ERR_INVALID_ARG


def test_the_wrappers_refuse_tensors_that_are_not_on_a_device():
    import torch
    q = torch.zeros(1, 2, 2, 8)
    for call in (lambda: vd.op_cross_attention(q, q, q), lambda: vd.op_rotary(q, torch.zeros(4, dtype=torch.float64)), lambda: vd.op_gate_norm(q[0], q[0])):
        with pytest.raises(vd.VdError) as e:
            call()
        assert e.value.status == vd.VD_ERR_INVALID_ARG and "device" in str(e.value)


def test_the_wrappers_refuse_sizes_that_would_wrap():
    """2^31 + 5 tokens of stride 0 as an int32 would be a negative number, 2^32 + 5 would be five."""
    import torch
    big = torch.zeros(1).expand(1, 2 ** 32 + 5, 1, 8)
    ok = torch.zeros(1, 2, 1, 8)
    for call in (lambda: vd._describe_cross_attention(ok, big, big, None, None, ok, 0), lambda: vd._describe_cross_attention(big, ok, ok, None, None, big, 0),
                 lambda: vd._describe_rotary(big, torch.zeros(4, dtype=torch.float64), None, "half", None, 1.0, 0, big),
                 lambda: vd._describe_rotary(ok, torch.zeros(4, dtype=torch.float64), None, "half", None, 1.0, 1 << 63, ok),
                 lambda: vd._describe_gate_norm(big[:, :, 0], None, None, None, None, "rms", 1e-6, None, None, False, None, 1.0, None, big[:, :, 0], None),
                 lambda: vd._describe_gate_norm(ok[:, :, 0], None, None, None, None, "rms", 1e-6, None, None, False, None, 1.0, 1 << 32, ok[:, :, 0], None)):
        with pytest.raises(vd.VdError) as e:
            call()
        assert e.value.status == vd.VD_ERR_INVALID_ARG and "device" not in str(e.value)


@pytest.mark.parametrize("which", range(3))
def test_cross_attention_refuses_an_output_that_is_an_input(which):
    """Rows are read while others are written."""
    at = [ctypes.c_void_p(4096 * (i + 1)) for i in range(3)]
    assert vd.lib().vd_op_cross_attention(ctypes.byref(xattn()), *at, None, at[which], None) == vd.VD_ERR_INVALID_ARG
    assert b"o is an input" in vd.lib().vd_last_error(None)


@pytest.mark.parametrize("heads", [(1 << 30) + 1, (1 << 31) - 1])
def test_rotary_refuses_heads_that_would_wrap(heads):
    """A thread steps over the heads by up to 1024: an int32 would turn negative behind the last of 2^31 - 1, and the thread go on there."""
    far = dict(batch=1, tokens=1, heads=heads, head_dim=8, rotary_dim=8, axis_pairs=(4, 0, 0, 0), x_head=0, y_head=8, y_token=8 * heads, y_batch=8 * heads)
    assert vd.lib().vd_op_rotary(ctypes.byref(rotary(**far)), P, P, P, ctypes.c_void_p(1 << 20), None) == vd.VD_ERR_INVALID_ARG
    assert b"rotary sizes" in vd.lib().vd_last_error(None)


def test_cross_attention_refuses_scales_that_overflow_in_units_of_log_2():
    l = vd.lib()
    for scale in (8.6e37, 3e38):
        assert l.vd_op_cross_attention(ctypes.byref(xattn(scale=scale)), P, P, P, None, ctypes.c_void_p(1 << 20), None) == vd.VD_ERR_INVALID_ARG
        assert b"scale" in l.vd_last_error(None)
    for scale in (2.0 ** 126, 1e-45):
        assert l.vd_op_cross_attention(ctypes.byref(xattn(scale=scale, batch=0)), None, None, None, None, None, None) == vd.VD_OK


def test_heads_without_channels_are_refused_by_the_library(monkeypatch):
    """Where no scale is given one follows from the number of channels, which may be none."""
    import torch
    monkeypatch.setattr(vd, "_on_device", lambda *a, **kw: None)
    x = torch.zeros(1, 2, 2, 0)
    desc = vd._describe_cross_attention(x, x, x, None, None, x, vd.VD_XATTN_AUTO)
    assert vd.lib().vd_op_cross_attention(ctypes.byref(desc), P, P, P, None, ctypes.c_void_p(1 << 20), None) == vd.VD_ERR_INVALID_ARG
    assert b"sizes" in vd.lib().vd_last_error(None)
