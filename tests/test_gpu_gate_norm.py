"""The seam of two blocks (gated residual add, modulated norm) against the definition in 64 bits."""
import itertools

import pytest

from tests import block_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vd():
    from paper_2602_00608_b200 import binding
    return binding


def _t(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def make(b, t, c, groups, x="f32", h="bf16", mod="bf16", seed=0, offset=0.5):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    mods = (0.3 * r(b, groups, 3, c)).to(_t(mod))
    return dict(x=(2 * r(b, t, c) + offset).to(_t(x)), h=r(b, t, c).to(_t(h)), gate=mods[:, :, 0], scale=mods[:, :, 1], shift=mods[:, :, 2],
                weight=1 + 0.1 * r(c), bias=0.1 * r(c), post_weight=1 + 0.1 * r(c))


def run(vd, a, **kw):
    import torch
    r, y = vd.op_gate_norm(**a, **kw)
    torch.cuda.synchronize()
    kw = {k: v for k, v in kw.items() if k not in ("x_out", "y", "want_x", "want_y")}
    want_r, br, want_y, by = block_ref.gate_norm(**a, **kw, x_dtype=None if r is None else r.dtype, y_dtype=None if y is None else y.dtype)
    if r is not None:
        block_ref.check(r, want_r, br)
    if y is not None:
        block_ref.check(y, want_y, by)
    return r, y


SIZES = [(1, 1, 64, 1), (8, 1, 1920, 1), (2, 37, 1920, 5), (3, 11, 1111, 11), (1, 5, 8, 2), (2, 3, 1, 3), (1, 2, 16384, 1), (1, 3, 8191, 2), (2, 9, 512, 4),
         (1, 4, 2048, 4), (2, 2, 4104, 1), (1, 130, 72, 13), (1, 7, 5000, 7), (1, 3, 100, 1), (1, 2, 12288, 2)]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("types", [("f32", "bf16", "bf16"), ("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("f32", "bf16", "f32")], ids="-".join)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_gate_norm_matches_the_definition(vd, kind, post, types, size):
    b, t, c, mod_tokens = size
    a = make(b, t, c, -(-t // mod_tokens), *types)
    if not post:
        a["post_weight"] = None
    run(vd, a, kind=kind, post_norm=post, residual_scale=0.7, mod_tokens=mod_tokens)


@pytest.mark.parametrize("size", [(2, 5, 192, 3), (1, 4, 333, 4)], ids=str)
@pytest.mark.parametrize("left_out", list(itertools.chain(
    [("gate",), ("scale",), ("shift",), ("weight",), ("bias",), ("post_weight",)], [("gate", "scale", "shift"), ("weight", "bias", "post_weight"),
                                                                             ("gate", "scale", "shift", "weight", "bias", "post_weight")])), ids="-".join)
def test_what_is_left_out(vd, size, left_out):
    b, t, c, m = size
    a = make(b, t, c, -(-t // m))
    a.update({n: None for n in left_out})
    run(vd, a, post_norm=True, mod_tokens=m)
    run(vd, {**a, "post_weight": None}, mod_tokens=m, kind="rms", want_x=False)
    run(vd, {**a, "scale": None, "shift": None, "weight": None, "bias": None}, post_norm=True, mod_tokens=m, want_y=False)
    run(vd, {**a, "h": None, "gate": None, "post_weight": None}, mod_tokens=m)                      # the first norm of a model
    run(vd, {**a, "h": None, "gate": None, "post_weight": None}, mod_tokens=m, want_x=False)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("size", [(2, 9, 256, 9), (1, 6, 1111, 2), (1, 3, 4096, 1)], ids=str)
def test_in_place_and_slices(vd, kind, size):
    import torch
    b, t, c, m = size
    a = make(b, t, c, -(-t // m))
    a["post_weight"] = None
    r, y = run(vd, a, kind=kind, mod_tokens=m)
    x, h = a["x"].clone(), a["h"].clone()
    got = vd.op_gate_norm(**{**a, "x": x, "h": h}, kind=kind, mod_tokens=m, x_out=x, y=h)
    torch.cuda.synchronize()
    assert got[0] is x and got[1] is h and torch.equal(x, r) and torch.equal(h, y)
    for pad in (8, 3):                                             # rows at aligned and odd places; a modulation that the batch shares
        wide = {n: torch.full((b, t, c + 2 * pad), 4.0, device="cuda", dtype=a[n].dtype) for n in ("x", "h")}
        out = {n: v.clone() for n, v in wide.items()}
        for n in wide:
            wide[n][..., pad:pad + c] = a[n]
        shared = {n: a[n][:1].expand(b, *a[n].shape[1:]) for n in ("gate", "scale", "shift")}
        s = {**a, **shared, "x": wide["x"][..., pad:pad + c], "h": wide["h"][..., pad:pad + c]}
        run(vd, s, kind=kind, mod_tokens=m, x_out=out["x"][..., pad:pad + c], y=out["h"][..., pad:pad + c])
        assert all((v[..., :pad] == 4).all() and (v[..., pad + c:] == 4).all() for v in out.values())


@pytest.mark.parametrize("c", [64, 1111, 1920, 6000])
def test_a_large_common_offset_does_not_cancel(vd, c):
    """Values around 1000 with a spread of one: a variance taken as a difference of two large sums would be noise."""
    a = make(2, 5, c, 1, h="f32", offset=1000.0)
    a["post_weight"] = None
    run(vd, a, kind="layer")


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_constant_and_zero_tokens(vd, kind):
    import torch
    x = torch.zeros((1, 3, 640), device="cuda")
    x[0, 1] = 3.0
    _, y = vd.op_gate_norm(x, kind=kind, eps=1e-6)
    torch.cuda.synchronize()
    assert (y[0, 0] == 0).all() and torch.isfinite(y).all()
    if kind == "layer":
        assert (y[0, 1] == 0).all()


def test_one_bad_token_stays_one(vd):
    import math
    import torch
    a = make(1, 40, 320, 1)
    r, y = run(vd, {**a, "post_weight": None})
    a["h"][0, 17, 100] = math.nan
    r2, y2 = vd.op_gate_norm(**{**a, "post_weight": None})
    torch.cuda.synchronize()
    keep = torch.arange(40, device="cuda") != 17
    assert torch.equal(r[:, keep], r2[:, keep]) and torch.equal(y[:, keep], y2[:, keep]) and torch.isnan(y2[0, 17]).all()


def test_empty_calls(vd):
    import torch
    x = torch.zeros((2, 0, 64), device="cuda")
    r, y = vd.op_gate_norm(x, x)
    assert r.shape == y.shape == (2, 0, 64)
