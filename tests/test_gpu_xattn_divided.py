"""Calls of the tensor-core attention whose items are divided by keys among the thread blocks of clusters: all of them, or what whole
rounds leave over.  That a size is shared out so is asked of the library, so that a changed rule does not drop a path from the tests."""
import math

import pytest

from tests import block_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vd():
    from paper_2602_00608_b200 import binding
    return binding


def make(b, tq, tk, h, hkv, d, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(8000 + seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    return r(b, tq, h, d).bfloat16(), r(b, tk, hkv, d).bfloat16(), (r(b, tk, hkv, d) + 0.25).bfloat16()


def ragged(vd, q, k, v, lens):
    """Against the definition, with NaN behind each length; twice, for the same bits."""
    import torch
    scale = q.shape[3] ** -0.5
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    behind = torch.arange(k.shape[1], device="cuda")[None, :, None, None] >= n[:, None, None, None]
    want = block_ref.attention(q, k.masked_fill(behind, 0), v.masked_fill(behind, 0), n, scale)
    k, v = k.masked_fill(behind, math.nan), v.masked_fill(behind, math.nan)
    o = vd.op_cross_attention(q, k, v, n, scale=scale)
    torch.cuda.synchronize()
    block_ref.check(o, *want)
    assert (o[n <= 0] == 0).all()
    again = vd.op_cross_attention(q, k, v, n, scale=scale)
    torch.cuda.synchronize()
    assert torch.equal(o.view(torch.int16), again.view(torch.int16))
    return o


REST = [(1, 5400, 6000, 8, 8, 64), (1, 5400, 6000, 8, 8, 128), (1, 2700, 5000, 16, 8, 40), (2, 1350, 6000, 16, 16, 72)]
ALL = [(1, 300, 5000, 2, 2, 64), (1, 130, 3001, 3, 1, 128), (2, 700, 2000, 5, 5, 96)]


@pytest.mark.parametrize("size", REST + ALL, ids=lambda s: "x".join(map(str, s)))
def test_full_lengths(vd, size):
    import torch
    q, k, v = make(*size, seed=1)
    splits, items, whole = vd.xattn_division(q, k, v)
    assert splits > 1 and items > whole and (whole > 0) == (size in REST)
    o = vd.op_cross_attention(q, k, v)
    torch.cuda.synchronize()
    block_ref.check(o, *block_ref.attention(q, k, v, None, size[5] ** -0.5))


# lengths of none, one, within a tile, tiles exactly, and all; every one of them among the last items, which are the divided ones
@pytest.mark.parametrize("turn", range(5))
@pytest.mark.parametrize("d", [64, 128])
def test_what_whole_rounds_leave_over_of_ragged_batches(vd, turn, d):
    b, tk = 5, 6000
    q, k, v = make(b, 1350, tk, 6, 6, d, seed=2)
    splits, items, whole = vd.xattn_division(q, k, v)
    assert splits > 1 and 0 < whole < items
    ragged(vd, q, k, v, [(0, 1, 3333, 2560, tk)[(i + turn) % b] for i in range(b)])


@pytest.mark.parametrize("turn", range(5))
@pytest.mark.parametrize("d", [64, 128])
def test_all_divided_of_ragged_batches(vd, turn, d):
    b, tk = 5, 3000
    q, k, v = make(b, 130, tk, 4, 2, d, seed=3)
    splits, items, whole = vd.xattn_division(q, k, v)
    assert splits > 1 and whole == 0
    ragged(vd, q, k, v, [(0, 1, 1333, 256, tk)[(i + turn) % b] for i in range(b)])


def test_the_division_of_other_calls(vd):
    import torch
    assert vd.xattn_division(*make(2, 300, 77, 4, 4, 64, seed=4))[0] == 1          # a tile of keys
    assert vd.xattn_division(*make(1, 300, 5000, 2, 2, 256, seed=4))[0] == 1       # wide heads
    assert vd.xattn_division(*make(1, 1, 5000, 2, 2, 64, seed=4)) is None          # few rows
    assert vd.xattn_division(*make(1, 300, 5000, 2, 2, 60, seed=4)) is None        # no tensor map
    assert vd.xattn_division(*(x.float() for x in make(1, 300, 500, 2, 2, 64, seed=4))) is None
    with pytest.raises(vd.VdError):
        vd.xattn_division(*make(1, 300, 500, 3, 2, 64, seed=4))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(3, 1, 700, 4, 2, 64), (3, 5, 300, 4, 4, 64), (2, 9, 100, 4, 2, 128), (3, 40, 90, 2, 2, 64), (2, 300, 700, 2, 2, 128), (2, 70, 300, 2, 1, 256)],
                         ids=lambda s: "x".join(map(str, s)))
def test_queries_expanded_over_the_batch(vd, dtype, size):
    """The same queries for every batch item, as a tensor of stride 0."""
    import torch
    b, tq, _, h, _, d = size
    q, k, v = make(*size, seed=5)
    if dtype == "f32":
        q, k, v = q.float(), k.float(), v.float()
    q = q[:1].expand(b, tq, h, d)
    o = vd.op_cross_attention(q, k, v)
    torch.cuda.synchronize()
    block_ref.check(o, *block_ref.attention(q, k, v, None, d ** -0.5))
