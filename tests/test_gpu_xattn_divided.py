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
    splits, items, whole, _ = vd.xattn_division(q, k, v)
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
    splits, items, whole, _ = vd.xattn_division(q, k, v)
    assert splits > 1 and 0 < whole < items
    ragged(vd, q, k, v, [(0, 1, 3333, 2560, tk)[(i + turn) % b] for i in range(b)])


@pytest.mark.parametrize("turn", range(5))
@pytest.mark.parametrize("d", [64, 128])
def test_all_divided_of_ragged_batches(vd, turn, d):
    b, tk = 5, 3000
    q, k, v = make(b, 130, tk, 4, 2, d, seed=3)
    splits, items, whole, _ = vd.xattn_division(q, k, v)
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


def divided_rows(vd, q, k, v):
    """A mask [B,Tq,H] of the rows whose items are divided."""
    import torch
    b, tq, h, d = q.shape
    hkv = k.shape[2]
    _, items, whole, _ = vd.xattn_division(q, k, v)
    tokens = 2 * (128 // (h // hkv))
    per = -(-tq // tokens)
    assert items == b * hkv * per
    at = torch.arange(items, device="cuda").view(b, hkv, per) >= whole
    return at.repeat_interleave(tokens, 2)[:, :, :tq].repeat_interleave(h // hkv, 1).transpose(1, 2)


@pytest.mark.parametrize("size,lens", [((1, 5400, 6000, 8, 8, 64), [6000]), ((1, 5400, 6000, 8, 8, 128), [5999]), ((5, 1350, 6000, 6, 6, 128), [6000, 0, 3333, 1, 0]),
                                       ((5, 130, 3000, 4, 2, 64), [0, 3000, 1, 0, 1333]), ((3, 700, 2000, 5, 5, 96), [2000, 200, 0])], ids=lambda s: "x".join(map(str, s)))
def test_rows_of_a_meeting_that_gave_up_are_nan(vd, size, lens):
    """A block that the others of its cluster do not tell anything (here: one that does not wait) answers NaN for its rows, and never with what it finds
    in their memory. Rows without keys stay zeros, whole items are not touched, and the next call is right again."""
    import torch
    q, k, v = make(*size, seed=6)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    divided = divided_rows(vd, q, k, v)
    assert divided.any()
    want, bound = block_ref.attention(q, k, v, n, size[5] ** -0.5)
    l = vd.lib()
    try:
        assert l.vd_debug_xattn_meeting_limit(-1) == vd.VD_OK
        o = vd.op_cross_attention(q, k, v, n)
        torch.cuda.synchronize()
    finally:
        l.vd_debug_xattn_meeting_limit(0)
    lost = divided & (n > 0)[:, None, None]
    assert torch.isnan(o[lost]).all()
    assert (o[n == 0] == 0).all()
    assert ((o.double() - want).abs() <= bound)[~lost].all()
    o = vd.op_cross_attention(q, k, v, n)
    torch.cuda.synchronize()
    block_ref.check(o, want, bound)


def test_a_block_that_comes_seconds_later_than_the_others(vd):
    """One block's whole items have 2^25 keys each, those of the others of its cluster none: they wait for it longer than a wait's
    usual second, and its share counts."""
    import torch
    b, tq, tk, d = 620, 17, 1 << 25, 64
    g = torch.Generator(device="cuda").manual_seed(8007)
    q = torch.randn(b, tq, 1, d, generator=g, device="cuda").bfloat16()
    k, v = (torch.empty(1, tk, 1, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g).expand(b, tk, 1, d) for _ in range(2))
    splits, items, whole, blocks = vd.xattn_division(q, k, v)
    assert items == b and splits > 1 and whole // blocks >= 4 and whole < b
    n = torch.zeros(b, dtype=torch.int32, device="cuda")
    n[0:whole:blocks] = tk                                         # all of block 0's
    n[whole:] = 300 + torch.arange(b - whole, device="cuda")
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    o = vd.op_cross_attention(q, k, v, n)
    end.record()
    torch.cuda.synchronize()
    assert start.elapsed_time(end) > 1100.0, "the block was not late"
    assert torch.isfinite(o).all() and (o[n == 0] == 0).all()
    few = slice(whole, b)
    block_ref.check(o[few], *block_ref.attention(q[few], k[few, :1000], v[few, :1000], n[few], d ** -0.5))
