"""Attention to states of another length against the definition in 64 bits: lengths from one to several tiles, ragged and empty
rows, grouped heads, head sizes, slices and expanded tensors, what lies behind a row's last key."""
import math

import pytest

from tests import block_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vd():
    from paper_2602_00608_b200 import binding
    return binding


def _types():
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}


def make(dtype, b, tq, tk, h, hkv, d, seed=0, factor=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(1000 + seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    return (factor * r(b, tq, h, d)).to(_types()[dtype]), r(b, tk, hkv, d).to(_types()[dtype]), (r(b, tk, hkv, d) + 0.25).to(_types()[dtype])


def run(vd, q, k, v, lens=None, scale=None, **kw):
    import torch
    scale = q.shape[3] ** -0.5 if scale is None else scale
    lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    o = vd.op_cross_attention(q, k, v, lens, scale=scale, **kw)
    torch.cuda.synchronize()
    block_ref.check(o, *block_ref.attention(q, k, v, lens, scale))
    return o


SIZES = [  # b, tq, tk, h, hkv, d
    (1, 1, 1, 1, 1, 64), (2, 1, 7, 4, 4, 64), (3, 1, 130, 8, 2, 128), (2, 3, 300, 6, 2, 80), (1, 17, 33, 5, 5, 40), (2, 64, 77, 3, 3, 64),
    (1, 127, 129, 2, 2, 128), (2, 128, 128, 2, 1, 64), (1, 129, 127, 4, 2, 96), (1, 255, 256, 3, 1, 128), (2, 257, 385, 2, 2, 72), (1, 300, 1, 2, 2, 64),
    (1, 513, 640, 2, 1, 32), (1, 1, 2049, 8, 1, 128), (1, 2, 5000, 4, 4, 64), (5, 31, 511, 7, 7, 128), (1, 40, 700, 30, 6, 64), (1, 9, 100, 16, 1, 128),
    (1, 130, 260, 3, 3, 256), (2, 5, 50, 2, 2, 1), (1, 16, 300, 2, 2, 128), (2, 1, 1000, 10, 1, 64), (1, 11, 77, 1, 1, 40), (1, 4, 500, 8, 4, 96), (3, 2, 4100, 12, 2, 128), (1, 8, 17, 2, 2, 72), (2, 1, 900, 3, 1, 256), (1, 19, 21, 2, 1, 7), (1, 70, 200, 2, 2, 160), (1, 20, 90, 1, 1, 255),
    # few items: their keys divided among a cluster; many: whole ones and divided ones in one call (148 SMs)
    (1, 300, 5000, 2, 2, 128), (1, 130, 3001, 3, 1, 64), (2, 700, 2000, 5, 5, 128), (1, 17, 9000, 1, 1, 64), (1, 50, 4000, 12, 2, 72), (1, 5400, 1100, 8, 8, 64), (1, 5400, 700, 8, 8, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_full_lengths(vd, dtype, size):
    run(vd, *make(dtype, *size))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(4, 1, 200, 4, 2, 64), (4, 33, 300, 2, 2, 128), (5, 140, 270, 3, 1, 80), (4, 300, 129, 2, 2, 64), (4, 2, 40, 2, 2, 7), (5, 100, 3000, 2, 2, 128),
                                  (5, 300, 2500, 2, 1, 64), (5, 5, 3000, 4, 2, 64), (5, 40, 3000, 6, 2, 80)],
                         ids=lambda s: "x".join(map(str, s)))
def test_ragged_lengths_with_garbage_behind_them(vd, dtype, size):
    """One row without keys, one of one key, one clamped from above, the others ragged; NaN, infinities and the type's lowest value behind each
    row's last key."""
    import torch
    b, _, tk = size[:3]
    q, k, v = make(dtype, *size, seed=1)
    lens = [0, 1, tk + 9, (2 * tk) // 3 + 1, tk // 12][:b]
    clean = [x.clone() for x in (k, v)]
    for i, n in enumerate(lens):
        n = min(n, tk)
        for x, bad in ((k, (math.nan, -math.inf, torch.finfo(k.dtype).min)), (v, (math.inf, math.nan, torch.finfo(k.dtype).max))):
            for j in range(3):
                x[i, n + j::3] = bad[j]
            clean[0 if x is k else 1][i, n:] = 0
    scale = q.shape[3] ** -0.5
    dev = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o = vd.op_cross_attention(q, k, v, dev, scale=scale)
    torch.cuda.synchronize()
    block_ref.check(o, *block_ref.attention(q, *clean, dev, scale))
    assert (o[0] == 0).all()
    neg = vd.op_cross_attention(q, k, v, torch.full((b,), -3, dtype=torch.int32, device="cuda"), scale=scale)
    torch.cuda.synchronize()
    assert (neg == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tq", [1, 200])
def test_no_keys_at_all(vd, dtype, tq):
    import torch
    q, k, v = make(dtype, 2, tq, 0, 4, 2, 64)
    out = torch.full_like(q, 7.0)
    vd.op_cross_attention(q, k, v, out=out)
    torch.cuda.synchronize()
    assert (out == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tq,tk", [(1, 900), (4, 3000), (150, 900)])
def test_scores_that_grow_from_tile_to_tile(vd, dtype, tq, tk):
    """The maximum of a row moves by far more than any threshold from one tile of keys to the next, up and down."""
    import torch
    q, k, v = make(dtype, 1, tq, tk, 2, 2, 64, seed=2)
    up = torch.sign(q.float().mean(1, keepdim=True))
    step = (torch.arange(tk, device="cuda") // 64 % 9).float().view(1, -1, 1, 1)
    k = (0.05 * k.float() + 0.8 * step * up).to(k.dtype)
    q = (q.float() * 0.5 + up).to(q.dtype)
    run(vd, q, k, v)
    run(vd, q, k.flip(1).contiguous(), v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tq", [1, 3, 150])
def test_large_scores(vd, dtype, tq):
    """Scores in the thousands: the softmax is one key's, nothing overflows."""
    q, k, v = make(dtype, 1, tq, 333, 2, 1, 128, seed=3, factor=400.0)
    run(vd, q, k, v, scale=0.25)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(2, 70, 150, 4, 2, 64), (2, 1, 150, 4, 2, 64), (3, 200, 90, 2, 2, 72)], ids=lambda s: "x".join(map(str, s)))
def test_slices_and_expanded_tensors(vd, dtype, size):
    import torch
    b, tq, tk, h, hkv, d = size
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(_types()[dtype])
    qkv = r(b, tq, h + 8, d)                                       # q a slice of a packed tensor
    kv = r(b, tk, 2, hkv, d)                                       # one projection
    o = torch.full((b, tq, h + 2, d), 3.0, device="cuda", dtype=qkv.dtype)
    lens = torch.tensor([tk, tk - 60, tk // 2][:b], dtype=torch.int32, device="cuda")
    q, k, v = qkv[:, :, 3:3 + h], kv[:, :, 0], kv[:, :, 1]
    vd.op_cross_attention(q, k, v, lens, out=o[:, :, 1:1 + h])
    torch.cuda.synchronize()
    block_ref.check(o[:, :, 1:1 + h], *block_ref.attention(q, k, v, lens, d ** -0.5))
    assert (o[:, :, 0] == 3).all() and (o[:, :, 1 + h:] == 3).all()
    # heads before tokens, one prompt for the whole batch, one value head for all
    q, k = r(b, h, tq, d).transpose(1, 2), r(1, hkv, tk, d).transpose(1, 2).expand(b, tk, hkv, d)
    v = r(1, tk, 1, d).expand(b, tk, hkv, d)
    out = torch.empty((b, h, tq, d), device="cuda", dtype=q.dtype).transpose(1, 2)
    run(vd, q, k, v, out=out)
    # rows that start at odd places
    q, k, v = (r(b, n, m, d + 3)[..., 1:1 + d] for n, m in ((tq, h), (tk, hkv), (tk, hkv)))
    run(vd, q, k, v)
    big = torch.full((b, tq, h, d + 5), 2.0, device="cuda", dtype=q.dtype)
    run(vd, q, k, v, out=big[..., 3:3 + d])
    assert (big[..., :3] == 2).all() and (big[..., 3 + d:] == 2).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tq", [1, 5, 160])
def test_nan_and_infinity_in_what_counts(vd, dtype, tq):
    """A NaN or an infinite score among a row's keys reaches that row, and no other."""
    import torch
    q, k, v = make(dtype, 2, tq, 300, 4, 2, 64, seed=6)
    want, bound = block_ref.attention(q, k, v, None, 0.125)
    for place in (3, 150, 299):
        for t, bad in ((k, math.nan), (v, math.nan), (q, math.nan)):
            x = [y.clone() for y in (q, k, v)]
            at = next(i for i, y in enumerate((q, k, v)) if y is t)
            x[at][1, 0 if at == 0 else place, 0, 5] = bad
            o = vd.op_cross_attention(*x, scale=0.125)
            torch.cuda.synchronize()
            hit = o[1, :, :2] if at else o[1, :1, :1]
            assert (torch.isnan(hit[..., 5]) if at == 2 else torch.isnan(hit)).all()
            clean = torch.ones_like(o, dtype=torch.bool)
            clean[1, slice(0, 1) if at == 0 else slice(None), slice(0, 1) if at == 0 else slice(0, 2)] = False
            assert ((o.double() - want).abs() <= bound)[clean].all()
    x = k.clone()
    x[0, 200, 1] = math.inf                                        # scores of + and - infinity: NaN where the sum has an infinity
    o = vd.op_cross_attention(q, x, v, scale=0.125)
    torch.cuda.synchronize()
    s = torch.einsum("thd,hd->th", q[0, :, 2:].float(), x[0, 200, 1].float().expand(2, 64))
    assert torch.isnan(o[0, :, 2:][~(s == -math.inf)]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(1, 300, 700, 4, 2, 64), (2, 1, 3000, 8, 2, 128), (2, 6, 90, 4, 2, 64), (1, 150, 6000, 2, 2, 128), (2, 1350, 500, 30, 30, 64), (1, 3000, 1500, 16, 16, 128)], ids=lambda s: "x".join(map(str, s)))
def test_same_bits_each_time_on_any_stream_and_in_a_graph(vd, dtype, size):
    import torch
    q, k, v = make(dtype, *size, seed=7)
    lens = torch.full((size[0],), size[2] - 5, dtype=torch.int32, device="cuda")
    first = run(vd, q, k, v, lens.tolist())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        others = [vd.op_cross_attention(q, k, v, lens) for _ in range(5)]
    both = [vd.op_cross_attention(q, k, v, lens) for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in others + both)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.graph(graph):
        vd.op_cross_attention(q, k, v, lens, out=out)
    q2 = make(dtype, *size, seed=8)[0]
    q.copy_(q2)
    lens.fill_(size[2] // 2)                                       # lengths are read on the device: a replay sees the present ones
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, vd.op_cross_attention(q, k, v, lens))
    block_ref.check(out, *block_ref.attention(q, k, v, lens, size[5] ** -0.5))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(2, 140, 300, 4, 2, 64), (1, 1, 500, 4, 1, 128)], ids=lambda s: "x".join(map(str, s)))
def test_the_plain_kernel_agrees(vd, dtype, size):
    run(vd, *make(dtype, *size, seed=9), lens=[size[2] - 3] * size[0], impl=vd.VD_XATTN_PLAIN)


@pytest.mark.parametrize("tq", [1, 130])
def test_offsets_beyond_32_bits(vd, tq):
    """Keys whose elements lie more than 2^31 elements behind the first one (a slice of a large cache)."""
    import torch
    b, tk, d = 2, 200, 64
    stride = (1 << 31) + 64
    cache = torch.zeros(stride + 2 * tk * d, dtype=torch.bfloat16, device="cuda")
    q, k, v = make("bf16", b, tq, tk, 1, 1, d, seed=10)
    far = [torch.as_strided(cache, (b, tk, 1, d), (stride, d, d, 1), at) for at in (0, tk * d)]
    for f, x in zip(far, (k, v)):
        f.copy_(x)
    run(vd, q, *far)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tq", [1, 2, 40])
def test_many_sequences(vd, dtype, tq):
    """More batch items than a CTA keeps lengths of, every length from none to all."""
    b, tk = 300, 150
    run(vd, *make(dtype, b, tq, tk, 2, 1, 64, seed=11), lens=[i % (tk + 1) for i in range(b)])


def test_a_first_call_can_be_captured():
    """In a process of its own: nothing of the library has run before the capture."""
    import subprocess
    import sys
    code = """
import torch
from paper_2602_00608_b200 import binding as vd
q, k, v = (torch.randn(1, n, 4, 64, device="cuda").bfloat16() for n in (200, 900, 900))
x = torch.randn(1, 200, 256, device="cuda")
freqs = vd.rotary_frequencies(64).cuda()
outs = [torch.empty_like(q), torch.empty_like(q), torch.empty_like(q[:, :1]), torch.empty_like(x), torch.empty_like(x), torch.empty_like(q.float())]
def step():
    vd.op_rotary(q, freqs, out=outs[0])
    vd.op_cross_attention(outs[0], k, v, out=outs[1])
    vd.op_cross_attention(outs[0][:, :1], k, v, out=outs[2])
    vd.op_gate_norm(x, x_out=outs[3], y=outs[4])
    vd.op_cross_attention(q.float(), k.float(), v.float(), out=outs[5])
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    step()
g.replay()
torch.cuda.synchronize()
first = [o.clone() for o in outs]
step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(first, outs))
print("captured")
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("size", [(300, 140, 77, 4, 2, 64), (90, 300, 128, 6, 6, 40), (80, 257, 17, 8, 8, 64), (150, 30, 100, 12, 4, 56), (2, 10800, 77, 4, 4, 64)], ids=lambda s: "x".join(map(str, s)))
def test_short_contexts_of_many_items(vd, size):
    """Contexts of one tile of keys where a CTA takes several items: every length from none to all, NaN behind each, large scores in between."""
    import torch
    b, _, tk = size[:3]
    q, k, v = make("bf16", *size, seed=12)
    q[::3] *= 100
    lens = torch.tensor([(7 * i + tk) % (tk + 1) if b > 2 else tk - 5 * i for i in range(b)], dtype=torch.int32, device="cuda")
    behind = torch.arange(tk, device="cuda")[None, :, None, None] >= lens[:, None, None, None]
    scale = q.shape[3] ** -0.5
    want = block_ref.attention(q, k.masked_fill(behind, 0), v.masked_fill(behind, 0), lens, scale)
    k.masked_fill_(behind, math.nan)
    v.masked_fill_(behind, math.nan)
    first = vd.op_cross_attention(q, k, v, lens, scale=scale)
    torch.cuda.synchronize()
    block_ref.check(first, *want)
    assert (first[lens == 0] == 0).all()
    again = vd.op_cross_attention(q, k, v, lens, scale=scale)
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(2, 150, 400, 4, 2, 64), (1, 70, 5000, 2, 1, 100), (3, 3, 900, 6, 2, 250), (2, 130, 300, 2, 2, 192), (2, 2, 300, 130, 1, 64), (1, 1, 2000, 2, 2, 33),
                                  (1, 700, 130, 20, 20, 128)], ids=lambda s: "x".join(map(str, s)))
def test_any_alignment_and_width(vd, dtype, size):
    """Heads that start at odd elements of odd rows, outputs too; ragged lengths with NaN behind them; what lies around the output stays."""
    import torch
    b, tq, tk, h, hkv, d = size
    q, k, v = make(dtype, *size, seed=13)
    lens = [tk, 0, tk // 2 + 1][:b]
    for i, n in enumerate(lens):
        k[i, n:], v[i, n:] = math.nan, math.nan
    clean = [x.nan_to_num() for x in (k, v)]
    wide = []
    for x in (q, k, v, q):
        w = torch.full((*x.shape[:3], d + 3), 7.0, dtype=x.dtype, device="cuda")
        w[..., 1:1 + d] = x
        wide.append(w)
    dev = torch.tensor(lens, dtype=torch.int32, device="cuda")
    at = [w[..., 1:1 + d] for w in wide]
    vd.op_cross_attention(*at[:3], dev, scale=d ** -0.5, out=at[3])
    torch.cuda.synchronize()
    block_ref.check(at[3], *block_ref.attention(q, *clean, dev, d ** -0.5))
    assert (wide[3][..., 0] == 7).all() and (wide[3][..., 1 + d:] == 7).all()


@pytest.mark.parametrize("size", [(1, 130, 260, 3, 3, 256), (3, 140, 300, 4, 2, 192), (5, 300, 129, 2, 1, 136), (40, 257, 130, 10, 10, 256), (2, 700, 1500, 6, 2, 200), (30, 40, 600, 24, 12, 256)],
                         ids=lambda s: "x".join(map(str, s)))
def test_wide_heads(vd, size):
    """Beyond 128 channels: every length from none to all, NaN behind each, scores that grow from tile to tile, the same bits again."""
    import torch
    b, _, tk = size[:3]
    q, k, v = make("bf16", *size, seed=14)
    k *= 1 + 8 * torch.arange(tk, device="cuda", dtype=k.dtype)[None, :, None, None] / tk
    lens = torch.tensor([tk - (i * tk) // max(1, b - 1) if b > 2 else tk - i for i in range(b)], dtype=torch.int32, device="cuda")
    behind = torch.arange(tk, device="cuda")[None, :, None, None] >= lens[:, None, None, None]
    scale = q.shape[3] ** -0.5
    want = block_ref.attention(q, k.masked_fill(behind, 0), v.masked_fill(behind, 0), lens, scale)
    k.masked_fill_(behind, math.nan)
    v.masked_fill_(behind, math.nan)
    first = vd.op_cross_attention(q, k, v, lens, scale=scale)
    torch.cuda.synchronize()
    block_ref.check(first, *want)
    assert (first[lens == 0] == 0).all()
    again = vd.op_cross_attention(q, k, v, lens, scale=scale)
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("size", [(3, 1, 3000, 8, 4, 256), (2, 4, 5000, 4, 2, 192), (5, 2, 900, 16, 2, 256), (40, 1, 700, 8, 8, 256), (4, 1, 2000, 2, 2, 136), (3, 8, 70, 4, 2, 200)],
                         ids=lambda s: "x".join(map(str, s)))
def test_wide_heads_of_few_rows(vd, size):
    """One to sixteen rows of a key head beyond 128 channels: lengths from none to all, NaN behind each, growing scores, the same bits again."""
    import torch
    b, _, tk = size[:3]
    q, k, v = make("bf16", *size, seed=15)
    k *= 1 + 8 * torch.arange(tk, device="cuda", dtype=k.dtype)[None, :, None, None] / tk
    lens = torch.tensor([tk - (i * tk) // (b - 1) for i in range(b)], dtype=torch.int32, device="cuda")
    behind = torch.arange(tk, device="cuda")[None, :, None, None] >= lens[:, None, None, None]
    scale = q.shape[3] ** -0.5
    want = block_ref.attention(q, k.masked_fill(behind, 0), v.masked_fill(behind, 0), lens, scale)
    k.masked_fill_(behind, math.nan)
    v.masked_fill_(behind, math.nan)
    first = vd.op_cross_attention(q, k, v, lens, scale=scale)
    torch.cuda.synchronize()
    block_ref.check(first, *want)
    assert (first[lens == 0] == 0).all()
    again = vd.op_cross_attention(q, k, v, lens, scale=scale)
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("size", [(4, 1, 77, 16, 2, 64), (6, 2, 128, 8, 1, 64), (40, 1, 500, 64, 4, 128), (3, 3, 100, 4, 2, 64), (5, 2, 90, 2, 2, 72), (5, 1, 1024, 4, 2, 64), (5, 4, 128, 2, 2, 128),
                                  (5, 4, 129, 2, 2, 128), (5, 1, 1025, 4, 2, 128), (3, 1, 513, 9, 1, 64), (3, 8, 129, 2, 2, 256), (75, 3, 700, 8, 2, 128)], ids=lambda s: "x".join(map(str, s)))
def test_few_rows_on_either_side_of_the_rules(vd, size):
    """Two to sixteen rows of a key head with contexts around the lengths at which another kernel takes them."""
    b, _, tk = size[:3]
    run(vd, *make("bf16", *size, seed=16), lens=[(5 * i + tk) % (tk + 1) if i % 3 else tk - i // 3 for i in range(b)])


@pytest.mark.parametrize("size", [(3, 5, 300, 4, 4, 64), (2, 8, 500, 8, 2, 80), (2, 11, 130, 6, 2, 64), (3, 2, 700, 16, 2, 128), (2, 17, 90, 1, 1, 96), (2, 1, 1000, 31, 1, 40), (70, 3, 40, 10, 5, 64),
                                  (3, 4, 600, 8, 2, 256)], ids=lambda s: "x".join(map(str, s)))
def test_few_rows_in_single_precision(vd, size):
    """Five to 33 rows of a key head, in groups of four: a length for each sequence, none and all among them."""
    b, _, tk = size[:3]
    run(vd, *make("f32", *size, seed=17), lens=[(5 * i + tk) % (tk + 1) if i % 3 else tk - i // 3 for i in range(b)])
