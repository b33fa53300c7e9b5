"""Rotary positions against the definition in 64 bits: layouts, parts of a head, axes, far positions, slices, in place."""
import pytest

from tests import block_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vd():
    from paper_2602_00608_b200 import binding
    return binding


def case(vd, dtype, b, t, h, d, pairs, layout, seed=0, base=10000.0, far=0, two_d=False):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((b, t, h, d), generator=g, device="cuda").to({"bf16": torch.bfloat16, "f32": torch.float32}[dtype])
    freqs = vd.rotary_frequencies(2 * sum(pairs), base, axis_pairs=pairs).cuda()
    pos = torch.randint(far - 50, far + 5000, (b, t, len(pairs)), generator=g, device="cuda", dtype=torch.int32)
    return x, freqs, pos


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("size", [(1, 1, 1, 64, (32,)), (3, 1, 40, 128, (64,)), (2, 77, 12, 80, (16,)), (1, 33, 3, 64, (12, 10, 10)), (2, 5, 2, 96, (8, 7, 0, 9)),
                                  (1, 300, 60, 64, (32,)), (2, 3, 5, 7, (2,)), (1, 9, 130, 256, (128,)), (1, 4, 2, 10, (5,)), (1, 2, 1, 1024, (512,)), (2, 6, 3, 2, (1,)),
                                  (1, 4, 3, 40, (3, 3)), (2, 2, 7, 72, (36,)), (1, 3, 4, 64, (4,))], ids=lambda s: "x".join(map(str, s[:4])) + "r" + "+".join(map(str, s[4])))
def test_rotary_matches_the_definition(vd, dtype, layout, size):
    import torch
    b, t, h, d, pairs = size
    x, freqs, pos = case(vd, dtype, b, t, h, d, pairs, layout)
    want, bound = block_ref.rotary(x, freqs, pos, pairs, layout)
    y = vd.op_rotary(x, freqs, pos, layout=layout, axis_pairs=pairs)
    torch.cuda.synchronize()
    block_ref.check(y, want, bound)
    z = x.clone()
    assert vd.op_rotary(z, freqs, pos, layout=layout, axis_pairs=pairs, out=z) is z                # in place
    torch.cuda.synchronize()
    assert torch.equal(z, y)
    # a slice of packed heads, into a slice of others, positions that the batch shares
    packed = torch.full((b, t, h + 3, d), 5.0, device="cuda", dtype=x.dtype)
    packed[:, :, 1:1 + h] = x
    out = torch.full((b, h + 2, t, d), 5.0, device="cuda", dtype=x.dtype)
    shared = pos[:1].expand(b, t, len(pairs))
    vd.op_rotary(packed[:, :, 1:1 + h], freqs, shared, layout=layout, axis_pairs=pairs, amplitude=1.25, out=out[:, 1:1 + h].transpose(1, 2))
    torch.cuda.synchronize()
    block_ref.check(out[:, 1:1 + h].transpose(1, 2), *block_ref.rotary(x, freqs, shared, pairs, layout, 1.25))
    assert (out[:, 0] == 5).all() and (out[:, 1 + h:] == 5).all()
    # rows at odd addresses
    odd = torch.empty((b, t, h, d + 3), device="cuda", dtype=x.dtype)[..., 1:1 + d]
    odd.copy_(x)
    assert torch.equal(vd.op_rotary(odd, freqs, pos, layout=layout, axis_pairs=pairs), y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("first", [0, 1000003, 2 ** 31 + 12345, -(2 ** 33)])
def test_far_positions_keep_their_angle(vd, dtype, first):
    """Against integer positions times the table in extended precision; an angle formed in fp32 would be off by radians."""
    import numpy as np
    import torch
    x, freqs, _ = case(vd, dtype, 1, 50, 3, 64, (32,), "half", seed=3)
    y = vd.op_rotary(x, freqs, None, first_position=first)
    torch.cuda.synchronize()
    turns = (first + np.arange(50)).astype(np.longdouble)[:, None] * freqs.cpu().numpy().astype(np.longdouble)[None]
    turns = (turns - np.rint(turns)).astype(np.float64)
    want, bound = block_ref.rotary(x, torch.ones(32, dtype=torch.float64), torch.zeros((1, 50, 1), device="cuda"), (32,), "half")
    c, s = (torch.from_numpy(f(2 * np.pi * turns)).cuda().view(1, 50, 1, 32) for f in (np.cos, np.sin))
    u, w = x.double()[..., :32], x.double()[..., 32:]
    want = torch.cat([u * c - w * s, u * s + w * c], 3)
    # (2^53 / 2^33: the product in 64 bits leaves 2^-20 of a turn at the farthest)
    far = 2 * np.pi * abs(first) * 2.0 ** -53
    bound = (u.abs() + w.abs()).repeat(1, 1, 1, 2) * (far + 2.0 ** -21 + 2.0 ** -23)
    block_ref.check(y, want, bound + block_ref.half_step(x.dtype) * (want.abs() + bound))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_scores_depend_on_distance_alone(vd, layout):
    """q at i and k at j: the product of the turned heads is the same wherever the pair stands."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k = (torch.randn((1, 1, 4, 64), generator=g, device="cuda") for _ in range(2))
    freqs = vd.rotary_frequencies(64).cuda()
    at = lambda x, p: vd.op_rotary(x, freqs, first_position=p, layout=layout).double()
    dots = [(at(q, p + 7) * at(k, p)).sum(3) for p in (0, 1, 1000, 500000)]
    # each factor is off by 2^-20.6 of its pair's length
    assert all((d - dots[0]).abs().max() <= 4 * 2.0 ** -20.6 * float(q.norm(dim=3).max() * k.norm(dim=3).max()) for d in dots)


def test_nothing_turns_and_nothing_there(vd):
    import torch
    x = torch.randn((2, 3, 4, 16), device="cuda")
    y = vd.op_rotary(x, torch.empty(0, dtype=torch.float64, device="cuda"), None, axis_pairs=(0,))
    torch.cuda.synchronize()
    assert torch.equal(x, y)
    assert vd.op_rotary(x[:, :0], vd.rotary_frequencies(16).cuda()).shape == (2, 0, 4, 16)


def test_graph_replays_see_the_present_positions(vd):
    import torch
    x, freqs, pos = case(vd, "bf16", 4, 1, 8, 64, (32,), "half", seed=6)
    y, graph = torch.empty_like(x), torch.cuda.CUDAGraph()
    vd.op_rotary(x, freqs, pos, out=y)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        vd.op_rotary(x, freqs, pos, out=y)
    pos += 17
    graph.replay()
    torch.cuda.synchronize()
    block_ref.check(y, *block_ref.rotary(x, freqs, pos, (32,), "half"))
