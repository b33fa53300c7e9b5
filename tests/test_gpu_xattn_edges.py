"""Attention to states of another length at the edges of its numbers: rows whose every score is minus infinity, weights that
underflow, one key, scores far from zero."""
import math

import pytest

from tests import block_ref

pytestmark = pytest.mark.gpu

WIDTHS = [64, 72, 128, 256]
CONTEXTS = [1, 17, 20, 77, 96, 100, 128, 150, 224, 256, 333]         # last tiles of every kind, alone and behind whole ones


@pytest.fixture(scope="module")
def vd():
    from paper_2602_00608_b200 import binding
    return binding


def make(dtype, b, tq, tk, h, hkv, d, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(7000 + seed)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    return tuple(torch.randn(s, generator=g, device="cuda").to(dt) for s in ((b, tq, h, d), (b, tk, hkv, d), (b, tk, hkv, d)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tq", [1, 3, 8, 40])
@pytest.mark.parametrize("d", WIDTHS)
def test_scores_of_minus_infinity(vd, dtype, tq, d):
    """A row all of whose scores are minus infinity is 0 / 0, as in the definition, whatever the number of keys; such scores beside finite ones
    weigh nothing."""
    import torch
    for tk in CONTEXTS:
        q, k, v = make(dtype, 2, tq, tk, 2, 2, d, seed=1)
        q[..., 0] = 1
        k[0, :, :, 0] = -math.inf
        few = min(tk, 3)
        k[1, few:, :, 0] = -math.inf
        o = vd.op_cross_attention(q, k, v, scale=0.125)
        torch.cuda.synchronize()
        assert torch.isnan(o[0]).all(), f"{tk} keys: {float(torch.isnan(o[0]).float().mean()):.2f} NaN"
        block_ref.check(o[1:], *block_ref.attention(q[1:], k[1:, :few], v[1:, :few], None, 0.125))


@pytest.mark.parametrize("tq", [1, 3, 8, 40])
@pytest.mark.parametrize("d", WIDTHS)
def test_weights_that_underflow_are_zero(vd, tq, d):
    """The first key's score is above the others' by 1024 (1477 in units of log 2: 2^-1477 is 0 in fp32), so the row is that key's value, however
    large the others' are (1e36 each: no sum of 100 of them overflows).  The output is v times a sum of ones and zeros over itself, rounded: exact, but
    for the probability's and the output's half steps."""
    import torch
    for tk in (17, 20, 77, 96, 100, 128):
        q, k, v = make("bf16", 1, tq, tk, 2, 2, d, seed=2)
        q.zero_()
        k.zero_()
        q[..., 0], k[:, 0, :, 0], v[:, 1:] = 64.0, 64.0, 1e36
        o = vd.op_cross_attention(q, k, v, scale=0.25)
        torch.cuda.synchronize()
        want = v[:, :1].double().expand(o.shape)
        off = ((o.double() - want).abs() - 2.01 * block_ref.BF16 * want.abs()).max()
        assert off <= 0, f"{tk} keys: off by {float((o.double() - want).abs().max()):.3g}"


@pytest.mark.parametrize("tq", [1, 3, 8, 40, 300])
@pytest.mark.parametrize("d", WIDTHS)
def test_one_key_is_its_value(vd, tq, d):
    """softmax of one score is 1: the output is v, bit for bit.  The same where one key's score is above all others by 200 in units of log 2 (their
    weights are 2^-200), in the first tile of keys or in one behind it."""
    import torch
    for tk in CONTEXTS:
        q, k, v = make("bf16", 2, tq, tk, 4, 2, d, seed=3)
        o = vd.op_cross_attention(q, k, v, torch.ones(2, dtype=torch.int32, device="cuda"))
        assert torch.equal(o, v[:, :1].repeat_interleave(2, 2).expand_as(o)), f"one of {tk} keys"
        for at in {0, tk // 3, tk // 2, tk - 1}:
            q[..., 0], k[..., 0] = 16.0, 0.0
            k[:, at, :, 0] = 512.0 + 16.0 * d
            o = vd.op_cross_attention(q, k, v, scale=0.25)
            assert torch.equal(o, v[:, at:at + 1].repeat_interleave(2, 2).expand_as(o)), f"key {at} of {tk}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tq", [1, 3, 8, 40, 300])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_far_from_zero(vd, dtype, tq, d, sign):
    """Scores of up to 2^107, above zero and below, whose size varies within a row: two keys share the largest, and the next is lower by
    thousands, so the row is the mean of the two values (weights 1 + 1; off by the half steps of the probabilities, which are alike, and of the output).
    Each score is one product of numbers of at most eight bits, exact in fp32; the scale is no power of two."""
    import torch
    half = block_ref.half_step(torch.bfloat16 if dtype == "bf16" else torch.float32)
    g = torch.Generator(device="cuda").manual_seed(7004)
    for tk in (77, 90, 150, 333, 3000):
        for e in (8, 16, 21, 24, 27, 30, 33, 40, 60, 98):
            q, k, v = make(dtype, 1, tq, tk, 2, 1, d, seed=4)
            q.zero_()
            k.zero_()
            q[..., 0] = 2.0 ** (e // 2)
            odd = (2 * torch.randint(64, 128, (tk,), generator=g, device="cuda") + 1).float()                    # 129 to 255
            less = 2.0 ** -torch.randint(1, e - 6, (tk,), generator=g, device="cuda").float() if sign > 0 else 1.0
            k[0, :, 0, 0] = sign * odd * less * 2.0 ** (e - e // 2)
            i, j = sorted(torch.randperm(tk, generator=g, device="cuda")[:2].tolist())
            k[0, [i, j], 0, 0] = sign * (251.0 if sign > 0 else 67.0) * 2.0 ** (e - e // 2)
            o = vd.op_cross_attention(q, k, v, scale=72.0 ** -0.5)
            torch.cuda.synchronize()
            one, two = v[0, i, 0].double(), v[0, j, 0].double()
            off = (o.double() - (one + two) / 2).abs() - 2.01 * half * (one.abs() + two.abs()) / 2
            assert (off <= 0).all(), f"{tk} keys, 2^{e}, the largest at {i} and {j}: {int((~(off <= 0)).sum())} values"
