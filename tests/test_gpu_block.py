"""The block operators together, as a world model's block uses them in front of the decoder: modulated norm, rotary q and k, attention
within the frames, gated residual, attention to a padded prompt, gated residual with norms on both sides; the result decoded."""
import pytest

from tests import block_ref, util

pytestmark = pytest.mark.gpu


def _weights(c, g):
    import torch
    lin = lambda n: torch.randn((c, n), generator=g, device="cuda") * c ** -0.5
    return {"qkv": lin(3 * c), "o1": lin(c), "q": lin(c), "kv": lin(2 * c), "o2": lin(c)}


def block(vd, w, x, mods, prompt, lens, pos, freqs, pairs, heads, dt):
    """One block on the library's operators; products by torch."""
    b, t, c = x.shape
    d = c // heads
    m = lambda i: mods[:, :, i]
    mm = lambda a, n: a @ w[n].to(dt)
    x1, y = vd.op_gate_norm(x, scale=m(0), shift=m(1), y=None if dt == x.dtype else x.new_empty(x.shape, dtype=dt))
    qkv = mm(y, "qkv").view(b, t, 3 * heads, d)
    qk = qkv[:, :, :2 * heads]
    vd.op_rotary(qk, freqs, pos, layout="interleaved", axis_pairs=pairs, out=qk)
    h = vd.op_cross_attention(qk[:, :, :heads], qk[:, :, heads:], qkv[:, :, 2 * heads:]).view(b, t, c)
    x2, y = vd.op_gate_norm(x1, mm(h, "o1"), gate=m(2), scale=m(3), shift=m(4), x_out=x1)
    kv = mm(prompt, "kv").view(b, prompt.shape[1], 2, heads, d)
    h = vd.op_cross_attention(mm(y, "q").view(b, t, heads, d), kv[:, :, 0], kv[:, :, 1], lens).view(b, t, c)
    return vd.op_gate_norm(x2, mm(h, "o2"), gate=m(5), kind="rms", post_norm=True, residual_scale=0.5, x_out=x2)


def block64(w, x, mods, prompt, lens, pos, freqs, pairs, heads):
    """The same in 64 bits from the definitions."""
    x, mods, prompt = x.double(), mods.double(), prompt.double()
    b, t, c = x.shape
    d = c // heads
    m = lambda i: mods[:, :, i]
    mm = lambda a, n: a @ w[n].double()
    _, _, y, _ = block_ref.gate_norm(x, scale=m(0), shift=m(1))
    qkv = mm(y, "qkv").view(b, t, 3 * heads, d)
    qk, _ = block_ref.rotary(qkv[:, :, :2 * heads], freqs, pos, pairs, "interleaved")
    h, _ = block_ref.attention(qk[:, :, :heads], qk[:, :, heads:], qkv[:, :, 2 * heads:], None, d ** -0.5)
    x, _, y, _ = block_ref.gate_norm(x, mm(h.view(b, t, c), "o1"), gate=m(2), scale=m(3), shift=m(4))
    kv = mm(prompt, "kv").view(b, prompt.shape[1], 2, heads, d)
    h, _ = block_ref.attention(mm(y, "q").view(b, t, heads, d), kv[:, :, 0], kv[:, :, 1], lens, d ** -0.5)
    x, _, y, _ = block_ref.gate_norm(x, mm(h.view(b, t, c), "o2"), gate=m(5), kind="rms", post_norm=True, residual_scale=0.5)
    return x, y


@pytest.mark.parametrize("dtype,tol", [("f32", 2e-5), ("bf16", 2e-2)])
@pytest.mark.parametrize("heads,d", [(4, 64), (2, 128), (5, 40)])
def test_a_block_matches_64_bits(dtype, tol, heads, d):
    """Relative 2-norm.  bf16: about twenty tensors rounded to 2^-8 at most (2^-9 on average) between x and the result, each carried with a
    factor of about one: sqrt(20) * 2^-9 = 0.9e-2.  fp32: the same with 2^-24, and sums of 2 c terms: 1e-6."""
    import torch
    from paper_2602_00608_b200 import binding as vd
    g = torch.Generator(device="cuda").manual_seed(11)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    b, t, c, n = 2, 150, heads * d, 33
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, mods, prompt = r(b, t, c), (0.3 * r(b, 1, 6, c)).to(dt), r(b, n, c).to(dt)
    lens = torch.tensor([n, 20], dtype=torch.int32, device="cuda")
    i = torch.arange(t, device="cuda", dtype=torch.int32)
    pos = torch.stack([i // 50, i % 50 // 10, i % 10], 1).expand(b, t, 3)
    pairs = (d // 2 - 2 * (d // 6), d // 6, d // 6)
    freqs = vd.rotary_frequencies(d, axis_pairs=pairs).cuda()
    w = {k: v.to(dt).float() for k, v in _weights(c, g).items()}
    old = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        got = block(vd, w, x.clone(), mods, prompt, lens, pos, freqs, pairs, heads, dt)
        torch.cuda.synchronize()
    finally:
        torch.backends.cuda.matmul.allow_tf32 = old
    want = block64(w, x, mods, prompt, lens, pos, freqs, pairs, heads)
    for a, e in zip(got, want):
        assert float((a.double() - e).norm() / e.norm()) <= tol


def test_a_block_in_front_of_the_decoder_in_one_graph():
    """A block step on the patches of a latent and the decode of it, captured together and replayed on new inputs."""
    import torch
    from paper_2602_00608_b200 import binding as vd, synth
    wl = synth.WORKLOADS[1]
    dec = vd.Decoder(wl.arch, wl.dtype, 8, 8, 1, wl.groups, wl.eps, synth.workload_weights(wl))
    g = torch.Generator(device="cuda").manual_seed(12)
    c, heads = 256, 4
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, mods, prompt, out = r(1, 64, c), 0.3 * r(1, 1, 6, c), r(1, 9, c), r(c, 4) * c ** -0.5
    i = torch.arange(64, device="cuda", dtype=torch.int32)
    pos = torch.stack([i // 8, i % 8], 1).unsqueeze(0)
    freqs, lens = vd.rotary_frequencies(64, axis_pairs=(16, 16)).cuda(), torch.tensor([7], dtype=torch.int32, device="cuda")
    w, frames = _weights(c, g), torch.empty((1,) + dec.out_shape, device="cuda")

    def step():
        _, y = block(vd, w, x.clone(), mods, prompt, lens, pos, freqs, (16, 16), heads, torch.float32)
        z = (y @ out).view(1, 8, 8, 4).permute(0, 3, 1, 2).contiguous()
        return dec.decode(z, frames)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x.copy_(r(1, 64, c))
    graph.replay()
    torch.cuda.synchronize()
    replayed = frames.clone()
    step()
    torch.cuda.synchronize()
    assert torch.equal(replayed, frames) and util.rel_l2(frames.cpu().numpy(), replayed.cpu().numpy()) == 0
    dec.check_status()
    dec.close()
