"""The two ways from torch tensors to the block operators: both launch the same, and refuse the same."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vd():
    from paper_2602_00608_b200 import binding
    return binding


def _calls(vd):
    import torch
    g = torch.Generator(device="cuda").manual_seed(21)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    q, kv, lens = r(2, 70, 4, 64).bfloat16(), r(2, 50, 2, 2, 64).bfloat16(), torch.tensor([50, 13], dtype=torch.int32, device="cuda")
    x, h, mods, w = r(2, 9, 96), r(2, 9, 96).bfloat16(), r(2, 3, 3, 96).bfloat16(), r(96)
    freqs, pos = vd.rotary_frequencies(32, axis_pairs=(8, 8)).cuda(), torch.randint(0, 99, (2, 70, 2), generator=g, device="cuda", dtype=torch.int32)
    mod = dict(gate=mods[:, :, 0], scale=mods[:, :, 1], shift=mods[:, :, 2], mod_tokens=3)
    return [
        lambda: vd.op_cross_attention(q, kv[:, :, 0], kv[:, :, 1], lens),
        lambda: vd.op_cross_attention(q.float(), kv[:, :, 0].float(), kv[:, :, 1].float(), scale=0.25, impl=vd.VD_XATTN_PLAIN),
        lambda: vd.op_rotary(q, freqs, pos, layout="interleaved", axis_pairs=(8, 8)),
        lambda: vd.op_rotary(q, freqs, pos[:, :, 0], amplitude=0.5),
        lambda: vd.op_rotary(q, freqs, first_position=77),
        lambda: vd.op_gate_norm(x, h, **mod, weight=w, bias=w),
        lambda: vd.op_gate_norm(x, h, **mod, kind="rms", post_norm=True, post_weight=w, residual_scale=0.5, want_x=False),
        lambda: vd.op_gate_norm(x, eps=1e-3, want_y=False),
    ], [
        (lambda: vd.op_cross_attention(q, kv[:, :, 0], kv[:, :, 1], lens.long()), "int32"),
        (lambda: vd.op_cross_attention(q, kv[:, :, 0].float(), kv[:, :, 1]), "one type"),
        (lambda: vd.op_cross_attention(q, kv[:, :, 0].half(), kv[:, :, 1].half()), "one type"),
        (lambda: vd.op_cross_attention(q.half(), kv[:, :, 0].half(), kv[:, :, 1].half()), "float32 or bfloat16"),
        (lambda: vd.op_cross_attention(q, kv[:, :, 0], kv[:1, :, 1]), "k and v"),
        (lambda: vd.op_cross_attention(q, kv[:, :, 0].cpu(), kv[:, :, 1]), "on cpu"),
        (lambda: vd.op_cross_attention(q[:, :, :3], kv[:, :, 0], kv[:, :, 1]), "attention sizes"),
        (lambda: vd.op_cross_attention(q, kv[:, :, 0], kv[:, :, 1], scale=-1.0), "scale"),
        (lambda: vd.op_cross_attention(q.transpose(1, 3), q.transpose(1, 3), q.transpose(1, 3)), "side by side"),
        (lambda: vd.op_rotary(q, freqs.float()), "float64"),
        (lambda: vd.op_rotary(q, freqs, pos, axis_pairs=(8, 7)), "positions|axis_pairs"),
        (lambda: vd.op_rotary(q, freqs, pos, axis_pairs=(16,)), "positions"),
        (lambda: vd.op_rotary(q, freqs, layout="both"), "layout"),
        (lambda: vd.op_rotary(q, freqs, axis_pairs=(8, 8)), "positions"),
        (lambda: vd.op_gate_norm(x, h, gate=mods[:, :, 0], mod_tokens=4, scale=mods[:, :2, 0]), "scale|side by side"),
        (lambda: vd.op_gate_norm(x, h, gate=mods[:, :, 0].float(), scale=mods[:, :, 1], mod_tokens=3), "one type"),
        (lambda: vd.op_gate_norm(x, gate=mods[:, :, 0], mod_tokens=3), "without h"),
        (lambda: vd.op_gate_norm(x, h, kind="batch"), "layer or rms"),
        (lambda: vd.op_gate_norm(x, h, weight=w.bfloat16()), "weight"),
        (lambda: vd.op_gate_norm(x, h, mod_tokens=0), "mod_tokens"),
        (lambda: vd.op_gate_norm(x, h, eps=0.0), "eps"),
    ]


def test_the_native_way_is_there_and_launches_the_same(vd, monkeypatch):
    import torch
    assert vd._calls(), "paper_2602_00608_b200/_vd_torch.so has not been built"
    good, _ = _calls(vd)
    taken = []
    native = vd._calls()

    class Watched:
        def __getattr__(self, name):
            def call(*a):
                r = getattr(native, name)(*a)
                taken.append((name, r))
                return r
            return call

    monkeypatch.setattr(vd, "_native", Watched())
    first = [f() for f in good]
    assert len(taken) == len(good) and all(r == vd.VD_OK for _, r in taken), taken
    monkeypatch.setattr(vd, "_native", False)
    again = [f() for f in good]
    torch.cuda.synchronize()
    flat = lambda outs: [t for o in outs for t in (o if isinstance(o, tuple) else (o,)) if t is not None]
    a, b = flat(first), flat(again)
    assert len(a) == len(b) and all(torch.equal(s, t) for s, t in zip(a, b))


@pytest.mark.parametrize("native", [True, False])
def test_both_ways_refuse(vd, monkeypatch, native):
    if not native:
        monkeypatch.setattr(vd, "_native", False)
    import re
    for i, (call, why) in enumerate(_calls(vd)[1]):
        with pytest.raises(vd.VdError) as e:
            call()
        assert e.value.status == vd.VD_ERR_INVALID_ARG and re.search(why, str(e.value)), (i, str(e.value))


@pytest.mark.parametrize("native", [True, False])
def test_calls_take_the_current_stream(vd, monkeypatch, native):
    """Work of another stream that a call's input waits for: a call on the wrong stream would see the old input."""
    import torch
    if not native:
        monkeypatch.setattr(vd, "_native", False)
    x = torch.zeros((64, 4096, 256), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            x.add_(1.0)
        r, _ = vd.op_gate_norm(x, want_y=False)
    torch.cuda.synchronize()
    assert (r == 20).all()


@pytest.mark.parametrize("native", [True, False])
def test_numbers_that_are_tensors_count_as_they_are_at_the_call(vd, monkeypatch, native):
    import torch
    if not native:
        monkeypatch.setattr(vd, "_native", False)
    g = torch.Generator(device="cuda").manual_seed(22)
    q = torch.randn((1, 9, 2, 64), generator=g, device="cuda")
    k, v, x = torch.randn_like(q), torch.randn_like(q), torch.randn((1, 9, 64), generator=g, device="cuda")
    freqs, n = vd.rotary_frequencies(64).cuda(), torch.tensor(0.5)
    calls = [lambda n: vd.op_cross_attention(q, k, v, scale=n), lambda n: vd.op_rotary(q, freqs, amplitude=n), lambda n: vd.op_gate_norm(x, x, residual_scale=n)[0],
             lambda n: vd.op_gate_norm(x, eps=n)[1]]
    for call in calls:
        for value in (0.5, 0.125):
            n.fill_(value)
            assert torch.equal(call(n), call(value))
