"""AdamW over many tensors, states in 32 and 8 bits, against its formula in double and its 8-bit states bit for bit.

Tolerances: in fp32 each operation rounds once, 2^-24 of its result.  m: three operations on |b1 m| + |(1 - b1) g|, and the factors' own
rounding: 5 2^-24 of that; v the same with one more.  The step's quotient: m's, the root's, a factor's and three operations' roundings relative to
its parts, 16 2^-24 of |m| terms over the denominator; then p: 3 2^-24 of |p| + lr (quotient + decay |p|)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
HALF = {"f32": 0.0, "bf16": 2.0 ** -8}


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _rows(shape, dtype, g, std=1.0, pad=0, fill=7.0):
    """Rows at a pitch wider than they are, what is behind them filled with something that is not to be touched."""
    import torch
    F = shape[-1]
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    buf = torch.full((*shape[:-1], -(-F // per) * per + pad * per), fill, device="cuda", dtype=dtype)
    buf[..., :F] = (std * torch.randn(*shape, generator=g, device="cuda")).to(dtype)
    return buf[..., :F], buf


SHAPES = [(1,), (3,), (16,), (255,), (257,), (4096,), (4100,), (1, 5), (7, 1), (5, 17), (33, 16), (100, 172), (64, 128), (300, 41), (2, 3, 24)]


def _make(dtype, seed, *, masters=False, pad=0, shapes=SHAPES):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    p, g1, ms = [], [], []
    for s in shapes:
        p.append(_rows(s, _dt(dtype), g, 0.1, pad)[0])
        g1.append(_rows(s, _dt(dtype), g, 0.01, 2 * pad, float("nan"))[0])
        if masters:
            m = _rows(s, torch.float32, g, 0.1, pad)[0]
            p[-1].copy_(m)
            ms.append(m)
    return p, g1, ms if masters else None


def _again(x):
    """A copy in rows at a pitch of its own."""
    import torch
    per = 16 // x.element_size()
    y = torch.zeros(*x.shape[:-1], -(-x.shape[-1] // per) * per, dtype=x.dtype, device="cuda")[..., :x.shape[-1]]
    return y.copy_(x)


def _flat(t):
    return t.reshape(-1, t.shape[-1])


def _reference(p, g, m, v, t, lr, b1, b2, eps, wd):
    """(p, m, v) in double, and how far each may be off."""
    p, g, m, v = (x.double() for x in (p, g, m, v))
    m1, am = b1 * m + (1 - b1) * g, (b1 * m).abs() + ((1 - b1) * g).abs()
    v1 = b2 * v + (1 - b2) * g * g
    tm, tv = 5 * E * am, 6 * E * v1
    den = (v1 / (1 - b2 ** t)).sqrt() + eps
    u, au = m1 / (1 - b1 ** t) / den, am / (1 - b1 ** t) / den
    p1 = p - lr * (u + wd * p)
    return (p1, 3 * E * (p.abs() + lr * (u.abs() + wd * p.abs())) + lr * 16 * E * au + 2 * E * p1.abs()), (m1, tm), (v1, tv)


def _near(got, want, tol, what):
    import torch
    got, tol = got.double(), tol.expand_as(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    ok = ~torch.isnan(want)
    off = float(((got - want).abs() - tol)[ok].max()) if ok.any() else 0.0
    assert off <= 0, f"{what}: over by {off}"


@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("dtype,masters", [("f32", False), ("bf16", False), ("bf16", True)])
def test_steps_in_32_bits(dtype, masters, pad):
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    p, g, ms = _make(dtype, 1, masters=masters, pad=pad)
    wd = [0.1 * (i % 3) for i in range(len(p))]
    opt = AdamW(p, g, masters=ms, lr=0.02, betas=(0.8, 0.95), eps=1e-6, weight_decay=wd)
    at = [x.clone() for x in (ms if masters else p)]
    held = [(torch.zeros_like(_flat(x), dtype=torch.float32), torch.zeros_like(_flat(x), dtype=torch.float32)) for x in p]
    for t in range(1, 4):
        before = [x.clone() for x in (ms if masters else p)]
        opt.step()
        for k, x in enumerate(p):
            F = x.shape[-1]
            (P, tp), (M, tm), (V, tv) = _reference(_flat(before[k]), _flat(g[k]), *held[k], t, 0.02, 0.8, 0.95, 1e-6, wd[k])
            m, v = opt.states[k]["m"], opt.states[k]["v"]
            _near(m[:, :F], M, tm, "m")
            _near(v[:, :F], V, tv, "v")
            assert not m[:, F:].any() and not v[:, F:].any()
            if masters:
                _near(_flat(ms[k]), P, tp, "master")
                assert torch.equal(ms[k].to(x.dtype), x)
            else:
                _near(_flat(x), P, tp + HALF[dtype] * P.abs(), "p")
            held[k] = (m[:, :F].clone(), v[:, :F].clone())
        for k in range(len(g)):
            g[k].mul_(0.7).add_(0.003)
    assert opt.steps == 3 and all(not torch.equal(a, b) for a, b in zip(at, ms if masters else p))
    for x in p:      # what is behind the rows
        if x.dim() > 1 and x.stride(-2) > x.shape[-1]:
            behind = torch.as_strided(x, (x.shape[-2], x.stride(-2) - x.shape[-1]), (x.stride(-2), 1), x.storage_offset() + x.shape[-1])
            assert bool((behind == 7).all())


def _pow2(k):
    """2^k for whole k, exactly (a power function need not be)."""
    import torch
    return ((k.long() + 1023) << 52).view(torch.float64)


def _held(x, root):
    """The 8-bit form by its definition: (codes as their values, scale) of flat blocks of 256."""
    import torch
    n = x.numel()
    b = torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)
    top = torch.where(torch.isfinite(b), b.abs(), 0).amax(1).double()
    k = torch.where(top > 0, torch.ceil(torch.log2(top / 448)), 0.0)
    k = torch.where((top > 0) & (top / 448 > _pow2(k)), k + 1, torch.where((top > 0) & (top / 448 <= _pow2(k - 1)), k - 1, k)).clamp(min=-126)
    scale = _pow2(k)[:, None]
    y = b.double() / scale
    # e4m3: three bits behind the point of a normal number, steps of 2^-9 below 2^-6
    step = _pow2(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    q = torch.round(y / step) * step
    if root:
        q = torch.where(b > 0, q.clamp(min=2.0 ** -9), q)
    return torch.where(torch.isfinite(b), q, torch.nan).view(-1)[:n], scale[:, 0]


@pytest.mark.parametrize("dtype,masters", [("f32", False), ("bf16", True), ("bf16", False)])
def test_states_in_8_bits_are_what_their_definition_says(dtype, masters):
    """The states before rounding are those of the same operations in fp32, one after the other, so the codes are the same."""
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    p, g, ms = _make(dtype, 2, masters=masters)
    g[5].mul_(1e-30)      # scales far below, some numbers zero, and a block that is all zero
    g[6].zero_()
    g[7].mul_(1e30)
    opt = AdamW(p, g, masters=ms, lr=0.01, betas=(0.9, 0.99), weight_decay=0.0, bits=8)
    for t in range(1, 4):
        before = [x.float().clone() for x in (ms if masters else p)]
        old = [{k: v.clone() for k, v in s.items()} for s in opt.states]
        opt.step()
        for k, x in enumerate(p):
            F, pitch = x.shape[-1], opt.states[k]["m"].shape[1]
            G = torch.nn.functional.pad(_flat(g[k]).float(), (0, pitch - F)).view(-1)
            wide = lambda n: old[k][n].float().view(-1) * old[k][n + "_scale"].repeat_interleave(256)[:G.numel()]  # noqa: E731
            m = wide("m") * 0.9 + G * (1 - 0.9)
            r = wide("v")
            v = (r * r) * 0.99 + (G * G) * (1 - 0.99)
            for name, want, root in (("m", m, False), ("v", v.sqrt(), True)):
                q, scale = _held(want, root)
                got = opt.states[k][name].float().view(-1).double()
                assert torch.equal(opt.states[k][name + "_scale"].double(), scale), (t, k, name)
                assert bool(((got == q) | (torch.isnan(got) & torch.isnan(q))).all()), (t, k, name)      # 1e30's square is none in fp32: NaN
            (P, tp), *_ = _reference(_flat(before[k]), _flat(g[k]), m.view(-1, pitch)[:, :F] * 0, v.view(-1, pitch)[:, :F] * 0, t, 0, 0.9, 0.99, 1e-8, 0)
            M, V = m.double().view(-1, pitch)[:, :F], v.double().view(-1, pitch)[:, :F]
            u = M / (1 - 0.9 ** t) / ((V / (1 - 0.99 ** t)).sqrt() + 1e-8)
            want = _flat(before[k]).double() - 0.01 * u
            tol = 4 * E * (_flat(before[k]).abs() + 0.01 * u.abs()) + 0.01 * 16 * E * u.abs() + 2.0 ** -126
            # roots below fp32's normal numbers have fewer bits
            tol = torch.where(V < 2.0 ** -120, tol + 0.02 * (u.abs() + 1), tol)
            _near(_flat(ms[k] if masters else x), want, tol if masters or dtype == "f32" else tol + HALF[dtype] * want.abs(), "p")
    assert any(bool((s["m_scale"] == 1).any()) for s in opt.states)


@pytest.mark.parametrize("bits", [8, 32])
def test_what_is_not_finite_stays_where_it_is(bits):
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    p, g, _ = _make("f32", 3, shapes=[(64, 40), (700,)])
    q, h = [_again(x) for x in p], [_again(x) for x in g]
    g[0][3, 7], g[1][500] = float("nan"), float("inf")
    a, b = AdamW(p, g, bits=bits), AdamW(q, h, bits=bits)
    for _ in range(2):
        a.step()
        b.step()
    for x, y in zip(p, q):
        bad = ~torch.isfinite(x)
        assert int(bad.sum()) == 1
        if bits == 32:
            assert torch.equal(x[~bad], y[~bad])
    for s, u in zip(a.states, b.states):
        for n in ("m", "v"):
            x, y = s[n].float(), u[n].float()
            assert int((~torch.isfinite(x)).sum()) == 1
            if bits == 32:
                assert torch.equal(x[torch.isfinite(x)], y[torch.isfinite(x)])


def test_many_tensors_and_a_large_one():
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    shapes = [(1 + i % 7, 8 + i % 5) for i in range(500)] + [(3000, 1001)]
    p, g, _ = _make("f32", 4, shapes=shapes)
    before = [x.clone() for x in p]
    AdamW(p, g, lr=0.1, weight_decay=0.0, eps=0.0).step()
    for x, y, d in zip(p, before, g):      # the first step: lr times the sign
        off = (x.double() - (y.double() - 0.1 * d.double().sign())).abs()
        assert float(off.max()) <= 0.1 * 16 * E + 4 * E * float(y.abs().max())


def test_resumed_states_go_on_as_they_would_have():
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    for bits in (8, 32):
        p, g, ms = _make("bf16", 5, masters=True)
        a = AdamW(p, g, masters=ms, bits=bits)
        a.step()
        q, h = [_again(x) for x in p], [_again(x) for x in ms]
        b = AdamW(q, g, masters=h, bits=bits, states=[{k: v.clone() for k, v in s.items()} for s in a.states], steps=a.steps)
        a.step()
        b.step()
        assert all(torch.equal(x, y) for x, y in zip(p + ms, q + h))


@pytest.mark.parametrize("bits", [8, 32])
def test_a_captured_step_counts_and_takes_the_rate_of_the_device(bits):
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    p, g, _ = _make("f32", 6)
    q, h = [_again(x) for x in p], [_again(x) for x in g]
    a, b = AdamW(p, g, bits=bits, on_device=True), AdamW(q, h, bits=bits)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    assert a.steps == 0
    for t in range(1, 5):
        if t == 3:
            a.set_lr(0.05)
            b.set_lr(0.05)
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        assert a.steps == t == b.steps
        for x, y, s, u in zip(p, q, a.states, b.states):
            # the factors are made by other functions: two roundings of 2^-24 apart in a step
            assert float((x - y).abs().max()) <= 1e-6 and torch.equal(s["m"].float(), u["m"].float())
        for x, y in zip(g, h):
            x.mul_(0.5)
            y.mul_(0.5)
    a.step()
    b.step()
    assert a.steps == 5


def test_on_another_stream_and_after_release():
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    p, g, _ = _make("f32", 7)
    q = [_again(x) for x in p]
    a, b = AdamW(p, g), AdamW(q, g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a.step(stream=s)
    b.step()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(p, q))
    a.release()
    with pytest.raises(RuntimeError, match="released"):
        a.step()


def test_refusals():
    import torch
    from paper_2309_03523_amd import binding
    from paper_2309_03523_amd.optimizer import AdamW
    p, g, _ = _make("f32", 8, shapes=[(4, 16), (9,)])
    for kw in (dict(bits=4), dict(lr=-1.0), dict(lr=float("nan")), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(weight_decay=[0.1]),
               dict(weight_decay=-0.1), dict(masters=[None]), dict(states=[]), dict(steps=-1)):
        with pytest.raises(ValueError):
            AdamW(p, g, **kw)
    for a, b in (([], []), (p, g[:1]), (p, [g[0], g[1][:8]]), (p, [g[0].cpu(), g[1]]), ([p[0].cpu(), p[1]], g), (p, [g[0].half(), g[1]])):
        with pytest.raises(ValueError):
            AdamW(a, b)
    for a, b, kw in (([p[0], p[0][1:2]], [g[0], g[0][2:3]], {}), ([p[0]], [p[0]], {}), (p, g, dict(masters=[torch.zeros(4, 16, device="cuda"), None]))):
        with pytest.raises(binding.DgcError):
            AdamW(a, b, **kw)
    s = AdamW(p, g, bits=8).states
    for bad in (dict(s[0], m=s[0]["m"][:2]), dict(s[0], m_scale=None), dict(s[0], v=s[0]["v"].float())):
        with pytest.raises((ValueError, binding.DgcError)):
            AdamW(p, g, bits=8, states=[bad, s[1]])
    one = AdamW(p, g)
    with pytest.raises(ValueError):
        one.set_lr(float("inf"))
    side = torch.zeros(6, 32, device="cuda")      # columns side by side in one buffer are apart
    AdamW([side[:, :16], side[:, 16:]], [torch.ones(6, 16, device="cuda")] * 2).step()
    assert bool((side != 0).all())
