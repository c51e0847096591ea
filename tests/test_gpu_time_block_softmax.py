"""The time block with softmax attention: against its formula in double, snapshot by snapshot from a cache, trained with AdamW, and a whole training
step in a graph.  Tolerances of the composite are those of the block's other tests: a few roundings of the element type for each of seven steps."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _params(block, seed):
    rng = np.random.RandomState(seed)
    host = {}
    for n, s in block.shapes.items():
        a = rng.randn(*s).astype(np.float32) * (s[-1] ** -0.5 if n.endswith("weight") and len(s) == 2 else 0.3)
        if n in ("norm1.weight", "norm2.weight"):
            a += 1.0
        block.set_param(n, a)
        host[n] = block.get_param(n)
    return host


def _norm(x, w, b, eps):
    v, m = x.var(-1, unbiased=False, keepdim=True), x.mean(-1, keepdim=True)
    return (x - m) / (v + eps).sqrt() * w + b


def _stored(dtype):
    """x as it is when it has been stored in `dtype`, and so its gradient."""
    import torch

    class Stored(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return x.to(dtype).double()

        @staticmethod
        def backward(ctx, g):
            return g.to(dtype).double()
    return Stored.apply


def _formula(block, P, x, keep=None, lengths=None, r=lambda t: t):
    """In double; r: what happens to each array that the block keeps in its element type."""
    import torch
    T, N, W = x.shape
    h, d = block.heads, W // block.heads
    n = r(_norm(x, P["norm1.weight"], P["norm1.bias"], block.eps))
    qkv = r(n @ P["qkv.weight"].t() + P["qkv.bias"])
    q, k, v = (t.reshape(T, N, h, d).permute(1, 2, 0, 3) for t in qkv.split(W, -1))
    i = torch.arange(T, device=x.device)
    away = i[:, None] - i
    s = d ** -0.5 * q @ k.transpose(-1, -2)
    if block.buckets:
        far = block.reach
        s = s + P["attn.bias"][:, block._map.long()[away.clamp(-far, far) + far]]
    sees = (away >= 0)[None, None].expand(N, 1, T, T)
    if keep is not None:
        sees = sees & (keep.t() != 0)[:, None, None, :]
    row = None
    if lengths is not None:
        sees = sees & (i < lengths[:, None])[:, None, None, :]
        row = (i < lengths[:, None])
    p = torch.softmax(torch.where(sees, s, -1e30), -1) * sees
    if row is not None:
        p = p * row[:, None, :, None]
    o = r((p @ v).permute(2, 0, 1, 3).reshape(T, N, W))
    m = r(x + o @ P["out.weight"].t() + P["out.bias"])
    u = r(r(_norm(m, P["norm2.weight"], P["norm2.bias"], block.eps)) @ P["up.weight"].t() + P["up.bias"])
    f = {"relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[block.act]
    return r(m + r(f(u)) @ P["down.weight"].t() + P["down.bias"])


def _near(got, want, rough, what=""):
    """want: the formula in double; rough: with every array rounded to the element type where the block keeps it, forward and backward, which flips
    the same number of relus and moves the scores as far.  The block adds a rounding of the weights and of the scores' gradients (bf16), and of its sums
    (2^-24 each, some hundred in a row, sqrt(100) 2^-24 in the mean: fp32's arrays are rounded by as much once), so its error has up to some
    three times rough's variance in bf16 and some ten times in fp32; of short vectors the norms scatter by as much again."""
    import torch
    got, want, rough = (t.detach().double().reshape(want.shape) for t in (got, want, rough))
    f32 = float((rough - want).norm()) < 1e-4 * float(want.norm())
    err, own = float((got - want).norm()), float((rough - want).norm())
    worst, own_worst = float((got - want).abs().max()), float((rough - want).abs().max())
    room = 12 if f32 else 3
    assert err <= room * own + 1e-6 * float(want.norm()) and worst <= 2 * room * own_worst + 4e-6 * float(want.abs().max()), f"{what}: {err} by {own}, worst {worst} by {own_worst}"
    assert not torch.isnan(got).any()


def _both(block, host, x, dy, keep=None, lengths=None):
    """(y, dx, gradients) by the formula, and with its arrays rounded."""
    import torch
    out = []
    for r in (lambda t: t, _stored(block.dtype)):
        P = {n: torch.from_numpy(a).cuda().double().requires_grad_() for n, a in host.items()}
        X = x.double().requires_grad_()
        y = _formula(block, P, X, keep, lengths, r)
        (y * dy.double()).sum().backward()
        out.append((y.detach(), r(X.grad), {n: r(p.grad) for n, p in P.items()}))
    return out


CASES = [(5, 7, 32, 2, 48, "gelu", 8), (33, 20, 64, 8, 100, "silu", 0), (16, 40, 128, 8, 256, "relu", 6), (150, 3, 64, 1, 64, "gelu", 16)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("how", ["all", "keep", "lengths"])
def test_forward_and_backward(case, how, dtype):
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    T, N, W, h, hidden, act, buckets = case
    block = TimeBlock(W, h, hidden, dtype=dtype, act=act, attention="softmax", buckets=buckets, reach=20)
    host = _params(block, T)
    g = torch.Generator(device="cuda").manual_seed(T + N)
    x, dy = (torch.randn(T, N, W, generator=g, device="cuda").to(block.dtype) for _ in range(2))
    keep = (torch.rand(T, N, generator=g, device="cuda") < 0.7).to(torch.uint8) if how == "keep" else None
    lengths = torch.randint(0, T + 1, (N,), generator=g, device="cuda", dtype=torch.int32) if how == "lengths" else None
    y, dx = torch.empty_like(x), torch.empty_like(x)
    block.forward(x, y, keep=keep, lengths=lengths)
    block.backward(dy, dX=dx)
    want, rough = _both(block, host, x, dy, keep, lengths)
    _near(y, want[0], rough[0], "y")
    _near(dx, want[1], rough[1], "dx")
    for n in block.names:
        got, ref, by = torch.from_numpy(block.get_param(n + ".grad")).cuda(), want[2][n], rough[2][n]
        if n == "qkv.bias":      # a key's bias has no gradient: softmax does not see it, and what is left is rounding
            got, ref, by = (torch.cat([t[:W], t[2 * W:]]) for t in (got, ref, by))
        _near(got, ref, by, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_snapshots_from_a_cache(dtype):
    """A window of 50, and the same as 20 snapshots at once, then one or several at a time, from the keys and values kept."""
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    T, N, W, h = 90, 6, 64, 4
    block = TimeBlock(W, h, 96, dtype=dtype, attention="softmax", buckets=8, reach=16)
    host = _params(block, 1)
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(T, N, W, generator=g, device="cuda").to(block.dtype)
    keep = (torch.rand(T, N, generator=g, device="cuda") < 0.8).to(torch.uint8)
    P = {n: torch.from_numpy(a).cuda().double() for n, a in host.items()}
    want, rough = (_formula(block, P, x.double(), keep, r=r) for r in (lambda t: t, _stored(block.dtype)))
    cache = torch.full((T + 3, N, 2 * W), float("nan"), dtype=block.dtype, device="cuda")
    y = torch.empty_like(x)
    at = 0
    for n in (20, 1, 1, 7, 35, 1, 1, 24):
        block.forward(x[at:at + n], y[at:at + n], cache=cache, at=at, keep=keep[:at + n].contiguous(), train=False)
        at += n
    assert at == T
    _near(y, want, rough)
    assert torch.isnan(cache[T:].float()).all()


@pytest.mark.parametrize("dtype,bits", [("f32", 32), ("bf16", 32), ("bf16", 8)])
def test_training_steps(dtype, bits):
    """Forward, backward, AdamW: the parameters are those of the formula's step from the gradients that backward left, and the gradients those of the parameters."""
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    from paper_2309_03523_amd.time_block import TimeBlock
    T, N, W, h = 16, 25, 64, 4
    block = TimeBlock(W, h, 96, dtype=dtype, attention="softmax", buckets=6, reach=12)
    _params(block, 3)
    params, grads = block.trained()
    opt = AdamW(params, grads, masters=True, lr=0.01, weight_decay=0.02, bits=bits)
    g = torch.Generator(device="cuda").manual_seed(5)
    x, target = (torch.randn(T, N, W, generator=g, device="cuda").to(block.dtype) for _ in range(2))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    for step in range(1, 4):
        host = {n: block.get_param(n) for n in block.names}
        block.forward(x, y)
        dy = (y.float() - target.float()).to(block.dtype)
        block.backward(dy, dX=dx)
        want, rough = _both(block, host, x, dy)
        for n in ("down.weight", "attn.bias", "qkv.weight"):
            _near(torch.from_numpy(block.get_param(n + ".grad")).cuda(), want[2][n], rough[2][n], n)
        before = [(m if m is not None else p).double().clone() for p, m in zip(params, opt.masters)]
        opt.step()
        for p, m, gr, b in zip(params, opt.masters, grads, before):
            if step == 1:      # the first step: lr times the sign, nearly
                u = gr.double() / (gr.double().abs() + 1e-8)
                new = b * (1 - 0.01 * 0.02) - 0.01 * u
                assert float(((m if m is not None else p).double() - new).abs().max()) <= 0.01 * 32 * 2.0 ** -24 + 8 * 2.0 ** -24 * float(b.abs().max())
            if m is not None:
                assert torch.equal(m.to(p.dtype), p)


def test_a_captured_training_step():
    """Forward, backward and AdamW in one graph, replayed with an eager block of the same sizes alive: the same bits as eager steps."""
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    from paper_2309_03523_amd.time_block import TimeBlock
    T, N, W, h = 12, 30, 64, 4
    g = torch.Generator(device="cuda").manual_seed(5)
    x, dy = (torch.randn(T, N, W, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    sides = []
    for on_device in (True, True):
        block = TimeBlock(W, h, 96, dtype="bf16", attention="softmax", buckets=6, reach=12)
        _params(block, 3)
        opt = AdamW(*block.trained(), masters=True, lr=0.01, on_device=on_device)
        sides.append((block, opt, torch.empty_like(x), torch.empty_like(x)))

    def step(side):
        block, opt, y, dx = side
        block.forward(x, y)
        block.backward(dy, dX=dx)
        opt.step()

    for side in sides:
        step(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(sides[0])
    for _ in range(4):
        graph.replay()
        step(sides[1])
        torch.cuda.synchronize()
        for a, b in zip(sides[0][0].trained(), sides[1][0].trained()):
            assert all(torch.equal(s, t) for s, t in zip(a, b))
        assert torch.equal(sides[0][2], sides[1][2]) and torch.equal(sides[0][3], sides[1][3])
    assert sides[0][1].steps == 5


def test_refusals():
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    for kw in (dict(attention="linear"), dict(attention="softmax", decay=[0.5, 0.5]), dict(attention="softmax", buckets=300), dict(attention="softmax", buckets=16, reach=2)):
        with pytest.raises((ValueError, RuntimeError)):
            TimeBlock(32, 2, 64, **kw)
    block, old = TimeBlock(32, 2, 64, attention="softmax"), TimeBlock(32, 2, 64)
    x, y = torch.zeros(4, 3, 32, device="cuda"), torch.zeros(4, 3, 32, device="cuda")
    s = torch.zeros(3, 2, 16, 16, device="cuda")
    cache = torch.zeros(10, 3, 64, device="cuda")
    for kw in (dict(S0=s), dict(SN=s), dict(reset=torch.zeros(4, 3, dtype=torch.uint8, device="cuda")), dict(cache=cache), dict(cache=cache, train=False, at=7),
               dict(cache=cache, train=False, at=-1), dict(cache=cache[:, :, :32], train=False), dict(cache=cache.bfloat16(), train=False),
               dict(cache=cache, train=False, lengths=torch.ones(3, dtype=torch.int32, device="cuda")), dict(keep=torch.ones(3, 4, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            block.forward(x, y, **kw)
    for kw in (dict(keep=torch.ones(4, 3, dtype=torch.uint8, device="cuda")), dict(cache=cache, train=False)):
        with pytest.raises(ValueError):
            old.forward(x, y, **kw)
