"""The time block: its operators run together, as they are used, against the same formulas in double with torch's gradients.

Tolerances: fp32 steps are each off by under 4e-6 of the magnitudes they add up, the chain has twelve and a norm multiplies by up to
1/std (about 1 here): 2e-4 of a tensor's largest value.  bf16 rounds the activations ten times on the way, by half a step 2^-8
each of the value at hand: 10 * 2^-8 of the root mean square, times up to 2 where the gradients add up two branches: 0.08."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _params(block, seed):
    rng = np.random.default_rng(seed)
    out = {}
    for n, s in block.shapes.items():
        if len(s) == 2:
            out[n] = rng.normal(0, s[1] ** -0.5, s).astype(np.float32)
        else:
            out[n] = ((1.0 if n.startswith("norm") and n.endswith("weight") else 0.0) + rng.normal(0, 0.2, s)).astype(np.float32)
    block.set_params(out)
    return {n: block.get_param(n) for n in out}      # as rounded


def _norm(x, w, b, eps):
    xc = x - x.mean(-1, keepdim=True)
    return xc / (xc.square().mean(-1, keepdim=True) + eps).sqrt() * w + b


def _formula(block, P, x, s0, lengths, reset):
    """Output and last state in double; P: dict of double tensors."""
    import torch
    T, N, W = x.shape
    h = block.heads
    d = W // h
    qkv = _norm(x, P["norm1.weight"], P["norm1.bias"], block.eps) @ P["qkv.weight"].t() + P["qkv.bias"]
    q, k, v = (t.reshape(T, N, h, d) for t in qkv.split(W, -1))
    S = s0
    g = block._decay.double()[None, :, None, None]
    o = []
    for t in range(T):
        link = g * S if reset is None else torch.where((reset[t] != 0)[:, None, None, None], 0.0, g * S)
        new = link + k[t][..., :, None] * v[t][..., None, :]
        on = torch.ones(N, dtype=torch.bool, device=x.device) if lengths is None else t < lengths
        S = torch.where(on[:, None, None, None], new, S)
        o.append(torch.where(on[:, None, None], (q[t][..., :, None] * S).sum(-2) * d ** -0.5, 0.0).reshape(N, W))
    m = x + torch.stack(o) @ P["out.weight"].t() + P["out.bias"]
    p = _norm(m, P["norm2.weight"], P["norm2.bias"], block.eps) @ P["up.weight"].t() + P["up.bias"]
    u = {"gelu": p * torch.special.ndtr(p), "relu": torch.relu(p), "silu": p * torch.sigmoid(p), "none": p}[block.act]
    return m + u @ P["down.weight"].t() + P["down.bias"], S


def _near(got, want, dtype):
    want = want.detach()
    err = (got.double() - want).abs().max()
    size = want.abs().max() if dtype == "f32" else want.square().mean().sqrt()
    if dtype == "f32":
        assert err <= 2e-4 * size
    else:
        assert (got.double() - want).square().mean().sqrt() <= 0.08 * size


CASES = [(5, 7, 32, 2, 48, "gelu"), (33, 20, 64, 8, 100, "silu"), (16, 40, 128, 8, 256, "relu"), (300, 2, 64, 1, 64, "gelu")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES)
def test_forward_and_backward(case, dtype):
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    T, N, W, h, hidden, act = case
    block = TimeBlock(W, h, hidden, dtype=dtype, act=act)
    host = _params(block, T)
    g = torch.Generator(device="cuda").manual_seed(T + N)
    x, dy = (torch.randn(T, N, W, generator=g, device="cuda").to(block.dtype) for _ in range(2))
    s0, dsn = (torch.randn(N, h, W // h, W // h, generator=g, device="cuda") for _ in range(2))
    reset = (torch.rand(T, N, generator=g, device="cuda") < 0.1).to(torch.uint8)
    y, sn, dx, ds0 = torch.empty_like(x), torch.empty_like(s0), torch.empty_like(x), torch.empty_like(s0)
    block.forward(x, y, S0=s0, SN=sn, reset=reset)
    block.backward(dy, dX=dx, dSN=dsn, dS0=ds0)
    P = {n: torch.from_numpy(a).cuda().double().requires_grad_() for n, a in host.items()}
    X, S = x.double().requires_grad_(), s0.double().requires_grad_()
    want, last = _formula(block, P, X, S, None, reset)
    ((want * dy.double()).sum() + (last * dsn.double()).sum()).backward()
    _near(y, want, dtype)
    _near(sn, last, dtype)
    _near(dx, X.grad, dtype)
    _near(ds0, S.grad, dtype)
    for n in P:
        _near(torch.from_numpy(block.get_param(n + ".grad")).cuda(), P[n].grad, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_windows_and_snapshots_chain(dtype):
    """One window of 40, and the same as a window of 33 and seven single snapshots with the states handed on, behind a structure encoder's
    rows of ragged sequences."""
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    T, N, W, h = 40, 30, 64, 4
    block = TimeBlock(W, h, 96, dtype=dtype)
    _params(block, 1)
    x = torch.randn(T, N, W, device="cuda").to(block.dtype)
    y, z = torch.empty_like(x), torch.empty_like(x)
    sn = torch.zeros(N, h, W // h, W // h, device="cuda")
    block.forward(x, y, SN=sn)
    s = torch.zeros_like(sn)
    block.forward(x[:33], z[:33], S0=s, SN=s, train=False)
    for t in range(33, T):
        block.forward(x[t:t + 1], z[t:t + 1], S0=s, SN=s, train=False)
    _near(z, y.double(), dtype)
    _near(s, sn.double(), "f32" if dtype == "f32" else dtype)
    with pytest.raises(RuntimeError, match="train=True"):
        block.backward(x)


def test_behind_a_structure_encoder():
    """A GCN layer's output goes through the block; rows behind a vertex' last snapshot keep to themselves."""
    import torch
    from paper_2309_03523_amd.runner import DeviceWorkload
    from paper_2309_03523_amd.time_block import TimeBlock
    from workloads import synth
    wl = synth.config1(seed=0, random_bias=True)
    wl.time_kind = "none"
    wl.params = {k: v for k, v in wl.params.items() if k.startswith("gcn")}
    wl.H0 = None
    dw = DeviceWorkload(wl)
    x = dw.forward()
    T, N, W = x.shape
    block = TimeBlock(W, 2, 2 * W)
    host = _params(block, 2)
    lengths = torch.randint(0, T + 1, (N,), device="cuda", dtype=torch.int32)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dy = torch.randn_like(x)
    for given in (None, lengths):      # the first call leaves its rows in the buffers
        block.forward(x, y, lengths=given)
        block.backward(dy, dX=dx)
    P = {n: torch.from_numpy(a).cuda().double().requires_grad_() for n, a in host.items()}
    X = x.double().requires_grad_()
    want, _ = _formula(block, P, X, torch.zeros(N, 2, W // 2, W // 2, dtype=torch.float64, device="cuda"), lengths, None)
    (want * dy.double()).sum().backward()
    _near(y, want, "f32")
    _near(dx, X.grad, "f32")
    for n in P:
        _near(torch.from_numpy(block.get_param(n + ".grad")).cuda(), P[n].grad, "f32")
    dw.layer.destroy()


def test_captured_step():
    """A training step captured after an eager one, replayed with other inputs while another size runs between."""
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    T, N, W = 12, 50, 32
    block = TimeBlock(W, 2, 64, dtype="bf16")
    _params(block, 3)
    x, dy = (torch.randn(T, N, W, device="cuda").to(torch.bfloat16) for _ in range(2))
    y, dx = torch.empty_like(x), torch.empty_like(x)

    def step():
        block.forward(x, y)
        block.backward(dy, dX=dx)

    step()
    torch.cuda.synchronize()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):        # sizes that no eager call has had are refused
        y.mul_(1.0)
        with pytest.raises(RuntimeError, match="eager call"):
            block.forward(x[:3], y[:3])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    small = torch.randn(1, 9, W, device="cuda").to(torch.bfloat16)
    for _ in range(3):
        x.mul_(0.8).add_(0.1)
        step()
        torch.cuda.synchronize()
        want = [y.clone(), dx.clone()] + [block.get_param(n + ".grad") for n in block.shapes]
        block.forward(small, torch.empty_like(small), train=False)
        y.zero_(), dx.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1])
        for n, a in zip(block.shapes, want[2:]):
            np.testing.assert_array_equal(block.get_param(n + ".grad"), a)


@pytest.mark.parametrize("T", [1, 9, 40])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_with_the_state_in_place(T, dtype):
    """SN given as S0 itself: the same output, state and gradients, bit for bit, as with states of their own."""
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    N, W, h = 13, 32, 2
    block = TimeBlock(W, h, 40, dtype=dtype)
    _params(block, 4)
    x, dy = (torch.randn(T, N, W, device="cuda").to(block.dtype) for _ in range(2))
    s0, dsn = (torch.randn(N, h, W // h, W // h, device="cuda") for _ in range(2))
    state = s0.clone()
    for turn in range(2):      # the second call finds the copy's place made
        out = []
        for given, left in ((s0, torch.empty_like(s0)), (state, state)):
            y, dx, ds0 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(s0)
            block.forward(x, y, S0=given, SN=left)
            block.backward(dy, dX=dx, dSN=dsn, dS0=ds0)
            out.append([y, left.clone(), dx, ds0] + [torch.from_numpy(block.get_param(n + ".grad")) for n in block.shapes])
        assert all(torch.equal(a, b) for a, b in zip(*out))
        s0.copy_(state)


def test_a_captured_training_step_with_the_state_in_place():
    """Truncated back-propagation through time: each replay starts from the state that the one before left."""
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    T, N, W, h = 6, 21, 32, 4
    block = TimeBlock(W, h, 64)
    _params(block, 5)
    x, dy = torch.randn(T, N, W, device="cuda"), torch.randn(T, N, W, device="cuda")
    y, dx, s = torch.empty_like(x), torch.empty_like(x), torch.zeros(N, h, W // h, W // h, device="cuda")

    def step():
        block.forward(x, y, S0=s, SN=s)
        block.backward(dy, dX=dx)

    want, first = [], s.clone()
    for _ in range(4):       # with states of their own
        left = torch.empty_like(s)
        block.forward(x, y, S0=first, SN=left)
        block.backward(dy, dX=dx)
        want.append([t.clone() for t in (y, dx, left)])
        first = left
    step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    s.zero_()
    for turn in range(4):
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, dx, s), want[turn]))
        block.forward(x[:2], y[:2].clone(), train=False)


def _busy(stream):
    """Some 50 ms of work ahead of what is enqueued on the stream next."""
    import torch
    with torch.cuda.stream(stream):
        a = torch.zeros(8192, 8192, device="cuda")
        for _ in range(6):
            a = a @ a


@pytest.mark.parametrize("hidden", [64, 100])      # a pitch of its own, and rows inside a wider one
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_calls_on_another_stream(dtype, hidden):
    """Parameters, gradients and buffers follow the stream that a call was given: nothing here waits but the block itself."""
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    T, N, W = 10, 300, 64
    g = torch.Generator(device="cuda").manual_seed(6)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    x, dy = (torch.randn(T, N, W, generator=g, device="cuda").to(dt) for _ in range(2))

    def results(stream):
        block = TimeBlock(W, 4, hidden, dtype=dtype)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        out = []
        for seed in (7, 8):
            _params(block, seed)
            if stream is not None:
                _busy(stream)
            block.forward(x, y, stream=stream)
            block.backward(dy, dX=dx, stream=stream)
            out += [block.get_param(n + ".grad") for n in block.shapes]
            if stream is not None:
                _busy(stream)
            z = torch.empty_like(x)
            block.forward(x, z, train=False, stream=stream)
            block.set_param("qkv.weight", np.zeros(block.shapes["qkv.weight"], np.float32))      # not before that call has read it
            out += [t.float().cpu().numpy() for t in (y, dx, z)]
            if stream is not None:
                _busy(stream)
            block.forward(x, z, train=False, stream=stream)
            block.release()
            used = [torch.full((T, N, k * W), float("nan"), device="cuda").to(dt) for k in (1, 1, 1, 3)]      # memory that was dropped
            torch.cuda.synchronize()
            out.append(z.float().cpu().numpy())
            del used
        return out

    want = results(None)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    got = results(stream)
    assert all(np.array_equal(a, b) for a, b in zip(want, got)), [bool(np.array_equal(a, b)) for a, b in zip(want, got)]


def test_new_sizes_are_refused_on_a_capturing_stream_that_is_not_the_current_one():
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    block = TimeBlock(32, 2, 64)
    x = torch.randn(4, 9, 32, device="cuda")
    y, s0 = torch.empty_like(x), torch.zeros(9, 2, 16, 16, device="cuda")
    block.forward(x, y, S0=s0, SN=torch.empty_like(s0))
    want, aside, graph = y.clone(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        on = torch.cuda.current_stream()
        with torch.cuda.stream(aside):
            with pytest.raises(RuntimeError, match="eager call"):
                block.forward(x[:3], y[:3], stream=on)
            with pytest.raises(RuntimeError, match="eager call"):
                block.forward(x, y, S0=s0, SN=s0, stream=on)
            block.forward(x, y, S0=s0, stream=on)
    for _ in range(2):
        y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_buffers_of_many_sizes():
    """A graph whose vertices come and go: what the block holds stays that of a few sizes, a captured size outlives them all, and memory
    that is let go under a queue of work is not given away early."""
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    W, h = 64, 4
    block = TimeBlock(W, h, 128)
    _params(block, 9)
    x = torch.randn(1, 4200, W, device="cuda")
    y = torch.empty_like(x)
    block.forward(x, y, train=False)
    want = y.clone()
    graph, z = torch.cuda.CUDAGraph(), torch.empty_like(x[:, :700])
    block.forward(x[:, :700], z, train=False)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        block.forward(x[:, :700], z, train=False)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for n in range(4000, 4060):
        block.forward(x[:, :n], y[:, :n], train=False)
        assert torch.equal(y[:, :n], want[:, :n])
    rows = 4200 * W * 4 * (1 + 3 + 1 + 1 + 2)      # n, qkv, o, m, u
    assert torch.cuda.memory_allocated() - before <= (block.SIZES + 1) * (rows + (1 << 16))
    for _ in range(2):
        z.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, want[:, :700])
    stream = torch.cuda.Stream()
    _busy(stream)
    out = [torch.empty(1, n, W, device="cuda") for n in range(3000, 3000 + 3 * block.SIZES)]
    for o in out:
        block.forward(x[:, :o.shape[1]], o, train=False, stream=stream)
    used = [torch.full((1, 3000, k * W), float("nan"), device="cuda") for k in (1, 3, 1, 1, 2) * 3 * block.SIZES]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[:, :o.shape[1]]) for o in out)
    del used


@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
def test_gradients_behind_the_activation_in_two_parts(act):
    """exact=True: the gradients that a rounded dy act'(p) reaches (up, its bias not, and what lies before it) come closer to the formula's, the others
    are the same bits; with RELU all are."""
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    T, N, W = 11, 60, 64
    g = torch.Generator(device="cuda").manual_seed(12)
    x, dy = (torch.randn(T, N, W, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    grads = []
    for exact in (False, True):
        block = TimeBlock(W, 4, 200, dtype="bf16", act=act, exact=exact)
        host = _params(block, 12)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        block.forward(x, y)
        block.backward(dy, dX=dx)
        grads.append({"x": dx.float().cpu().numpy(), **{n: block.get_param(n + ".grad") for n in block.shapes}})
    same = {n for n in grads[0] if np.array_equal(grads[0][n], grads[1][n])}
    assert same == (set(grads[0]) if act == "relu" else {"up.bias", "down.weight", "down.bias"})
    P = {n: torch.from_numpy(a).cuda().double().requires_grad_() for n, a in host.items()}
    X = x.double().requires_grad_()
    want, _ = _formula(block, P, X, torch.zeros(N, 4, 16, 16, dtype=torch.float64, device="cuda"), None, None)
    (want * dy.double()).sum().backward()
    for n in ("x", "up.weight"):
        w = X.grad if n == "x" else P[n].grad
        _near(torch.from_numpy(grads[1][n]).cuda(), w, "bf16")


def _near_in_rows(got, want, limit, name):
    """Every row's error within `limit` of the tensor's root mean square, every element's within five times that.

    An activation's rounding is off by at most half a step, 2^-8 of it.  From X to Y there are seven of them (n, q/k/v, o, m, n2, u, Y), ten
    with the gradients' way back, doubled where two branches add up: 0.08, as for the whole tensor.  Of a row that is a bound as well: the
    products' rows have norms near 1, so a row's error is a sum of as many roundings.  A row's elements scatter about it: five deviations hold
    a hundred thousand of them.  States are sums of k and v, two roundings each (n, then the product's): 4 * 2^-8 = 0.016, rounded up to 0.02; the first state's
    gradient is one of q (2) and of o's gradient (du, n2's, m's, o's and Y's own twice over the branches): 10 * 2^-8 = 0.04."""
    want = want.detach()
    rms = want.square().mean().sqrt()
    err = got.double() - want
    row = err.square().mean(-1).sqrt() if want.dim() > 1 else err.abs() / 5
    assert bool((row <= limit * rms).all()), (name, float(row.max() / rms))
    assert bool((err.abs() <= 5 * limit * rms).all()), (name, float(err.abs().max() / rms))


def _formula_with_sides(block, P, x, s0, lengths, reset, above):
    """_formula with RELU's side of zero given: the slope there is a step, so an argument that a rounding carries over zero, one in a hundred
    of them, changes its gradient by all of it (two in a hundred of the squares: 0.1 to 0.2 of the root mean square)."""
    import torch
    nothing = {k: torch.zeros_like(P[k]) for k in ("down.weight", "down.bias")}
    m, S = _formula(block, {**P, **nothing}, x, s0, lengths, reset)
    p = _norm(m, P["norm2.weight"], P["norm2.bias"], block.eps) @ P["up.weight"].t() + P["up.bias"]
    return m + torch.where(above, p, 0.0) @ P["down.weight"].t() + P["down.bias"], S


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("case", CASES + [(130, 33, 96, 12, 200, "silu"), (32, 70, 128, 4, 512, "gelu")])
def test_bf16_row_by_row(case, ragged):
    """A defect in one token, one sequence or the last tile shows, where the whole tensor's mean hides it."""
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    T, N, W, h, hidden, act = case
    block = TimeBlock(W, h, hidden, dtype="bf16", act=act)
    host = _params(block, T + 1)
    g = torch.Generator(device="cuda").manual_seed(T * N)
    x, dy = (torch.randn(T, N, W, generator=g, device="cuda").to(block.dtype) for _ in range(2))
    s0, dsn = (torch.randn(N, h, W // h, W // h, generator=g, device="cuda") for _ in range(2))
    reset = (torch.rand(T, N, generator=g, device="cuda") < 0.05).to(torch.uint8)
    lengths = torch.randint(0, T + 1, (N,), generator=g, device="cuda", dtype=torch.int32) if ragged else None
    y, sn, dx, ds0 = torch.empty_like(x), torch.empty_like(s0), torch.empty_like(x), torch.empty_like(s0)
    block.forward(x, y, S0=s0, SN=sn, reset=reset, lengths=lengths)
    block.backward(dy, dX=dx, dSN=dsn, dS0=ds0)
    P = {n: torch.from_numpy(a).cuda().double().requires_grad_() for n, a in host.items()}
    X, S = x.double().requires_grad_(), s0.double().requires_grad_()
    if act == "relu":
        want, last = _formula_with_sides(block, P, X, S, lengths, reset, block._buffers[T, N, True]["pre"] > 0)
    else:
        want, last = _formula(block, P, X, S, lengths, reset)
    ((want * dy.double()).sum() + (last * dsn.double()).sum()).backward()
    _near_in_rows(y, want, 0.08, "y")
    _near_in_rows(dx, X.grad, 0.08, "dx")
    _near_in_rows(sn.flatten(2), last.flatten(2), 0.02, "sn")
    _near_in_rows(ds0.flatten(2), S.grad.flatten(2), 0.04, "ds0")
    for n in P:
        _near_in_rows(torch.from_numpy(block.get_param(n + ".grad")).cuda(), P[n].grad, 0.08, n)


def test_a_state_in_place_on_another_stream():
    """The copy of the first state is made, and used, on the call's stream."""
    import torch
    from paper_2309_03523_amd.time_block import TimeBlock
    T, N, W, h = 6, 400, 64, 4
    block = TimeBlock(W, h, 64)
    _params(block, 14)
    x, dy = torch.randn(T, N, W, device="cuda"), torch.randn(T, N, W, device="cuda")
    first = torch.randn(N, h, W // h, W // h, device="cuda")
    y, dx, s = torch.empty_like(x), torch.empty_like(x), torch.empty_like(first)
    block.forward(x, y, S0=first, SN=s)
    block.backward(dy, dX=dx)
    want = [t.clone() for t in (y, dx, s)]
    s.copy_(first)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    _busy(stream)
    block.forward(x, y, S0=s, SN=s, stream=stream)
    block.backward(dy, dX=dx, stream=stream)
    used = [torch.full_like(first, float("nan")) for _ in range(4)]
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((y, dx, s), want))
    del used
