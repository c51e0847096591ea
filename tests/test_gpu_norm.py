"""Layer norm and its gradients on the device against the formulas in double precision: every kernel shape (row
widths around the steps of the lanes and vectors), both element types, pitches with NaN in the padding, rows in
place, the added residual gradient, and the calls a user may make of it (another stream, a replayed graph).

Tolerances count roundings.  An output of the element type is off by half a step of it, eps/2 relative, and by the fp32
arithmetic before it: with n = F terms in tree order a sum is off by at most (log2 F + 8) 2^-24 of the sum of magnitudes, which
for inputs of mean 0.5 and deviation 1.5 is under 24 * 2^-24 in each of mean and variance; the few further operations on
numbers up to |x - m| r |gamma| (below 8) make that 1e-5 absolute at most.  A column sum over R rows in fp32 registers of at most 512 terms,
then double: 512 * 2^-24 of the magnitudes in the worst case, 3e-5 of them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _dt(dtype):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]


def _rows(rng, R, F, dtype, mean=0.0, std=1.0, extra=0):
    """A [R, F] view at a wider pitch whose padding is NaN, and its values in double."""
    import torch
    per = 4 if dtype == "f32" else 8
    ld = -(-F // per) * per + extra * per
    buf = torch.full((R, ld), float("nan"), dtype=_dt(dtype), device="cuda")
    buf[:, :F] = torch.from_numpy(rng.normal(mean, std, (R, F))).cuda().to(_dt(dtype))
    return buf, buf[:, :F], buf[:, :F].double().cpu().numpy()


def _pad_is_nan(buf, F):
    import torch
    return bool(torch.isnan(buf[:, F:]).all())


def _forward(x, gamma, beta, eps):
    m = x.mean(1, keepdims=True)
    r = 1 / np.sqrt(((x - m) ** 2).mean(1, keepdims=True) + eps)
    return (x - m) * r * gamma + beta, m[:, 0], r[:, 0]


WIDTHS = [1, 3, 16, 17, 32, 33, 100, 128, 129, 172, 256, 257, 512, 513, 1000, 1025, 2048, 2049, 4096, 4097, 8192]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", WIDTHS)
def test_forward(F, dtype):
    import torch
    from paper_2309_03523_amd import binding
    rng = np.random.default_rng(F)
    R = 67 if F > 512 else 301
    _, x, X = _rows(rng, R, F, dtype, 0.5, 1.5, extra=F % 3)
    buf, y, _ = _rows(rng, R, F, dtype, extra=1)
    gamma, beta = rng.normal(1, 0.2, F).astype(np.float32), rng.normal(0, 0.2, F).astype(np.float32)
    mean, rstd = torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    eps = 1e-3
    binding.norm_forward(x, y, gamma=torch.from_numpy(gamma).cuda(), beta=torch.from_numpy(beta).cuda(), mean=mean, rstd=rstd, eps=eps)
    want, m, r = _forward(X, gamma.astype(np.float64), beta.astype(np.float64), eps)
    got = y.double().cpu().numpy()
    # rows that are nearly constant have a large rstd: an error of x - m counts that many times
    tol = HALF[dtype] * np.abs(want) + 1e-5 * np.maximum(1, r)[:, None]
    assert (np.abs(got - want) <= tol).all()
    assert np.abs(mean.cpu().numpy() - m).max() <= 24 * 2.0 ** -24 * np.abs(X).max()
    assert (np.abs(rstd.cpu().numpy() / r - 1) <= 1e-5 * np.maximum(1, r)).all()
    assert _pad_is_nan(buf, F)
    # without weights, in place
    binding.norm_forward(x, x, eps=eps)
    want, _, _ = _forward(X, 1.0, 0.0, eps)
    assert (np.abs(x.double().cpu().numpy() - want) <= HALF[dtype] * np.abs(want) + 1e-5 * np.maximum(1, r)[:, None]).all()


def _backward(dy, x, m, r, gamma, add):
    xh = (x - m[:, None]) * r[:, None]
    g = dy * gamma
    dx = r[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True)) + add
    return dx, (dy * xh).sum(0), dy.sum(0), np.abs(dy * xh).sum(0), np.abs(dy).sum(0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", WIDTHS)
def test_backward(F, dtype):
    import torch
    from paper_2309_03523_amd import binding
    rng = np.random.default_rng(1000 + F)
    R = 67 if F > 512 else 1301
    _, x, X = _rows(rng, R, F, dtype, 0.5, 1.5, extra=F % 3)
    _, dy, DY = _rows(rng, R, F, dtype)
    _, add, ADD = _rows(rng, R, F, dtype, extra=1)
    buf, dx, _ = _rows(rng, R, F, dtype, extra=2)
    gamma = rng.normal(1, 0.2, F).astype(np.float32)
    _, m, r = _forward(X, 1.0, 0.0, 1e-3)
    m, r = m.astype(np.float32), r.astype(np.float32)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    ws = torch.full((binding.norm_workspace_bytes(R, F) // 4,), float("nan"), device="cuda")
    dgamma, dbeta = torch.empty(F, device="cuda"), torch.empty(F, device="cuda")
    binding.norm_backward(dy, x, dev(m), dev(r), dx, gamma=dev(gamma), add=add, dgamma=dgamma, dbeta=dbeta, workspace=ws)
    want, dg, db, mag_g, mag_b = _backward(DY, X, m.astype(np.float64), r.astype(np.float64), gamma.astype(np.float64), ADD)
    scale = r.astype(np.float64)[:, None] * (np.abs(DY).max(1, keepdims=True) + 1) * np.maximum(1, np.abs((X - m[:, None]) * r[:, None]).max(1, keepdims=True))
    tol = HALF[dtype] * np.abs(want) + 24 * 2.0 ** -24 * 2 * scale
    assert (np.abs(dx.double().cpu().numpy() - want) <= tol).all()
    assert (np.abs(dgamma.cpu().numpy() - dg) <= 3e-5 * mag_g + 1e-30).all()
    assert (np.abs(dbeta.cpu().numpy() - db) <= 3e-5 * mag_b + 1e-30).all()
    assert _pad_is_nan(buf, F)
    # no weights, no residual gradient, one of the two sums, in place of dy
    g2 = torch.full((F,), -7.0, device="cuda")
    binding.norm_backward(dy, x, dev(m), dev(r), dy, dbeta=g2, workspace=ws)
    want, _, _, _, _ = _backward(DY, X, m.astype(np.float64), r.astype(np.float64), 1.0, 0.0)
    assert (np.abs(dy.double().cpu().numpy() - want) <= HALF[dtype] * np.abs(want) + 24 * 2.0 ** -24 * 2 * scale).all()
    assert torch.equal(g2, dbeta)


def test_gradient_against_differences():
    """The gradient in fp32 against central differences of the forward formula in double."""
    import torch
    from paper_2309_03523_amd import binding
    rng = np.random.default_rng(5)
    R, F, eps = 3, 20, 1e-5
    x, dy = rng.normal(0, 1, (R, F)).astype(np.float32), rng.normal(0, 1, (R, F)).astype(np.float32)
    gamma, beta = rng.normal(1, 0.3, F), rng.normal(0, 0.3, F)
    xd, out, dx = torch.from_numpy(x).cuda(), torch.empty(R, F, device="cuda"), torch.empty(R, F, device="cuda")
    mean, rstd = torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    g = torch.from_numpy(gamma.astype(np.float32)).cuda()
    binding.norm_forward(xd, out, gamma=g, mean=mean, rstd=rstd, eps=eps)
    binding.norm_backward(torch.from_numpy(dy).cuda(), xd, mean, rstd, dx, gamma=g)
    h = 1e-5
    for _ in range(20):
        d = rng.normal(0, 1, (R, F))
        x64, g64 = x.astype(np.float64), gamma.astype(np.float32).astype(np.float64)
        slope = ((_forward(x64 + h * d, g64, beta, eps)[0] - _forward(x64 - h * d, g64, beta, eps)[0]) * dy).sum() / (2 * h)
        got = (dx.double().cpu().numpy() * d).sum()
        assert abs(got - slope) <= 1e-5 * np.abs(dx.double().cpu().numpy() * d).sum()


def test_no_rows_and_one_row():
    import torch
    from paper_2309_03523_amd import binding
    for R in (0, 1):
        x = torch.randn(R, 40, device="cuda")
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
        dg, db = torch.full((40,), 5.0, device="cuda"), torch.full((40,), 5.0, device="cuda")
        binding.norm_forward(x, y, mean=mean, rstd=rstd)
        ws = torch.empty(binding.norm_workspace_bytes(R, 40), dtype=torch.uint8, device="cuda")
        binding.norm_backward(x, x, mean, rstd, dx, dgamma=dg, dbeta=db, workspace=ws)
        want = x.sum(0) if R else torch.zeros(40, device="cuda")     # of no rows: zeros
        assert torch.equal(db, want)


def test_values_that_are_not_finite_stay_in_their_row():
    import torch
    from paper_2309_03523_amd import binding
    x = torch.randn(64, 96, device="cuda")
    clean = torch.empty_like(x)
    binding.norm_forward(x, clean)
    x[5, 3], x[17, 0] = float("nan"), float("inf")
    y = torch.empty_like(x)
    binding.norm_forward(x, y)
    bad = torch.zeros(64, dtype=torch.bool, device="cuda")
    bad[5] = bad[17] = True
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], clean[~bad])


def test_streams_graphs_and_repeats():
    """A call on another stream, and one captured and replayed with eager work between, give the eager call's bits."""
    import torch
    from paper_2309_03523_amd import binding
    R, F = 20011, 136
    x, dy = torch.randn(R, F, device="cuda"), torch.randn(R, F, device="cuda")
    ws = torch.empty(binding.norm_workspace_bytes(R, F), dtype=torch.uint8, device="cuda")

    def step(out, stream=None):
        binding.norm_forward(x, out[0], mean=out[1], rstd=out[2], stream=stream)
        binding.norm_backward(dy, x, out[1], out[2], out[3], dgamma=out[4], dbeta=out[5], workspace=ws, stream=stream)

    def room():
        return [torch.empty(*s, device="cuda") for s in ((R, F), (R,), (R,), (R, F), (F,), (F,))]

    want, other, graph_out = room(), room(), room()
    step(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    step(other, s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(graph_out)
    for k in range(3):
        x.mul_(1.5)
        step(want)
        torch.cuda.synchronize()
        for t in graph_out:
            t.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, graph_out)), k
