"""Softmax attention with a learned bias by buckets, forward and backward, against its formulas in double.

Tolerances count roundings against magnitudes.  A result of the element type is off by half a step of it.  Before that, fp32: a score is off by
(d + 16) 2^-23 of the sum of its terms' sizes (the matrix unit cuts its sums off) and 2^-22 of itself and the statistic that is taken from it, which is
the relative error of its weight; sums of n weights by n 2^-23.  Weights, and products, below fp32's smallest normal number
may count as zero: TINY each.  bf16 rounds weights, and the gradients of scores, to half a step once before
they are summed."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
FILL = -7.0
TINY = 2.0 ** -126


def _dt(dtype):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]


def _case(Tq, Tk, N, heads, d, dtype, seed, *, kv=None, causal=True, buckets=0, reach=0, absent=0.0, ragged=False, first=False, batch_first=False, fused=False):
    import torch
    from paper_2309_03523_amd import binding
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, kv = _dt(dtype), kv or heads

    def rows(T, F, fill=None):
        shape = (N, T, F + 16) if batch_first else (T, N, F + 16)      # wider rows: strides that are not the width
        t = torch.randn(*shape, generator=g, device="cuda") if fill is None else torch.full(shape, fill, device="cuda")
        t = t.to(dt)[..., 8:8 + F]
        return t.transpose(0, 1) if batch_first else t

    c = dict(q=rows(Tq, heads * d), k=rows(Tk, kv * d), v=rows(Tk, kv * d), do=rows(Tq, heads * d))
    if fused:       # one buffer, as a fused product leaves it
        c["q"], c["k"], c["v"] = torch.randn(Tk, N, (heads + 2 * kv) * d, generator=g, device="cuda").to(dt).split([heads * d, kv * d, kv * d], -1)
    kw = dict(heads=heads, kv_heads=kv, scale=d ** -0.5, causal=causal)
    if buckets:
        kw["bias"] = torch.randn(heads, buckets, generator=g, device="cuda")
        kw["bias_map"] = torch.from_numpy(binding.attn_buckets(buckets, reach, causal=causal)).cuda()
    if absent:
        kw["keep"] = ((torch.rand(Tk, N, generator=g, device="cuda") >= absent) * 3).to(torch.uint8)
    if ragged:
        kw["lengths"] = torch.randint(-1, Tk + 2, (N,), generator=g, device="cuda", dtype=torch.int32)
    if first:
        kw["first"] = torch.randint(-2, Tk + 2, (N,), generator=g, device="cuda", dtype=torch.int32)
    c.update(kw=kw, rows=rows, dims=(Tq, Tk, N, heads, kv, d), dtype=dtype)
    return c


def _ws(c, backward, fill=255):
    import torch
    from paper_2309_03523_amd import binding
    Tq, Tk, N, heads, kv, d = c["dims"]
    b, m = c["kw"].get("bias"), c["kw"].get("bias_map")
    n = binding.attn_workspace_bytes(Tq, Tk, N, heads, d, kv_heads=kv, dtype=c["dtype"], causal=c["kw"]["causal"], buckets=b.shape[1] if b is not None else 0,
                                     reach=m.shape[0] // 2 if m is not None else 0, backward=backward)
    assert n >= 0
    return torch.full((n,), fill, dtype=torch.uint8, device="cuda") if n else None


def _forward(c, **more):
    import torch
    from paper_2309_03523_amd import binding
    Tq, Tk, N, heads, kv, d = c["dims"]
    o, lse = c["rows"](Tq, heads * d, FILL), torch.full((N, heads, Tq), FILL, device="cuda")
    binding.attn_forward(c["q"], c["k"], c["v"], o, lse=lse, workspace=_ws(c, False), **{**c["kw"], **more})
    return o, lse


def _backward(c, o, lse, **more):
    import torch
    from paper_2309_03523_amd import binding
    Tq, Tk, N, heads, kv, d = c["dims"]
    dq, dk, dv = c["rows"](Tq, heads * d, FILL), c["rows"](Tk, kv * d, FILL), c["rows"](Tk, kv * d, FILL)
    b = c["kw"].get("bias")
    db = torch.full_like(b, FILL) if b is not None else None
    binding.attn_backward(c["q"], c["k"], c["v"], o, lse, c["do"], dq, dk, dv, dbias=db, workspace=_ws(c, True), **{**c["kw"], **more})
    return dq, dk, dv, db


def _split(x, heads, wide=True):
    T, N, F = x.shape
    return (x.double() if wide else x).reshape(T, N, heads, F // heads).permute(1, 2, 0, 3).contiguous()


def _join(x):
    N, h, T, d = x.shape
    return x.permute(2, 0, 1, 3).reshape(T, N, h * d)


def _parts(c):
    """Which (n, i, j) are seen, which queries and keys are tokens, and the distances."""
    import torch
    Tq, Tk, N, *_ = c["dims"]
    kw = c["kw"]
    i, j = torch.arange(Tq, device="cuda"), torch.arange(Tk, device="cuda")
    at = (kw["first"].long() if "first" in kw else torch.full((N,), Tk - Tq, device="cuda"))[:, None] + i
    n = kw["lengths"].long().clamp(0, Tk) if "lengths" in kw else torch.full((N,), Tk, device="cuda")
    row, key = (at >= 0) & (at < n[:, None]), j < n[:, None]
    there = key & (kw["keep"].t() != 0) if "keep" in kw else key
    away = at[:, :, None] - j
    sees = row[:, :, None] & there[:, None, :]
    return sees & (away >= 0) if kw["causal"] else sees, row, key, there, away


def _reference(c, o=None, lse=None):
    """(value, magnitude) of each output; with o and lse those of the gradients for them."""
    import torch
    Tq, Tk, N, heads, kv, d = c["dims"]
    kw, g, dtype = c["kw"], heads // kv, c["dtype"]
    sees, row, key, there, away = _parts(c)
    bits = lambda x, ok: torch.where(ok.t()[:, :, None], x, 0)  # noqa: E731
    Q, K, V = _split(bits(c["q"], row), heads), _split(bits(c["k"], there), kv).repeat_interleave(g, 1), _split(bits(c["v"], there), kv).repeat_interleave(g, 1)
    s = kw["scale"]
    S, A = s * (Q @ K.transpose(-1, -2)), abs(s) * (Q.abs() @ K.abs().transpose(-1, -2))
    if "bias" in kw:
        r = kw["bias_map"].shape[0] // 2
        which = kw["bias_map"].long()[away.clamp(-r, r) + r].clamp(max=kw["bias"].shape[1] - 1)
        B = kw["bias"].double()[:, which].transpose(0, 1)
        S, A = S + B, A + B.abs()
    m = sees[:, None]
    S = torch.where(m, S, -torch.inf)
    pr = HALF[dtype] if dtype == "bf16" else 0.0
    if o is None:
        L = torch.logsumexp(S, -1)
        P = torch.exp(S - torch.where(L == -torch.inf, 0.0, L)[..., None])
        e = torch.where(m, (d + 16) * 2.0 ** -23 * A + 2.0 ** -22 * (S.abs() + 2), 0.0).amax(-1)       # of a weight
        O, mag = P @ V, P @ V.abs()
        tol = HALF[dtype] * O.abs() + (2 * e + (Tk + 8) * 2.0 ** -23 + pr)[..., None] * mag + TINY * (V.abs().sum(-2, keepdim=True) + Tk)
        return (O, tol), (L, e + (Tk + 8) * 2.0 ** -23 + 2.0 ** -22 * torch.where(L == -torch.inf, 0.0, L).abs()), row
    ok = (lse.double() > -torch.inf) & row[:, None]
    l = torch.where(ok, lse.double(), 0.0)[..., None]
    P = torch.where(m & ok[..., None], torch.exp(S - l), 0.0)
    live = lambda x: torch.where(ok[..., None], _split(x, heads), 0.0)  # noqa: E731
    G, O = live(c["do"]), live(o)
    Q = torch.where(ok[..., None], Q, 0.0)
    dP, aP = G @ V.transpose(-1, -2), G.abs() @ V.abs().transpose(-1, -2)
    D, aD = (G * O).sum(-1, keepdim=True), (G * O).abs().sum(-1, keepdim=True)
    dS = P * (dP - D)
    e = torch.where(m, (d + 16) * 2.0 ** -23 * A + 2.0 ** -22 * (torch.where(m, S, 0.0).abs() + l.abs() + 2), 0.0)
    eS = (P * (e + (d + 16) * 2.0 ** -23) + TINY) * (aP + aD + 1) + pr * dS.abs()
    fold = lambda x: x.reshape(N, kv, g, Tk, d).sum(2)  # noqa: E731
    n = (max(Tq * g, Tk) + 8) * 2.0 ** -23
    t = lambda x: x.transpose(-1, -2)  # noqa: E731
    half = HALF[dtype]
    dq, dk, dv = s * (dS @ K), fold(s * (t(dS) @ Q)), fold(t(P) @ G)
    s = abs(s)
    tq = half * dq.abs() + s * ((eS + n * dS.abs()) @ (K.abs() + TINY)) + Tk * TINY
    tk = half * dk.abs() + fold(s * (t(eS + n * dS.abs()) @ (Q.abs() + TINY)) + Tq * TINY)
    tv = half * dv.abs() + fold(t(P * (e + n + pr) + TINY) @ (G.abs() + 1) + Tq * TINY)
    db = tb = None
    if "bias" in kw:
        nb = kw["bias"].shape[1]
        hot = torch.nn.functional.one_hot(which, nb).double() * m[:, 0][..., None]
        sums = lambda x: torch.einsum("nhij,nijb->hb", x, hot)  # noqa: E731
        db = sums(dS)
        # A table takes at most every pair of its distance, one after the other: not more than the pairs of one query in one bucket times queries.
        tb = sums(eS - pr * dS.abs()) + (N * max(Tq, Tk) + 64) * 2.0 ** -24 * sums(dS.abs()) + half * 0 + 2.0 ** -24 * db.abs()
    return (dq, tq), (dk, tk), (dv, tv), (db, tb), (row, key)


def _near(got, want, tol, what):
    import torch
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf].to(got.dtype)), what
    off = (got.double() - want)[~inf].abs() - tol[~inf]
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 0, f"{what}: over by {worst}, at most {float(tol.max())} allowed"


def _check_forward(c, o, lse):
    import torch
    (O, to), (L, tl), row = _reference(c)
    rows = row.t()[:, :, None].expand_as(o)
    assert bool((o[~rows] == FILL).all()) and bool((lse[~row[:, None].expand_as(lse)] == FILL).all())
    _near(torch.where(rows, o, 0), torch.where(rows, _join(O), 0), _join(to), "o")
    r = row[:, None].expand_as(lse)
    _near(torch.where(r, lse, 0), torch.where(r, L, 0), tl, "lse")


def _check_backward(c, o, lse, got):
    import torch
    wants = _reference(c, o, lse)
    row, key = wants[4]
    for x, ok, (want, tol), what in zip(got, (row, key, key), wants, ("dq", "dk", "dv")):
        rows = ok.t()[:, :, None].expand_as(x)
        assert bool((x[~rows] == FILL).all()), what
        _near(torch.where(rows, x, 0), torch.where(rows, _join(want), 0), _join(tol), what)
    if got[3] is not None:
        _near(got[3], *wants[3], "dbias")


def _both(c):
    o, lse = _forward(c)
    _check_forward(c, o, lse)
    _check_backward(c, o, lse, _backward(c, o, lse))


LENGTHS = [(1, 1, 5), (2, 3, 3), (15, 16, 3), (17, 17, 3), (32, 32, 2), (20, 33, 2), (64, 64, 2), (1, 64, 3), (1, 65, 3), (3, 130, 2), (16, 300, 2), (17, 66, 2),
           (65, 65, 2), (100, 129, 2), (257, 257, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Tq,Tk,N", LENGTHS)
def test_lengths(Tq, Tk, N, dtype):
    _both(_case(Tq, Tk, N, 2, 16, dtype, Tq + Tk, buckets=8, reach=9, causal=Tk % 3 != 0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [8, 16, 24, 32, 40, 64, 72, 96, 128])
@pytest.mark.parametrize("T", [7, 29, 70])
def test_widths(d, T, dtype):
    _both(_case(T, T, 2, 3, d, dtype, d + T, buckets=6 if d != 24 else 0, reach=20 if d != 24 else 0))
    one = _case(1, T + 70, 2, 3, d, dtype, d)
    _check_forward(one, *_forward(one))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv", [(4, 4), (4, 2), (3, 1), (8, 1), (6, 2), (16, 1)])
@pytest.mark.parametrize("Tq,Tk", [(12, 12), (1, 90), (5, 100), (80, 80)])
def test_shared_heads(heads, kv, Tq, Tk, dtype):
    _both(_case(Tq, Tk, 3, heads, 16, dtype, heads + Tk, kv=kv, buckets=8, reach=32, ragged=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Tq,Tk", [(9, 9), (30, 30), (50, 60), (1, 200), (7, 140), (150, 150), (90, 200)])
@pytest.mark.parametrize("how", ["absent", "most absent", "ragged", "first", "all", "batch first"])
def test_masks(how, Tq, Tk, causal, dtype):
    kw = {"absent": dict(absent=0.3), "most absent": dict(absent=0.97), "ragged": dict(ragged=True), "first": dict(first=True),
          "all": dict(absent=0.4, ragged=True, first=True, buckets=10, reach=50, kv=1), "batch first": dict(batch_first=True, ragged=True, buckets=4, reach=2)}[how]
    _both(_case(Tq, Tk, 6, 2, 24, dtype, Tk, causal=causal, **kw))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("T,reach", [(30, 5), (30, 1024), (300, 4), (300, 100), (300, 1024), (400, 64)])
def test_bias_beyond_and_within_reach(T, reach, causal, dtype):
    _both(_case(T, T, 2, 2, 32, dtype, T + reach, causal=causal, buckets=8 if reach > 4 else 4, reach=reach))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_the_most_shared_memory(d, dtype):
    _both(_case(200, 200, 2, 2, d, dtype, d, causal=False, buckets=256, reach=1024))


def test_any_map_and_numbers_beyond_the_buckets():
    import torch
    for T in (20, 100):
        c = _case(T, T, 3, 2, 16, "f32", 3, causal=False, buckets=6, reach=12)
        c["kw"]["bias_map"] = torch.randint(0, 9, (25,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.uint8)
        _both(c)


def test_one_buffer_for_queries_keys_and_values():
    import torch
    from paper_2309_03523_amd import binding
    for T in (20, 90):
        c = _case(T, T, 4, 4, 16, "bf16", 8, kv=2, fused=True, buckets=8, reach=8)
        o, lse = _forward(c)
        _check_forward(c, o, lse)
        room = torch.full((T, 4, 128), FILL, dtype=torch.bfloat16, device="cuda")
        dq, dk, dv = room.split([64, 32, 32], -1)
        db = torch.empty_like(c["kw"]["bias"])
        binding.attn_backward(c["q"], c["k"], c["v"], o, lse, c["do"], dq, dk, dv, dbias=db, workspace=_ws(c, True), **c["kw"])
        _check_backward(c, o, lse, (dq, dk, dv, db))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [12, 24, 100])
def test_repeated_rows_as_inputs(T, dtype):
    """Strides of 0: one query for all sequences, one sequence's keys for all."""
    c = _case(T, T, 3, 2, 16, dtype, 4, buckets=4, reach=4)
    c["q"] = c["q"][:, :1].expand(T, 3, 32)
    c["k"] = c["k"][:1].expand(T, 3, 32)
    c["do"] = c["do"][:, :1].expand(T, 3, 32)
    _both(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,Tq", [(14, 14), (30, 30), (60, 60), (100, 100), (90, 1), (90, 6)])
def test_what_masked_rows_hold_reaches_nothing(T, Tq, dtype):
    """NaN and infinities in absent keys, behind sequences and in queries that are no tokens: the same bits as with zeros there."""
    import torch
    c = _case(Tq, T, 5, 2, 16, dtype, T, absent=0.4, ragged=True, buckets=8, reach=16, causal=T != 60)
    if Tq == 1:
        c["kw"]["first"] = c["kw"]["lengths"].clamp(0, T) - 1
    sees, row, key, there, _ = _parts(c)
    some = sees.any(-1) & row
    got = []
    for fill in (0.0, float("nan"), float("inf")):
        x = dict(c)
        for n, ok in (("q", some), ("k", there), ("v", there), ("do", some)):
            x[n] = torch.where(ok.t()[:, :, None], c[n], fill).to(c[n].dtype)
        o, lse = _forward(x)
        got.append((o, lse, *_backward(x, o, lse)))
    assert all(torch.isfinite(t[t != -torch.inf]).all() for t in got[0])
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("T", [14, 30, 60, 100, 200])
def test_a_token_that_is_not_finite_reaches_what_sees_it(T, value, dtype):
    import torch
    J = T // 2
    c = _case(T, T, 2, 2, 16, dtype, T, buckets=4, reach=8)
    clean_o, clean_lse = _forward(c)
    clean = _backward(c, clean_o, clean_lse)
    x = dict(c, v=c["v"].clone())
    x["v"][J, 0, 3] = value      # head 0's column 3
    o, lse = _forward(x)
    # lse does not depend on v, but the order of its sum may: it is held to its formula.  What is of another sequence or head keeps its bits.
    _near(lse, *_reference(c)[1], "lse")
    assert torch.equal(o[:, 1], clean_o[:, 1]) and torch.equal(o[:, 0, 16:], clean_o[:, 0, 16:])
    assert not torch.isfinite(o[J:, 0, 3]).any() and torch.isfinite(o[:J]).all()
    _check_forward(dict(c, v=torch.where(torch.isfinite(x["v"]), x["v"], 0)), torch.where((torch.arange(T, device="cuda") >= J)[:, None, None] & (torch.arange(32, device="cuda") == 3), _zeroed(c, J)[0], o), lse)
    # A key: scores of the queries from J on; gradients of earlier queries stay as they were.
    x = dict(c, k=c["k"].clone())
    x["k"][J, 0, 3] = value
    o, lse = _forward(x)
    assert torch.isfinite(o[:J]).all() and torch.isfinite(o[:, 1]).all() and torch.isfinite(o[:, 0, 16:]).all()
    dq, dk, dv, _ = _backward(x, o, lse)
    assert torch.isfinite(dq[:J]).all() and torch.isfinite(dq[:, 1]).all() and torch.isfinite(dq[:, 0, 16:]).all()
    _rows_near(dq[:J], clean[0][:J], c, clean_o, clean_lse, 0, slice(0, J))
    # A query or its output's gradient: keys behind it stay as they were.
    for name in ("q", "do"):
        x = dict(c, **{name: c[name].clone()})
        x[name][J, 0, 3] = value
        o, lse = _forward(x)
        _, dk, dv, _ = _backward(x, o, lse)
        for g, w, k in ((dk, clean[1], 1), (dv, clean[2], 2)):
            assert torch.isfinite(g[J + 1:]).all() and torch.isfinite(g[:, 1]).all() and torch.isfinite(g[:, 0, 16:]).all()
            _rows_near(g[J + 1:], w[J + 1:], c, clean_o, clean_lse, k, slice(J + 1, T))


def _zeroed(c, J):
    import torch
    v = c["v"].clone()
    v[J, 0, 3] = 0
    return _forward(dict(c, v=v))


def _rows_near(got, clean, c, o, lse, which, rows):
    """Both within the tolerance of the formula: the slow way sums in another order."""
    want, tol = _reference(c, o, lse)[which]
    _near(got, _join(want)[rows], _join(tol)[rows], "rows that do not see it")
    _near(clean, _join(want)[rows], _join(tol)[rows], "clean rows")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,Tq", [(12, 12), (30, 30), (100, 100), (100, 1)])
def test_biases_that_mask(T, Tq, dtype):
    """-inf and the type's lowest value as biases: what has others to see does not see those; rows of -inf alone are empty, rows of the lowest value alone even."""
    import torch
    for low in (-float("inf"), torch.finfo(torch.float32).min):
        c = _case(Tq, T, 2, 2, 16, dtype, T, buckets=4, reach=3, causal=True)
        c["kw"]["bias_map"] = torch.tensor([0, 0, 0, 0, 1, 2, 3], dtype=torch.uint8, device="cuda")
        c["kw"]["bias"][0, 1:] = low         # head 0 sees itself alone
        c["kw"]["bias"][1, :] = low
        o, lse = _forward(c)
        own = c["v"][T - Tq:, :, :16]
        assert torch.equal(o[..., :16], own)
        if low == -float("inf"):
            assert bool((o[..., 16:] == 0).all()) and bool((lse[:, 1] == low).all())
        else:
            sees = torch.arange(T - Tq, T, device="cuda")
            mean = c["v"][..., 16:].double().cumsum(0)[sees] / (sees + 1)[:, None, None]
            assert bool(((o[..., 16:].double() - mean).abs() <= (HALF[dtype] * 2 + T * 2.0 ** -23) * c["v"].double().abs().amax()).all())
            assert bool((lse[:, 1] == low).all())
        got = _backward(c, o, lse)
        assert all(torch.isfinite(x).all() for x in got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Tq,Tk", [(20, 20), (40, 50), (1, 300), (130, 130)])
def test_large_scores(Tq, Tk, dtype):
    """Scores of some hundreds: weights of 1 and 0, no overflow."""
    c = _case(Tq, Tk, 2, 2, 32, dtype, 5, buckets=4, reach=4)
    c["kw"]["scale"] = 8.0
    _both(c)
    c["kw"]["scale"] = -0.3
    _both(c)
    c["kw"]["scale"] = 0.0
    _both(c)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("T,kv", [(10, 4), (31, 2), (75, 2), (40, 1)])
def test_gradients_against_autograd_in_double(T, kv, causal):
    import torch
    c = _case(T, T, 3, 4, 16, "f32", T, kv=kv, causal=causal, buckets=6, reach=11, absent=0.2)
    o, lse = _forward(c)
    got = _backward(c, o, lse)
    leaves = [c[n].double().clone().requires_grad_() for n in ("q", "k", "v")] + [c["kw"]["bias"].double().clone().requires_grad_()]
    sees, *_, away = _parts(c)
    Q, K, V = _split(leaves[0], 4), _split(leaves[1], kv).repeat_interleave(4 // kv, 1), _split(leaves[2], kv).repeat_interleave(4 // kv, 1)
    S = 0.25 * (Q @ K.transpose(-1, -2)) + leaves[3][:, c["kw"]["bias_map"].long()[away.clamp(-11, 11) + 11]].transpose(0, 1)
    some = sees.any(-1)[:, None, :, None]
    P = torch.where(some, torch.softmax(torch.where(sees[:, None], S, -1e30), -1) * sees[:, None], 0.0)
    loss = (_join(P @ V) * c["do"].double()).sum()
    for g, leaf, (_, tol) in zip(got, leaves, _reference(c, o, lse)[:4]):
        want = torch.autograd.grad(loss, leaf, retain_graph=True)[0]
        tol = _join(tol) if tol.dim() == 4 else tol
        # o's own rounding enters D: once more the size of the tolerance
        _near(g, want, 2 * tol, "gradient")


def test_gradients_against_differences():
    import torch
    c = _case(9, 9, 2, 2, 8, "f32", 1, buckets=4, reach=5)
    o, lse = _forward(c)
    got = _backward(c, o, lse)
    loss = lambda x: float((_reference(x)[0][0] * _split(c["do"], 2)).sum())  # noqa: E731
    h = 2.0 ** -10
    rng = np.random.RandomState(0)
    for g, name in zip(got, ("q", "k", "v", "bias")):
        base = c["kw"]["bias"] if name == "bias" else c[name]
        for _ in range(6):
            at = tuple(int(rng.randint(s)) for s in base.shape)
            side = []
            for sign in (1, -1):
                t = base.double().clone()
                t[at] += sign * h
                x = dict(c, kw=dict(c["kw"]))
                if name == "bias":
                    x["kw"]["bias"] = t
                else:
                    x[name] = t
                side.append(loss(x))
            # central differences: h^2 / 6 of the third derivative, a few times the largest input cubed
            assert abs((side[0] - side[1]) / (2 * h) - float(g[at])) < 1e-4


@pytest.mark.parametrize("Tq,Tk", [(16, 16), (32, 32), (1, 2000), (200, 200)])
def test_the_same_bits_twice_and_on_other_streams(Tq, Tk):
    import torch
    c = _case(Tq, Tk, 40, 4, 32, "bf16", 2, buckets=16, reach=40, absent=0.1, ragged=Tq > 1)
    o, lse = _forward(c)
    first = (o, lse, *_backward(c, o, lse))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o, lse = _forward(c)
        other = (o, lse, *_backward(c, o, lse))
    s.synchronize()
    for a, b in zip(first, other):
        assert torch.equal(a, b)


@pytest.mark.parametrize("Tq,Tk", [(16, 16), (1, 2000), (100, 100)])
def test_replayed_graphs(Tq, Tk):
    """Two captured graphs with a workspace each, replayed in turn with eager work between; new inputs in place."""
    import torch
    from paper_2309_03523_amd import binding
    cs = [_case(Tq, Tk, 8, 4, 32, "bf16", s, buckets=8, reach=16) for s in (1, 2)]
    graphs = []
    for c in cs:
        heads, d = 4, 32
        out = [torch.zeros(Tq, 8, heads * d, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, heads, Tq, device="cuda")]
        out += [torch.zeros_like(c[n]) for n in ("q", "k", "v")] + [torch.zeros_like(c["kw"]["bias"])]
        ws = (_ws(c, False), _ws(c, True))

        def call(c=c, out=out, ws=ws):
            binding.attn_forward(c["q"], c["k"], c["v"], out[0], lse=out[1], workspace=ws[0], **c["kw"])
            binding.attn_backward(c["q"], c["k"], c["v"], out[0], out[1], c["do"], out[2], out[3], out[4], dbias=out[5], workspace=ws[1], **c["kw"])

        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append((g, out))
    for turn in range(3):
        for c, (g, out) in zip(cs, graphs):
            g.replay()
        for c, (g, out) in zip(cs, graphs):
            o, lse = _forward(c)
            for a, b in zip(out, (o, lse, *_backward(c, o, lse))):
                assert torch.equal(a, b), turn
            for n in ("q", "k", "v", "do"):
                c[n].mul_(0.5).add_(0.1)
        torch.cuda.synchronize()


@pytest.mark.parametrize("Tq,Tk", [(20, 20), (100, 100)])
def test_single_gradients(Tq, Tk):
    """Each gradient asked for alone is the one that comes with all."""
    import torch
    from paper_2309_03523_amd import binding
    c = _case(Tq, Tk, 3, 2, 16, "f32", 6, buckets=4, reach=9)
    o, lse = _forward(c)
    every = _backward(c, o, lse)
    for k in range(4):
        out = [torch.full_like(x, FILL) if x.dim() == 2 else c["rows"](x.shape[0], 32, FILL) for x in every]
        args = [out[x] if x == k else None for x in range(4)]
        binding.attn_backward(c["q"], c["k"], c["v"], o, lse, c["do"], *args[:3], dbias=args[3], workspace=_ws(c, True), **c["kw"])
        assert torch.equal(out[k], every[k])


def test_nothing_to_do():
    import torch
    for Tq, Tk, N in ((0, 0, 3), (0, 5, 3), (0, 50, 3), (4, 4, 0)):
        c = _case(Tq, Tk, N, 2, 16, "f32", 0, buckets=4, reach=4)
        o, lse = _forward(c)
        dq, dk, dv, db = _backward(c, o, lse)
        assert bool((db == 0).all()) and bool((dk == 0).all()) and bool((dv == 0).all())
    c = _case(6, 6, 4, 2, 16, "f32", 0)
    c["kw"]["lengths"] = torch.zeros(4, dtype=torch.int32, device="cuda")
    o, lse = _forward(c)
    assert all(bool((x == FILL).all()) for x in (o, lse, *_backward(c, o, lse)[:3]))


def test_positions_far_away():
    """first at the ends of its range: every query is no token."""
    import torch
    for Tq, Tk in ((5, 20), (5, 100), (20, 100)):
        for at in (-2 ** 31, 2 ** 31 - 1):
            c = _case(Tq, Tk, 2, 2, 16, "f32", 0, buckets=4, reach=4)
            c["kw"]["first"] = torch.full((2,), at, dtype=torch.int32, device="cuda")
            o, lse = _forward(c)
            dq, dk, dv, db = _backward(c, o, lse)
            assert bool((o == FILL).all()) and bool((lse == FILL).all()) and bool((dq == FILL).all()) and all(bool((x == 0).all()) for x in (dk, dv, db))


def test_steps_against_a_growing_cache_are_the_forward_pass():
    """Snapshot by snapshot against the keys kept so far, sequences of different ages: the rows of one pass over all."""
    import torch
    from paper_2309_03523_amd import binding
    T, N, heads, d = 70, 5, 4, 16
    c = _case(T, T, N, heads, d, "bf16", 9, kv=2, buckets=8, reach=30)
    whole, lse = _forward(c)
    (O, to), (L, tl), _ = _reference(c)
    ws = torch.empty(max(16, binding.attn_workspace_bytes(1, T, N, heads, d, kv_heads=2, dtype="bf16", buckets=8, reach=30)), dtype=torch.uint8, device="cuda")
    for t in (0, 1, 15, 16, 33, 63, 64, 69):
        ages = torch.tensor([t, max(t - 1, 0), t // 2, 0, t], dtype=torch.int32, device="cuda")
        q = torch.stack([c["q"][a, n] for n, a in enumerate(ages.tolist())])[None]
        o, l = torch.empty_like(q), torch.empty(N, heads, 1, device="cuda")
        binding.attn_forward(q, c["k"], c["v"], o, lse=l, first=ages, lengths=ages + 1, workspace=ws, **c["kw"])
        at, n = ages.long(), torch.arange(N, device="cuda")
        _near(o[0], _join(O)[at, n], _join(to)[at, n], f"step {t}")
        _near(l[..., 0], L[n, :, at], tl[n, :, at], f"lse of step {t}")


def test_offsets_beyond_32_bits():
    """A cache of rows 2^33 bytes apart, as a view of a larger one has them."""
    import torch
    from paper_2309_03523_amd import binding
    free, _ = torch.cuda.mem_get_info()
    T, heads, d = 66, 2, 16
    if free < 40 << 30:
        pytest.skip("needs 17 GiB")
    step = 2 ** 27 // 2
    room = torch.empty(T * step * 2 + 64, dtype=torch.bfloat16, device="cuda")      # rows 2^27 bytes apart: the last at 2^33 bytes and more
    k, v = (torch.as_strided(room, (T, 1, heads * d), (step * 2, heads * d, 1), at) for at in (0, 32))
    g = torch.Generator(device="cuda").manual_seed(1)
    for t in (k, v):
        t.copy_(torch.randn(T, 1, heads * d, generator=g, device="cuda"))
    q = torch.randn(T, 1, heads * d, generator=g, device="cuda").to(torch.bfloat16)
    for rows in (T, 1):
        got, want = (torch.empty(rows, 1, heads * d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        binding.attn_forward(q[T - rows:], k, v, got, heads=heads)
        binding.attn_forward(q[T - rows:], k.contiguous(), v.contiguous(), want, heads=heads)
        assert torch.equal(got, want)


def test_forms_of_one_call_agree():
    """A window padded with keys behind its sequences goes another way through the library: the same values."""
    import torch
    from paper_2309_03523_amd import binding
    T, N, heads, d = 30, 4, 2, 32
    c = _case(T, T, N, heads, d, "f32", 11, buckets=8, reach=16)
    o, lse = _forward(c)
    got = _backward(c, o, lse)
    pad = lambda x: torch.cat([x, torch.full((60, N, heads * d), float("nan"), device="cuda")])  # noqa: E731
    kw = dict(c["kw"], first=torch.zeros(N, dtype=torch.int32, device="cuda"), lengths=torch.full((N,), T, dtype=torch.int32, device="cuda"))
    x = dict(c, q=pad(c["q"]), k=pad(c["k"]), v=pad(c["v"]), do=pad(c["do"]), kw=kw, dims=(90, 90, N, heads, heads, d))
    ox, lx = _forward(x)
    other = _backward(x, ox, lx)
    (O, to), (L, tl), _ = _reference(c)
    _near(ox[:T], _join(O), _join(to), "o")
    for k, (a, b) in enumerate(zip(got, other)):
        want, tol = _reference(c, o, lse)[k]
        _near(b[:T] if k < 3 else b, _join(want) if k < 3 else want, 2 * (_join(tol) if k < 3 else tol), "gradient")
        assert k == 3 or bool((b[T:] == FILL).all())
