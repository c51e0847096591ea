"""Softmax attention at numbers of sequences where workgroups take one after the other, and at lengths where a key's gradients are summed in parts: against the
formulas in double, with the tolerances of test_gpu_attn.  A launch holds at most 2048 workgroups of windows (backward 1024, with shared heads 4096 waves of all key
heads), 512 to 1024 that sum the bias' gradient of longer sequences, and parts of 256 queries at least."""
import pytest

from test_gpu_attn import FILL, _backward, _both, _case, _check_backward, _check_forward, _forward, _join, _near, _parts, _reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv,d", [(8, 8, 16), (2, 2, 16), (3, 3, 24), (4, 2, 32), (2, 1, 64)])
@pytest.mark.parametrize("Tq,Tk", [(5, 5), (12, 16), (30, 30)])
def test_windows_of_many_sequences(Tq, Tk, heads, kv, d, dtype):
    c = _case(Tq, Tk, 5003, heads, d, dtype, Tk + d, kv=kv, buckets=6, reach=10, absent=0.2, ragged=True)
    o, lse = _forward(c)
    _check_forward(c, o, lse)
    _check_backward(c, o, lse, _backward(c, o, lse))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [9, 31, 50])
def test_windows_of_many_sequences_at_positions_of_their_own(T, dtype):
    _both(_case(T, T, 4999, 4, 16, dtype, T, kv=2, buckets=6, reach=10, ragged=True, first=True, causal=T != 31))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv", [(4, 4), (4, 2)])
@pytest.mark.parametrize("T", [11, 28])
def test_what_masked_rows_hold_reaches_no_later_sequence(T, heads, kv, dtype):
    """NaN and infinities in absent keys and behind sequences: the same bits as with zeros there."""
    import torch
    c = _case(T, T, 4999, heads, 16, dtype, T, kv=kv, absent=0.4, ragged=True, buckets=8, reach=16)
    sees, row, key, there, _ = _parts(c)
    some = sees.any(-1) & row
    got = []
    for fill in (0.0, float("nan"), -float("inf")):
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
@pytest.mark.parametrize("T,N,heads,kv,d", [(16, 3001, 8, 8, 16), (28, 3001, 4, 4, 16), (28, 4801, 4, 2, 16), (130, 61, 16, 16, 16), (130, 61, 16, 4, 64)])
def test_one_key_that_is_not_finite_among_many_sequences(T, N, heads, kv, d, dtype):
    """Other sequences keep their bits, and so do heads that do not read that key; earlier queries of its own sequence have the formula's gradients."""
    import torch
    c = _case(T, T, N, heads, d, dtype, T, kv=kv, buckets=4, reach=8, absent=0.1)
    c["kw"]["keep"][0] = 1      # every query sees something
    J, n, g = T // 2, N - 2, heads // kv
    c["kw"]["keep"][J, n] = 1
    o, lse = _forward(c)
    clean = (o, lse, *_backward(c, o, lse))
    for name in ("k", "v"):
        x = dict(c, **{name: c[name].clone()})
        x[name][J, n, 3] = float("inf")      # key head 0
        o, lse = _forward(x)
        got = (o, lse, *_backward(x, o, lse))
        others = torch.arange(N, device="cuda") != n
        for a, b in zip(got[:1] + got[2:5], clean[:1] + clean[2:5]):
            mine = d * (g if a.shape[2] == heads * d else 1)
            assert torch.equal(a[:, others], b[:, others]) and torch.equal(a[:, n, mine:], b[:, n, mine:])
        assert torch.equal(got[1][others], clean[1][others]) and torch.equal(got[1][n, g:], clean[1][n, g:]) and torch.equal(got[5][g:], clean[5][g:])
        assert torch.isfinite(got[0][:J]).all() and torch.isfinite(got[2][:J]).all()
        (O, to), (L, tl), _ = _reference(c)
        _near(got[0][:J], _join(O)[:J], _join(to)[:J], "o")
        want, tol = _reference(c, clean[0], clean[1])[0]
        if name == "v":      # lse of later queries does not count here, of earlier ones it is the same
            _near(got[1][n], L[n], tl[n], "lse")
        _near(got[2][:J], _join(want)[:J], 2 * _join(tol)[:J], "dq")      # for an o and lse in another order of sums: once more their size


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,heads,kv,d,causal", [(130, 60, 16, 16, 16, True), (200, 50, 12, 4, 32, False), (70, 300, 8, 8, 64, True), (100, 90, 6, 1, 128, True)])
def test_the_bias_gradient_over_several_rounds(T, N, heads, kv, d, causal, dtype):
    _both(_case(T, T, N, heads, d, dtype, T, kv=kv, causal=causal, buckets=8, reach=20, absent=0.1, ragged=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["all", "ragged", "both sides"])
def test_gradients_of_keys_in_parts(how, dtype):
    kw = {"all": {}, "ragged": dict(ragged=True, absent=0.2), "both sides": dict(causal=False)}[how]
    _both(_case(1100, 1100, 1, 4, 16, dtype, 7, kv=1, buckets=8, reach=100, **kw))
    _both(_case(600, 700, 2, 6, 40, dtype, 8, kv=2, buckets=8, reach=30, **kw))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["q", "do"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_gradients_of_keys_in_parts_with_a_query_that_is_not_finite(value, name, dtype):
    """Keys behind it have the formula's gradients, whichever part they are summed in; earlier ones, which it sees, are not finite in its column or row."""
    import torch
    T, J = 1100, 700
    c = _case(T, T, 1, 4, 16, dtype, 7, kv=1, buckets=8, reach=100)
    clean_o, clean_lse = _forward(c)
    x = dict(c, **{name: c[name].clone()})
    x[name][J, 0, 3] = value      # head 0
    o, lse = _forward(x)
    assert torch.equal(o[:J], clean_o[:J]) and torch.equal(o[J + 1:], clean_o[J + 1:])
    dq, dk, dv, _ = _backward(x, o, lse)
    wants = _reference(c, clean_o, clean_lse)
    for got, (want, tol) in ((dk, wants[1]), (dv, wants[2])):
        assert not torch.isfinite(got[:J + 1]).all()
        _near(got[J + 1:], _join(want)[J + 1:], _join(tol)[J + 1:], "keys behind it")
    rest = torch.arange(T, device="cuda") != J
    _near(dq[rest], _join(wants[0][0])[rest], _join(wants[0][1])[rest], "dq")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Tq,Tk,N,heads,kv,d", [(1, 5000, 3, 4, 4, 16), (1, 3000, 2, 4, 2, 64), (2, 2100, 2, 2, 2, 32), (7, 3000, 2, 8, 2, 32), (16, 2600, 1, 4, 1, 128), (1, 700, 300, 8, 8, 16)])
def test_a_few_queries_against_split_keys(Tq, Tk, N, heads, kv, d, dtype):
    c = _case(Tq, Tk, N, heads, d, dtype, Tk, kv=kv, buckets=8, reach=40, absent=0.1)
    _check_forward(c, *_forward(c))
    c = _case(Tq, Tk, N, heads, d, dtype, Tk, kv=kv, buckets=8, reach=40, ragged=True, first=True)
    o, lse = _forward(c)
    _check_forward(c, o, lse)
    assert o.shape[0] == Tq and bool((o[~_parts(c)[1].t()] == FILL).all())
