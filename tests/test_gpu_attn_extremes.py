"""Softmax attention where tokens hold numbers at the ends of their type's range: what a query does not see, and rows that are no
tokens, reach nothing, whatever the products with them come to; scores of any size that fp32 holds have weights.

Where outputs are compared bit for bit, only what must not count differs between the two calls.  Other tolerances are those of the formulas in test_gpu_attn."""
import pytest

from test_gpu_attn import HALF, _backward, _case, _forward, _join, _near, _reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", ["one product", "lowest", "highest"])
@pytest.mark.parametrize("T", [12, 16, 30, 32, 60, 100])
def test_products_with_later_keys_that_overflow(T, what, dtype):
    """A finite key whose products with earlier queries are infinite, or infinities of both signs: those queries keep their bits."""
    import torch
    J = T - 1 - T // 4
    c = _case(T, T, 3, 4, 16, dtype, T, kv=2 if T % 3 else 4, buckets=4, reach=8)
    low = torch.finfo(c["k"].dtype).min
    q, k = c["q"].clone(), c["k"].clone()
    if what == "one product":      # of one query and one key, in a column where no other key has anything
        q[J // 2, 1, 3] = 2.0 ** 70
        k[..., 3] = 0.0
    x = dict(c, q=q, k=k)
    clean = _forward(x)
    x["k"] = k.clone()
    if what == "one product":
        x["k"][J, 1, 3] = 2.0 ** 70
    else:
        x["k"][J, 1] = low if what == "lowest" else -low
    o, lse = _forward(x)
    assert torch.equal(o[:, 0], clean[0][:, 0]) and torch.equal(o[:, 2], clean[0][:, 2])
    assert torch.isfinite(clean[0][:J]).all() and torch.equal(o[:J], clean[0][:J]) and torch.equal(lse[..., :J], clean[1][..., :J])
    want, got = (_backward(dict(y, kw=c["kw"]), *clean) for y in (dict(c, q=q, k=k), x))      # of the same o and lse
    assert torch.isfinite(want[0][:J]).all() and torch.equal(got[0][:J], want[0][:J])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [16, 30, 60, 100, 150, 200])
def test_a_key_of_weight_zero_that_is_not_finite(T, dtype, causal):
    """Scores of -inf with a key that is -inf where all queries are positive: the queries' gradients and the bias' are those without that key.  Rows
    that only fill a tile up have no part in it."""
    import torch
    J = 5
    c = _case(T, T, 3, 2, 16, dtype, T, buckets=4, reach=4, causal=causal)
    c["q"] = c["q"].clone()
    c["q"][..., 3] = c["q"][..., 3].abs() + 0.125
    c["q"][..., 16 + 3] = c["q"][..., 16 + 3].abs() + 0.125
    x = dict(c, k=c["k"].clone())
    x["k"][J, :, 3] = x["k"][J, :, 16 + 3] = -float("inf")
    keep = torch.ones(T, 3, dtype=torch.uint8, device="cuda")
    keep[J] = 0
    without = dict(c, kw=dict(c["kw"], keep=keep))
    o, lse = _forward(x)
    (O, to), (L, tl), _ = _reference(without)
    _near(o, _join(O), _join(to), "o")
    _near(lse, L, tl, "lse")
    dq, _, _, db = _backward(x, o, lse)
    wants = _reference(without, o, lse)
    other = [e for e in range(32) if e % 16 != 3]
    _near(dq[..., other], _join(wants[0][0])[..., other], _join(wants[0][1])[..., other], "dq")      # in column 3 a zero meets the infinity
    _near(db, *wants[3], "dbias")


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [16, 30, 60, 100, 150, 200])
def test_gradients_of_a_key_of_weight_zero_that_is_not_finite(T, dtype, causal):
    """The same: its own are zero, the other keys' those without it."""
    import torch
    J = 5
    c = _case(T, T, 3, 2, 16, dtype, T, buckets=4, reach=4, causal=causal)
    c["q"] = c["q"].clone()
    c["q"][..., 3] = c["q"][..., 3].abs() + 0.125
    c["q"][..., 16 + 3] = c["q"][..., 16 + 3].abs() + 0.125
    x = dict(c, k=c["k"].clone())
    x["k"][J, :, 3] = x["k"][J, :, 16 + 3] = -float("inf")
    keep = torch.ones(T, 3, dtype=torch.uint8, device="cuda")
    keep[J] = 0
    without = dict(c, kw=dict(c["kw"], keep=keep))
    o, lse = _forward(x)
    _, dk, dv, _ = _backward(x, o, lse)
    wants = _reference(without, o, lse)
    for got, (want, tol), name in ((dk, wants[1], "dk"), (dv, wants[2], "dv")):
        _near(got, _join(want), _join(tol), name)
    assert bool((dk[J] == 0).all()) and bool((dv[J] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("Tq,Tk", [(20, 30), (40, 60), (70, 100), (5, 100), (1, 90), (130, 200), (600, 700)])
def test_keys_behind_every_query(Tq, Tk, value, dtype):
    """A cache's rows that are not filled yet, with nothing but positions to mask them: no query sees them, their gradients are zero."""
    import torch
    c = _case(Tq, Tk, 2, 4, 16, dtype, Tk, kv=2, buckets=4, reach=8)
    first = (Tk - Tq) // 2
    c["kw"]["first"] = torch.tensor([first, 0], dtype=torch.int32, device="cuda")
    seen = torch.stack([torch.arange(Tk, device="cuda") < f + Tq for f in (first, 0)], 1)[..., None]
    got = []
    for fill in (0.0, value):
        x = dict(c, k=torch.where(seen, c["k"], fill).to(c["k"].dtype), v=torch.where(seen, c["v"], fill).to(c["v"].dtype))
        o, lse = _forward(x)
        got.append((o, lse, *_backward(x, o, lse)))
    for name, a, b in zip(("o", "lse", "dq", "dk", "dv", "dbias"), *got):
        assert torch.isfinite(a).all() and torch.equal(a, b), name
    for g in got[1][3:5]:
        assert bool((torch.where(seen, 0, g) == 0).all())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e6, 1e10, 1e17])
@pytest.mark.parametrize("Tq,Tk", [(16, 16), (30, 30), (60, 60), (1, 300), (8, 300), (150, 150), (300, 300)])
def test_scores_far_beyond_what_a_weight_can_tell(Tq, Tk, size, dtype, causal):
    """Scores of up to `size`, whole multiples of a step beside which biases are nothing, no two alike: the largest takes all.  Two columns hold a score's
    digits, so products and their sums are exact.  o: the weight's rounding and o's own, each half a step of the type, and fp32's.  lse: the
    largest score rounded once, and the logarithm of its weight, whose exponent is off by three roundings of the score."""
    import math
    import torch
    c = _case(Tq, Tk, 2, 2, 32, dtype, 5, causal=causal, buckets=4, reach=4)
    c["kw"]["scale"] = 1.0
    g = torch.Generator(device="cuda").manual_seed(3)
    step = 2.0 ** round(math.log2(size / Tk))
    k, q = torch.zeros_like(c["k"]), torch.zeros_like(c["q"])
    for n in range(2):
        for h in range(2):
            rank = torch.randperm(Tk, generator=g, device="cuda")
            k[:, n, h * 32 + 7], k[:, n, h * 32 + 20] = (rank // 128 * 128 * step).to(k.dtype), (rank % 128 * step).to(k.dtype)
            sign = torch.where(torch.rand(Tq, generator=g, device="cuda") < 0.5, 1.0, -1.0).to(q.dtype)
            q[:, n, h * 32 + 7] = q[:, n, h * 32 + 20] = sign
    c.update(q=q, k=k)
    o, lse = _forward(c)
    (O, _), (L, _), _ = _reference(c)
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    assert float((o.double() - _join(O)).abs().max()) <= (2.02 * HALF[dtype] + 2.0 ** -20) * float(c["v"].double().abs().max())
    assert bool(((lse.double() - L).abs() <= 2.0 ** -22 * L.abs() + 2.0 ** -20).all())
    for x in _backward(c, o, lse):
        assert torch.isfinite(x).all()
