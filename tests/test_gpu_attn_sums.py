"""How exactly the softmax attention's bias gradient is summed over millions of pairs whose parts nearly cancel.

Its terms dS and their sums are held in fp32, whatever the tensors' type.  fp32 roundings have no side that they prefer, so errors of n terms grow with the root of n;
the same formula in fp32 torch operations, which round as often, says how large that is on the same inputs.  A kernel whose terms or sums are all off to one side
is off by n times as much, which at these numbers of pairs is 4 to 15 times what the roundings come to.  Each side's error is the norm over heads x buckets (24 and more numbers)
of independent errors: a factor of 3 between two such norms leaves room for their scatter and for the kernel's own order of sums."""
import pytest

from test_gpu_attn import _backward, _case, _forward, _parts, _split

pytestmark = pytest.mark.gpu


def _bias_gradient(c, o, lse, dtype):
    """By the formula, in `dtype`, some sequences at a time."""
    import torch
    Tq, Tk, N, heads, kv, d = c["dims"]
    kw = c["kw"]
    sees, *_, away = _parts(c)
    r = kw["bias_map"].shape[0] // 2
    which = kw["bias_map"].long()[away[0].clamp(-r, r) + r]       # every sequence's alike
    sums = torch.zeros(heads, Tq, Tk, dtype=dtype, device="cuda")
    for a in range(0, N, 100):
        b = slice(a, a + 100)
        split = lambda x, h: _split(x[:, b], h, False).to(dtype)  # noqa: E731
        Q, K, V, G, O = split(c["q"], heads), split(c["k"], kv), split(c["v"], kv), split(c["do"], heads), split(o, heads)
        K, V = (x.repeat_interleave(heads // kv, 1) for x in (K, V))
        S = kw["scale"] * (Q @ K.transpose(-1, -2).contiguous()) + kw["bias"].to(dtype)[:, which]
        P = torch.exp(S - lse[b].to(dtype)[..., None])
        dS = P * (G @ V.transpose(-1, -2).contiguous() - (G * O).sum(-1, keepdim=True))
        sums += torch.where(sees[b, None], dS, 0).sum(0)
    out = torch.zeros(heads, kw["bias"].shape[1], dtype=dtype, device="cuda")
    return out.index_add_(1, which.reshape(-1), sums.reshape(heads, -1))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,heads,kv,d,causal", [(200, 2000, 4, 4, 32, True), (200, 2000, 4, 2, 32, False), (150, 1500, 3, 3, 64, True), (96, 3000, 3, 1, 128, True),
                                                   (16, 40000, 4, 4, 16, True), (30, 10000, 4, 2, 32, True)])
def test_the_bias_gradient_of_many_pairs(T, N, heads, kv, d, causal, dtype):
    c = _case(T, T, N, heads, d, dtype, T + d, kv=kv, causal=causal, buckets=8, reach=12)
    o, lse = _forward(c)
    import torch
    got = _backward(c, o, lse)[3].double()
    want = _bias_gradient(c, o, lse, torch.float64)
    plain = _bias_gradient(c, o, lse, torch.float32).double()
    err, by = float((got - want).norm()), float((plain - want).norm())
    assert err <= 3 * by, f"off by {err / float(want.norm())} of the norm, where fp32 operations are by {by / float(want.norm())}"
