"""Softmax attention and AdamW at the ends of the ranges that the header gives: heads, sequences, distances, sizes; and with what may be left out."""
import pytest

from test_gpu_attn import _both, _case, _check_forward, _forward, _ws

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv", [(1024, 1024), (1024, 1), (999, 3)])
@pytest.mark.parametrize("Tq,Tk", [(5, 5), (20, 30), (40, 40), (70, 70), (1, 300), (3, 300)])
def test_the_most_heads(Tq, Tk, heads, kv, dtype):
    _both(_case(Tq, Tk, 2, heads, 8, dtype, Tk, kv=kv, buckets=4, reach=6))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Tq,Tk", [(16, 16), (30, 30), (50, 50), (150, 150), (1, 300), (9, 300)])
def test_one_bucket_and_no_reach(Tq, Tk, causal, dtype):
    """A map of one entry: one number for all distances."""
    import torch
    c = _case(Tq, Tk, 3, 2, 32, dtype, Tk, causal=causal)
    c["kw"].update(bias=torch.tensor([[0.5], [-2.0]], device="cuda"), bias_map=torch.zeros(1, dtype=torch.uint8, device="cuda"))
    _both(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Tq,Tk", [(16, 16), (30, 30), (50, 50), (150, 150), (1, 3000), (9, 3000)])
def test_statistics_may_be_left_out(Tq, Tk, dtype):
    import torch
    from paper_2309_03523_amd import binding
    c = _case(Tq, Tk, 3, 2, 32, dtype, Tk, buckets=4, reach=6)
    o, lse = _forward(c)
    _check_forward(c, o, lse)
    again = torch.empty_like(o)
    binding.attn_forward(c["q"], c["k"], c["v"], again, workspace=_ws(c, False), **c["kw"])
    assert torch.equal(o, again)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nearly_as_many_sequences_as_a_launch_takes(dtype):
    """Of one token each: it attends to itself, so o is v, dv the output's gradient, and nothing else has one."""
    import torch
    from paper_2309_03523_amd import binding
    N, dt = 8388600, {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator(device="cuda").manual_seed(0)
    q, k, v, do = (torch.randn(1, N, 8, generator=g, device="cuda").to(dt) for _ in range(4))
    o, dq, dk, dv = (torch.full_like(v, 7) for _ in range(4))
    lse = torch.empty(N, 1, 1, device="cuda")
    binding.attn_forward(q, k, v, o, heads=1, lse=lse)
    assert torch.equal(o, v)
    s = (q.double() * k.double()).sum(-1)[0]
    assert float((lse[:, 0, 0].double() - s).abs().max()) <= 24 * 2.0 ** -23 * float((q.double() * k.double()).abs().sum(-1).max())
    ws = torch.empty(binding.attn_workspace_bytes(1, 1, N, 1, 8, dtype=dtype, backward=True), dtype=torch.uint8, device="cuda")
    binding.attn_backward(q, k, v, o, lse, do, dq, dk, dv, heads=1, workspace=ws)
    # P is e^(s - lse) with both of one value; dP and D are the same sum in two orders, 8 terms and the roundings of them
    near = 16 * 2.0 ** -23 * (do.double() * v.double()).abs().sum(-1, keepdim=True)
    assert bool((dq.double().abs() <= near * k.double().abs() * 1.01 + 1e-30).all()) and bool((dk.double().abs() <= near * q.double().abs() * 1.01 + 1e-30).all())
    assert float((dv.double() - do.double()).abs().max()) <= (2.0 ** -20 + (0 if dtype == "f32" else 2.0 ** -8)) * float(do.double().abs().max())


@pytest.mark.parametrize("F", [41, 48])
def test_adamw_of_more_than_32_bits_of_places(F):
    """One tensor of 2^32 places and some: its last rows are stepped as a tensor of those rows alone is."""
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 30 GiB")
    R, tail = 2 ** 32 // 48 + 1000, 2048
    R += -R % 16      # the last rows begin at a scale's first place: 16 rows of 48 are 3 blocks of 256
    p, g = (torch.zeros(R, 48, dtype=torch.bfloat16, device="cuda")[:, :F] for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(1)
    for x in (p, g):
        for rows in (slice(0, tail), slice(R - tail, R)):
            x[rows] = torch.randn(tail, F, generator=gen, device="cuda").to(x.dtype)
    big = AdamW([p], [g], bits=8, lr=0.1)
    small = []
    for rows in (slice(0, tail), slice(R - tail, R)):
        q, h = (torch.zeros(tail, 48, dtype=torch.bfloat16, device="cuda")[:, :F] for _ in range(2))
        q.copy_(p[rows]), h.copy_(g[rows])
        small.append((rows, AdamW([q], [h], bits=8, lr=0.1)))
    for _ in range(2):
        big.step()
        for _, opt in small:
            opt.step()
    for rows, opt in small:
        assert torch.equal(p[rows], opt.params[0]) and bool((p[rows] != 0).any())
        for n in ("m", "v"):
            assert torch.equal(big.states[0][n][rows].view(torch.uint8), opt.states[0][n].view(torch.uint8))
            blocks = slice(rows.start * 48 // 256, rows.stop * 48 // 256)
            assert torch.equal(big.states[0][n + "_scale"][blocks], opt.states[0][n + "_scale"])
    assert not p[tail:tail + 1000].any() and not p[R // 2:R // 2 + 1000].any()
