"""The operators of the time block, as cases that can be timed and checked: row-wise layer norm, products
with bias, activation and residual, and linear attention with a decay per head, each forward and backward.

`run` computes them in elementary torch operations in 32 bits, or, where `own` is set, through the public
binding of this repository.  `exact` computes them in 64 bits from their definitions.
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-5


# ------------------------------------------------------------------------------------ the cases


def _norm(**kw):
    return dict(dict(op="norm", way="forward", dtype="bf16", R=1000, F=128, affine=True, add=False), **kw)


def _linear(**kw):
    return dict(dict(op="linear", way="forward", dtype="bf16", R=1000, K=128, M=128, act="none", bias=True, residual=False,
                     pre=False), **kw)


def _attn(**kw):
    return dict(dict(op="attn", way="forward", dtype="bf16", T=16, N=1000, heads=8, dk=16, dv=16, state=True, reset=0.0,
                     ragged=False, batch_first=False), **kw)


def listed():
    return [
        # A batch that leaves the card idle: a thousand rows of an odd width. Latency counts.
        _norm(name="norm_forward_small", dtype="f32", R=1000, F=172),
        # Embeddings of 32 snapshots of 100 000 vertices before a training step: output and statistics.
        _norm(name="norm_forward_rows", R=3200000, F=128),
        # Its gradients on wide fp32 rows, the gradient of the residual branch added on the way.
        _norm(name="norm_backward_wide", way="backward", dtype="f32", R=500000, F=256, add=True),
        # A handful of vertices served at once, wide weights: the weights' bytes and latency count.
        _linear(name="linear_forward_few_rows", R=8, K=1024, M=4096, act="silu", residual=True),
        # Node features of an odd width into the model's width, fp32.
        _linear(name="linear_forward_features", dtype="f32", R=100000, K=172, M=128, act="relu"),
        # The widening product of a feed-forward part over a training batch; the pre-activation is kept.
        _linear(name="linear_forward_expand", R=800000, K=128, M=512, act="gelu", pre=True),
        # The gradients of the same product.
        _linear(name="linear_backward_expand", way="backward", R=400000, K=128, M=512, act="gelu"),
        # Gradients of a square fp32 product over an odd number of rows.
        _linear(name="linear_backward_square", way="backward", dtype="f32", R=60001, K=256, M=256, act="relu"),
        # Windows of 16 snapshots of 100 000 vertices, 8 heads of 16, from zero states.
        _attn(name="attn_forward_windows", T=16, N=100000, state=False),
        # Gradients over ragged windows with resets (vertices that come and go), states chained.
        _attn(name="attn_backward_ragged", way="backward", T=32, N=20000, heads=4, dk=32, dv=32, reset=0.05, ragged=True),
        # A few long sequences, stored one after the other: work has to be split over the length.
        _attn(name="attn_forward_long", T=8192, N=4, heads=8, dk=64, dv=64, batch_first=True),
        # One new snapshot for 4000 vertices: every state is read and written once.
        _attn(name="attn_forward_step", dtype="f32", T=1, N=4000, heads=8, dk=64, dv=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "linear", "linear", "attn", "attn"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    way = rng.choice(["forward", "backward"])
    if op == "norm":
        F = _log_int(rng, 8, 8192)
        R = _log_int(rng, 1, min(3000000, 2e8 / F))
        return _norm(way=way, dtype=dtype, R=R, F=F, affine=rng.random() < 0.8, add=way == "backward" and rng.random() < 0.5)
    if op == "linear":
        K, M = _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)
        most = 4e10 if dtype == "bf16" else 1.5e10
        R = _log_int(rng, 1, max(1, min(800000, most / (K * M), 2e8 / (K + M))))
        act = rng.choice(["none", "relu", "gelu", "silu"])
        fwd = way == "forward"
        return _linear(way=way, dtype=dtype, R=R, K=K, M=M, act=act, bias=rng.random() < 0.8, residual=fwd and rng.random() < 0.5,
                       pre=fwd and act != "none" and rng.random() < 0.5)
    heads = rng.choice([1, 2, 3, 4, 8, 16])
    dk, dv = rng.choice([8, 16, 32, 64, 128]), rng.choice([8, 16, 24, 32, 40, 64, 128])
    if rng.random() < 0.5:
        dv = dk
    T = rng.choice([1, _log_int(rng, 2, 64), _log_int(rng, 2, 64), _log_int(rng, 65, 8192)])
    chunks = -(-T // 64)
    most = min(100000, 1e8 / (heads * T * min(T, 64)), 8e7 / (heads * chunks * dk * dv), 1.5e8 / (T * heads * (dk + dv)),
               1e7 / (heads * chunks * chunks))
    N = _log_int(rng, 1, max(1, most))
    return _attn(way=way, dtype=dtype, T=T, N=N, heads=heads, dk=dk, dv=dv, state=rng.random() < 0.6,
                 reset=rng.choice([0.0, 0.0, 0.05, 0.3]), ragged=rng.random() < 0.4, batch_first=rng.random() < 0.4)


# ------------------------------------------------------------------------------------ their inputs


def _pitch(n, dtype):
    per = 16 // SIZE[dtype]
    return -(-n // per) * per


def _tensor(g, shape, dtype, std=1.0, mean=0.0):
    """Rows at a pitch that is a multiple of 16 bytes, as every tensor of this library has them."""
    buf = torch.randn(*shape[:-1], _pitch(shape[-1], dtype), generator=g, device="cuda")
    return buf.mul_(std).add_(mean).to(DT[dtype])[..., :shape[-1]]


def _room(shape, dtype):
    return torch.zeros(*shape[:-1], _pitch(shape[-1], dtype), dtype=DT[dtype], device="cuda")[..., :shape[-1]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c, dt = case, case["dtype"]
    s = {"case": c}
    if c["op"] == "norm":
        R, F = c["R"], c["F"]
        s["x"] = _tensor(g, (R, F), dt, 1.5, 0.5)
        s["gamma"] = 1.0 + 0.2 * torch.randn(F, generator=g, device="cuda") if c["affine"] else None
        s["beta"] = 0.2 * torch.randn(F, generator=g, device="cuda") if c["affine"] else None
        if c["way"] == "forward":
            s["y"] = _room((R, F), dt)
            s["mean"], s["rstd"] = (torch.empty(R, device="cuda") for _ in range(2))
        else:
            x = s["x"].double()
            m = x.mean(1)
            s["mean"], s["rstd"] = m.float(), (x.sub_(m[:, None]).square_().mean(1) + EPS).rsqrt().float()
            s["dy"] = _tensor(g, (R, F), dt)
            s["add"] = _tensor(g, (R, F), dt) if c["add"] else None
            s["dx"] = _room((R, F), dt)
            s["dgamma"], s["dbeta"] = (torch.empty(F, device="cuda") for _ in range(2))
    elif c["op"] == "linear":
        R, K, M = c["R"], c["K"], c["M"]
        s["x"] = _tensor(g, (R, K), dt)
        s["w"] = _tensor(g, (M, K), dt, K ** -0.5)
        if c["way"] == "forward":
            s["bias"] = 0.3 * torch.randn(M, generator=g, device="cuda") if c["bias"] else None
            s["residual"] = _tensor(g, (R, M), dt) if c["residual"] else None
            s["y"] = _room((R, M), dt)
            s["pre"] = _room((R, M), dt) if c["pre"] else None
        else:
            s["dy"] = _tensor(g, (R, M), dt)
            s["pre"] = _tensor(g, (R, M), dt) if c["act"] != "none" else None
            s["dx"], s["dw"] = _room((R, K), dt), _room((M, K), dt)
            s["dbias"] = torch.empty(M, device="cuda") if c["bias"] else None
    else:
        T, N, h, dk, dv = (c[k] for k in ("T", "N", "heads", "dk", "dv"))

        def rows(d, made=None):
            shape = (N, T, d) if c["batch_first"] else (T, N, d)
            t = made(shape, dt) if made else _tensor(g, shape, dt)
            return t.transpose(0, 1) if c["batch_first"] else t

        s["q"], s["k"], s["v"] = rows(h * dk), rows(h * dk), rows(h * dv)
        s["scale"] = dk ** -0.5
        s["decay"] = 1.0 - 2.0 ** -(2.0 + 6.0 * torch.arange(h, device="cuda", dtype=torch.float32) / h)
        s["s0"] = torch.randn(N, h, dk, dv, generator=g, device="cuda") if c["state"] else None
        s["reset"] = (torch.rand(T, N, generator=g, device="cuda") < c["reset"]).to(torch.uint8) if c["reset"] else None
        s["lengths"] = torch.randint(0, T + 1, (N,), generator=g, device="cuda", dtype=torch.int32) if c["ragged"] else None
        if c["way"] == "forward":
            s["o"] = rows(h * dv, _room)
            s["sn"] = torch.empty(N, h, dk, dv, device="cuda") if c["state"] else None
        else:
            s["do"] = rows(h * dv)
            s["dsn"] = torch.randn(N, h, dk, dv, generator=g, device="cuda") if c["state"] else None
            s["dq"], s["dk"], s["dv"] = rows(h * dk, _room), rows(h * dk, _room), rows(h * dv, _room)
            s["ds0"] = torch.empty(N, h, dk, dv, device="cuda") if c["state"] else None
    return s


def work(case):
    c, e = case, SIZE[case["dtype"]]
    if c["op"] == "norm":
        n = c["R"] * c["F"]
        if c["way"] == "forward":
            return {"bytes": 2 * n * e + 8 * c["R"] + 8 * c["F"], "flops": 8 * n}
        return {"bytes": (4 if c["add"] else 3) * n * e + 8 * c["R"] + 12 * c["F"], "flops": 14 * n}
    if c["op"] == "linear":
        R, K, M = c["R"], c["K"], c["M"]
        if c["way"] == "forward":
            return {"bytes": e * (R * K + M * K + R * M * (1 + c["residual"] + c["pre"])), "flops": 2 * R * K * M}
        return {"bytes": e * (2 * R * K + 2 * M * K + R * M * (1 + (c["act"] != "none"))), "flops": 4 * R * K * M}
    T, N, h, dk, dv = (c[k] for k in ("T", "N", "heads", "dk", "dv"))
    share = 0.5 if c["ragged"] else 1.0
    # A token and head: the recurrence's two products, or the pairs of tokens of a short window where they are less.
    fl = min(4 * dk * dv, (T + 1) * (dk + dv) + (4 * dk * dv if c["state"] else 0))
    states = 4 * N * h * dk * dv
    if c["way"] == "forward":
        return {"bytes": share * e * T * N * h * 2 * (dk + dv) + (2 * states if c["state"] else 0), "flops": share * T * N * h * fl}
    return {"bytes": share * e * T * N * h * (4 * dk + 3 * dv) + (3 * states if c["state"] else 0),
            "flops": share * T * N * h * 3 * fl}


# ------------------------------------------------------------------------------------ plain forms


def _norm_forward(s):
    x = s["x"].float()
    m = x.mean(1, keepdim=True)
    xc = x - m
    r = torch.rsqrt((xc * xc).mean(1, keepdim=True) + EPS)
    y = xc * r
    if s["gamma"] is not None:
        y = y * s["gamma"] + s["beta"]
    return {"y": y.to(s["x"].dtype), "mean": m[:, 0], "rstd": r[:, 0]}


def _norm_backward(s):
    dy, r = s["dy"].float(), s["rstd"][:, None]
    xh = (s["x"].float() - s["mean"][:, None]) * r
    g = dy * s["gamma"] if s["gamma"] is not None else dy
    dx = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    if s["add"] is not None:
        dx = dx + s["add"].float()
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}


def _act(p, act):
    if act == "relu":
        return torch.where(p > 0, p, torch.zeros_like(p))
    if act == "gelu":
        return 0.5 * p * torch.erfc(p * -0.5 ** 0.5)
    return p / (1 + torch.exp(-p)) if act == "silu" else p


def _act_slope(p, act):
    if act == "relu":
        return (p > 0).to(p.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(p * -0.5 ** 0.5) + p * torch.exp(-0.5 * p * p) * (2 * math.pi) ** -0.5
    a = 1 / (1 + torch.exp(-p))
    return a * (1 + p * (1 - a))


def _linear_forward(s):
    p = s["x"].float() @ s["w"].float().t()
    if s["bias"] is not None:
        p = p + s["bias"]
    y = _act(p, s["case"]["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    dt = s["x"].dtype
    return {"y": y.to(dt), "pre": p.to(dt) if s["pre"] is not None else None}


def _linear_backward(s):
    dp = s["dy"].float()
    if s["pre"] is not None:
        dp = dp * _act_slope(s["pre"].float(), s["case"]["act"])
    dt = s["x"].dtype
    return {"dx": (dp @ s["w"].float()).to(dt), "dw": (dp.t() @ s["x"].float()).to(dt),
            "dbias": dp.sum(0) if s["dbias"] is not None else None}


def _powers(decay, n):
    """decay[h] ** n for a tensor of whole numbers, -> [..., h], in 64 bits; 0 where n is negative."""
    p = torch.exp2(n.clamp(min=0)[..., None].double() * torch.log2(decay.double()))
    return torch.where(n[..., None] >= 0, p, 0.0).float()


def _causal(a, b, c, decay, run):
    """sum over j <= i of one run of decay^(i-j) (a_i . b_j) c_j, for a, b [N,h,T,*], c [N,h,T,*], run [N,T]: in chunks of 64
    tokens, the earlier chunks through their sums of b^T c."""
    N, h, T, _ = a.shape
    C = min(64, T)
    n = -(-T // C)
    pad = n * C - T

    def chunks(x):
        return torch.nn.functional.pad(x, (0, 0, 0, pad)).reshape(N, h, n, C, x.shape[-1])

    a, b, c = chunks(a), chunks(b), chunks(c)
    run = torch.cat([run, run[:, -1:].expand(N, pad)], 1).reshape(N, 1, n, C)
    at = torch.arange(C, device=a.device)
    pair = _powers(decay, at[:, None] - at).permute(2, 0, 1)[None, :, None]
    seen = (run[..., :, None] == run[..., None, :])
    out = torch.matmul(torch.matmul(a, b.transpose(-1, -2)) * pair * seen, c)
    if n > 1:
        last = run[..., -1:]
        sums = torch.matmul((b * (_powers(decay, C - 1 - at).t()[None, :, None] * (run == last))[..., None]).transpose(-1, -2), c)
        ci = torch.arange(n, device=a.device)
        far = _powers(decay, C * (ci[:, None] - 1 - ci)).permute(2, 0, 1)[None]
        ends = last[..., 0]
        before = torch.cat([ends[..., :1] - 1, ends[..., :-1]], -1)
        far = far * (before[..., :, None] == ends[..., None, :])
        entering = torch.matmul(far, sums.flatten(-2)).reshape(sums.shape)
        out = out + torch.matmul(a, entering) * (_powers(decay, at + 1).t()[None, :, None] * (run == before[..., None]))[..., None]
    return out.reshape(N, h, n * C, -1)[:, :, :T]


def _attn_parts(s, bits):
    """q, k, v (and do) as [N,h,T,*], zero behind each sequence, the runs between resets and the lengths."""
    c = s["case"]
    T, N, h = c["T"], c["N"], c["heads"]
    dev = s["q"].device
    n = s["lengths"].long() if s["lengths"] is not None else torch.full((N,), T, device=dev)
    t = torch.arange(T, device=dev)
    live = t < n[:, None]
    run = s["reset"].t().long().cumsum(1) if s["reset"] is not None else torch.zeros(N, T, dtype=torch.long, device=dev)
    x = [torch.where(live[:, None, :, None], s[k].permute(1, 0, 2).reshape(N, T, h, -1).transpose(1, 2).to(bits), 0.0)
         for k in ("q", "k", "v", "do") if k in s]
    return x, n, t, live, run


def _back(x):
    """[N,h,T,d] -> [T,N,h*d]."""
    N, h, T, d = x.shape
    return x.permute(2, 0, 1, 3).reshape(T, N, h * d)


def _state_weights(s, n, t, live, run):
    """What each token's k^T v, and the state at the start, keeps of itself in the last state; and the first state in each token."""
    last = torch.where(n > 0, run.gather(1, (n - 1).clamp(min=0)[:, None])[:, 0], 0)
    keep = _powers(s["decay"], n[:, None] - 1 - t) * ((run == last[:, None]) & live)[..., None]
    start = _powers(s["decay"], n) * (last == 0)[:, None]
    first = _powers(s["decay"], t + 1)[None] * ((run == 0) & live)[..., None]
    return keep.transpose(1, 2)[..., None], start[..., None, None], first.transpose(1, 2)[..., None]


def _attn_forward(s):
    (q, k, v), n, t, live, run = _attn_parts(s, torch.float32)
    o = _causal(q, k, v, s["decay"], run)
    sn = None
    if s["s0"] is not None:
        keep, start, first = _state_weights(s, n, t, live, run)
        o = o + first * torch.matmul(q, s["s0"])
        sn = torch.matmul((k * keep).transpose(-1, -2), v) + start * s["s0"]
    return {"o": _back(o * s["scale"]).to(s["q"].dtype), "sn": sn}


def _attn_backward(s):
    (q, k, v, do), n, t, live, run = _attn_parts(s, torch.float32)
    do = do * s["scale"]
    dq = _causal(do, v, k, s["decay"], run)
    turned, runs = [x.flip(2) for x in (q, k, v, do)], run.flip(1)
    dk = _causal(turned[2], turned[3], turned[0], s["decay"], runs).flip(2)
    dv = _causal(turned[1], turned[0], turned[3], s["decay"], runs).flip(2)
    ds0 = None
    if s["s0"] is not None:
        keep, start, first = _state_weights(s, n, t, live, run)
        dq = dq + first * torch.matmul(do, s["s0"].transpose(-1, -2))
        dk = dk + keep * torch.matmul(v, s["dsn"].transpose(-1, -2))
        dv = dv + keep * torch.matmul(k, s["dsn"])
        ds0 = torch.matmul((q * first).transpose(-1, -2), do) + start * s["dsn"]
    dt = s["q"].dtype
    return {"dq": _back(dq).to(dt), "dk": _back(dk).to(dt), "dv": _back(dv).to(dt), "ds0": ds0}


PLAIN = {"norm": (_norm_forward, _norm_backward), "linear": (_linear_forward, _linear_backward),
         "attn": (_attn_forward, _attn_backward)}


def _workspace(s, size):
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(16, size()), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _run_own(s):
    from paper_2309_03523_amd import binding as b
    c = s["case"]
    if c["op"] == "norm":
        if c["way"] == "forward":
            b.norm_forward(s["x"], s["y"], gamma=s["gamma"], beta=s["beta"], mean=s["mean"], rstd=s["rstd"], eps=EPS)
            return {k: s[k] for k in ("y", "mean", "rstd")}
        b.norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["dx"], gamma=s["gamma"], add=s["add"], dgamma=s["dgamma"],
                        dbeta=s["dbeta"], workspace=_workspace(s, lambda: b.norm_workspace_bytes(c["R"], c["F"])))
        return {k: s[k] for k in ("dx", "dgamma", "dbeta")}
    if c["op"] == "linear":
        if c["way"] == "forward":
            b.linear_forward(s["x"], s["w"], s["y"], bias=s["bias"], act=c["act"], residual=s["residual"], pre=s["pre"])
            return {k: s[k] for k in ("y", "pre")}
        ws = _workspace(s, lambda: b.linear_workspace_bytes(c["R"], c["K"], c["M"], dtype=c["dtype"]))
        b.linear_backward(s["dy"], s["x"], s["w"], pre=s["pre"], act=c["act"], dx=s["dx"], dw=s["dw"], dbias=s["dbias"],
                          workspace=ws)
        return {k: s[k] for k in ("dx", "dw", "dbias")}
    ws = _workspace(s, lambda: b.decay_attn_workspace_bytes(c["T"], c["N"], c["heads"], c["dk"], c["dv"],
                                                            backward=c["way"] == "backward"))
    if c["way"] == "forward":
        b.decay_attn_forward(s["q"], s["k"], s["v"], s["decay"], s["o"], heads=c["heads"], scale=s["scale"], s0=s["s0"],
                             sn=s["sn"], lengths=s["lengths"], reset=s["reset"], workspace=ws)
        return {k: s[k] for k in ("o", "sn")}
    b.decay_attn_backward(s["q"], s["k"], s["v"], s["decay"], s["do"], s["dq"], s["dk"], s["dv"], heads=c["heads"],
                          scale=s["scale"], s0=s["s0"], dsn=s["dsn"], ds0=s["ds0"], lengths=s["lengths"], reset=s["reset"],
                          workspace=ws)
    return {k: s[k] for k in ("dq", "dk", "dv", "ds0")}


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    return PLAIN[c["op"]][c["way"] == "backward"](state)


# ------------------------------------------------------------------------------------ from the definitions, in 64 bits


def exact(case, seed):
    s, c = prepare(case, seed), case
    wide = lambda k: s[k].double() if s[k] is not None else None  # noqa: E731
    if c["op"] == "norm":
        x = wide("x")
        if c["way"] == "forward":
            var, m = torch.var_mean(x, 1, correction=0)
            r = 1 / torch.sqrt(var + EPS)
            y = (x - m[:, None]) * r[:, None]
            return {"y": y * wide("gamma") + wide("beta") if c["affine"] else y, "mean": m, "rstd": r}
        dy, r = wide("dy"), wide("rstd")[:, None]
        xh = (x - wide("mean")[:, None]) * r
        g = dy * wide("gamma") if c["affine"] else dy
        dx = r * (g - (g.sum(1, keepdim=True) + xh * (g * xh).sum(1, keepdim=True)) / c["F"])
        return {"dx": dx + wide("add") if c["add"] else dx, "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}
    if c["op"] == "linear":
        f = {"none": lambda p: p, "relu": torch.relu, "gelu": lambda p: p * torch.special.ndtr(p),
             "silu": lambda p: p * torch.sigmoid(p)}[c["act"]]
        x, w = wide("x"), wide("w")
        if c["way"] == "forward":
            p = torch.mm(x, w.t())
            p = p + wide("bias") if c["bias"] else p
            return {"y": f(p) + wide("residual") if c["residual"] else f(p), "pre": p if c["pre"] else None}
        dp = wide("dy")
        if c["act"] != "none":
            p = wide("pre").requires_grad_()
            dp, = torch.autograd.grad(f(p), p, dp)
        return {"dx": torch.mm(dp, w), "dw": torch.mm(dp.t().contiguous(), x), "dbias": dp.sum(0) if c["bias"] else None}
    # The recurrence, token by token; a sequence that has ended keeps its state.
    T, N, h, dk, dv = (c[k] for k in ("T", "N", "heads", "dk", "dv"))
    if T * (1 if c["way"] == "forward" else 2) > 20000 or T * N * h * dk * dv > 3e11:
        return None
    gone = s["reset"].bool() if s["reset"] is not None else torch.zeros(T, N, dtype=torch.bool, device="cuda")
    n = s["lengths"] if s["lengths"] is not None else torch.full((N,), T, device="cuda")
    link = (s["decay"].double()[None, None] * (~gone)[..., None])[..., None, None]
    live = (torch.arange(T, device="cuda")[:, None] < n)[..., None, None, None]
    ends = (torch.arange(T, device="cuda")[:, None] == n - 1)[..., None, None, None]
    heads = lambda k, d: s[k].reshape(T, N, h, d)  # noqa: E731
    Q, K, V = heads("q", dk), heads("k", dk), heads("v", dv)
    S = wide("s0") if c["state"] else torch.zeros(N, h, dk, dv, dtype=torch.float64, device="cuda")
    forward = c["way"] == "forward"
    out = torch.zeros(T, N, h, dv if forward else dk, dtype=torch.float64, device="cuda")
    D = None if forward else heads("do", dv)
    for t in range(T):
        S = torch.where(live[t], link[t] * S + K[t].double()[..., :, None] * V[t].double()[..., None, :], S)
        if forward:
            out[t] = torch.where(live[t][..., 0], s["scale"] * (Q[t].double()[..., :, None] * S).sum(-2), 0.0)
        else:
            out[t] = torch.where(live[t][..., 0], s["scale"] * (S * D[t].double()[..., None, :]).sum(-1), 0.0)
    if forward:
        return {"o": out.reshape(T, N, h * dv), "sn": S if c["state"] else None}
    G = torch.zeros_like(S)
    last = wide("dsn") if c["state"] else torch.zeros_like(S)
    outk, outv = torch.zeros_like(out), torch.zeros(T, N, h, dv, dtype=torch.float64, device="cuda")
    for t in range(T - 1, -1, -1):
        G = torch.where(ends[t], last, G)
        G = torch.where(live[t], G + s["scale"] * Q[t].double()[..., :, None] * D[t].double()[..., None, :], G)
        outk[t] = torch.where(live[t][..., 0], (G * V[t].double()[..., None, :]).sum(-1), 0.0)
        outv[t] = torch.where(live[t][..., 0], (K[t].double()[..., :, None] * G).sum(-2), 0.0)
        G = torch.where(live[t], link[t] * G, G)
    ds0 = torch.where((n == 0)[:, None, None, None], last, G) if c["state"] else None
    return {"dq": out.reshape(T, N, h * dk), "dk": outk.reshape(T, N, h * dk), "dv": outv.reshape(T, N, h * dv), "ds0": ds0}
