"""Softmax attention over snapshots with a learned bias by buckets of distance, its gradients, and AdamW steps over many
tensors, as cases that can be timed and checked.

`run` computes them in elementary torch operations in 32 bits, or, where `own` is set, through the public
modules of this repository.  `exact` computes them in 64 bits from their definitions.
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
BLOCK = 256                       # numbers that share a scale in an 8-bit state
LR, BETAS, EPS, DECAY = 1e-3, (0.9, 0.999), 1e-8, 0.01


# ------------------------------------------------------------------------------------ the cases


def _attn(**kw):
    c = dict(dict(op="attn", way="forward", dtype="bf16", T=16, N=1000, heads=8, d=16, causal=True, buckets=0, reach=0, absent=0.0,
                  ragged=False, batch_first=False), **kw)
    c.setdefault("rows", c["T"])       # queries: the last `rows` tokens of a sequence
    c.setdefault("kv_heads", c["heads"])
    return c


def _adamw(**kw):
    return dict(dict(op="adamw", dtype="f32", bits=32, blocks=1, width=128, hidden=512), **kw)


def listed():
    return [
        # A dozen snapshots of a hundred vertices in fp32: a batch that leaves the card idle. Latency counts.
        _attn(name="attn_forward_small", dtype="f32", T=12, N=100, heads=4, d=32, buckets=8, reach=8),
        # Windows of 16 snapshots of 100 000 vertices, 8 heads of 16.
        _attn(name="attn_forward_windows", N=100000, buckets=16, reach=16),
        # A few long histories, stored one after the other, through a block's forward pass.
        _attn(name="attn_forward_long", T=8192, N=4, heads=8, d=64, buckets=32, reach=128, batch_first=True),
        # Histories of an odd length looked at from both sides, fp32.
        _attn(name="attn_forward_both_sides", dtype="f32", T=1001, N=16, heads=8, d=64, causal=False, buckets=32, reach=128),
        # A new snapshot for 2000 vertices that have seen up to 512: their keys and values are read once.
        _attn(name="attn_forward_step", rows=1, T=512, N=2000, heads=8, d=64, buckets=32, reach=128, ragged=True),
        # The same for two vertices with long histories, four heads to a key: too few sequences to fill the card.
        _attn(name="attn_forward_step_long", rows=1, T=65536, N=2, heads=16, kv_heads=4, d=128),
        # Gradients over ragged windows of vertices that come and go.
        _attn(name="attn_backward_windows", way="backward", T=32, N=20000, heads=4, d=32, buckets=16, reach=32, absent=0.1, ragged=True),
        # Gradients of long histories whose heads share keys.
        _attn(name="attn_backward_long", way="backward", T=4096, N=4, heads=8, kv_heads=2, d=64, buckets=32, reach=128, batch_first=True),
        # Gradients in fp32 at odd sizes, both sides.
        _attn(name="attn_backward_f32", way="backward", dtype="f32", T=101, N=200, heads=4, d=40, causal=False, buckets=16, reach=64),
        # The parameters of one time block: twelve small tensors. Latency counts.
        _adamw(name="adamw_block"),
        # A large model in fp32: 151 tensors and 53 million parameters.
        _adamw(name="adamw_wide", blocks=12, width=584, hidden=2400),
        # Parameters and gradients in bf16 beside fp32 masters, states in 8 bits.
        _adamw(name="adamw_8bit", dtype="bf16", bits=8, blocks=9, width=960, hidden=3840),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if rng.random() < 0.25:
        width = 8 * _log_int(rng, 1, 128)
        hidden = _log_int(rng, 8, 4096)
        most = 1e8 / (4 * width * width + 2 * width * hidden)
        return _adamw(dtype=dtype, bits=rng.choice([8, 32]), blocks=_log_int(rng, 1, max(1, min(16, most))), width=width, hidden=hidden)
    heads = rng.choice([1, 2, 3, 4, 6, 8, 16])
    kv_heads = rng.choice([h for h in (heads, heads, heads // 2, heads // 4, 1) if h and heads % h == 0])
    d = rng.choice([8, 16, 16, 24, 32, 40, 64, 64, 96, 128])
    kind = rng.choice(["window", "window", "long", "long", "step"])
    way = "forward" if kind == "step" else rng.choice(["forward", "backward"])
    pairs = (3e9 if dtype == "bf16" else 3e8) * 16 / (d + 16) / (2.5 if way == "backward" else 1)
    # A row with one key has no gradient but its rounding's: backward windows are not as short as that.
    T = {"window": _log_int(rng, 1 if way == "forward" else 6, 64), "long": _log_int(rng, 65, min(8192, (pairs / heads) ** 0.5)),
         "step": _log_int(rng, 2, 65536)}[kind]
    rows = 1 if kind == "step" else T
    most = min(100000, pairs / (heads * rows * T), 8e7 / (heads * rows * d), 1.3e8 / (kv_heads * T * d))
    N = _log_int(rng, 1 if way == "forward" or kind == "long" else min(8, most), max(1, most))
    buckets = rng.choice([0, 8, 16, 32, 64])
    return _attn(way=way, dtype=dtype, T=T, rows=rows, N=N, heads=heads, kv_heads=kv_heads, d=d, causal=kind == "step" or rng.random() < 0.75,
                 buckets=buckets, reach=_log_int(rng, buckets, 512) if buckets else 0, absent=rng.choice([0.0, 0.0, 0.1, 0.5]),
                 ragged=rng.random() < 0.4, batch_first=rng.random() < 0.4)


# ------------------------------------------------------------------------------------ their inputs


def _bucket_map(buckets, reach, causal):
    """Bucket of each distance -reach .. reach (query's position minus key's): half of one side's buckets for single distances, the
    other half growing to `reach`; keys that follow the query have the upper half of them where they are seen."""
    side = buckets if causal else buckets // 2
    single = max(1, side // 2)
    grown = [min(side - 1, a if a < single else
                 single + int(math.log(a / single) / max(math.log(max(reach, single + 1) / single), 1e-9) * (side - single) + 1e-9))
             for a in range(reach + 1)]
    ahead = [grown[0] if causal else side + grown[a] for a in range(reach, 0, -1)]
    return torch.tensor(ahead + grown, dtype=torch.uint8, device="cuda")


def _prepare_attn(c, g):
    T, rows, N, h, kv, d, dt = (c[k] for k in ("T", "rows", "N", "heads", "kv_heads", "d", "dtype"))

    def seq(n, width, made=torch.randn):
        t = made(*((N, n, width) if c["batch_first"] else (n, N, width)), device="cuda", **({"generator": g} if made is torch.randn else {})).to(DT[dt])
        return t.transpose(0, 1) if c["batch_first"] else t

    s = {"q": seq(rows, h * d), "k": seq(T, kv * d), "v": seq(T, kv * d), "scale": d ** -0.5}
    s["bias"] = 0.5 * torch.randn(h, c["buckets"], generator=g, device="cuda") if c["buckets"] else None
    s["bias_map"] = _bucket_map(c["buckets"], c["reach"], c["causal"]) if c["buckets"] else None
    s["keep"] = (torch.rand(T, N, generator=g, device="cuda") >= c["absent"]).to(torch.uint8) if c["absent"] else None
    s["lengths"] = torch.randint(rows if rows < T else 0, T + 1, (N,), generator=g, device="cuda", dtype=torch.int32) if c["ragged"] else None
    s["first"] = s["lengths"] - rows if c["ragged"] and rows < T else None
    if c["way"] == "forward":
        s["o"], s["lse"] = seq(rows, h * d, torch.zeros), torch.zeros(N, h, rows, device="cuda")
        return s
    made = _attn_forward(dict(s, case=c))       # what the forward pass left
    s["o"], s["lse"] = made["o"].transpose(0, 1).contiguous().transpose(0, 1) if c["batch_first"] else made["o"], made["lse"]
    s["do"] = seq(rows, h * d)
    s["dq"], s["dk"], s["dv"] = seq(rows, h * d, torch.zeros), seq(T, kv * d, torch.zeros), seq(T, kv * d, torch.zeros)
    s["dbias"] = torch.zeros(h, c["buckets"], device="cuda") if c["buckets"] else None
    return s


def _shapes(c):
    """The tensors of `blocks` time blocks, and of large models some behind them: (rows, columns) each, vectors in one row."""
    W, H = c["width"], c["hidden"]
    one = [(1, W), (1, W), (3 * W, W), (1, 3 * W), (W, W), (1, W), (1, W), (1, W), (H, W), (1, H), (W, H), (1, W)]
    return one * c["blocks"] + ([(W, W), (1, W), (1, W), (1, W), (H, W), (1, H), (W, H)] if c["blocks"] > 9 else [])


def _pitch(columns):
    return -(-columns // 16) * 16


def _cut(flat, shapes, whole=False):
    """The tensors that lie one after the other in a flat buffer, each from a multiple of BLOCK on, rows at a pitch of whole 16s."""
    views, at = [], 0
    for R, F in shapes:
        n = R * _pitch(F)
        v = flat[at:at + n].view(R, _pitch(F))
        views.append(v if whole else v[:, :F])
        at += -(-n // BLOCK) * BLOCK
    return views


def _scales(top):
    """The least power of two, and its inverse, times which e4m3's largest number, 448, is at least `top`; 1 for 0."""
    f, e = torch.frexp(top)
    k = torch.where(top > 0, torch.where(f <= 0.875, e - 9, e - 8).clamp(min=-126), 0).to(torch.int32)
    return ((127 + k) << 23).view(torch.float32), ((127 - k) << 23).view(torch.float32)


def _held(x, root=False):
    """Numbers in 8 bits with a scale for each BLOCK; roots that are not zero stay so."""
    b = x.view(-1, BLOCK)
    scale, inverse = _scales(b.abs().amax(1))
    y = b * inverse[:, None]
    if root:
        y = torch.where(b > 0, y.clamp(min=2.0 ** -9), y)
    return y.to(torch.float8_e4m3fn).view(-1), scale


def _prepare_adamw(c, g):
    shapes = _shapes(c)
    total = sum(-(-R * _pitch(F) // BLOCK) * BLOCK for R, F in shapes)
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for v in _cut(inside, shapes):
        v.fill_(True)
    rand = lambda std: torch.where(inside, std * torch.randn(total, generator=g, device="cuda"), 0.0)  # noqa: E731
    p = rand(0.05)
    s = {"shapes": shapes, "t": 100, "p": p.to(DT[c["dtype"]]), "g": rand(1e-3).to(DT[c["dtype"]]),
         "master": p if c["dtype"] == "bf16" else None}
    m, root = rand(3e-4), rand(1e-3).abs() + torch.where(inside, 1e-5, 0.0)
    if c["bits"] == 8:
        (s["m"], s["m_scale"]), (s["v"], s["v_scale"]) = _held(m), _held(root, True)
    else:
        s["m"], s["v"] = m, root * root
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return dict((_prepare_attn if case["op"] == "attn" else _prepare_adamw)(case, g), case=case)


def work(case):
    c = case
    if c["op"] == "adamw":
        n = sum(R * F for R, F in _shapes(c))
        state = 16 if c["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * (state + 12), "flops": 16 * n}     # 12: fp32 p, p, g; or the master twice and p and g in bf16
    T, rows, N, h, kv, d, e = *(c[k] for k in ("T", "rows", "N", "heads", "kv_heads", "d")), SIZE[c["dtype"]]
    share = 0.5 if c["ragged"] else 1.0
    q, k, stats = e * N * rows * h * d, e * N * T * kv * d * share, 4 * N * h * rows
    if rows == T:
        q, stats = q * share, stats * share
    pairs = N * h * rows * T * (share if rows < T else 1 / 3 if c["ragged"] else 1.0) * (0.5 if c["causal"] and rows == T > 1 else 1.0)
    if c["way"] == "forward":
        return {"bytes": 2 * q + 2 * k + stats, "flops": 4 * pairs * d}
    return {"bytes": 4 * q + 4 * k + stats, "flops": 10 * pairs * d}


# ------------------------------------------------------------------------------------ plain forms


def _split(x, heads):
    """[T, N, heads * d] -> [N, heads, T, d] in 32 bits."""
    T, N, F = x.shape
    return x.float().reshape(T, N, heads, F // heads).permute(1, 2, 0, 3).contiguous()


def _joined(x, like):
    N, h, T, d = x.shape
    return x.permute(2, 0, 1, 3).reshape(T, N, h * d).to(like.dtype)


def _seen(s):
    """[N or 1, rows] positions of the queries, [N or 1, 1, 1, rows, T] whether a query sees a key, [N or 1, rows] whether it is one."""
    c, dev = s["case"], s["q"].device
    i, j = torch.arange(c["rows"], device=dev), torch.arange(c["T"], device=dev)
    at = i + (s["first"][:, None].long() if s["first"] is not None else c["T"] - c["rows"])
    at = at.reshape(-1, c["rows"])
    n = s["lengths"].long()[:, None] if s["lengths"] is not None else torch.full((1, 1), c["T"], device=dev)
    live = (at >= 0) & (at < n)
    ok = (j < n)[:, None, :] & live[:, :, None]
    if s["keep"] is not None:
        ok = ok & (s["keep"].t() != 0)[:, None, :]
    if c["causal"]:
        ok = ok & (j <= at[:, :, None])
    return at, ok[:, None, None], live


def _scores(s, q, k):
    """[N, kv_heads, heads of each, rows, T]."""
    c = s["case"]
    N, h, rows, d = q.shape
    x = torch.matmul(q.reshape(N, c["kv_heads"], -1, d), k.transpose(-1, -2)).mul_(s["scale"]).reshape(N, c["kv_heads"], h // c["kv_heads"], rows, -1)
    at, ok, live = _seen(s)
    if s["bias"] is not None:
        away = (at[:, :, None] - torch.arange(c["T"], device=q.device)).clamp(-c["reach"], c["reach"]) + c["reach"]
        b = s["bias"][:, s["bias_map"][away].long()].transpose(0, 1)
        x = x.add_(b.reshape(b.shape[0], c["kv_heads"], -1, rows, c["T"]))
    return x, ok, live


def _attn_forward(s):
    q, k, v = _split(s["q"], s["case"]["heads"]), _split(s["k"], s["case"]["kv_heads"]), _split(s["v"], s["case"]["kv_heads"])
    x, ok, live = _scores(s, q, k)
    x = torch.where(ok, x, -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-3e38)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    N, kv, g, rows, T = x.shape
    o = torch.matmul(x.reshape(N, kv, g * rows, T), v).reshape(N, kv, g, rows, -1) / torch.where(total > 0, total, 1.0)
    lse = (m + torch.log(total)).reshape(N, kv * g, rows)
    lse = torch.where(total.reshape(N, kv * g, rows) > 0, lse, -math.inf)
    return {"o": _joined(o.reshape(N, kv * g, rows, -1), s["q"]), "lse": torch.where(live[:, None], lse, 0.0)}


def _diagonals(x, rows, T):
    """Sums of [h, rows, T] along its diagonals: [h, rows + T - 1], by i - j + T - 1."""
    x = torch.nn.functional.pad(x.flip(-1), (0, rows)).flatten(1)
    return x[:, :rows * (T + rows - 1)].view(-1, rows, T + rows - 1).sum(1)


def _attn_backward(s):
    c = s["case"]
    q, k, v = _split(s["q"], c["heads"]), _split(s["k"], c["kv_heads"]), _split(s["v"], c["kv_heads"])
    do, o = _split(s["do"], c["heads"]), _split(s["o"], c["heads"])
    x, ok, live = _scores(s, q, k)
    N, kv, g, rows, T = x.shape
    lse = s["lse"].reshape(N, kv, g, rows, 1)
    p = torch.where(ok, x.sub_(torch.where(lse > -math.inf, lse, 0.0)).exp_(), 0.0)
    flat = lambda y: y.reshape(N, kv, g * rows, -1)  # noqa: E731
    dv = torch.matmul(flat(p).transpose(-1, -2), flat(do))
    delta = torch.where(live[:, None], (do * o).sum(-1), 0.0).reshape(N, kv, g, rows, 1)
    ds = p.mul_(torch.matmul(flat(do), v.transpose(-1, -2)).view(N, kv, g, rows, T).sub_(delta))
    dq = torch.matmul(flat(ds), k).mul_(s["scale"]).reshape(N, kv * g, rows, -1)
    dk = torch.matmul(flat(ds).transpose(-1, -2), flat(q)).mul_(s["scale"])
    dbias = None
    if s["bias"] is not None:
        sums = _diagonals(ds.reshape(N, kv * g, rows, T).sum(0), rows, T)
        away = (torch.arange(rows + T - 1, device=sums.device) - (rows - 1)).clamp(-c["reach"], c["reach"]) + c["reach"]
        dbias = torch.zeros_like(s["bias"]).index_add_(1, s["bias_map"][away].long(), sums)
    return {"dq": _joined(dq, s["q"]), "dk": _joined(dk, s["k"]), "dv": _joined(dv, s["v"]), "dbias": dbias}


def _factors(t):
    return 1 / (1 - BETAS[0] ** t), (1 - BETAS[1] ** t) ** -0.5


def _adamw_step(s):
    s["t"] += 1
    (b1, b2), (c1, c2) = BETAS, _factors(s["t"])
    g, eight = s["g"].float(), s["case"]["bits"] == 8
    wide = lambda n: (s[n].float().view(-1, BLOCK) * s[n + "_scale"][:, None]).view(-1)  # noqa: E731
    m, v = (wide("m"), wide("v").square()) if eight else (s["m"], s["v"])
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    root = v.sqrt()
    p = s["master"] if s["master"] is not None else s["p"].float()
    p = p - LR * ((m * c1) / (root * c2 + EPS) + DECAY * p)
    if s["master"] is not None:
        s["master"].copy_(p)
    s["p"].copy_(p)
    if eight:
        for n, (codes, scale) in (("m", _held(m)), ("v", _held(root, True))):
            s[n].copy_(codes)
            s[n + "_scale"].copy_(scale)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _adamw_out(s)


def _adamw_out(s):
    return {k: s[k] for k in ("p", "master", "m", "v", "m_scale", "v_scale") if s.get(k) is not None}


def _run_own(s):
    c = s["case"]
    if c["op"] == "adamw":
        if "opt" not in s:       # a program makes it once, over its parameters, gradients and states
            from paper_2309_03523_amd.optimizer import AdamW
            cut = lambda n, whole=False: _cut(s[n], s["shapes"], whole)  # noqa: E731
            states = [dict(m=m, v=v) for m, v in zip(cut("m", True), cut("v", True))]
            if c["bits"] == 8:
                at = 0
                for x, (R, F) in zip(states, s["shapes"]):
                    n = -(-R * _pitch(F) // BLOCK)
                    x.update(m_scale=s["m_scale"][at:at + n], v_scale=s["v_scale"][at:at + n])
                    at += n
            s["opt"] = AdamW(cut("p"), cut("g"), masters=cut("master") if s["master"] is not None else None, states=states, steps=s["t"],
                             lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY, bits=c["bits"])
        s["opt"].step()
        return _adamw_out(s)
    from paper_2309_03523_amd import binding as b
    kw = dict(heads=c["heads"], kv_heads=c["kv_heads"], scale=s["scale"], causal=c["causal"], first=s["first"], lengths=s["lengths"], keep=s["keep"],
              bias=s["bias"], bias_map=s["bias_map"])
    if "workspace" not in s:
        size = b.attn_workspace_bytes(c["rows"], c["T"], c["N"], c["heads"], c["d"], kv_heads=c["kv_heads"], dtype=c["dtype"], causal=c["causal"],
                                      buckets=c["buckets"], reach=c["reach"], backward=c["way"] == "backward")
        s["workspace"] = torch.empty(max(16, size), dtype=torch.uint8, device="cuda")
    if c["way"] == "forward":
        b.attn_forward(s["q"], s["k"], s["v"], s["o"], lse=s["lse"], workspace=s["workspace"], **kw)
        return {k: s[k] for k in ("o", "lse")}
    b.attn_backward(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["dq"], s["dk"], s["dv"], dbias=s["dbias"], workspace=s["workspace"], **kw)
    return {k: s[k] for k in ("dq", "dk", "dv", "dbias")}


def run(state):
    if own:
        return _run_own(state)
    if state["case"]["op"] == "adamw":
        return _adamw_step(state)
    return (_attn_forward if state["case"]["way"] == "forward" else _attn_backward)(state)


# ------------------------------------------------------------------------------------ from the definitions, in 64 bits


def _exact_adamw(s):
    t, g = s["t"] + 1, s["g"].double()
    if s["case"]["bits"] == 8:
        m, r = (s[n].double() * s[n + "_scale"].double().repeat_interleave(BLOCK) for n in ("m", "v"))
        v = r * r
    else:
        m, v = s["m"].double(), s["v"].double()
    m = BETAS[0] * m + (1 - BETAS[0]) * g
    v = BETAS[1] * v + (1 - BETAS[1]) * g * g
    p = (s["master"] if s["master"] is not None else s["p"]).double()
    p = p * (1 - LR * DECAY) - LR * (m / (1 - BETAS[0] ** t)) / (torch.sqrt(v / (1 - BETAS[1] ** t)) + EPS)
    out = {"p": p, "master": p if s["master"] is not None else None}
    return dict(out, m=m, v=v) if s["case"]["bits"] == 32 else dict(out, m=None, v=None, m_scale=None, v_scale=None)


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "adamw":
        return _exact_adamw(s)
    T, rows, N, h, kv, d = (c[k] for k in ("T", "rows", "N", "heads", "kv_heads", "d"))
    dev = s["q"].device
    n = s["lengths"].long() if s["lengths"] is not None else torch.full((N,), T, device=dev)
    first = s["first"].long() if s["first"] is not None else torch.full((N,), T - rows, device=dev)
    at = first[:, None] + torch.arange(rows, device=dev)
    live = (at >= 0) & (at < n[:, None])
    key = torch.arange(T, device=dev)
    there = key < n[:, None]
    if s["keep"] is not None:
        there = there & s["keep"].t().bool()
    head = lambda x, k: x[..., k * d:(k + 1) * d].transpose(0, 1).double().contiguous()  # noqa: E731
    forward = c["way"] == "forward"
    out = {"o": torch.zeros(rows, N, h * d, dtype=torch.float64, device=dev), "lse": torch.zeros(N, h, rows, dtype=torch.float64, device=dev)} if forward else \
        {"dq": torch.zeros(rows, N, h * d, dtype=torch.float64, device=dev), "dk": torch.zeros(T, N, kv * d, dtype=torch.float64, device=dev),
         "dv": torch.zeros(T, N, kv * d, dtype=torch.float64, device=dev),
         "dbias": torch.zeros(h, c["buckets"], dtype=torch.float64, device=dev) if c["buckets"] else None}
    step = max(1, int(1.5e9 // (rows * T)))           # sequences at a time
    for a in range(0, N, step):
        b = slice(a, min(N, a + step))
        apart = at[b, :, None] - key
        sees = there[b, None, :] & live[b, :, None]
        if c["causal"]:
            sees = sees & (apart >= 0)
        which = s["bias_map"].long()[apart.clamp(-c["reach"], c["reach"]) + c["reach"]] if c["buckets"] else None
        for x in range(h):
            y = x // (h // kv)
            Q, K, V = head(s["q"][:, b], x), head(s["k"][:, b], y), head(s["v"][:, b], y)
            S = torch.bmm(Q, K.transpose(1, 2).contiguous()) * s["scale"]
            if c["buckets"]:
                S = S + s["bias"][x].double()[which]
            S = S.masked_fill(~sees, -math.inf)
            mine = slice(x * d, (x + 1) * d)
            if forward:
                L = torch.logsumexp(S, -1)
                P = torch.exp(S - L.clamp(min=-1e300)[..., None])
                out["o"][:, b, mine] = torch.bmm(P, V).transpose(0, 1)
                out["lse"][b, x] = torch.where(live[b], L, 0.0)
                continue
            P = torch.exp(S - s["lse"][b, x].double().clamp(min=-1e300)[..., None])
            G, O = head(s["do"][:, b], x), head(s["o"][:, b], x)
            D = P * (torch.bmm(G, V.transpose(1, 2).contiguous()) - (G * O).sum(-1, keepdim=True))
            D = torch.where(sees, D, 0.0)
            theirs = slice(y * d, (y + 1) * d)
            out["dq"][:, b, mine] = (s["scale"] * torch.bmm(D, K)).transpose(0, 1)
            out["dk"][:, b, theirs] += (s["scale"] * torch.bmm(D.transpose(1, 2).contiguous(), Q)).transpose(0, 1)
            out["dv"][:, b, theirs] += torch.bmm(P.transpose(1, 2).contiguous(), G).transpose(0, 1)
            if c["buckets"]:
                out["dbias"][x] += torch.bincount(which.reshape(-1), weights=D.reshape(-1), minlength=c["buckets"])
    return out
