"""A pre-norm time block over snapshots, built of the library's operators: a trainable time encoder whose state is carried
from window to window (as H0 / HN of the recurrent layers), to stand behind a structure encoder or another block.

    n = norm1(x);  q, k, v = qkv(n);  o = linear attention with a decay per head over every vertex' sequence, or
                                          softmax attention with a learned bias by buckets of distance
    m = x + out(o);  y = m + down(act(up(norm2(m))))

x, y are [T, N, width], snapshots by vertices, float32 or bfloat16.  Every step runs in the HIP library
(binding.norm_*, linear_*, decay_attn_*, attn_*); PyTorch supplies device memory and the stream.
"""
from __future__ import annotations

import numpy as np

from . import binding

NAMES = ["norm1.weight", "norm1.bias", "qkv.weight", "qkv.bias", "out.weight", "out.bias", "norm2.weight", "norm2.bias",
         "up.weight", "up.bias", "down.weight", "down.bias"]


class TimeBlock:
    """width = heads * size of a head (a multiple of 8, at most 128); hidden: width between up and down.  decay: one number in
    [0, 1] a head, default 1 - 2^-(2 + 6 h / heads), memories of 4 to some 200 snapshots.  exact: binding.linear_backward's, for
    the gradients behind the activation.

    attention="softmax": every snapshot attends to itself and those before it, with a learned bias, the parameter "attn.bias" [heads, buckets]: of
    the distances' `buckets` (0: no bias) half hold one distance each and the rest grow up to `reach` (binding.attn_buckets).  Then no state is carried: a new
    snapshot attends to the keys and values of those before it, which the caller keeps in a cache.

    Parameters are fp32, (out, in), named as in NAMES; set_param copies them in, get_param reads one or "<name>.grad": they and release()
    wait for the device, forward and backward only enqueue.  A block runs one call at a time.  Its buffers are made at the first call
    with new sizes, so a call may be captured into a HIP graph after an eager one of the same sizes.  Those of the last SIZES sizes
    and all that a captured call uses are kept until release()."""

    attention, buckets = "decay", 0
    SIZES = 8      # a program trains, evaluates and steps at a few sizes; the vertices of a served graph change in number for ever

    def __init__(self, width: int, heads: int, hidden: int, *, dtype: str = "f32", act: str = "gelu", decay=None, eps: float = 1e-5,
                 exact: bool = False, attention: str = "decay", buckets: int = 16, reach: int = 32, device="cuda:0"):
        import torch
        if attention not in ("decay", "softmax") or (attention == "softmax" and decay is not None):
            raise ValueError("attention must be decay or softmax; only the former has decays")
        if heads < 1 or width % heads or (width // heads) % 8 or width // heads > 128:
            raise ValueError("width must be heads times a multiple of 8 that is at most 128")
        if hidden < 1 or act not in binding.LINEAR_ACT or dtype not in binding.DTYPE:
            raise ValueError("unknown activation or element type, or hidden < 1")
        self.width, self.heads, self.hidden, self.act, self.eps, self.exact = width, heads, hidden, act, float(eps), bool(exact)
        self.dtype_name, self.dtype = dtype, {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.attention, self.buckets = attention, int(buckets) if attention == "softmax" else 0
        bias_map = binding.attn_buckets(self.buckets, reach) if self.buckets else None
        self.reach = int(reach) if self.buckets else 0
        g = np.asarray(decay if decay is not None else 1.0 - 2.0 ** -(2.0 + 6.0 * np.arange(heads) / heads), np.float32).reshape(-1)
        if g.size != heads or not ((g >= 0) & (g <= 1)).all():
            raise ValueError("decay must hold one number in [0, 1] for each head")
        self._decay = torch.from_numpy(g).to(self.device)
        W = width
        self.shapes = {"norm1.weight": (W,), "norm1.bias": (W,), "qkv.weight": (3 * W, W), "qkv.bias": (3 * W,), "out.weight": (W, W),
                       "out.bias": (W,), "norm2.weight": (W,), "norm2.bias": (W,), "up.weight": (hidden, W), "up.bias": (hidden,),
                       "down.weight": (W, hidden), "down.bias": (W,)}
        self.names = list(NAMES)
        if self.buckets:
            self.names.append("attn.bias")
            self.shapes["attn.bias"] = (heads, self.buckets)
        self._map = torch.from_numpy(bias_map).to(self.device) if self.buckets else None
        self._p = {n: self._room(s, self._kind(n)) for n, s in self.shapes.items()}
        for n in ("norm1.weight", "norm2.weight"):
            self._p[n].fill_(1.0)
        self._g = {}
        self._buffers = {}
        self._last = None
        self._settle()

    def _kind(self, name: str):
        import torch
        return self.dtype if len(self.shapes[name]) == 2 and name != "attn.bias" else torch.float32

    def _grads(self):
        if not self._g:
            self._g = {n: self._room(s, self._kind(n)) for n, s in self.shapes.items()}
        return self._g

    def trained(self):
        """(parameters, gradients): the device tensors in the order of `names`, as an optimizer takes them (optimizer.AdamW(*block.trained())).  They
        stay where they are; backward writes the gradients.  attn.bias is one row."""
        g = self._grads()
        self._settle()
        flat = lambda t, n: t.view(1, -1) if n == "attn.bias" else t  # noqa: E731
        return [flat(self._p[n], n) for n in self.names], [flat(g[n], n) for n in self.names]

    def _room(self, shape, dtype):
        """Zeroed rows at a pitch that is a multiple of 16 bytes."""
        import torch
        if shape == self.shapes.get("attn.bias"):       # one piece, as the library takes it
            return torch.zeros(shape, dtype=dtype, device=self.device)
        per = 16 // torch.empty(0, dtype=dtype).element_size()
        buf = torch.zeros(*shape[:-1], -(-shape[-1] // per) * per, dtype=dtype, device=self.device)
        return buf[..., :shape[-1]]

    def _settle(self):
        """Waits for the device: calls that were given other streams and replayed graphs read and write what the block holds."""
        import torch
        torch.cuda.synchronize(self.device)

    # -- parameters (these calls synchronise, as those of a layer do)
    def set_param(self, name: str, value):
        import torch
        v = torch.from_numpy(np.ascontiguousarray(value, np.float32))
        if tuple(v.shape) != self.shapes[name]:
            raise ValueError(f"{name} must have shape {self.shapes[name]}")
        self._settle()
        self._p[name].copy_(v.to(self._p[name].dtype))
        self._settle()

    def set_params(self, params: dict):
        for k, v in params.items():
            self.set_param(k, v)

    def get_param(self, name: str) -> np.ndarray:
        """The parameter as the kernels use it, or "<name>.grad" after a backward, as fp32."""
        if name.endswith(".grad"):
            if name[:-5] not in self._g:
                raise RuntimeError("no gradient yet: run a backward first")
            self._settle()
            return self._g[name[:-5]].float().cpu().numpy()
        self._settle()
        return self._p[name].float().cpu().numpy()

    # -- memory
    def release(self):
        """Drops the buffers of all sizes once the device has done with them; graphs captured before must not be replayed after it."""
        self._settle()
        self._buffers.clear()
        self._last = None

    def _capturing(self, stream) -> bool:
        """Whether the call's stream, or the current one of the block's device, is being captured."""
        import torch
        if torch.cuda.current_device() == self.device.index:
            if torch.cuda.is_current_stream_capturing():
                return True
        else:
            with torch.cuda.device(self.device):
                if torch.cuda.is_current_stream_capturing():
                    return True
        if stream is None:
            return False
        with torch.cuda.stream(stream):
            return torch.cuda.is_current_stream_capturing()

    def _made(self, T: int, N: int, train: bool, stream, kept: int = 0):
        import torch
        key = (T, N, train, kept) if kept else (T, N, train)
        b = self._buffers.pop(key, None)
        if b is not None:
            self._buffers[key] = b      # the last to go
            return b
        if self._capturing(stream):      # memory made now would belong to the graph, and be cleared in it
            raise RuntimeError("these sizes are new to the block: make one eager call of them before the captured one")
        W, Hd, h = self.width, self.hidden, self.heads
        b = {"n": self._room((T, N, W), self.dtype), "qkv": self._room((T, N, 3 * W), self.dtype), "o": self._room((T, N, W), self.dtype),
             "m": self._room((T, N, W), self.dtype), "u": self._room((T, N, Hd), self.dtype)}
        if self.attention == "softmax":
            size = lambda Tk, back: binding.attn_workspace_bytes(T, Tk, N, h, W // h, dtype=self.dtype_name, buckets=self.buckets, reach=self.reach, backward=back)  # noqa: E731
            ws = max([size(kept or T, False), size(T, True)] if train else [size(kept or T, False)])      # it grows with the keys
        else:
            ws = binding.decay_attn_workspace_bytes(T, N, h, W // h, W // h, backward=train)
        if train:
            R = T * N
            b["n2"], b["pre"] = self._room((T, N, W), self.dtype), self._room((T, N, Hd), self.dtype)
            for k in ("mean1", "rstd1", "mean2", "rstd2"):
                b[k] = torch.empty(R, device=self.device)
            b["du"], b["dw"], b["dm"] = self._room((T, N, Hd), self.dtype), self._room((T, N, W), self.dtype), self._room((T, N, W), self.dtype)
            b["dqkv"] = self._room((T, N, 3 * W), self.dtype)
            size = lambda k, m, act: binding.linear_workspace_bytes(R, k, m, dtype=self.dtype_name, act=act, exact=self.exact)  # noqa: E731
            ws = max(ws, binding.norm_workspace_bytes(R, W), size(W, 3 * W, "none"), size(W, W, "none"), size(W, Hd, self.act),
                     size(Hd, W, "none"))
            b["lse"] = torch.empty(N, h, T, device=self.device) if self.attention == "softmax" else None
            self._grads()
        else:
            b["n2"] = b["n"]       # nothing is read again
        b["ws"] = torch.empty(max(ws, 16), dtype=torch.uint8, device=self.device)
        if stream is not None:     # the zeros above were written on the current stream
            stream.wait_stream(torch.cuda.current_stream(self.device))
        b["home"], b["done"], b["captured"] = torch.cuda.current_stream(self.device), None, False
        self._buffers[key] = b
        for k in [k for k, s in self._buffers.items() if not s["captured"]][:-self.SIZES]:
            old = self._buffers.pop(k)
            if old["done"] is not None:      # the allocator hands its memory to what is enqueued on that stream from here on
                old["home"].wait_event(old["done"])
        return b

    def _used(self, b, stream):
        """Notes where a call ran that uses a set of buffers: in a graph, or, for the stream that they were made on, on another one."""
        import torch
        on = stream if stream is not None else torch.cuda.current_stream(self.device)
        if self._capturing(stream):
            b["captured"] = True
        elif on != b["home"]:
            b["done"] = b["done"] or torch.cuda.Event()
            b["done"].record(on)

    def _kept(self, b, S0, stream):
        """A copy of the first state, which the call is about to overwrite, for backward."""
        import torch
        shape = (b["m"].shape[1], self.heads, self.width // self.heads, self.width // self.heads)
        if S0.shape != shape or S0.dtype != torch.float32 or S0.device != self.device:
            raise ValueError(f"S0 must be float32 {list(shape)} on the block's device")
        on = stream if stream is not None else torch.cuda.current_stream(self.device)
        if "s0" not in b:
            if self._capturing(stream):
                raise RuntimeError("a state in place is new to these sizes: make one eager call of it before the captured one")
            with torch.cuda.stream(b["home"]):
                b["s0"] = torch.empty(shape, device=self.device)
            on.wait_stream(b["home"])
        with torch.cuda.stream(on):
            b["s0"].copy_(S0)
        return b["s0"]

    def _blank(self, t, lengths, stream):
        """Rows behind the sequences hold what an earlier call left; no attention and no gradient there is zero."""
        import torch
        if lengths is not None:
            with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(self.device)):
                t.zero_()

    @staticmethod
    def _overlap(a, b) -> bool:
        """Whether two tensors share memory; rows side by side in one buffer do not."""
        if a is None or b is None or not a.numel() or not b.numel():
            return False
        size = lambda t: t.element_size()  # noqa: E731
        last = lambda t: t.data_ptr() + (sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1) * size(t)  # noqa: E731
        if a.data_ptr() >= last(b) or b.data_ptr() >= last(a):
            return False
        rows = [s for n, s in zip(a.shape[:-1], a.stride()) if n > 1]
        if not rows or a.stride() != b.stride() or a.shape[:-1] != b.shape[:-1] or size(a) != size(b) or not min(rows) or any(s % min(rows) for s in rows):
            return True
        pitch, first = min(rows) * size(a), b.data_ptr() - a.data_ptr()
        return not a.shape[-1] * size(a) <= first % pitch <= pitch - b.shape[-1] * size(b)

    def _rows(self, t, name: str, like=None):
        if t.dim() != 3 or t.shape[2] != self.width or t.dtype != self.dtype or t.device != self.device:
            raise ValueError(f"{name} must be [T, N, {self.width}] of the block's element type and device")
        if like is not None and t.shape != like.shape:
            raise ValueError(f"{name} must have the shape of X, {list(like.shape)}, not {list(t.shape)}")

    # -- the path
    def forward(self, X, Y, *, S0=None, SN=None, lengths=None, reset=None, keep=None, cache=None, at: int = 0, train: bool = True, stream=None):
        """Y = block(X).  S0, SN fp32 [N, heads, d, d]: states entering and leaving the window (SN may be S0, of which train=True then
        keeps a copy); lengths, reset as binding.decay_attn_forward has them (rows behind a sequence take part in the row-wise steps
        alone).  train=True keeps what backward reads, X and S0 among it, so Y must lie apart from X; with train=False Y may be X.
        T = 1 with train=False is the form for one new snapshot.

        With softmax attention there are no states and resets.  keep uint8 [T, N], as binding.attn_forward has it: snapshots that nobody attends to.  cache
        [S, N, 2 width], rows at least, of the block's element type, with train=False: X are snapshots at .. at + T - 1; their keys and values are written
        to those rows, and they attend to all rows up to their own, of which keep [at + T, N] may mask some.  `at` is one for all vertices, and a captured call
        keeps it."""
        self._last = None
        if self.attention == "softmax":
            if S0 is not None or SN is not None or reset is not None:
                raise ValueError("softmax attention has no states and no resets")
            if cache is not None:
                if train or lengths is not None:
                    raise ValueError("a cache goes with train=False and without lengths")
                if cache.dim() != 3 or cache.shape[1:] != (X.shape[1], 2 * self.width) or cache.dtype != self.dtype or cache.device != self.device:
                    raise ValueError(f"cache must be [S, {X.shape[1]}, {2 * self.width}] of the block's element type and device")
                if at < 0 or at + X.shape[0] > cache.shape[0]:
                    raise ValueError("the snapshots must fit the cache")
        elif keep is not None or cache is not None:
            raise ValueError("keep and cache go with softmax attention")
        self._rows(X, "X")
        self._rows(Y, "Y", X)
        if train and self._overlap(X, Y):
            raise ValueError("with train=True Y must lie apart from X, which backward reads")
        T, N = X.shape[:2]
        b = self._made(T, N, train, stream, cache.shape[0] if cache is not None else 0)
        try:
            if train and self._overlap(S0, SN):
                S0 = self._kept(b, S0, stream)
            self._forward(b, X, Y, S0, SN, lengths, reset if self.attention == "decay" else keep, cache, at, stream)
        finally:
            self._used(b, stream)
        self._last = (b, X, S0, lengths, reset if self.attention == "decay" else keep) if train else None
        return Y

    def _softmax(self):
        """What every call of the attention has."""
        return dict(heads=self.heads, scale=(self.width // self.heads) ** -0.5, bias=self._p.get("attn.bias"), bias_map=self._map)

    def _forward(self, b, X, Y, S0, SN, lengths, mask, cache, at, stream):
        p, W = self._p, self.width
        q, k, v = b["qkv"][..., :W], b["qkv"][..., W:2 * W], b["qkv"][..., 2 * W:]
        binding.norm_forward(X, b["n"], gamma=p["norm1.weight"], beta=p["norm1.bias"], mean=b.get("mean1"), rstd=b.get("rstd1"), eps=self.eps,
                             stream=stream)
        if cache is None:
            binding.linear_forward(b["n"], p["qkv.weight"], b["qkv"], bias=p["qkv.bias"], stream=stream)
        else:       # keys and values to where they stay
            end = at + X.shape[0]
            binding.linear_forward(b["n"], p["qkv.weight"][:W], q, bias=p["qkv.bias"][:W], stream=stream)
            binding.linear_forward(b["n"], p["qkv.weight"][W:], cache[at:end], bias=p["qkv.bias"][W:], stream=stream)
            k, v = cache[:end, :, :W], cache[:end, :, W:]
        self._blank(b["o"], lengths, stream)
        if self.attention == "softmax":
            binding.attn_forward(q, k, v, b["o"], lengths=lengths, keep=mask, lse=b.get("lse"), workspace=b["ws"], stream=stream, **self._softmax())
        else:
            binding.decay_attn_forward(q, k, v, self._decay, b["o"], heads=self.heads, scale=(W // self.heads) ** -0.5, s0=S0, sn=SN, lengths=lengths,
                                       reset=mask, workspace=b["ws"], stream=stream)
        binding.linear_forward(b["o"], p["out.weight"], b["m"], bias=p["out.bias"], residual=X, stream=stream)
        binding.norm_forward(b["m"], b["n2"], gamma=p["norm2.weight"], beta=p["norm2.bias"], mean=b.get("mean2"), rstd=b.get("rstd2"),
                             eps=self.eps, stream=stream)
        binding.linear_forward(b["n2"], p["up.weight"], b["u"], bias=p["up.bias"], act=self.act, pre=b.get("pre"), stream=stream)
        binding.linear_forward(b["u"], p["down.weight"], Y, bias=p["down.bias"], residual=b["m"], stream=stream)

    def backward(self, dY, *, dX=None, dSN=None, dS0=None, stream=None):
        """Gradients of the last forward with train=True: of the parameters (get_param("<name>.grad")), of X into dX if given
        (dX may be dY), and of S0 into dS0.  X, S0, lengths, reset and keep of that forward must be unchanged."""
        if self._last is None:
            raise RuntimeError("backward follows a forward with train=True")
        b, X, S0, lengths, mask = self._last
        if self.attention == "softmax" and (dSN is not None or dS0 is not None):
            raise ValueError("softmax attention has no states")
        self._rows(dY, "dY", X)
        if dX is not None:
            self._rows(dX, "dX", X)
        try:
            self._backward(b, X, S0, lengths, mask, dY, dX, dSN, dS0, stream)
        finally:
            self._used(b, stream)

    def _backward(self, b, X, S0, lengths, mask, dY, dX, dSN, dS0, stream):
        p, g, W, ws = self._p, self._g, self.width, b["ws"]
        cut = lambda t: (t[..., :W], t[..., W:2 * W], t[..., 2 * W:])  # noqa: E731
        lin = lambda dy, x, n, dx, **kw: binding.linear_backward(dy, x, p[n + ".weight"], dx=dx, dw=g[n + ".weight"], dbias=g[n + ".bias"],  # noqa: E731
                                                                  workspace=ws, stream=stream, **kw)
        lin(dY, b["u"], "down", b["du"])
        lin(b["du"], b["n2"], "up", b["dw"], pre=b["pre"], act=self.act, exact=self.exact)
        binding.norm_backward(b["dw"], b["m"], b["mean2"], b["rstd2"], b["dm"], gamma=p["norm2.weight"], add=dY, dgamma=g["norm2.weight"],
                              dbeta=g["norm2.bias"], workspace=ws, stream=stream)
        lin(b["dm"], b["o"], "out", b["dw"])
        self._blank(b["dqkv"], lengths, stream)
        if self.attention == "softmax":
            binding.attn_backward(*cut(b["qkv"]), b["o"], b["lse"], b["dw"], *cut(b["dqkv"]), lengths=lengths, keep=mask, dbias=g.get("attn.bias"),
                                  workspace=ws, stream=stream, **self._softmax())
        else:
            binding.decay_attn_backward(*cut(b["qkv"]), self._decay, b["dw"], *cut(b["dqkv"]), heads=self.heads, scale=(W // self.heads) ** -0.5, s0=S0,
                                        dsn=dSN, ds0=dS0, lengths=lengths, reset=mask, workspace=ws, stream=stream)
        lin(b["dqkv"], b["n"], "qkv", b["dw"])
        binding.norm_backward(b["dw"], X, b["mean1"], b["rstd1"], dX if dX is not None else b["dw"], gamma=p["norm1.weight"], add=b["dm"],
                              dgamma=g["norm1.weight"], dbeta=g["norm1.bias"], workspace=ws, stream=stream)
