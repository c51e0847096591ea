"""AdamW over the parameters of whatever the library trains: one launch for all tensors, states in 32 or 8 bits.

    m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p - lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay p)

The step runs in the HIP library (binding.adamw_*); PyTorch supplies device memory and the stream.
"""
from __future__ import annotations

from . import binding


class AdamW:
    """params, grads: device tensors of rows [..., F] or vectors [F], float32 or bfloat16, all on one device.  masters: fp32 copies that are stepped in
    place of bfloat16 parameters (which receive them rounded): True makes them, a list gives them (None: none for that tensor; never for a float32 one).
    weight_decay: one number or one a tensor.  bits: 32, or 8 (e4m3 numbers of m and of sqrt(v) with a power of two for each 256).

    states: to resume, the list `states` of an optimizer of the same tensors and bits, and steps, the number of steps done.  The list holds a dict for each
    tensor: m, v and, with bits=8, m_scale, v_scale; rows at binding.adamw_pitch(F) places, 8-bit ones as float8_e4m3fn.

    on_device=True keeps the number of steps and the learning rate on the device, so that a step that is captured into a graph counts, and takes the rate
    of set_lr, when it is replayed; without it a step is not captured.  The optimizer keeps its tensors and their addresses: writing new values into them is seen, putting other
    tensors in their place is not.  After parameters that have masters were set from outside, call reload().  It runs one call at a time: a step only enqueues, the
    constructor, release(), reload() and the number of steps on the device wait for the device."""

    def __init__(self, params, grads, *, masters=None, states=None, steps: int = 0, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay=0.01, bits: int = 32, on_device: bool = False):
        import torch
        params, grads = list(params), list(grads)
        n = len(params)
        if masters is not None and not isinstance(masters, bool):
            masters = list(masters)
        if n == 0 or len(grads) != n or (isinstance(masters, list) and len(masters) != n) or (states is not None and len(states) != n):
            raise ValueError("params must not be empty; grads, masters and states go with them, one each")
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        decays = [float(weight_decay)] * n if not isinstance(weight_decay, (list, tuple)) else [float(x) for x in weight_decay]
        if len(decays) != n or not all(x >= 0 for x in decays):
            raise ValueError("weight_decay must be one number >= 0, or one for each parameter")
        b1, b2 = (float(x) for x in betas)
        if not (0 <= b1 < 1 and 0 <= b2 < 1 and eps >= 0 and int(steps) >= 0):
            raise ValueError("betas must be in [0, 1), eps and steps >= 0")
        dev = params[0].device
        if dev.type != "cuda" or any(t.device != dev for t in params + grads):
            raise ValueError("parameters and gradients must be on one device")
        if any(p.shape != g.shape or p.dim() < 1 for p, g in zip(params, grads)):
            raise ValueError("a gradient must have its parameter's shape")
        self.device, self.bits, self.betas, self.eps = dev, bits, (b1, b2), float(eps)
        self._handle, self._steps, self._at, self._lr_at = None, int(steps), None, None
        self.lr = self._checked(lr)
        self.params, self.grads = params, grads
        with torch.cuda.device(dev):
            if masters is True:
                masters = [self._copied(p) if p.dtype == torch.bfloat16 else None for p in params]
            self.masters = masters or [None] * n
            self.states = [dict(s) for s in states] if states is not None else [self._state(p) for p in params]
            if on_device:
                self._at, self._lr_at = torch.full((1,), self._steps, dtype=torch.int64, device=dev), torch.full((1,), self.lr, device=dev)
            torch.cuda.synchronize(dev)      # what was made here may be used on any stream
            self._handle = binding.adamw_create([dict(s, p=p, g=g, master=m, weight_decay=w) for p, g, m, s, w in zip(params, grads, self.masters, self.states, decays)],
                                                bits, dev.index)

    @staticmethod
    def _checked(lr) -> float:
        lr = float(lr)
        if not 0 <= lr < float("inf"):
            raise ValueError("lr must be finite and >= 0")
        return lr

    @staticmethod
    def _copied(p):
        """An fp32 copy in rows of its own, at a pitch that is a multiple of 16 bytes."""
        import torch
        F = p.shape[-1]
        t = torch.zeros(*p.shape[:-1], -(-F // 4) * 4, device=p.device)[..., :F]
        return t.copy_(p)

    def _state(self, p):
        import torch
        F = p.shape[-1]
        pitch = binding.adamw_pitch(F)
        R = p.numel() // F if F else 0
        if self.bits == 32:
            return {k: torch.zeros(R, pitch, device=p.device) for k in ("m", "v")}
        s = {k: torch.zeros(R, pitch, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn) for k in ("m", "v")}
        return dict(s, **{k + "_scale": torch.ones(-(-R * pitch // 256), device=p.device) for k in ("m", "v")})

    def step(self, *, stream=None):
        """One step from the gradients as they are when it runs."""
        if self._handle is None:
            raise RuntimeError("the optimizer was released")
        t = self._steps + 1
        binding.adamw_step(self._handle, self.device.index, t, lr=self.lr, beta1=self.betas[0], beta2=self.betas[1], eps=self.eps, steps=self._at,
                           lr_at=self._lr_at, stream=stream)
        self._steps = t

    def set_lr(self, lr: float, *, stream=None):
        """The learning rate of the steps from here on; with on_device it is enqueued."""
        import torch
        self.lr = self._checked(lr)
        if self._lr_at is not None:
            with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(self.device)):
                self._lr_at.fill_(self.lr)

    @property
    def steps(self) -> int:
        """Steps done; with on_device as the device has counted them (waits for it)."""
        import torch
        if self._at is None:
            return self._steps
        torch.cuda.synchronize(self.device)
        return int(self._at.item())

    def reload(self):
        """Takes the parameters' values into their masters (waits for the device)."""
        import torch
        torch.cuda.synchronize(self.device)
        for p, m in zip(self.params, self.masters):
            if m is not None:
                m.copy_(p)
        torch.cuda.synchronize(self.device)

    def release(self):
        """Frees the library's table once the device has done with it; graphs captured before must not be replayed after it."""
        import torch
        if self._handle is not None:
            torch.cuda.synchronize(self.device)
            binding.adamw_destroy(self._handle)
            self._handle = None

    def __del__(self):
        try:
            if getattr(self, "_handle", None) is not None:
                binding.adamw_destroy(self._handle)
        except Exception:
            pass
