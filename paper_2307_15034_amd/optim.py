"""AdamW over all tensors of a model at once (the fno_adamw_* and fno_grad_norm
calls), on torch tensors.

PyTorch supplies memory and streams only; every step runs in the HIP kernels.
"""
from __future__ import annotations

import ctypes
from array import array
from operator import attrgetter
from typing import Dict, List, Optional, Sequence, Union

import torch

from . import binding as B
from .layer import DTYPE_CODES, _addr, _external, _stream_of

_dtype_of = attrgetter("dtype")


class AdamW:
    """AdamW on the lists `params` and `grads`.

    params: float32, float16 or bfloat16 tensors of any shapes (complex weights
    as their (re, im) pairs); grads: float32 or the parameter's type, the same
    shapes.  All contiguous, on one GPU, 16-byte aligned, none overlapping
    another.  masters: the float32 values that 16-bit parameters round (one
    entry each, None for a float32 parameter or to go without), made by
    `make_masters`.  weight_decay: one value, or one per tensor.

    state_bits 32 keeps the moments as float32, 8 as codes with a scale per
    256 elements (one value, or one per tensor).  `states` takes up moments
    that exist (one dict per tensor: exp_avg and exp_avg_sq, with
    exp_avg_scale and exp_avg_sq_scale in 8 bits), after `step` steps;
    otherwise they start at zero.

    The object writes the addresses of its tensors down once and keeps their
    storage; `set_grads` (and `step(grads=...)`) takes other gradients.  A
    parameter that is to change its storage needs a new object.

    device_control: the step number, the clipped scale and the skip of
    non-finite gradients live on the GPU; each `step` then follows one
    `clip_grads` (and is refused otherwise, unless clip_grads was captured:
    its replays are not seen here), nothing is read by the host, and both can
    be captured in a HIP graph.  Calls of one object belong on one stream (or on streams that
    wait for each other); what the object makes itself is filled when the
    constructor returns, so that any stream may take the first call.  The
    caller's tensors are the caller's: where `stream` is given, it has waited
    for their values, and they stay until its work is done.
    """

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor],
                 masters: Optional[Sequence[Optional[torch.Tensor]]] = None,
                 states: Optional[Sequence[Dict[str, torch.Tensor]]] = None, lr: float = 1e-3,
                 betas: Sequence[float] = (0.9, 0.999), eps: float = 1e-8,
                 weight_decay: Union[float, Sequence[float]] = 1e-2,
                 state_bits: Union[int, Sequence[int]] = 32, step: int = 0,
                 device_control: bool = False):
        self.params = list(params)
        n = len(self.params)
        if n == 0:
            raise ValueError("params is empty")
        self.device = self.params[0].device
        self.masters = self._per_tensor(masters if masters is not None else [None] * n, "masters")
        self.state_bits = self._per_tensor([state_bits] * n if isinstance(state_bits, int)
                                           else state_bits, "state_bits")
        decay = self._per_tensor([weight_decay] * n if isinstance(weight_decay, (int, float))
                                 else weight_decay, "weight_decay")
        for b in self.state_bits:
            if b not in (32, 8):
                raise ValueError(f"state_bits {b}, expected 32 or 8")
        if step < 0:
            raise ValueError(f"step {step}, expected at least 0")
        self._steps = int(step)
        self.desc = B.FnoAdamwDesc(float(lr), float(betas[0]), float(betas[1]), float(eps))
        self.states: List[Dict[str, torch.Tensor]] = (
            [self._zero_state(p, b) for p, b in zip(self.params, self.state_bits)]
            if states is None else [dict(s) for s in self._per_tensor(states, "states")])
        self._list = (B.FnoAdamwTensor * n)()
        seen = set()
        for i, (t, p) in enumerate(zip(self._list, self.params)):
            if p.dtype not in DTYPE_CODES:
                raise ValueError(f"params[{i}]: dtype {p.dtype}, expected float32, float16 or "
                                 "bfloat16")
            t.param = _addr(p, None, None, f"params[{i}]", self.device) or None
            t.param_dtype, t.n = DTYPE_CODES[p.dtype], p.numel()
            m = self.masters[i]
            if m is not None and p.dtype == torch.float32:
                raise ValueError(f"masters[{i}]: a float32 parameter has none")
            t.master = _addr(m, p.shape, torch.float32, f"masters[{i}]", self.device) or None
            t.state_bits, t.weight_decay = self.state_bits[i], float(decay[i])
            own = [t.param, t.master] + self._set_state(t, i)
            own = [v for v in own if v] if t.n else []
            if len(set(own)) != len(own) or seen & set(own):
                raise ValueError(f"params[{i}]: a parameter, master or state is used twice")
            seen |= set(own)
        # the tensors with 8-bit states, as `moments` reads them
        self._eight = [i for i, b in enumerate(self.state_bits) if b == 8]
        self._eight_sizes = [self.params[i].numel() for i in self._eight]
        self._eight_list = (B.FnoAdamwTensor * max(1, len(self._eight)))(
            *[self._list[i] for i in self._eight])
        self.set_grads(grads)
        self.control: Optional[torch.Tensor] = None
        self._clipped = self._replayed = False  # a clip_grads awaits its step; one was captured
        if device_control:
            c = B.FnoAdamwControl(step=self._steps, lr_factor=1.0, grad_scale=1.0)
            self.control = torch.frombuffer(bytearray(bytes(c)), dtype=torch.uint8).to(self.device)
            self._norm = self.control[32:36].view(torch.float32)[0]
            self._factor = self.control[44:48].view(torch.float32)
            self._ws = torch.empty(B.fno_grad_norm_workspace_size(self._list, n),
                                   dtype=torch.uint8, device=self.device)
            self._control_at = self.control.data_ptr()
            self._ws_at, self._ws_bytes = self._ws.data_ptr(), self._ws.numel()
        # memory that torch handed out here, and the streams whose work it outlives
        self._made = [v for s in self.states for v in s.values()] if states is None else []
        if device_control:
            self._made += [self.control, self._ws]
        home = torch.cuda.current_stream(self.device)
        self._outlives = {home.cuda_stream}
        if self._made:
            home.synchronize()

    # -- construction ------------------------------------------------------------
    def _per_tensor(self, v, name):
        v = list(v)
        if len(v) != len(self.params):
            raise ValueError(f"{name}: {len(v)} entries for {len(self.params)} parameters")
        return v

    @staticmethod
    def make_masters(params: Sequence[torch.Tensor]) -> List[Optional[torch.Tensor]]:
        """float32 copies of the 16-bit parameters (None for float32 ones)."""
        return [None if p.dtype == torch.float32 else p.detach().float().clone() for p in params]

    @staticmethod
    def _zero_state(p, bits):
        z = dict(device=p.device)
        if bits == 32:
            return {k: torch.zeros(p.numel(), dtype=torch.float32, **z)
                    for k in ("exp_avg", "exp_avg_sq")}
        blocks = -(-p.numel() // B.FNO_ADAMW_BLOCK)
        return {"exp_avg": torch.zeros(p.numel(), dtype=torch.int8, **z),
                "exp_avg_sq": torch.zeros(p.numel(), dtype=torch.uint8, **z),
                "exp_avg_scale": torch.zeros(blocks, dtype=torch.float32, **z),
                "exp_avg_sq_scale": torch.zeros(blocks, dtype=torch.float32, **z)}

    def _set_state(self, t, i):
        s, n = self.states[i], t.n
        blocks = -(-n // B.FNO_ADAMW_BLOCK)
        want = ({"exp_avg": (n, torch.float32), "exp_avg_sq": (n, torch.float32)}
                if t.state_bits == 32 else
                {"exp_avg": (n, torch.int8), "exp_avg_sq": (n, torch.uint8),
                 "exp_avg_scale": (blocks, torch.float32),
                 "exp_avg_sq_scale": (blocks, torch.float32)})
        if set(s) != set(want):
            raise ValueError(f"states[{i}]: {sorted(s)}, expected {sorted(want)}")
        got = []
        for k, (count, dtype) in want.items():
            if s[k].numel() != count:
                raise ValueError(f"states[{i}].{k}: {s[k].numel()} elements, expected {count}")
            got.append(_addr(s[k], None, dtype, f"states[{i}].{k}", self.device) or None)
            setattr(t, k, got[-1])
        return got

    def set_grads(self, grads: Sequence[torch.Tensor]) -> None:
        """Takes `grads` as the gradients of the following steps."""
        grads = self._per_tensor(grads, "grads")
        addr = []
        for i, (p, g) in enumerate(zip(self.params, grads)):
            if g is None:
                raise ValueError(f"grads[{i}] is required")
            if g.dtype not in (torch.float32, p.dtype):
                raise ValueError(f"grads[{i}]: dtype {g.dtype}, expected float32 or {p.dtype}")
            addr.append(_addr(g, p.shape, None, f"grads[{i}]", self.device))
        for t, g, a in zip(self._list, grads, addr):
            t.grad, t.grad_dtype = a or None, DTYPE_CODES[g.dtype]
        self.grads = grads
        # what the addresses point to stays, whatever becomes of the tensors
        self._held = [v.untyped_storage() for v in self.params + self.grads + [
            m for m in self.masters if m is not None] + [
                v for s in self.states for v in s.values()]]

    # -- the calls ---------------------------------------------------------------
    def _on(self, stream):
        s = _stream_of(self.device, stream)
        if s not in self._outlives:
            for t in self._made:
                t.record_stream(_external(self.device, s))
            self._outlives.add(s)
        return s

    def clip_grads(self, max_norm: float = float("inf"), loss_scale: float = 1.0,
                   stream: Optional[int] = None) -> torch.Tensor:
        """The global norm of the gradients over `loss_scale` (returned, a
        scalar tensor that later calls overwrite), and the next step's
        gradient scale, step number and skip, on the device."""
        if self.control is None:
            raise ValueError("clip_grads needs device_control=True")
        if not loss_scale > 0:
            raise ValueError(f"loss_scale {loss_scale}, expected more than 0")
        s = self._on(stream)
        B.fno_grad_norm(self.desc, self._list, len(self.params), max_norm, 1.0 / loss_scale,
                        self._control_at, self._ws_at, self._ws_bytes, s)
        self._clipped = True
        if stream is None:
            self._replayed |= torch.cuda.is_current_stream_capturing()
        else:
            with torch.cuda.stream(_external(self.device, s)):
                self._replayed |= torch.cuda.is_current_stream_capturing()
        return self._norm

    def step(self, grads: Optional[Sequence[torch.Tensor]] = None, lr: Optional[float] = None,
             stream: Optional[int] = None) -> None:
        """One step (with device_control: the one that clip_grads prepared).
        lr: the learning rate from this step on."""
        if grads is not None:
            if self.control is not None:
                raise ValueError("set_grads before clip_grads: the clip reads the gradients")
            self.set_grads(grads)
        if self.control is not None and not (self._clipped or self._replayed):
            raise ValueError("with device_control every step follows a clip_grads of its own")
        if lr is not None:
            self.desc.lr = float(lr)
        s = self._on(stream)
        if self.control is not None:
            B.fno_adamw_step(self.desc, self._list, len(self.params), 0, self._control_at, s)
            self._clipped = False
        else:
            B.fno_adamw_step(self.desc, self._list, len(self.params), self._steps + 1, 0, s)
            self._steps += 1

    @property
    def steps(self) -> int:
        """Steps taken, those left out for gradients that are not finite not
        among them (with device_control read from the device, behind the
        current stream's work)."""
        return self._steps if self.control is None else self.read_control()["step"]

    def set_lr_factor(self, factor: float) -> None:
        """Multiplies lr on the device (a schedule for captured steps), in the
        order of the current stream."""
        if self.control is None:
            raise ValueError("set_lr_factor needs device_control=True")
        self._factor.fill_(float(factor))

    def read_control(self) -> Dict[str, float]:
        """The control block's fields (waits for the current stream)."""
        if self.control is None:
            raise ValueError("read_control needs device_control=True")
        c = B.FnoAdamwControl.from_buffer_copy(bytes(self.control.cpu().numpy()))
        return {k: getattr(c, k) for k, _ in c._fields_ if k not in ("arrived", "reserved")}

    def _all_fit(self, tensors, dtype) -> bool:
        """_addr's checks for the read-out's tensors, a check at a time over all
        of them: with a hundred small tensors the call is as long as its checks."""
        T = torch.Tensor
        return (all(issubclass(c, T) for c in set(map(type, tensors))) and
                list(map(T.numel, tensors)) == self._eight_sizes and
                set(map(_dtype_of, tensors)) == {dtype} and
                all(map(T.is_contiguous, tensors)) and
                set(map(T.get_device, tensors)) == {self.device.index})

    def moments(self, exp_avg: Optional[Sequence[torch.Tensor]] = None,
                exp_avg_sq: Optional[Sequence[torch.Tensor]] = None,
                dtype: torch.dtype = torch.float32, stream: Optional[int] = None):
        """The moments as values, two lists: 32-bit states themselves, 8-bit
        ones read out into tensors of the parameter's element count, made here
        in `dtype` or the caller's (then a full list of one type each; entries
        of 32-bit states stay as they are)."""
        eight = self._eight
        s = self._on(stream)
        outs, ptrs = [], []
        for k, given in (("exp_avg", exp_avg), ("exp_avg_sq", exp_avg_sq)):
            if given is None:
                if stream is not None:
                    raise ValueError(f"{k} is required where a stream is given")
                given = [torch.empty(self.params[i].numel(), dtype=dtype, device=self.device)
                         if b == 8 else self.states[i][k] for i, b in enumerate(self.state_bits)]
            given = self._per_tensor(given, k)
            outs.append(given)
            if not eight:
                continue
            if not ptrs:
                _addr(given[eight[0]], None, None, f"{k}[{eight[0]}]", self.device)
                dtype = getattr(given[eight[0]], "dtype", None)
                if dtype not in DTYPE_CODES:
                    raise ValueError(f"{k}: dtype {dtype}, expected float32, float16 or bfloat16")
            sub = [given[i] for i in eight]
            if not self._all_fit(sub, dtype):
                for i, n, t in zip(eight, self._eight_sizes, sub):
                    _addr(t, None, dtype, f"{k}[{i}]", self.device)
                    if t is None or t.numel() != n:
                        raise ValueError(f"{k}[{i}]: a tensor of {n} elements is required")
            addr = map(torch.Tensor.data_ptr, sub)
            addr = array("Q", addr)      # a third of the time of a ctypes array's making
            ptrs.append((ctypes.c_void_p * len(sub)).from_buffer(addr))
        if not eight:
            return outs[0], outs[1]
        B.fno_adamw_moments(self._eight_list, len(eight), DTYPE_CODES[dtype], ptrs[0], ptrs[1], s)
        return outs[0], outs[1]
