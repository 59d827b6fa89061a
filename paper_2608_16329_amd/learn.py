"""The learning operators over PyTorch-ROCm tensors (C ABI in include/mlip.h).

`Learner` wraps one mlip_learn context, `AdamW` one optimiser plan.  Every
tensor is the caller's, outputs too (but for the optimiser's moments); the
arithmetic runs in the library's HIP kernels, and there is no fallback.
"""
from __future__ import annotations

from typing import Optional

import numpy as np

from . import binding as b

_GATES = {"chosen": b.MLIP_GATES_CHOSEN, "all": b.MLIP_GATES_ALL}


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


class _OnStream:
    """A stream of its own that is put in order with the caller's current one."""

    def _bind(self, stream) -> None:
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the MLIP library runs only on the GPU")
        self.torch = torch
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self.device = self.stream.device
        self._raw = self.stream.cuda_stream
        # (the current stream's handle alone: a stream object for every call takes longer than the call's checks)
        self._current, self._device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        self._dtypes = {torch.float32: b.MLIP_F32, torch.bfloat16: b.MLIP_BF16}

    def _run(self, call, *args) -> None:
        """The call's work after what the current stream has, and what it gets next after the call's."""
        if self._device() != self.device.index:
            with self.torch.cuda.device(self.device):
                return self._run(call, *args)
        if self._current(self.device.index) == self._raw:
            call(*args)
            return
        current = self.torch.cuda.current_stream(self.device)
        self.stream.wait_stream(current)
        call(*args)
        current.wait_stream(self.stream)

    def _dense(self, t, name: str, dtype, *shape):
        if t.dtype is dtype and t.shape == shape and t.device == self.device and t.is_contiguous():
            return
        _need(t.device == self.device, f"{name} is on {t.device}, not {self.device}")
        _need(t.dtype == dtype, f"{name} is {t.dtype}, not {dtype}")
        _need(tuple(t.shape) == shape, f"{name} has shape {tuple(t.shape)}, not {shape}")
        _need(t.is_contiguous(), f"{name} is not contiguous")

    def _rows(self, t, name: str) -> int:
        """The values between the rows of a 2-d f32 or bf16 tensor."""
        if t.dim() == 2 and t.dtype in self._dtypes and t.device == self.device and t.is_contiguous():
            return t.shape[1]
        _need(t.device == self.device, f"{name} is on {t.device}, not {self.device}")
        _need(t.dtype in self._dtypes, f"{name} is {t.dtype}, not float32 or bfloat16")
        _need(t.dim() == 2, f"{name} has {t.dim()} dimensions, not 2")
        n, m = t.shape
        _need(m == 0 or t.stride(1) == 1 or m == 1, f"{name} has rows of values that are not next to each other")
        stride = t.stride(0) if n > 1 else m
        _need(stride >= m, f"{name} has rows that overlap")
        return stride


class Learner(_OnStream):
    """One mlip_learn context bound to a stream (default: the current one).

    A call made while another stream is current waits for that stream's work,
    and the work that stream gets afterwards waits for the call's."""

    def __init__(self, stream=None):
        self.ctx = None
        self._kept = {}
        self._bind(stream)
        with self.torch.cuda.device(self.device):
            self.ctx = b.mlip_learn_create(self.stream.cuda_stream)

    def close(self) -> None:
        if self.ctx:
            b.mlip_learn_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def memory_bytes(self) -> int:
        return b.mlip_learn_memory_bytes(self.ctx)

    # -- routing ---------------------------------------------------------------

    def _route_params(self, logits, top_k: int, kinds, allowed, gates_of: str):
        t = self.torch
        stride = self._rows(logits, "logits")
        n, n_experts = logits.shape
        _need(gates_of in _GATES, f"gates_of is {gates_of!r}, not 'chosen' or 'all'")
        _need((kinds is None) == (allowed is None), "kinds and allowed go together")
        if kinds is not None:
            self._dense(kinds, "kinds", t.int32, n)
            _need(allowed.dim() == 2, "allowed is not 2-d")
            self._dense(allowed, "allowed", t.uint8, allowed.shape[0], n_experts)
        return self._params(b.mlip_route_params, n_experts, top_k, 0 if kinds is None else allowed.shape[0],
                            _GATES[gates_of], self._dtypes[logits.dtype], max(stride, n_experts))

    def _params(self, kind, *values):
        """A parameter structure, kept: the same few come again in every step."""
        p = self._kept.get((kind, values))
        if p is None:
            if len(self._kept) >= 64:
                self._kept.clear()
            p = self._kept[(kind, values)] = kind(*values)
            if kind is b.mlip_heads_params:
                p.count = b.mlip_heads_weight_count(p)
        return p

    def route(self, logits, experts, gates, counts, loss, *, kinds=None, allowed=None, gates_of: str = "chosen") -> None:
        """Route the rows of `logits` (f32 or bf16 [n, E], rows may be apart) to
        their experts.shape[1] largest experts: experts int32 [n, k], gates f32
        [n, k], counts int32 [E + 1], loss f32 [1] (mlip_route).  kinds int32 [n]
        and allowed uint8 [kinds, E] say which experts a row may use."""
        t = self.torch
        _need(experts.dim() == 2, "experts is not 2-d")
        p = self._route_params(logits, experts.shape[1], kinds, allowed, gates_of)
        n, n_experts = logits.shape
        self._dense(experts, "experts", t.int32, n, p.top_k)
        self._dense(gates, "gates", t.float32, n, p.top_k)
        self._dense(counts, "counts", t.int32, n_experts + 1)
        self._dense(loss, "loss", t.float32, 1)
        self._run(b.mlip_route, self.ctx, p, n, _ptr(logits), _ptr(kinds), _ptr(allowed), _ptr(experts), _ptr(gates),
                  _ptr(counts), _ptr(loss))

    def route_backward(self, logits, experts, counts, dlogits, *, dgates=None, dloss=None, kinds=None, allowed=None,
                       gates_of: str = "chosen") -> None:
        """dlogits (the logits' type, [n, E]) of sum(dgates gates) + dloss loss,
        from what `route` was given and what it wrote (mlip_route_backward)."""
        t = self.torch
        _need(experts.dim() == 2, "experts is not 2-d")
        p = self._route_params(logits, experts.shape[1], kinds, allowed, gates_of)
        n, n_experts = logits.shape
        self._dense(experts, "experts", t.int32, n, p.top_k)
        self._dense(counts, "counts", t.int32, n_experts + 1)
        self._dense(dlogits, "dlogits", logits.dtype, n, n_experts)
        if dgates is not None:
            self._dense(dgates, "dgates", t.float32, n, p.top_k)
        if dloss is not None:
            self._dense(dloss, "dloss", t.float32, 1)
        self._run(b.mlip_route_backward, self.ctx, p, n, _ptr(logits), _ptr(kinds), _ptr(allowed), _ptr(experts), _ptr(counts),
                  _ptr(dgates), _ptr(dloss), _ptr(dlogits))

    def group(self, experts, offsets, order) -> None:
        """The entries of `experts` (int32, any shape: [n, k] or one species per
        atom) by expert: offsets int32 [E + 1], order int32 [entries] (mlip_group)."""
        t = self.torch
        m = experts.numel()
        _need(offsets.dim() == 1 and offsets.shape[0] >= 2, "offsets is not 1-d with at least 2 places")
        self._dense(experts, "experts", t.int32, *experts.shape)
        self._dense(offsets, "offsets", t.int32, offsets.shape[0])
        self._dense(order, "order", t.int32, m)
        self._run(b.mlip_group, self.ctx, m, offsets.shape[0] - 1, _ptr(experts), _ptr(offsets), _ptr(order))

    # -- energy heads ------------------------------------------------------------

    def heads(self, x, weights, offsets, order, *, hidden: int, top_k: int = 1, gates=None, denergy=None, energy=None,
              dx=None, dweights=None, dgates=None) -> None:
        """Energy heads `weights` (f32 [E, values], tables as in the potential's
        blob) over the rows of `x` (f32 or bf16 [n, width], rows may be apart),
        grouped by `group` (mlip_heads).  Outputs that are given are written:
        energy f32 [n] and, of sum(denergy energy), dx (x's type, [n, width]),
        dweights f32 [E, values] and dgates f32 [n, top_k]."""
        t = self.torch
        stride = self._rows(x, "x")
        n, width = x.shape
        _need(weights.dim() == 2, "weights is not 2-d")
        n_experts, values = weights.shape
        p = self._params(b.mlip_heads_params, n_experts, width, hidden, top_k, self._dtypes[x.dtype], max(stride, width))
        if p.count and values * n_experts != p.count:
            raise ValueError(f"weights has {values} values a head, {width} inputs and {hidden} layers need {p.count // n_experts}")
        self._dense(weights, "weights", t.float32, n_experts, values)
        self._dense(offsets, "offsets", t.int32, n_experts + 1)
        self._dense(order, "order", t.int32, n * top_k)
        for v, name, dtype, shape in ((gates, "gates", t.float32, (n, top_k)), (denergy, "denergy", t.float32, (n,)),
                                      (energy, "energy", t.float32, (n,)), (dx, "dx", x.dtype, (n, width)),
                                      (dweights, "dweights", t.float32, (n_experts, values)),
                                      (dgates, "dgates", t.float32, (n, top_k))):
            if v is not None:
                self._dense(v, name, dtype, *shape)
        self._run(b.mlip_heads, self.ctx, p, n, _ptr(x), _ptr(weights), _ptr(offsets), _ptr(order), _ptr(gates), _ptr(denergy),
                  _ptr(energy), _ptr(dx), _ptr(dweights), _ptr(dgates))


class AdamW(_OnStream):
    """AdamW over lists of contiguous tensors (f32 or bf16, gradients of either
    type in the same order), moments in 32 or 8 bits (mlip_adamw_step).

    The tensors' places are taken once: later gradients have to be written to
    the same tensors.  decay: one truth value a tensor, whether weight_decay
    applies (default: to those with two dimensions or more).  The moments are `m`
    and `v`, flat over the tensors back to back, with 8 bits codes beside
    `m_exp` and `v_exp`; they start as zeros, may be read, and are overwritten
    in place (opt.m.copy_(saved)): the plan holds their places.

    into: tensors that new parameters go to, like `params`; `new_m`, `new_v`
    (`new_m_exp`, `new_v_exp`) receive the new moments.  A step then changes
    nothing that it reads; `accept` makes what it wrote the next step's start
    and the old values the place to write to."""

    m, v, m_exp, v_exp, new_m, new_v, new_m_exp, new_v_exp = (
        property(lambda self, name=name: self._moments[name]) for name in
        ("m", "v", "m_exp", "v_exp", "new_m", "new_v", "new_m_exp", "new_v_exp"))

    def __init__(self, params, grads, *, bits: int = 32, decay=None, into=None, stream=None):
        self.plan = None
        self._bind(stream)
        t = self.torch
        params, grads = list(params), list(grads)
        into = None if into is None else list(into)
        decay = [p.dim() >= 2 for p in params] if decay is None else list(decay)
        _need(len(params) == len(grads) == len(decay) and len(params) == len(into if into is not None else params),
              "params, grads, into and decay differ in length")
        _need(bits in (8, 32), f"bits is {bits}, not 32 or 8")
        kinds, here = self._dtypes, self.device.index
        for k, (p, g) in enumerate(zip(params, grads)):
            if (p.dtype in kinds and g.dtype in kinds and p.get_device() == here == g.get_device() and p.shape == g.shape
                    and p.is_contiguous() and g.is_contiguous()):
                continue
            _need(p.dtype in kinds, f"params[{k}] is {p.dtype}, not float32 or bfloat16")
            _need(g.dtype in kinds, f"grads[{k}] is {g.dtype}, not float32 or bfloat16")
            self._dense(p, "a tensor of params", p.dtype, *p.shape)
            self._dense(g, "a tensor of grads", g.dtype, *p.shape)
        for p, q in zip(params, into or []):
            self._dense(q, "a tensor of into", p.dtype, *p.shape)
        table = np.zeros(len(params), b.ADAMW_TENSOR)
        table["param_dev"] = [p.data_ptr() for p in params]
        table["into_dev"] = [q.data_ptr() for q in into] if into is not None else 0
        table["grad_dev"] = [g.data_ptr() for g in grads]
        table["n"] = [p.numel() for p in params]
        table["param_dtype"] = [self._dtypes[p.dtype] for p in params]
        table["grad_dtype"] = [self._dtypes[g.dtype] for g in grads]
        table["decay"] = [bool(d) for d in decay]
        self._hold = (params, grads, into)
        self.bits, self._twice, self._reverse = bits, into is not None, False
        with t.cuda.device(self.device):
            self.plan = b.mlip_adamw_create(table, bits, self.stream.cuda_stream)
            n, blocks = b.mlip_adamw_state_count(self.plan)

            def zeros(m, dtype):
                return t.zeros(m, dtype=dtype, device=self.device)
            kind = t.float32 if bits == 32 else t.uint8
            held = {"m": (n, kind), "v": (n, kind)}
            if bits == 8:
                held.update(m_exp=(blocks, t.uint8), v_exp=(blocks, t.uint8))
            self._moments = dict.fromkeys(("m_exp", "v_exp", "new_m_exp", "new_v_exp"))
            for name, of in held.items():
                self._moments[name] = zeros(*of)
                self._moments["new_" + name] = zeros(*of) if self._twice else self._moments[name]
        # the moments' zeros are written by the current stream
        self.stream.wait_stream(t.cuda.current_stream(self.device))
        self._states()
        self._written = self._from

    def _states(self) -> None:
        self._from = b.mlip_adamw_state(_ptr(self.m), _ptr(self.v), _ptr(self.m_exp), _ptr(self.v_exp))
        self._into = b.mlip_adamw_state(_ptr(self.new_m), _ptr(self.new_v), _ptr(self.new_m_exp), _ptr(self.new_v_exp))

    def close(self) -> None:
        if self.plan:
            b.mlip_adamw_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def step(self, step: int, *, lr: float, beta1: float = 0.9, beta2: float = 0.99, eps: float = 1e-8,
             weight_decay: float = 0.0, grad_scale: float = 1.0, seed: int = 0) -> None:
        """Step number `step` (from 1).  seed: of the rounding of 8-bit moments, another one each step."""
        p = b.mlip_adamw_params(step, lr, beta1, beta2, eps, weight_decay, grad_scale, seed & 0xFFFFFFFF)
        self._run(b.mlip_adamw_step, self.plan, p, self._from, self._into, self._reverse)
        self._written = self._into

    def accept(self) -> None:
        """With `into`: the next step starts from what the last one wrote."""
        _need(self._twice, "accept() is for a plan with into")
        self._reverse = not self._reverse
        k = self._moments
        for name in ("m", "v", "m_exp", "v_exp"):
            k[name], k["new_" + name] = k["new_" + name], k[name]
        self._states()

    def moments(self, m, v) -> None:
        """The values that 8-bit moments as the last step wrote them stand for,
        accepted or not (before the first step: the start's), f32 [elements] each."""
        self._dense(m, "m", self.torch.float32, self.m.shape[0])
        self._dense(v, "v", self.torch.float32, self.m.shape[0])
        self._run(b.mlip_adamw_moments, self.plan, self._written, _ptr(m), _ptr(v))
