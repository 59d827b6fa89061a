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


def _at(r):
    """The places of a Rows8's codes and exponents."""
    if r is None:
        return None, None
    codes, exps, _, _ = r._held
    return codes.data_ptr(), exps.data_ptr()


class _OnStream:
    """A stream of its own that is put in order with the caller's current one."""

    def _bind(self, stream) -> None:
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the MLIP library runs only on the GPU")
        self.torch = torch
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self.device = self.stream.device
        self._index = self.device.index
        self._raw = self.stream.cuda_stream
        # (the current stream's handle alone: a stream object for every call takes longer than the call's checks)
        self._current, self._device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        self._dtypes = {torch.float32: b.MLIP_F32, torch.bfloat16: b.MLIP_BF16}

    def _run(self, call, *args) -> None:
        """The call's work after what the current stream has, and what it gets next after the call's."""
        if self._device() != self._index:
            with self.torch.cuda.device(self.device):
                return self._run(call, *args)
        if self._current(self._index) == self._raw:
            call(*args)
            return
        current = self.torch.cuda.current_stream(self.device)
        self.stream.wait_stream(current)
        call(*args)
        current.wait_stream(self.stream)

    def _dense(self, t, name: str, dtype, *shape):
        if t.dtype is dtype and t.shape == shape and t.get_device() == self._index and t.is_contiguous():
            return
        _need(t.device == self.device, f"{name} is on {t.device}, not {self.device}")
        _need(t.dtype == dtype, f"{name} is {t.dtype}, not {dtype}")
        _need(tuple(t.shape) == shape, f"{name} has shape {tuple(t.shape)}, not {shape}")
        _need(t.is_contiguous(), f"{name} is not contiguous")

    def _matrix(self, t, name: str):
        """Rows, values of a row, values between rows and mlip_dtype of a 2-d f32 or bf16 tensor."""
        kind = self._dtypes.get(t.dtype)
        if kind is not None and t.get_device() == self._index and t.is_contiguous():
            shape = t.shape
            if len(shape) == 2:
                n, m = shape
                return n, m, m, kind
        stride = self._rows(t, name)
        return *t.shape, stride, kind

    def _rows(self, t, name: str) -> int:
        """The values between the rows of a 2-d f32 or bf16 tensor."""
        if t.dtype in self._dtypes and t.get_device() == self._index and t.is_contiguous():
            shape = t.shape
            if len(shape) == 2:
                return shape[1]
        if t.get_device() != self._index:
            raise ValueError(f"{name} is on {t.device}, not {self.device}")
        if t.dtype not in self._dtypes:
            raise ValueError(f"{name} is {t.dtype}, not float32 or bfloat16")
        if t.dim() != 2:
            raise ValueError(f"{name} has {t.dim()} dimensions, not 2")
        n, m = t.shape
        if m > 1 and t.stride(1) != 1:
            raise ValueError(f"{name} has rows of values that are not next to each other")
        stride = t.stride(0) if n > 1 else m
        if stride < m:
            raise ValueError(f"{name} has rows that overlap")
        return stride


def _bytes(t, name: str, *shape):
    _need(t.element_size() == 1 and not t.is_floating_point(), f"{name} is {t.dtype}, not uint8")
    _need(tuple(t.shape) == shape and t.is_contiguous(), f"{name} has shape {tuple(t.shape)}, not {shape}, or is not contiguous")
    return t


class Rows8:
    """Places for `rows` rows of `width` values in 8 bits (mlip_pack8): codes uint8
    [rows, width rounded up to 128s], exps uint8 [rows, blocks of 128 rounded up to
    fours], allocated here unless given (both, contiguous)."""

    codes, exps, rows, width = (property(lambda self, k=k: self._held[k]) for k in range(4))

    def __init__(self, rows: int, width: int, *, codes=None, exps=None, device=None):
        import torch
        _need(rows >= 0, f"rows is {rows}")
        _need(1 <= width <= 65536, f"width is {width}, not in 1..65536")
        _need((codes is None) == (exps is None), "codes and exps go together")
        shapes = (rows, b.mlip_row8_codes(width)), (rows, b.mlip_row8_exps(width))
        if codes is None:
            device = torch.device("cuda") if device is None else device
            codes, exps = (torch.empty(s, dtype=torch.uint8, device=device) for s in shapes)
        _need(codes.device == exps.device, f"codes are on {codes.device}, exps on {exps.device}")
        self._held = _bytes(codes, "codes", *shapes[0]), _bytes(exps, "exps", *shapes[1]), rows, width


class Weights8:
    """Places for `experts` matrices [outputs, inputs] in 8 bits (mlip_pack8_weights):
    codes and exps, and, with `transposed`, t_codes and t_exps of their transposes,
    which gradients in x need (otherwise None)."""

    codes, exps, t_codes, t_exps, experts, outputs, inputs = (property(lambda self, k=k: self._held[k]) for k in range(7))

    def __init__(self, experts: int, outputs: int, inputs: int, *, transposed: bool = True, device=None):
        import torch
        _need(1 <= experts <= 256, f"experts is {experts}, not in 1..256")
        _need(1 <= outputs <= 65536 and 1 <= inputs <= 65536, f"{outputs} outputs and {inputs} inputs are not in 1..65536")
        device = torch.device("cuda") if device is None else device

        def places(rows, width):
            return (torch.empty((experts, rows, b.mlip_row8_codes(width)), dtype=torch.uint8, device=device),
                    torch.empty((experts, (rows + 127) // 128, b.mlip_row8_exps(width)), dtype=torch.uint8, device=device))
        self._held = (*places(outputs, inputs), *(places(inputs, outputs) if transposed else (None, None)), experts, outputs, inputs)


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


    # -- wide layers of experts ----------------------------------------------------

    def _packed(self, r: Rows8, name: str, rows: int, width: int) -> None:
        codes, _, has, wide = r._held
        if has == rows and wide == width and codes.get_device() == self._index:
            return
        if codes.device != self.device:
            raise ValueError(f"{name} is on {codes.device}, not {self.device}")
        raise ValueError(f"{name} has {has} rows of {wide} values, not {rows} of {width}")

    def _expert_offsets(self, offsets, experts: int) -> None:
        if offsets is None:
            if experts != 1:
                raise ValueError(f"{experts} experts need offsets")
        else:
            self._dense(offsets, "offsets", self.torch.int32, experts + 1)

    def sort(self, x, offsets, order, xs, places) -> None:
        """The rows of `x` (f32 or bf16 [n, width], rows may be apart) in the order
        that `group` found: xs (x's type) [n k, width], rows of entries without an
        expert left as they are (None: places alone); places int32 [n, k], where each
        entry stands or -1 (mlip_sort).  The gradient in x is `combine` of xs' gradient."""
        t = self.torch
        n, width, stride, kind = self._matrix(x, "x")
        _need(places.dim() == 2, "places is not 2-d")
        _need(offsets.dim() == 1 and offsets.shape[0] >= 2, "offsets is not 1-d with at least 2 places")
        top_k = places.shape[1]
        self._dense(places, "places", t.int32, n, top_k)
        self._dense(offsets, "offsets", t.int32, offsets.shape[0])
        self._dense(order, "order", t.int32, n * top_k)
        if xs is not None:
            self._dense(xs, "xs", x.dtype, n * top_k, width)
        p = self._params(b.mlip_rows_params, offsets.shape[0] - 1, top_k, width, kind)
        self._run(b.mlip_sort, self.ctx, p, n, _ptr(x), stride, _ptr(offsets), _ptr(order), _ptr(xs), _ptr(places))

    def combine(self, y, places, out, *, gates=None) -> None:
        """out (y's type, [n, width]): each row's sum of the rows of `y` ([n k, width],
        rows may be apart) at its `places`, times its gates f32 [n, k] (mlip_combine)."""
        t = self.torch
        m, width, stride, kind = self._matrix(y, "y")
        _need(places.dim() == 2, "places is not 2-d")
        n, top_k = places.shape
        if m != n * top_k:
            raise ValueError(f"y has {m} rows, not {n} x {top_k}")
        self._dense(places, "places", t.int32, n, top_k)
        self._dense(out, "out", y.dtype, n, width)
        if gates is not None:
            self._dense(gates, "gates", t.float32, n, top_k)
        p = self._params(b.mlip_rows_params, 1, top_k, width, kind)
        self._run(b.mlip_combine, self.ctx, p, n, _ptr(y), stride, _ptr(places), _ptr(gates), _ptr(out))

    def combine_backward(self, dout, y, places, dy, *, gates=None, dgates=None) -> None:
        """Of sum(dout out): dy (dout's type, [n k, width], rows that are no place left as
        they are) and, where it is given, dgates f32 [n, k], which alone needs `y`
        (otherwise None may stand there) (mlip_combine_backward)."""
        t = self.torch
        rows, width, stride, kind = self._matrix(dout, "dout")
        _need(places.dim() == 2, "places is not 2-d")
        n, top_k = places.shape
        if rows != n:
            raise ValueError(f"dout has {rows} rows, not {n}")
        self._dense(places, "places", t.int32, n, top_k)
        self._dense(dy, "dy", dout.dtype, n * top_k, width)
        if gates is not None:
            self._dense(gates, "gates", t.float32, n, top_k)
        y_stride = width
        if dgates is not None:
            _need(y is not None, "dgates needs y")
            self._dense(dgates, "dgates", t.float32, n, top_k)
            y_stride = self._rows(y, "y")
            if not (y.dtype == dout.dtype and tuple(y.shape) == (n * top_k, width)):
                raise ValueError(f"y is {y.dtype} {tuple(y.shape)}, not {dout.dtype} {(n * top_k, width)}")
        p = self._params(b.mlip_rows_params, 1, top_k, width, kind)
        self._run(b.mlip_combine_backward, self.ctx, p, n, _ptr(dout), stride, _ptr(y) if dgates is not None else None,
                  y_stride, _ptr(places), _ptr(gates), _ptr(dy), _ptr(dgates))

    def pack8(self, x, rows8: Rows8, *, offsets=None, order=None, top_k: int = 1) -> None:
        """The rows of `x` (f32 or bf16 [n, width], rows may be apart) in 8 bits, or,
        with what `group` wrote, their n top_k entries in the experts' order, rows of
        entries without an expert left as they are (mlip_pack8)."""
        t = self.torch
        n, width, stride, kind = self._matrix(x, "x")
        _need((offsets is None) == (order is None), "offsets and order go together")
        _need(order is not None or top_k == 1, "top_k is 1 without an order")
        experts = 1
        if offsets is not None:
            _need(offsets.dim() == 1 and offsets.shape[0] >= 2, "offsets is not 1-d with at least 2 places")
            experts = offsets.shape[0] - 1
            self._dense(offsets, "offsets", t.int32, experts + 1)
            self._dense(order, "order", t.int32, n * top_k)
        self._packed(rows8, "rows8", n * top_k, width)
        p = self._params(b.mlip_rows_params, experts, top_k, width, kind)
        self._run(b.mlip_pack8, self.ctx, p, n, x.data_ptr(), stride, _ptr(offsets), _ptr(order), *_at(rows8))

    def unpack8(self, rows8: Rows8, x) -> None:
        """The values of rows in 8 bits into x, f32 or bf16 [rows, width] (mlip_unpack8)."""
        if x.dtype not in self._dtypes:
            raise ValueError(f"x is {x.dtype}, not float32 or bfloat16")
        _, _, n, width = rows8._held
        self._packed(rows8, "rows8", n, width)
        self._dense(x, "x", x.dtype, n, width)
        p = self._params(b.mlip_rows_params, 1, 1, width, self._dtypes[x.dtype])
        self._run(b.mlip_unpack8, self.ctx, p, n, *_at(rows8), x.data_ptr())

    def _matrices(self, w8: Weights8, name: str) -> None:
        codes = w8._held[0]
        if codes.get_device() != self._index:
            raise ValueError(f"{name} is on {codes.device}, not {self.device}")

    def pack8_weights(self, w, w8: Weights8) -> None:
        """Matrices (f32 or bf16 [experts, outputs, inputs]) in 8 bits, and their
        transposes where w8 has places for them (mlip_pack8_weights)."""
        if w.dtype not in self._dtypes:
            raise ValueError(f"w is {w.dtype}, not float32 or bfloat16")
        self._matrices(w8, "w8")
        self._dense(w, "w", w.dtype, w8.experts, w8.outputs, w8.inputs)
        p = self._params(b.mlip_product8_params, w8.experts, w8.inputs, w8.outputs, self._dtypes[w.dtype])
        self._run(b.mlip_pack8_weights, self.ctx, p, _ptr(w), _ptr(w8.codes), _ptr(w8.exps), _ptr(w8.t_codes),
                  _ptr(w8.t_exps))

    def product8(self, x8: Rows8, w8: Weights8, y, *, offsets=None, bias=None, transposed: bool = False) -> None:
        """y (f32 or bf16 [m, outputs]): each packed row's product with its expert's
        matrix, plus bias f32 [experts, outputs]; offsets int32 [experts + 1] as `group`
        writes them for rows in the experts' order (one expert needs none), rows from the
        last one on left as they are.  transposed: with the transposes, [m, inputs] from
        rows of `outputs` values, the gradient in x (mlip_product8)."""
        t = self.torch
        if y.dtype not in self._dtypes:
            raise ValueError(f"y is {y.dtype}, not float32 or bfloat16")
        codes, exps, t_codes, t_exps, experts, n_out, n_in = w8._held
        if transposed:
            _need(t_codes is not None, "w8 has no transposes")
            codes, exps, n_out, n_in = t_codes, t_exps, n_in, n_out
        self._matrices(w8, "w8")
        m = x8._held[2]
        self._packed(x8, "x8", m, n_in)
        self._dense(y, "y", y.dtype, m, n_out)
        self._expert_offsets(offsets, experts)
        if bias is not None:
            self._dense(bias, "bias", t.float32, experts, n_out)
        p = self._params(b.mlip_product8_params, experts, n_in, n_out, self._dtypes[y.dtype])
        self._run(b.mlip_product8, self.ctx, p, m, *_at(x8), codes.data_ptr(), exps.data_ptr(), _ptr(offsets), _ptr(bias),
                  y.data_ptr())

    def product8_weights(self, dy8: Rows8, x8: Rows8, dweights, *, offsets=None, dbias=None) -> None:
        """The matrices' gradients, f32 [experts, outputs, inputs], and dbias f32
        [experts, outputs], from packed rows (mlip_product8_weights)."""
        t = self.torch
        _need(dweights.dim() == 3, "dweights is not 3-d")
        experts, n_out, n_in = dweights.shape
        m = x8._held[2]
        self._packed(x8, "x8", m, n_in)
        self._packed(dy8, "dy8", m, n_out)
        self._dense(dweights, "dweights", t.float32, experts, n_out, n_in)
        self._expert_offsets(offsets, experts)
        if dbias is not None:
            self._dense(dbias, "dbias", t.float32, experts, n_out)
        p = self._params(b.mlip_product8_params, experts, n_in, n_out, b.MLIP_F32)
        self._run(b.mlip_product8_weights, self.ctx, p, m, *_at(dy8), *_at(x8), _ptr(offsets), dweights.data_ptr(),
                  _ptr(dbias))

    def activate8(self, z, kept: Optional[Rows8] = None, h=None, *, h8: Optional[Rows8] = None, residual=None) -> None:
        """h = residual + silu(z) of the rows of `z` (f32 or bf16 [n, width], rows may be
        apart, residual too) into h (z's type) and, packed, h8; z itself, packed, into
        `kept` for the backward pass (mlip_activate8)."""
        n, width, stride, kind = self._matrix(z, "z")
        residual_stride = width
        if residual is not None:
            residual_stride = self._rows(residual, "residual")
            if not (residual.dtype == z.dtype and residual.shape == z.shape):
                raise ValueError(f"residual is {residual.dtype} {tuple(residual.shape)}, not {z.dtype} {tuple(z.shape)}")
        if h is not None:
            self._dense(h, "h", z.dtype, n, width)
        if kept is not None:
            self._packed(kept, "kept", n, width)
        if h8 is not None:
            self._packed(h8, "h8", n, width)
        p = self._params(b.mlip_rows_params, 1, 1, width, kind)
        self._run(b.mlip_activate8, self.ctx, p, n, z.data_ptr(), stride, _ptr(residual), residual_stride, _ptr(h), *_at(h8),
                  *_at(kept))

    def activate8_backward(self, kept: Rows8, dh, dz=None, *, dz8: Optional[Rows8] = None) -> None:
        """dz = dh silu'(z) with the z that was kept, into dz (dh's type, [n, width]) and,
        packed, dz8; dh's rows may be apart (mlip_activate8_backward)."""
        n, width, stride, kind = self._matrix(dh, "dh")
        self._packed(kept, "kept", n, width)
        if dz is not None:
            self._dense(dz, "dz", dh.dtype, n, width)
        if dz8 is not None:
            self._packed(dz8, "dz8", n, width)
        p = self._params(b.mlip_rows_params, 1, 1, width, kind)
        self._run(b.mlip_activate8_backward, self.ctx, p, n, *_at(kept), dh.data_ptr(), stride, _ptr(dz), *_at(dz8))


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
