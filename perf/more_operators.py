"""Timed cases of the operators that layers of experts wider than the energy heads
are made of: rows brought into the experts' order and back with weights, rows
and weights in 8 bits with a power of two for every 128 values, products of them
over grouped rows, and activations that keep 8 bits for the backward pass.  Each
case has a plain form in elementary torch operations and a definition in 64 bits.
"""
import math

import torch

own = False

F32, BF16 = "float32", "bfloat16"
BLOCK = 128         # values that share a power of two


def _mix(name, **over):
    c = dict(name=name, op="mix", rows=1, width=128, experts=4, top_k=1, dtype=F32, weights=True, skew=0.0, empty=0.0, spare=0,
             train=True)
    c.update(over)
    return c


def _pack(name, **over):
    c = dict(name=name, op="pack", rows=1, width=128, experts=4, top_k=1, dtype=F32, sort=True, skew=0.0, empty=0.0, spare=0)
    c.update(over)
    return c


def _layer(name, **over):
    c = dict(name=name, op="layer", rows=1, inputs=128, outputs=128, experts=1, dtype=BF16, bias=True, skew=0.0, empty=0.0,
             train=False)
    c.update(over)
    return c


def _silu(name, **over):
    c = dict(name=name, op="silu", rows=1, width=128, dtype=BF16, residual=False, spare=0)
    c.update(over)
    return c


def listed():
    return [
        # one new atom, two of eight experts: launches and latency
        _mix("mix-one-atom", experts=8, top_k=2, train=False),
        # a ragged batch: three experts an atom, some of them nobody's, rows of
        # an odd width that lie further apart than they are long
        _mix("mix-ragged-33k", rows=32767, width=385, experts=29, top_k=3, skew=1.0, empty=0.03, spare=3),
        # the largest training batch of wide rows in 16 bits
        _mix("mix-train-262k-bf16", rows=262144, width=1024, experts=16, top_k=2, dtype=BF16, skew=0.5),
        # descriptors of a small batch, brought into order on the way
        _pack("pack-ragged-5k", rows=4999, width=193, experts=6, empty=0.02, skew=1.0, spare=2),
        # two entries for each of many rows
        _pack("pack-131k-bf16", rows=131072, width=1024, experts=16, top_k=2, dtype=BF16),
        # one row through one wide layer: the weights' bytes and latency
        _layer("layer-one-row", inputs=1024, outputs=1024),
        # evaluation of a ragged batch, eight experts
        _layer("layer-serve-4k", rows=4093, inputs=1024, outputs=2048, experts=8, skew=1.0, empty=0.02),
        # first layer of experts over descriptors, odd sizes, 32 bits outside
        _layer("layer-train-odd-30k", rows=30001, inputs=385, outputs=321, experts=6, dtype=F32, skew=0.5, empty=0.01, train=True),
        # a training step of the widest layer
        _layer("layer-train-65k", rows=65536, inputs=1024, outputs=4096, experts=8, skew=0.5, train=True),
        # activations of one small cell
        _silu("silu-cell-108", rows=108, width=64, dtype=F32),
        # an odd width, residual
        _silu("silu-odd-30k", rows=30001, width=321, dtype=F32, residual=True, spare=3),
        # a large batch of the widest layer
        _silu("silu-65k", rows=65536, width=4096),
    ]


def _log(rng, low, high):
    return round(math.exp(rng.uniform(math.log(low), math.log(high))))


def _width(rng, high):
    """Multiples of 64 and anything else."""
    w = _log(rng, 1, high)
    return min(high, (w + 63) // 64 * 64) if rng.random() < 0.5 else w


def draw(rng):
    """Another case of the same ranges, at most as much work as the largest listed one of its operator."""
    op = rng.choice(["mix", "pack", "layer", "layer", "silu"])
    spare = rng.choice([0, 0, rng.randint(1, 9)])
    empty = rng.choice([0.0, rng.uniform(0.0, 0.2)])
    skew = rng.choice([0.0, rng.uniform(0.0, 2.0)])
    if op in ("mix", "pack"):
        experts = _log(rng, 1, 256)
        top_k = rng.choice([1, 2, rng.randint(1, min(experts, 8))])
        top_k = min(top_k, experts)
        width = _width(rng, 4096)
        dtype = rng.choice([F32, BF16])
        most = (262144 if op == "mix" else 131072) * 2 * 1024 // (width * top_k * (2 if dtype == F32 else 1))
        rows = _log(rng, 1, max(1, min(524288 // top_k, most)))
        if op == "mix":
            c = _mix("", rows=rows, width=width, experts=experts, top_k=top_k, dtype=dtype, skew=skew, empty=empty, spare=spare,
                     weights=rng.random() < 0.8, train=rng.random() < 0.7)
        else:
            sort = rng.random() < 0.6
            c = _pack("", rows=rows, width=width, experts=experts, top_k=top_k if sort else 1, dtype=dtype, sort=sort, skew=skew,
                      empty=empty if sort else 0.0, spare=spare)
    elif op == "layer":
        experts = rng.choice([1, _log(rng, 1, 64)])
        inputs, outputs = _width(rng, 4096), _width(rng, 4096)
        while inputs * outputs * experts > 8 * 1024 * 4096:
            experts = (experts + 1) // 2
            if experts == 1:
                break
        most = 65536 * 1024 * 4096 // (inputs * outputs)
        c = _layer("", inputs=inputs, outputs=outputs, experts=experts, rows=_log(rng, 1, max(1, min(262144, most, 2 ** 28 // max(inputs, outputs)))),
                   dtype=rng.choice([F32, BF16, BF16]), bias=rng.random() < 0.7, skew=skew, empty=empty if experts > 1 else 0.0,
                   train=rng.random() < 0.5)
    else:
        width = _width(rng, 4096)
        c = _silu("", width=width, rows=_log(rng, 1, min(524288, 65536 * 4096 // (2 * width))), dtype=rng.choice([F32, BF16]),
                  residual=rng.random() < 0.5, spare=spare)
    del c["name"]
    return c


def _size(c):
    return 2 if c["dtype"] == BF16 else 4


def work(case):
    c, s = case, _size(case)
    n = c["rows"]
    if c["op"] == "mix":
        w, m = c["width"], round(n * c["top_k"] * (1 - c["empty"]))
        ids, g = 4 * n * c["top_k"], 4 * n * c["top_k"] if c["weights"] else 0
        # rows in, in order out, places; in order in, rows out
        b = (n + m) * w * s + 2 * ids + (m + n) * w * s + ids + g
        f = 2 * m * w
        if c["train"]:
            # the outputs' gradient and the experts' outputs in, their gradient out; and back to rows
            b += (n + m) * w * s + (m * w * s if c["weights"] else 0) + 2 * g + ids + (m + n) * w * s + ids
            f += (4 if c["weights"] else 1) * m * w
        return {"bytes": b, "flops": f}
    if c["op"] == "pack":
        w, m = c["width"], round(n * c["top_k"] * (1 - c["empty"]))
        packed = m * (w + (w + BLOCK - 1) // BLOCK)
        return {"bytes": n * w * s + (4 * n * c["top_k"] if c["sort"] else 0) + 2 * packed + m * w * s, "flops": 3 * m * w}
    if c["op"] == "layer":
        K, N, E, m = c["inputs"], c["outputs"], c["experts"], round(n * (1 - c["empty"]))
        bias = 4 * E * N if c["bias"] else 0
        used = min(E, m)
        if not c["train"]:
            return {"bytes": m * (K + N) * s + used * N * K + bias, "flops": 2 * m * K * N}
        # weights in, their gradient out; rows and outputs' gradient in, outputs and rows' gradient out
        return {"bytes": 2 * m * (K + N) * s + 8 * E * N * K + 2 * bias, "flops": 6 * m * K * N}
    w = c["width"]
    kept = n * (w + (w + BLOCK - 1) // BLOCK)
    return {"bytes": n * w * s * (5 if c["residual"] else 4) + 2 * kept, "flops": 16 * n * w}


# ---- inputs ------------------------------------------------------------------

def _rng(seed, device):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g


def _device():
    return torch.device("cuda:0" if torch.cuda.is_available() else "cpu")


def _spaced(t, spare):
    """The same values in rows that are `spare` elements further apart than they are long."""
    if not spare:
        return t
    wide = torch.full((t.shape[0], t.shape[1] + spare), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _values(g, dev, n, width, dtype):
    """Activations: rows of different size, some with nothing in them."""
    x = torch.randn((n, width), generator=g, device=dev)
    size = torch.exp(torch.randn((n, 1), generator=g, device=dev))
    x.mul_(torch.where(torch.rand((n, 1), generator=g, device=dev) < 0.01, 0.0, size))
    return x.to(getattr(torch, dtype))


def _grouped(c, g, dev):
    """Experts of each row (-1: none) with shares that are equal or fall off, and their grouping."""
    n, E, K = c["rows"], c["experts"], c.get("top_k", 1)
    share = torch.exp(-c["skew"] * torch.arange(E, device=dev, dtype=torch.float32) / max(1, E - 1) * 3.0)
    noise = -torch.log(-torch.log(torch.rand((n, E), generator=g, device=dev).clamp_(1e-7, 1 - 1e-7)))
    experts = torch.topk(share.log() + noise, K, dim=1).indices.to(torch.int32)
    if c["empty"]:
        experts[torch.rand((n, K), generator=g, device=dev) < c["empty"]] = -1
    flat = experts.reshape(-1).long()
    key = torch.where(flat >= 0, flat, E)
    order = torch.sort(key, stable=True).indices
    counts = torch.bincount(key, minlength=E + 1)
    offsets = torch.cat([counts.new_zeros(1), counts[:E].cumsum(0)])
    return offsets.to(torch.int32), order.to(torch.int32)


def _mix_inputs(c, g, dev):
    n, K, w = c["rows"], c["top_k"], c["width"]
    kind = getattr(torch, c["dtype"])
    offsets, order = _grouped(c, g, dev)
    s = dict(case=c, offsets=offsets, order=order, x=_spaced(_values(g, dev, n, w, c["dtype"]), c["spare"]),
             y=_spaced(_values(g, dev, n * K, w, c["dtype"]), c["spare"]), gates=None)
    if c["weights"]:
        s["gates"] = torch.softmax(torch.randn((n, K), generator=g, device=dev), dim=1)
    if c["train"]:
        s["dout"] = _values(g, dev, n, w, c["dtype"])
        s["dxs"] = _values(g, dev, n * K, w, c["dtype"])
    if own:
        from paper_2608_16329_amd import Learner
        s["learner"] = Learner()
        s["places"] = torch.empty((n, K), dtype=torch.int32, device=dev)
        # rows behind the last expert's stay as they are
        out = dict(xs=torch.zeros((n * K, w), dtype=kind, device=dev), out=torch.empty((n, w), dtype=kind, device=dev))
        if c["train"]:
            out["dy"] = torch.zeros((n * K, w), dtype=kind, device=dev)
            out["dx"] = torch.empty((n, w), dtype=kind, device=dev)
            if c["weights"]:
                out["dgates"] = torch.empty((n, K), device=dev)
        s["out"] = out
    return s


def _pack_inputs(c, g, dev):
    n, w = c["rows"], c["width"]
    s = dict(case=c, offsets=None, order=None, x=_spaced(_values(g, dev, n, w, c["dtype"]), c["spare"]))
    if c["sort"]:
        s["offsets"], s["order"] = _grouped(c, g, dev)
    if own:
        from paper_2608_16329_amd import Learner, Rows8
        m = n * c["top_k"]
        s["learner"], s["rows8"] = Learner(), Rows8(m, w, device=dev)
        s["rows8"].codes.zero_()
        s["rows8"].exps.zero_()
        s["values"] = torch.empty((m, w), dtype=s["x"].dtype, device=dev)
    return s


def _layer_inputs(c, g, dev):
    n, K, N, E = c["rows"], c["inputs"], c["outputs"], c["experts"]
    kind = getattr(torch, c["dtype"])
    s = dict(case=c, x=_values(g, dev, n, K, c["dtype"]), weights=torch.randn((E, N, K), generator=g, device=dev) / math.sqrt(K),
             offsets=None, bias=None)
    if E > 1:
        # rows that stand in the experts' order already
        s["offsets"] = _grouped(c, g, dev)[0]
    if c["bias"]:
        s["bias"] = torch.randn((E, N), generator=g, device=dev)
    if c["train"]:
        s["dy"] = _values(g, dev, n, N, c["dtype"])
    if own:
        from paper_2608_16329_amd import Learner, Rows8, Weights8
        s["learner"] = Learner()
        s["w8"] = Weights8(E, N, K, transposed=c["train"], device=dev)
        s["x8"] = Rows8(n, K, device=dev)
        out = dict(y=torch.zeros((n, N), dtype=kind, device=dev))
        if c["train"]:
            s["dy8"] = Rows8(n, N, device=dev)
            out["dx"] = torch.zeros((n, K), dtype=kind, device=dev)
            out["dweights"] = torch.empty((E, N, K), device=dev)
            if c["bias"]:
                out["dbias"] = torch.empty((E, N), device=dev)
        else:
            # weights that are learned already are packed once
            s["learner"].pack8_weights(s["weights"], s["w8"])
        s["out"] = out
    elif not c["train"]:
        s["weights_held"] = _held_weights(s["weights"])
    return s


def _silu_inputs(c, g, dev):
    n, w = c["rows"], c["width"]
    z = torch.randn((n, w), generator=g, device=dev).mul_(2.0).to(getattr(torch, c["dtype"]))
    s = dict(case=c, z=_spaced(z, c["spare"]), dh=_spaced(_values(g, dev, n, w, c["dtype"]), c["spare"]), residual=None)
    if c["residual"]:
        s["residual"] = _values(g, dev, n, w, c["dtype"])
    if own:
        from paper_2608_16329_amd import Learner, Rows8
        s["learner"], s["kept"] = Learner(), Rows8(n, w, device=dev)
        s["out"] = dict(h=torch.empty((n, w), dtype=z.dtype, device=dev), dz=torch.empty((n, w), dtype=z.dtype, device=dev))
    return s


def prepare(case, seed):
    dev = _device()
    g = _rng(seed, dev)
    return {"mix": _mix_inputs, "pack": _pack_inputs, "layer": _layer_inputs, "silu": _silu_inputs}[case["op"]](dict(case), g, dev)


# ---- one pass ----------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if op == "mix":
        return _run_mix(state) if own else _plain_mix(state)
    if op == "pack":
        return _run_pack(state) if own else _plain_pack(state)
    if op == "layer":
        return _run_layer(state) if own else _plain_layer(state)
    return _run_silu(state) if own else _plain_silu(state)


def _run_mix(s):
    c, L, out, places = s["case"], s["learner"], s["out"], s["places"]
    L.sort(s["x"], s["offsets"], s["order"], out["xs"], places)
    L.combine(s["y"], places, out["out"], gates=s["gates"])
    if c["train"]:
        L.combine_backward(s["dout"], s["y"], places, out["dy"], gates=s["gates"], dgates=out.get("dgates"))
        L.combine(s["dxs"], places, out["dx"])
    return out


def _run_pack(s):
    L, c = s["learner"], s["case"]
    L.pack8(s["x"], s["rows8"], offsets=s["offsets"], order=s["order"], top_k=c["top_k"])
    L.unpack8(s["rows8"], s["values"])
    return s["values"]


def _run_layer(s):
    c, L, out = s["case"], s["learner"], s["out"]
    if c["train"]:
        L.pack8_weights(s["weights"], s["w8"])
    L.pack8(s["x"], s["x8"])
    L.product8(s["x8"], s["w8"], out["y"], offsets=s["offsets"], bias=s["bias"])
    if c["train"]:
        L.pack8(s["dy"], s["dy8"])
        L.product8(s["dy8"], s["w8"], out["dx"], offsets=s["offsets"], transposed=True)
        L.product8_weights(s["dy8"], s["x8"], out["dweights"], offsets=s["offsets"], dbias=out.get("dbias"))
    return out


def _run_silu(s):
    L, out = s["learner"], s["out"]
    L.activate8(s["z"], s["kept"], out["h"], residual=s["residual"])
    L.activate8_backward(s["kept"], s["dh"], out["dz"])
    return out


# ---- plain forms -------------------------------------------------------------

def _pow2(e):
    """2^e in float32, -126 <= e <= 127, from its bits."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _exponent(size):
    """The exponent of a block whose largest value is `size`: all of it fits in codes up to 448."""
    bits = size.view(torch.int32)
    return ((bits >> 23) - 135 + ((bits & 0x7FFFFF) > 0x600000).to(torch.int32)).clamp(-100, 120)


def _rounded(t, e):
    """t, in 8 bits relative to 2^e: 4 exponent and 3 mantissa bits beside the sign, to nearest even."""
    fine = t.isfinite()
    y = torch.where(fine, t, 0.0) * _pow2(-e)
    ey = ((y.abs().view(torch.int32) >> 23) - 127).clamp(min=-6)
    return torch.where(fine, torch.round(y * _pow2(3 - ey)) * _pow2(ey - 3) * _pow2(e), math.nan)


def _held(x):
    """The values that rows in 8 bits stand for, float32."""
    n, w = x.shape
    nb = (w + BLOCK - 1) // BLOCK
    t = x.float()
    if w != nb * BLOCK:
        t = torch.cat([t, t.new_zeros((n, nb * BLOCK - w))], 1)
    t = t.reshape(n, nb, BLOCK)
    size = torch.where(t.isfinite(), t.abs(), 0.0).amax(2, keepdim=True)
    return _rounded(t, _exponent(size)).reshape(n, nb * BLOCK)[:, :w]


def _held_weights(weights):
    """The same for matrices, with a power of two for every 128 x 128 values."""
    E, N, K = weights.shape
    nb, kb = (N + BLOCK - 1) // BLOCK, (K + BLOCK - 1) // BLOCK
    t = weights.new_zeros((E, nb * BLOCK, kb * BLOCK))
    t[:, :N, :K] = weights
    t = t.view(E, nb, BLOCK, kb, BLOCK)
    size = torch.where(t.isfinite(), t.abs(), 0.0).amax((2, 4), keepdim=True)
    return _rounded(t, _exponent(size)).reshape(E, nb * BLOCK, kb * BLOCK)[:, :N, :K].contiguous()


def _plain_places(s):
    """Where each row's entries stand in the experts' order, and the rows of those that have an expert."""
    order, m = s["order"].long(), s["offsets"][-1].long()
    at = torch.arange(order.numel(), device=order.device)
    places = torch.empty_like(order)
    places[order] = torch.where(at < m, at, -1)
    return places, at < m


def _plain_mix(s):
    c, K, kind = s["case"], s["case"]["top_k"], s["x"].dtype
    n, w = s["x"].shape
    places, there = _plain_places(s)
    row = s["order"].long() // K
    out = {"xs": torch.where(there[:, None], s["x"][row], 0.0)}
    has = (places >= 0)[:, None]
    y = torch.where(has, s["y"][places.clamp(min=0)].float(), 0.0)
    gate = None if s["gates"] is None else s["gates"].reshape(-1, 1)
    out["out"] = (y if gate is None else y * gate).view(n, K, w).sum(1).to(kind)
    if c["train"]:
        d = s["dout"].float()[row]
        if gate is not None:
            d = d * gate[s["order"].long()]
        out["dy"] = torch.where(there[:, None], d, 0.0).to(kind)
        out["dx"] = torch.where(has, s["dxs"][places.clamp(min=0)].float(), 0.0).view(n, K, w).sum(1).to(kind)
        if gate is not None:
            out["dgates"] = (y.view(n, K, w) * s["dout"].float()[:, None, :]).sum(2)
    return out


def _plain_pack(s):
    held = _held(s["x"]).to(s["x"].dtype)
    if s["order"] is None:
        return held
    m = s["offsets"][-1].long()
    there = torch.arange(s["order"].numel(), device=m.device) < m
    return torch.where(there[:, None], held[s["order"].long() // s["case"]["top_k"]], 0.0)


def _parts(s):
    """First and last row of each expert."""
    if s["offsets"] is None:
        return [(0, s["x"].shape[0])]
    ends = s["offsets"].tolist()
    return list(zip(ends[:-1], ends[1:]))


def _plain_layer(s):
    c, kind = s["case"], s["x"].dtype
    n, K, N = c["rows"], c["inputs"], c["outputs"]
    x = _held(s["x"])
    W = _held_weights(s["weights"]) if c["train"] else s["weights_held"]
    y = x.new_zeros((n, N))
    if c["train"]:
        dy, dx = _held(s["dy"]), x.new_zeros((n, K))
        dW, db = torch.zeros_like(W), x.new_zeros((c["experts"], N))
    for e, (a, b) in enumerate(_parts(s)):
        if a == b:
            continue
        y[a:b] = x[a:b] @ W[e].t()
        if c["bias"]:
            y[a:b] += s["bias"][e]
        if c["train"]:
            dx[a:b] = dy[a:b] @ W[e]
            dW[e] = dy[a:b].t() @ x[a:b]
            db[e] = dy[a:b].sum(0)
    out = {"y": y.to(kind)}
    if c["train"]:
        out.update(dx=dx.to(kind), dweights=dW)
        if c["bias"]:
            out["dbias"] = db
    return out


def _plain_silu(s):
    kind, z = s["z"].dtype, s["z"].float()
    h = z / (1 + torch.exp(-z))
    if s["residual"] is not None:
        h = h + s["residual"].float()
    z = _held(s["z"])
    sg = 1 / (1 + torch.exp(-z))
    return {"h": h.to(kind), "dz": (s["dh"].float() * (sg * (1 + z * (1 - sg)))).to(kind)}


# ---- the definitions in 64 bits ------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"mix": _exact_mix, "pack": _exact_pack, "layer": _exact_layer, "silu": _exact_silu}[case["op"]](s)


def _exact_pow2(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_held(x, matrix=False):
    """x [..., a, b] in 8 bits: blocks of 128 along b, of 128 x 128 for a matrix."""
    x = x.double()
    out = torch.empty_like(x)
    a, b = x.shape[-2:]
    tall = BLOCK if matrix else 1
    for j in range(0, b, BLOCK):
        part = x[..., j:j + BLOCK]
        top = part.abs().amax(-1)
        if matrix:
            top = torch.stack([t.amax(-1) for t in top.split(tall, -1)], -1)
        f, q = torch.frexp(top)                       # top = f 2^q, 1/2 <= f < 1
        e = torch.where(f > 0.875, q - 8, q - 9)
        e = torch.where(top == 0, -100, e).clamp(-100, 120)
        unit = _exact_pow2(e)
        if matrix:
            unit = unit.repeat_interleave(tall, -1)[..., :a]
        rel = part / unit[..., None]
        step = _exact_pow2((torch.frexp(rel)[1] - 1).clamp(min=-6) - 3)
        out[..., j:j + BLOCK] = torch.round(rel / step) * step * unit[..., None]
    return out


def _exact_mix(s):
    c, K = s["case"], s["case"]["top_k"]
    n, w = s["x"].shape
    order, m = s["order"].long(), int(s["offsets"][-1])
    mine = order[:m]
    rows = torch.div(mine, K, rounding_mode="floor")
    gate = torch.ones(n * K, dtype=torch.float64, device=order.device)
    if s["gates"] is not None:
        gate = s["gates"].double().reshape(-1)

    def back(t, factor):
        return torch.zeros((n, w), dtype=torch.float64, device=t.device).index_add_(0, rows, t[:m].double() * factor[:, None])

    def forth(t, factor):
        full = torch.zeros((n * K, w), dtype=torch.float64, device=t.device)
        full[:m] = t.double()[rows] * factor[:, None]
        return full

    ones = torch.ones(m, dtype=torch.float64, device=order.device)
    out = {"xs": forth(s["x"], ones), "out": back(s["y"], gate[mine])}
    if c["train"]:
        out["dy"], out["dx"] = forth(s["dout"], gate[mine]), back(s["dxs"], ones)
        if s["gates"] is not None:
            dots = torch.zeros(n * K, dtype=torch.float64, device=order.device)
            dots[mine] = (s["dout"].double()[rows] * s["y"][:m].double()).sum(1)
            out["dgates"] = dots.view(n, K)
    return out


def _exact_pack(s):
    held = _exact_held(s["x"])
    if s["order"] is None:
        return held
    m = int(s["offsets"][-1])
    out = torch.zeros((s["order"].numel(), held.shape[1]), dtype=torch.float64, device=held.device)
    out[:m] = held[torch.div(s["order"][:m].long(), s["case"]["top_k"], rounding_mode="floor")]
    return out


def _exact_layer(s):
    c = s["case"]
    n, K, N = c["rows"], c["inputs"], c["outputs"]
    x, W = _exact_held(s["x"]), _exact_held(s["weights"], matrix=True)
    ends = [0, n] if s["offsets"] is None else s["offsets"].tolist()
    out = {"y": torch.zeros((n, N), dtype=torch.float64, device=x.device)}
    if c["train"]:
        dy = _exact_held(s["dy"])
        out.update(dx=torch.zeros_like(x), dweights=torch.zeros_like(W))
        if c["bias"]:
            out["dbias"] = torch.zeros((c["experts"], N), dtype=torch.float64, device=x.device)
    for e in range(c["experts"]):
        r = slice(ends[e], ends[e + 1])
        out["y"][r] = torch.matmul(x[r], W[e].t().contiguous())
        if c["bias"]:
            out["y"][r] += s["bias"][e].double()
        if c["train"]:
            out["dx"][r] = torch.matmul(dy[r], W[e])
            out["dweights"][e] = torch.matmul(dy[r].t().contiguous(), x[r])
            if c["bias"]:
                out["dbias"][e] = dy[r].sum(0)
    return out


def _exact_silu(s):
    z = s["z"].double()
    h = z * torch.sigmoid(z)
    if s["residual"] is not None:
        h = h + s["residual"].double()
    kept = _exact_held(s["z"]).requires_grad_(True)
    dz = torch.autograd.grad(torch.nn.functional.silu(kept), kept, s["dh"].double())[0]
    return {"h": h, "dz": dz}
