"""Timed cases of the operators that learn the potential's tables: routing atoms
to energy heads with a balance loss, the heads over rows grouped by head with
their gradients, and an AdamW step over all tables' tensors.  Each case has a
plain form in elementary torch operations and a definition in 64 bits.
"""
import math

import torch

own = False

F32, BF16 = "float32", "bfloat16"
WIDTH = 64          # hidden width of a head
ENC = 128           # hidden width of an encoder table
BLOCK = 256         # elements that share a scale in 8-bit states
BETA1, BETA2, EPS, DECAY, LR, STEP, GRAD_SCALE = 0.9, 0.99, 1e-8, 0.01, 1e-3, 7, 0.5


def _route(name, **over):
    c = dict(name=name, op="route", rows=1, experts=4, top_k=1, dtype=F32, kinds=0, gates="chosen", empty=0.0, spare=0,
             backward=True)
    c.update(over)
    return c


def _heads(name, **over):
    c = dict(name=name, op="heads", rows=1, width=128, hidden=4, experts=6, top_k=1, dtype=F32, want="train", skew=0.0,
             empty=0.0, spare=0)
    c.update(over)
    return c


def _adamw(name, **over):
    c = dict(name=name, op="adamw", species=1, k=32, lmax=3, enc_hidden=3, reg_hidden=4, bits=32, param=F32, grad=F32)
    c.update(over)
    return c


def listed():
    return [
        # one small cell, four heads: launches and latency
        _route("route-cell-108", rows=108),
        # a ragged batch: six kinds of atom with heads of their own, padded
        # rows, rows further apart than they are long
        _route("route-ragged-131k", rows=131071, experts=29, top_k=3, kinds=6, empty=0.03, spare=3),
        # evaluation of a large system, logits in 16 bits, no gradient
        _route("route-serve-1m-bf16", rows=1048576, experts=16, top_k=2, dtype=BF16, gates="all", backward=False),
        # the largest batch and many heads
        _route("route-train-2m", rows=2097152, experts=64, top_k=4, kinds=16, empty=0.01),
        # one new atom: energy and its gradient in the descriptor
        _heads("heads-one-atom", want="gradient"),
        # an MD step of a six-component system: energies and gradients
        _heads("heads-md-262k", rows=262144, want="gradient", skew=0.5),
        # a small ragged batch of training structures
        _heads("heads-train-5k", rows=4994, empty=0.02, skew=1.0),
        # two of eight heads for each atom, wide descriptors in 16 bits
        _heads("heads-mixture-131k-bf16", rows=131071, width=192, experts=8, top_k=2, dtype=BF16, empty=0.01),
        # the largest training batch
        _heads("heads-train-1m", rows=1048576, skew=0.5),
        # one element: 18 tensors
        _adamw("adamw-unary"),
        # six components: 348 tensors, states in 8 bits, gradients in 16
        _adamw("adamw-hea6-8bit", species=6, bits=8, grad=BF16),
        # sixteen components with the widest basis: 2,208 tensors
        _adamw("adamw-16-species", species=16, k=64),
    ]


def _log(rng, low, high):
    return round(math.exp(rng.uniform(math.log(low), math.log(high))))


def draw(rng):
    """Another case of the same ranges, at most as much work as the largest listed one of its operator."""
    op = rng.choice(["route", "heads", "adamw"])
    if op == "route":
        experts = _log(rng, 2, 256)
        c = _route("", experts=experts, rows=_log(rng, 1, min(2097152, 2097152 * 64 // experts)),
                   top_k=rng.randint(1, min(experts, 8)), dtype=rng.choice([F32, BF16]), kinds=rng.choice([0, 0, 1, 6, 16]),
                   gates=rng.choice(["chosen", "all"]), empty=rng.choice([0.0, rng.uniform(0.0, 0.2)]),
                   spare=rng.choice([0, 0, rng.randint(1, 9)]), backward=rng.random() < 0.7)
    elif op == "heads":
        experts = _log(rng, 1, 64)
        c = _heads("", experts=experts, top_k=rng.choice([1, 1, rng.randint(1, min(experts, 4))]),
                   width=rng.choice([16, 32, 64, 128, 128, 192, 256, 384, rng.randint(1, 384)]), hidden=rng.randint(1, 8),
                   dtype=rng.choice([F32, F32, BF16]), want=rng.choice(["energy", "gradient", "train", "train"]),
                   skew=rng.choice([0.0, rng.uniform(0.0, 2.0)]), empty=rng.choice([0.0, rng.uniform(0.0, 0.2)]),
                   spare=rng.choice([0, 0, rng.randint(1, 9)]))
        most = 1048576 * _macs(_heads("")) // (_macs(c) * c["top_k"])
        c["rows"] = _log(rng, 1, min(1048576, most * 128 // max(c["width"], 128)))
    else:
        c = _adamw("", species=rng.randint(1, 16), k=rng.choice([16, 32, 64]), lmax=rng.randint(0, 5),
                   enc_hidden=rng.randint(1, 3), reg_hidden=rng.randint(1, 8), bits=rng.choice([32, 8]),
                   param=rng.choice([F32, F32, BF16]), grad=rng.choice([F32, BF16]))
        while sum(_sizes(c)) > sum(_sizes(_adamw("", species=16, k=64))):
            c["species"] -= 1
    del c["name"]
    return c


def _macs(c):
    """Multiplications of one row through one head."""
    return WIDTH * c["width"] + (c["hidden"] - 1) * WIDTH * WIDTH + WIDTH


def _head_values(width, hidden):
    return WIDTH * width + WIDTH + (hidden - 1) * (WIDTH * WIDTH + WIDTH) + WIDTH + 1


def _segments(c):
    """(elements, whether it is a matrix) of every tensor of the potential's blob, in its order."""
    enc = [(ENC, False), (ENC, False)] + [(ENC * ENC, True), (ENC, False)] * (c["enc_hidden"] - 1) \
        + [(c["k"] * ENC, True), (c["k"], False)]
    head = [(WIDTH * (c["lmax"] + 1) * c["k"], True), (WIDTH, False)] \
        + [(WIDTH * WIDTH, True), (WIDTH, False)] * (c["reg_hidden"] - 1) + [(WIDTH, False), (1, False)]
    return enc * c["species"] ** 2 + head * c["species"]


def _sizes(c):
    return [n for n, _ in _segments(c)]


def work(case):
    c = case
    if c["op"] == "route":
        size = 2 if c["dtype"] == BF16 else 4
        n, kinds = c["rows"], 4 * c["rows"] if c["kinds"] else 0
        # forward: logits, kinds; experts and gates.  Backward: logits, kinds, experts and their gradients; logits' gradient
        b = n * c["experts"] * size + kinds + 8 * n * c["top_k"]
        f = 5 * n * c["experts"]
        if c["backward"]:
            b += 2 * n * c["experts"] * size + kinds + 8 * n * c["top_k"]
            f += 9 * n * c["experts"]
        return {"bytes": b, "flops": f}
    if c["op"] == "heads":
        size = 2 if c["dtype"] == BF16 else 4
        n, e = c["rows"], c["rows"] * c["top_k"]
        weights = 4 * c["experts"] * _head_values(c["width"], c["hidden"])
        mixed = 4 * e if c["top_k"] > 1 else 0                       # gates
        b = n * c["width"] * size + weights + 4 * e + 4 * e + mixed + 4 * n   # descriptors, ids, grouping, energies
        times = 1
        if c["want"] != "energy":
            b += n * c["width"] * size
            times = 2
        if c["want"] == "train":
            b += weights + 4 * n + mixed
            times = 3
        return {"bytes": b, "flops": 2 * times * e * _macs(c)}
    n = sum(_sizes(c))
    state = 16 if c["bits"] == 32 else 4
    b = n * (2 * (2 if c["param"] == BF16 else 4) + (2 if c["grad"] == BF16 else 4) + state)
    if c["bits"] == 8:
        b += n * (2 + 8)                                              # the moments' values, given back
    return {"bytes": b, "flops": 15 * n}


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


def _route_inputs(c, g, dev):
    n, E = c["rows"], c["experts"]
    kinds = allowed = None
    logits = torch.randn((n, E), generator=g, device=dev) * 2.0
    if c["kinds"]:
        kinds = torch.randint(0, c["kinds"], (n,), generator=g, device=dev, dtype=torch.int32)
        allowed = (torch.rand((c["kinds"], E), generator=g, device=dev) < 0.6).to(torch.uint8)
        allowed[torch.arange(c["kinds"], device=dev), torch.arange(c["kinds"], device=dev) % E] = 1
        if c["empty"]:
            # padded atoms have no kind, and nothing that means something in their rows
            gone = torch.rand((n,), generator=g, device=dev) < c["empty"]
            kinds[gone] = -1
            logits[gone] = float("nan")
    elif c["empty"]:
        logits[torch.rand((n,), generator=g, device=dev) < c["empty"]] = float("-inf")
    s = dict(case=c, logits=_spaced(logits.to(getattr(torch, c["dtype"])), c["spare"]), kinds=kinds, allowed=allowed)
    if c["backward"]:
        s["dgates"] = torch.randn((n, c["top_k"]), generator=g, device=dev)
        s["dloss"] = torch.full((1,), 0.01, device=dev)
    if own:
        from paper_2608_16329_amd import Learner
        s["learner"] = Learner()
        s["chosen"] = torch.empty((n, c["top_k"]), dtype=torch.int32, device=dev)
        s["weight"] = torch.empty((n, c["top_k"]), device=dev)
        s["counts"] = torch.empty((E + 1,), dtype=torch.int32, device=dev)
        s["loss"] = torch.empty((1,), device=dev)
        if c["backward"]:
            s["dlogits"] = torch.empty((n, E), dtype=s["logits"].dtype, device=dev)
    return s


def _heads_inputs(c, g, dev):
    n, E, D, K = c["rows"], c["experts"], c["width"], c["top_k"]
    # squared norms of moments: positive, most of them small
    x = 0.5 * torch.randn((n, D), generator=g, device=dev).square()
    scale = torch.cat([torch.full((m,), 1.0 / math.sqrt(fan)) for m, fan in
                       [(WIDTH * D, D), (WIDTH, D)] + [(WIDTH * WIDTH, WIDTH), (WIDTH, WIDTH)] * (c["hidden"] - 1)
                       + [(WIDTH + 1, WIDTH)]]).to(dev)
    weights = torch.randn((E, scale.numel()), generator=g, device=dev) * scale
    # shares of the heads: equal, or falling off
    share = torch.exp(-c["skew"] * torch.arange(E, device=dev, dtype=torch.float32) / max(1, E - 1) * 3.0)
    noise = -torch.log(-torch.log(torch.rand((n, E), generator=g, device=dev).clamp_(1e-7, 1 - 1e-7)))
    experts = torch.topk(share.log() + noise, K, dim=1).indices.to(torch.int32)
    if c["empty"]:
        experts[torch.rand((n, K), generator=g, device=dev) < c["empty"]] = -1
    s = dict(case=c, x=_spaced(x.to(getattr(torch, c["dtype"])), c["spare"]), weights=weights, experts=experts, gates=None,
             denergy=None)
    if K > 1:
        s["gates"] = torch.softmax(torch.randn((n, K), generator=g, device=dev), dim=1)
    if c["want"] == "train":
        s["denergy"] = torch.randn((n,), generator=g, device=dev)
    if own:
        from paper_2608_16329_amd import Learner
        s["learner"] = Learner()
        out = dict(offsets=torch.empty((E + 1,), dtype=torch.int32, device=dev),
                   order=torch.empty((n * K,), dtype=torch.int32, device=dev), energy=torch.empty((n,), device=dev))
        if c["want"] != "energy":
            out["dx"] = torch.empty((n, D), dtype=s["x"].dtype, device=dev)
        if c["want"] == "train":
            out["dweights"] = torch.empty_like(weights)
            if K > 1:
                out["dgates"] = torch.empty_like(s["gates"])
        s["out"] = out
    return s


def _adamw_inputs(c, g, dev):
    sizes = _sizes(c)
    n = sum(sizes)
    param = (torch.randn((n,), generator=g, device=dev) * 0.1).to(getattr(torch, c["param"]))
    grad = (torch.randn((n,), generator=g, device=dev) * 1e-2).to(getattr(torch, c["grad"]))
    m = torch.randn((n,), generator=g, device=dev) * 1e-3
    v = torch.randn((n,), generator=g, device=dev).square() * 1e-5
    count = torch.tensor(sizes, device=dev)
    s = dict(case=c, param=param, grad=grad, sizes=sizes, count=count, seed=int(torch.randint(1 << 31, (1,), generator=g, device=dev)),
             decay=torch.tensor([w for _, w in _segments(c)], device=dev))
    if c["bits"] == 8:
        # blocks of up to 256 elements, none across two tensors
        s["blocks"] = torch.tensor([min(BLOCK, z - b) for z in sizes for b in range(0, z, BLOCK)], device=dev)
        block = _block_of(s)
        s["m"], s["m_exp"], _ = _held(m, block, s["blocks"].numel(), torch.full_like(m, 0.5), 3)
        s["v"], s["v_exp"], _ = _held(v, block, s["blocks"].numel(), torch.full_like(m, 0.5), 4)
    else:
        s["m"], s["v"] = m, v
    if own:
        from paper_2608_16329_amd import AdamW
        s["param_new"] = torch.empty_like(param)
        s["opt"] = AdamW(param.split(sizes), grad.split(sizes), bits=c["bits"], decay=[w for _, w in _segments(c)],
                         into=s["param_new"].split(sizes))
        for name in ("m", "v", "m_exp", "v_exp"):
            if name in s:
                getattr(s["opt"], name).copy_(s[name])
        if c["bits"] == 8:
            s["values"] = [torch.empty((n,), device=dev) for _ in range(2)]
    return s


def prepare(case, seed):
    dev = _device()
    g = _rng(seed, dev)
    return {"route": _route_inputs, "heads": _heads_inputs, "adamw": _adamw_inputs}[case["op"]](dict(case), g, dev)


# ---- one pass ----------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if op == "route":
        return _run_route(state) if own else _plain_route(state)
    if op == "heads":
        return _run_heads(state) if own else _plain_heads(state)
    return _run_adamw(state) if own else _plain_adamw(state)


def _run_route(s):
    c, L = s["case"], s["learner"]
    L.route(s["logits"], s["chosen"], s["weight"], s["counts"], s["loss"], kinds=s["kinds"], allowed=s["allowed"],
            gates_of=c["gates"])
    out = {"experts": s["chosen"], "gates": s["weight"], "counts": s["counts"], "loss": s["loss"]}
    if c["backward"]:
        L.route_backward(s["logits"], s["chosen"], s["counts"], s["dlogits"], dgates=s["dgates"], dloss=s["dloss"],
                         kinds=s["kinds"], allowed=s["allowed"], gates_of=c["gates"])
        out["dlogits"] = s["dlogits"]
    return out


def _run_heads(s):
    c, L, out = s["case"], s["learner"], s["out"]
    L.group(s["experts"], out["offsets"], out["order"])
    L.heads(s["x"], s["weights"], out["offsets"], out["order"], hidden=c["hidden"], top_k=c["top_k"], gates=s["gates"],
            denergy=s["denergy"], energy=out["energy"], dx=out.get("dx"), dweights=out.get("dweights"),
            dgates=out.get("dgates"))
    return out


def _run_adamw(s):
    opt = s["opt"]
    opt.step(STEP, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY, grad_scale=GRAD_SCALE, seed=s["seed"])
    out = {"param": s["param_new"]}
    if s["case"]["bits"] == 8:
        opt.moments(*s["values"])
        out["m"], out["v"] = s["values"]
    else:
        out["m"], out["v"] = opt.new_m, opt.new_v
    return out


# ---- plain forms -------------------------------------------------------------

def _plain_route(s):
    c, logits = s["case"], s["logits"].float()
    n, E, K = c["rows"], c["experts"], c["top_k"]
    open_ = logits != -math.inf
    if s["kinds"] is not None:
        kind = s["kinds"].long()
        open_ = open_ & (kind >= 0)[:, None] & (s["allowed"][kind.clamp(min=0)] != 0)
    z = torch.where(open_, logits, -math.inf)
    live = open_.any(1)
    top = torch.where(live, z.amax(1), 0.0)
    e = torch.exp(z - top[:, None])
    p = e / torch.where(live, e.sum(1), 1.0)[:, None]
    # the largest logits, equal ones in the order of their heads
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :K]
    there = open_.gather(1, order)
    weight = torch.where(there, p.gather(1, order), 0.0)
    if c["gates"] == "chosen":
        weight = weight / torch.where(live, weight.sum(1), 1.0)[:, None]
    chosen = torch.where(there, order, -1)
    counts = torch.bincount(torch.where(there, order, E).reshape(-1), minlength=E + 1)[:E]
    rows = live.sum()
    share = counts.float() / counts.sum().clamp(min=1)
    loss = E * (share * p.sum(0)).sum() / rows.clamp(min=1)
    out = {"experts": chosen.to(torch.int32), "gates": weight, "counts": torch.cat([counts, rows[None]]).to(torch.int32),
           "loss": loss.reshape(1)}
    if c["backward"]:
        h = (s["dloss"] * E / rows.clamp(min=1) * share)[None, :].expand(n, E)
        dgate = torch.where(there, s["dgates"], 0.0)
        if c["gates"] == "all":
            h = h.scatter_add(1, order, dgate)
        d = p * (h - (p * h).sum(1, keepdim=True))
        if c["gates"] == "chosen":
            d = d.scatter_add(1, order, weight * (dgate - (weight * dgate).sum(1, keepdim=True)))
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _parts(row, width, hidden):
    """The matrices and vectors of one head."""
    sizes = [WIDTH * width, WIDTH] + [WIDTH * WIDTH, WIDTH] * (hidden - 1) + [WIDTH, 1]
    t = row.split(sizes)
    return [t[0].view(WIDTH, width)] + [m.view(WIDTH, WIDTH) for m in t[2:-2:2]], t[1:-2:2], t[-2], t[-1]


def _plain_heads(s):
    c = s["case"]
    n, E, D, K, H = c["rows"], c["experts"], c["width"], c["top_k"], c["hidden"]
    x, weights = s["x"].float(), s["weights"].float()
    flat = s["experts"].reshape(-1).long()
    key = torch.where(flat >= 0, flat, E)
    order = torch.sort(key, stable=True).indices
    counts = torch.bincount(key, minlength=E + 1)
    offsets = torch.cat([counts.new_zeros(1), counts[:E].cumsum(0)])
    value = x.new_zeros(n * K)
    gate = None if s["gates"] is None else s["gates"].reshape(-1)
    dvalue = s["denergy"] if s["denergy"] is not None else x.new_ones(n)
    dvalue = dvalue.repeat_interleave(K) if K > 1 else dvalue
    dentry = dvalue if gate is None else dvalue * gate
    dx = x.new_zeros((n * K, D)) if c["want"] != "energy" else None
    dweights = torch.zeros_like(weights) if c["want"] == "train" else None
    # each head's matrices on its own rows, one layer after another
    for e, mine in enumerate(order.split(counts.tolist())[:E]):
        if not mine.numel():
            continue
        A, b, a, last = _parts(weights[e], D, H)
        xe = x[mine // K]
        z = xe @ A[0].t() + b[0]
        y, pre = z * torch.sigmoid(z), [z]
        seen = [xe, y]
        for t in range(1, H):
            z = y @ A[t].t() + b[t]
            y = y + z * torch.sigmoid(z)
            pre.append(z)
            seen.append(y)
        value[mine] = y @ a + last
        if c["want"] == "energy":
            continue
        d = dentry[mine]
        u = d[:, None] * a
        grads = [d.sum().reshape(1), d @ y]
        for t in range(H - 1, -1, -1):
            sg = torch.sigmoid(pre[t])
            gz = u * sg * (1 + pre[t] * (1 - sg))
            if c["want"] == "train":
                grads += [gz.sum(0), (gz.t() @ seen[t]).reshape(-1)]
            u = gz @ A[t] + (u if t else 0)
        dx[mine] = u
        if c["want"] == "train":
            dweights[e] = torch.cat(grads[::-1])
    energy = value if gate is None else value * gate
    out = {"offsets": offsets.to(torch.int32), "order": order.to(torch.int32), "energy": energy.view(n, K).sum(1)}
    if dx is not None:
        out["dx"] = (dx.view(n, K, D).sum(1) if K > 1 else dx).to(s["x"].dtype)
    if dweights is not None:
        out["dweights"] = dweights
        if gate is not None:
            out["dgates"] = (value * dvalue).view(n, K)
    return out


def _block_of(s):
    return torch.repeat_interleave(torch.arange(s["blocks"].numel(), device=s["blocks"].device), s["blocks"])


def _pow2(e):
    """2^e in float32, -126 <= e <= 127, from its bits."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _held(x, block, blocks, u, mant):
    """x in 8 bits: of the m's 4 exponent and 3 mantissa bits beside the sign, of the
    v's (x >= 0) 4 and 4, relative to the block's power of two 2^e > max |x|; t
    + u rounded down, u in [0, 1).  Codes, e + 127, and the values they stand for."""
    size = x.abs()
    fine = size.isfinite()
    top = torch.zeros(blocks, dtype=x.dtype, device=x.device)
    top = top.scatter_reduce(0, block, torch.where(fine, size, 0.0), "amax")
    e = ((top.view(torch.int32) >> 23) - 126).clamp(-126, 126)
    y = torch.where(fine, size, 0.0) * _pow2(-e)[block]
    ey = ((y.view(torch.int32) >> 23) - 127).clamp(min=-14)
    whole = torch.floor(y * _pow2(mant - ey) + u).to(torch.int32)
    code = (((ey + 14) << mant) + whole).clamp(max=126 if mant == 3 else 254)
    if mant == 4:
        code = torch.where((size > 0) & (code == 0), 1, code)
    code = torch.where(fine, code, 127 if mant == 3 else 255)
    if mant == 3:
        code = code | ((x < 0) & fine).to(torch.int32) << 7
    code = code.to(torch.uint8)
    return code, (e + 127).to(torch.uint8), _value(code, (e + 127)[block], mant)


def _value(code, e, mant):
    c = code.to(torch.int32)
    if mant == 3:
        sign, c = 1.0 - 2.0 * (c >> 7).float(), c & 127
    ec = c >> mant
    base = (c & ((1 << mant) - 1)) + torch.where(ec > 0, 1 << mant, 0)
    v = base.float() * _pow2(ec.clamp(min=1) - 15 - mant) * _pow2(e.to(torch.int32) - 127)
    v = torch.where(c == (127 if mant == 3 else 255), math.nan, v)
    return v * sign if mant == 3 else v


def _dice(seed, n, device):
    """32 mixed bits for each element, from the seed and its place."""
    h = (torch.arange(n, device=device) * 0x9E3779B1 + seed) & 0xFFFFFFFF
    h = ((h ^ (h >> 15)) * 0x2C1B3C6D) & 0xFFFFFFFF
    h = ((h ^ (h >> 12)) * 0x297A2D39) & 0xFFFFFFFF
    return h ^ (h >> 15)


def _plain_adamw(s):
    c, p, g = s["case"], s["param"].float(), s["grad"].float() * GRAD_SCALE
    block = _block_of(s) if c["bits"] == 8 else None
    m, v = s["m"], s["v"]
    if c["bits"] == 8:
        m, v = _value(m, s["m_exp"][block], 3), _value(v, s["v_exp"][block], 4)
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    keep = torch.where(s["decay"], 1 - LR * DECAY, 1.0).repeat_interleave(s["count"])
    q = p * keep - (LR / (1 - BETA1 ** STEP)) * (m / (torch.sqrt(v) * (1 / math.sqrt(1 - BETA2 ** STEP)) + EPS))
    if c["bits"] == 8:
        dice = _dice(s["seed"], p.numel(), p.device)
        m = _held(m, block, s["blocks"].numel(), (dice & 0xFFFF).float() * 2.0 ** -16, 3)[2]
        v = _held(v, block, s["blocks"].numel(), (dice >> 16).float() * 2.0 ** -16, 4)[2]
    return {"param": q.to(s["param"].dtype), "m": m, "v": v}


# ---- the definitions in 64 bits ------------------------------------------------

def exact(case, seed):
    if case["op"] == "route":
        return _exact_route(case, seed)
    if case["op"] == "heads":
        return _exact_heads(case, seed)
    return _exact_adamw(case, seed)


def _exact_route(case, seed):
    s = prepare(case, seed)
    E, K = case["experts"], case["top_k"]
    logits = s["logits"].double().clone()
    if s["kinds"] is not None:
        table = torch.cat([s["allowed"] == 0, torch.ones((1, E), dtype=torch.bool, device=logits.device)])
        logits[table[s["kinds"].long()]] = -math.inf             # kind -1 reads the added row
    dead = (logits == -math.inf).all(1)
    logits[dead] = 0.0
    logits.requires_grad_(True)
    p = torch.softmax(logits, 1) * (~dead)[:, None]
    ids = torch.sort(logits.detach(), dim=1, descending=True, stable=True).indices[:, :K]
    z = logits.gather(1, ids)
    there = (z != -math.inf) & ~dead[:, None]
    if case["gates"] == "chosen":
        gates = torch.softmax(z, 1) * (~dead)[:, None]
    else:
        gates = p.gather(1, ids)
    used = torch.zeros(E, dtype=torch.float64, device=p.device)
    used.index_add_(0, ids[there], torch.ones_like(ids[there], dtype=torch.float64))
    rows = (~dead).sum()
    loss = E / rows.clamp(min=1) / used.sum().clamp(min=1) * (p @ used).sum()
    out = {"experts": torch.where(there, ids, -1).to(torch.int32), "gates": gates.detach(),
           "counts": torch.cat([used, rows[None]]).to(torch.int32), "loss": loss.detach().reshape(1)}
    if case["backward"]:
        total = (gates * s["dgates"].double() * there).sum() + s["dloss"].double()[0] * loss
        d = torch.autograd.grad(total, logits)[0]
        out["dlogits"] = torch.where((logits == -math.inf) | dead[:, None], 0.0, d.detach())
    return out


def _exact_heads(case, seed):
    s = prepare(case, seed)
    n, E, D, K, H = case["rows"], case["experts"], case["width"], case["top_k"], case["hidden"]
    train = case["want"] == "train"
    W = s["weights"].double()
    value = torch.zeros((n, K), dtype=torch.float64, device=W.device)
    dx = torch.zeros((n, D), dtype=torch.float64, device=W.device)
    dW = torch.zeros_like(W)
    up = s["denergy"].double() if s["denergy"] is not None else torch.ones(n, dtype=torch.float64, device=W.device)
    gates = s["gates"].double() if s["gates"] is not None else torch.ones((n, K), dtype=torch.float64, device=W.device)
    for e in range(E):
        for k in range(K):
            for rows in (s["experts"][:, k] == e).nonzero()[:, 0].split(131072):
                x = s["x"][rows].double().requires_grad_(True)
                w = W[e].clone().requires_grad_(True)
                A, b, a, last = _parts(w, D, H)
                y = torch.nn.functional.silu(x @ A[0].t() + b[0])
                for t in range(1, H):
                    y = y + torch.nn.functional.silu(y @ A[t].t() + b[t])
                v = y @ a + last
                value[rows, k] = v.detach()
                if case["want"] != "energy":
                    gx, gw = torch.autograd.grad((v * up[rows] * gates[rows, k]).sum(), (x, w))
                    dx[rows] += gx
                    dW[e] += gw
    out = {"offsets": None, "order": None, "energy": (value * gates).sum(1)}
    if case["want"] != "energy":
        out["dx"] = dx
    if train:
        out["dweights"] = dW
        if K > 1:
            out["dgates"] = value * up[:, None]
    return out


def _exact_adamw(case, seed):
    s = prepare(case, seed)
    sizes, bits = s["sizes"], case["bits"]
    p, g = s["param"].double(), s["grad"].double() * GRAD_SCALE
    block = _block_of(s) if bits == 8 else None

    def decode(code, e, mant):
        c = code.long()
        sign = 1.0 if mant == 4 else 1.0 - 2.0 * (c >= 128).double()
        c = c if mant == 4 else c % 128
        ec, f = torch.div(c, 2 ** mant, rounding_mode="floor"), (c % 2 ** mant).double() / 2 ** mant
        rel = torch.where(ec > 0, (1 + f) * torch.pow(2.0, (ec - 15).double()), f * 2.0 ** -14)
        return sign * rel * torch.pow(2.0, (e.double() - 127)[block])

    def encode(x, u, mant):
        top = torch.zeros(s["blocks"].numel(), dtype=torch.float64, device=x.device).scatter_reduce(0, block, x.abs(), "amax")
        scale = torch.pow(2.0, torch.floor(torch.log2(top.clamp(min=2.0 ** -126))) + 1)[block]
        rel = x.abs() / scale
        step = torch.pow(2.0, torch.floor(torch.log2(rel.clamp(min=2.0 ** -14))) - mant)
        near = torch.floor(rel / step + u) * step
        if mant == 4:
            near = torch.where((x > 0) & (near == 0), step, near)
        return torch.sign(x) * near * scale

    m = decode(s["m"], s["m_exp"], 3) if bits == 8 else s["m"].double()
    v = decode(s["v"], s["v_exp"], 4) if bits == 8 else s["v"].double()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    new = []
    for q, mi, vi, matrix in zip(p.split(sizes), m.split(sizes), v.split(sizes), s["decay"].tolist()):
        q = q * (1 - LR * DECAY) if matrix else q
        new.append(q - LR * (mi / (1 - BETA1 ** STEP)) / ((vi / (1 - BETA2 ** STEP)).sqrt() + EPS))
    if bits == 8:
        dice = _dice(s["seed"], p.numel(), p.device)
        m = encode(m, (dice % 65536).double() / 65536, 3)
        v = encode(v, torch.div(dice, 65536, rounding_mode="floor").double() / 65536, 4)
    return {"param": torch.cat(new), "m": m, "v": v}
