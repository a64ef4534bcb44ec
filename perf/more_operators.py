"""Performance cases of experts in 4 bits, of whole layers of experts for few tokens, and of clipped gradients.

Five operators.  `quantize` takes matrices to 4-bit floating point with a scale for each 32 and gives the values that they stand for;
`linear` takes activations to 4 bits and through one product with weights that are kept so; `experts` runs the products of all experts over
the tokens that were routed to them, in 4 bits, and sums each token's results; `layer` takes a few tokens through a whole layer of experts,
from the router's logits to the sum (weights in 8 or 4 bits); `clip` takes the norm of many gradients and clips them by it.

Where `own` is true `run` makes the calls of this framework, else it computes the same from elementary torch operations in 32 bits.
`exact` is the definition in 64 bits.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}

SMALL = 32                       # values that share a scale, a power of two, in 4 bits (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6)
ROW = 256                        # rows in 4 bits are laid out in whole runs of so many
LEAST, MOST = -126, 125          # exponents of scales

BLOCK = 128                      # values that share a scale in 8 bits (e4m3)
LARGEST = 448.0
SMALLEST = 1e-30                 # a block whose largest magnitude is below this is scaled as if it were this


def _quantize(name, experts, rows, cols, type):
    return {"name": name, "kind": "quantize", "experts": experts, "rows": rows, "cols": cols, "type": type}


def _linear(name, rows, inputs, outputs, type):
    return {"name": name, "kind": "linear", "rows": rows, "inputs": inputs, "outputs": outputs, "type": type}


def _experts(name, tokens, experts, k, inputs, outputs, type, skew=False, padding=False):
    return {"name": name, "kind": "experts", "tokens": tokens, "experts": experts, "k": k, "inputs": inputs, "outputs": outputs,
            "type": type, "skew": skew, "padding": padding}


def _layer(name, tokens, experts, k, width, hidden, type, bits, score="softmax", bias=False, renormalize=True, scale=1.0, gelu=False,
           padding=False):
    return {"name": name, "kind": "layer", "tokens": tokens, "experts": experts, "k": k, "width": width, "hidden": hidden, "type": type,
            "bits": bits, "score": score, "bias": bias, "renormalize": renormalize, "scale": scale, "gelu": gelu, "padding": padding}


def _clip(name, tensors, total, type, out, clipped=True, norm_alone=False):
    return {"name": name, "kind": "clip", "tensors": tensors, "total": total, "type": type, "out": out, "clipped": clipped,
            "norm_alone": norm_alone}


def listed():
    return [
        # a trained layer's matrices are brought to 4 bits to be served: a large matrix each, in 16 bits
        _quantize("quantize_weights", 4, 4096, 4096, "bf16"),
        # master weights of odd size: no row starts where the one before suggests, the last block is short
        _quantize("quantize_odd", 1, 777, 1001, "fp32"),
        # one token through one layer: the weights are read once, for one row
        _linear("linear_one_token", 1, 4096, 4096, "bf16"),
        # a batch with odd sizes throughout
        _linear("linear_odd", 777, 1100, 1001, "fp16"),
        # a long prompt through a wide layer: the largest product
        _linear("linear_large", 8192, 8192, 8192, "bf16"),
        # a few conversations at once through one matrix of each expert, unequally popular experts, odd sizes
        _experts("experts_batch_odd", 24, 100, 5, 1000, 1100, "fp16", skew=True),
        # a long prompt with padded places
        _experts("experts_prompt", 4093, 64, 4, 2048, 2048, "bf16", skew=True, padding=True),
        # one token of a conversation through a whole layer whose weights are kept in 8 bits
        _layer("layer_one_token", 1, 64, 6, 2048, 1408, "bf16", 8),
        # a few conversations at once, sigmoid scores with a bias that balances the load, odd sizes, a place that is padding
        _layer("layer_few_odd", 5, 100, 5, 1000, 700, "fp16", 4, score="sigmoid", bias=True, scale=2.5, padding=True),
        # as many tokens as such a call takes: most experts are met, each by few
        _layer("layer_sixteen", 16, 128, 8, 4096, 1024, "bf16", 4, gelu=True),
        # the gradients of a small model of sixteen experts: nothing but latency
        _clip("clip_small", 3, 13_000, "fp32", "fp32"),
        # the gradients of a large model, from a bias to matrices, to the 16-bit buffer that is sent to the other workers
        _clip("clip_large", 300, 400_000_000, "fp32", "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Any sizes the listed ones stand for: 1 to 8192 rows (a layer: 1 to 16), 64 to 8192 columns, 8 to 256 experts of which 1 to 8 are
    taken, 1 to 400 gradients, bounded by what the largest listed case of the kind costs."""
    kind = rng.choice(["quantize", "linear", "linear", "experts", "layer", "layer", "clip"])
    type = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if kind == "quantize":
        while True:
            experts, rows, cols = rng.choice([1, 1, 3, 8]), _log(rng, 1, 8192), _log(rng, 1, 8192)
            if experts * rows * cols <= 1 << 26:
                return _unnamed(_quantize("", experts, rows, cols, type))
    if kind == "linear":
        while True:
            rows, inputs, outputs = _log(rng, 1, 16384), _log(rng, 64, 8192), _log(rng, 64, 8192)
            if rows * inputs * outputs <= 4e11 and rows * max(inputs, outputs) <= 1 << 26:
                return _unnamed(_linear("", rows, inputs, outputs, type))
    if kind == "experts":
        while True:
            tokens, experts, k = _log(rng, 1, 8192), _log(rng, 8, 128), rng.randint(1, 8)
            inputs, outputs = _log(rng, 64, 4096), _log(rng, 64, 4096)
            tiles = tokens * k // BLOCK + min(experts, tokens * k)
            if tokens * k * inputs * outputs <= 6e10 and tiles * inputs * outputs <= 1 << 30 and experts * inputs * outputs <= 1 << 28:
                return _unnamed(_experts("", tokens, experts, k, inputs, outputs, type, rng.random() < 0.5, rng.random() < 0.3))
    if kind == "layer":
        # (results in 16 bits: in 32 a value that lies next to a border of its 8 or 4 bits would count, whichever way it is rounded)
        type = rng.choice(["bf16", "bf16", "fp16"])
        while True:
            tokens, experts, k = rng.randint(1, 16), _log(rng, 8, 256), rng.randint(1, 8)
            width, hidden = _log(rng, 64, 4096), _log(rng, 64, 2048)
            if tokens * k * width * hidden <= 1 << 29 and experts * width * hidden <= 1 << 29:
                score = rng.choice(["softmax", "sigmoid"])
                return _unnamed(_layer("", tokens, experts, k, width, hidden, type, rng.choice([8, 4]), score,
                                       score == "sigmoid" and rng.random() < 0.7, rng.random() < 0.6, rng.choice([1.0, 2.5]),
                                       rng.random() < 0.3, tokens > 1 and rng.random() < 0.3))
    tensors = _log(rng, 1, 400)
    return _unnamed(_clip("", tensors, max(tensors, _log(rng, 1000, 400_000_000)), type, rng.choice([type, "fp32", "bf16"]),
                          rng.random() < 0.7, rng.random() < 0.3))


def _unnamed(case):
    del case["name"]
    return case


# ---- inputs ------------------------------------------------------------------------------------------------------
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _activations(rows, cols, dtype, gen):
    """Normal values, a few columns much larger than the rest, as a network's activations are."""
    x = torch.randn((rows, cols), generator=gen, device="cuda")
    large = torch.rand(cols, generator=gen, device="cuda") < 0.01
    return (x * torch.where(large, 20.0, 1.0)).to(dtype)


def _blocks_of(cols):
    return -(-cols // BLOCK)


def _weights8(experts, outputs, inputs, gen):
    """Weights as a checkpoint has them: e4m3 values [experts, outputs, whole blocks of inputs], zeros at the end, and a
    scale for each square [experts, blocks of outputs, blocks of inputs]."""
    nb, kb = _blocks_of(outputs), _blocks_of(inputs)
    w = torch.zeros((experts, nb * BLOCK, kb * BLOCK), device="cuda")
    w[:, :outputs, :inputs].normal_(0.0, 1.0 / math.sqrt(inputs), generator=gen)
    tiles = w.view(experts, nb, BLOCK, kb, BLOCK)
    top = tiles.abs().amax((2, 4), keepdim=True).clamp_min(SMALLEST)
    values = (tiles * (LARGEST / top)).clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
    scales = (top / LARGEST).view(experts, nb, kb)
    return values.view(experts, nb * BLOCK, kb * BLOCK)[:, :outputs].contiguous(), scales.contiguous()


def _weights4(experts, outputs, inputs, gen):
    """Weights as a checkpoint has them: two values a byte [experts, outputs, whole runs of 256 inputs / 2], the first in the low bits,
    and the exponents of the scales plus 127 [experts, outputs, whole runs / 32]; zeros at the end."""
    whole = -(-inputs // ROW) * ROW
    values = torch.empty((experts, outputs, whole // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((experts, outputs, whole // SMALL), dtype=torch.uint8, device="cuda")
    for e0 in range(0, experts, 16):
        w = torch.zeros((min(16, experts - e0), outputs, whole), device="cuda")
        w[:, :, :inputs].normal_(0.0, 1.0 / math.sqrt(inputs), generator=gen)
        b = w.view(-1, SMALL)
        e = _exponents(b)
        q = _nearest(torch.ldexp(b, -e[:, None]))
        q = (q + 8 * (b < 0)).to(torch.uint8).view(w.shape[0], outputs, whole // 2, 2)
        values[e0:e0 + 16] = q[..., 0] + 16 * q[..., 1]
        scales[e0:e0 + 16] = (e + 127).to(torch.uint8).view(w.shape[0], outputs, -1)
    return values, scales


def _sizes_of(case, gen):
    """Sizes of a model's gradients: a few matrices hold nearly all of it, many vectors nearly nothing."""
    n, total = case["tensors"], case["total"]
    share = torch.exp(2.5 * torch.randn(n, generator=torch.Generator().manual_seed(n + total)))
    sizes = (share / share.sum() * (total - n)).long() + 1
    sizes[0] += total - int(sizes.sum())
    return sizes.tolist()


def prepare(case, seed):
    gen, kind, dtype = _generator(seed), case["kind"], TYPES[case["type"]]
    s = {"case": case}
    if kind == "quantize":
        x = _activations(case["experts"] * case["rows"], case["cols"], dtype, gen)
        s["x"] = x.view(case["experts"], case["rows"], case["cols"])
    elif kind == "linear":
        s["x"] = _activations(case["rows"], case["inputs"], dtype, gen)
        s["w"], s["ws"] = _weights4(1, case["outputs"], case["inputs"], gen)
    elif kind == "experts":
        T, E, k = case["tokens"], case["experts"], case["k"]
        s["x"] = _activations(T, case["inputs"], dtype, gen)
        s["w"], s["ws"] = _weights4(E, case["outputs"], case["inputs"], gen)
        popular = torch.randn(E, generator=gen, device="cuda") * (1.0 if case["skew"] else 0.0)
        logits = torch.randn((T, E), generator=gen, device="cuda") + popular
        ids = torch.argsort(logits, dim=1, descending=True)[:, :k].to(torch.int32)
        weights = torch.softmax(torch.gather(logits, 1, ids.long()), 1)
        if case["padding"]:
            out = torch.rand(T, generator=gen, device="cuda") < 0.03
            ids[out], weights[out] = -1, 0.0
        s["ids"], s["weights"] = ids.contiguous(), weights.contiguous()
    elif kind == "layer":
        T, E, D, H = case["tokens"], case["experts"], case["width"], case["hidden"]
        s["x"] = _activations(T, D, dtype, gen)
        popular = torch.randn(E, generator=gen, device="cuda") * 0.5
        s["logits"] = torch.randn((T, E), generator=gen, device="cuda") * 1.5 + popular
        if case["padding"]:
            s["logits"][T // 2] = -math.inf
        s["bias"] = -0.001 * torch.round(popular * 100.0) if case["bias"] else None
        make = _weights8 if case["bits"] == 8 else _weights4
        s["up"], s["up_scales"] = make(E, 2 * H, D, gen)                   # rows of the gate, then rows that it multiplies
        s["down"], s["down_scales"] = make(E, D, H, gen)
    else:
        sizes = _sizes_of(case, gen)
        s["grads"] = torch.empty(case["total"], dtype=dtype, device="cuda").normal_(generator=gen).split(sizes)
        for i, g in enumerate(s["grads"]):
            g.mul_(10.0 ** -(i % 4))                                        # (an infrequent parameter's are small)
        s["bucket"] = torch.empty(case["total"], dtype=TYPES[case["out"]], device="cuda")
        s["out"] = s["bucket"].split(sizes)
        norm = math.sqrt(sum(float((g.float() * g.float()).sum(dtype=torch.float64)) for g in s["grads"]))
        s["limit"] = norm * (0.37 if case["clipped"] else 1.9)
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------
def _exponents(b):
    """Exponents of the scales of blocks [..., 32] in 32 bits: the largest magnitude, were it rounded to a bit after its first, is at most 6
    of them."""
    top = b.abs().amax(-1)
    return (((top.view(torch.int32) + (1 << 21)) >> 23) - 129).clamp(LEAST, MOST)


def _nearest(v):
    """Which of the eight magnitudes of 4 bits is nearest to v's; of two as near the even one."""
    a = v.abs()
    return ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int())


def _magnitudes(device):
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=device)


def _rounded4(x):
    """x, whose last dimension is cut into blocks of 32, as its 4-bit values and scales say, in 32 bits."""
    cols = x.shape[-1]
    whole = torch.nn.functional.pad(x, (0, -cols % SMALL))
    b = whole.view(-1, SMALL)
    e = _exponents(b)[:, None]
    q = _magnitudes(x.device)[_nearest(torch.ldexp(b, -e))]
    return torch.ldexp(torch.where(b < 0, -q, q), e).view(whole.shape)[..., :cols]


def _rounded8(x):
    """The same in 8 bits, in blocks of 128."""
    cols = x.shape[-1]
    whole = torch.nn.functional.pad(x, (0, -cols % BLOCK))
    b = whole.view(*x.shape[:-1], -1, BLOCK)
    top = b.abs().amax(-1, keepdim=True).clamp_min(SMALLEST)
    q = (b * (LARGEST / top)).clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn).float()
    return (q * (top / LARGEST)).view(whole.shape)[..., :cols]


def _weights_are4(values, scales, cols):
    low, high = (values & 15).long(), (values >> 4).long()
    code = torch.stack([low, high], -1).view(*values.shape[:-1], -1)
    m = _magnitudes(values.device)
    v = torch.cat([m, -m])[code].view(*scales.shape, SMALL)
    return torch.ldexp(v, (scales.int() - 127)[..., None]).view(*values.shape[:-1], -1)[..., :cols]


def _weights_are8(values, scales, cols):
    n, kb = values.shape[-2], scales.shape[-1]
    rows = torch.arange(n, device=values.device) // BLOCK
    tiles = values.float().view(*values.shape[:-1], kb, BLOCK) * scales[..., rows, :][..., None]
    return tiles.view(values.shape)[..., :cols]


def _plain_quantize(s):
    return _rounded4(s["x"].float()).to(s["x"].dtype)


def _plain_linear(s):
    w = _weights_are4(s["w"][0], s["ws"][0], s["case"]["inputs"])
    return (_rounded4(s["x"].float()) @ w.t()).to(s["x"].dtype)


def _plain_experts(s):
    case, x, ids = s["case"], s["x"].float(), s["ids"].long()
    T, E, k, K, N = case["tokens"], case["experts"], case["k"], case["inputs"], case["outputs"]
    # every expert's rows begin a tile of their own, of 128 rows, or of one where there are few
    rows = BLOCK if T * k >= 2 * E else 1
    tiles = T * k // rows + min(E, T * k)
    flat, slots = ids.reshape(-1), torch.arange(T * k, device=x.device)
    group = torch.where(flat >= 0, flat, torch.full_like(flat, E))
    counts = (group[None, :] == torch.arange(E + 1, device=x.device)[:, None]).sum(1)
    first, tile_end = torch.cumsum(counts, 0) - counts, torch.cumsum((counts[:E] + rows - 1) // rows, 0)
    tile_first = torch.cat([tile_end - (counts[:E] + rows - 1) // rows, tile_end.new_full((1,), tiles)])
    order = torch.argsort(group, stable=True)
    sorted_group = group[order]
    at = tile_first[sorted_group] * rows + (slots - first[sorted_group]) * (sorted_group < E)
    slot_at = torch.full((tiles * rows + 1,), -1, device=x.device, dtype=torch.long)
    slot_at[at] = torch.where(sorted_group < E, order, torch.full_like(order, -1))
    place = torch.empty_like(flat)
    place[order] = at
    slot_at, there = slot_at[:-1], (slot_at[:-1] >= 0)[:, None]
    expert = torch.searchsorted(tile_end, torch.arange(tiles, device=x.device), right=True).clamp_max(E - 1)
    w = _weights_are4(s["w"][expert], s["ws"][expert], K)
    a = torch.where(there, _rounded4(x)[slot_at.clamp_min(0) // k], torch.zeros((), device=x.device)).view(tiles, rows, K)
    y = torch.cat([torch.bmm(a, w.transpose(1, 2)).view(-1, N), x.new_zeros((1, N))])
    return (s["weights"][:, :, None] * y[place].view(T, k, N)).sum(1).to(s["x"].dtype)


def _plain_route(s):
    """(ids, weights) of the experts with the k best keys: the logits, or with a bias the scores plus it."""
    case, l, bias = s["case"], s["logits"].float(), s["bias"]
    soft, k = case["score"] == "softmax", case["k"]
    if soft:
        e = torch.where(l == -math.inf, torch.zeros_like(l), torch.exp(l - l.amax(1, keepdim=True)))
        score = e / e.sum(1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-l))
    key = l if bias is None else torch.where(l == -math.inf, l, score + bias)
    order = torch.sort(key, dim=1, descending=True, stable=True)
    ids, there = order.indices[:, :k], order.values[:, :k] > -math.inf
    if soft and case["renormalize"]:
        chosen = torch.where(there, torch.gather(l, 1, ids), torch.full_like(l[:, :k], -math.inf))
        share = torch.where(there, torch.exp(chosen - chosen.amax(1, keepdim=True)), torch.zeros_like(chosen))
    else:
        share = torch.where(there, torch.gather(score, 1, ids), torch.zeros_like(l[:, :k]))
    total = share.sum(1, keepdim=True)
    part = torch.where(total > 0, share / total, torch.zeros_like(share)) if case["renormalize"] else share
    return torch.where(there, ids, torch.full_like(ids, -1)).to(torch.int32), part * case["scale"]


def _activated(u, case, erf, exp):
    gate, up = u[..., :case["hidden"]], u[..., case["hidden"]:]
    if case["gelu"]:
        return 0.5 * gate * (1.0 + erf(gate * math.sqrt(0.5))) * up
    return gate / (1.0 + exp(-gate)) * up


def _plain_layer(s):
    case, x = s["case"], s["x"].float()
    T, k, D, H = case["tokens"], case["k"], case["width"], case["hidden"]
    ids, weights = _plain_route(s)
    at = ids.reshape(-1).clamp_min(0).long()
    rounded, are = (_rounded8, _weights_are8) if case["bits"] == 8 else (_rounded4, _weights_are4)
    rows = rounded(x)[:, None].expand(T, k, D).reshape(T * k, D, 1)
    u = torch.bmm(are(s["up"][at], s["up_scales"][at], D), rows)[:, :, 0]
    h = rounded(_activated(u, case, torch.erf, torch.exp))
    y = torch.bmm(are(s["down"][at], s["down_scales"][at], H), h[:, :, None]).view(T, k, D)
    y = torch.where(ids[:, :, None] >= 0, weights[:, :, None] * y, torch.zeros_like(y)).sum(1)
    return {"y": y.to(s["x"].dtype), "ids": ids, "weights": weights}


def _plain_clip(s):
    total = torch.stack([(g.double() * g.double()).sum() for g in s["grads"]]).sum()
    norm = torch.sqrt(total)
    if s["case"]["norm_alone"]:
        return norm.float()
    factor = torch.where(norm > s["limit"], s["limit"] / norm, torch.ones_like(norm)).float()
    s["bucket"].copy_(torch.cat([g.float() * factor for g in s["grads"]]))
    return {"norm": norm.float(), "clipped": s["bucket"]}


# ---- the framework's calls ---------------------------------------------------------------------------------------
def _own_quantize(s):
    from paper_1505_04956_amd import micro
    return micro.expand(micro.quantize(s["x"]), s["x"].dtype)


def _own_linear(s):
    from paper_1505_04956_amd import micro
    return micro.linear(s["x"], micro.Micro(s["w"][0], s["ws"][0], s["case"]["inputs"]))


def _own_experts(s):
    from paper_1505_04956_amd import micro
    return micro.experts(s["x"], s["ids"], s["weights"], micro.Micro(s["w"], s["ws"], s["case"]["inputs"]))


def _own_layer(s):
    from paper_1505_04956_amd import experts, layer, micro
    c = s["case"]
    rule = experts.Rule(c["k"], score=experts.SOFTMAX if c["score"] == "softmax" else experts.SIGMOID, renormalize=c["renormalize"],
                        scale=c["scale"])
    kept = experts.Blocks if c["bits"] == 8 else micro.Micro
    y, ids, weights = layer.layer(s["x"], s["logits"], rule, kept(s["up"], s["up_scales"], c["width"]),
                                  kept(s["down"], s["down_scales"], c["hidden"]), bias=s["bias"],
                                  activation=layer.GELU if c["gelu"] else layer.SILU)
    return {"y": y, "ids": ids, "weights": weights}


def _own_clip(s):
    from paper_1505_04956_amd import gradients
    if s["case"]["norm_alone"]:
        return gradients.norm(s["grads"])
    return {"norm": gradients.clip(s["grads"], s["limit"], out=s["out"]), "clipped": s["bucket"]}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"quantize": _own_quantize, "linear": _own_linear, "experts": _own_experts, "layer": _own_layer, "clip": _own_clip}[kind](state)
    return {"quantize": _plain_quantize, "linear": _plain_linear, "experts": _plain_experts, "layer": _plain_layer, "clip": _plain_clip}[kind](state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def _bytes4(rows, cols):
    return rows * cols / 2 + rows * -(-cols // SMALL)


def _met(case):
    """Experts that some token goes to, were all as popular."""
    return case["experts"] * (1.0 - (1.0 - case["k"] / case["experts"]) ** case["tokens"])


def work(case):
    size = SIZE[case["type"]]
    if case["kind"] == "quantize":
        n = case["experts"] * case["rows"] * case["cols"]
        return {"bytes": 2 * n * size, "flops": 2 * n}
    if case["kind"] == "linear":
        rows, K, N = case["rows"], case["inputs"], case["outputs"]
        return {"bytes": rows * (K + N) * size + _bytes4(N, K), "flops": 2 * rows * N * K}
    if case["kind"] == "experts":
        T, k, K, N = case["tokens"], case["k"], case["inputs"], case["outputs"]
        return {"bytes": T * (K + N) * size + 8 * T * k + _met(case) * _bytes4(N, K), "flops": 2 * T * k * N * K}
    if case["kind"] == "layer":
        T, k, D, H = case["tokens"], case["k"], case["width"], case["hidden"]
        one = _bytes4(2 * H, D) + _bytes4(D, H) if case["bits"] == 4 else 3 * H * D + 4 * (_blocks_of(2 * H) * _blocks_of(D) + _blocks_of(D) * _blocks_of(H))
        return {"bytes": _met(case) * one + 2 * T * D * size + T * (4 * case["experts"] + 8 * k), "flops": 6 * T * k * D * H}
    n = case["total"]
    return {"bytes": n * size + (0 if case["norm_alone"] else n * SIZE[case["out"]]), "flops": (2 if case["norm_alone"] else 3) * n}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------
def _exact4(v):
    """v, a 32-bit number by definition, with its last dimension brought to 4 bits and back."""
    v = v.float().double()
    out = []
    for part in v.split(1 << 14, 0):
        cut = torch.nn.functional.pad(part, (0, -part.shape[-1] % SMALL)).unflatten(-1, (-1, SMALL))
        top = cut.abs().amax(-1, keepdim=True)
        e = torch.floor(torch.log2(top.clamp_min(1e-300)))
        e = e - (torch.exp2(e) > top).double() + (torch.exp2(e + 1) <= top).double()     # (a logarithm may be off next to a whole number)
        e = (e + (top >= 1.75 * torch.exp2(e)).double() - 2).clamp(LEAST, MOST)
        m = (cut / torch.exp2(e)).abs()
        step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
        near = (torch.round(m / step) * step).clamp_max(6.0)                             # (to even: of steps here, of the last bit in 4 bits)
        out.append((torch.sign(cut) * near * torch.exp2(e)).flatten(-2)[..., :part.shape[-1]])
    return torch.cat(out)


def _exact8(v):
    out = []
    for part in v.float().split(BLOCK, -1):
        top = part.abs().amax(-1, keepdim=True).clamp_min(SMALLEST)
        q = (part * (LARGEST / top)).clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
        out.append(q.double() * (top / LARGEST).double())
    return torch.cat(out, -1)


def _full4(values, scales, cols):
    v = values.int()
    code = torch.stack([v % 16, v // 16], -1).flatten(-2)
    m = code % 8
    size = torch.where(m < 2, 0.5 * m, torch.where(m % 2 == 0, 1.0, 1.5).double() * torch.exp2(torch.div(m, 2, rounding_mode="floor").double() - 1))
    grid = torch.exp2(scales.double() - 127).repeat_interleave(SMALL, -1)
    return (torch.where(code >= 8, -size, size) * grid)[..., :cols]


def _full8(values, scales, cols):
    grid = scales.double().repeat_interleave(BLOCK, -2).repeat_interleave(BLOCK, -1)
    return (values.double() * grid[..., :values.shape[-2], :values.shape[-1]])[..., :cols]


def _exact_experts(case, s):
    q, y = _exact4(s["x"]), torch.zeros((case["tokens"], case["outputs"]), dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        t, j = torch.nonzero(s["ids"] == e, as_tuple=True)
        if len(t):
            y[t] += s["weights"].double()[t, j][:, None] * (q[t] @ _full4(s["w"][e], s["ws"][e], case["inputs"]).t())
    return y


def _exact_layer(case, s):
    l, bias, k = s["logits"].double(), s["bias"], case["k"]
    inside = l > -math.inf
    p = torch.sigmoid(l) if case["score"] == "sigmoid" else torch.nan_to_num(torch.softmax(l, 1))
    rank = l if bias is None else (p + bias.double()).masked_fill(~inside, -math.inf)
    ids = torch.argsort(rank, dim=1, descending=True, stable=True)[:, :k]
    real = torch.gather(inside, 1, ids)
    w = torch.gather(p, 1, ids) * real
    if case["renormalize"]:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    w = w * case["scale"]
    to, full = (_exact8, _full8) if case["bits"] == 8 else (_exact4, _full4)
    q, y = to(s["x"]), torch.zeros((case["tokens"], case["width"]), dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        t, j = torch.nonzero((ids == e) & real, as_tuple=True)
        if len(t):
            u = q[t] @ full(s["up"][e], s["up_scales"][e], case["width"]).t()
            h = to(_activated(u, case, torch.erf, torch.exp))
            y[t] += w[t, j][:, None] * (h @ full(s["down"][e], s["down_scales"][e], case["hidden"]).t())
    return {"y": y, "ids": None, "weights": w}


def _exact_clip(case, s):
    norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(part.double()) ** 2) for g in s["grads"] for part in g.split(1 << 26)))
    if case["norm_alone"]:
        return torch.tensor(norm, dtype=torch.float64)
    factor = min(1.0, s["limit"] / norm) if norm else 1.0
    return {"norm": torch.tensor(norm, dtype=torch.float64), "clipped": torch.cat([g.double() for g in s["grads"]]).mul_(factor)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quantize":
        return _exact4(s["x"].flatten(0, 1)).view(s["x"].shape)
    if case["kind"] == "linear":
        return _exact4(s["x"]) @ _full4(s["w"][0], s["ws"][0], case["inputs"]).t()
    return {"experts": _exact_experts, "layer": _exact_layer, "clip": _exact_clip}[case["kind"]](case, s)
