"""The routed experts in 64 bits, from their definitions, on the CPU; and what the 32-bit steps of the definitions are."""
import torch

BLOCK, LARGEST, SMALLEST = 128, 448.0, 1e-30
U = 2.0 ** -24                                   # half a unit in the last place of 32-bit numbers


def blocks(n):
    return -(-n // BLOCK)


def inside(logits, bias):
    ok = logits.double() > -float("inf")
    ok |= torch.isnan(logits.double())
    return ok if bias is None else ok & (bias.double() != -float("inf"))


def scores(logits, score, bias):
    """[T, E] scores in 64 bits, 0 where an expert is out."""
    l, ok = logits.double(), inside(logits, bias)
    if score == "sigmoid":
        return torch.where(ok, torch.sigmoid(l), torch.zeros_like(l))
    masked = torch.where(ok, l, torch.full_like(l, -1e300))
    e = torch.where(ok, torch.exp(masked - masked.amax(1, keepdim=True)), torch.zeros_like(l))
    return e / e.sum(1, keepdim=True).clamp_min(1e-300)


def keys(logits, score, bias):
    ok = inside(logits, bias)
    k = logits.double() if bias is None else scores(logits, score, bias) + bias.double()
    return torch.where(ok, k, torch.full_like(k, -float("inf")))


def group_values(logits, score, bias, groups, two):
    by = keys(logits, score, bias)
    if two and bias is None:
        s = scores(logits, score, bias)
        by = torch.where(inside(logits, bias), s, torch.full_like(s, -float("inf")))
    best = torch.sort(by.view(by.shape[0], groups, -1), dim=2, descending=True).values
    return best[:, :, 0] + best[:, :, 1] if two else best[:, :, 0]


def choose(logits, score, bias, k, groups, kept, two):
    """ids by the definition (keys in 64 bits; ties lowest index first)."""
    key = keys(logits, score, bias).clone()
    T, E = key.shape
    if groups > 1:
        value = group_values(logits, score, bias, groups, two)
        order = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :kept]
        stays = torch.zeros(T, groups, dtype=torch.bool).scatter_(1, order, True)
        key[~stays.repeat_interleave(E // groups, 1)] = -float("inf")
    o = torch.sort(key, dim=1, descending=True, stable=True)
    ids = o.indices[:, :k].clone()
    ids[o.values[:, :k] == -float("inf")] = -1
    return ids.int()


def chosen_weights(logits, score, bias, ids, renormalize, scale, differentiable=False):
    """weights of given ids in 64 bits; `logits` may be a 64-bit leaf."""
    l, ok, there = logits.double(), inside(logits.detach(), bias), ids >= 0
    at = ids.clamp_min(0).long()
    if score == "sigmoid":
        s = torch.sigmoid(torch.where(ok, l, torch.zeros_like(l)))
        share = torch.gather(s, 1, at) * there
        if renormalize:
            total = share.sum(1, keepdim=True)
            share = share / torch.where(total > 0, total, torch.ones_like(total))
    elif renormalize:
        c = torch.where(there, torch.gather(l, 1, at), torch.full_like(share_like(l, ids), -1e300))
        e = torch.exp(c - c.detach().amax(1, keepdim=True)) * there
        share = e / e.sum(1, keepdim=True).clamp_min(1e-300)
    else:
        m = torch.where(ok, l, torch.full_like(l, -1e300))
        e = torch.exp(m - m.detach().amax(1, keepdim=True)) * ok
        share = torch.gather(e / e.sum(1, keepdim=True).clamp_min(1e-300), 1, at) * there
    return share * scale


def share_like(l, ids):
    return l.new_zeros(ids.shape)


def scale_of(top):
    """(scale, inverse) of blocks with these largest magnitudes, in the 32-bit steps of the definition."""
    bad = ~torch.isfinite(top)
    m = torch.where(bad, torch.ones_like(top), top).clamp_min(SMALLEST)
    scale = m * torch.tensor(1.0 / LARGEST, dtype=torch.float32)
    inverse = torch.tensor(LARGEST, dtype=torch.float32) * torch.reciprocal(m)
    return torch.where(bad, torch.full_like(top, float("nan")), scale), inverse


def to_blocks(x):
    """x [rows, cols] float32 to (values [rows, kb, 128] e4m3, scales [kb, rows]) in blocks along the columns."""
    rows, cols = x.shape
    w = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    top = torch.where(torch.isfinite(w), w, torch.full_like(w, float("inf"))).abs().amax(-1)
    scale, inverse = scale_of(top)
    q = (w * inverse[:, :, None]).clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
    return q, scale.t().contiguous()


def to_squares(x):
    rows, cols = x.shape
    w = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK, 0, -rows % BLOCK)).view(blocks(rows), BLOCK, blocks(cols), BLOCK)
    scale, inverse = scale_of(w.abs().amax((1, 3)))
    q = (w * inverse[:, None, :, None]).clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
    return q.view(blocks(rows) * BLOCK, -1)[:rows], scale


def from_blocks(values, scales):
    """64-bit matrix [rows, 128 * kb] of values [rows, 128 * kb] or [rows, kb, 128] and scales [kb, rows]."""
    kb, rows = scales.shape
    return (values.double().view(rows, kb, BLOCK) * scales.t().double()[:, :, None]).reshape(rows, kb * BLOCK)


def from_squares(values, scales):
    grid = scales.double().repeat_interleave(BLOCK, 0).repeat_interleave(BLOCK, 1)
    return values.double() * grid[:values.shape[0]]


def rounded(x):
    """x as its 8-bit blocks say, in 64 bits, its own columns."""
    return from_blocks(*to_blocks(x))[:, :x.shape[1]]


def order_of(ids, E):
    """(offsets, blocks, slots, places) of ids [T, k], as lists."""
    flat = ids.reshape(-1).tolist()
    rows = [[s for s, e in enumerate(flat) if e == x] for x in range(E)] if len(flat) * E < 1 << 22 else None
    if rows is None:
        rows = [[] for _ in range(E)]
        for s, e in enumerate(flat):
            if 0 <= e < E:
                rows[e].append(s)
    offsets, blks, slots, places = [0], [0], [], [-1] * len(flat)
    for r in rows:
        for s in r:
            places[s] = len(slots)
            slots.append(s)
        offsets.append(len(slots))
        blks.append(blks[-1] + blocks(len(r)))
    return offsets, blks, slots + [-1] * (len(flat) - len(slots)), places
