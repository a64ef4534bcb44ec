"""4-bit blocks and layers of experts in 64 bits, from their definitions, on the CPU."""
import numpy as np
import torch

from tests import experts_rules as R

U = R.U
NUMBERS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
BORDERS = (NUMBERS[1:] + NUMBERS[:-1]) / 2
SMALL, RUN = 32, 256


def exponents(top):
    """Exponents of the scales of blocks with these largest magnitudes (64-bit tensors of finite numbers)."""
    m, e = np.frexp(top.numpy())                                    # top = m * 2^e, m in [0.5, 1)
    e = e - 3 + (m >= 0.875)
    return torch.from_numpy(np.where(top.numpy() == 0, -126, np.clip(e, -126, 125)).astype(np.int64))


def nearest(v):
    """Which of the eight numbers is nearest to |v|, of two as near the even one."""
    a = v.abs()
    up = torch.searchsorted(BORDERS, a, right=False)                # borders below a
    tie = torch.zeros_like(up, dtype=torch.bool)
    for i, b in enumerate(BORDERS.tolist()):
        tie |= (a == b) & (i % 2 == 1)                              # between i (odd) and i + 1 (even): up
    return up + tie.long()


def to_four(x):
    """x [rows, cols] (values float32 can hold) to (codes [rows, whole] 0 .. 15, scale bytes [rows, whole / 32]), whole runs of 256."""
    v = torch.nn.functional.pad(x.double(), (0, -x.shape[1] % RUN)).view(x.shape[0], -1, SMALL)
    bad = ~torch.isfinite(v).all(-1)
    w = torch.where(bad[..., None], torch.zeros_like(v), v)
    e = exponents(w.abs().amax(-1))
    q = nearest(w * torch.exp2(-e.double())[..., None])
    code = q + 8 * torch.signbit(w).long()
    return code.view(x.shape[0], -1), torch.where(bad, torch.full_like(e, 255), e + 127)


def packed(code):
    c = code.view(code.shape[0], -1, 2)
    return (c[..., 0] + 16 * c[..., 1]).to(torch.uint8)


def from_four(code, scales):
    """64-bit matrix of codes [..., n] and scale bytes [..., n / 32]."""
    s = torch.where(scales.long() == 255, torch.full(scales.shape, float("nan"), dtype=torch.float64), torch.exp2(scales.double() - 127))
    v = NUMBERS[code.long() % 8] * torch.where(code.long() >= 8, -1.0, 1.0).double()
    return v * s.repeat_interleave(SMALL, -1)


def codes(values):
    v = values.cpu().long()
    return torch.stack([v % 16, v // 16], -1).flatten(-2)


def matrix_of(m):
    """64-bit [..., rows, cols] that a Micro on the GPU stands for."""
    return from_four(codes(m.values), m.scales.cpu())[..., :m.cols]


def four(x):
    code, s = to_four(x)
    return from_four(code, s)[:, :x.shape[1]]


def product_bound(magnitudes, K):
    """Errors of a product in 4 bits: an instruction, 128 columns, is within 2 units of 2^-24 ... of the magnitudes that it and those before it
    added (measured: 1.21e-7 = 2.03 U, so 3 U here); then up to sixteen partial sums are added, a half-unit each."""
    return magnitudes * (3 * (K / 128 + 2) + 16) * U


def eight_bound(magnitudes, K):
    """Errors of a product in 8 bits whose blocks are summed by the 16-bit instruction, as in the tests of the 8-bit products: 4 sums of 32
    within 6 half-units, a scale, an addition a block; then sixteen partial sums."""
    return magnitudes * ((4 * 6 + 4 + K / 128) * 2 + 16) * U


def activated(g, u, gelu):
    f = 0.5 * g * (1 + torch.erf(g / 2 ** 0.5)) if gelu else g * torch.sigmoid(g)
    return f * u


def activated_bound(g, u, dg, du, gelu):
    """How far a 32-bit f(g) u is off: both derivatives are below 1.13; the exponential, the division or the error function and three products
    are within 12 half-units of f, those of 1 + erf of 4 half-units of |g|."""
    f = activated(g, torch.ones_like(u), gelu)
    return (1.13 * dg + 12 * U * f.abs() + (4 * U * g.abs() if gelu else 0)) * (u.abs() + du) + f.abs() * du + 2 * U * (f * u).abs() + 1e-37


def four_bound(h, d):
    """(4-bit values of h, how far those of any h' within d of h may be): a rounding may fall the other way, and so may a block's scale."""
    pad = -h.shape[1] % SMALL
    v, dd = (torch.nn.functional.pad(t, (0, pad)).view(h.shape[0], -1, SMALL) for t in (h, d))
    of = lambda w, e: torch.sign(w) * NUMBERS[nearest(w * torch.exp2(-e.double()))] * torch.exp2(e.double())  # noqa: E731
    top = v.abs()
    e0 = exponents(top.amax(-1))[..., None]
    value, off = of(v, e0), torch.zeros_like(v)
    for e in (exponents((top - dd).clamp_min(0).amax(-1))[..., None], exponents((top + dd).amax(-1))[..., None]):
        for w in (v - dd, v + dd):
            off = torch.maximum(off, (of(w, e) - value).abs())
    flat = lambda t: t.view(h.shape[0], -1)[:, :h.shape[1]]  # noqa: E731
    return flat(value), flat(off)


def _e4m3(x):
    return x.float().clamp(-448, 448).to(torch.float8_e4m3fn).double()


def eight_bound_of(h, d):
    """The same in 8 bits: a value times the scale's inverse is off by d and by what the largest is off, and three roundings."""
    pad = -h.shape[1] % R.BLOCK
    v, dd = (torch.nn.functional.pad(t, (0, pad)).view(h.shape[0], -1, R.BLOCK) for t in (h, d))
    top = v.abs().amax(-1, keepdim=True).clamp_min(R.SMALLEST)
    dt = dd.amax(-1, keepdim=True)
    value = _e4m3(v * (448 / top)) * (top / 448)
    off = torch.zeros_like(v)
    rel = (dt / top + 6 * U).clamp_max(0.5)
    for w in (v - dd, v + dd):
        for s in (1 - 2 * rel, 1 + 2 * rel):
            off = torch.maximum(off, (_e4m3(w * (448 / top) * s) * (top / 448) - value).abs() * (1 + 2 * rel))
    off = off + value.abs() * 2 * rel
    flat = lambda t: t.view(h.shape[0], -1)[:, :h.shape[1]]  # noqa: E731
    return flat(value), flat(off)


def layer(x, ids, weights, up, down, bits, gelu):
    """(y, bound) in 64 bits of a layer on rows x (values float32 can hold); up [E, 2H, D] and down [E, N, H] are 64-bit matrices, ids and
    weights the ones that were used.  The bound is on a 32-bit result, before its last rounding."""
    T, k, H = x.shape[0], ids.shape[1], down.shape[2]
    to = four if bits == 4 else R.rounded
    bound, of_h = (product_bound, four_bound) if bits == 4 else (eight_bound, eight_bound_of)
    q = to(x)
    y, off = torch.zeros(T, down.shape[1], dtype=torch.float64), torch.zeros(T, down.shape[1], dtype=torch.float64)
    total = torch.zeros_like(y)
    for t in range(T):
        for j in range(k):
            e = int(ids[t, j])
            if e < 0:
                continue
            u = up[e] @ q[t]
            du = bound(up[e].abs() @ q[t].abs(), x.shape[1])
            h = activated(u[:H], u[H:], gelu)
            dh = activated_bound(u[:H], u[H:], du[:H], du[H:], gelu)
            v, dv = of_h(h[None], dh[None])
            w = float(weights[t, j])
            part = down[e] @ v[0]
            mags = down[e].abs() @ (v[0].abs() + dv[0])
            y[t] += w * part
            off[t] += abs(w) * (down[e].abs() @ dv[0] + bound(mags, H))
            total[t] += abs(w) * mags
    return y, off + total * (k * H / 128 + 40) * U
