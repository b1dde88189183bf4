"""Plain 64-bit implementations of what surrounds the projections of a transformer block (products with 4-bit weights, norms before and after a block, the AdamW step),
with how far fp32 arithmetic and the outputs' rounding may be from them.

u = 2^-23 stands for one fp32 operation, as in operators_ref; a sum of n products is off by at most (n + 8) u of the sum of their absolute values in any order; a
bf16 output by 2^-8 of its value, an fp32 one by 2^-24.  Errors are carried through to first order; SLACK covers their products."""
import torch

from tests.operators_ref import ROUND, U, check  # noqa: F401

SLACK = 1.01
E4M3_MAX = 448.0


def rounded(value, off, dtype):
    off = SLACK * off
    return value, off + ROUND[dtype] * (value.abs() + off)


# ---- 4-bit weights ------------------------------------------------------------------------------

def w4_weights(codes, scales, group):
    return codes.double() * scales.double().repeat_interleave(group, 1)[:, :codes.shape[1]]


def w4_quantise(W, group):
    """(codes, scales) by the INT family's rule, in fp32: s = amax / 7, c = rne(w (7 / amax)); a group of zeros has 1."""
    N, K = W.shape
    G = -(-K // group)
    v = torch.nn.functional.pad(W, (0, G * group - K)).view(N, G, group)
    amax = v.abs().amax(-1)
    seven = torch.full_like(amax, 7.0)
    inv = torch.where(amax == 0, torch.ones_like(amax), seven / amax)
    codes = (v * inv[:, :, None]).round().clamp(-7, 7).view(N, -1)[:, :K].to(torch.int8)
    return codes, torch.where(amax == 0, torch.ones_like(amax), amax / seven)


def w4_fwd(X, codes, scales, group, bias, dtype):
    W, x = w4_weights(codes, scales, group), X.double()
    b = torch.zeros(W.shape[0], dtype=torch.float64, device=X.device) if bias is None else bias.double()
    # three terms of an fp32 row make three sums; then the scales, the groups' and wavefronts' sums, the bias
    n = (3 if X.dtype == torch.float32 else 1) * X.shape[1]
    return rounded(x @ W.t() + b, (n + 24) * U * (x.abs() @ W.abs().t() + b.abs()), dtype)


def w4_bwd(dY, codes, scales, group, dtype):
    W, g = w4_weights(codes, scales, group), dY.double()
    return rounded(g @ W, (3 * dY.shape[1] + 24) * U * (g.abs() @ W.abs()), dtype)


# ---- norms before and after a block -------------------------------------------------------------

def rows_of(offsets, M, device):
    """Sequence of each row, -1 for rows of none."""
    if offsets is None:
        return torch.zeros(M, dtype=torch.int64, device=device)
    row = torch.arange(M, device=device)
    s = (row[:, None] >= offsets[None, 1:]).sum(1)
    return torch.where((s < offsets.shape[0] - 1) & (row >= offsets[0]), s, -1)


def norm(kind, x, eps, off=0.0):
    """(values, 1 / deviation, bound of the values' error, of the deviation's relative error) for rows x that are off by up to `off`."""
    D = x.shape[-1]
    if kind == "none":
        return x, torch.ones_like(x[:, :1]), off + torch.zeros_like(x), torch.zeros_like(x[:, :1])
    off = off + torch.zeros_like(x)
    if kind == "layer":
        m = x.mean(-1, keepdim=True)
        off = off + off.mean(-1, keepdim=True) + (D + 8) * U * x.abs().mean(-1, keepdim=True) + U * (x.abs() + m.abs())
        x = x - m
    r = 1.0 / ((x * x).mean(-1, keepdim=True) + eps).sqrt()
    rel = 0.5 * ((D + 10) * U + 2 * (x.abs() * off).mean(-1, keepdim=True) * r * r) + 4 * U
    n = x * r
    return n, r, r * off + n.abs() * (rel + U), rel


def norm_grad(kind, n, r, off_n, rel, dn, off_dn):
    """(gradient at the norm's input, bound)."""
    if kind == "none":
        return dn, off_dn
    D = n.shape[-1]
    u = (dn * n).mean(-1, keepdim=True)
    eu = (off_dn * n.abs() + dn.abs() * off_n).mean(-1, keepdim=True) + (D + 10) * U * (dn * n).abs().mean(-1, keepdim=True)
    w, ew = torch.zeros_like(u), torch.zeros_like(u)
    if kind == "layer":
        w = dn.mean(-1, keepdim=True)
        ew = off_dn.mean(-1, keepdim=True) + (D + 10) * U * dn.abs().mean(-1, keepdim=True)
    size = dn.abs() + w.abs() + (n * u).abs()
    return r * (dn - w - n * u), r * (off_dn + ew + off_n * u.abs() + n.abs() * eu + (4 * U + rel) * size)


def _vec(w, like):
    return torch.ones(like.shape[-1], dtype=torch.float64, device=like.device) if w is None else w.double()


def _mod(t, s, like, default):
    return torch.full_like(like, default) if t is None else t.double()[s]


def block_fwd(h, y, offsets, gate, scale, shift, w_post, w_pre, post, pre, eps, alpha, x_dtype):
    """dict of (value, bound) of the rows that belong to sequences: their numbers, ho, x."""
    rows = (rows_of(offsets, h.shape[0], h.device) >= 0).nonzero()[:, 0]
    s = rows_of(offsets, h.shape[0], h.device)[rows]
    H = h.double()[rows]
    out = dict(rows=rows)
    off = torch.zeros_like(H)
    if y is not None:
        p, _, op, _ = norm(post, y.double()[rows], eps)
        b = _mod(gate, s, H, 1.0) * _vec(w_post, H)
        ho = alpha * H + b * p
        off = b.abs() * op + 4 * U * ((alpha * H).abs() + (b * p).abs())
        out["ho"] = rounded(ho, off, h.dtype)
        H = ho
    n, _, on, _ = norm(pre, H, eps, off)
    a, c = (1.0 + _mod(scale, s, H, 0.0)) * _vec(w_pre, H), _mod(shift, s, H, 0.0)
    a_size = (1.0 + _mod(scale, s, H, 0.0).abs()) * _vec(w_pre, H).abs()  # (1 + scale may cancel)
    out["x"] = rounded(n * a + c, a.abs() * on + 4 * U * ((n * a_size).abs() + c.abs()), x_dtype)
    return out


def block_bwd(ho, y, offsets, gate, scale, w_post, w_pre, dho, dx, post, pre, eps, alpha, h_dtype, y_dtype):
    """dict of (value, bound) for dh, dy (of the rows of sequences), dgate, dscale, dshift, dw_post, dw_pre."""
    first = dx if dx is not None else dho
    where = rows_of(offsets, first.shape[0], first.device)
    rows = (where >= 0).nonzero()[:, 0]
    s = where[rows]
    S = 1 if offsets is None else offsets.shape[0] - 1
    member = (torch.arange(S, device=first.device)[:, None] == s).double()
    like = first.double()[rows]
    zero = torch.zeros_like(like)
    G, oG = (zero, zero) if dho is None else (dho.double()[rows], zero)
    out = dict(rows=rows)
    count = rows.numel() + 64  # additions that a value of a sum goes through, at most
    f32 = torch.float32
    wr, wp = _vec(w_pre, like), _vec(w_post, like)
    one = 1.0 + (torch.zeros(S, like.shape[1], dtype=torch.float64, device=like.device) if scale is None else scale.double())
    one_size = 2.0 + one.abs()
    g = torch.ones(S, like.shape[1], dtype=torch.float64, device=like.device) if gate is None else gate.double()
    if dx is not None:
        d = like if dx is first else dx.double()[rows]
        n, r, on, rel = norm(pre, ho.double()[rows], eps)
        dn = d * one[s] * wr
        t, ot = norm_grad(pre, n, r, on, rel, dn, 3 * U * (d * one_size[s] * wr).abs())
        G, oG = G + t, oG + ot + 2 * U * (G.abs() + t.abs())
        q = member @ (d * n)
        oq = member @ (d.abs() * on) + count * U * (member @ (d * n).abs())
        out["dshift"] = rounded(member @ d, count * U * (member @ d.abs()), f32)
        out["dscale"] = rounded(wr * q, wr.abs() * oq + 2 * U * (wr * q).abs(), f32)
        out["dw_pre"] = rounded((one * q).sum(0), (one_size * oq).sum(0) + (S + 8) * U * (one_size * q.abs()).sum(0), f32)
    a = alpha if y is not None else 1.0
    out["dh"] = rounded(a * G, abs(a) * oG + U * (a * G).abs(), h_dtype)
    if y is not None:
        p, r, op, rel = norm(post, y.double()[rows], eps)
        b = g[s] * wp
        dp = G * b
        out["dy"] = rounded(*norm_grad(post, p, r, op, rel, dp, b.abs() * oG + 3 * U * dp.abs()), y_dtype)
        q = member @ (G * p)
        oq = member @ (oG * p.abs() + G.abs() * op) + count * U * (member @ (G * p).abs())
        out["dgate"] = rounded(wp * q, wp.abs() * oq + 2 * U * (wp * q).abs(), f32)
        out["dw_post"] = rounded((g * q).sum(0), (g.abs() * oq).sum(0) + (S + 8) * U * (g * q).abs().sum(0), f32)
    return out


# ---- AdamW --------------------------------------------------------------------------------------

def adamw(p, g, m, v, lr, t, beta1, beta2, eps, wd, gs=1.0):
    """dict of (value, bound before the parameter's own rounding) of one step in 64 bits, of fp32 states.  e = 2^-24 is the rounding of an operation or of a constant."""
    e = 2.0 ** -24
    p, g, m, v = p.double(), g.double() * gs, m.double(), v.double()
    m1, om = beta1 * m + (1 - beta1) * g, 5 * e * ((beta1 * m).abs() + ((1 - beta1) * g).abs())
    v1 = beta2 * v + (1 - beta2) * g * g
    ov = 7 * e * v1                                    # no term is negative
    mh, vh = m1 / (1 - beta1 ** t), v1 / (1 - beta2 ** t)
    den = vh.sqrt() + eps
    # of the quotient: the correction's rounding and division, half of v's and of its correction's, the root, eps and the sum, the division, lr and its product
    step = lr * mh / den
    ostep = lr * om / (1 - beta1 ** t) / den + 14 * e * step.abs()
    keep = (1 - lr * wd) * p
    return dict(p=(keep - step, SLACK * (ostep + 5 * e * (p.abs() + step.abs()))), m=(m1, SLACK * om), v=(v1, SLACK * ov))


def power_scale(amax):
    """The smallest power of two s with amax <= 448 s (1 for zero)."""
    s = torch.exp2(torch.ceil(torch.log2(amax.double() / E4M3_MAX)))
    s = torch.where(amax.double() > E4M3_MAX * s, 2 * s, s)
    s = torch.where(amax.double() <= E4M3_MAX * s / 2, s / 2, s)
    return torch.where(amax == 0, torch.ones_like(s), s.clamp(min=2.0 ** -126)).float()


def random_bits(seed, t, count):
    """Two 20-bit numbers for each place, by the rule of the states in 8 bits, in 64-bit integers."""
    mask = 0xFFFFFFFF
    h = torch.arange(count, dtype=torch.int64) ^ ((seed * 0x9E3779B1 + t * 0x6A09E667) & mask)
    for k, shift in ((0x9E3779B1, 16), (0x6A09E667, 15), (0xBB67AE85, 16)):
        h = (h * k) & mask
        h = h ^ (h >> shift)
    return h & 0xFFFFF, ((h * 0x3C6EF373) & mask) >> 12


def e4m3_random(x, bits):
    """0 <= x <= 448 to the grid of E4M3: up where the cut part is above 1 - bits / 2^20 of a step."""
    x = x.double()
    step = torch.exp2(torch.floor(torch.log2(x.clamp(min=2.0 ** -6)))) / 8
    return torch.floor(x / step + bits.double() / 2 ** 20) * step
