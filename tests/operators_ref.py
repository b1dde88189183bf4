"""Plain 64-bit implementations of the operators around a quantised projection, with how far fp32 sums and the outputs' rounding may be from them.

u = 2^-23 stands for one fp32 operation (twice the unit roundoff: the matrix core's own rounding is not documented); a sum of n products is off by at most
(n + 8) u of the sum of their absolute values in any order; a bf16 output by 2^-8 of its value, an fp32 one by 2^-24."""
import torch

U = 2.0 ** -23
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24, torch.float64: 0.0}


def masked(A, B, ranks):
    """The pool in 64 bits, zeros beyond each adapter's rank (whatever the arrays hold there)."""
    R = A.shape[1]
    keep = torch.arange(R, device=A.device)[None, :] < ranks.clamp(0, R)[:, None]
    return torch.where(keep[:, :, None], A.double(), 0.0), torch.where(keep[:, None, :], B.double(), 0.0)


def adapter_fwd(X, Yin, A, B, ranks, scales, ids):
    """(Y, bound on what a right answer in bf16 is off by)."""
    A, B = masked(A, B, ranks)
    Y, off = Yin.double(), torch.zeros(Yin.shape, dtype=torch.float64, device=X.device)
    K, R = A.shape[2], A.shape[1]
    for s in range(A.shape[0]):
        m = (ids == s).nonzero()[:, 0]
        if m.numel() == 0:
            continue
        x, c = X[m].double(), scales[s].double()
        T = x @ A[s].t()
        Tabs = x.abs() @ A[s].abs().t()
        Y[m] += c * (T @ B[s].t())
        # T: K products and the cut to two bf16 terms (2^-16 covers both and the scale's product); then two sums of R products and the last addition
        off[m] = c.abs() * (((K + 8) * U * Tabs + 2.0 ** -16 * T.abs()) @ B[s].abs().t() + (2 * R + 10) * U * (T.abs() @ B[s].abs().t()))
    off += 4 * U * Yin.double().abs()
    return Y, off + ROUND[torch.bfloat16] * (Y.abs() + off)


def adapter_bwd(X, dXin, A, B, ranks, scales, ids, dY):
    """dict of (value, bound) for dX, dA, dB."""
    dtype = X.dtype
    A, B = masked(A, B, ranks)
    f = dict(dtype=torch.float64, device=X.device)
    dX = torch.zeros(X.shape, **f) if dXin is None else dXin.double()
    oX, dA, dB, oA, oB = torch.zeros(X.shape, **f), torch.zeros_like(A), torch.zeros_like(B), torch.zeros_like(A), torch.zeros_like(B)
    K, R, N = A.shape[2], A.shape[1], B.shape[1]
    cut = 2.0 ** -16 if dtype == torch.bfloat16 else 2.0 ** -22
    base = dX.abs()
    for s in range(A.shape[0]):
        m = (ids == s).nonzero()[:, 0]
        if m.numel() == 0:
            continue
        n = m.numel()
        x, c, g = X[m].double(), scales[s].double(), dY[m].double()
        T, Tabs = x @ A[s].t(), x.abs() @ A[s].abs().t()
        dT, dTabs = g @ B[s], g.abs() @ B[s].abs()
        dX[m] += c * (dT @ A[s])
        oX[m] = c.abs() * (((N + 8) * U * dTabs + cut * dT.abs()) @ A[s].abs() + (3 * R + 10) * U * (dT.abs() @ A[s].abs()))
        dA[s], dB[s] = c * (dT.t() @ x), c * (g.t() @ T)
        # three terms hold all of T (dT), six products all but 2^-22 of theirs; up to six sums of n products, their parts and the scale
        oA[s] = c.abs() * (((N + 8) * U * dTabs).t() @ x.abs() + (6 * n + 64) * U * (dT.abs().t() @ x.abs()))
        oB[s] = c.abs() * (g.abs().t() @ ((K + 8) * U * Tabs) + (3 * n + 64) * U * (g.abs().t() @ T.abs()))
    oX = oX + 4 * U * base
    r32 = ROUND[torch.float32]
    return dict(dX=(dX, oX + ROUND[dtype] * (dX.abs() + oX)), dA=(dA, oA + r32 * (dA.abs() + oA)), dB=(dB, oB + r32 * (dB.abs() + oB)))


def _turn(pos, inv_freq, pairs, M):
    axis = [a for a, p in enumerate(pairs) for _ in range(p)]
    if not axis:
        return None
    rows = pos.double()[torch.arange(M, device=pos.device) % pos.shape[0]]
    t = rows[:, axis] * inv_freq.double()
    return torch.cos(t)[:, None, :], torch.sin(t)[:, None, :]


def _members(D, P, pairing):
    i = torch.arange(P)
    return (i, i + P) if pairing == "half" else (2 * i, 2 * i + 1)


def _rotate(y, cs, a, b, sign=1.0):
    if cs is None:
        return y
    c, s = cs[0], sign * cs[1]
    out = y.clone()
    out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., a] * s + y[..., b] * c
    return out


def _both(y, a, b, P):
    """|value| of each value, of a rotated one |a| + |b| of its pair."""
    out = y.abs().clone()
    if P:
        out[..., a] = out[..., b] = y[..., a].abs() + y[..., b].abs()
    return out


def qk_fwd(x, w, pos, inv_freq, pairs, pairing, norm, eps):
    """(value, bound) of the heads x (M x H x D)."""
    M, H, D = x.shape
    P = sum(pairs)
    a, b = _members(D, P, pairing)
    cs = _turn(pos, inv_freq, pairs, M)
    n = x.double()
    if norm:
        n = n / ((n * n).mean(-1, keepdim=True) + eps).sqrt() * (1.0 if w is None else w.double())
    y = _rotate(n, cs, a, b)
    # the mean's relative error is at most (D + 8) u / 2, half of it in the root; an angle's 2^-24 of half a turn, cosine and sine 4 u
    off = ((D / 4 + 12) * U + 4e-7) * _both(n, a, b, P)
    return y, off + ROUND[x.dtype] * (y.abs() + off)


def qk_bwd(x, w, pos, inv_freq, pairs, pairing, norm, eps, dy, chain=512):
    """((dx, bound), (dw, bound) or None).  chain: additions that a value of dw goes through one after another."""
    M, H, D = dy.shape
    P = sum(pairs)
    a, b = _members(D, P, pairing)
    cs = _turn(pos, inv_freq, pairs, M)
    g = _rotate(dy.double(), cs, a, b, -1.0)
    gabs = _both(dy.double(), a, b, P)
    c = (D / 2 + 24) * U + 6e-7
    if not norm:
        off = c * gabs
        return (g, off + ROUND[dy.dtype] * (g.abs() + off)), None
    w = torch.ones(D, dtype=torch.float64, device=dy.device) if w is None else w.double()
    rstd = 1.0 / ((x.double() ** 2).mean(-1, keepdim=True) + eps).sqrt()
    xh = x.double() * rstd
    dw, dwabs = (g * xh).sum((0, 1)), (gabs * xh.abs()).sum((0, 1))
    gw = g * w
    dx = rstd * (gw - xh * (gw * xh).mean(-1, keepdim=True))
    gwabs = gabs * w.abs()
    off = c * rstd * (gwabs + xh.abs() * (gwabs * xh.abs()).mean(-1, keepdim=True))
    return (dx, off + ROUND[dy.dtype] * (dx.abs() + off)), (dw, (c + chain * U) * dwabs)


def check(got, want, what):
    value, bound = want
    assert got.shape == value.shape, what
    far = (got.double() - value).abs() - bound
    assert not torch.isnan(far).any(), f"{what}: NaN"
    assert (far <= 0).all(), f"{what}: {int((far > 0).sum())} of {far.numel()} values off, the worst by {float(far.max()):.3g} beyond its bound"
