"""Plain implementations in 64 bits of the loss, the embedding with its gradient, and dropout, with bounds on what the kernels'
roundings may add up to.  Tensors may live on any device.

Bounds.  U = 2^-24 is half a step of fp32, `half_step` that of a type.  A sum of n products or terms in fp32, in any order, is off
by at most n U (1 + small) times the sum of magnitudes; the matrix unit may cut off instead of rounding (a whole step), so its sums
count 2 n U.  SAFE covers terms of second order."""
import numpy as np
import torch

import paper_2512_14628_amd as pkg

U = 2.0 ** -24
SAFE = 1.01
TYPES = {pkg.TYPE_F32: torch.float32, pkg.TYPE_BF16: torch.bfloat16, pkg.TYPE_F16: torch.float16}


def half_step(kind):
    return torch.finfo(TYPES[kind]).eps / 2


def least(kind):
    """Half of the smallest step of a type (values below its normal range)."""
    f = torch.finfo(TYPES[kind])
    return f.tiny * f.eps / 2


def rounded(kind, value, bound):
    """The bound of a value that carries `bound` and is then rounded to the type."""
    return SAFE * (bound + half_step(kind) * (value.abs() + bound)) + least(kind)


def loss_reference(kind, X, W, labels, mean, scale, label=None):
    """{name: (value, bound)}; X, W of the type, labels int64.  Rows without a target are not looked at.  `label`: what the gradient of
    the label's own logit is off by, relative to itself, behind its fp32 steps (dX's share, G's); None: as the other classes'."""
    V, D = W.shape
    n = X.shape[0]
    f64 = torch.float64
    at = ((labels >= 0) & (labels < V)).nonzero()[:, 0]
    x, w, y = X[at].to(f64), W.to(f64), labels[at]
    rows = torch.arange(at.numel(), device=X.device)
    count = at.numel()
    l = x @ w.T
    # products of 16-bit values are exact in fp32, those of fp32 values are rounded: one more U
    dl = (x.abs() @ w.abs().T) * (2 * (D + 1) * U)
    worst = dl.amax(1) if count else dl.new_zeros(0)
    lse = torch.logsumexp(l, 1)
    p = torch.exp(l - lse[:, None])
    # exponentials: the difference's rounding and that of its product with log2 e move the exponent by 2 U |l - max|, weighted by the
    # term itself (t exp(-t) < 1), the instruction adds 2 U; sums of V terms, a factor for every join, the logarithm 2 U
    ds = (V + 64) * U
    dlse = worst + ds + 4 * U * (lse.abs() + l.abs().amax(1) if count else 0)
    loss = lse - l[rows, y]
    out = {}

    def spread(value, bound):
        a, b = value.new_zeros(n), value.new_zeros(n)
        a[at], b[at] = value, bound
        return a, b

    dloss = SAFE * (dlse + dl[rows, y] + 2 * U * (lse.abs() + loss.abs()))
    out["lse"] = spread(lse, SAFE * dlse)
    out["loss"] = spread(loss, dloss)
    div = max(count, 1) if mean else 1
    total = loss.sum() / div
    out["total"] = (total, dloss.sum() / div + 2 * U * total.abs())
    g = scale / div
    # p's own relative error: the logit's and the largest one's, the sum's, the exponential's (up to |l - max| 4 U); then the type's
    span = (l - l.amax(1, keepdim=True)).abs() if count else l
    dp = p * (dl + worst[:, None] + ds + 4 * U * (1 + span) + 4 * U)
    P = p.clone()
    P[rows, y] -= 1
    # (in 16 bits up to two roundings: of the exponential that is held, then of the gradient made of it)
    unit = 2.0 ** -15 if kind == pkg.TYPE_F16 else 1.0
    dP = dp + SAFE * (P.abs() + dp) * (2 * half_step(kind) + 4 * U) + 2 * unit * least(kind) + (2.0 ** -125 if kind != pkg.TYPE_F32 else 0)
    dPx, dPw = dP, dP
    if label is not None:
        dPx, dPw = dP.clone(), dP.clone()
        own = dp[rows, y] + SAFE * (P[rows, y].abs() + dp[rows, y]) * 4 * U
        for share, into in zip(label, (dPx, dPw)):
            into[rows, y] = own + SAFE * share * P[rows, y].abs() + (2 * unit * least(kind) if share else 0)
    dx = (P @ w) * g
    ddx = abs(g) * (dPx @ w.abs() + 2 * (V + 64) * U * ((P.abs() + dPx) @ w.abs())) + 4 * U * dx.abs()
    a, b = X.new_zeros((n, D), dtype=f64), X.new_zeros((n, D), dtype=f64)
    a[at], b[at] = dx, rounded(kind, dx, ddx)
    out["dX"] = (a, b)
    dw = (P.T @ x) * g
    ddw = abs(g) * (dPw.T @ x.abs() + 2 * (count + 2) * U * ((P.abs() + dPw).T @ x.abs())) + 4 * U * dw.abs()
    out["G"] = (dw, ddw)             # before it is rounded (or added and rounded)
    return out


def embedding_reference(kind, W, ids, scale):
    V = W.shape[0]
    token = (ids >= 0) & (ids < V)
    y = torch.where(token[:, None], W[torch.where(token, ids, 0)].double() * scale, 0.0)
    return y, rounded(kind, y, y.abs() * U)


def embedding_gradient_reference(V, dY, ids, scale):
    """Value and bound before the rounding: a row's terms are added one by one, in parts or not, then scaled."""
    token = ((ids >= 0) & (ids < V)).nonzero()[:, 0]
    f64 = torch.float64
    total, size = (torch.zeros((V, dY.shape[1]), dtype=f64, device=dY.device) for _ in range(2))
    many = torch.zeros(V, dtype=f64, device=dY.device)
    total.index_add_(0, ids[token], dY[token].to(f64))
    size.index_add_(0, ids[token], dY[token].to(f64).abs())
    many.index_add_(0, ids[token], torch.ones(token.numel(), dtype=f64, device=dY.device))
    return total * scale, abs(scale) * (many[:, None] + 2) * U * size


def philox_words(groups, call, seed):
    """Philox4x32-10 with Python's whole numbers kept in numpy's 64 bits: [groups, 4]."""
    low, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    g = np.asarray(groups, np.uint64)
    c = [g & low, g >> s32, np.full_like(g, call & 0xFFFFFFFF), np.full_like(g, call >> 32)]
    for r in range(10):
        k = [np.uint64(((seed & 0xFFFFFFFF) + r * 0x9E3779B9) & 0xFFFFFFFF), np.uint64(((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)]
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> s32) ^ c[1] ^ k[0], b & low, (a >> s32) ^ c[3] ^ k[1], a & low]
    return np.stack(c, -1)


def dropout_kept(n, p, seed, call, first=0):
    """Which of the elements first .. first + n - 1 stay, and the factor of those that do."""
    groups = np.arange(first // 8, (first + n + 7) // 8, dtype=np.uint64)
    w = philox_words(groups, call, seed)
    halves = np.stack((w & np.uint64(0xFFFF), w >> np.uint64(16)), -1).reshape(-1)[first % 8:first % 8 + n]
    t = min(65535, int(np.floor(65536 * p + 0.5)))
    return halves >= t, 65536 / (65536 - t)


def dropout_reference(kind, X, kept, factor, residual=None):
    y = torch.where(kept, X.double() * factor, 0.0)
    bound = y.abs() * 2 * U
    if residual is not None:
        y = y + residual.double()
        bound = bound + U * (y.abs() + bound)
    # (to nearest, a value of half a step above the type's largest or more is infinite: fp16 65504 + 16, and the factor is up to 65536)
    f = torch.finfo(TYPES[kind])
    over = y.abs() >= f.max * (1 + 2 * half_step(kind) / (4 - 2 * f.eps))
    return torch.where(over, torch.copysign(torch.full_like(y, float("inf")), y), y), rounded(kind, y, bound)


def close(got, value, bound, what=""):
    off = (got.double() - value).abs()
    bad = ~((off <= bound) | (got.double() == value))
    assert not bad.any(), "%s: %d of %d off, at %s: got %s, want %s, bound %s" % (
        what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), got[bad][0].item(), value[bad][0].item(), bound[bad][0].item())
