"""Plain 64-bit implementations of the operators that fit the output layer and hold it
in four bits (cross entropy and its gradients, clipping by the norm, microscaled
4-bit matrices), on the CPU, and the error bounds that 32-bit sums of the same
formulas keep (plain_scores has the rules)."""
import math

import torch

from plain_scores import EPS, rounding


def cross_entropy(x, weight, target, bias=None, grad=None):
    """dict of the loss, dx, dweight, dbias in 64 bits, and "bounds" of each; tensors on the CPU."""
    N, P, dtype = x.shape[0], weight.shape[0], x.dtype
    X, W, t = x.double(), weight.double(), target.long()
    b = torch.zeros(P, dtype=torch.float64) if bias is None else bias.double()
    z = X @ W.T + b
    fin = lambda v: torch.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0)  # noqa: E731
    err = (X.shape[1] + 8) * EPS * (fin(X).abs() @ fin(W).abs().T + fin(b).abs())  # of a logit: a sum of D products and the bias
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = e.sum(1, keepdim=True)
    p = e / total
    has = (t >= 0) & (t < P)
    label = t.clamp(0, P - 1)[:, None]
    zt = z.gather(1, label)
    loss = torch.where(total == 0, torch.full_like(top, math.inf), top - zt + total.log())[:, 0]
    away = fin((z - top).abs())
    # a term of the sum: its logit's error, that of its exponent's product and of the exponential; then the sum
    pe = fin(p) * (err + 4 * EPS * away + 4 * EPS)
    lerr = pe.sum(1, keepdim=True) + (P / 64 + 64) * EPS
    lbound = (lerr + err.gather(1, label) + 4 * EPS * (fin((top - zt).abs()) + fin(total.log().abs())))[:, 0]
    # (the largest logit's own error is in its term and in top - zt)
    lbound = lbound + (err * (z == top)).amax(1)
    g = torch.ones(N, dtype=torch.float64) if grad is None else grad.double()
    inside = has & (g != 0) & (total[:, 0] != 0)
    dz = p.clone()
    dz[torch.arange(N), label[:, 0]] -= 1.0
    dz = torch.where(inside[:, None], g[:, None] * dz, torch.zeros((), dtype=torch.float64))
    near = fin(p) * (err + (err * (z == top)).amax(1, keepdim=True) + lerr + 4 * EPS * away + 8 * EPS) + 2 * EPS * fin(dz / torch.where(g == 0, 1.0, g)[:, None]).abs()
    if N > 64 and X.shape[1] >= 512:  # exponentials held in 20 bits on their way
        near = near + 2.0 ** -18 * fin(p) + 2.0 ** -32
    derr = torch.where(inside[:, None], fin(g).abs()[:, None] * near, torch.zeros((), dtype=torch.float64))
    rel, least = rounding(dtype)
    if dtype is torch.float16:  # times a power of two that takes the largest |g| to 2^14 at least
        least = least * 2.0 ** -14 * 2 * float(fin(g).abs().max()) if N else 0.0
    rounded = derr + rel * (fin(dz).abs() + derr) + least * inside[:, None]
    Xin = torch.where(inside[:, None], X, torch.zeros((), dtype=torch.float64))
    out = dict(loss=torch.where(has, loss, torch.zeros((), dtype=torch.float64)),
               dx=torch.where(inside[:, None], dz @ W, torch.zeros((), dtype=torch.float64)), dweight=dz.T @ Xin, dbias=dz.sum(0))
    xe = rounded @ fin(W).abs() + (P + 16) * EPS * (fin(dz).abs() @ fin(W).abs())
    we = rounded.T @ fin(Xin).abs() + (N + 16) * EPS * (fin(dz).abs().T @ fin(Xin).abs())
    be = derr.sum(0) + (N + 16) * EPS * fin(dz).abs().sum(0)
    orel, oleast = rounding(dtype)
    out["bounds"] = dict(loss=lbound + EPS * fin(loss).abs(), dx=xe * (1 + orel) + orel * fin(out["dx"]).abs() + oleast,
                         dweight=we * (1 + orel) + orel * fin(out["dweight"]).abs() + oleast, dbias=be + EPS * fin(out["dbias"]).abs() + 1e-40)
    return out


def clip(tensors, max_norm):
    """(norm, scaled tensors) in 64 bits."""
    norm = math.sqrt(sum(float((t.double() ** 2).sum()) for t in tensors))
    by = max_norm / norm if max_norm < norm < math.inf else 1.0
    return norm, [t.double() * by for t in tensors]


CODES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def micro(x):
    """(codes [rows, D] 0..15, scale bytes [rows, ceil(D/32)]) by the definition, one value at a time."""
    rows, D = x.shape
    codes, scales = torch.zeros(rows, D, dtype=torch.int64), torch.zeros(rows, (D + 31) // 32, dtype=torch.int64)
    for n in range(rows):
        for c in range(0, D, 32):
            v = [float(a) for a in x[n, c:c + 32].double()]
            top = max(abs(a) if not math.isnan(a) else math.inf for a in v)
            if math.isinf(top):
                scales[n, c // 32] = 255
                continue
            s = max(math.frexp(top)[1] - 1 + 125, 0) if top > 0 else 0
            scales[n, c // 32] = s
            for i, a in enumerate(v):
                y = abs(a) * 2.0 ** (127 - s)
                best = min(range(8), key=lambda k: (abs(CODES[k] - y), k % 2))
                codes[n, c + i] = best + (8 if math.copysign(1.0, a) < 0 else 0)
    return codes, scales


def micro_values(codes, scales):
    v = torch.tensor(CODES + [-c for c in CODES], dtype=torch.float64)[codes]
    unit = torch.where(scales == 255, torch.full((), math.nan, dtype=torch.float64), torch.exp2(scales.double() - 127))
    return v * unit.repeat_interleave(32, 1)[:, :codes.shape[1]]
