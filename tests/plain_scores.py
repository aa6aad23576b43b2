"""Plain 64-bit implementations of the operators that make log-likelihoods
(projection with adapters, logits to log-likelihoods, label masks), on the CPU,
and the error bounds that 32-bit sums of the same formulas keep.

A bound follows the formula: a sum of n products kept in 32 bits is off by at
most n 2^-24 times the sum of the products' magnitudes, every further operation
by 2^-24 of its result, and the output's rounding comes last."""
import math

import numpy as np
import torch

EPS = 2.0 ** -24


def rounding(dtype):
    """(relative, absolute) error of one rounding to the type."""
    # (half the spacing of 24, 8 and 11 significant bits, and of the subnormals)
    return {torch.float32: (EPS, 2.0 ** -150), torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float16: (2.0 ** -11, 2.0 ** -25)}[dtype]


def project(x, weight, bias=None, a=None, b=None, scale=None, adapter=None, out_dtype=torch.float32):
    """(outputs, bound) in 64 bits; tensors on the CPU."""
    X, W = x.double(), weight.double()
    y, mag = X @ W.T, X.abs() @ W.abs().T
    if bias is not None:
        y, mag = y + bias.double(), mag + bias.double().abs()
    err = (X.shape[1] + 8) * EPS * mag
    if adapter is not None and a is not None:
        for n, g in enumerate(adapter.tolist()):
            if not 0 <= g < a.shape[0]:
                continue
            s = 1.0 if scale is None else float(scale[g])
            A, B = a[g].double(), b[g].double()
            u, um = s * (A @ X[n]), abs(s) * (A.abs() @ X[n].abs())
            y[n] += B @ u
            # u: a sum of D products, then held in 16 bits of mantissa; its products: a sum of 2 R
            err[n] += B.abs() @ ((X.shape[1] + 8) * EPS * um + 2.0 ** -16 * u.abs()) + (2 * A.shape[0] + 8) * EPS * (B.abs() @ um)
    rel, least = rounding(out_dtype)
    return y, err * (1 + rel) + rel * y.abs() + least


def loglikes(logits, normalize=True, scale=1.0, log_prior=None, request=None, history=None, repetition=None,
             presence=None, frequency=None, bias=None, mask=None, mask_of=None):
    """(outputs, bound) in 64 bits; arguments as wfstdec.loglikes, on the CPU."""
    N, V = logits.shape
    y, bound = np.zeros((N, V)), np.zeros((N, V))
    for n in range(N):
        z = logits[n].double().numpy().copy()
        size = np.abs(np.where(np.isfinite(z), z, 0.0))
        q = n if request is None else int(request[n])
        if history is not None and 0 <= q < len(history[0]) - 1:
            off = np.clip(history[0].numpy(), 0, len(history[1]))
            ids = history[1].numpy()[off[q]:off[q + 1]] if off[q] < off[q + 1] else np.zeros(0, np.int32)
            c = np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V)
            rho = 1.0 if repetition is None else float(repetition[q])
            less = (0.0 if presence is None else float(presence[q])) + (0.0 if frequency is None else float(frequency[q])) * c
            with np.errstate(invalid="ignore"):
                had = np.where(z > 0, z / rho, z * rho) - less
            z = np.where(c > 0, had, z)
            size = np.where(c > 0, size * max(rho, 1.0 / rho) + np.abs(less), size)
        if bias is not None and 0 <= q < len(bias[0]) - 1:
            off = np.clip(bias[0].numpy(), 0, len(bias[1]))
            add = np.zeros(V)
            for i in range(off[q], off[q + 1]):
                if 0 <= int(bias[1][i]) < V:
                    add[int(bias[1][i])] = float(bias[2][i])
            z, size = z + add, size + np.abs(add)
        if mask is not None:
            m = n if mask_of is None else int(mask_of[n])
            if 0 <= m < mask.shape[0]:
                bits = np.unpackbits(mask[m].contiguous().numpy().astype("<i4").view(np.uint8), bitorder="little")[:V]
                z = np.where(bits == 1, z, -np.inf)
        err = 6 * EPS * size
        lse = lerr = 0.0
        shift = 0.0
        if normalize:
            top = np.max(np.where(np.isnan(z), -np.inf, z))
            shift = top if top > -np.inf else 0.0
            with np.errstate(invalid="ignore", over="ignore"):
                p = np.exp(z - shift)
            total = p.sum()
            with np.errstate(divide="ignore", invalid="ignore"):
                lse = math.log(total) if total > 0 else (-np.inf if total == 0 else np.nan)
            if np.isfinite(total) and total > 0:
                away = np.where(p > 0, np.abs(np.where(np.isfinite(z), z, shift) - shift), 0.0)
                # each term: its own error, that of its exponent's product and of the exponential; then the sum
                lerr = float((p * (err + 4 * EPS * away + 4 * EPS)).sum() / total) + (V / 64 + 64) * EPS + 2 * EPS * abs(lse)
        prior = np.zeros(V) if log_prior is None else log_prior.double().numpy()
        with np.errstate(invalid="ignore"):
            y[n] = np.where(np.isneginf(z), -np.inf, scale * ((z - shift) - lse - prior))
            far = np.abs(np.where(np.isfinite(z), z, 0.0) - shift) + (abs(lse) if np.isfinite(lse) else 0.0) + np.abs(prior)
        bound[n] = scale * (err + lerr + 4 * EPS * far) * (1 + 4 * EPS) + 2 * EPS * np.abs(np.where(np.isfinite(y[n]), y[n], 0.0)) + 1e-40
    return torch.from_numpy(y), torch.from_numpy(bound)


def label_masks(g, num_pdfs, offsets, states):
    """int32 words [N, ceil(num_pdfs / 32)] of a graph dict's labels."""
    words = (num_pdfs + 31) // 32
    out = np.zeros((len(offsets) - 1, words * 32), np.uint8)
    rp = g["row_ptr"].astype(np.int64)
    for n in range(len(offsets) - 1):
        for s in states[max(0, offsets[n]):min(offsets[n + 1], len(states))]:
            if 0 <= s < len(rp) - 1:
                l = g["ilabel"][rp[s]:rp[s + 1]]
                out[n, l[l > 0] - 1] = 1
    return np.packbits(out, axis=1, bitorder="little").view("<i4").reshape(len(offsets) - 1, words)


def close(got, want, bound):
    """Finite values within the bound, the others equal (NaN with NaN)."""
    got = got.detach().cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN in other places"
    odd = ~fine & ~torch.isnan(want)
    assert torch.equal(got[odd], want[odd]), "infinities differ"
    off = (got - want).abs()[fine] - bound[fine]
    assert not off.numel() or float(off.max()) <= 0, f"{float(off.max())} beyond the bound, {int((off > 0).sum())} of {off.numel()}"
