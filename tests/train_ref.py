"""Plain 64-bit implementations of the training-side calls, and the rounding bounds the tests hold the kernels to."""
import numpy as np
import torch

import oracle

U32 = 2.0 ** -24     # half a step of fp32, relative
U16 = 2.0 ** -11     # of binary16


def patches(u, k):
    """[n][c][H][W] -> [n][c][H][W][k*k], positions clamped to the image."""
    p = (k - 1) // 2
    pad = np.pad(u, ((0, 0), (0, 0), (p, p), (p, p)), mode="edge")
    H, W = u.shape[2:]
    return np.stack([pad[:, :, a:a + H, b:b + W] for a in range(k) for b in range(k)], -1)


def grads(lr, coef, idx, gamma, dict_, gout, r, k, mode, compact=False, bilinear=False):
    """Gradients of the regression in fp64 and, for each, the sum of the magnitudes of its terms: every rounding of a kernel is at most a
    small multiple of that sum. mode: dense, listed (idx [n][s][H][W]; compact: values by rank) or global (idx [s]).
    Returns (grad_coef, grad_dict, grad_gamma or None), (magnitudes of the same)."""
    u = (oracle.bilinear_upsample if bilinear else oracle.bicubic_upsample)(lr, r).astype(np.float64)
    # |taps| of the up-sampling sum to at most 1.375 an axis (1 when bilinear): the magnitudes behind a value of u
    mag_u = np.full_like(u, 1.375 ** 2 * np.abs(lr[np.isfinite(lr)]).max(initial=0.0))
    d, phi, g = dict_.astype(np.float64), coef.astype(np.float64), gout.astype(np.float64)
    D, n = d.shape[0], u.shape[0]
    G = (g[..., None] * patches(u, k)).sum(1)
    Gm = (np.abs(g)[..., None] * patches(mag_u, k)).sum(1)

    def both(weights, atoms):
        """(gradient of the planes, gradient of the atoms) and their magnitudes."""
        one = np.einsum("nhwj,lj->nlhw", G, atoms, optimize=True), np.einsum("nlhw,nhwj->lj", weights, G, optimize=True)
        two = np.einsum("nhwj,lj->nlhw", Gm, np.abs(atoms), optimize=True), np.einsum("nlhw,nhwj->lj", np.abs(weights), Gm, optimize=True)
        return one, two

    if mode == "dense":
        (gc, gd), (mc, md) = both(phi, d)
        return (gc, gd, None), (mc, md, None)
    if mode == "global":
        at = idx.astype(np.int64)
        w = np.ones(len(at)) if gamma is None else gamma.astype(np.float64)
        (gc, A), (mc, mA) = both(phi if compact else phi[:, at], d[at] * w[:, None])
        gd, md = np.zeros_like(d), np.zeros_like(d)
        np.add.at(gd, at, w[:, None] * A)
        np.add.at(md, at, np.abs(w)[:, None] * mA)
        gg, mg = (d[at] * A).sum(1), (np.abs(d[at]) * mA).sum(1)
        if not compact:
            full, fullm = np.zeros_like(phi), np.zeros_like(phi)
            for q, a in enumerate(at):
                full[:, a] += gc[:, q]
                fullm[:, a] += mc[:, q]
            gc, mc = full, fullm
        return (gc, gd, gg), (mc, md, mg)
    at = np.minimum(idx.astype(np.int64), D - 1)
    keep = np.zeros((n, D) + u.shape[2:])
    np.put_along_axis(keep, at, 1.0, 1)
    if compact:
        weights = np.zeros_like(keep)
        np.put_along_axis(weights, at, phi, 1)
    else:
        weights = phi * keep
    (gc, gd), (mc, md) = both(weights, d)
    if compact:
        gc, mc = np.take_along_axis(gc, at, 1), np.take_along_axis(mc, at, 1)
    else:
        gc, mc = gc * keep, mc * keep
    return (gc, gd, None), (mc, md, None)


def balance(coef, idx, mask, per_frame):
    """(loss, counts, share, slope) in fp64 and a function from a weight to the gradient."""
    phi = coef.astype(np.float64)
    n, D, H, W = phi.shape
    s = idx.shape[1]
    on = np.ones((n, H, W), bool) if mask is None else mask != 0
    mag = np.where(on[:, None], np.abs(phi), 0.0)
    total = mag.sum(1, keepdims=True)
    small = total < np.finfo(np.float32).tiny
    p = np.where(small, 1.0 / D, mag / np.where(small, 1.0, total)) * on[:, None]
    counts = np.zeros((n, D), np.int64)
    for f in range(n):
        listed = idx[f][:, on[f]].reshape(-1)
        counts[f] = np.bincount(listed[listed < D], minlength=D)[:D]
    T = on.sum((1, 2)).astype(np.float64)
    if per_frame:
        slope = D * counts / (s * n * np.maximum(T, 1)[:, None] ** 2)
    else:
        slope = np.broadcast_to(D * counts.sum(0) / (s * max(T.sum(), 1) ** 2), (n, D)).copy()
    sums = p.sum((2, 3))
    share = sums / np.maximum(T, 1)[:, None]

    def gradient(weight):
        a = slope[:, :, None, None]
        with np.errstate(invalid="ignore"):
            g = weight * np.sign(np.where(on[:, None], phi, 0.0)) * (a - (a * p).sum(1, keepdims=True)) / np.where(small, 1.0, total)
        return np.where(small | ~on[:, None], 0.0, g)

    return (slope * sums).sum(), counts, share, slope, gradient, np.where(small, 1.0, total), p


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0):
    """One step in fp64 (torch tensors)."""
    g = g.double() * grad_scale
    m = beta1 * m.double() + (1 - beta1) * g
    v = beta2 * v.double() + (1 - beta2) * g * g
    p = p.double()
    return p - lr * weight_decay * p - lr * (m / (1 - beta1 ** t)) / ((v / (1 - beta2 ** t)).sqrt() + eps), m, v


def to(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
