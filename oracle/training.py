"""Operators of a training step around the layers in 64 bits, from their formulas: layer norm, the
cross entropy of a linear classifier, orthogonalised updates.  NumPy only."""
import numpy as np


def layer_norm(x, gamma, beta, eps):
    """Rows of x -> (y, mean, rstd)."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def codes(y, s_y):
    return np.clip(np.rint(y / np.float64(np.float32(s_y))), -127, 127).astype(np.int8)


def layer_norm_backward(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) for the statistics the forward pass kept."""
    dy, x, mean, rstd = (np.asarray(a, np.float64) for a in (dy, x, mean, rstd))
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def logits(h, w, bias):
    l = np.asarray(h, np.float64) @ np.asarray(w, np.float64).T
    return l if bias is None else l + np.asarray(bias, np.float64)


def kept(target, classes, ignore_index):
    return (target != ignore_index) & (target >= 0) & (target < classes)


def cross_entropy(h, w, bias, target, ignore_index=-100):
    """(loss, lse) of every row; a row that is left out has loss 0."""
    l = logits(h, w, bias)
    top = l.max(1)
    base = np.where(np.isfinite(top), top, 0)
    with np.errstate(divide="ignore"):
        lse = base + np.log(np.exp(l - base[:, None]).sum(1))
    k = kept(target, w.shape[0], ignore_index)
    hit = l[np.arange(len(target)), np.where(k, target, 0)]
    with np.errstate(invalid="ignore"):
        loss = np.where(np.isneginf(hit), np.inf, lse - hit)
    return np.where(k, loss, 0.0), lse


def cross_entropy_backward(h, w, bias, target, dloss, ignore_index=-100):
    """(dh, dw, dbias, dl)."""
    l = logits(h, w, bias)
    _, lse = cross_entropy(h, w, bias, target, ignore_index)
    k = kept(target, w.shape[0], ignore_index) & ~np.isneginf(lse)
    with np.errstate(invalid="ignore"):
        dl = np.exp(l - np.where(np.isneginf(lse), 0, lse)[:, None])
    dl[np.arange(len(target))[k], target[k]] -= 1
    dl = np.where(k[:, None], dl * np.where(k, dloss, 0)[:, None], 0)
    h = np.where(kept(target, w.shape[0], ignore_index)[:, None], h, 0)
    return dl @ np.asarray(w, np.float64), dl.T @ np.asarray(h, np.float64), dl.sum(0), dl


def orthogonalise(g, steps=5, a=3.4445, b=-4.7750, c=2.0315, eps=1e-7, scale=1.0):
    """One matrix -> (update, Frobenius norms of X before every step)."""
    a, b, c, eps = (np.float64(np.float32(v)) for v in (a, b, c, eps))
    x = np.asarray(g, np.float64)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / (np.linalg.norm(x) + eps)
    norms = []
    for _ in range(steps):
        norms.append(np.linalg.norm(x))
        m = x @ x.T
        x = a * x + (b * m + c * (m @ m)) @ x
    return scale * (x.T if tall else x), norms
