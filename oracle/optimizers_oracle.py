"""fp64 oracle of the Muon and AdamW steps, written from their formulas in plain numpy.

TEST INFRASTRUCTURE ONLY, like orthdion_oracle.py: no code is shared with the HIP path.

Muon (published quintic Newton-Schulz iteration):
    M = mu M + G,  B = G + mu M (Nesterov) or M,  X_0 = B / (||B||_F + eps)
    X_k+1 = a X_k + (b S + c S S) X_k,  S = X_k X_k^T
    X = (1 - lr wd) X - lr scale X_K
A zero B gives X_K = 0; a B with a NaN or an infinity gives NaN everywhere.

AdamW:
    t = t + 1,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
    x = (1 - lr wd) x - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
"""
from __future__ import annotations

import numpy as np

__all__ = ["newton_schulz", "newton_schulz_path", "muon_step", "adamw_step"]


def newton_schulz_path(a, coeffs, eps=1e-7):
    """[X_0, .., X_K], as the shorter side has it: X is wide or square."""
    a = np.asarray(a, dtype=np.float64)
    if a.shape[0] > a.shape[1]:
        a = a.T
    if not np.all(np.isfinite(a)):
        return [np.full_like(a, np.nan)] * (len(coeffs) + 1)
    norm = np.sqrt(np.sum(a * a)) + eps
    x = a / norm if norm > 0 else np.zeros_like(a)
    path = [x]
    for ca, cb, cc in coeffs:
        s = x @ x.T
        x = ca * x + (cb * s + cc * (s @ s)) @ x
        path.append(x)
    return path


def newton_schulz(a, coeffs, eps=1e-7):
    x = newton_schulz_path(a, coeffs, eps)[-1]
    return x.T if np.shape(a)[0] > np.shape(a)[1] else x


def muon_step(x, g, m, coeffs, mu, lr, weight_decay, scale, nesterov=True, eps=1e-7):
    """(X, M, O) after one step, in fp64."""
    m = mu * np.asarray(m, dtype=np.float64) + np.asarray(g, dtype=np.float64)
    o = newton_schulz(g + mu * m if nesterov else m, coeffs, eps)
    return (1 - lr * weight_decay) * np.asarray(x, dtype=np.float64) - lr * scale * o, m, o


def adamw_step(x, g, m, v, t, lr, beta1, beta2, eps, weight_decay):
    """(x, m, v) after step t (counted from 1), in fp64."""
    g = np.asarray(g, dtype=np.float64)
    m = beta1 * np.asarray(m, dtype=np.float64) + (1 - beta1) * g
    v = beta2 * np.asarray(v, dtype=np.float64) + (1 - beta2) * g * g
    x = (1 - lr * weight_decay) * np.asarray(x, dtype=np.float64)
    return x - lr * (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps), m, v
