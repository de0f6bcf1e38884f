"""Plain CPU oracle of the vocabulary projection's calls: row quantisation, the product in
8-bit integers, the softmax cross entropy over the vocabulary and its gradients.

TEST INFRASTRUCTURE ONLY, as ``cmsd_oracle``: numpy in float64 (integers where the
quantity is whole), the definitions written out, and no code shared with the library.
Beside each float result stands ``size``: the sum of the magnitudes that it adds up, which
a bound on the rounding of any order of summation is a multiple of.
"""
from __future__ import annotations

import numpy as np

__all__ = ["quantize_rows", "head_logits", "head_loss", "head_loss_grad"]


def quantize_rows(x):
    """Codes int8 and scales float32 of the rows of x (float64 holding float32 values)."""
    n = len(x)
    codes = np.zeros(x.shape, np.int8)
    scales = np.zeros(n, np.float32)
    for r in range(n):
        top = np.max(np.abs(x[r]))
        if not np.isfinite(top):
            scales[r] = np.nan
            continue
        scales[r] = np.float32(top / 127.0)
        if scales[r] > 0:
            codes[r] = np.clip(np.rint(x[r] / np.float64(scales[r])), -127, 127).astype(np.int8)
    return codes, scales


def head_logits(codes, scales, weight_codes, weight_scales, scale):
    """Logits float64 from the codes: the sum of products is whole, the scales multiply it."""
    s = codes.astype(np.int64) @ weight_codes.astype(np.int64).T
    return s.astype(np.float64) * np.float64(scale) * scales.astype(np.float64)[:, None] \
        * weight_scales.astype(np.float64)[None, :]


def head_loss(hidden, weight, labels, scale):
    """loss, lse, logits and the logits' size."""
    z = scale * (hidden @ weight.T)
    size = abs(scale) * (np.abs(hidden) @ np.abs(weight).T)
    top = z.max(1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(1))
    loss = np.zeros(len(hidden))
    for n, y in enumerate(labels):
        if y >= weight.shape[0]:
            loss[n] = np.nan
        elif y >= 0:
            loss[n] = lse[n] - z[n, y]
    return loss, lse, z, size


def head_loss_grad(hidden, weight, labels, grad_loss, scale):
    """(grad_hidden, its size, grad_weight, its size, d, softmax)."""
    _, lse, z, _ = head_loss(hidden, weight, labels, scale)
    p = np.exp(z - lse[:, None])
    d = p.copy()
    for n, y in enumerate(labels):
        if 0 <= y < weight.shape[0]:
            d[n, y] -= 1.0
            d[n] *= grad_loss[n] * scale
        else:
            d[n] = 0.0
    return d @ weight, np.abs(d) @ np.abs(weight), d.T @ hidden, np.abs(d).T @ np.abs(hidden), d, p
