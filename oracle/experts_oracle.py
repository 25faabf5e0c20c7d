"""Plain binary64 definitions of the router, the experts' products and the 4-bit rows, one expert, row or block at a time.
Arrays are float64 (already widened from their storage type); nothing is rounded here."""
from __future__ import annotations

import math

import numpy as np
import torch

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def gate_topk_ref(logits: np.ndarray, k: int, full: bool):
    """ids [T, k] and weights [T, k]: the k largest logits, the lower index first among equal ones."""
    T, E = logits.shape
    ids = np.empty((T, k), np.int32)
    weight = np.zeros((T, k))
    for t in range(T):
        row = logits[t]
        key = np.where(np.isnan(row), np.inf, row)
        order = sorted(range(E), key=lambda e: (not np.isnan(row[e]), -key[e], e))[:k]
        ids[t] = order
        if row[order[0]] == -np.inf:
            continue
        over = row if full else row[order]
        with np.errstate(invalid="ignore"):
            weight[t] = np.exp(row[order] - row[order[0]]) / np.exp(over - row[order[0]]).sum()
    return ids, weight


def gate_topk_backward_ref(logits: np.ndarray, ids: np.ndarray, grad_weight: np.ndarray, full: bool) -> np.ndarray:
    """dL/dlogits from the softmax's Jacobian, diag(p) - p p^T, over the chosen logits or over all of them."""
    T, E = logits.shape
    out = np.zeros((T, E))
    for t in range(T):
        over = np.arange(E) if full else ids[t]
        row = logits[t, over]
        if row.max() == -np.inf:
            continue
        p = np.exp(row - row.max())
        p /= p.sum()
        g = np.zeros(E)
        g[ids[t]] = grad_weight[t]
        out[t, over] = (np.diag(p) - np.outer(p, p)) @ g[over]
    return out


def _erf(v: np.ndarray) -> np.ndarray:
    return torch.erf(torch.from_numpy(np.ascontiguousarray(v))).numpy()


def activation_ref(v: np.ndarray, act: str) -> np.ndarray:
    if act == "relu":
        return np.maximum(v, 0.0)
    if act == "gelu":
        return v * 0.5 * (1.0 + _erf(v / math.sqrt(2.0)))
    return v


def activation_slope_ref(v: np.ndarray, act: str) -> np.ndarray:
    if act == "relu":
        return (v > 0).astype(np.float64)
    if act == "gelu":
        return 0.5 * (1.0 + _erf(v / math.sqrt(2.0))) + v * np.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)
    return np.ones_like(v)


def expert_forward_ref(x, w, bias, offsets, act):
    """pre, out [rows, d_out] and the sums of magnitudes behind pre (for error bounds); rows without an expert stay 0."""
    pre = np.zeros((x.shape[0], w.shape[1]))
    size = np.zeros_like(pre)
    for e in range(w.shape[0]):
        lo, hi = offsets[e], offsets[e + 1]
        pre[lo:hi] = x[lo:hi] @ w[e].T
        size[lo:hi] = np.abs(x[lo:hi]) @ np.abs(w[e]).T
        if bias is not None:
            pre[lo:hi] += bias[e]
            size[lo:hi] += np.abs(bias[e])
    return pre, activation_ref(pre, act), size


def expert_backward_input_ref(grad_out, w, offsets, act, pre):
    """grad_x and the sums of magnitudes behind the product (before the slope)."""
    grad_x = np.zeros((grad_out.shape[0], w.shape[2]))
    size = np.zeros_like(grad_x)
    for e in range(w.shape[0]):
        lo, hi = offsets[e], offsets[e + 1]
        grad_x[lo:hi] = grad_out[lo:hi] @ w[e]
        size[lo:hi] = np.abs(grad_out[lo:hi]) @ np.abs(w[e])
    slope = np.ones_like(grad_x) if act == "none" else activation_slope_ref(pre, act)
    return grad_x * slope, grad_x, slope, size


def expert_backward_weight_ref(grad_out, x, offsets, E):
    """grad_w, grad_bias and the sums of magnitudes behind them."""
    grad_w = np.zeros((E, grad_out.shape[1], x.shape[1]))
    grad_b = np.zeros((E, grad_out.shape[1]))
    size_w, size_b = np.zeros_like(grad_w), np.zeros_like(grad_b)
    for e in range(E):
        g, v = grad_out[offsets[e]:offsets[e + 1]], x[offsets[e]:offsets[e + 1]]
        grad_w[e], size_w[e] = g.T @ v, np.abs(g).T @ np.abs(v)
        grad_b[e], size_b[e] = g.sum(axis=0), np.abs(g).sum(axis=0)
    return grad_w, grad_b, size_w, size_b


def mx4_quantize_ref(x: np.ndarray):
    """codes [rows, d / 2] and scales [rows, d / 32]: per block the scale, per number the nearest code by distance."""
    rows, d = x.shape
    codes = np.zeros((rows, d), np.uint8)
    scales = np.zeros((rows, d // 32), np.uint8)
    for i in range(rows):
        for b in range(d // 32):
            block = x[i, 32 * b:32 * b + 32]
            if not np.isfinite(block).all():
                scales[i, b] = 255
                continue
            top = np.abs(block).max()
            s = -127 if top == 0 else max(math.frexp(top)[1] - 3, -127)
            scales[i, b] = s + 127
            mag = np.ldexp(np.abs(block), -s)
            dist = np.abs(mag[:, None] - E2M1[None, :])
            near = dist == dist.min(axis=1, keepdims=True)
            # of two codes equally near the even one; above 6 the largest
            pick = np.array([min(np.flatnonzero(n), key=lambda c: c % 2) for n in near])
            codes[i, 32 * b:32 * b + 32] = pick | (np.signbit(block) << 3)
    return codes[:, 0::2] | (codes[:, 1::2] << 4), scales


def mx4_values_ref(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    nibble = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[:-1] + (-1,))
    value = np.where(nibble & 8, -1.0, 1.0) * E2M1[nibble & 7]
    scale = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return value * np.repeat(scale, 32, axis=-1)
