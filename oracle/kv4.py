"""Norm, rotation and cache write, and attention over a 4-bit KV cache (oracle, NumPy, CPU).  Test infrastructure only.

`normed_rotated` is the definition in float64:
  y_i = x_i / sqrt(mean(x^2) + eps) * (offset + w_i),  a_i = p f_i (i < d/2),
  o_i = y_i cos a_i - y_(i+d/2) sin a_i,  o_(i+d/2) = y_(i+d/2) cos a_i + y_i sin a_i.

A cache row of d values is quantized in groups of 32 as weights are
(oracle.quantize) and stands for RNE_bf16(RN_f32(scale * code + offset)).
The byte order of the two caches is a reading, written here as one address
per value: `k_address` and `v_address` give the byte and the nibble of value i
of position p, and the index of its (scale, offset) pair, in a head of P
positions (P a multiple of 32).
"""
from __future__ import annotations

import numpy as np

from .q4nx import bf16_to_f32, dequant_bf16
from .quantize import quantize


def normed_rotated(x, weight_bits, offset, eps, positions, inv_freq):
    """x [T][heads][d] float32 (weight_bits [d] or None, inv_freq [d/2] float32 or None) -> float64."""
    y = np.asarray(x, np.float64)
    if weight_bits is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + np.float64(np.float32(eps)))
        y = y * (np.float64(np.float32(offset)) + bf16_to_f32(weight_bits).astype(np.float64))
    if inv_freq is not None:
        a = np.asarray(positions, np.float64)[:, None, None] * np.asarray(inv_freq, np.float32).astype(np.float64)
        h = y.shape[-1] // 2
        lo, hi = y[..., :h], y[..., h:]
        y = np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], -1)
    return y


def k_address(p, i, P, d):
    return p * (d // 2) + (i // 8) * 4 + i % 4, (i // 4) % 2, p * (d // 32) + i // 32


def v_address(p, i, P, d):
    blk, a, h, r = p // 32, (p // 16) % 2, (p // 4) % 4, p % 4
    byte = blk * 16 * d + (i // 64) * 1024 + ((((h * 16) + i % 16) * 2 + (i // 32) % 2) * 2 + a) * 4 + r
    return byte, (i // 16) % 2, blk * d + (i // 32) * 32 + h * 8 + a * 4 + r


def padded(L):
    return -(-L // 32) * 32


def write_rows(cache, rows, heads, positions, n_heads, L, address):
    """Quantizes rows [n][d] (float32) into cache (uint8, all of one cache): row t to (heads[t], positions[t])."""
    P = padded(L)
    d = rows.shape[-1]
    codes, scales, offsets = quantize(rows)
    pairs = cache[n_heads * P * d // 2:].view(np.uint16).reshape(-1, 2)
    i = np.arange(d)
    for t, (h, p) in enumerate(zip(heads, positions)):
        byte, nibble, pair = address(p, i, P, d)
        at = h * P * d // 2 + byte
        keep = np.where(nibble == 1, 0x0F, 0xF0).astype(np.uint8)
        for nib in (0, 1):                       # two values share a byte
            m = nibble == nib
            cache[at[m]] = (cache[at[m]] & keep[m]) | (codes[t, m] << (4 * nib)).astype(np.uint8)
        pairs[h * P * (d // 32) + pair, 0] = scales[t, i // 32]
        pairs[h * P * (d // 32) + pair, 1] = offsets[t, i // 32]


def read_rows(cache, heads, positions, n_heads, L, d, address):
    """The values (bf16 bits, [n][d]) of rows (heads[t], positions[t])."""
    P = padded(L)
    pairs = cache[n_heads * P * d // 2:].view(np.uint16).reshape(-1, 2)
    i = np.arange(d)
    heads, positions = np.asarray(heads)[:, None], np.asarray(positions)[:, None]
    byte, nibble, pair = address(positions, i, P, d)
    b = cache[heads * P * d // 2 + byte]
    codes = np.where(nibble == 1, b >> 4, b & 15).astype(np.uint8)
    pr = pairs[heads * P * (d // 32) + pair][:, ::32]          # one pair a group
    return dequant_bf16(codes, np.ascontiguousarray(pr[..., 0]), np.ascontiguousarray(pr[..., 1]))


def attention(q_bits, K_bits, V_bits, n, window, scale):
    """q [T][H][d], K and V [G][>= n][d] (bf16 bits) of one sequence of n positions, the T rows its last ones ->
    o [T][H][d] float64, sum_j p_j |v_j| and the largest sum_i |q_i k_ji| of each row (for tolerances)."""
    q = bf16_to_f32(q_bits).astype(np.float64)
    K, V = bf16_to_f32(K_bits[:, :n]).astype(np.float64), bf16_to_f32(V_bits[:, :n]).astype(np.float64)
    T, H, d = q.shape
    hg = H // K.shape[0]
    o, bound, dots = np.zeros((T, H, d)), np.zeros((T, H, d)), np.zeros((T, H, 1))
    for t in range(T):
        p = n - T + t
        if p < 0:
            continue
        j0 = max(0, p - window + 1) if window else 0
        for h in range(H):
            k, v = K[h // hg, j0:p + 1], V[h // hg, j0:p + 1]
            s = scale * (k @ q[t, h])
            w = np.exp(s - s.max())
            w /= w.sum()
            o[t, h], bound[t, h] = w @ v, w @ np.abs(v)
            dots[t, h] = (np.abs(k) @ np.abs(q[t, h])).max()
    return o, bound, dots
