"""CPU oracle for token-by-token generation: the paged int8 key / value cache, attention over it, rules on logits.
TEST INFRASTRUCTURE ONLY; shares no code with the kernels.

The cache holds what the boundary codec (oracle/codec.py) makes of every token's key and value row, 64 elements to a
scale; keys of the rotary block are rotated in 64 bits and rounded to fp32 once before that.  Attention of a new token
sees the tokens before the call and, of the new ones, those that its mask names.  Plain numpy in float64, one sequence
and one head at a time.

The pool is a dict of numpy arrays in the layout of the C ABI: k_codes [pages, kv, page, dh], v_codes [pages, kv, dh,
page], k_scales / v_scales [pages, kv, dh / 64, page] fp32 values (already rounded to bf16 with scale_bits = 16).
"""
from __future__ import annotations

import math

import numpy as np

from oracle import codec


def rotate(x, pos):
    """x [n, heads, dh] float64, pos [n]: pairs (2i, 2i+1) turned by pos * 10000^(-2i/dh)."""
    dh = x.shape[2]
    ang = np.asarray(pos, dtype=np.float64)[:, None] * 10000.0 ** (-np.arange(0, dh, 2, dtype=np.float64) / dh)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    out = np.empty_like(x)
    out[..., 0::2] = x[..., 0::2] * c - x[..., 1::2] * s
    out[..., 1::2] = x[..., 0::2] * s + x[..., 1::2] * c
    return out


def append(pool, table, page, b, past, k, v, scale_bits):
    """k, v [n, kv, dh] fp32 (rotated already) go to the tokens past .. of sequence b."""
    for name, x in (("k", k), ("v", v)):
        n, kv, dh = x.shape
        codes, scales = codec.encode(np.ascontiguousarray(x, dtype=np.float32).reshape(-1), 64, scale_bits)
        if scale_bits == 16:
            scales = codec.bf16_bits_to_f32(scales)
        codes, scales = codes.reshape(n, kv, dh), scales.reshape(n, kv, dh // 64)
        for i in range(n):
            p, o = table[b, (past + i) // page], (past + i) % page
            if not 0 <= p < pool["k_codes"].shape[0]:
                continue
            if name == "k":
                pool["k_codes"][p, :, o, :] = codes[i]
            else:
                pool["v_codes"][p, :, :, o] = codes[i]
            pool[name + "_scales"][p, :, :, o] = scales[i]


def read(pool, table, page, b, tokens):
    """k, v [n, kv, dh] float64 of the tokens (a list) of sequence b, and whether their page is one of the pool's."""
    n, (_, kv, _, dh) = len(tokens), pool["k_codes"].shape
    k, v, there = np.zeros((n, kv, dh)), np.zeros((n, kv, dh)), np.zeros(n, dtype=bool)
    for i, j in enumerate(tokens):
        p, o = table[b, j // page], j % page
        if 0 <= p < pool["k_codes"].shape[0]:
            there[i] = True
            with np.errstate(invalid="ignore"):
                k[i] = pool["k_codes"][p, :, o].astype(np.float64) * np.repeat(pool["k_scales"][p, :, :, o].astype(np.float64), 64, axis=1)
                v[i] = pool["v_codes"][p, :, :, o].astype(np.float64) * np.repeat(pool["v_scales"][p, :, :, o].astype(np.float64), 64, axis=1)
    return k, v, there


def keep(pool, table, page, b, past, kept, tokens):
    """The draft tokens kept[j] of sequence b move to the places j."""
    old = {n: a.copy() for n, a in pool.items()}
    cap, pages = table.shape[1] * page, pool["k_codes"].shape[0]
    for j, u in enumerate(kept):
        if not 0 <= u < tokens or past + u >= cap:
            continue
        sp, so = table[b, (past + u) // page], (past + u) % page
        dp, do = table[b, (past + j) // page], (past + j) % page
        if not (0 <= sp < pages and 0 <= dp < pages):
            continue
        pool["k_codes"][dp, :, do] = old["k_codes"][sp, :, so]
        for n in ("v_codes", "k_scales", "v_scales"):
            pool[n][dp, :, :, do] = old[n][sp, :, :, so]


def attention(q, k, v, see):
    """q [n, H, dh], k and v [m, kv, dh], see [n, m] -> out [n, H, dh]; the weights' mean of |v| (same shape), the largest
    sum_d |q_d k_jd| / sqrt(dh) of a row and head [n, H], for error bounds."""
    n, H, dh = q.shape
    kv = k.shape[1]
    out, mean_abs, size = np.zeros((n, H, dh)), np.zeros((n, H, dh)), np.zeros((n, H))
    for h in range(H):
        g = h // (H // kv)
        s = q[:, h] @ k[:, g].T / math.sqrt(dh)
        s = np.where(see, s, -np.inf)
        top = s.max(axis=1, keepdims=True, initial=-np.inf)
        p = np.where(see, np.exp(s - np.where(np.isfinite(top), top, 0.0)), 0.0)
        total = p.sum(axis=1, keepdims=True)
        p = p / np.where(total == 0, 1.0, total)
        out[:, h] = p @ v[:, g]
        mean_abs[:, h] = p @ np.abs(v[:, g])
        size[:, h] = np.where(see, np.abs(q[:, h]) @ np.abs(k[:, g]).T / math.sqrt(dh), 0.0).max(axis=1, initial=0.0)
    return out, mean_abs, size


def adjust(x, history, repetition, frequency, presence, bias_ids, bias, allowed):
    """One row of logits x [vocab] float64; history, bias_ids lists of ids; allowed [vocab] bool or None."""
    out = x.copy()
    vocab = x.size
    times = np.zeros(vocab)
    for v in history:
        if 0 <= v < vocab:
            times[v] += 1
    for v in np.nonzero(times)[0]:
        y = out[v] / repetition if out[v] > 0 else out[v] * repetition
        out[v] = y - frequency * times[v] - presence
    for v, b in zip(bias_ids, bias):
        if 0 <= v < vocab:
            out[v] += b
    if allowed is not None:
        out[~allowed] = -np.inf
    return out
