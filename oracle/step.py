"""The serving step around grouped-query attention in float64 (numpy, CPU):
step tables, rotary positions, the append to blocks of 8-bit codes, attention
over them.  Plain loops over the definitions; no code of the library's.

Layouts are the library's: codes uint8 (E4M3) or int8 [pages, kv heads, 64, D],
scales float32 [pages, kv heads]; bf16 tensors come as uint16 bit patterns.
"""
from __future__ import annotations

import numpy as np

from .formats import bf16_bits_to_f64, e4m3_bits_to_f64

PAGE = 64


def pages_of(tokens: int) -> int:
    return -(-tokens // PAGE)


def step_tables(seq_lens, new_lens, free_pages, taken, block_table, num_pages, max_tokens):
    """Returns (block_table, new_indptr, slots, positions, requests, taken_out)."""
    table = np.array(block_table, dtype=np.int32)
    width = table.shape[1]
    at, short = min(max(int(taken), 0), len(free_pages)), 0
    indptr, slots, positions, requests = [0], [], [], []
    for b in range(len(seq_lens)):
        s = min(max(int(seq_lens[b]), 0), PAGE * width)
        n = min(max(int(new_lens[b]), 0), s)
        for k in range(pages_of(s - n), pages_of(s)):
            if at < len(free_pages):
                table[b, k] = free_pages[at]
                at += 1
            else:
                table[b, k] = -1
                short += 1
        for p in range(s - n, s):
            page = int(table[b, p // PAGE])
            slots.append(page * PAGE + p % PAGE if 0 <= page < num_pages else -1)
            positions.append(p)
            requests.append(b)
        indptr.append(len(slots))

    def padded(x, fill):
        return np.array((x + [fill] * max_tokens)[:max_tokens], dtype=np.int32)

    return (table, np.array(indptr, dtype=np.int32), padded(slots, -1), padded(positions, 0), padded(requests, -1),
            np.array([at, short], dtype=np.int32))


def rope(x, positions, inv_freq, pair_axis, interleaved, scale=1.0):
    """x float64 [tokens, heads, rot]; positions [axes, tokens]."""
    out = np.empty_like(x)
    half = x.shape[-1] // 2
    for j in range(half):
        angle = positions[pair_axis[j]].astype(np.float64) * inv_freq[j]
        c, s = np.cos(angle)[:, None] * scale, np.sin(angle)[:, None] * scale
        ia, ib = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        out[..., ia] = x[..., ia] * c - x[..., ib] * s
        out[..., ib] = x[..., ib] * c + x[..., ia] * s
    return out


# the non-negative values of either code, ascending, and the codes they belong to
_E4M3 = e4m3_bits_to_f64(np.arange(127, dtype=np.uint8))


def encode(values, int8: bool):
    """Round to the nearest code (ties to the even one); past the largest, the largest; NaN: 0x7f or 0."""
    v = np.asarray(values, dtype=np.float64)
    if int8:
        return np.clip(np.rint(np.where(np.isnan(v), 0.0, v)), -127, 127).astype(np.int8)
    a = np.minimum(np.abs(np.where(np.isnan(v), 0.0, v)), 448.0)
    hi = np.searchsorted(_E4M3, a).clip(0, 126)
    lo = (hi - 1).clip(0, 126)
    up, down = _E4M3[hi] - a, a - _E4M3[lo]
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    return np.where(np.isnan(v), np.uint8(0x7F), code | np.where(np.signbit(v), np.uint8(0x80), np.uint8(0)))


def decode(codes, int8: bool):
    return np.asarray(codes).astype(np.float64) if int8 else e4m3_bits_to_f64(np.asarray(codes))


def gqa_append(x_bits, slots, codes, scales, int8: bool):
    """One of K and V; returns new (codes, scales).  x_bits uint16 [rows, kv heads, D]."""
    codes, scales = codes.copy(), scales.copy()
    x = bf16_bits_to_f64(x_bits)
    top = 127.0 if int8 else 448.0
    t = 0
    while t < len(slots):
        page = int(slots[t]) // PAGE
        if slots[t] < 0 or page >= codes.shape[0]:
            t += 1
            continue
        end = t
        while end < len(slots) and slots[end] >= 0 and slots[end] // PAGE == page:
            end += 1
        places = [int(s) % PAGE for s in slots[t:end]]
        for h in range(codes.shape[1]):
            rows = x[t:end, h]
            finite = np.abs(rows[np.isfinite(rows)])
            amax = finite.max() if finite.size else 0.0
            e = -126
            while amax > top * 2.0 ** e:
                e += 1
            if 0 not in places:
                old = int(np.floor(np.log2(float(scales[page, h]))))
                if e > old:
                    for r in range(max(places)):
                        if r not in places:
                            codes[page, h, r] = encode(decode(codes[page, h, r], int8) * 2.0 ** (old - e), int8)
                else:
                    e = old
            for r, place in zip(rows, places):
                codes[page, h, place] = encode(r * 2.0 ** -e, int8)
            scales[page, h] = np.float32(2.0 ** e)
        t = end
    return codes, scales


def gqa_attend(q_bits, k_codes, v_codes, k_scales, v_scales, block_table, seq_lens, q_chunk, softmax_scale, int8):
    """Returns (out, lse, weight of |V| in out, largest sum of |q k| * softmax_scale of a row): the last two bound
    what a rounding of a weight or of a product can do."""
    q = bf16_bits_to_f64(q_bits)
    n, hq, d = q.shape
    hk = k_codes.shape[1]
    g = hq // hk
    out, mass = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    lse, spread = np.full((n, hq), -np.inf), np.zeros((n, hq))
    width = block_table.shape[1]
    for b in range(len(seq_lens)):
        s = min(max(int(seq_lens[b]), 0), PAGE * width)
        held = [(k, int(p)) for k, p in enumerate(block_table[b, :pages_of(s)]) if 0 <= p < k_codes.shape[0]]
        if not held:
            continue
        pos = np.concatenate([np.arange(k * PAGE, (k + 1) * PAGE) for k, _ in held])
        for h in range(hk):
            keys = np.concatenate([decode(k_codes[p, h], int8) * np.float64(k_scales[p, h]) for _, p in held])
            vals = np.concatenate([decode(v_codes[p, h], int8) * np.float64(v_scales[p, h]) for _, p in held])
            for i in range(q_chunk):
                see = pos < s - q_chunk + i + 1
                if not see.any():
                    continue
                row = b * q_chunk + i
                rows = q[row, h * g:(h + 1) * g]
                z = softmax_scale * (rows @ keys[see].T)
                top = z.max(-1, keepdims=True)
                w = np.exp(z - top)
                total = w.sum(-1, keepdims=True)
                out[row, h * g:(h + 1) * g] = (w / total) @ vals[see]
                mass[row, h * g:(h + 1) * g] = (w / total) @ np.abs(vals[see])
                lse[row, h * g:(h + 1) * g] = (top + np.log(total))[:, 0]
                spread[row, h * g:(h + 1) * g] = softmax_scale * (np.abs(rows) @ np.abs(keys[see]).T).max(-1)
    return out, lse, mass, spread
