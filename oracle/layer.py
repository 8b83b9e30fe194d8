"""The latent-attention layer around the cache in float64 (numpy, CPU): the rows
that are appended and the bytes they become, the projections between heads and
latents, causal attention of ragged prompts.  Plain loops over the definitions; no
code of the library's.

bf16 tensors come as uint16 bit patterns; pools are the library's: bf16 bits or
E4M3 codes [pages, 64, 576] (with float32 scales [pages, 64]), or 656-byte rows.
"""
from __future__ import annotations

import numpy as np

from .formats import bf16_bits_to_f64, ds_rows_to_f64, e4m3_bits_to_f64
from .step import encode, rope

PAGE, LATENT, NOPE, ROPE = 64, 512, 128, 64
BF16, E4M3, LATENT_ROWS = 0, 1, 2


def round_bf16(x):
    """float64 to bf16 bits, one rounding to nearest even (NaN: 0x7fc0)."""
    x = np.asarray(x, dtype=np.float64)
    m, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
    step = np.exp2(np.maximum(e - 8, -133).astype(np.float64))   # a bf16 step at this magnitude
    y = np.where(np.isfinite(x), np.rint(np.where(np.isfinite(x), x, 0.0) / step) * step, x)
    with np.errstate(over="ignore"):
        f = y.astype(np.float32)
    bits = (f.view(np.uint32) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), bits)


def new_rows(latent_bits, key_bits, weight_bits=None, eps=0.0, positions=None, inv_freq=None, pair_axis=None,
             interleaved=False, scale=1.0):
    """(latent rows rounded to fp32, key rows), both as float64."""
    x = bf16_bits_to_f64(latent_bits)
    if weight_bits is not None:
        with np.errstate(all="ignore"):
            x = x * bf16_bits_to_f64(weight_bits) / np.sqrt((x * x).sum(-1, keepdims=True) / LATENT + np.float64(np.float32(eps)))
    with np.errstate(over="ignore"):
        y = x.astype(np.float32).astype(np.float64)
    r = bf16_bits_to_f64(key_bits)
    if positions is not None:
        r = rope(r[:, None, :], positions, inv_freq, pair_axis, interleaved, scale)[:, 0]
    return y, r


def _finite_top(x):
    return np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)


def row_bytes(latent, key, kv_dtype):
    """Rows as they are stored: (bf16 bits | E4M3 codes | 656 bytes, scales or None)."""
    if kv_dtype == BF16:
        return round_bf16(np.concatenate([latent, key], -1)), None
    if kv_dtype == E4M3:
        y = np.concatenate([latent, key], -1)
        top = _finite_top(y).astype(np.float32)
        scale = np.where(top > 0, np.maximum(top / np.float32(448.0), np.float32(2.0 ** -126)), np.float32(1.0)).astype(np.float32)
        with np.errstate(all="ignore"):   # (the quotient is one of fp32: a value 2^-24 beside a tie of codes is on it)
            return encode(y.astype(np.float32) / scale[:, None], False), scale
    n = latent.shape[0]
    out = np.zeros((n, 656), np.uint8)
    for t in range(4):
        tile = latent[:, 128 * t:128 * t + 128]
        top = _finite_top(tile)
        for i in range(n):
            e = 0
            if top[i] > 0:
                e = -126
                while e < 63 and top[i] > 448.0 * 2.0 ** e:
                    e += 1
            out[i, 128 * t:128 * t + 128] = encode(tile[i] * 2.0 ** -e, False)
            out[i, 512 + 4 * t:516 + 4 * t] = np.array([2.0 ** e], "<f4").view(np.uint8)
    out[:, 528:] = round_bf16(key).astype("<u2").view(np.uint8).reshape(n, 128)
    return out, None


def put_rows(pool, scales, slots, rows, row_scales):
    """The pool and scales with row t at slots[t]; slots outside are skipped."""
    pool, scales = pool.copy(), None if scales is None else scales.copy()
    for t, s in enumerate(slots):
        if 0 <= s < PAGE * pool.shape[0]:
            pool[s // PAGE, s % PAGE] = rows[t]
            if scales is not None:
                scales[s // PAGE, s % PAGE] = row_scales[t]
    return pool, scales


def read_rows(pool, scales, kv_dtype):
    """The pool's values, float64 [pages, 64, 576]."""
    if kv_dtype == BF16:
        return bf16_bits_to_f64(pool)
    if kv_dtype == E4M3:
        return e4m3_bits_to_f64(pool) * scales.astype(np.float64)[..., None]
    return ds_rows_to_f64(pool).reshape(-1, PAGE, 576)


def gather(pool, scales, kv_dtype, block_table, begin, indptr, max_rows, fill):
    """bf16 bits [max_rows, 576]: `fill` where no request's row is, zeros for tokens without a page."""
    with np.errstate(all="ignore"):
        values = round_bf16(read_rows(pool, scales, kv_dtype).astype(np.float32))
    out = np.full((max_rows, 576), fill, np.uint16)
    for b in range(block_table.shape[0]):
        for r in range(indptr[b], min(indptr[b + 1], max_rows)):
            at = int(begin[b]) + r - int(indptr[b])
            page = int(block_table[b, at // PAGE]) if 0 <= at < PAGE * block_table.shape[1] else -1
            out[r] = values[page, at % PAGE] if 0 <= page < pool.shape[0] else 0
    return out


def project(x_bits, w_bits, transpose):
    """Per head: x [n, h, in] times w [h, in, out] (transpose: [h, out, in]); also the sums of magnitudes."""
    x, w = bf16_bits_to_f64(x_bits), bf16_bits_to_f64(w_bits)
    if transpose:
        w = w.transpose(0, 2, 1)
    return np.matmul(x.transpose(1, 0, 2), w).transpose(1, 0, 2), np.matmul(np.abs(x).transpose(1, 0, 2), np.abs(w)).transpose(1, 0, 2)


def prefill(q_bits, k_bits, key_bits, v_bits, q_indptr, kv_indptr, softmax_scale):
    """Returns (out, lse, weight of |V| in out, largest sum of |q k| * softmax_scale of a row), rows of no request 0."""
    q, k, key, v = (bf16_bits_to_f64(t) for t in (q_bits, k_bits, key_bits, v_bits))
    n, heads = q.shape[:2]
    out, mass = np.zeros((n, heads, v.shape[-1])), np.zeros((n, heads, v.shape[-1]))
    lse, spread = np.full((n, heads), -np.inf), np.zeros((n, heads))
    for b in range(len(q_indptr) - 1):
        q0, q1, k0, k1 = q_indptr[b], q_indptr[b + 1], kv_indptr[b], kv_indptr[b + 1]
        for h in range(heads):
            keys = np.concatenate([k[k0:k1, h], key[k0:k1]], -1)
            for i in range(q1 - q0):
                see = (k1 - k0) - (q1 - q0) + i + 1
                if see <= 0:
                    continue
                z = softmax_scale * (keys[:see] @ q[q0 + i, h])
                top = z.max()
                w = np.exp(z - top)
                out[q0 + i, h] = (w / w.sum()) @ v[k0:k0 + see, h]
                mass[q0 + i, h] = (w / w.sum()) @ np.abs(v[k0:k0 + see, h])
                lse[q0 + i, h] = top + np.log(w.sum())
                spread[q0 + i, h] = softmax_scale * (np.abs(keys[:see]) @ np.abs(q[q0 + i, h])).max()
    return out, lse, mass, spread
