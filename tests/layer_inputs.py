"""Inputs of the latent-attention layer's tests: host arrays, and their device tensors."""
import numpy as np
import torch

import oracle
from paper_2609_37626_amd import binding as B
from paper_2609_37626_amd.workloads import encode_e4m3_per_token, encode_fp8_latent_rows, f32_to_bf16_bits
from tests.step_inputs import bf16, bf16_bits, to_bf16

PAGE = 64
FORMATS = {"bf16": B.KV_BF16, "e4m3": B.KV_FP8_E4M3, "latent": B.KV_FP8_LATENT}
FREQ = 10000.0 ** (-np.arange(32) / 32.0)


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def rng_of(seed):
    return np.random.Generator(np.random.PCG64(seed))


def pool_of(rng, pages, kv_dtype):
    """N(0, 1) rows in the pool's format, and their scales (per-token fp8)."""
    x = rng.standard_normal((pages, PAGE, 576), dtype=np.float32)
    if kv_dtype == B.KV_BF16:
        return f32_to_bf16_bits(x), None
    if kv_dtype == B.KV_FP8_E4M3:
        return encode_e4m3_per_token(x)
    return encode_fp8_latent_rows(x * np.exp2(rng.integers(-3, 1, (pages, PAGE, 1))).astype(np.float32)), None


def to_pool(pool, kv_dtype):
    return to_bf16(pool) if kv_dtype == B.KV_BF16 else dev(pool)


def pool_bytes(t):
    """A pool's or scales' bytes on the host."""
    return t.contiguous().view(torch.uint8).cpu().numpy()


def table_of(rng, held, pages, fill=-1):
    perm = rng.permutation(pages).astype(np.int32)
    table, off = np.full((len(held), max(1, max(held))), fill, np.int32), 0
    for b, n in enumerate(held):
        table[b, :n] = perm[off:off + n]
        off += n
    return table


def rope_of(interleaved=False, axis=None, scale=1.0):
    return B.make_rope(64, FREQ, pair_axis=axis, interleaved=interleaved, scale=scale)


def key_tolerance(key_bits, want, interleaved, scale=1.0):
    """What the turn's fp32 leaves beside its rounding: 2^-20 of the pair."""
    x = np.abs(oracle.bf16_bits_to_f64(key_bits))
    pair = x[..., 0::2] + x[..., 1::2] if interleaved else x[..., :32] + x[..., 32:]
    return 2.0 ** -20 * abs(scale) * (np.repeat(pair, 2, -1) if interleaved else np.concatenate([pair, pair], -1))


class Prompts:
    """One ragged batch: new[b] query rows over old[b] + new[b] keys (old[b] may be negative: rows that see none)."""

    def __init__(self, new, old, heads, seed, q_scale=1.0, packed=True):
        rng = rng_of(seed)
        self.new, self.heads = np.array(new), heads
        self.keys = np.maximum(self.new + np.array(old), 0)
        self.q_indptr = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.kv_indptr = np.concatenate([[0], np.cumsum(self.keys)]).astype(np.int32)
        rows, keys = int(self.q_indptr[-1]), int(self.kv_indptr[-1])
        self.q = bf16(rng, rows, heads, 192, scale=q_scale)
        self.kv = bf16(rng, keys, heads, 256)      # each head's key dims, then its value
        self.key = bf16(rng, keys, 64)
        self.scale = np.float32(192 ** -0.5)
        self.packed = packed

    def run(self, lse=True, spare=3, stream=None):
        """Outputs with `spare` rows behind the last sequence, filled before the call."""
        rows = int(self.q_indptr[-1])
        q = torch.full((rows + spare, self.heads, 192), float("nan"), dtype=torch.bfloat16, device="cuda")
        q[:rows] = to_bf16(self.q)
        kv = to_bf16(self.kv)
        k, v = kv[..., :128], kv[..., 128:]
        if not self.packed:
            k, v = k.contiguous(), v.contiguous()
        out = torch.full((rows + spare, self.heads, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        l = torch.full((rows + spare, self.heads), 7.0, device="cuda") if lse else None
        ws = torch.empty(B.mla_prefill_workspace_size(len(self.new), rows + spare, self.heads), dtype=torch.uint8, device="cuda")
        B.splash_mla_prefill(q, k, to_bf16(self.key), v, dev(self.q_indptr), dev(self.kv_indptr), out, l, ws,
                             softmax_scale=float(self.scale), stream=stream)
        torch.cuda.synchronize()
        assert bool((out[rows:] == 7.0).all()) and (l is None or bool((l[rows:] == 7.0).all()))
        return out[:rows], None if l is None else l[:rows]

    def oracle(self):
        return oracle.layer.prefill(self.q, self.kv[..., :128], self.key, self.kv[..., 128:], self.q_indptr, self.kv_indptr,
                                    np.float64(self.scale))


def assert_prefill(out, lse, ref, keys, label=""):
    """A score is a sum of 192 exact products in fp32 times a constant: off by at most 194 roundings (2^-24) of the
    sum of magnitudes, `spread`; its exponent's argument and exp2 add 2^-23 of `spread` and 2^-21.  A weight is off
    by dz relative, and by half a step of bf16, 2^-8, where it meets V.  Sums over the keys round once a key at
    most, and once a part that is joined.  Output: bf16, 2^-8."""
    want, want_lse, mass, spread = ref
    dz = 198 * 2.0 ** -24 * spread + 2.0 ** -21
    sums = (keys + 80) * 2.0 ** -24
    tol = 2.0 ** -8 * np.abs(want) + 1.01 * (2.0 ** -8 + 2 * dz + 2 * sums)[..., None] * mass
    o = out.float().cpu().numpy().astype(np.float64)
    err = np.abs(o - want)
    print(f"{label}: out {err.max() if err.size else 0:.2e}", flush=True)
    assert np.all(err <= tol), (label, float((err - tol).max()))
    if lse is not None:
        l, empty = lse.cpu().numpy().astype(np.float64), np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(l), empty), label
        assert np.all(o[empty] == 0), label
        d = np.abs(np.where(empty, 0, l) - np.where(empty, 0, want_lse))
        assert np.all(d <= dz + sums + 2.0 ** -22 * np.abs(np.where(empty, 0, want_lse))), (label, float(d.max()))
