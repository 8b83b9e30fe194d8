"""Inputs of the grouped-query tests: host arrays, and their device tensors."""
import numpy as np
import torch

import oracle
from paper_2609_37626_amd import binding as B
from paper_2609_37626_amd.workloads import f32_to_bf16_bits

PAGE = 64


def bf16(rng, *shape, scale=1.0):
    return f32_to_bf16_bits(rng.standard_normal(shape, dtype=np.float32) * np.float32(scale))


def to_bf16(bits, device="cuda"):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(device).view(torch.bfloat16)


def bf16_bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def blocks(rng, pages, kv_heads, dim, int8, exponents=(-9, -5)):
    """N(0, 1) blocks times powers of two of their own, encoded with those scales: codes, scales."""
    x = rng.standard_normal((pages, kv_heads, PAGE, dim))
    top = 20.0 if int8 else 60.0
    codes = oracle.step.encode(x * top, int8)
    scales = np.exp2(rng.integers(*exponents, size=(pages, kv_heads), endpoint=True)).astype(np.float32)
    return codes, scales


class Attend:
    """One attention problem over a random page placement."""

    def __init__(self, lens, kv_heads, group, dim, q_chunk, int8, seed, extra_pages=3, exponents=(-9, -5), q_scale=1.0):
        rng = np.random.Generator(np.random.PCG64(seed))
        self.lens = np.array(lens, dtype=np.int32)
        self.q_chunk, self.int8, self.dim, self.kv_heads, self.group = q_chunk, int8, dim, kv_heads, group
        held = [-(-int(max(s, 0)) // PAGE) for s in lens]
        width, pages = max(1, max(held)), sum(held) + extra_pages
        perm = rng.permutation(pages).astype(np.int32)
        self.table = np.full((len(lens), width), -1, dtype=np.int32)
        off = 0
        for b, n in enumerate(held):
            self.table[b, :n] = perm[off:off + n]
            off += n
        self.k, self.ks = blocks(rng, pages, kv_heads, dim, int8, exponents)
        self.v, self.vs = blocks(rng, pages, kv_heads, dim, int8, exponents)
        self.q = bf16(rng, len(lens) * q_chunk, kv_heads * group, dim, scale=q_scale)
        self.scale = np.float32(dim ** -0.5)

    def poison(self):
        """NaN codes and scales in every place that no history reaches (int8: -128)."""
        used = np.zeros((self.k.shape[0], PAGE), dtype=bool)
        for b, s in enumerate(self.lens):
            for j in range(int(s)):
                if j // PAGE < self.table.shape[1] and self.table[b, j // PAGE] >= 0:
                    used[self.table[b, j // PAGE], j % PAGE] = True
        bad = np.int8(-128) if self.int8 else np.uint8(0xFF)
        for codes in (self.k, self.v):
            codes.transpose(0, 2, 1, 3)[~used] = bad
        for scales in (self.ks, self.vs):
            scales[~used.any(1)] = np.nan
        return self

    def desc(self):
        return B.make_gqa_desc(len(self.lens), self.kv_heads * self.group, self.kv_heads, self.dim, self.table.shape[1],
                               self.k.shape[0], B.GQA_INT8 if self.int8 else B.GQA_E4M3)

    def device(self):
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
        return dict(q=to_bf16(self.q), k_pages=dev(self.k), v_pages=dev(self.v), k_scales=dev(self.ks), v_scales=dev(self.vs),
                    block_table=dev(self.table), seq_lens=dev(self.lens))

    def outputs(self):
        n = len(self.lens) * self.q_chunk
        return (torch.full((n, self.kv_heads * self.group, self.dim), 7.0, dtype=torch.bfloat16, device="cuda"),
                torch.full((n, self.kv_heads * self.group), 7.0, dtype=torch.float32, device="cuda"))

    def workspace(self):
        return torch.empty(B.gqa_workspace_size(self.desc(), self.q_chunk), dtype=torch.uint8, device="cuda")

    def attend(self):
        out, lse = self.outputs()
        t = self.device()
        B.splash_gqa_attend(t["q"], t["k_pages"], t["v_pages"], t["k_scales"], t["v_scales"], t["block_table"],
                            t["seq_lens"], self.q_chunk, out, lse, self.desc(), self.workspace())
        torch.cuda.synchronize()
        return out, lse

    def oracle(self):
        return oracle.step.gqa_attend(self.q, self.k, self.v, self.ks, self.vs, self.table, self.lens, self.q_chunk,
                                      self.scale, self.int8)


def tolerances(ref, keys, dim):
    """Element-wise bounds on |out - exact| and |lse - exact|.

    A score is a sum of `dim` exact products in fp32: off by at most dim + 2
    roundings (2^-24 each) of the sum of magnitudes, `spread`, the last two for
    the block's scale and softmax_scale * log2 e; its exponent's argument and
    exp2 add 2^-24 |z| (in `spread` again) and 2^-22.  A weight therefore is off
    by dz relative, and by half a step of fp16, 2^-11, where it meets V (or by
    2^-25 of a sum of at least 2^6 where it is subnormal).  The sums of weights
    and of products over the keys round to fp32 once a key at most.  Output:
    bf16, half a step 2^-8."""
    out, lse, mass, spread = ref
    dz = (dim + 6) * 2.0 ** -24 * spread + 2.0 ** -21
    sums = (keys + 64) * 2.0 ** -24
    tol_out = 2.0 ** -8 * np.abs(out) + (2.0 ** -11 + 2 * dz + 2 * sums)[..., None] * mass * 1.01 + \
        keys * 2.0 ** -31 * (mass.max(-1, keepdims=True) if mass.size else 0)
    return tol_out, dz + sums + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse), lse, 0))


def assert_close(out, lse, ref, keys, dim, label=""):
    tol_out, tol_lse = tolerances(ref, keys, dim)
    o, l = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    empty = np.isneginf(ref[1])
    assert np.array_equal(np.isneginf(l), empty), label
    assert np.all(o[empty] == 0), label
    err_o, err_l = np.abs(o - ref[0]), np.abs(np.where(empty, 0, l) - np.where(empty, 0, ref[1]))
    print(f"{label}: out {err_o.max():.2e} of {tol_out.max():.2e}, lse {err_l.max():.2e}", flush=True)
    assert np.all(err_o <= tol_out), (label, float((err_o - tol_out).max()))
    assert np.all(err_l <= tol_lse), (label, float((err_l - tol_lse).max()))
