"""splash_mla_append and splash_mla_gather against the float64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_37626_amd import binding as B
from tests.layer_inputs import (FORMATS, FREQ, PAGE, bf16, bf16_bits, dev, key_tolerance, pool_bytes, pool_of, rng_of, rope_of,
                                table_of, to_bf16, to_pool)

pytestmark = pytest.mark.gpu
L = oracle.layer


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def check_append(fmt, latent, key, slots, pages, weight=None, eps=1e-6, positions=None, interleaved=False, axis=None, scale=1.0,
                 before=0, seed=0):
    """Appends to a random pool and compares every byte of it: the latent's exactly, the key's to its rounding and
    2^-20 of the pair, whose magnitude may also decide a per-token scale."""
    kind, n = FORMATS[fmt], len(slots)
    rng = rng_of(seed + 1000)
    pool, scales = pool_of(rng, pages, kind)
    rows = np.concatenate([bf16(rng, n, before), latent, key], -1)
    wide = to_bf16(rows)
    d_pool, d_scales = to_pool(pool, kind), None if scales is None else dev(scales)
    desc = B.make_desc(2, 16, 4, pages, kind, d_scales)
    axes = None if positions is None else np.atleast_2d(positions)
    B.splash_mla_append(wide[:, before:before + 512], wide[:, before + 512:], dev(np.asarray(slots, np.int32)), d_pool, d_scales,
                        desc, norm_weight=None if weight is None else to_bf16(weight), norm_eps=eps,
                        positions=None if positions is None else dev(np.asarray(positions, np.int32)),
                        rope=None if positions is None else rope_of(interleaved, axis, scale))
    torch.cuda.synchronize()
    y, r = L.new_rows(latent, key, weight, eps, axes, FREQ, np.zeros(32, int) if axis is None else axis, interleaved, scale)
    want, want_scales = L.put_rows(pool, scales, slots, *L.row_bytes(y, r, kind))
    got = d_pool.view(torch.int16).cpu().numpy().view(np.uint16) if kind == B.KV_BF16 else d_pool.cpu().numpy()
    got_scales = None if scales is None else d_scales.cpu().numpy()
    real = [(t, s) for t, s in enumerate(slots) if 0 <= s < PAGE * pages]
    mine = np.zeros((pages, PAGE), bool)
    for _, s in real:
        mine[s // PAGE, s % PAGE] = True
    assert np.array_equal(got[~mine], pool[~mine])          # every other row as it was
    if scales is not None:
        assert np.array_equal(got_scales[~mine], scales[~mine], equal_nan=True)
    if not real:
        return
    t, at = np.array([t for t, _ in real]), np.array([s for _, s in real])
    g, w = got[at // PAGE, at % PAGE], want[at // PAGE, at % PAGE]
    more = key_tolerance(key, r, interleaved, scale)[t] if positions is not None else np.zeros((len(t), 64))
    fin = np.isfinite(r[t])
    if kind != B.KV_FP8_E4M3:
        same = 512 if kind == B.KV_BF16 else 528
        if kind == B.KV_BF16:
            nan = (w[:, :512] & 0x7FFF) > 0x7F80
            assert np.array_equal(g[:, :512][~nan], w[:, :512][~nan]) and np.all((g[:, :512][nan] & 0x7FFF) > 0x7F80)
            bits = g[:, 512:]
        else:
            nan = (w[:, :512] & 0x7F) == 0x7F
            assert np.array_equal(g[:, :512][~nan], w[:, :512][~nan]) and np.all((g[:, :512][nan] & 0x7F) == 0x7F)
            assert np.array_equal(g[:, 512:same], w[:, 512:same])
            bits = np.ascontiguousarray(g[:, 528:]).view("<u2")
        v = oracle.bf16_bits_to_f64(bits)
        assert np.array_equal(np.isfinite(v), fin)
        err = np.abs(np.where(fin, v, 0) - np.where(fin, r[t], 0))
        assert np.all(err <= 2.0 ** -8 * np.abs(np.where(fin, r[t], 0)) + np.where(fin, more, 0) + 2.0 ** -134), err.max()
        return
    gs, ws = got_scales[at // PAGE, at % PAGE].astype(np.float64), want_scales[at // PAGE, at % PAGE].astype(np.float64)
    assert np.all(np.abs(gs - ws) <= 2.0 ** -23 * ws + np.nan_to_num(more).max(-1) / 448)
    yy = np.concatenate([y[t], r[t]], -1)
    v = oracle.e4m3_bits_to_f64(g)
    assert np.array_equal(np.isnan(v), np.isnan(yy))
    ok = np.isfinite(yy)
    assert np.all((v == np.copysign(448.0, yy))[np.isinf(yy)])
    # half a step of E4M3 (2^-4, below its normals 2^-10 of the scale), the quotient's roundings
    tol = gs[:, None] * (2.0 ** -10) + np.where(ok, np.abs(yy), 0) * (2.0 ** -4 + 2.0 ** -20) + \
        np.concatenate([np.zeros((len(t), 512)), np.nan_to_num(more)], -1)
    with np.errstate(all="ignore"):
        assert np.all((np.abs(v * gs[:, None] - yy) <= tol)[ok])
    exact = (gs == ws)
    assert np.array_equal(g[exact][:, :512][~np.isnan(yy[exact][:, :512])], w[exact][:, :512][~np.isnan(yy[exact][:, :512])])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,norm,before", [(1, True, 0), (3, False, 8), (67, True, 1536), (1030, True, 0)])
def test_append(fmt, interleaved, n, norm, before):
    rng = rng_of(n)
    pages = n // 40 + 2
    latent, key = bf16(rng, n, 512), bf16(rng, n, 64)
    latent = oracle.layer.round_bf16(oracle.bf16_bits_to_f64(latent) * np.exp2(rng.integers(-9, 9, (n, 1))))
    slots = rng.permutation(pages * PAGE)[:n].astype(np.int32)
    check_append(fmt, latent, key, slots, pages, bf16(rng, 512) if norm else None,
                 positions=rng.integers(0, 1 << 20, n), interleaved=interleaved, before=before, seed=n)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_skips_slots_outside_the_pool(fmt):
    rng = rng_of(5)
    check_append(fmt, bf16(rng, 7, 512), bf16(rng, 7, 64), [-1, 128, 5, 1 << 30, -(1 << 31), 127, (1 << 31) - 1], 2)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_without_rope_takes_the_key_as_it_is(fmt):
    rng = rng_of(6)
    key = bf16(rng, 4, 64)
    key[2, 5], key[3, :] = 0x7F80, 0x8000          # an infinity, zeros of the other sign
    check_append(fmt, bf16(rng, 4, 512), key, [1, 2, 70, 0], 2, bf16(rng, 512))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("axes", [2, 4])
def test_append_several_axes(fmt, axes):
    rng = rng_of(axes)
    check_append(fmt, bf16(rng, 40, 512), bf16(rng, 40, 64), rng.permutation(128)[:40], 2, bf16(rng, 512),
                 positions=rng.integers(0, 9999, (axes, 40)), axis=np.arange(32) % axes, scale=1.25, interleaved=axes == 4)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("norm", [False, True])
def test_append_values_out_of_the_ordinary(fmt, norm):
    """Zero rows, NaN, infinities, the type's largest and smallest values, and magnitudes on both sides of every
    scale's border."""
    rng = rng_of(8)
    latent, key = bf16(rng, 12, 512), bf16(rng, 12, 64)
    latent[0], key[0] = 0, 0
    latent[1, 3] = 0x7FC0                             # NaN
    latent[2, 200], latent[2, 400] = 0x7F80, 0xFF80   # infinities
    latent[3] = 0x7F7F                                # the largest
    latent[4], key[4] = 0x0001, 0x0001                # the smallest
    latent[5, :128], latent[5, 128:256] = 0, 0x0080
    latent[6, 0], latent[7, 0] = 0x43E0, 0x43E1       # 448 and the next value, the rows' largest
    latent[8, 130], latent[9, 130] = 0x3F60, 0x3F61   # 0.875 and the next
    latent[8, 128:256], latent[9, 128:256] = 0x3F60, 0x3F61
    key[10, 7] = 0x7FC0
    check_append(fmt, latent, key, rng.permutation(128)[:12], 2, bf16(rng, 512) if norm else None, eps=0.0 if norm else 1.0)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_and_gather_past_4_gib(fmt):
    kind = FORMATS[fmt]
    width = 656 if fmt == "latent" else 576
    pages = (1 << 32) // (PAGE * (1152 if fmt == "bf16" else width)) + 9
    rng = rng_of(9)
    n = 70
    latent, key = bf16(rng, n, 512), bf16(rng, n, 64)
    pool = torch.zeros((pages, PAGE, width), dtype=torch.bfloat16 if fmt == "bf16" else torch.uint8, device="cuda")
    scales = torch.ones((pages, PAGE), device="cuda") if fmt == "e4m3" else None
    desc = B.make_desc(1, 16, 2, pages, kind, scales)
    slots = (pages - 2) * PAGE + np.arange(n)
    B.splash_mla_append(to_bf16(latent), to_bf16(key), dev(slots.astype(np.int32)), pool, scales, desc)
    assert int(pool[:pages - 2].count_nonzero()) == 0
    want, ws = L.row_bytes(*L.new_rows(latent, key), kind)
    small = [np.zeros((2, PAGE, width), want.dtype), None if ws is None else np.ones((2, PAGE), np.float32)]
    small = L.put_rows(*small, np.arange(n), want, ws)
    outs = torch.empty((n, 576), dtype=torch.bfloat16, device="cuda")
    B.splash_mla_gather(pool, dev(np.array([[pages - 2, pages - 1]], np.int32)), dev(np.array([0, n], np.int32)), outs[:, :512],
                        outs[:, 512:], desc)
    torch.cuda.synchronize()
    ref = L.gather(*small, kind, np.array([[0, 1]], np.int32), [0], [0, n], n, 0)
    assert np.array_equal(bf16_bits(outs), ref)


def check_gather(fmt, lens, begin=None, spare=0, cut=0, seed=0, first=0, bad=(), one_buffer=True):
    kind, rng = FORMATS[fmt], rng_of(seed)
    held = [-(-(int(n) + (0 if begin is None else int(begin[b]))) // PAGE) for b, n in enumerate(lens)]
    pages = sum(held) + 2
    pool, scales = pool_of(rng, pages, kind)
    table = table_of(rng, held, pages)
    for b, k, page in bad:
        table[b, k] = page
    indptr = (first + np.concatenate([[0], np.cumsum(lens)])).astype(np.int32)
    rows = max(int(indptr[-1]) + spare - cut, 0)
    fill = np.uint16(0x40E0)   # 7.0
    if one_buffer:
        out = torch.full((rows, 576), 7.0, dtype=torch.bfloat16, device="cuda")
        latent, key = out[:, :512], out[:, 512:]
    else:
        latent, key = (torch.full((rows, w), 7.0, dtype=torch.bfloat16, device="cuda") for w in (512, 64))
    d_scales = None if scales is None else dev(scales)
    desc = B.make_desc(len(lens), 16, table.shape[1], pages, kind, d_scales)
    B.splash_mla_gather(to_pool(pool, kind), dev(table), dev(indptr), latent, key, desc,
                        key_begin=None if begin is None else dev(np.array(begin, np.int32)))
    torch.cuda.synchronize()
    want = L.gather(pool, scales, kind, table, np.zeros(len(lens), int) if begin is None else begin, indptr, rows, fill)
    got = np.concatenate([bf16_bits(latent), bf16_bits(key)], -1)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("lens", [[1], [64], [65], [0, 1, 0, 63, 7, 0], [129, 0, 200], [3000, 1, 517]])
def test_gather(fmt, lens):
    check_gather(fmt, lens, seed=len(lens))
    check_gather(fmt, lens, begin=[(37 * b) % 130 for b in range(len(lens))], spare=11, seed=1, one_buffer=False)


@pytest.mark.parametrize("fmt", FORMATS)
def test_gather_many_requests(fmt):
    rng = rng_of(3)
    check_gather(fmt, rng.integers(0, 3, 900), seed=4)
    check_gather(fmt, [0] * 200 + [5] + [0] * 300 + [70] + [0] * 10, seed=5, spare=3)


@pytest.mark.parametrize("fmt", FORMATS)
def test_gather_of_rows_outside(fmt):
    check_gather(fmt, [100, 90], cut=30, seed=6)                       # outputs end inside a request
    check_gather(fmt, [100, 90], first=13, seed=7)                     # rows before the first are left
    check_gather(fmt, [130, 90], bad=[(0, 1, -1), (1, 0, 1 << 20)], seed=8)   # pages outside the pool: zeros


@pytest.mark.parametrize("fmt", FORMATS)
def test_gather_of_tokens_outside_the_table(fmt):
    check_gather(fmt, [70], begin=[-3], seed=9)
    kind, rng = FORMATS[fmt], rng_of(10)
    pool, scales = pool_of(rng, 2, kind)
    d_scales = None if scales is None else dev(scales)
    out = torch.full((100, 576), 7.0, dtype=torch.bfloat16, device="cuda")
    desc = B.make_desc(1, 16, 1, 2, kind, d_scales)
    B.splash_mla_gather(to_pool(pool, kind), dev(np.array([[1]], np.int32)), dev(np.array([0, 100], np.int32)), out[:, :512],
                        out[:, 512:], desc)
    torch.cuda.synchronize()
    want = L.gather(pool, scales, kind, np.array([[1]], np.int32), [0], [0, 100], 100, 0)
    assert np.array_equal(bf16_bits(out), want) and not bf16_bits(out)[64:].any()


def test_nothing_to_do():
    desc = B.make_desc(0, 16, 1, 1, B.KV_BF16)
    pool = torch.zeros((1, PAGE, 576), dtype=torch.bfloat16, device="cuda")
    none = torch.empty((0, 576), dtype=torch.bfloat16, device="cuda")
    B.splash_mla_append(none[:, :512], none[:, 512:], dev(np.zeros(0, np.int32)), pool, None, desc)
    B.splash_mla_gather(pool, torch.empty((0, 1), dtype=torch.int32, device="cuda"), dev(np.zeros(1, np.int32)), none[:, :512],
                        none[:, 512:], desc)
    torch.cuda.synchronize()
    assert not pool_bytes(pool).any()
