"""The oracle of the calls around the latent cache against values that are not its own (CPU)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_37626_amd.workloads import f32_to_bf16_bits

L = oracle.layer


def f64(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float64))


def test_round_bf16_is_torchs_rounding():
    rng = np.random.Generator(np.random.PCG64(0))
    x = rng.integers(0, 1 << 32, 200000, dtype=np.uint64).astype(np.uint32).view(np.float32)   # NaN, infinities, subnormals
    x = np.concatenate([x, np.float32([0.0, -0.0, 3.3961775e38, 1.0 + 2.0 ** -8, 1.0 + 3 * 2.0 ** -8, 2.0 ** -134])])
    want = torch.from_numpy(x).bfloat16()
    with np.errstate(invalid="ignore"):
        got = L.round_bf16(x.astype(np.float64))
    nan = np.isnan(x)
    assert np.array_equal(got[~nan], want.view(torch.int16).numpy().view(np.uint16)[~nan])
    assert np.all(got[nan] == 0x7FC0)


def test_new_rows_norm_and_turn():
    rng = np.random.Generator(np.random.PCG64(1))
    latent, key, weight = (f32_to_bf16_bits(rng.standard_normal(s, dtype=np.float32)) for s in ((5, 512), (5, 64), (512,)))
    freq, pos = 0.5 ** np.arange(32), np.arange(5, dtype=np.int32) * 1000
    y, r = L.new_rows(latent, key, weight, 1e-3, pos[None], freq, np.zeros(32, dtype=int))
    x = f64(oracle.bf16_bits_to_f64(latent))
    want = torch.nn.functional.rms_norm(x, (512,), f64(oracle.bf16_bits_to_f64(weight)), float(np.float32(1e-3)))
    np.testing.assert_allclose(y, want.numpy(), rtol=2.0 ** -24 + 1e-12)
    k = oracle.bf16_bits_to_f64(key)
    turned = (k[:, :32] + 1j * k[:, 32:]) * np.exp(1j * pos[:, None] * freq)
    np.testing.assert_allclose(r, np.concatenate([turned.real, turned.imag], -1), atol=1e-12)
    y, r = L.new_rows(latent, key)
    assert np.array_equal(y, oracle.bf16_bits_to_f64(latent)) and np.array_equal(r, k)


def test_row_bytes_by_hand():
    latent, key = np.zeros((2, 512)), np.zeros((2, 64))
    latent[0, 0], latent[0, 1], latent[0, 200], key[0, 3] = 448.0, -1.0, 449.0, 2.0 ** -10
    latent[1, 0], key[1, 0] = np.inf, 896.0
    codes, scale = L.row_bytes(latent, key, L.E4M3)
    assert scale.tolist() == [np.float32(449.0) / np.float32(448.0), 2.0]
    assert codes[0, 200] == 0x7E and codes[1, 512] == 0x7E and codes[1, 0] == 0x7E and codes[1, 1] == 0
    rows, none = L.row_bytes(latent, key, L.LATENT_ROWS)
    assert none is None
    scales = rows[:, 512:528].copy().view("<f4")
    assert scales.tolist() == [[1.0, 2.0, 1.0, 1.0], [1.0, 1.0, 1.0, 1.0]]   # 449 is past 448; zeros and infinities alone: 1
    assert rows[0, 0] == 0x7E and rows[0, 1] == 0xB8 and rows[0, 200] == 0x76 and rows[1, 0] == 0x7E
    assert rows[0, 528 + 6:528 + 8].copy().view("<u2")[0] == f32_to_bf16_bits(np.float32([2.0 ** -10]))[0]
    bits, none = L.row_bytes(latent, key, L.BF16)
    assert none is None and bits[0, 0] == 0x43E0 and bits[1, 0] == 0x7F80


@pytest.mark.parametrize("kind", [0, 1, 2])
def test_rows_come_back_as_they_were_put(kind):
    rng = np.random.Generator(np.random.PCG64(2))
    latent, key = np.exp2(rng.integers(-3, 3, (6, 512))), np.exp2(rng.integers(-3, 3, (6, 64)))
    latent[:, 0] = 448.0 if kind else 256.0     # the scales are 1
    rows, scales = L.row_bytes(latent, key, kind)
    shape, t = {0: ((3, 64, 576), np.uint16), 1: ((3, 64, 576), np.uint8), 2: ((3, 64, 656), np.uint8)}[kind]
    slots = np.array([130, 64, -1, 191, 192, 0])
    pool, pool_scales = L.put_rows(np.zeros(shape, t), np.ones((3, 64), np.float32) if kind == 1 else None, slots, rows, scales)
    got = L.read_rows(pool, pool_scales, kind)
    for i in (0, 1, 3, 5):
        assert np.array_equal(got[slots[i] // 64, slots[i] % 64], np.concatenate([latent[i], key[i]]))
    assert np.count_nonzero(got.any(-1)) == 4
    table = np.array([[2, 9], [0, 1]], np.int32)
    out = L.gather(pool, pool_scales, kind, table, np.array([2, 64]), np.array([1, 2, 4]), 6, 0x1234)
    assert np.all(out[[0, 4, 5]] == 0x1234)
    values = oracle.bf16_bits_to_f64(out)
    assert np.array_equal(values[1], np.concatenate([latent[0], key[0]])) and np.array_equal(values[2], np.concatenate([latent[1], key[1]]))
    assert np.all(out[3] == 0)                                           # token 65 of page 1: nothing written there
    assert np.all(L.gather(pool, pool_scales, kind, table, np.array([64, -1]), np.array([0, 1, 2]), 2, 7) == 0)   # no page; before 0


def test_projections_and_prefill_match_torch():
    rng = np.random.Generator(np.random.PCG64(3))

    def bits(*shape):
        return f32_to_bf16_bits(rng.standard_normal(shape, dtype=np.float32))

    x, w = bits(3, 2, 8), bits(2, 8, 5)
    got, mass = L.project(x, w, False)
    X, W = f64(oracle.bf16_bits_to_f64(x)), f64(oracle.bf16_bits_to_f64(w))
    np.testing.assert_allclose(got, torch.einsum("nhd,hdc->nhc", X, W).numpy(), atol=1e-12)
    assert np.all(mass >= np.abs(got) - 1e-12)
    np.testing.assert_allclose(L.project(bits(3, 2, 5), w, True)[0].shape, (3, 2, 8))
    q, k, key, v = bits(9, 2, 192), bits(12, 2, 128), bits(12, 64), bits(12, 2, 128)
    out, lse, mass, spread = L.prefill(q, k, key, v, [1, 4, 4, 9], [0, 7, 9, 12], 0.1)
    assert np.all(out[0] == 0) and np.isneginf(lse[0]).all() and np.isneginf(lse[[4, 5]]).all() and np.all(out[[4, 5]] == 0)
    Q, K, R, V = (f64(oracle.bf16_bits_to_f64(t)) for t in (q, k, key, v))
    K = torch.cat([K, R[:, None].expand(-1, 2, -1)], -1)
    for rows, keys in ((slice(1, 4), slice(0, 7)), (slice(6, 9), slice(9, 12))):
        n, m = rows.stop - rows.start, keys.stop - keys.start
        mask = torch.arange(m)[None] <= m - n + torch.arange(n)[:, None]
        want = torch.nn.functional.scaled_dot_product_attention(Q[rows].transpose(0, 1), K[keys].transpose(0, 1),
                                                                V[keys].transpose(0, 1), attn_mask=mask, scale=0.1)
        np.testing.assert_allclose(out[rows], want.transpose(0, 1).numpy(), atol=1e-12)
        z = torch.einsum("nhd,khd->nhk", Q[rows], K[keys]) * 0.1
        z = z.masked_fill(~mask[:, None], -torch.inf)
        np.testing.assert_allclose(lse[rows], torch.logsumexp(z, -1).numpy(), atol=1e-12)
    assert np.all(mass[1:4] >= np.abs(out[1:4]) - 1e-12) and np.all(spread[1:4] > 0)
