"""The step oracle against values that are not its own (CPU)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_37626_amd.workloads import f32_to_bf16_bits

S = oracle.step


def test_encode_matches_torch_float8_and_rounds_int8_to_even():
    rng = np.random.Generator(np.random.PCG64(0))
    x = np.concatenate([rng.uniform(-448, 448, 20000), rng.uniform(-0.02, 0.02, 5000)]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(S.encode(x, False), want)
    assert S.encode([0.5, 1.5, -2.5, 200.0, -200.0, np.nan], True).tolist() == [0, 2, -2, 127, -127, 0]
    assert S.encode([np.inf, -np.inf, 1e9], False).tolist() == [0x7E, 0xFE, 0x7E]
    assert S.encode([np.nan], False).tolist() == [0x7F]


def test_attend_matches_torch_float64_attention():
    rng = np.random.Generator(np.random.PCG64(1))
    lens, q_chunk, hk, g, d = [130, 65], 3, 2, 4, 64
    table = np.array([[4, 0, 2], [1, 3, -1]], dtype=np.int32)
    codes = [S.encode(rng.standard_normal((5, hk, 64, d)) * 50, False) for _ in range(2)]
    scales = [np.exp2(rng.integers(-8, -4, (5, hk))).astype(np.float32) for _ in range(2)]
    q = f32_to_bf16_bits(rng.standard_normal((6, hk * g, d), dtype=np.float32))
    out, lse, mass, spread = S.gqa_attend(q, codes[0], codes[1], scales[0], scales[1], table, lens, q_chunk, 0.125, False)
    full = [torch.from_numpy(c).view(torch.float8_e4m3fn).double() * torch.from_numpy(s).double()[:, :, None, None]
            for c, s in zip(codes, scales)]
    qt = torch.from_numpy(oracle.bf16_bits_to_f64(q))
    for b, s in enumerate(lens):
        k, v = [f[table[b, :-(-s // 64)]].transpose(0, 1).reshape(hk, -1, d)[:, :s].repeat_interleave(g, 0) for f in full]
        rows = qt[b * q_chunk:(b + 1) * q_chunk].transpose(0, 1)
        mask = torch.arange(s)[None] <= s - q_chunk + torch.arange(q_chunk)[:, None]
        want = torch.nn.functional.scaled_dot_product_attention(rows, k, v, attn_mask=mask, scale=0.125)
        np.testing.assert_allclose(out[b * q_chunk:(b + 1) * q_chunk], want.transpose(0, 1).numpy(), atol=1e-12)
    assert np.all(mass >= np.abs(out) - 1e-12) and np.all(spread > 0) and np.all(np.isfinite(lse))


def test_attend_of_one_key_returns_its_value_and_of_none_nothing():
    rng = np.random.Generator(np.random.PCG64(2))
    k = S.encode(rng.standard_normal((1, 1, 64, 64)) * 50, True)
    one = np.ones((1, 1), dtype=np.float32)
    q = f32_to_bf16_bits(rng.standard_normal((2, 1, 64), dtype=np.float32))
    out, lse, _, _ = S.gqa_attend(q, k, k, one, one, np.zeros((1, 1), np.int32), [1], 2, 1.0, True)
    assert np.all(out[0] == 0) and np.isneginf(lse[0, 0])
    assert np.array_equal(out[1, 0], k[0, 0, 0].astype(np.float64))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_is_a_complex_turn_and_keeps_relative_positions(interleaved):
    rng = np.random.Generator(np.random.PCG64(3))
    x, y = rng.standard_normal((2, 4, 3, 16))
    freq, axis = 0.1 ** np.arange(8), np.array([0, 0, 1, 1, 1, 2, 2, 2])
    p = rng.integers(0, 1000, (3, 4))
    pairs = (lambda z: z[..., 0::2] + 1j * z[..., 1::2]) if interleaved else (lambda z: z[..., :8] + 1j * z[..., 8:])
    want = pairs(x) * np.exp(1j * p[axis].T * freq)[:, None]
    np.testing.assert_allclose(pairs(S.rope(x, p, freq, axis, interleaved)), want, atol=1e-12)
    dot = lambda shift: (S.rope(x, p + shift, freq, axis, interleaved) * S.rope(y, p + shift + 5, freq, axis, interleaved)).sum(-1)
    np.testing.assert_allclose(dot(0), dot(77), atol=1e-9)


def test_append_scales_and_rescaling():
    # 448 * 2^-7 = 3.5 holds 3.5 and not 3.75; an older block at 2^-9 goes to 2^-6
    codes = S.encode(np.full((1, 1, 64, 64), 100.0), False)
    scales = np.full((1, 1), 2.0 ** -9, dtype=np.float32)
    rows = np.zeros((1, 1, 64), dtype=np.float32)
    for value, e in [(3.5, -7), (3.75, -6), (0.1, -9)]:
        rows[0, 0, 3] = value
        c, s = S.gqa_append(f32_to_bf16_bits(rows), [5], codes, scales, False)
        assert s[0, 0] == 2.0 ** e
        kept = S.decode(c[0, 0, :5], False) * s[0, 0]
        assert np.all(np.abs(kept - 100 * 2.0 ** -9) <= 100 * 2.0 ** -9 * 2.0 ** -4)
        assert np.array_equal(c[0, 0, 6:], codes[0, 0, 6:])
        bf = oracle.bf16_bits_to_f64(f32_to_bf16_bits(rows))[0, 0, 3]
        assert abs(S.decode(c[0, 0, 5], False)[3] * s[0, 0] - bf) <= abs(bf) * 2.0 ** -4
    # place 0 starts the block anew: the old scale does not hold it up
    c, s = S.gqa_append(f32_to_bf16_bits(rows), [0], codes, np.full((1, 1), 8.0, np.float32), False)
    assert s[0, 0] == 2.0 ** -12 and 0.1 <= 448 * 2.0 ** -12


def test_tables_cover_every_new_token_once():
    rng = np.random.Generator(np.random.PCG64(4))
    lens = rng.integers(0, 400, 20)
    new = np.minimum(rng.integers(0, 200, 20), lens)
    held = [S.pages_of(s - n) for s, n in zip(lens, new)]
    perm = rng.permutation(200).astype(np.int32)
    table = np.full((20, 7), -1, np.int32)
    off = 0
    for b, n in enumerate(held):
        table[b, :n] = perm[off:off + n]
        off += n
    out, indptr, slots, positions, requests, taken = S.step_tables(lens, new, perm[off:], 0, table, 200, 4096)
    assert indptr[-1] == new.sum() and len(set(slots[:indptr[-1]].tolist())) == new.sum()
    assert taken.tolist() == [sum(S.pages_of(s) for s in lens) - sum(held), 0]
    for b in range(20):
        rows = slice(indptr[b], indptr[b + 1])
        assert positions[rows].tolist() == list(range(lens[b] - new[b], lens[b])) and set(requests[rows]) <= {b}
        assert np.array_equal(slots[rows] // 64, out[b, positions[rows] // 64])
    assert np.all(slots[indptr[-1]:] == -1) and np.all(requests[indptr[-1]:] == -1)
