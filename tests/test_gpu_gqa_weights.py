"""splash_gqa_attend where softmax weights and V block scales lie far apart and decide the result together."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_37626_amd import binding as B
from paper_2609_37626_amd.workloads import f32_to_bf16_bits
from tests.step_inputs import PAGE, Attend, assert_close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def levelled(lens, kv_heads, group, dim, q_chunk, int8, seed, levels):
    """Page p of a history holds scores of about levels(p) powers of two, and its V block a scale of 2^-levels(p), so
    that every page has a like part in the output.  Dim 0 carries the level: queries 32 there, codes level by level."""
    rng = np.random.Generator(np.random.PCG64(seed))
    p = Attend(lens, kv_heads, group, dim, q_chunk, int8, seed)
    n, hq, d = len(lens) * q_chunk, kv_heads * group, dim
    q = rng.standard_normal((n, hq, d)).astype(np.float32)
    q[..., 0] = 32.0
    p.q = f32_to_bf16_bits(q)
    per_code = 32.0 * 2.0 ** -3 * float(p.scale) * np.log2(np.e)  # powers of two of one unit of the code in dim 0
    top = 120 if int8 else 448
    p.ks[:] = 2.0 ** -3
    for x, lo, hi in ((p.k, -2, 2), (p.v, 32, 120)):   # (V: no code is small beside its block's largest)
        vals = rng.integers(lo, hi, x.shape, endpoint=True) * rng.choice([-1.0, 1.0], x.shape)
        x[:] = oracle.step.encode(vals, int8)
    for row, s in zip(p.table, lens):
        for at in range(-(-s // PAGE)):
            code = np.clip(np.round(levels(at) / per_code), -top, top)
            p.k[row[at], :, :, 0] = oracle.step.encode(np.full((kv_heads, PAGE), code), int8)
            held = oracle.step.decode(p.k[row[at], :1, :1, 0], int8)[0, 0] * per_code
            p.vs[row[at]] = 2.0 ** -round(held)
    return p


def check(p, label):
    out, lse = p.attend()
    ref = p.oracle()
    # The bound of a plain problem holds: with no V code small beside its block's
    # largest, what a block's weights lose below 2^-40 of its largest weight is
    # far under the 2^-11 of the weighted |V| that it counts.
    assert_close(out, lse, ref, int(max(p.lens)), p.dim, label)
    assert np.abs(ref[0]).max() > 0


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
@pytest.mark.parametrize("order", ["falling", "rising", "mixed"])
@pytest.mark.parametrize("dim,group,q_chunk", [(64, 4, 1), (64, 9, 8), (128, 8, 1), (128, 8, 4), (128, 16, 8), (256, 2, 1), (256, 8, 8)])
def test_attend_low_scores_under_large_v_scales(int8, order, dim, group, q_chunk):
    # a page of one wave every fourth (or second): levels 33 powers apart from one to its next
    levels = {"falling": lambda at: 33 - 66 * (at // 4 % 2), "rising": lambda at: 66 * (at // 4 % 2) - 33,
              "mixed": lambda at: (at * 37) % 64 - 32}[order]
    check(levelled([300, 700, 64, 5], 2, group, dim, q_chunk, int8, seed=dim + group, levels=levels), f"d{dim} g{group} q{q_chunk} {order}")


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
def test_attend_low_scores_under_large_v_scales_over_many_workgroups(int8):
    # (tiles cut between workgroups, and parts of them joined)
    check(levelled([9000, 3000, 130], 1, 8, 128, 2, int8, seed=3, levels=lambda at: (at * 29) % 44 - 22), "split")


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
def test_attend_two_pages_of_one_wave(int8):
    # page 4 after page 0 in one wave: scores 32 powers of two down, V's scale 2^31 up: a third of the output
    p = levelled([5 * PAGE], 1, 1, 64, 1, int8, seed=4, levels=lambda at: 16 if at == 0 else -16 if at == 4 else -80)
    p.vs[:] = 2.0 ** -31
    p.vs[p.table[0, 4]] = 1.0
    check(p, "two pages")


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
@pytest.mark.parametrize("dim,kv_heads,group", [(64, 2, 4), (128, 1, 16), (128, 8, 1), (256, 2, 8)])
def test_attend_of_few_rows_keeps_weights_past_fp16(int8, dim, kv_heads, group):
    """Values that nearly cancel: bf16's half step of a small result does not hide what a weight was rounded by.

    Two fp16 terms hold a weight to 2^-22 (2^-11 of what 2^-11 leaves), where tolerances() counts 2^-11; the rest of
    its bound stands: bf16's half step, the scores' dz and the sums."""
    rng = np.random.Generator(np.random.PCG64(60 + dim))
    p = Attend([2] * 96, kv_heads, group, dim, 1, int8, seed=61 + dim, exponents=(-7, -7))
    first = rng.integers(8, 40, (kv_heads, dim)) * 2 * rng.choice([-1, 1], (kv_heads, dim))
    for b in range(96):   # the second token's value is -3/2 of the first's
        for place, x in ((0, first), (1, -first * 3 // 2)):
            p.v[p.table[b, 0], :, place] = oracle.step.encode(x.astype(np.float64), int8)
    out, lse = p.attend()
    ref = p.oracle()
    exact, mass, spread = ref[0], ref[2], ref[3]
    dz = (dim + 6) * 2.0 ** -24 * spread + 2.0 ** -21
    sums = (2 + 64) * 2.0 ** -24
    tol = 2.0 ** -8 * np.abs(exact) + (2.0 ** -22 + 2 * dz + 2 * sums)[..., None] * mass * 1.01
    err = np.abs(out.float().cpu().numpy().astype(np.float64) - exact)
    assert (2.0 ** -8 * np.abs(exact) < 2.0 ** -13 * mass).any()   # results that cancel are there
    assert np.all(err <= tol), float((err / tol).max())


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
@pytest.mark.parametrize("power", [8, 10, 18, 24, 27, 30, 40, 60, 100])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("lens,group,q_chunk", [([300, 64, 5], 4, 1), ([9000, 130, 3], 8, 4), ([200, 66], 16, 8)])
def test_attend_scores_past_fp32s_whole_numbers(int8, power, sign, lens, group, q_chunk):
    """Scores of +-2^power and more, where neighbouring fp32 values lie far apart: the keys of the largest score share
    the weight evenly, all others have none; every score positive, or every score negative."""
    rng = np.random.Generator(np.random.PCG64(70 + power))
    dim = 64
    p = Attend(lens, 1, group, dim, q_chunk, int8, seed=71 + power)
    q = np.zeros((len(lens) * q_chunk, group, dim), dtype=np.float32)
    q[..., 0] = np.exp2(np.float32(power + 3)) * rng.integers(64, 128, q.shape[:2]).astype(np.float32) / 64   # (bf16 holds these)
    p.q = f32_to_bf16_bits(q)
    level = rng.integers(1, 4, p.k.shape[:3])
    p.k[:] = 0
    p.k[..., 0] = oracle.step.encode(sign * level.astype(np.float64), int8)
    p.ks[:] = 1.0
    out, lse = p.attend()
    o, l = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    V = oracle.step.decode(p.v, int8) * p.vs[..., None, None].astype(np.float64)
    for b, s in enumerate(lens):
        at = [(p.table[b, j // PAGE], j % PAGE) for j in range(s)]
        for i in range(q_chunk):
            n, row = s - q_chunk + i + 1, b * q_chunk + i
            if n <= 0:
                assert np.all(o[row] == 0) and np.all(np.isneginf(l[row]))
                continue
            have = np.array([sign * level[page, 0, place] for page, place in at[:n]])
            vals = np.array([V[page, 0, place] for page, place in at[:n]])[have == have.max()]
            exact, mass = vals.mean(0), np.abs(vals).mean(0)
            # bf16's half step, and equal weights: 2^-11 where one fp16 term holds them, and one rounding a key
            tol = 2.0 ** -8 * np.abs(exact) + (2.0 ** -11 + (n + 64) * 2.0 ** -24) * mass * 1.01
            assert np.all(np.abs(o[row] - exact) <= tol)
            z = have.max() * 0.125 * q[row, :, 0].astype(np.float64)
            # roundings of log2 e, its product with softmax_scale, the block's factor, the score, two sums, ln 2, its product
            assert np.all(np.abs(l[row] - (z + np.log(len(vals)))) <= 8 * 2.0 ** -24 * np.abs(z) + 2.0 ** -18)
