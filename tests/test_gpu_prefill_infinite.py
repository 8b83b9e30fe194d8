"""splash_mla_prefill over values and scores that are not finite, wherever the keys lie: in the first step of a tile or a
piece, in steps that every row sees, on the diagonal; in tiles of both widths, one after the other, whole and cut."""
import numpy as np
import pytest
import torch

from paper_2609_37626_amd import binding as B
from tests.layer_inputs import Prompts, assert_prefill, dev

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")

# new rows, keys before them, heads, and the request that is looked at
CALLS = {
    "4 waves": ([300, 20], [420, 0], 2, 0),
    "4 waves, tile after tile": ([600, 601, 599, 7], [0, 30, 64, 0], 64, 1),
    "4 waves, cut": ([300] + [10] * 23, [8000] + [3] * 23, 2, 0),
    "8 waves, cut": ([520, 300], [4000, 2900], 2, 0),
    "8 waves": ([1024], [4096], 72, 0),
}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


class Call:
    """Inputs of N(0, 1); every query's first dim is 64, every key's 0, so that a key's own first dim sets its score apart."""

    def __init__(self, name, seed=0):
        new, old, self.heads, b = CALLS[name]
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()
        self.q_indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.kv_indptr = np.concatenate([[0], np.cumsum(np.array(new) + old)]).astype(np.int32)
        rows, keys = int(self.q_indptr[-1]), int(self.kv_indptr[-1])
        self.q, self.kv, self.key = randn(rows, self.heads, 192), randn(keys, self.heads, 256), randn(keys, 64)
        self.q[..., 0], self.kv[..., 0] = 64.0, 0.0
        self.b, self.new, self.old = b, new[b], old[b]
        self.q0, self.k0, self.h = int(self.q_indptr[b]), int(self.kv_indptr[b]), self.heads - 1

    def tokens(self):
        """One of the first half step, of the second, in steps that all rows see, and on the diagonal."""
        seen_by_all = max(self.old - 130, 70)
        return [3, 40, seen_by_all, self.old + self.new // 3]

    def sees(self, token):
        """The request's rows that see a token, as rows of the call."""
        return slice(self.q0 + max(0, token - self.old), self.q0 + self.new)

    def run(self):
        out = torch.full((self.q.shape[0], self.heads, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.q.shape[0], self.heads), 7.0, device="cuda")
        ws = torch.empty(B.mla_prefill_workspace_size(len(self.q_indptr) - 1, self.q.shape[0], self.heads), dtype=torch.uint8, device="cuda")
        B.splash_mla_prefill(self.q, self.kv[..., :128], self.key, self.kv[..., 128:], dev(self.q_indptr), dev(self.kv_indptr), out, lse, ws)
        torch.cuda.synchronize()
        return out, lse


def same(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("apart", [0.0, -64.0], ids=["a weight like others", "a weight that underflows"])
@pytest.mark.parametrize("value", [INF, -INF, NAN])
def test_a_value_reaches_the_rows_that_see_it_and_no_other(name, apart, value):
    """exp(-64 * 64 / sqrt(192)) is 0 in fp32; the definition's weight is not 0, and the value is infinite with it."""
    for token in Call(name).tokens():
        c = Call(name)
        c.kv[c.k0 + token, c.h, 0] = apart
        clean, clean_lse = c.run()
        assert bool(clean.isfinite().all())
        c.kv[c.k0 + token, c.h, 128 + 77] = value
        out, lse = c.run()
        rows = c.sees(token)
        got = out[rows, c.h, 77].clone()
        assert bool((got.isnan() if np.isnan(value) else got == value).all()), (token, got)
        out[rows, c.h, 77] = clean[rows, c.h, 77]
        assert same(out, clean) and torch.equal(lse, clean_lse), token


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("low", [3, 130])
def test_infinities_before_a_score_that_takes_all_weight(name, low):
    """Old weights times exp2 of the distance to the new score: 0 in fp32."""
    c = Call(name)
    high = c.tokens()[3]
    c.kv[c.k0 + high, c.h, 0] = 64.0
    clean, clean_lse = c.run()
    c.kv[c.k0 + low, c.h, 128 + 3] = -INF
    c.kv[c.k0 + low, c.h, 128 + 127] = INF
    out, lse = c.run()
    rows = c.sees(low)
    assert bool((out[rows, c.h, 3] == -INF).all()) and bool((out[rows, c.h, 127] == INF).all())
    for at in (3, 127):
        out[rows, c.h, at] = clean[rows, c.h, at]
    assert same(out, clean) and torch.equal(lse, clean_lse)


@pytest.mark.parametrize("name", CALLS)
def test_infinities_of_both_signs_are_nan(name):
    c = Call(name)
    clean, _ = c.run()
    first, _, middle, late = c.tokens()
    c.kv[c.k0 + first, c.h, 128], c.kv[c.k0 + middle, c.h, 128], c.kv[c.k0 + middle, c.h, 129] = INF, -INF, INF
    c.kv[c.k0 + late, c.h, 129] = -INF
    out, _ = c.run()
    rows, last = c.sees(middle), c.sees(late)
    assert bool(out[rows, c.h, 0].isnan().all()) and bool(out[last, c.h, 1].isnan().all())
    assert bool((out[rows.start:last.start, c.h, 1] == INF).all())
    out[c.sees(first), c.h, :2] = clean[c.sees(first), c.h, :2]
    assert same(out, clean)


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("shared", [False, True], ids=["k", "key"])
@pytest.mark.parametrize("value", [INF, -INF, NAN])
def test_scores_that_are_not_finite(name, shared, value):
    """A score of +inf or NaN makes its row NaN; one of -inf has no weight: as without the key."""
    for token in Call(name).tokens()[1:]:
        c = Call(name)
        heads = slice(0, c.heads) if shared else slice(c.h, c.h + 1)
        column = c.key[:, 5] if shared else c.kv[:, c.h, 9]
        c.q[..., 133 if shared else 9] = 2.0            # the sign of the score is the key's
        clean, clean_lse = c.run()
        column[c.k0 + token] = value
        out, lse = c.run()
        rows = c.sees(token)
        if value == -INF:
            c.kv[c.k0 + token, heads, 0], column[c.k0 + token] = -64.0, 0.0        # (weight 0 of fp32: the same sums)
            lone, lone_lse = c.run()
            assert same(out, lone) and torch.equal(lse, lone_lse), token
            continue
        assert bool(out[rows, heads].isnan().all()) and bool(lse[rows, heads].isnan().all()), token
        out[rows, heads], lse[rows, heads] = clean[rows, heads], clean_lse[rows, heads]
        assert same(out, clean) and torch.equal(lse, clean_lse), token


@pytest.mark.parametrize("name", CALLS)
def test_rows_whose_every_score_is_minus_infinity(name):
    """No weight at all: zeros, whatever the values are."""
    c = Call(name)
    c.kv[:, c.h, 0] = -INF
    c.kv[c.k0 + 5, c.h, 128:] = INF
    c.kv[c.k0 + c.tokens()[2], c.h, 128:] = NAN
    out, lse = c.run()
    assert bool((out[:, c.h] == 0).all()) and bool(lse[:, c.h].isneginf().all())
    assert bool(out[:, 0].isfinite().all()) and bool(lse[:, 0].isfinite().all())


@pytest.mark.parametrize("new,old,heads", [([2000], [-1000], 2), ([900, 300], [-890, 5000], 2), ([1500] * 3, [-700] * 3, 40)])
def test_rows_that_see_no_key_in_long_calls(new, old, heads):
    """More queries than keys, cut and one tile after the other: the first rows are empty, the others as without them."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()
    keys = np.maximum(np.array(new) + old, 0)
    rows, total = sum(new), int(keys.sum())
    q, kv, key = randn(rows, heads, 192), randn(total, heads, 256), randn(total, 64)

    def run(q, q_at, kv_at):
        out, lse = torch.full((q.shape[0], heads, 128), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((q.shape[0], heads), 7.0, device="cuda")
        ws = torch.empty(B.mla_prefill_workspace_size(len(q_at) - 1, q.shape[0], heads), dtype=torch.uint8, device="cuda")
        B.splash_mla_prefill(q, kv[..., :128], key, kv[..., 128:], dev(np.array(q_at, np.int32)), dev(np.array(kv_at, np.int32)), out, lse, ws)
        torch.cuda.synchronize()
        return out, lse

    q_at, kv_at = np.concatenate([[0], np.cumsum(new)]), np.concatenate([[0], np.cumsum(keys)])
    out, lse = run(q, q_at, kv_at)
    for b in range(len(new)):
        empty = max(0, new[b] - int(keys[b]))
        mine = slice(q_at[b], q_at[b] + empty)
        assert bool((out[mine] == 0).all()) and bool(lse[mine].isneginf().all())
        rest = slice(q_at[b] + empty, q_at[b + 1])
        # float64 over some of the other rows
        for n in {rest.start, (rest.start + rest.stop) // 2, rest.stop - 1}:
            see = int(keys[b]) - (int(q_at[b + 1]) - n) + 1
            k = torch.cat([kv[kv_at[b]:kv_at[b] + see, :, :128], key[kv_at[b]:kv_at[b] + see, None].expand(-1, heads, -1)], -1).double().cpu()
            v = kv[kv_at[b]:kv_at[b] + see, :, 128:].double().cpu()
            z = (k * q[n].double().cpu()).sum(-1) / 192 ** 0.5
            w = torch.softmax(z, 0)
            want, mass = (w[..., None] * v).sum(0), (w[..., None] * v.abs()).sum(0)
            # bf16's half step of the output, and of each weight; scores of a few hundred sums of fp32, |z| < 2^5
            assert bool(((out[n].double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -10) * mass).all()), (b, n)
            # lse: 198 roundings of a score's magnitudes, below 2^6
            assert bool(((lse[n].double().cpu() - torch.logsumexp(z, 0)).abs() <= 198 * 2.0 ** -18 + 2.0 ** -10).all())


@pytest.mark.parametrize("new,old,heads", [([200], [824], 2), ([40], [6000], 1), ([1024], [4096], 72), ([3], [0], 1)])
def test_values_at_the_end_of_the_range(new, old, heads):
    """Values of 2^129 / nk or the type's largest power of two, and weights that come close to the most that moves no
    reference: all scores behind the first 32 keys 6.8 powers of two above theirs."""
    p = Prompts(new, old, heads, seed=6)
    keys, ones = int(p.keys[0]), np.uint16(0x3F80)
    p.q[:], p.kv[..., :128], p.key[:] = 0, 0, 0
    p.q[..., 0] = ones
    p.scale = np.float32(6.8 * np.log(2.0))
    p.kv[32:, :, 0] = ones
    p.kv[..., 128:] = (p.kv[..., 128:] & 0x8000) + ((127 + min(127, 129 - int(np.ceil(np.log2(keys))))) << 7)
    p.kv[..., 128:160] &= 0x7FFF      # sums of one sign
    out, lse = p.run()
    some = sorted({0, heads - 1})
    p.q, p.kv, p.heads = p.q[:, some], p.kv[:, some], len(some)
    assert_prefill(out[:, some], lse[:, some], p.oracle(), keys, f"{new} over {old}, {heads} heads")
