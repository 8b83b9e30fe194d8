"""Serving steps read back more often: the append's V side in a far pool, a history block by block, prompts attended."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_37626_amd import binding as B
from tests.step_inputs import PAGE, assert_close, bf16, bf16_bits, blocks, to_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def same_codes(got, want, int8):
    nan = (want & 0x7F) == 0x7F if not int8 else np.zeros(want.shape, bool)
    return np.array_equal(got[~nan], want[~nan]) and bool(np.all((got[nan] & 0x7F) == 0x7F))


@pytest.mark.parametrize("batch", [1, 1000], ids=["prompts", "decode"])
def test_append_past_4_gib_on_both_sides(batch):
    # K and V of their own in the last pages of a 2^32-byte pool: a few rows, and a run of rows
    rng = np.random.Generator(np.random.PCG64(50))
    near, far = 4, (1 << 32) // (8 * PAGE * 128) + 9
    host = [blocks(rng, near, 8, 128, False) for _ in range(2)]
    pools = [torch.zeros((far, 8, PAGE, 128), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.ones((far, 8), dtype=torch.float32, device="cuda") for _ in range(2)]
    for pool, scale, (c, s) in zip(pools, scales, host):
        pool[far - near:], scale[far - near:] = dev(c), dev(s)
    slots = np.array([3, PAGE + 1, PAGE + 2] + [3 * PAGE + r for r in range(20, 45)], dtype=np.int32)
    rows = [bf16(rng, len(slots), 8, 128, scale=2.0) for _ in range(2)]
    want = [oracle.step.gqa_append(x, slots, c, s, False) for x, (c, s) in zip(rows, host)]
    desc = B.make_gqa_desc(batch, 32, 8, 128, 3, far)
    B.splash_gqa_append(*[to_bf16(x) for x in rows], dev(slots + np.int32((far - near) * PAGE)), *pools, *scales, desc)
    torch.cuda.synchronize()
    for pool, scale, (c, s) in zip(pools, scales, want):
        assert same_codes(pool[far - near:].cpu().numpy(), c, False)
        assert np.array_equal(scale[far - near:].cpu().numpy(), s)
        assert int(pool[:far - near].count_nonzero()) == 0 and bool((scale[:far - near] == 1).all())


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
@pytest.mark.parametrize("dim", [64, 256])
def test_append_token_by_token_read_back_at_every_page(int8, dim):
    # growing and shrinking rows, K and V of their own, compared after every eighth token and at each page's end
    rng = np.random.Generator(np.random.PCG64(51))
    host = [blocks(rng, 3, 2, dim, int8) for _ in range(2)]
    c, s = [dev(a) for a, _ in host], [dev(b) for _, b in host]
    desc = B.make_gqa_desc(1, 2, 2, dim, 3, 3, B.GQA_INT8 if int8 else B.GQA_E4M3)
    at = [2 * PAGE + r for r in range(PAGE)] + list(range(PAGE)) + [PAGE, PAGE + 1]   # pages 2, 0, 1
    for t, slot in enumerate(at):
        rows = [bf16(rng, 1, 2, dim, scale=2.0 ** ((7 * t + 3 * side) % 23 - 11 + t // 16)) for side in range(2)]
        B.splash_gqa_append(*[to_bf16(x) for x in rows], dev(np.array([slot], np.int32)), *c, *s, desc)
        host = [oracle.step.gqa_append(x, [slot], hc, hs, int8) for x, (hc, hs) in zip(rows, host)]
        if t % 8 == 7 or slot % PAGE == PAGE - 1 or t == len(at) - 1:
            for side in range(2):
                assert np.array_equal(s[side].cpu().numpy(), host[side][1]), (t, side)
                assert same_codes(c[side].cpu().numpy(), host[side][0], int8), (t, side)


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
@pytest.mark.parametrize("dim,kv_heads,group", [(64, 2, 4), (128, 1, 8), (256, 2, 2)])
def test_a_prompt_step_and_its_attention(int8, dim, kv_heads, group):
    """Prompts of several requests: tables, rope, append and the attention of every prompt row, a call a request."""
    S = oracle.step
    rng = np.random.Generator(np.random.PCG64(52))
    lens = np.array([130, 1, 64, 77], np.int32)
    batch, width = len(lens), 3
    pages, rows = batch * width, int(lens.sum()) + 5
    heads = kv_heads * group
    table, taken, taken_out = dev(np.full((batch, width), -1, np.int32)), dev(np.zeros(2, np.int32)), dev(np.zeros(2, np.int32))
    indptr, slots, pos, req = (dev(np.zeros(n, np.int32)) for n in (batch + 1, rows, rows, rows))
    seq, free = dev(lens), rng.permutation(pages).astype(np.int32)
    B.splash_step_tables(seq, 0, dev(free), taken, taken_out, table, pages, indptr, slots, pos, req, new_lens=seq)
    want = S.step_tables(lens, lens, free, 0, np.full((batch, width), -1, np.int32), pages, rows)
    for a, b in zip((table, indptr, slots, pos, req, taken_out), want):
        assert np.array_equal(a.cpu().numpy(), b)
    qkv = to_bf16(bf16(rng, rows, heads + 2 * kv_heads, dim))
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    turned = torch.empty((rows, heads, dim), dtype=torch.bfloat16, device="cuda")
    B.splash_rope(q, pos, B.make_rope(dim, 10000.0 ** (-np.arange(dim // 2) * 2.0 / dim)), out=turned, x2=k)
    kind = torch.int8 if int8 else torch.uint8
    cache = [torch.full((pages, kv_heads, PAGE, dim), 0x7F, dtype=kind, device="cuda") for _ in range(2)]
    scales = [torch.full((pages, kv_heads), float("nan"), dtype=torch.float32, device="cuda") for _ in range(2)]
    host = [S.gqa_append(bf16_bits(x), want[2], c.cpu().numpy(), s.cpu().numpy(), int8)
            for x, c, s in zip((k, v), cache, scales)]
    code = B.GQA_INT8 if int8 else B.GQA_E4M3
    B.splash_gqa_append(k, v, slots, *cache, *scales, B.make_gqa_desc(batch, heads, kv_heads, dim, width, pages, code))
    for c, s, (hc, hs) in zip(cache, scales, host):
        assert np.array_equal(c.cpu().numpy(), hc) and np.array_equal(s.cpu().numpy(), hs, equal_nan=True)
    one = B.make_gqa_desc(1, heads, kv_heads, dim, width, pages, code)
    for b, n in enumerate(int(x) for x in lens):
        at = int(want[1][b])
        out = torch.empty((n, heads, dim), dtype=torch.bfloat16, device="cuda")
        lse = torch.empty((n, heads), dtype=torch.float32, device="cuda")
        ws = torch.empty(B.gqa_workspace_size(one, n), dtype=torch.uint8, device="cuda")
        B.splash_gqa_attend(turned[at:at + n], *cache, *scales, table[b:b + 1], seq[b:b + 1], n, out, lse, one, ws)
        ref = S.gqa_attend(bf16_bits(turned[at:at + n]), host[0][0], host[1][0], host[0][1], host[1][1], want[0][b:b + 1],
                           lens[b:b + 1], n, np.float32(dim ** -0.5), int8)
        assert_close(out, lse, ref, n, dim, f"prompt of {n}")
