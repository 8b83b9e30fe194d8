"""splash_mla_prefill against the float64 oracle, and the layer's two forms against each other."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_37626_amd import binding as B
from tests.layer_inputs import (FORMATS, FREQ, PAGE, Prompts, assert_prefill, bf16, bf16_bits, dev, rng_of, rope_of, table_of,
                                to_bf16, to_pool)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def check(p, label="", lse=True):
    out, l = p.run(lse)
    assert_prefill(out, l, p.oracle(), max(1, int(p.keys.max())), label)
    return out, l


@pytest.mark.parametrize("new,old,heads", [
    ([1], [0], 1), ([1], [200], 3), ([2], [0], 2), ([31], [0], 1), ([32], [1], 1), ([33], [0], 2), ([64], [0], 1),
    ([65], [63], 1), ([127], [0], 1), ([128], [0], 3), ([129], [0], 1), ([192], [64], 2), ([300], [77], 2), ([257], [0], 5),
])
def test_one_prompt(new, old, heads):
    check(Prompts(new, old, heads, seed=new[0] + heads), f"{new} over {old}, {heads} heads")


@pytest.mark.parametrize("heads", [1, 4, 20])
def test_ragged(heads):
    check(Prompts([5, 0, 130, 1, 64, 17, 0, 200], [0, 40, 3, 129, 0, 700, 0, 64], heads, seed=heads), f"{heads} heads")


def test_many_requests():
    rng = rng_of(2)
    check(Prompts(rng.integers(0, 4, 150), rng.integers(0, 90, 150), 2, seed=3))
    check(Prompts([0] * 100 + [3] + [0] * 64 + [140], [0] * 50 + [9] * 116, 1, seed=4))


@pytest.mark.parametrize("heads", [1, 3])
def test_few_rows_over_a_long_history(heads):
    check(Prompts([7, 40, 1], [9000, 3001, 6000], heads, seed=5), f"{heads} heads")


@pytest.mark.parametrize("new,old,heads", [([800], [0], 80), ([1000, 1100, 7], [0, 30, 0], 40), ([520, 900], [4000, 10], 2),
                                           ([1, 300, 4096], [0, 0, 0], 25), ([256, 257, 255], [6000, 6000, 6001], 3)])
def test_tiles_whole_and_cut(new, old, heads):
    """Long and short tiles in both widths, whole and over several workgroups: some heads against the oracle."""
    p = Prompts(new, old, heads, seed=sum(new))
    out, lse = p.run()
    some = sorted({0, heads // 2, heads - 1})[:3 if max(new) < 2000 else 1]
    p.q, p.kv, p.heads = p.q[:, some], p.kv[:, some], len(some)
    assert_prefill(out[:, some], lse[:, some], p.oracle(), int(p.keys.max()), f"{new} over {old}, {heads} heads")


def test_more_requests_than_are_ordered():
    rng = rng_of(16)
    check(Prompts(rng.integers(0, 3, 300), rng.integers(0, 40, 300), 1, seed=17))
    p = Prompts([900] + [2] * 299, [100] + [0] * 299, 2, seed=18)
    check(p, "one long prompt before 299 short ones")


def test_rows_that_see_no_key():
    # more query rows than keys: the first ones see none
    check(Prompts([70, 200, 3, 130], [-69, -140, -3, -130], 2, seed=6))


def test_without_lse_and_with_separate_keys_and_values():
    check(Prompts([100, 40], [5, 0], 2, seed=7), lse=False)
    check(Prompts([100, 40], [5, 0], 2, seed=7, packed=False))


@pytest.mark.parametrize("q_scale", [0.0, 30.0, 300.0])
def test_scores_of_other_magnitudes(q_scale):
    check(Prompts([150, 33], [100, 0], 2, seed=8, q_scale=q_scale), f"queries times {q_scale}")


def test_scores_that_grow_along_the_keys():
    """The reference moves at every step."""
    p = Prompts([140], [260], 1, seed=9)
    at = np.arange(p.kv.shape[0])[:, None]
    p.q[..., :128], p.q[..., 128:] = 0x3F80, 0                                     # ones
    p.kv[:, 0, :128] = oracle.layer.round_bf16(np.broadcast_to(at * 0.05, (400, 128)))
    check(p, "growing")
    p.kv[:, 0, :128] = p.kv[::-1, 0, :128]
    check(p, "falling")


@pytest.mark.parametrize("value", [0x7FC0, 0x7F80, 0xFF80], ids=["nan", "inf", "-inf"])
@pytest.mark.parametrize("where", ["k", "key", "v"])
def test_what_a_row_does_not_see_does_not_touch_it(value, where):
    """One token of one request holds a value that is not finite: rows before it, and other requests, are as without it."""
    p = Prompts([150, 90, 20], [33, 0, 7], 2, seed=10)
    clean, clean_lse = p.run()
    token = 33 + 70                     # request 0's row 70 is the first that sees it
    if where == "k":
        p.kv[token, 1, 17] = value
    elif where == "key":
        p.key[token, 3] = value
    else:
        p.kv[token, 1, 128 + 77] = value
    out, lse = p.run()
    touched = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    if where == "v":
        touched[70:150, 1, 77] = True
    else:
        touched[70:150, slice(1, 2) if where == "k" else slice(0, 2)] = True
    assert torch.equal(out[~touched], clean[~touched])
    rows = touched.any(-1)
    if where == "v":
        assert torch.equal(lse, clean_lse)
        want = {0x7FC0: float("nan"), 0x7F80: float("inf"), 0xFF80: float("-inf")}[value]
        got = out[70:150, 1, 77]
        assert bool(got.isnan().all() if value == 0x7FC0 else (got == want).all())
    else:
        assert torch.equal(lse[~rows], clean_lse[~rows])
        if value == 0x7FC0:
            assert bool(out[rows].isnan().all()) and bool(lse[rows].isnan().all())


def test_scores_of_minus_infinity():
    """A key that scores -inf has no weight; a row whose every score is -inf is empty."""
    p = Prompts([3], [2], 1, seed=11)
    p.q[..., :128], p.q[..., 128:] = 0x3F80, 0
    p.kv[1, 0, 0] = 0xFF80
    out, lse = check(p, "one key")
    p.kv[:, 0, 0] = 0xFF80
    out, lse = p.run()
    assert bool((out == 0).all()) and bool(lse.isneginf().all())


def test_indptr_outside_its_range_is_cut_off():
    p = Prompts([100, 60], [0, 10], 2, seed=12)
    full, _ = p.run(spare=0)
    p.q_indptr, p.kv_indptr = np.array([0, 100, 160], np.int32), np.array([0, 100, 170], np.int32)
    out, lse = (torch.full((160, 2, n), 7.0, dtype=t, device="cuda").squeeze(-1) for n, t in ((128, torch.bfloat16), (1, torch.float32)))
    kv = to_bf16(p.kv)
    ws = torch.empty(B.mla_prefill_workspace_size(3, 160, 2), dtype=torch.uint8, device="cuda")
    B.splash_mla_prefill(to_bf16(p.q), kv[..., :128], to_bf16(p.key), kv[..., 128:], dev(np.array([-5, 100, 160, 1 << 30], np.int32)),
                         dev(np.array([-9, 100, 170, 1 << 30], np.int32)), out, lse, ws)
    torch.cuda.synchronize()
    assert torch.equal(out, full)


def test_same_bits_again_and_on_another_stream():
    p = Prompts([300, 70, 5], [0, 1000, 64], 4, seed=13)
    out, lse = p.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again, lse2 = p.run()
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    torch.cuda.synchronize()
    third, _ = p.run(stream=s)
    assert torch.equal(out, third)


def test_captured_and_replayed():
    """One graph of the layer's calls, replayed with other inputs and eager work between."""
    rng = rng_of(14)
    heads, rows = 4, 90
    q, kv, key = to_bf16(bf16(rng, rows, heads, 192)), to_bf16(bf16(rng, rows, heads, 256)), to_bf16(bf16(rng, rows, 64))
    w = to_bf16(bf16(rng, heads, 256, 512, scale=512 ** -0.5))
    latent = to_bf16(bf16(rng, rows, 512))
    indptr, slots, positions = dev(np.array([0, 30, 90], np.int32)), dev(np.arange(rows, dtype=np.int32)), dev(np.arange(rows, dtype=np.int32))
    pool = torch.zeros((2, PAGE, 656), dtype=torch.uint8, device="cuda")
    desc, rope = B.make_desc(2, 16, 2, 2, B.KV_FP8_LATENT), rope_of(True)
    table = dev(np.array([[0, 1], [1, 0]], np.int32))
    ws = torch.empty(B.mla_prefill_workspace_size(2, rows, heads), dtype=torch.uint8, device="cuda")

    def outputs():
        return [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in
                ((rows, heads, 128), (rows, heads, 576), (rows, heads, 128), (rows, 576))]

    def calls(out, packed, y, dense):
        B.splash_mla_append(latent, key, slots, pool, None, desc, positions=positions, rope=rope)
        B.splash_mla_gather(pool, table, indptr, dense[:, :512], dense[:, 512:], desc)
        B.splash_mla_absorb_q(q, w[:, :128], packed, positions=positions, rope=rope)
        B.splash_mla_expand_out(packed_out, w[:, 128:], y)
        B.splash_mla_prefill(q, kv[..., :128], key, kv[..., 128:], indptr, indptr, out, None, ws)

    packed_out = to_bf16(bf16(rng, rows, heads, 512))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph, captured = torch.cuda.CUDAGraph(), outputs()
    with torch.cuda.stream(s):
        calls(*outputs())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        calls(*captured)
    for turn in range(4):
        for t in (q, kv, key, latent, packed_out):
            t.copy_(torch.randn(t.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        stored, eager = pool.clone(), outputs()
        pool.zero_()
        calls(*eager)
        torch.cuda.synchronize()
        assert torch.equal(stored, pool)
        for a, b in zip(captured, eager):
            assert torch.equal(a, b), turn


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("interleaved", [False, True])
def test_the_expanded_and_the_absorbed_form_agree(fmt, interleaved):
    """A step of requests with old and new tokens: their rows into the cache, the history back, both forms of the
    attention of the last 4 tokens, each against the float64 attention of what the cache holds."""
    rng = rng_of(15)
    kind, heads, chunk = FORMATS[fmt], 32, 4
    lens = np.array([4, 5, 64, 130, 257], np.int32)
    batch, total = len(lens), int(lens.sum())
    held = [-(-int(s) // PAGE) for s in lens]
    pages = sum(held) + 1
    table = table_of(rng, held, pages)
    indptr = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    pos = np.concatenate([np.arange(s) for s in lens]).astype(np.int32)
    slots = np.concatenate([table[b, np.arange(s) // PAGE] * PAGE + np.arange(s) % PAGE for b, s in enumerate(lens)]).astype(np.int32)
    rows = to_bf16(bf16(rng, total, 576))
    norm, w = to_bf16(bf16(rng, 512)), to_bf16(bf16(rng, heads, 256, 512, scale=512 ** -0.5))
    pool = torch.zeros((pages, PAGE, 656 if fmt == "latent" else 576), dtype=torch.bfloat16 if fmt == "bf16" else torch.uint8, device="cuda")
    scales = torch.ones((pages, PAGE), device="cuda") if fmt == "e4m3" else None
    desc = B.make_desc(batch, heads, table.shape[1], pages, kind, scales)
    rope = rope_of(interleaved)
    d_table, d_indptr, d_lens = dev(table), dev(indptr), dev(lens)
    B.splash_mla_append(rows[:, :512], rows[:, 512:], dev(slots), pool, scales, desc, norm_weight=norm, positions=dev(pos), rope=rope)
    q = to_bf16(bf16(rng, batch * chunk, heads, 192))
    q_pos = dev(np.concatenate([np.arange(s - chunk, s) for s in lens]).astype(np.int32))

    packed = torch.empty((batch * chunk, heads, 576), dtype=torch.bfloat16, device="cuda")
    B.splash_mla_absorb_q(q, w[:, :128], packed, positions=q_pos, rope=rope)
    latent_out = torch.empty((batch * chunk, heads, 512), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((batch * chunk, heads), device="cuda")
    ws = torch.empty(B.workspace_size(batch, chunk, heads), dtype=torch.uint8, device="cuda")
    B.splash_mla_attend(packed, pool, d_table, d_lens, chunk, latent_out, lse, desc, ws)
    absorbed = torch.empty((batch * chunk, heads, 128), dtype=torch.bfloat16, device="cuda")
    B.splash_mla_expand_out(latent_out, w[:, 128:], absorbed)

    dense = torch.empty((total, 576), dtype=torch.bfloat16, device="cuda")
    B.splash_mla_gather(pool, d_table, d_indptr, dense[:, :512], dense[:, 512:], desc)
    kv = (dense[:, :512].float() @ w.float().flatten(0, 1).T.contiguous()).bfloat16().unflatten(-1, (heads, 256))
    turned = q.clone()
    B.splash_rope(turned[..., 128:], q_pos, rope)
    expanded, lse2 = torch.empty_like(absorbed), torch.empty_like(lse)
    ws2 = torch.empty(B.mla_prefill_workspace_size(batch, batch * chunk, heads), dtype=torch.uint8, device="cuda")
    B.splash_mla_prefill(turned, kv[..., :128], dense[:, 512:], kv[..., 128:], dev(np.arange(batch + 1, dtype=np.int32) * chunk),
                         d_indptr, expanded, lse2, ws2)
    torch.cuda.synchronize()

    # float64 over what the cache holds
    f = lambda t: t.double().cpu().numpy()
    held_rows, ww, qq = f(dense), f(w), oracle.bf16_bits_to_f64(bf16_bits(q))
    qq[..., 128:] = oracle.step.rope(qq[..., 128:], q_pos.cpu().numpy()[None], FREQ, np.zeros(32, int), interleaved)
    worst = {"absorbed": 0.0, "expanded": 0.0, "lse": 0.0}
    for b in range(batch):
        c = held_rows[indptr[b]:indptr[b + 1]]
        for h in range(heads):
            keys = np.concatenate([c[:, :512] @ ww[h, :128].T, c[:, 512:]], -1)
            values = c[:, :512] @ ww[h, 128:].T
            for i in range(chunk):
                n = b * chunk + i
                see = lens[b] - chunk + i + 1
                z = keys[:see] @ qq[n, h] / np.sqrt(192.0)
                p = np.exp(z - z.max())
                want, total_w = (p / p.sum()) @ values[:see], z.max() + np.log(p.sum())
                size = (p / p.sum()) @ np.abs(values[:see]) + np.abs(want)
                for name, t in (("absorbed", absorbed), ("expanded", expanded)):
                    worst[name] = max(worst[name], float(np.max(np.abs(f(t[n, h]) - want) / size.max())))
                worst["lse"] = max(worst["lse"], abs(float(lse[n, h]) - total_w), abs(float(lse2[n, h]) - total_w))
    print(fmt, worst, flush=True)
    # Each form rounds its queries, keys or values and its output to bf16 once or twice (2^-8 each) and its weights to
    # at most 2^-8; scores of |z| <= 8 whose keys and queries are rounded are off by 2^-7 |z| at most, weights by as much
    assert worst["absorbed"] < 0.125 and worst["expanded"] < 0.125 and worst["lse"] < 0.125
