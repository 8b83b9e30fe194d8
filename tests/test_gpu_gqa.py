"""splash_gqa_attend and splash_gqa_append against the float64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_37626_amd import binding as B
from tests.step_inputs import PAGE, Attend, assert_close, bf16, blocks, to_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def check(p, label=""):
    out, lse = p.attend()
    assert_close(out, lse, p.oracle(), max(1, int(max(p.lens))), p.dim, label)
    return out, lse


EDGES = [0, 1, 63, 64, 65, 129, 700, 5]


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kv_heads,group,q_chunk", [(2, 1, 1), (1, 8, 1), (2, 16, 1), (3, 5, 3), (1, 4, 8), (2, 40, 1),
                                                    (1, 9, 8), (1, 33, 4)])
def test_attend_edge_lengths(int8, dim, kv_heads, group, q_chunk):
    p = Attend(EDGES, kv_heads, group, dim, q_chunk, int8, seed=dim + group)
    check(p.poison(), f"d{dim} hk{kv_heads} g{group} q{q_chunk}")


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
@pytest.mark.parametrize("dim,group,q_chunk", [(64, 4, 1), (128, 8, 1), (128, 8, 4), (128, 16, 4), (256, 2, 8), (256, 8, 4)])
def test_attend_long_and_ragged(int8, dim, group, q_chunk):
    check(Attend([20000, 17, 4097, 9000, 640], 1, group, dim, q_chunk, int8, seed=7).poison(), f"d{dim} g{group} q{q_chunk}")


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
@pytest.mark.parametrize("dim,kv_heads,group,q_chunk", [(64, 2, 4, 1), (128, 3, 2, 4), (128, 1, 16, 8), (256, 2, 16, 4)])
def test_attend_edges_beside_a_long_history(int8, dim, kv_heads, group, q_chunk):
    # (a table row past 16 pages: tiles are cut, short and empty ones among them)
    check(Attend([0, 1, 1100, 63, 0, 64, 65, 2, 0], kv_heads, group, dim, q_chunk, int8, seed=28).poison())


@pytest.mark.parametrize("dim,q_chunk,lens", [(128, 150, [150, 400, 149, 90]), (256, 70, [70, 1300]), (64, 200, [1500, 3])])
def test_attend_long_chunks(dim, q_chunk, lens):
    # a prompt's rows: several row blocks, most pages seen in part
    check(Attend(lens, 1, 2, dim, q_chunk, False, seed=29).poison(), f"d{dim} q{q_chunk}")


@pytest.mark.parametrize("dim,kv_heads,group", [(64, 1, 4), (256, 1, 2)])
def test_attend_one_history_over_the_whole_chip(dim, kv_heads, group):
    # (more parts of a tile than a wave of the join has lanes)
    check(Attend([120000], kv_heads, group, dim, 1, False, seed=31).poison())


@pytest.mark.parametrize("kv_heads,group,dim,q_chunk", [(1, 1024, 128, 1), (128, 8, 64, 1), (128, 1, 256, 2), (2, 300, 64, 2)])
def test_attend_most_heads(kv_heads, group, dim, q_chunk):
    check(Attend([130, 0, 1300], kv_heads, group, dim, q_chunk, False, seed=32).poison())


def test_attend_many_requests():
    rng = np.random.Generator(np.random.PCG64(5))
    check(Attend(rng.integers(0, 200, 700), 2, 4, 64, 1, False, seed=8).poison())


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
def test_attend_scales_far_apart_and_sharp_scores(int8):
    # block scales over forty powers of two: the largest V block decides, in
    # fp32, whatever the weights; large queries make one key win
    check(Attend([1000, 300], 2, 4, 128, 2, int8, seed=9, exponents=(-30, 10), q_scale=2.0 ** -8))
    check(Attend([1000, 300], 2, 4, 128, 2, int8, seed=10, q_scale=30.0))


@pytest.mark.parametrize("softmax_scale", [2.0 ** -60, 2.0 ** 60])
@pytest.mark.parametrize("lens", [[70, 200, 3], [70, 2000, 3]], ids=["whole", "split"])
def test_attend_scales_at_the_ends_of_fp32(lens, softmax_scale):
    # the scale of a block of zeros, and one whose product with softmax_scale is
    # past fp32; all keys are zeros, so every weight is the same
    p = Attend(lens, 1, 4, 128, 2, False, seed=30)
    p.k[:] = 0
    p.ks[:] = 2.0 ** -126 if softmax_scale < 1 else 2.0 ** 120
    p.scale = np.float32(softmax_scale)
    desc = p.desc
    p.desc = lambda: B.make_gqa_desc(len(lens), 4, 1, 128, p.table.shape[1], p.k.shape[0], softmax_scale=softmax_scale)
    assert bytes(desc())[:32] == bytes(p.desc())[:32]
    check(p)


def test_attend_nan_codes_stay_with_the_rows_that_see_them():
    # the last chunk token's V holds a NaN: earlier rows of the chunk are whole
    p = Attend([200, 64, 130], 1, 4, 128, 4, False, seed=11)
    ref = Attend([200, 64, 130], 1, 4, 128, 4, False, seed=11).oracle()
    for b, s in enumerate(p.lens):
        p.v[p.table[b, (s - 1) // PAGE], 0, (s - 1) % PAGE, 5] = 0x7F
        p.k[p.table[b, (s - 2) // PAGE], 0, (s - 2) % PAGE, 9] = 0xFF
    out, lse = p.attend()
    o = out.float().cpu().numpy()
    for b in range(3):
        rows = o[4 * b:4 * b + 2]      # see neither token
        np.testing.assert_allclose(rows, ref[0][4 * b:4 * b + 2], atol=2e-2)
        assert np.isnan(o[4 * b + 2:4 * b + 4]).all()  # a NaN key: every weight
        p.k[p.table[b, (p.lens[b] - 2) // PAGE], 0, (p.lens[b] - 2) % PAGE, 9] = 0
    out, lse = p.attend()
    o = out.float().cpu().numpy()
    nan = np.isnan(o)
    want = np.zeros_like(nan)
    want[3::4, :, 5] = True            # the last row of each chunk, dim 5
    assert np.array_equal(nan, want) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("lens", [[200, 64, 130], [9000, 64, 130]], ids=["whole", "split"])
def test_attend_nan_and_infinite_queries_stay_in_their_rows(lens):
    p = Attend(lens, 2, 4, 64, 2, False, seed=11)
    ref = p.oracle()
    p.q[1, 3, 7] = 0x7FC0
    p.q[4, 6, 0] = 0x7F80
    out, lse = p.attend()
    o, l = out.float().cpu().numpy(), lse.cpu().numpy()
    for row, head in ((1, 3), (4, 6)):
        assert np.isnan(o[row, head]).all() and np.isnan(l[row, head])
        o[row, head], l[row, head] = ref[0][row, head], ref[1][row, head]
    np.testing.assert_allclose(o, ref[0], atol=2e-2)
    np.testing.assert_allclose(l, ref[1], atol=1e-4)


def test_attend_calls_side_by_side_on_two_streams():
    ps = [Attend([5000, 70], 2, 8, 128, 1, False, seed=26), Attend([3000, 1, 900], 1, 16, 64, 2, True, seed=27)]
    want = [p.attend() for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    state = [(p.device(), p.workspace(), p.outputs()) for p in ps]
    torch.cuda.synchronize()
    for _ in range(5):
        for p, s, (t, ws, (out, lse)) in zip(ps, streams, state):
            B.splash_gqa_attend(t["q"], t["k_pages"], t["v_pages"], t["k_scales"], t["v_scales"], t["block_table"],
                                t["seq_lens"], p.q_chunk, out, lse, p.desc(), ws, stream=s)
    torch.cuda.synchronize()
    for (a, la), (_, _, (b, lb)) in zip(want, state):
        assert torch.equal(a, b) and torch.equal(la, lb)


def test_attend_skips_pages_outside_the_pool():
    p = Attend([300, 500, 60], 2, 4, 64, 2, True, seed=12)
    p.table[0, 1], p.table[1, 7], p.table[2, 0] = -1, p.k.shape[0], 1 << 30
    check(p)
    p.lens = np.array([10 ** 9, -5, 60], dtype=np.int32)  # past the table row, negative
    check(p)
    # the places of skipped pages read nothing of the pool's first page either
    p = Attend([300, 500, 60], 2, 4, 64, 2, False, seed=12)
    p.table[p.table == 0] = -1
    p.table[0, 2] = -1
    p.poison()
    p.ks[0] = p.vs[0] = np.nan
    p.k[0] = p.v[0] = 0xFF
    check(p)


def test_attend_is_deterministic_and_independent_of_placement():
    p = Attend([3000, 70, 1], 2, 8, 128, 1, False, seed=13)
    a, la = p.attend()
    b, lb = p.attend()
    assert torch.equal(a, b) and torch.equal(la, lb)
    perm = np.random.Generator(np.random.PCG64(14)).permutation(p.k.shape[0])
    inverse = np.argsort(perm)
    p.k, p.v, p.ks, p.vs = p.k[perm], p.v[perm], p.ks[perm], p.vs[perm]
    p.table = np.where(p.table >= 0, inverse[np.maximum(p.table, 0)], -1).astype(np.int32)
    c, lc = p.attend()
    assert torch.equal(a, c) and torch.equal(la, lc)


def test_attend_pool_past_4_gib():
    # blocks of a 2^32-byte pool, only its last pages in use
    p = Attend([150, 90], 8, 4, 128, 1, False, seed=15, extra_pages=0)
    pages, far = p.k.shape[0], (1 << 32) // (8 * PAGE * 128) + 9
    t = p.device()
    big = {}
    for side in "kv":
        big[side] = torch.zeros((far, 8, PAGE, 128), dtype=torch.uint8, device="cuda")
        big[side][far - pages:] = t[side + "_pages"]
        big[side + "s"] = torch.ones((far, 8), dtype=torch.float32, device="cuda")
        big[side + "s"][far - pages:] = t[side + "_scales"]
    table = torch.where(t["block_table"] >= 0, t["block_table"] + (far - pages), -1).int()
    desc = B.make_gqa_desc(2, 32, 8, 128, p.table.shape[1], far)
    out, lse = p.outputs()
    B.splash_gqa_attend(t["q"], big["k"], big["v"], big["ks"], big["vs"], table, t["seq_lens"], 1, out, lse, desc,
                        p.workspace())
    assert_close(out, lse, p.oracle(), 150, 128)
    # and the append writes there
    rng = np.random.Generator(np.random.PCG64(16))
    x = bf16(rng, 2, 8, 128)
    slots = np.array([(far - 1) * PAGE + 3, (far - 2) * PAGE + 1], dtype=np.int32)
    want_c, want_s = oracle.step.gqa_append(x, slots - (far - pages) * PAGE, p.k, p.ks, False)
    B.splash_gqa_append(to_bf16(x), to_bf16(x), torch.from_numpy(slots).cuda(), big["k"], big["v"], big["ks"], big["vs"], desc)
    assert np.array_equal(big["k"][far - pages:].cpu().numpy(), want_c)
    assert np.array_equal(big["ks"][far - pages:].cpu().numpy(), want_s)
    assert int(big["k"][:far - pages].count_nonzero()) == 0


def test_attend_without_lse_on_another_stream_and_idle():
    p = Attend([100, 5], 1, 4, 64, 1, False, seed=17)
    want, _ = p.attend()
    t, ws = p.device(), p.workspace()
    out, _ = p.outputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.splash_gqa_attend(t["q"], t["k_pages"], t["v_pages"], t["k_scales"], t["v_scales"], t["block_table"], t["seq_lens"], 1,
                        out, None, p.desc(), ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    idle = B.make_gqa_desc(0, 4, 1, 64, 2, p.k.shape[0])
    B.splash_gqa_attend(t["q"][:0], t["k_pages"], t["v_pages"], t["k_scales"], t["v_scales"], t["block_table"][:0, :2],
                        t["seq_lens"][:0], 1, out[:0], None, idle, ws)


def test_attend_replays_in_a_graph():
    p = Attend([3000, 64, 700, 1], 2, 8, 128, 2, False, seed=18)
    t, ws, desc = p.device(), p.workspace(), p.desc()
    out, lse = p.outputs()

    def call():
        B.splash_gqa_attend(t["q"], t["k_pages"], t["v_pages"], t["k_scales"], t["v_scales"], t["block_table"],
                            t["seq_lens"], 2, out, lse, desc, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for lens in ([3000, 64, 700, 1], [2, 64, 100, 0], [2999, 1, 699, 64]):
        p.lens = np.array(lens, dtype=np.int32)
        t["seq_lens"].copy_(torch.from_numpy(p.lens))
        t["q"].copy_(t["q"] * 0.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        a, la = out.clone(), lse.clone()
        out.fill_(3), lse.fill_(3)
        call()
        torch.cuda.synchronize()
        assert torch.equal(a, out) and torch.equal(la, lse), lens
    p.q = (t["q"].view(torch.int16).cpu().numpy()).view(np.uint16)
    assert_close(out, lse, p.oracle(), 3000, 128)


# -------------------------------------------------------------- append ---

def run_append(k, v, slots, cache, scales, int8, heads, dim, strided=False, batch=1):
    pages = cache[0].shape[0]
    desc = B.make_gqa_desc(batch, heads, heads, dim, 1, pages, B.GQA_INT8 if int8 else B.GQA_E4M3)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    kt, vt = to_bf16(k), to_bf16(v)
    if strided:  # keys and values side by side in one row, behind the queries
        row = torch.zeros((k.shape[0], 3 * heads, dim), dtype=torch.bfloat16, device="cuda")
        row[:, heads:2 * heads], row[:, 2 * heads:] = kt, vt
        kt, vt = row[:, heads:2 * heads], row[:, 2 * heads:]
    c, s = [dev(x) for x in cache], [dev(x) for x in scales]
    B.splash_gqa_append(kt, vt, dev(np.array(slots, dtype=np.int32)), c[0], c[1], s[0], s[1], desc)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in c], [x.cpu().numpy() for x in s]


def check_append(k, v, slots, int8, heads, dim, seed, pages=12, exponents=(-9, -5), strided=False):
    rng = np.random.Generator(np.random.PCG64(seed))
    cache, scales = zip(*[blocks(rng, pages, heads, dim, int8, exponents) for _ in range(2)])
    want = [oracle.step.gqa_append(x, slots, c, s, int8) for x, c, s in zip((k, v), cache, scales)]
    for batch in (1, 1000):   # laid out for prompts (from 8 rows on), and for decode steps
        got_c, got_s = run_append(k, v, slots, cache, scales, int8, heads, dim, strided, batch)
        for (want_c, want_s), gc, gs in zip(want, got_c, got_s):
            assert np.array_equal(gs, want_s)
            nan = (want_c & 0x7F) == 0x7F if not int8 else np.zeros(want_c.shape, bool)
            assert np.array_equal(gc[~nan], want_c[~nan]) and np.all((gc[nan] & 0x7F) == 0x7F)


SLOTS = {
    "one": [64 * 3 + 17],
    "starts": [64 * 3],
    "decode": [64 * p + r for p, r in [(2, 0), (9, 63), (4, 31), (0, 1), (11, 62)]],
    "prompt": list(range(64 * 5 + 40, 64 * 6)) + list(range(64 * 2, 64 * 3)) + list(range(64 * 7, 64 * 7 + 33)),
    "skips": [-1, 64 * 1 + 5, -1, 64 * 12, 64 * 4 + 1, 64 * 4 + 3, -(1 << 31), 2 ** 31 - 1],
    "backwards": [64 * 3 + r for r in (9, 4, 63, 2)],
    "page": list(range(64 * 8, 64 * 9)),
    # short and long runs in one stretch of the list, over its 32- and 64-row ends
    "mixed": sum(([64 * p + r for r in range(at, at + n)] for p, at, n in
                  [(0, 5, 1), (1, 0, 8), (2, 55, 9), (3, 63, 1), (4, 0, 2), (5, 10, 40), (6, 1, 1), (7, 2, 7), (8, 0, 1), (9, 20, 3)]),
                 []) + [64 * 10 + r for r in (7, 3, 30, 1, 2, 9, 8, 40, 50, 49)] + [64 * 11 + 62, 64 * 11 + 60],
}


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
@pytest.mark.parametrize("heads,dim", [(1, 64), (3, 128), (2, 256)])
@pytest.mark.parametrize("name", sorted(SLOTS))
def test_append(int8, heads, dim, name):
    rng = np.random.Generator(np.random.PCG64(20))
    n = len(SLOTS[name])
    for scale in (1.0, 2.0 ** -6, 30.0):
        check_append(bf16(rng, n, heads, dim, scale=scale), bf16(rng, n, heads, dim, scale=scale), SLOTS[name], int8, heads,
                     dim, seed=21, strided=scale == 1.0)


@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
def test_append_special_values(int8):
    # zeros, subnormals, the largest magnitudes, borders of a power of two,
    # infinities and NaN, ties
    top = np.array([0x0000, 0x8000, 0x0001, 0x007F, 0x7F7F, 0xFF7F, 0x7F80, 0xFF80, 0x7FC0, 0x3F80, 0x43E0, 0x43E1, 0x42FE,
                    0x42FF, 0x4300, 0x3F00, 0x3FC0, 0x4020, 0x3B00], dtype=np.uint16)
    rng = np.random.Generator(np.random.PCG64(22))
    for row in range(len(top)):
        x = np.zeros((2, 1, 64), dtype=np.uint16)
        x[0, 0, :] = top[row]
        x[1, 0, :] = rng.permutation(np.resize(top[:row + 1], 64))
        for slots in ([64 * 2 + 7, 64 * 2 + 8], [64 * 3, 64 * 3 + 1]):
            check_append(x, x[::-1].copy(), slots, int8, 1, 64, seed=23, pages=5)
            check_append(x, x[::-1].copy(), slots, int8, 1, 64, seed=23, pages=5, exponents=(-126, -120))


def test_append_a_history_token_by_token():
    # the growing block, read back after every page
    rng = np.random.Generator(np.random.PCG64(24))
    cache, scales = zip(*[blocks(rng, 3, 2, 64, False) for _ in range(2)])
    want = [(c, s) for c, s in zip(cache, scales)]
    x = bf16(rng, 130, 2, 64)
    grow = np.repeat(np.arange(-65, 65), 1)
    bits = np.clip((x & 0x7F80).astype(np.int32) + ((grow // 16)[:, None, None] << 7), 0x80, 0x7E00) | (x & 0x807F)
    x = bits.astype(np.uint16)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    c, s = [dev(a) for a in cache], [dev(a) for a in scales]
    desc = B.make_gqa_desc(1, 2, 2, 64, 3, 3)
    for t in range(130):
        B.splash_gqa_append(to_bf16(x[t:t + 1]), to_bf16(x[t:t + 1]), dev(np.array([t], np.int32)), c[0], c[1], s[0], s[1], desc)
        want = [oracle.step.gqa_append(x[t:t + 1], [t], wc, ws, False) for wc, ws in want]
    for i in range(2):
        assert np.array_equal(s[i].cpu().numpy(), want[i][1])
        assert np.array_equal(c[i].cpu().numpy(), want[i][0])


def test_binding_refuses_tensors_that_the_kernels_do_not_take():
    p = Attend([100, 5], 2, 4, 64, 1, False, seed=25)
    t, ws, desc = p.device(), p.workspace(), p.desc()
    out, lse = p.outputs()

    def call(**kw):
        a = {**t, "out": out, "lse": lse, "workspace": ws, **kw}
        B.splash_gqa_attend(a["q"], a["k_pages"], a["v_pages"], a["k_scales"], a["v_scales"], a["block_table"], a["seq_lens"],
                            1, a["out"], a["lse"], desc, a["workspace"])

    for kw in (dict(q=t["q"].float()), dict(q=t["q"][:1]), dict(k_pages=t["k_pages"][1:]), dict(v_pages=t["v_pages"].view(torch.int8)),
               dict(k_scales=t["k_scales"].T.contiguous().T), dict(seq_lens=t["seq_lens"].long()),
               dict(block_table=t["block_table"][:, :1]), dict(out=out.transpose(1, 2).contiguous().transpose(1, 2)),
               dict(lse=lse.cpu()), dict(workspace=ws[:16])):
        with pytest.raises(B.SplashError):
            call(**kw)
    x = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache = (t["k_pages"], t["v_pages"], t["k_scales"], t["v_scales"])
    for k, s in ((x.float(), slots), (x[:, :1], slots), (x, slots.long()), (x, torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(B.SplashError):
            B.splash_gqa_append(k, k, s, *cache, desc)
