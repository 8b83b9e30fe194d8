"""splash_step_tables, splash_rope, and whole serving steps, against the float64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_37626_amd import binding as B
from tests.step_inputs import PAGE, assert_close, bf16, bf16_bits, to_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def i32(*shape):
    return torch.full(shape, 77, dtype=torch.int32, device="cuda")


# -------------------------------------------------------------- tables ---

def run_tables(lens, new, free, taken, table, pages, rows, q_chunk=1):
    b = len(lens)
    t, out = dev(table), i32(2)
    indptr, slots, positions, requests = i32(b + 1), i32(rows), i32(rows), i32(rows)
    B.splash_step_tables(dev(np.array(lens, np.int32)), q_chunk, dev(np.array(free, np.int32)),
                         dev(np.array([taken, 5], np.int32)), out, t, pages, indptr, slots, positions, requests,
                         new_lens=None if new is None else dev(np.array(new, np.int32)))
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (t, indptr, slots, positions, requests, out)]


def check_tables(lens, new, spare=5, taken=0, width=None, padding=0, short=0, seed=0, q_chunk=1, rows=None):
    rng = np.random.Generator(np.random.PCG64(seed))
    given = [q_chunk] * len(lens) if new is None else new
    s = [max(0, int(x)) for x in lens]
    n = [min(max(0, int(y)), x) for x, y in zip(s, given)]
    held = [oracle.step.pages_of(a - c) for a, c in zip(s, n)]
    need = sum(oracle.step.pages_of(a) for a in s) - sum(held)
    width = width or max([1] + [oracle.step.pages_of(a) for a in s])
    pages = sum(held) + need + spare + taken
    perm = rng.permutation(pages).astype(np.int32)
    table = np.full((len(lens), width), -7, np.int32)
    off = 0
    for b, k in enumerate(held):
        k = min(k, width)
        table[b, :k] = perm[off:off + k]
        off += k
    free = perm[off:off + taken + need - short] if short else perm[off:]
    rows = sum(n) + padding if rows is None else rows
    want = oracle.step.step_tables(lens, given, free, taken, table, pages, rows)
    got = run_tables(lens, new, free, taken, table, pages, rows, q_chunk)
    for name, a, b in zip(("table", "indptr", "slots", "positions", "requests", "taken"), got, want):
        assert np.array_equal(a, b), name


@pytest.mark.parametrize("lens,new", [
    ([5], [5]), ([64], [1]), ([65], [1]), ([0], [0]), ([1], [1]), ([128, 0, 64, 1], [128, 0, 0, 1]),
    ([63, 64, 65, 127, 128, 129], [63, 1, 2, 64, 65, 129]), ([1000] * 3, [0, 0, 0]),
])
def test_tables_small(lens, new):
    check_tables(lens, new)
    check_tables(lens, new, taken=3, padding=70)


@pytest.mark.parametrize("batch,hi,new_hi", [(256, 4096, 1), (1023, 300, 9), (1025, 300, 9), (8192, 130, 3), (40, 9000, 5000)])
def test_tables_random(batch, hi, new_hi):
    rng = np.random.Generator(np.random.PCG64(batch))
    lens = rng.integers(0, hi, batch)
    new = np.minimum(rng.integers(0, new_hi, batch, endpoint=True), lens)
    check_tables(lens, new, padding=33, taken=2, seed=batch)


def test_tables_of_a_query_chunk():
    check_tables([4, 64, 66, 2], None, q_chunk=4)   # the last request is shorter than the chunk


@pytest.mark.parametrize("short", [1, 7, 30])
def test_tables_when_the_free_list_runs_out(short):
    check_tables([500, 64, 700, 1, 800], [300, 1, 700, 1, 70], short=short, seed=3)


def test_tables_without_room_for_every_row_and_without_requests():
    check_tables([500, 200], [500, 200], rows=300)
    check_tables([500, 200], [500, 200], rows=0)
    got = run_tables([], [], [1, 2], 1, np.zeros((0, 4), np.int32), 8, 3)
    assert got[1].tolist() == [0] and got[2].tolist() == [-1] * 3 and got[5].tolist() == [1, 0]


def test_tables_clamp_what_lies_outside():
    check_tables([-3, 1000, 100], [5, 40, -2], width=4)
    check_tables([10, 100], [50, 100], taken=0)
    # taken past the list, and a table entry outside the pool
    table = np.array([[99, -7], [0, -7]], np.int32)
    got = run_tables([70, 70], [10, 70], [1, 2, 3], 10, table, 5, 80)
    want = oracle.step.step_tables([70, 70], [10, 70], [1, 2, 3], 10, table, 5, 80)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)


# ---------------------------------------------------------------- rope ---

def check_rope(x_bits, got_bits, positions, freq, axis, interleaved, scale=1.0):
    """bf16's half step 2^-8, and in fp32 the angle (2^-25 of a turn), sine and cosine, products: 2^-20 of the pair."""
    x = oracle.bf16_bits_to_f64(x_bits)
    want = oracle.step.rope(x, positions, freq, axis, interleaved, scale)
    half = x.shape[-1] // 2
    pair = np.abs(x[..., 0::2]) + np.abs(x[..., 1::2]) if interleaved else np.abs(x[..., :half]) + np.abs(x[..., half:])
    pair = np.repeat(pair, 2, -1) if interleaved else np.concatenate([pair, pair], -1)
    err = np.abs(oracle.bf16_bits_to_f64(got_bits) - want)
    assert np.all(err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * abs(scale) * pair), err.max()


@pytest.mark.parametrize("rot", [2, 6, 32, 64, 80, 128, 256])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("axes,tokens", [(1, 1), (3, 37), (4, 700)])
def test_rope(rot, interleaved, axes, tokens):
    rng = np.random.Generator(np.random.PCG64(rot))
    heads, kv_heads = 5, 2
    freq = 10000.0 ** (-np.arange(rot // 2) * 2.0 / rot)
    axis = rng.integers(0, axes, rot // 2)
    pos = rng.integers(0, 1 << 20, (axes, tokens)).astype(np.int32)
    pos[:, 0] = 0 if tokens > 1 else (1 << 31) - 1
    q, k = bf16(rng, tokens, heads, rot), bf16(rng, tokens, kv_heads, rot)
    rope = B.make_rope(rot, freq, pair_axis=axis, num_axes=axes, interleaved=interleaved)
    out, out2 = torch.empty_like(to_bf16(q)), torch.empty_like(to_bf16(k))
    B.splash_rope(to_bf16(q), dev(pos), rope, out=out, x2=to_bf16(k), out2=out2)
    check_rope(q, bf16_bits(out), pos, freq, axis, interleaved)
    check_rope(k, bf16_bits(out2), pos, freq, axis, interleaved)
    both, both2 = to_bf16(q), to_bf16(k)   # in place
    B.splash_rope(both, dev(pos), rope, x2=both2)
    assert torch.equal(both, out) and torch.equal(both2, out2)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("head,offset,rot", [(576, 512, 64), (128, 0, 64), (67, 3, 64), (129, 1, 128), (100, 20, 80)])
def test_rope_views_leave_the_rest_of_a_row(interleaved, head, offset, rot):
    rng = np.random.Generator(np.random.PCG64(head))
    rows = to_bf16(bf16(rng, 19, 6, head))
    before = rows.clone()
    freq, axis = 0.9 ** np.arange(rot // 2), np.zeros(rot // 2, int)
    pos = rng.integers(0, 5000, (1, 19)).astype(np.int32)
    rope = B.make_rope(rot, freq, interleaved=interleaved, scale=1.25)
    view = rows[:, 1:5, offset:offset + rot]
    B.splash_rope(view, dev(pos[0]), rope)
    check_rope(bf16_bits(before[:, 1:5, offset:offset + rot]), bf16_bits(view), pos, freq, axis, interleaved, 1.25)
    rows[:, 1:5, offset:offset + rot] = before[:, 1:5, offset:offset + rot]
    assert torch.equal(rows, before)
    # heads outside tokens: [heads, tokens, rot] memory
    turned = before[:, 1:5, offset:offset + rot].transpose(0, 1).contiguous().transpose(0, 1)
    B.splash_rope(turned, dev(pos[0]), rope)
    check_rope(bf16_bits(before[:, 1:5, offset:offset + rot]), bf16_bits(turned), pos, freq, axis, interleaved, 1.25)


def test_rope_of_text_positions_on_every_axis():
    rng = np.random.Generator(np.random.PCG64(41))
    x = bf16(rng, 50, 3, 64)
    freq, axis = 0.8 ** np.arange(32), np.arange(32) % 3
    pos = rng.integers(0, 9000, 50).astype(np.int32)
    out = to_bf16(x)
    B.splash_rope(out, dev(pos).expand(3, -1), B.make_rope(64, freq, pair_axis=axis))
    check_rope(x, bf16_bits(out), np.broadcast_to(pos, (3, 50)), freq, axis, False)


def test_rope_refuses_other_shapes():
    x, rope = torch.zeros((3, 2, 8), dtype=torch.bfloat16, device="cuda"), B.make_rope(8, [1.0] * 4)
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    for args in ((x[:, :, :6], pos), (x.float(), pos), (x[:2], pos), (x, pos.long()), (x.cpu(), pos),
                 (x, torch.zeros((2, 3), dtype=torch.int32, device="cuda")), (x.transpose(1, 2).contiguous().transpose(1, 2), pos)):
        with pytest.raises(B.SplashError):
            B.splash_rope(*args, rope)


# --------------------------------------------------------- whole steps ---

@pytest.mark.parametrize("int8", [False, True], ids=["e4m3", "int8"])
@pytest.mark.parametrize("captured", [False, True], ids=["eager", "captured"])
def test_serving_steps(int8, captured):
    """A prompt step and decode steps: tables, rope on queries and keys, append, attend; the oracle goes the same way."""
    S = oracle.step
    rng = np.random.Generator(np.random.PCG64(30))
    batch, hk, g, d, width, q_chunk = 5, 2, 4, 64, 6, 2
    pages = batch * width
    freq = 10000.0 ** (-np.arange(d // 2) * 2.0 / d)
    axis = np.array([0] * 8 + [1] * 12 + [2] * 12)
    rope = B.make_rope(d, freq, pair_axis=axis)
    code = B.GQA_INT8 if int8 else B.GQA_E4M3
    desc = B.make_gqa_desc(batch, hk * g, hk, d, width, pages, code)
    free = rng.permutation(pages).astype(np.int32)
    kind = torch.int8 if int8 else torch.uint8
    cache = [torch.full((pages, hk, PAGE, d), 0x7F, dtype=kind, device="cuda") for _ in range(2)]
    scales = [torch.full((pages, hk), float("nan"), dtype=torch.float32, device="cuda") for _ in range(2)]
    host = [(np.full((pages, hk, PAGE, d), 0x7F, np.int8 if int8 else np.uint8), np.full((pages, hk), np.nan, np.float32))
            for _ in range(2)]
    table, free_d = torch.full((batch, width), -1, dtype=torch.int32, device="cuda"), dev(free)
    host_table = np.full((batch, width), -1, np.int32)
    taken, taken_out = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.gqa_workspace_size(desc, q_chunk), dtype=torch.uint8, device="cuda")
    lens = np.array([70, 1, 64, 200, 130])

    def prompt():
        seq, rows = dev(lens.astype(np.int32)), int(lens.sum()) + 9
        indptr, slots, pos, req = i32(batch + 1), i32(rows), i32(rows), i32(rows)
        B.splash_step_tables(seq, 0, free_d, taken, taken_out, table, pages, indptr, slots, pos, req, new_lens=seq)
        want = S.step_tables(lens, lens, free, 0, host_table, pages, rows)
        for a, b in zip((table, indptr, slots, pos, req, taken_out), want):
            assert np.array_equal(a.cpu().numpy(), b)
        kv = to_bf16(bf16(rng, rows, 2 * hk, d))
        turned = torch.empty((rows, hk, d), dtype=torch.bfloat16, device="cuda")
        kv2 = torch.empty_like(kv)
        B.splash_rope(kv[:, :hk], pos.repeat(3, 1), rope, out=turned)
        kv2[:, :hk], kv2[:, hk:] = turned, kv[:, hk:]
        B.splash_gqa_append(kv2[:, :hk], kv2[:, hk:], slots, cache[0], cache[1], scales[0], scales[1], desc)
        for i in range(2):
            host[i] = S.gqa_append(bf16_bits(kv2[:, hk * i:hk * (i + 1)]), want[2], *host[i], int8)
            assert np.array_equal(cache[i].cpu().numpy(), host[i][0])
            assert np.array_equal(scales[i].cpu().numpy(), host[i][1], equal_nan=True)
        host_table[:] = want[0]

    prompt()
    rows = batch * q_chunk
    seq = dev(lens.astype(np.int32))
    indptr, slots, pos, req = i32(batch + 1), i32(rows), i32(rows), i32(rows)
    pos3 = torch.zeros((3, rows), dtype=torch.int32, device="cuda")
    qkv = torch.zeros((rows, hk * g + 2 * hk, d), dtype=torch.bfloat16, device="cuda")
    q = torch.empty((rows, hk * g, d), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((rows, hk * g), dtype=torch.float32, device="cuda")
    k_rows, v_rows = qkv[:, hk * g:hk * g + hk], qkv[:, hk * g + hk:]

    def step():
        B.splash_step_tables(seq, q_chunk, free_d, taken, taken_out, table, pages, indptr, slots, pos, req)
        pos3.copy_(pos.expand(3, -1))
        B.splash_rope(qkv[:, :hk * g], pos3, rope, out=q, x2=k_rows)
        B.splash_gqa_append(k_rows, v_rows, slots, cache[0], cache[1], scales[0], scales[1], desc)
        B.splash_gqa_attend(q, cache[0], cache[1], scales[0], scales[1], table, seq, q_chunk, out, lse, desc, ws)
        taken.copy_(taken_out)

    taken.copy_(taken_out)
    state = [x.clone() for x in (table, taken, *cache, *scales)]
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        torch.cuda.synchronize()
        for x, was in zip((table, taken, *cache, *scales), state):
            x.copy_(was)
    at = int(sum(S.pages_of(s) for s in lens))
    for turn in range(6):
        lens = lens + q_chunk
        seq.copy_(dev(lens.astype(np.int32)))
        fresh = bf16(rng, rows, hk * g + 2 * hk, d, scale=2.0 ** (turn - 2))
        qkv.copy_(to_bf16(fresh))
        torch.cuda.synchronize()
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        want = S.step_tables(lens, [q_chunk] * batch, free, at, host_table, pages, rows)
        for a, b in zip((table, indptr, slots, pos, req, taken_out), want):
            assert np.array_equal(a.cpu().numpy(), b), turn
        host_table[:], at = want[0], int(want[5][0])
        p3 = np.broadcast_to(want[3], (3, rows))
        check_rope(fresh[:, :hk * g], bf16_bits(q), p3, freq, axis, False)
        check_rope(fresh[:, hk * g:hk * g + hk], bf16_bits(k_rows), p3, freq, axis, False)
        for i, x in enumerate((k_rows, v_rows)):
            host[i] = S.gqa_append(bf16_bits(x), want[2], *host[i], int8)
            assert np.array_equal(cache[i].cpu().numpy(), host[i][0]), turn
            assert np.array_equal(scales[i].cpu().numpy(), host[i][1], equal_nan=True), turn
        ref = S.gqa_attend(bf16_bits(q), host[0][0], host[1][0], host[0][1], host[1][1], host_table, lens, q_chunk,
                           np.float32(d ** -0.5), int8)
        assert_close(out, lse, ref, int(lens.max()), d, f"step {turn}")


def test_tables_and_rope_before_the_latent_attention():
    """The same tables and the rotary part of packed rows in front of splash_mla_attend."""
    rng = np.random.Generator(np.random.PCG64(31))
    batch, heads, pages, width = 3, 16, 12, 4
    lens = np.array([100, 1, 65], np.int32)
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    taken, taken_out = torch.zeros(2, dtype=torch.int32, device="cuda"), i32(2)
    rows = int(lens.sum())
    indptr, slots, pos, req = i32(batch + 1), i32(rows), i32(rows), i32(rows)
    seq = dev(lens)
    B.splash_step_tables(seq, 0, dev(rng.permutation(pages).astype(np.int32)), taken, taken_out, table, pages, indptr, slots,
                         pos, req, new_lens=seq)
    freq = 10000.0 ** (-np.arange(32) / 32.0)
    rope = B.make_rope(64, freq, interleaved=True)
    latent = to_bf16(bf16(rng, rows, 1, 576))
    B.splash_rope(latent[..., 512:], pos, rope)
    pool = torch.zeros((pages * 64, 576), dtype=torch.bfloat16, device="cuda")
    pool[slots.long()] = latent[:, 0]
    q = to_bf16(bf16(rng, batch, heads, 576))
    B.splash_rope(q[..., 512:], (seq - 1).int(), rope)
    out = torch.empty((batch, heads, 512), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((batch, heads), dtype=torch.float32, device="cuda")
    desc = B.make_desc(batch, heads, width, pages)
    ws = torch.empty(B.workspace_size(batch, 1, heads), dtype=torch.uint8, device="cuda")
    B.splash_mla_attend(q, pool, table, seq, 1, out, lse, desc, ws)
    torch.cuda.synchronize()
    history = oracle.bf16_bits_to_f64(bf16_bits(latent[:, 0]))
    at = indptr.cpu().numpy()
    for b in range(batch):
        keys = history[at[b]:at[b + 1]]
        z = oracle.bf16_bits_to_f64(bf16_bits(q[b])) @ keys.T * desc.softmax_scale
        w = np.exp(z - z.max(-1, keepdims=True))
        want = (w / w.sum(-1, keepdims=True)) @ keys[:, :512]
        assert np.abs(out[b].float().cpu().numpy() - want).max() <= 1e-2   # the latent attention's bar
