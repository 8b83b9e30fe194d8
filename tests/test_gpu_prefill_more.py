"""splash_mla_prefill where there are more tiles than workgroups, over the widest strides, and beside itself; the
projections and the gather over the same strides."""
import numpy as np
import pytest
import torch

from paper_2609_37626_amd import binding as B
from tests.layer_inputs import PAGE, Prompts, assert_prefill, bf16, dev, rng_of, rope_of, to_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def some_heads(p, heads, label):
    """The call over all heads, some of them against the oracle."""
    out, lse = p.run()
    p.q, p.kv, p.heads = p.q[:, heads], p.kv[:, heads], len(heads)
    assert_prefill(out[:, heads], lse[:, heads], p.oracle(), int(p.keys.max()), label)


def test_more_tiles_than_workgroups_in_the_requests_order():
    rng = rng_of(31)
    p = Prompts(rng.integers(0, 4, 400), rng.integers(0, 30, 400), 4, seed=32)
    some_heads(p, [0, 1, 2, 3], "400 short prompts")
    some_heads(Prompts(rng.integers(0, 4, 400), rng.integers(0, 30, 400), 20, seed=39), [0, 19], "400 short prompts, 20 heads")
    p = Prompts([700, 0, 300] + [1] * 270, [0, 5, 900] + [3] * 270, 40, seed=33)
    some_heads(p, [0, 39], "two long prompts before 270 tokens")


@pytest.mark.parametrize("new,old,heads", [([130] * 9, [0, 7, 64, 100, 31, 500, 1, 2, 3], 40), ([390, 20, 650], [0, 0, 0], 64),
                                           ([500, 420, 610], [0, 30, 0], 64), ([18] * 34, [0] * 34, 32),
                                           ([515, 510], [3000, 2950], 56), ([300, 700], [4100, 3300], 56)])
def test_more_tiles_than_workgroups(new, old, heads):
    """Both tile widths, last tiles that are not full, groups that are not."""
    some_heads(Prompts(new, old, heads, seed=sum(new)), [0, heads - 1], f"{new} over {old}, {heads} heads")


def test_no_request_has_rows():
    """Room for more tiles than workgroups, and none of them: nothing is written."""
    rows, heads = 2000, 64
    q, kv, key = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((rows, heads, 192), (900, heads, 256), (900, 64)))
    out, lse = torch.full((rows, heads, 128), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((rows, heads), 7.0, device="cuda")
    ws = torch.empty(B.mla_prefill_workspace_size(2, rows, heads), dtype=torch.uint8, device="cuda")
    for at in ([5, 5, 5], [0, 0, 0], [2000, 2000, 2000]):
        B.splash_mla_prefill(q, kv[..., :128], key, kv[..., 128:], dev(np.array(at, np.int32)), dev(np.array([0, 400, 900], np.int32)),
                             out, lse, ws)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all()) and bool((lse == 7.0).all())


def inputs(rng, rows, heads):
    return (to_bf16(bf16(rng, rows, heads, 192)), to_bf16(bf16(rng, rows, heads, 256)), to_bf16(bf16(rng, rows, 64)),
            torch.empty((rows, heads, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, heads), device="cuda"))


def attend(x, at, ws, stream=None):
    q, kv, key, out, lse = x
    B.splash_mla_prefill(q, kv[..., :128], key, kv[..., 128:], at, at, out, lse, ws, stream=stream)


def test_two_graphs_share_a_workspace_and_take_other_lengths():
    """Whole tiles in one, cut ones in the other, by turns, with lengths that change between the replays."""
    rng = rng_of(34)
    many, few = inputs(rng, 1500, 70), inputs(rng, 1600, 2)
    at_many, at_few = dev(np.array([0, 700, 1500], np.int32)), dev(np.array([0, 1500, 1600], np.int32))
    ws = torch.empty(B.mla_prefill_workspace_size(2, 1600, 70), dtype=torch.uint8, device="cuda")
    attend(many, at_many, ws)
    attend(few, at_few, ws)
    torch.cuda.synchronize()
    graphs = []
    for x, at in ((many, at_many), (few, at_few)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            attend(x, at, ws)
    own = torch.empty_like(ws)
    for a, b in ((700, 1500), (1, 1600), (1499, 10), (1500, 800)):
        at_many.copy_(dev(np.array([0, a, 1500], np.int32)))
        at_few.copy_(dev(np.array([0, b, 1600], np.int32)))
        for x in (many, few):
            x[0].copy_(torch.randn(x[0].shape, device="cuda"))
            x[3].fill_(7.0)
        graphs[0].replay()
        graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        for x, at in ((many, at_many), (few, at_few)):
            out, lse = x[3].clone(), x[4].clone()
            attend(x, at, own)
            torch.cuda.synchronize()
            assert torch.equal(out, x[3]) and torch.equal(lse, x[4]), (a, b)


def test_two_calls_at_once():
    rng = rng_of(35)
    x = [inputs(rng, 1500, 70), inputs(rng, 1600, 2)]
    at = [dev(np.array([0, 700, 1500], np.int32)), dev(np.array([0, 1500, 1600], np.int32))]
    ws = [torch.empty(B.mla_prefill_workspace_size(2, 1600, 70), dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = []
    for i in range(2):
        attend(x[i], at[i], ws[i])
        torch.cuda.synchronize()
        want.append((x[i][3].clone(), x[i][4].clone()))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for i in range(2):
            attend(x[i], at[i], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(x[i][3], want[i][0]) and torch.equal(x[i][4], want[i][1])


def test_offsets_past_32_bits():
    """Rows 2^24 elements apart, as many as take offsets past 2^31 and 2^32 elements."""
    rows, heads, stride = 290, 2, 1 << 24
    rng = rng_of(36)
    big = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda")   # 9.7 GB
    wide = lambda first, shape: torch.as_strided(big, (rows, *shape), (stride, *([shape[1], 1] if len(shape) == 2 else [1])), first)
    q, kv, key, y = wide(0, (heads, 192)), wide(1024, (heads, 256)), wide(2048, (64,)), wide(4096, (heads, 128))
    p = Prompts([rows], [0], heads, seed=37)
    q.copy_(to_bf16(p.q))
    kv.copy_(to_bf16(p.kv))
    key.copy_(to_bf16(p.key))
    at = dev(np.array([0, rows], np.int32))
    out, lse = torch.empty((rows, heads, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, heads), device="cuda")
    ws = torch.empty(B.mla_prefill_workspace_size(1, rows, heads), dtype=torch.uint8, device="cuda")
    B.splash_mla_prefill(q, kv[..., :128], key, kv[..., 128:], at, at, out, lse, ws)
    want = p.run(spare=0)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    w = to_bf16(bf16(rng, heads, 256, 512, scale=512 ** -0.5))
    pos, rope = dev(np.arange(rows, dtype=np.int32)), rope_of(True)
    packed = [torch.empty((rows, heads, 576), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.splash_mla_absorb_q(q, w[:, :128], packed[0], positions=pos, rope=rope)
    B.splash_mla_absorb_q(to_bf16(p.q), w[:, :128], packed[1], positions=pos, rope=rope)
    dense = torch.empty((rows, heads, 128), dtype=torch.bfloat16, device="cuda")
    latent_out = packed[1][..., :512].contiguous()
    B.splash_mla_expand_out(latent_out, w[:, 128:], y)
    B.splash_mla_expand_out(latent_out, w[:, 128:], dense)
    torch.cuda.synchronize()
    assert torch.equal(packed[0], packed[1]) and torch.equal(y, dense)
    # through the cache and back
    latent, back, back_key = wide(8192, (512,)), wide(16384, (512,)), wide(32768, (64,))
    latent.copy_(to_bf16(bf16(rng, rows, 512)))
    pool = torch.zeros((5, PAGE, 576), dtype=torch.bfloat16, device="cuda")
    desc = B.make_desc(1, 16, 5, 5, B.KV_BF16)
    B.splash_mla_append(latent, key, pos, pool, None, desc)
    B.splash_mla_gather(pool, dev(np.arange(5, dtype=np.int32)[None]), at, back, back_key, desc)
    torch.cuda.synchronize()
    assert torch.equal(back, latent) and torch.equal(back_key, key)


def test_one_row_of_any_stride():
    """A single row's stride is never walked: views whose row stride is not a multiple of 8."""
    rng = rng_of(38)
    base = to_bf16(bf16(rng, 2, 577))
    latent, key = base[:1, :512], base[:1, 512:576]
    pool = torch.zeros((1, PAGE, 576), dtype=torch.bfloat16, device="cuda")
    desc, slot = B.make_desc(1, 16, 1, 1, B.KV_BF16), dev(np.array([3], np.int32))
    B.splash_mla_append(latent, key, slot, pool, None, desc)
    got, got_key = torch.zeros((2, 577), dtype=torch.bfloat16, device="cuda")[:1, :512], torch.zeros((2, 65), dtype=torch.bfloat16, device="cuda")[:1, :64]
    B.splash_mla_gather(pool, dev(np.zeros((1, 1), np.int32)), dev(np.array([0, 1], np.int32)), got, got_key, desc,
                        key_begin=dev(np.array([3], np.int32)))
    torch.cuda.synchronize()
    assert torch.equal(got, latent) and torch.equal(got_key, key)
