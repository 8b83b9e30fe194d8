"""splash_mla_prefill at its largest sizes: rows, requests and tiles up to the limits, offsets past 2^32 elements."""
import pytest
import torch

from paper_2609_37626_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GiB of GPU memory")
    B.lib()


def indptr(lengths):
    return torch.nn.functional.pad(lengths.cumsum(0), (1, 0)).int().cuda()


@pytest.mark.parametrize("batch,new,old,heads", [(16000, (0, 3), (0, 4), 128), (1 << 20, (32, 32), (0, 0), 1), (1 << 20, (0, 64), (0, 1), 1),
                                                 (300, (0, 4000), (0, 3000), 9)])
def test_many_requests_and_rows(batch, new, old, heads):
    gen = torch.Generator()
    gen.manual_seed(batch + heads)
    lengths = lambda lo, hi: torch.randint(lo, hi + 1, (batch,), generator=gen)
    nq = lengths(*new)
    nk = nq + lengths(*old)
    q_at, kv_at = indptr(nq), indptr(nk)
    rows, keys = min(int(q_at[-1]), 1 << 25), min(int(kv_at[-1]), 1 << 25)      # (what lies past is cut off)
    normal = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_()
    q, k, key, v = normal(rows, heads, 192), normal(keys, heads, 128), normal(keys, 64), normal(keys, heads, 128)
    out = torch.full((rows, heads, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((rows, heads), 1e30, device="cuda")      # (what no row has: of 5 million near 7 some are 7.0 to the bit)
    ws = torch.empty(B.mla_prefill_workspace_size(batch, rows, heads), dtype=torch.uint8, device="cuda")
    B.splash_mla_prefill(q, k, key, v, q_at, kv_at, out, lse, ws)
    torch.cuda.synchronize()
    assert not bool(lse.isnan().any()) and not bool((lse == 1e30).any())
    some = [b for b in {0, 1, batch // 3, batch // 2, batch - 2, batch - 1} if int(kv_at[b + 1]) <= keys and int(q_at[b + 1]) <= rows]
    assert len(some) >= 3
    for b in some:
        q0, q1, k0, k1 = (int(t[i]) for t in (q_at, kv_at) for i in (b, b + 1))
        for n in {q0, (q0 + q1) // 2, q1 - 1} if q1 > q0 else ():
            see = (k1 - k0) - (q1 - n) + 1
            kk = torch.cat([k[k0:k0 + see].double(), key[k0:k0 + see, None].double().expand(-1, heads, -1)], -1)
            z = (kk * q[n].double()).sum(-1) / 192 ** 0.5
            w, vv = torch.softmax(z, 0), v[k0:k0 + see].double()
            want, mass = (w[..., None] * vv).sum(0), (w[..., None] * vv.abs()).sum(0)
            # half a step of bf16 for the output and for each weight; scores' 198 roundings of magnitudes below 2^5
            assert bool(((out[n].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -10) * mass).all()), (b, n)
            assert bool(((lse[n].double() - torch.logsumexp(z, 0)).abs() <= 198 * 2.0 ** -19 + 2.0 ** -10).all()), (b, n)
