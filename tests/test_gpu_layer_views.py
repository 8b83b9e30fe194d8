"""Views of one token, row, key or head: what a stride over them says is not looked at, in any call around the latent cache."""
import numpy as np
import pytest
import torch

from paper_2609_37626_amd import binding as B
from tests.layer_inputs import PAGE, dev

pytestmark = pytest.mark.gpu
ODD = [577, 3, (1 << 25) + 1]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def bf16(*shape):
    return torch.randn(shape, device="cuda").bfloat16()


def odd(t, stride, *dims):
    """The same memory, with `stride` over the dimensions (of one element) that are named."""
    assert all(t.shape[d] == 1 for d in dims)
    return t.as_strided(t.shape, [stride if d in dims else s for d, s in enumerate(t.stride())], t.storage_offset())


def zeros(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16, device="cuda")


@pytest.mark.parametrize("stride", ODD)
def test_cache(stride):
    latent, key, pool = bf16(1, 512), bf16(1, 64), zeros(1, PAGE, 576)
    desc, slot = B.make_desc(1, 16, 1, 1, B.KV_BF16), dev(np.array([3], np.int32))
    B.splash_mla_append(odd(latent, stride, 0), odd(key, stride, 0), slot, pool, None, desc)
    back, back_key = zeros(1, 512), zeros(1, 64)
    B.splash_mla_gather(pool, dev(np.zeros((1, 1), np.int32)), dev(np.array([0, 1], np.int32)), odd(back, stride, 0),
                        odd(back_key, stride, 0), desc, key_begin=slot)
    torch.cuda.synchronize()
    assert torch.equal(back, latent) and torch.equal(back_key, key)
    assert int(pool.count_nonzero()) == int(latent.count_nonzero() + key.count_nonzero())


@pytest.mark.parametrize("stride", ODD)
@pytest.mark.parametrize("n,h,dims", [(1, 3, [0]), (5, 1, [1]), (1, 1, [0, 1])])
def test_projections(stride, n, h, dims):
    q, w, x = bf16(n, h, 192), bf16(h, 128, 512), bf16(n, h, 512)
    packed, y = [zeros(n, h, 576) for _ in range(2)], [zeros(n, h, 128) for _ in range(2)]
    w_odd = odd(w, stride, 0) if h == 1 else w
    B.splash_mla_absorb_q(q, w, packed[0])
    B.splash_mla_absorb_q(odd(q, stride, *dims), w_odd, packed[1])
    B.splash_mla_expand_out(x, w, y[0])
    B.splash_mla_expand_out(x, w_odd, odd(y[1], stride, *dims))
    torch.cuda.synchronize()
    assert torch.equal(packed[0], packed[1]) and torch.equal(y[0], y[1]) and bool(y[0].any()) and bool(packed[0].any())


@pytest.mark.parametrize("stride", ODD)
@pytest.mark.parametrize("rows,keys,heads", [(1, 70, 2), (40, 1, 2), (70, 70, 1), (1, 1, 3), (1, 1, 1), (1, 2000, 1)])
def test_prefill(stride, rows, keys, heads):
    q, k, key, v = bf16(rows, heads, 192), bf16(keys, heads, 128), bf16(keys, 64), bf16(keys, heads, 128)
    q_at, kv_at = dev(np.array([0, rows], np.int32)), dev(np.array([0, keys], np.int32))
    ws = torch.empty(B.mla_prefill_workspace_size(1, rows, heads), dtype=torch.uint8, device="cuda")
    of = lambda n: ([0] if n == 1 else []) + ([1] if heads == 1 else [])
    views = (odd(q, stride, *of(rows)), odd(k, stride, *of(keys)), odd(key, stride, 0) if keys == 1 else key, odd(v, stride, *of(keys)))
    outs = []
    for q, k, key, v in ((q, k, key, v), views):
        out, lse = zeros(rows, heads, 128), torch.zeros((rows, heads), device="cuda")
        B.splash_mla_prefill(q, k, key, v, q_at, kv_at, out, lse, ws)
        outs.append((out, lse))
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]) and bool(outs[0][0].any())
