"""splash_mla_prefill: what a row's bits depend on."""
import numpy as np
import pytest
import torch

from paper_2609_37626_amd import binding as B
from tests.layer_inputs import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


@pytest.mark.parametrize("new,old,heads", [([300, 20], [420, 0], 2), ([600, 601, 7], [0, 30, 0], 64), ([520, 300], [4000, 2900], 2),
                                           ([1024], [4096], 72)])
@pytest.mark.parametrize("factor", [30.0, 0.01])
def test_a_row_depends_on_its_own_values(new, old, heads, factor):
    """Other queries of its tile, other requests and other heads: their values reach no row, whose reference moves by its
    own scores alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()
    q_at = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    kv_at = np.concatenate([[0], np.cumsum(np.array(new) + old)]).astype(np.int32)
    rows, keys = int(q_at[-1]), int(kv_at[-1])
    q, kv, key = randn(rows, heads, 192), randn(keys, heads, 256), randn(keys, 64)
    ws = torch.empty(B.mla_prefill_workspace_size(len(new), rows, heads), dtype=torch.uint8, device="cuda")

    def run():
        out, lse = torch.empty((rows, heads, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, heads), device="cuda")
        B.splash_mla_prefill(q, kv[..., :128], key, kv[..., 128:], dev(q_at), dev(kv_at), out, lse, ws)
        torch.cuda.synchronize()
        return out, lse

    out, lse = run()
    mine = torch.zeros((rows, heads), dtype=torch.bool, device="cuda")
    mine[:new[0]:3, heads - 1] = True                                  # every third row of the first request
    q *= torch.where(mine, 1.0, factor).bfloat16()[..., None]
    kv[:, :heads - 1] *= factor
    kv[int(kv_at[1]):] *= factor
    key[int(kv_at[1]):] *= factor
    again, lse_again = run()
    assert torch.equal(out[mine], again[mine]) and torch.equal(lse[mine], lse_again[mine])
    assert not torch.equal(out[~mine], again[~mine])
