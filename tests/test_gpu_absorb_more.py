"""splash_mla_absorb_q where a workgroup takes more than one batch of 64 tokens, against the float64 oracle."""
import pytest
import torch

from paper_2609_37626_amd import binding as B
from tests.layer_inputs import bf16, rng_of, to_bf16
from tests.test_gpu_layer_project import check_absorb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


# 192, 256, 128, 128, 256, 128, 256, 256, 192 and 64 tokens a workgroup; one chunk and several, last batches and chunks that
# are whole and that are not, heads that fill the XCDs evenly and that do not
@pytest.mark.parametrize("n,h", [(129, 128), (256, 128), (257, 64), (1100, 8), (2500, 20), (4100, 3), (640, 40), (321, 130), (193, 127),
                                 (513, 16)])
def test_absorb_of_more_tokens(n, h):
    check_absorb(n, h, interleaved=bool(n % 2), seed=n + h)


@pytest.mark.parametrize("interleaved", [False, True])
def test_absorb_of_more_tokens_in_views(interleaved):
    check_absorb(300, 56, interleaved, wide=True, seed=3)
    check_absorb(700, 23, interleaved, axes=2, scale=0.75, seed=4)


@pytest.mark.parametrize("n,h", [(300, 64), (1100, 20)])
def test_tokens_that_are_not_finite_stay_alone_in_later_batches(n, h):
    rng = rng_of(n)
    q, w = to_bf16(bf16(rng, n, h, 192)), to_bf16(bf16(rng, h, 128, 512))
    a, b = (torch.empty((n, h, 576), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.splash_mla_absorb_q(q, w, a)
    at = [0, 63, 64, 130, 191, 192, n - 1]
    q[at, h - 1, 5] = float("nan")
    B.splash_mla_absorb_q(q, w, b)
    torch.cuda.synchronize()
    assert bool(b[at, h - 1, :512].isnan().all())
    b[at, h - 1] = a[at, h - 1]
    assert torch.equal(a, b)


def test_the_same_call_again():
    """Loads of one batch go where another was read: the same bits each time."""
    rng = rng_of(5)
    q, w = to_bf16(bf16(rng, 2000, 24, 192)), to_bf16(bf16(rng, 24, 128, 512))
    a, b = (torch.empty((2000, 24, 576), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.splash_mla_absorb_q(q, w, a)
    for _ in range(20):
        b.fill_(7.0)
        B.splash_mla_absorb_q(q, w, b)
        torch.cuda.synchronize()
        assert torch.equal(a, b)
