"""splash_rope over tensors whose rows overlap or are woven into each other."""
import numpy as np
import pytest
import torch

from paper_2609_37626_amd import binding as B
from tests.step_inputs import bf16, to_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def test_rope_refuses_overlapping_rows_and_views():
    rope = B.make_rope(64, 0.9 ** np.arange(32))
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    rows = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    x = rows[:5 * 2 * 64].view(5, 2, 64)
    for strides in ((64, 64), (128, 32), (64, 96), (96, 64)):
        y = rows.as_strided((5, 2, 64), (*strides, 1))
        with pytest.raises(B.SplashError):
            B.splash_rope(y, pos, rope)
        with pytest.raises(B.SplashError):
            B.splash_rope(torch.zeros_like(x), pos, rope, out=y)
    other = torch.zeros_like(x)
    for kw in (dict(x2=x), dict(x2=other, out2=x), dict(out=other, x2=other)):
        with pytest.raises(B.SplashError):
            B.splash_rope(x, pos, rope, **kw)


@pytest.mark.parametrize("rot,token,head", [(64, 128, 192), (8, 24, 8 + 24 * 2), (6, 14, 7)])
def test_rope_of_rows_woven_into_each_other(rot, token, head):
    # (the rows of one head between those of another, no element shared)
    rng = np.random.Generator(np.random.PCG64(rot))
    heads = 2
    x = to_bf16(bf16(rng, 5, heads, rot))
    pos = torch.arange(5, dtype=torch.int32, device="cuda") * 37
    rope = B.make_rope(rot, 0.9 ** np.arange(rot // 2))
    want = torch.empty_like(x)
    B.splash_rope(x, pos, rope, out=want)
    memory = torch.full((4 * token + (heads - 1) * head + rot,), 7.0, dtype=torch.bfloat16, device="cuda")
    y = memory.as_strided((5, heads, rot), (token, head, 1))
    y.copy_(x)
    before = memory.clone()
    B.splash_rope(y, pos, rope)
    assert torch.equal(y, want)
    y.copy_(x)
    assert torch.equal(memory, before)
