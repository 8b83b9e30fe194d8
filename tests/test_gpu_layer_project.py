"""splash_mla_absorb_q and splash_mla_expand_out against the float64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_37626_amd import binding as B
from tests.layer_inputs import FREQ, bf16, dev, key_tolerance, rng_of, rope_of, to_bf16

pytestmark = pytest.mark.gpu
L = oracle.layer


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def near(got, want, sums, terms):
    """bf16's half step, and a rounding to fp32 for each of the sum's products."""
    g = got.float().cpu().numpy().astype(np.float64)
    err = np.abs(g - want)
    print(f"{err.max() if err.size else 0:.2e}", flush=True)
    assert np.all(err <= 2.0 ** -8 * np.abs(want) + (terms + 2) * 2.0 ** -24 * sums), err.max()


def check_absorb(n, h, interleaved=False, rope=True, seed=0, wide=False, axes=None, scale=1.0):
    rng = rng_of(seed)
    q, w = bf16(rng, n, h, 192), bf16(rng, h, 128, 512, scale=512 ** -0.5)
    d_q = to_bf16(q)
    if wide:   # q heads before tokens, and the weight's rows among others
        store = torch.full((h, n, 200), float("nan"), dtype=torch.bfloat16, device="cuda")
        store[..., 8:] = d_q.transpose(0, 1)
        d_q = store[..., 8:].transpose(0, 1)
        rows = torch.full((h, 256, 520), float("nan"), dtype=torch.bfloat16, device="cuda")
        rows[:, 128:, :512] = to_bf16(w)
        d_w = rows[:, 128:, :512]
    else:
        d_w = to_bf16(w)
    out = torch.full((n, h, 576), 7.0, dtype=torch.bfloat16, device="cuda")
    axis = np.zeros(32, int) if axes is None else np.arange(32) % axes
    positions = rng.integers(0, 1 << 20, (axes or 1, n)).astype(np.int32)
    B.splash_mla_absorb_q(d_q, d_w, out, positions=dev(positions if axes else positions[0]) if rope else None,
                          rope=rope_of(interleaved, axis if axes else None, scale) if rope else None)
    torch.cuda.synchronize()
    near(out[..., :512], *L.project(q[..., :128], w, False), 128)
    x = oracle.bf16_bits_to_f64(q[..., 128:])
    if rope:
        want = oracle.step.rope(x, positions, FREQ, axis, interleaved, scale)
        err = np.abs(out[..., 512:].float().cpu().numpy() - want)
        assert np.all(err <= 2.0 ** -8 * np.abs(want) + key_tolerance(q[..., 128:], want, interleaved, scale))
    else:
        assert torch.equal(out[..., 512:].view(torch.int16), d_q[..., 128:].contiguous().view(torch.int16))


@pytest.mark.parametrize("n,h", [(1, 1), (1, 128), (2, 3), (15, 5), (16, 2), (17, 20), (63, 4), (64, 1), (65, 7), (200, 9), (1500, 1)])
def test_absorb(n, h):
    check_absorb(n, h, interleaved=bool(n % 2), seed=n + h)


@pytest.mark.parametrize("interleaved", [False, True])
def test_absorb_views_axes_and_scale(interleaved):
    check_absorb(37, 5, interleaved, wide=True, seed=1)
    check_absorb(70, 2, interleaved, axes=3, scale=0.5, seed=2)


def test_absorb_without_rope():
    check_absorb(40, 3, rope=False, seed=3)


def check_expand(n, h, seed=0, wide=False):
    rng = rng_of(seed)
    x, w = bf16(rng, n, h, 512), bf16(rng, h, 128, 512, scale=512 ** -0.5)
    d_w, y = to_bf16(w), torch.full((n, h, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    if wide:
        rows = torch.full((h, 256, 520), float("nan"), dtype=torch.bfloat16, device="cuda")
        rows[:, 128:, :512] = d_w
        d_w = rows[:, 128:, :512]
        store = torch.full((h, n + 1, 136), 7.0, dtype=torch.bfloat16, device="cuda")
        y = store[:, :n, :128].transpose(0, 1)
    B.splash_mla_expand_out(to_bf16(x), d_w, y)
    torch.cuda.synchronize()
    near(y, *L.project(x, w, True), 512)
    if wide:
        assert bool((store[:, n:] == 7.0).all()) and bool((store[..., 128:] == 7.0).all())


@pytest.mark.parametrize("n,h", [(1, 1), (1, 128), (2, 3), (15, 5), (16, 2), (17, 20), (63, 4), (64, 1), (65, 7), (200, 9), (1500, 1)])
def test_expand(n, h):
    check_expand(n, h, seed=n + h)


@pytest.mark.parametrize("n,h", [(33, 128), (64, 130), (129, 129), (700, 20), (650, 40), (4100, 1), (1025, 7)])
def test_expand_of_more_tokens(n, h):
    """32, 64 and 128 tokens a workgroup, heads fewer and more than the XCDs."""
    check_expand(n, h, seed=n + h)


def test_expand_views():
    check_expand(37, 5, wide=True, seed=1)


@pytest.mark.parametrize("n", [1, 20])
def test_one_token_or_row_that_is_not_finite_stays_with_its_own(n):
    """NaN and infinities of one token's row reach that token alone."""
    rng = rng_of(n)
    q, w = to_bf16(bf16(rng, n, 2, 192)), to_bf16(bf16(rng, 2, 128, 512))
    a, b = (torch.empty((n, 2, 576), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.splash_mla_absorb_q(q, w, a)
    q[n - 1, 1, 5] = float("nan")
    B.splash_mla_absorb_q(q, w, b)
    torch.cuda.synchronize()
    assert bool(b[n - 1, 1, :512].isnan().all()) and torch.equal(a[:n - 1], b[:n - 1]) and torch.equal(a[:, 0], b[:, 0])
    x, w = to_bf16(bf16(rng, n, 2, 512)), to_bf16(bf16(rng, 2, 128, 512))
    c, d = (torch.empty((n, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.splash_mla_expand_out(x, w, c)
    x[0, 0, 500] = float("inf")
    B.splash_mla_expand_out(x, w, d)
    torch.cuda.synchronize()
    assert not bool(d[0, 0].isfinite().any()) and torch.equal(c[1:], d[1:]) and torch.equal(c[:, 1], d[:, 1])


def test_no_tokens_or_heads():
    none = torch.empty((0, 3, 192), dtype=torch.bfloat16, device="cuda")
    w = torch.empty((3, 128, 512), dtype=torch.bfloat16, device="cuda")
    B.splash_mla_absorb_q(none, w, torch.empty((0, 3, 576), dtype=torch.bfloat16, device="cuda"))
    B.splash_mla_expand_out(torch.empty((0, 3, 512), dtype=torch.bfloat16, device="cuda"), w,
                            torch.empty((0, 3, 128), dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
