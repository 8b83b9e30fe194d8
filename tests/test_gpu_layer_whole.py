"""A whole latent-attention step, from a token's rows to value heads, in its absorbed and its expanded form, each against the
float64 attention of what the cache holds: within what the documented roundings leave."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_37626_amd import binding as B
from tests.layer_inputs import FORMATS, FREQ, PAGE, bf16, bf16_bits, dev, rng_of, rope_of, table_of, to_bf16

pytestmark = pytest.mark.gpu

# A rounding to bf16 is off by at most half a step, 2^-8 of the value, evenly over it: 2^-8 / sqrt(3) in the mean square,
# where the value is a power of two, and less elsewhere.
EPS = 2.0 ** -8 / np.sqrt(3.0)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def spread(z_scale, q_lat, q_rope, q_nope, c, w_uk, w_uv, dense_rounds):
    """The attention of one row and head over rows c [keys, 576], and the variances that independent roundings to bf16 give
    its values: (y, lse, {form: variance of y}, {form: variance of the lse}, the weights' sum of |y_j|).  A score's error dz_j moves y by
    sum_j w_j dz_j (y_j - y) and the lse by sum_j w_j dz_j; a weight's, relative, by w_j y_j."""
    q = np.concatenate([q_lat, q_rope])
    z = z_scale * (c @ q)
    w = np.exp(z - z.max())
    lse = z.max() + np.log(w.sum())
    w /= w.sum()
    yj = c[:, :512] @ w_uv.T
    y = w @ yj
    apart = yj - y
    s2, e2, w2 = z_scale ** 2, EPS ** 2, w ** 2
    moved = (c * w[:, None]).T @ apart                  # [576, 128]: of y by an entry of the query
    mean = w @ c
    weights, out = e2 * w2 @ np.maximum(yj ** 2, apart ** 2), e2 * y ** 2
    o = w @ c[:, :512]
    absorbed = s2 * e2 * (q ** 2 @ moved ** 2) + weights + e2 * (w_uv ** 2 @ o ** 2) + out
    absorbed_lse = s2 * e2 * (q ** 2 @ mean ** 2)
    k = c[:, :512] @ w_uk.T
    dz2 = s2 * e2 * (k ** 2 @ q_nope ** 2)              # of each key: its 128 dims rounded
    values = e2 * w2 @ yj ** 2
    if dense_rounds:                                    # the history's rows come back rounded
        dz2 = dz2 + s2 * e2 * (c ** 2 @ q ** 2)
        values = values + e2 * w2 @ (c[:, :512] ** 2 @ w_uv.T ** 2)
    expanded = s2 * e2 * (q_rope ** 2 @ moved[512:] ** 2) + (w2 * dz2) @ apart ** 2 + values + weights + out
    expanded_lse = s2 * e2 * (q_rope ** 2 @ mean[512:] ** 2) + w2 @ dz2
    return y, lse, {"absorbed": absorbed, "expanded": expanded}, {"absorbed": absorbed_lse, "expanded": expanded_lse}, w @ np.abs(yj)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("interleaved", [False, True])
def test_both_forms_are_as_near_as_their_roundings(fmt, interleaved):
    rng = rng_of(41)
    kind, heads, chunk, scale = FORMATS[fmt], 16, 3, 192 ** -0.5
    lens = np.array([3, 4, 65, 200, 321], np.int32)
    batch, total = len(lens), int(lens.sum())
    held = [-(-int(s) // PAGE) for s in lens]
    pages = sum(held) + 1
    table = table_of(rng, held, pages)
    indptr = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    pos = np.concatenate([np.arange(s) for s in lens]).astype(np.int32)
    slots = np.concatenate([table[b, np.arange(s) // PAGE] * PAGE + np.arange(s) % PAGE for b, s in enumerate(lens)]).astype(np.int32)
    rows, norm = to_bf16(bf16(rng, total, 576)), to_bf16(bf16(rng, 512))
    w = to_bf16(bf16(rng, heads, 256, 512, scale=512 ** -0.5))
    pool = torch.zeros((pages, PAGE, 656 if fmt == "latent" else 576), dtype=torch.bfloat16 if fmt == "bf16" else torch.uint8, device="cuda")
    scales = torch.ones((pages, PAGE), device="cuda") if fmt == "e4m3" else None
    desc, rope = B.make_desc(batch, heads, table.shape[1], pages, kind, scales), rope_of(interleaved)
    d_table, d_indptr, d_lens = dev(table), dev(indptr), dev(lens)
    q, q_pos = to_bf16(bf16(rng, batch * chunk, heads, 192)), np.concatenate([np.arange(s - chunk, s) for s in lens]).astype(np.int32)

    B.splash_mla_append(rows[:, :512], rows[:, 512:], dev(slots), pool, scales, desc, norm_weight=norm, positions=dev(pos), rope=rope)
    new = lambda *shape: torch.empty((batch * chunk, heads, *shape), dtype=torch.bfloat16, device="cuda")
    packed, latent_out, got = new(576), new(512), {"absorbed": new(128), "expanded": new(128)}
    lse = {form: torch.empty((batch * chunk, heads), device="cuda") for form in got}
    B.splash_mla_absorb_q(q, w[:, :128], packed, positions=dev(q_pos), rope=rope)
    ws = torch.empty(B.workspace_size(batch, chunk, heads), dtype=torch.uint8, device="cuda")
    B.splash_mla_attend(packed, pool, d_table, d_lens, chunk, latent_out, lse["absorbed"], desc, ws)
    B.splash_mla_expand_out(latent_out, w[:, 128:], got["absorbed"])
    dense = torch.empty((total, 576), dtype=torch.bfloat16, device="cuda")
    B.splash_mla_gather(pool, d_table, d_indptr, dense[:, :512], dense[:, 512:], desc)
    kv = (dense[:, :512].float() @ w.float().flatten(0, 1).T.contiguous()).bfloat16().unflatten(-1, (heads, 256))
    turned = q.clone()
    B.splash_rope(turned[..., 128:], dev(q_pos), rope)
    ws2 = torch.empty(B.mla_prefill_workspace_size(batch, batch * chunk, heads), dtype=torch.uint8, device="cuda")
    B.splash_mla_prefill(turned, kv[..., :128], dense[:, 512:], kv[..., 128:], dev(np.arange(batch + 1, dtype=np.int32) * chunk),
                         d_indptr, got["expanded"], lse["expanded"], ws2)
    torch.cuda.synchronize()

    host = pool.view(torch.int16).cpu().numpy().view(np.uint16) if fmt == "bf16" else pool.cpu().numpy()
    cache = oracle.layer.read_rows(host, None if scales is None else scales.cpu().numpy(), kind).reshape(-1, 576)
    ww, qq = w.double().cpu().numpy(), oracle.bf16_bits_to_f64(bf16_bits(q))
    qq[..., 128:] = oracle.step.rope(qq[..., 128:], q_pos[None], FREQ, np.zeros(32, int), interleaved)
    mass, (err, var, lse_err, lse_var) = [], ({form: [] for form in got} for _ in range(4))
    for b in range(batch):
        c = cache[slots[indptr[b]:indptr[b + 1]]]
        for n in range(b * chunk, b * chunk + chunk):
            see = int(q_pos[n]) + 1
            for h in range(heads):
                y, l, v, lv, size = spread(scale, qq[n, h, :128] @ ww[h, :128], qq[n, h, 128:], qq[n, h, :128], c[:see], ww[h, :128],
                                           ww[h, 128:], fmt == "e4m3")
                mass.append(size)
                for form in got:
                    err[form].append(got[form][n, h].double().cpu().numpy() - y)
                    var[form].append(v[form])
                    lse_err[form].append(float(lse[form][n, h]) - l)
                    lse_var[form].append(lv[form])
    for form in got:
        e, s = np.array(err[form]), np.sqrt(np.array(var[form]))
        le, ls = np.array(lse_err[form]), np.sqrt(np.array(lse_var[form]))
        ratio, lse_ratio = np.linalg.norm(e) / np.linalg.norm(s), np.linalg.norm(le) / np.linalg.norm(ls)
        print(fmt, interleaved, form, f"of the roundings' mean square: out {ratio:.3f}, lse {lse_ratio:.3f}; largest "
              f"{np.max(np.abs(e) / s):.2f} and {np.max(np.abs(le) / ls):.2f}", flush=True)
        # The mean square over 30,720 values of 240 rows (240 lse's) stays within a tenth of what it is expected to be, and
        # no value strays 8 of its own (sums of independent roundings have no longer tails than a normal one).  Scores' fp32
        # sums (2^-24 of 576 magnitudes, or 6e-6 of them on the fp8 pipe, a score of 16 or less) add 1e-4 of a weight.
        small = 1e-4 * np.array(mass)
        assert np.linalg.norm(e) <= 1.1 * np.linalg.norm(s) + np.linalg.norm(small) and np.all(np.abs(e) <= 8.0 * s + small), form
        assert np.linalg.norm(le) <= 1.1 * np.linalg.norm(ls) + 1e-4 * np.sqrt(le.size) and np.all(np.abs(le) <= 8.0 * ls + 1e-4), form
