"""Refusals of the calls around the latent cache, before any launch (no GPU): the C
entry points on addresses that are never read, and the binding's tensor checks."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2609_37626_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20
BAD, UNSUPPORTED, MISALIGNED, SMALL = (B.SPLASH_ERR_INVALID_ARGUMENT, B.SPLASH_ERR_UNSUPPORTED, B.SPLASH_ERR_MISALIGNED,
                                       B.SPLASH_ERR_WORKSPACE_TOO_SMALL)
NAN, INF = float("nan"), float("inf")


def desc(**kw):
    d = B.MlaDesc()
    d.batch, d.num_heads, d.page_size, d.max_pages_per_seq, d.num_pages = 4, 128, 64, 8, 24
    d.dim_qk, d.dim_v, d.kv_dtype, d.kv_scales, d.softmax_scale = 576, 512, B.KV_FP8_E4M3, FAKE, 0.07
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def turn(rot=64, axes=1, scale=1.0, freq=None, axis=None, none=False):
    n = max(1, rot // 2)
    freq = (ctypes.c_double * n)(*([1.0] * n if freq is None else freq))
    d = B.RopeDesc(rot, 0, axes, scale, freq, None if axis is None else (ctypes.c_uint8 * n)(*axis))
    if none:
        d.inv_freq = None
    return d


def append(d, latent=FAKE, ls=2112, key=FAKE, ks=2112, norm=FAKE, eps=1e-6, pos=FAKE, ps=4, rope=None, slots=FAKE, n=4,
           pages=FAKE, scales=FAKE):
    return B.lib().splash_mla_append(latent, ls, key, ks, norm, eps, pos, ps, rope, slots, n, pages, scales,
                                     None if d is None else d, None)


def gather(d, pages=FAKE, table=FAKE, begin=FAKE, indptr=FAKE, rows=4, latent=FAKE, ls=576, key=FAKE, ks=576):
    return B.lib().splash_mla_gather(pages, table, begin, indptr, rows, latent, ls, key, ks, None if d is None else d, None)


def absorb(q=FAKE, qt=20 * 192, qh=192, w=FAKE, wh=256 * 512, wr=512, pos=FAKE, ps=4, rope=None, n=4, heads=20, out=2 * FAKE):
    return B.lib().splash_mla_absorb_q(q, qt, qh, w, wh, wr, pos, ps, rope, n, heads, out, None)


def expand(x=FAKE, w=FAKE, wh=256 * 512, wr=512, n=4, heads=20, y=2 * FAKE, yt=20 * 128, yh=128):
    return B.lib().splash_mla_expand_out(x, w, wh, wr, n, heads, y, yt, yh, None)


def prefill(q=FAKE, qt=20 * 192, qh=192, k=FAKE, kt=20 * 256, kh=256, key=FAKE, ks=64, v=FAKE, vt=20 * 256, vh=256, qi=FAKE,
            ki=FAKE, b=2, rows=8, keys=8, heads=20, scale=0.07, out=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 40, views=(1, 1, 1)):
    r = [B.MlaRows(x, t, h) if on else None for on, (x, t, h) in zip(views, ((q, qt, qh), (k, kt, kh), (v, vt, vh)))]
    p = [None if x is None else bytes(x) for x in r]
    return B.lib().splash_mla_prefill(p[0], p[1], key, ks, p[2], qi, ki, b, rows, keys, heads, scale, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("mutate,status", [
    (dict(batch=-1), BAD), (dict(max_pages_per_seq=0), BAD), (dict(num_pages=0), BAD), (dict(kv_scales=None), BAD),
    (dict(softmax_scale=0.0), BAD), (dict(page_size=16), UNSUPPORTED), (dict(kv_dtype=9), UNSUPPORTED),
    (dict(num_pages=(1 << 25) + 1), UNSUPPORTED), (dict(dim_qk=512), BAD), (dict(num_heads=8), UNSUPPORTED),
])
def test_bad_descriptor(mutate, status):
    d = desc(**mutate)
    assert append(d, scales=d.kv_scales) == status and gather(d) == status
    assert B.lib().splash_last_error()


def test_append_arguments():
    d = desc()
    assert append(None) == BAD and append(d, n=-1) == BAD and append(d, ls=-8) == BAD and append(d, ks=-8) == BAD
    for name in ("latent", "key", "slots", "pages"):
        assert append(d, **{name: None}) == BAD, name
    for name in ("latent", "key", "norm", "pages"):
        assert append(d, **{name: FAKE + 8}) == MISALIGNED, name
    assert append(d, slots=FAKE + 2) == MISALIGNED and append(desc(kv_scales=FAKE + 2), scales=FAKE + 2) == MISALIGNED
    assert append(d, ls=513) == MISALIGNED and append(d, ks=68) == MISALIGNED
    assert append(d, scales=FAKE + 64) == BAD            # other scales than the attention's
    for eps in (-1e-6, NAN, INF):
        assert append(d, eps=eps) == BAD
    assert append(d, n=(1 << 25) + 1) == UNSUPPORTED
    nothing = dict(latent=None, key=None, slots=None, pages=None)
    assert append(d, n=0, **nothing) == B.SPLASH_OK and append(desc(batch=0), **nothing) == B.SPLASH_OK


@pytest.mark.parametrize("call", [lambda **kw: append(desc(), **kw), absorb])
def test_turns(call):
    assert call(rope=turn(none=True)) == BAD and call(rope=turn(scale=NAN)) == BAD
    for rot in (32, 62, 66, 128):
        assert call(rope=turn(rot=rot)) == BAD
    assert call(rope=turn(axes=0)) == BAD and call(rope=turn(axes=5)) == BAD
    assert call(rope=turn(freq=[1.0] * 31 + [INF])) == BAD
    assert call(rope=turn(axis=[0] * 31 + [1])) == BAD and call(rope=turn(axes=2, axis=[0] * 31 + [2])) == BAD
    assert call(rope=turn(), pos=None) == BAD and call(rope=turn(), pos=FAKE + 2) == MISALIGNED
    assert call(rope=turn(axes=2), ps=3) == BAD and call(rope=turn(axes=2), ps=-4) == BAD


def test_gather_arguments():
    d = desc()
    assert gather(None) == BAD and gather(d, rows=-1) == BAD and gather(d, ls=504) == BAD and gather(d, ks=56) == BAD
    for name in ("pages", "table", "indptr", "latent", "key"):
        assert gather(d, **{name: None}) == BAD, name
    for name in ("pages", "latent", "key"):
        assert gather(d, **{name: FAKE + 8}) == MISALIGNED, name
    for name in ("table", "begin", "indptr"):
        assert gather(d, **{name: FAKE + 2}) == MISALIGNED, name
    assert gather(desc(kv_scales=FAKE + 2)) == MISALIGNED
    assert gather(d, ls=580) == MISALIGNED and gather(d, ks=68) == MISALIGNED
    assert gather(d, rows=(1 << 25) + 1) == UNSUPPORTED and gather(desc(max_pages_per_seq=1 << 25)) == UNSUPPORTED
    nothing = dict(pages=None, table=None, indptr=None, latent=None, key=None)
    assert gather(d, rows=0, **nothing) == B.SPLASH_OK and gather(desc(batch=0), **nothing) == B.SPLASH_OK


@pytest.mark.parametrize("call,inp,out", [(absorb, "q", "out"), (expand, "x", "y")])
def test_projection_arguments(call, inp, out):
    assert call(n=-1) == BAD and call(heads=-1) == BAD and call(wh=-8) == BAD and call(wr=-8) == BAD
    for name in (inp, "w", out):
        assert call(**{name: None}) == BAD, name
        assert call(**{name: FAKE + 8}) == MISALIGNED, name
    assert call(**{out: FAKE}) == BAD
    assert call(wh=516) == MISALIGNED and call(wr=513) == MISALIGNED
    assert call(heads=1025) == UNSUPPORTED and call(n=(1 << 24) + 1) == UNSUPPORTED
    assert call(n=1 << 24, heads=17) == UNSUPPORTED
    for kw in (dict(n=0), dict(heads=0)):
        assert call(**{inp: None, "w": None, out: None}, **kw) == B.SPLASH_OK


def test_projection_strides():
    assert absorb(qt=-8) == BAD and absorb(qh=-8) == BAD and absorb(qt=100) == MISALIGNED and absorb(qh=196) == MISALIGNED
    assert expand(yt=-8) == BAD and expand(yh=-8) == BAD and expand(yt=20 * 128 + 4) == MISALIGNED and expand(yh=132) == MISALIGNED
    assert expand(yh=120) == BAD and expand(yt=19 * 128) == BAD                    # rows overlap
    assert expand(yt=128, yh=3 * 128) == BAD and expand(yt=0) == BAD and expand(yh=0) == BAD
    assert expand(yt=(1 << 63) - 8, yh=(1 << 62)) == BAD


def test_prefill_arguments():
    for i in range(3):
        assert prefill(views=[j != i for j in range(3)]) == BAD
    for name in ("b", "rows", "keys", "heads"):
        assert prefill(**{name: -1}) == BAD, name
    for name in ("qt", "qh", "kt", "kh", "ks", "vt", "vh"):
        assert prefill(**{name: -8}) == BAD, name
        assert prefill(**{name: 1028}) == MISALIGNED, name
    for name in ("qt", "kt", "ks", "vt"):
        assert prefill(**{name: (1 << 24) + 8}) == UNSUPPORTED, name
    for name in ("q", "k", "key", "v", "qi", "ki", "out", "ws"):
        assert prefill(**{name: None}) == BAD, name
    for name in ("q", "k", "key", "v", "out", "ws"):
        assert prefill(**{name: FAKE + 8}) == MISALIGNED, name
    for name in ("qi", "ki", "lse"):
        assert prefill(**{name: FAKE + 2}) == MISALIGNED, name
    for scale in (0.0, -1.0, NAN, INF, 3e38):
        assert prefill(scale=scale) == BAD, scale
    need = B.mla_prefill_workspace_size(2, 8, 20)
    assert need > 0 and prefill(ws_bytes=need - 1) == SMALL and prefill(ws_bytes=0) == SMALL
    assert prefill(heads=1025) == UNSUPPORTED and prefill(rows=(1 << 25) + 1) == UNSUPPORTED
    assert prefill(keys=(1 << 25) + 1) == UNSUPPORTED and prefill(b=(1 << 20) + 1) == UNSUPPORTED
    assert prefill(rows=1 << 25, heads=64) == UNSUPPORTED          # rows * heads
    assert prefill(rows=1 << 20, heads=1024, b=1 << 12) == UNSUPPORTED   # tiles
    nothing = dict(q=None, k=None, key=None, v=None, qi=None, ki=None, out=None, lse=None, ws=None, ws_bytes=0)
    for name in ("b", "rows", "heads"):
        assert prefill(**{name: 0}, **nothing) == B.SPLASH_OK, name
    assert B.lib().splash_mla_prefill_workspace_size(-1, 8, 8) == 0


def test_binding_refuses_host_tensors():
    def bf16(*shape):
        return torch.zeros(*shape, dtype=torch.bfloat16)

    def i32(*shape):
        return torch.zeros(*shape, dtype=torch.int32)

    pool, d = bf16(2, 64, 576), B.make_desc(1, 128, 2, 2, B.KV_BF16)
    rope = B.make_rope(64, [1.0] * 32)
    for call in (lambda: B.splash_mla_append(bf16(3, 512), bf16(3, 64), i32(3), pool, None, d),
                 lambda: B.splash_mla_gather(pool, i32(1, 2), i32(2), bf16(3, 512), bf16(3, 64), d),
                 lambda: B.splash_mla_absorb_q(bf16(3, 2, 192), bf16(2, 128, 512), bf16(3, 2, 576)),
                 lambda: B.splash_mla_absorb_q(bf16(3, 192), bf16(2, 128, 512), bf16(3, 2, 576)),
                 lambda: B.splash_mla_expand_out(bf16(3, 2, 512), bf16(2, 128, 512), bf16(3, 2, 128)),
                 lambda: B.splash_mla_expand_out(bf16(3), bf16(2, 128, 512), bf16(3, 2, 128)),
                 lambda: B.splash_mla_prefill(bf16(3, 2, 192), bf16(3, 2, 128), bf16(3, 64), bf16(3, 2, 128), i32(2), i32(2),
                                              bf16(3, 2, 128), None, torch.zeros(8, dtype=torch.uint8)),
                 lambda: B._turn_args(None, rope, 3, -1), lambda: B._turn_args(i32(4), rope, 3, -1),
                 lambda: B._turn_args(torch.zeros(3), rope, 3, -1), lambda: B._turn_args(i32(6)[::2], rope, 3, -1),
                 lambda: B.mla_prefill_workspace_size(-1, 3, 2)):
        with pytest.raises(B.SplashError):
            call()


def test_layer_checks_under_host_sanitizers(tmp_path):
    """The checks over random and extreme arguments, built with host sanitizers against stubs of the launchers."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    csrc, exe = os.path.join(ROOT, "paper_2609_37626_amd", "csrc"), tmp_path / "layer_fuzz"
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
                        "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                        "-Xarch_host", "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                        os.path.join(csrc, "api.cpp"), os.path.join(csrc, "layer_api.cpp"),
                        os.path.join(ROOT, "tests", "sanitize", "launch_stubs.cpp"),
                        os.path.join(ROOT, "tests", "sanitize", "layer_fuzz.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe), "200000"], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    assert r.stdout.startswith("ok ") and all(int(n) > 300 for n in r.stdout.split()[1:])   # launches of each call
