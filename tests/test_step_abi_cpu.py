"""Refusals of the serving-step calls, before any launch (no GPU): the C entry
points on addresses that are never read, and the binding's tensor checks."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2609_37626_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20
BAD, UNSUPPORTED, MISALIGNED, SMALL = (B.SPLASH_ERR_INVALID_ARGUMENT, B.SPLASH_ERR_UNSUPPORTED, B.SPLASH_ERR_MISALIGNED,
                                       B.SPLASH_ERR_WORKSPACE_TOO_SMALL)


def desc(**kw):
    d = B.make_gqa_desc(4, 16, 2, 64, 8, 24)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def attend(d, q=FAKE, k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, bt=FAKE, seq=FAKE, q_chunk=1, out=FAKE, lse=FAKE, ws=FAKE,
           ws_bytes=1 << 40):
    return B.lib().splash_gqa_attend(q, k, v, ks, vs, bt, seq, q_chunk, out, lse, None if d is None else ctypes.byref(d),
                                     ws, ws_bytes, None)


def append(d, k=FAKE, v=FAKE, ts=128, hs=64, slots=FAKE, n=4, kp=FAKE, vp=FAKE, ks=FAKE, vs=FAKE):
    return B.lib().splash_gqa_append(k, v, ts, hs, slots, n, kp, vp, ks, vs, None if d is None else ctypes.byref(d), None)


@pytest.mark.parametrize("mutate,status", [
    (dict(batch=-1), BAD), (dict(max_pages_per_seq=0), BAD), (dict(num_pages=0), BAD),
    (dict(softmax_scale=0.0), BAD), (dict(softmax_scale=float("inf")), BAD),
    (dict(page_size=16), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(num_heads=15), UNSUPPORTED),
    (dict(num_heads=0), UNSUPPORTED), (dict(num_kv_heads=0), UNSUPPORTED), (dict(num_heads=2048), UNSUPPORTED),
    (dict(num_heads=258, num_kv_heads=129), UNSUPPORTED), (dict(code_type=2), UNSUPPORTED),
    (dict(num_pages=(1 << 25) + 1), UNSUPPORTED), (dict(max_pages_per_seq=1 << 25), UNSUPPORTED),
])
def test_bad_gqa_descriptor(mutate, status):
    assert attend(desc(**mutate)) == status
    assert append(desc(**mutate)) == status
    d = desc(**mutate)
    assert B.lib().splash_gqa_workspace_size(ctypes.byref(d), 1) == 0
    assert B.lib().splash_last_error()


def test_gqa_attend_arguments():
    assert attend(None) == BAD and attend(desc(), q_chunk=0) == BAD
    for name in ("q", "k", "v", "ks", "vs", "bt", "seq", "out", "ws"):
        assert attend(desc(), **{name: None}) == BAD, name
    for name in ("q", "k", "v", "out", "ws"):
        assert attend(desc(), **{name: FAKE + 8}) == MISALIGNED, name
    for name in ("ks", "vs", "bt", "seq", "lse"):
        assert attend(desc(), **{name: FAKE + 2}) == MISALIGNED, name
    assert attend(desc(), ws_bytes=0) == SMALL
    need = B.gqa_workspace_size(desc(), 1)
    assert attend(desc(), ws_bytes=need - 1) == SMALL
    assert attend(desc(batch=1 << 20, max_pages_per_seq=1 << 11)) == UNSUPPORTED
    assert attend(desc(batch=(1 << 31) - 1, num_heads=1024, num_kv_heads=128, max_pages_per_seq=(1 << 31) - 1),
                  q_chunk=(1 << 31) - 1) == UNSUPPORTED
    assert attend(desc(batch=0), q=None, k=None, v=None, ks=None, vs=None, bt=None, seq=None, out=None, ws=None,
                  ws_bytes=0) == B.SPLASH_OK


def test_gqa_append_arguments():
    assert append(None) == BAD and append(desc(), n=-1) == BAD
    assert append(desc(), ts=-8) == BAD and append(desc(), hs=-8) == BAD
    for name in ("k", "v", "slots", "kp", "vp", "ks", "vs"):
        assert append(desc(), **{name: None}) == BAD, name
    for name in ("k", "v", "kp", "vp"):
        assert append(desc(), **{name: FAKE + 8}) == MISALIGNED, name
    for name in ("slots", "ks", "vs"):
        assert append(desc(), **{name: FAKE + 2}) == MISALIGNED, name
    assert append(desc(), ts=100) == MISALIGNED and append(desc(), hs=4) == MISALIGNED
    assert append(desc(), n=(1 << 24) + 1) == UNSUPPORTED   # 2 KV heads
    assert append(desc(batch=0), n=(1 << 24) + 1) == B.SPLASH_OK
    assert append(desc(), n=0, k=None, v=None, slots=None, kp=None, vp=None, ks=None, vs=None) == B.SPLASH_OK


def tables(seq=FAKE, new=FAKE, q_chunk=1, batch=4, free=FAKE, num_free=8, taken=FAKE, taken_out=FAKE + 64, table=FAKE,
           width=8, pages=24, rows=4, indptr=FAKE, slots=FAKE, pos=FAKE, req=FAKE):
    return B.lib().splash_step_tables(seq, new, q_chunk, batch, free, num_free, taken, taken_out, table, width, pages, rows,
                                      indptr, slots, pos, req, None)


def test_step_tables_arguments():
    for kw in (dict(batch=-1), dict(rows=-1), dict(num_free=-1), dict(q_chunk=-1), dict(width=0), dict(pages=0),
               dict(taken_out=FAKE)):
        assert tables(**kw) == BAD, kw
    for name in ("seq", "free", "taken", "taken_out", "table", "indptr", "slots", "pos", "req"):
        assert tables(**{name: None}) == BAD, name
        assert tables(**{name: FAKE + 66}) == MISALIGNED, name
    assert tables(new=FAKE + 2) == MISALIGNED
    assert tables(taken_out=FAKE + 4) == BAD and tables(taken=FAKE + 4, taken_out=FAKE) == BAD   # overlap
    assert tables(batch=8193) == UNSUPPORTED and tables(pages=(1 << 25) + 1) == UNSUPPORTED
    assert tables(batch=8192, width=1 << 13) == UNSUPPORTED


def rope(n=4, heads=2, rot=64, axes=1, freq=None, axis=None, scale=1.0, x=FAKE, y=FAKE, strides=(128, 64, 128, 64),
         pos=FAKE, pos_stride=4, views=1):
    half = max(1, rot // 2)
    freq = (ctypes.c_double * half)(*([1.0] * half if freq is None else freq))
    axis = None if axis is None else (ctypes.c_uint8 * half)(*axis)
    d = B.RopeDesc(rot, 0, axes, scale, freq, axis)
    v = (B.RopeView * 2)(*[B.RopeView(x, y, *strides, heads)] * 2)
    return B.lib().splash_rope(v, views, pos, pos_stride, n, ctypes.byref(d), None)


def test_rope_arguments():
    assert rope(views=0) == BAD and rope(views=3) == BAD and rope(n=-1) == BAD and rope(heads=-1) == BAD
    assert rope(axes=0) == BAD and rope(axes=5) == BAD and rope(scale=float("nan")) == BAD
    assert rope(rot=63) == UNSUPPORTED and rope(rot=0) == UNSUPPORTED and rope(rot=258) == UNSUPPORTED
    assert rope(heads=65537) == UNSUPPORTED and rope(n=(1 << 25) + 1) == UNSUPPORTED
    assert rope(freq=[1.0] * 31 + [float("inf")]) == BAD
    assert rope(axis=[0] * 31 + [1]) == BAD and rope(axes=2, axis=[0] * 31 + [2]) == BAD
    assert rope(x=None) == BAD and rope(y=None) == BAD and rope(pos=None) == BAD
    assert rope(x=FAKE + 1) == MISALIGNED and rope(pos=FAKE + 2) == MISALIGNED
    assert rope(strides=(-1, 64, 128, 64)) == BAD
    assert rope(strides=(128, 64, 256, 128)) == BAD            # in place, other strides
    assert rope(y=FAKE * 2, strides=(128, 64, 128, 32)) == BAD  # rows of y overlap
    assert rope(axes=2, axis=[0, 1] * 16, pos_stride=3) == BAD
    assert rope(n=0, x=None, y=None, pos=None) == B.SPLASH_OK
    L, one = B.lib(), B.make_rope(4, [1.0, 0.5])
    assert L.splash_rope(None, 1, FAKE, 4, 4, ctypes.byref(one), None) == BAD
    assert L.splash_rope((B.RopeView * 1)(), 1, FAKE, 4, 4, None, None) == BAD


def test_binding_refuses_host_tensors_and_bad_descriptors():
    with pytest.raises(B.SplashError):
        B.make_rope(8, [1.0] * 3)
    with pytest.raises(B.SplashError):
        B.make_rope(8, [1.0] * 4, pair_axis=[0, 0, 1, 4])
    assert B.make_rope(8, np.ones(4), pair_axis=[0, 2, 1, 1]).num_axes == 3
    x = torch.zeros(2, 1, 8, dtype=torch.bfloat16)
    with pytest.raises(B.SplashError):
        B.splash_rope(x, torch.zeros(2, dtype=torch.int32), B.make_rope(8, [1.0] * 4))
    with pytest.raises(B.SplashError):
        B.gqa_workspace_size(desc(head_dim=80), 1)


def test_step_checks_under_host_sanitizers(tmp_path):
    """The checks over random and extreme arguments, built with host sanitizers against stubs of the launchers."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    csrc, exe = os.path.join(ROOT, "paper_2609_37626_amd", "csrc"), tmp_path / "step_fuzz"
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
                        "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                        "-Xarch_host", "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                        os.path.join(csrc, "api.cpp"), os.path.join(csrc, "step_api.cpp"),
                        os.path.join(ROOT, "tests", "sanitize", "launch_stubs.cpp"),
                        os.path.join(ROOT, "tests", "sanitize", "step_fuzz.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe), "200000"], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    assert r.stdout.startswith("ok ") and int(r.stdout.split()[1]) > 1000   # calls that reached a launch
