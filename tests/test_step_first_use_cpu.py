"""The step calls' first use from several threads (no GPU): what they set up is whole when it says so."""
import sys

import pytest
import torch

from paper_2609_37626_amd import binding as B

pytestmark = pytest.mark.skipif(not hasattr(torch._C, "_cuda_getDevice"), reason="torch without a GPU runtime")


def test_setup_says_it_is_done_last(monkeypatch):
    for name in ("_device", "_raw_stream", "_I32T", "_F32T", "_BF16T"):
        monkeypatch.setattr(B, name, None)
    monkeypatch.setattr(B, "_CODES", {})
    seen = []

    def look(frame, event, arg):   # at every line: what another thread would go by
        if frame.f_code is B._types.__code__:
            seen.append((B._device is not None, all(x is not None for x in (B._raw_stream, B._I32T, B._F32T, B._BF16T))
                         and set(B._CODES) == {B.GQA_E4M3, B.GQA_INT8}))
        return look

    before = sys.gettrace()
    sys.settrace(look)
    try:
        B._types()
    finally:
        sys.settrace(before)
    assert len(seen) > 3 and seen[-1] == (True, True)
    assert all(whole for done, whole in seen if done)
