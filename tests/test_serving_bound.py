"""Bound calls around the verification without a GPU: what a loop changes in place is held against the tensors that were bound."""
import numpy as np
import pytest

from paper_2511_21699_amd import binding as B


class _Calls:
    """Stands for the library: counts the calls that get there."""

    def __init__(self):
        self.made = 0

    def _call(self, *args):
        self.made += 1
        return B.CB_OK

    cb_append_kv_device = cb_chunk_attention_device = _call


def _verifier(hq=4, hkv=2, d=64):
    v = object.__new__(B.Verifier)
    v.cfg, v.ctx, v._F, v._stream = B.make_config(hq, hkv, d, "f32", "f32", 2, 16, 4, 20), None, _Calls(), lambda stream: None
    return v


@pytest.mark.parametrize("which", ["chunk", "append", "append, keys and values only", "append of trees"])
@pytest.mark.parametrize("short", ["all", "q", "k", "v", "out", "parent"])
def test_offsets_that_outgrow_the_tensors_are_refused(which, short):
    import torch
    rows = lambda name: 5 if short in ("all", name) else 9  # noqa: E731
    q, out = torch.zeros(rows("q"), 4, 64), torch.zeros(rows("out"), 4, 64)
    k, v, parent = torch.zeros(rows("k"), 2, 64), torch.zeros(rows("v"), 2, 64), torch.zeros(rows("parent"), dtype=torch.int32)
    ver, kv = _verifier(), B.CbKvLayer()
    kv_len, off = np.array([3, 4], dtype=np.int32), np.array([0, 2, 5], dtype=np.int32)
    if which == "chunk":
        call, bounded = ver.bind_chunk_attention(q, kv, kv_len, off, out), ("all", "q", "out")
    elif which == "append":
        call, bounded = ver.bind_append_kv(q, k, v, B.head_prep(), kv, kv_len, off, out), ("all", "q", "k", "v", "out")
    elif which == "append of trees":
        call, bounded = ver.bind_append_kv(q, k, v, B.head_prep(), kv, kv_len, off, out, d_parent=parent), ("all", "q", "k", "v", "out", "parent")
    else:
        call, bounded = ver.bind_append_kv(None, k, v, B.head_prep(), kv, kv_len, off, None), ("all", "k", "v")
    call()
    off[:] = 0, 1, 4  # fewer
    call()
    assert ver._F.made == 2
    off[2] = 6
    if short in bounded:
        with pytest.raises(ValueError, match="token_offsets"):
            call()
        assert ver._F.made == 2
    else:
        call()
        assert ver._F.made == 3
        off[2] = 10
        with pytest.raises(ValueError, match="token_offsets"):
            call()
    off[2] = 5
    call()
