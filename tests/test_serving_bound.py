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
    import torch
    v.workspace = torch.zeros(1)
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


@pytest.mark.parametrize("which", ["q", "k", "v", "out", "parent", "q_weight", "k_weight", "inv_freq"])
def test_tensors_of_another_device_are_refused(which):
    """(Here the context's device is the CPU; a kernel would be given an address of the other one.)"""
    import torch
    place = lambda name, t: t.to("meta") if name == which else t  # noqa: E731
    ver = _verifier()
    q, out = place("q", torch.zeros(5, 4, 64)), place("out", torch.zeros(5, 4, 64))
    k, v, parent = place("k", torch.zeros(5, 2, 64)), place("v", torch.zeros(5, 2, 64)), place("parent", torch.zeros(5, dtype=torch.int32))
    prep = B.head_prep(place("q_weight", torch.ones(64)), place("k_weight", torch.ones(64)), 1e-6, place("inv_freq", torch.ones(16)))
    with pytest.raises(ValueError, match=which + ".*meta"):
        ver.bind_append_kv(q, k, v, prep, B.CbKvLayer(), [3], [0, 5], out, d_parent=parent)
    if which in ("q", "out"):
        with pytest.raises(ValueError, match=which + ".*meta"):
            ver.bind_chunk_attention(q, B.CbKvLayer(), [3], [0, 5], out)


@pytest.mark.parametrize("which", ["logits", "d_rows", "d_tokens", "logprob", "entropy", "top_tokens", "top_logprobs"])
def test_logits_of_another_device_are_refused(which):
    import torch
    ver = _verifier()
    ver._F.cb_token_logprobs_device = ver._F._call
    t = dict(logits=torch.zeros(3, 20), d_rows=torch.zeros(3, dtype=torch.int32), d_tokens=torch.zeros(3, dtype=torch.int32), logprob=torch.zeros(3), entropy=torch.zeros(3),
             top_tokens=torch.zeros(3, 2, dtype=torch.int32), top_logprobs=torch.zeros(3, 2))

    def bind():
        return ver.bind_token_logprobs(t["logits"], t["d_tokens"], 2, t["logprob"], t["entropy"], t["top_tokens"], t["top_logprobs"], d_rows=t["d_rows"])
    bind()()
    t[which] = t[which].to("meta")
    with pytest.raises(ValueError, match=which + ".*meta"):
        bind()
