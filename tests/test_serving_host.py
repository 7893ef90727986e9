"""The calls around the verification without a GPU: every refusal comes from the host's checks, before anything is launched."""
import ctypes as C

import numpy as np
import pytest

from paper_2511_21699_amd import binding as B

A = 1 << 20  # an address nobody reads


def test_the_reference_is_right_on_hand_made_inputs():
    from .serving_reference import chunk_attention, depths, prepared, token_logprobs
    assert depths([-1, 0, 0, 2]) == [0, 1, 1, 2]
    x = np.zeros((1, 1, 16))
    x[0, 0, 0], x[0, 0, 3] = 1.0, 2.0
    y, _ = prepared(x, None, 0.0, [np.pi / 2] * 8, False, [1])
    assert np.allclose(y[0, 0, [0, 8, 3, 11]], [0, 1, 0, 2])
    y, _ = prepared(x, None, 0.0, [np.pi / 2] * 8, True, [1])
    assert np.allclose(y[0, 0, [0, 1, 2, 3]], [0, 1, -2, 0])
    y, _ = prepared(x, np.full(16, 3.0), 0.0, None, False, [7])
    assert np.allclose((y ** 2).mean(), 9.0)
    k = np.ones((3, 1, 4))
    v = np.arange(3.0)[:, None, None] * np.ones((3, 1, 4))
    out, _, _ = chunk_attention(np.ones((2, 2, 4)), [k], [v], [1], [0, 2], 1.0)
    assert np.allclose(out[:, :, 0], [[0.5, 0.5], [1.0, 1.0]])
    lp, ent, top, tops = token_logprobs([0.0, 1.0, 1.0, -np.inf], 3, 3)
    assert lp == -np.inf and list(top) == [1, 2, 0] and np.isclose(np.exp(tops).sum(), 1.0)
    assert np.isclose(ent, -(np.exp(tops) * tops).sum())
    assert token_logprobs([-np.inf] * 4, 0, 2)[:2] == (-np.inf, 0.0)


def test_null_contexts_are_refused():
    L = B.load()
    one = (C.c_int32 * 2)(0, 1)
    kv, prep = B.CbKvLayer(A, A, 8, None, 0, 0), B.CbHeadPrep()
    assert L.cb_append_kv_device(None, None, 1, A, 8, A, 8, A, 8, C.byref(prep), C.byref(kv), one, one, None, A) == B.CB_EINVAL
    assert b"context" in L.cb_last_error(None)
    assert L.cb_chunk_attention_device(None, None, 1, A, C.byref(kv), one, one, A) == B.CB_EINVAL
    assert L.cb_token_logprobs_device(None, None, A, 8, 1, 1, None, None, None, None, 0, None, None) == B.CB_EINVAL


def test_head_prep_checks_its_tensors():
    import torch
    p = B.head_prep(torch.ones(64), None, 1e-5, torch.ones(16), interleaved=True)
    assert (p.rotary_dim, p.interleaved, p.k_weight) == (32, 1, None)
    assert B.head_prep().rotary_dim == 0
    with pytest.raises(ValueError):
        B.head_prep(torch.ones(64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        B.head_prep(inv_freq=torch.ones(32)[::2])


CFG = dict(Hq=32, Hkv=8, D=128, qkv_dtype="bf16", logits_dtype="bf16", max_batch=4, max_nodes=16, max_depth=4, vocab=20)


def _check(fn, *args):
    err = C.create_string_buffer(256)
    L = B.load()
    rc = getattr(L, "cb_debug_check_" + fn)(*args, err)
    return rc, err.value.decode()


def _ints(*x):
    return (C.c_int32 * len(x))(*x)


def _append(cfg=CFG, batch=2, q=A, qs=4096, k=2 * A, ks=1024, v=3 * A, vs=1024, prep=None, kv=None, kv_len=(5, 0), offsets=(0, 3, 4), parent=None, out=8 * A):
    cfg = B.make_config(**cfg)
    prep = B.CbHeadPrep(None, None, A, 1e-6, 128, 0) if prep is None else prep
    kv = B.CbKvLayer(4 * A, 5 * A, 64, None, 0, 0) if kv is None else kv
    c = C.c_int64
    p = C.c_void_p
    return _check("append", C.byref(cfg), batch, p(q), c(qs), p(k), c(ks), p(v), c(vs), C.byref(prep), C.byref(kv), _ints(*kv_len), _ints(*offsets), p(parent), p(out))


@pytest.mark.parametrize("kw, code, text", [
    (dict(), B.CB_OK, ""),
    (dict(q=None, out=None, qs=-1), B.CB_OK, ""),
    (dict(q=8 * A), B.CB_OK, ""),                                           # in place
    (dict(offsets=(0, 0, 0), q=None, k=None, v=None, out=None), B.CB_OK, ""),  # nothing new
    (dict(offsets=(0, 0, 4)), B.CB_OK, ""),
    (dict(kv_len=(61, 63)), B.CB_OK, ""),                                   # up to the cache's end
    (dict(parent=A), B.CB_OK, ""),
    (dict(k=None), B.CB_EINVAL, "null"),
    (dict(q=None), B.CB_EINVAL, "both or neither"),
    (dict(out=None), B.CB_EINVAL, "both or neither"),
    (dict(batch=5, kv_len=(0,) * 5, offsets=(0,) * 6), B.CB_EINVAL, "batch"),
    (dict(batch=0), B.CB_EINVAL, "batch"),
    (dict(q=A + 8), B.CB_EINVAL, "aligned"),
    (dict(v=A + 2), B.CB_EINVAL, "aligned"),
    (dict(qs=4095 + 8), B.CB_EINVAL, "multiples of 16"),
    (dict(qs=4088), B.CB_EINVAL, "less than its heads"),
    (dict(ks=512), B.CB_EINVAL, "less than its heads"),
    (dict(vs=-1024), B.CB_EINVAL, "less than its heads"),
    (dict(vs=1 << 40), B.CB_EINVAL, "2^32"),
    (dict(offsets=(1, 3, 4)), B.CB_EINVAL, "must be 0"),
    (dict(offsets=(0, 3, 2)), B.CB_EINVAL, "falls"),
    (dict(kv_len=(5, -1)), B.CB_EINVAL, "negative"),
    (dict(kv_len=(62, 0)), B.CB_ECAP, "does not fit"),
    (dict(kv_len=(2 ** 31 - 1, 0)), B.CB_ECAP, "does not fit"),
    (dict(offsets=(0, 17, 18), parent=A), B.CB_ECAP, "max_nodes"),
    (dict(prep=B.CbHeadPrep(None, None, A, 1e-6, 24, 0)), B.CB_EINVAL, "rotary_dim"),
    (dict(prep=B.CbHeadPrep(None, None, A, 1e-6, 144, 0)), B.CB_EINVAL, "rotary_dim"),
    (dict(prep=B.CbHeadPrep(None, None, None, 1e-6, 128, 0)), B.CB_EINVAL, "inv_freq"),
    (dict(prep=B.CbHeadPrep(A, None, None, -1.0, 0, 0)), B.CB_EINVAL, "norm_eps"),
    (dict(prep=B.CbHeadPrep(A, None, None, float("nan"), 0, 0)), B.CB_EINVAL, "norm_eps"),
    (dict(prep=B.CbHeadPrep(A + 4, None, None, 0.0, 0, 0)), B.CB_EINVAL, "aligned"),
    (dict(q=8 * A + 16), B.CB_EINVAL, "overlaps q"),
    (dict(q=8 * A, qs=6144), B.CB_EINVAL, "overlaps q"),
    (dict(out=3 * A), B.CB_EINVAL, "overlaps k or v"),
    (dict(kv=B.CbKvLayer(4 * A, 5 * A + 4, 64, None, 0, 0)), B.CB_EINVAL, "cache"),
    (dict(kv=B.CbKvLayer(4 * A, None, 64, None, 0, 0)), B.CB_EINVAL, "cache"),
    (dict(kv=B.CbKvLayer(4 * A, 5 * A, 64, None, 0, 7)), B.CB_EINVAL, "layout"),
    (dict(cfg=dict(CFG, block_size=16), kv=B.CbKvLayer(4 * A, 5 * A, 64, None, 4, 0)), B.CB_EINVAL, "block table"),
    (dict(cfg=dict(CFG, block_size=16), kv=B.CbKvLayer(4 * A, 5 * A, 64, A, 1, 0), kv_len=(14, 0)), B.CB_ECAP, "does not fit"),
])
def test_append_checks_its_arguments(kw, code, text):
    rc, err = _append(**kw)
    assert rc == code and text in err, (rc, err)


@pytest.mark.parametrize("kw, code, text", [
    (dict(), B.CB_OK, ""),
    (dict(out=A), B.CB_OK, ""),
    (dict(offsets=(0, 0, 0), q=None, out=None), B.CB_OK, ""),
    (dict(offsets=(0, 40, 41), kv_len=(20, 63)), B.CB_OK, ""),  # longer than a tree may be
    (dict(q=None), B.CB_EINVAL, "null"),
    (dict(out=A + 16), B.CB_EINVAL, "overlaps"),
    (dict(q=A + 4), B.CB_EINVAL, "aligned"),
    (dict(kv_len=(62, 0)), B.CB_ECAP, "does not fit"),
    (dict(offsets=(0, -1, 3)), B.CB_EINVAL, "falls"),
    (dict(batch=9), B.CB_EINVAL, "batch"),
])
def test_chunk_attention_checks_its_arguments(kw, code, text):
    a = dict(batch=2, q=A, kv_len=(5, 0), offsets=(0, 3, 4), out=8 * A)
    a.update(kw)
    cfg, kv = B.make_config(**CFG), B.CbKvLayer(4 * A, 5 * A, 64, None, 0, 0)
    rc, err = _check("chunk", C.byref(cfg), a["batch"], C.c_void_p(a["q"]), C.byref(kv), _ints(*a["kv_len"]), _ints(*a["offsets"]), C.c_void_p(a["out"]))
    assert rc == code and text in err, (rc, err)


def test_chunk_attention_counts_rows_in_32_bits():
    cfg, kv = B.make_config(**CFG), B.CbKvLayer(4 * A, 5 * A, 1 << 30, None, 0, 0)
    for n, code in ((1 << 28, B.CB_OK), ((1 << 28) + 1, B.CB_EINVAL)):  # four heads to a kv head
        rc, err = _check("chunk", C.byref(cfg), 1, C.c_void_p(1 << 60), C.byref(kv), _ints(5), _ints(0, n), C.c_void_p(1 << 61))
        assert rc == code and (rc == B.CB_OK or "too many tokens" in err)


@pytest.mark.parametrize("kw, code, text", [
    (dict(), B.CB_OK, ""),
    (dict(logits=A + 2), B.CB_OK, ""),
    (dict(n=0, logits=None), B.CB_OK, ""),
    (dict(n=9, rows=A), B.CB_OK, ""),
    (dict(tokens=None, lp=None), B.CB_OK, ""),
    (dict(k=0, ids=None, tops=None), B.CB_OK, ""),
    (dict(logits=None), B.CB_EINVAL, "null"),
    (dict(logits=A + 1), B.CB_EINVAL, "misaligned"),
    (dict(ent=A + 2), B.CB_EINVAL, "misaligned"),
    (dict(n=9), B.CB_EINVAL, "9 results of 8"),
    (dict(n=-1), B.CB_EINVAL, "results"),
    (dict(stride=19), B.CB_EINVAL, "logits_stride"),
    (dict(stride=1 << 40), B.CB_EINVAL, "logits_stride"),
    (dict(k=21), B.CB_EINVAL, "top_k"),                      # (the vocabulary has 20)
    (dict(k=-1), B.CB_EINVAL, "top_k"),
    (dict(k=33, vocab=1000, stride=1000), B.CB_EINVAL, "top_k"),
    (dict(ids=None), B.CB_EINVAL, "top_k without"),
    (dict(tops=None), B.CB_EINVAL, "top_k without"),
    (dict(tokens=None), B.CB_EINVAL, "both or neither"),
    (dict(lp=None), B.CB_EINVAL, "both or neither"),
])
def test_token_logprobs_checks_its_arguments(kw, code, text):
    a = dict(logits=A, stride=20, rows_of=8, n=8, rows=None, tokens=A, lp=A, ent=A, k=5, ids=A, tops=A, vocab=20)
    a.update(kw)
    cfg, p = B.make_config(**dict(CFG, vocab=a["vocab"])), C.c_void_p
    rc, err = _check("logprobs", C.byref(cfg), p(a["logits"]), C.c_int64(a["stride"]), a["rows_of"], a["n"], p(a["rows"]), p(a["tokens"]), p(a["lp"]), p(a["ent"]), a["k"],
                     p(a["ids"]), p(a["tops"]))
    assert rc == code and text in err, (rc, err)


@pytest.mark.parametrize("seed", range(60))
def test_the_plan_covers_a_chunk(seed):
    """Splits cover the longest sequence, jobs are counted as the kernel counts them, and options are kept to."""
    rng = np.random.default_rng(seed)
    g, hkv, d, dtype = int(rng.choice([1, 2, 4, 5, 16])), int(rng.choice([1, 2, 8])), int(rng.choice([64, 128])), str(rng.choice(["bf16", "f32"]))
    batch, max_splits = int(rng.choice([1, 3, 64])), int(rng.choice([0, 1, 7]))
    n = [int(rng.choice([0, 1, 1, 7, 64, 700, 5000])) for _ in range(batch)]
    n[int(rng.integers(batch))] = 1 + int(rng.integers(300))
    s = [int(rng.choice([0, 1, 100, 3000, 70000, 10**6])) for _ in range(batch)]
    cfg = B.make_config(g * hkv, hkv, d, dtype, dtype, batch, int(rng.choice([1, 64])), 1, 100, 16, max_splits)
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    L, ip = B.load(), C.POINTER(C.c_int32)
    for rows, splits in ((0, 0), (64, 0), (128, 5), (256, 1), (0, 64)):
        plan = (C.c_int32 * 5)()
        assert L.cb_debug_chunk_plan(C.byref(cfg), batch, np.array(s, dtype=np.int32).ctypes.data_as(ip), off.ctypes.data_as(ip), splits, rows, plan) == B.CB_OK
        tile, ns, keys, jobs, tiles = plan
        assert tile in ((16, 32) if dtype == "f32" else (64, 128, 256) if d == 128 else (64, 128))
        if rows and dtype == "bf16":
            assert tile == min(rows, 256 if d == 128 else 128)
        assert tiles == max(-(-x * g // tile) for x in n)
        assert 1 <= ns <= 1024 and (max_splits == 0 or ns <= max_splits) and (splits == 0 or ns <= splits)
        if batch == 1:
            assert keys % 32 == 0 and ns == -(-(s[0] + n[0]) // keys) and jobs == tiles * hkv * ns
