"""The calls around the verification as a serving program makes them: a prompt in chunks, single tokens, draft trees and their
compaction on one cache, probabilities of what came out; captured into graphs, on other streams, between the verifications' calls."""
import math

import numpy as np
import pytest

from paper_2511_21699_amd import binding as B
from .serving_gpu import Batch, to_np
from .serving_reference import attention_tolerance, chunk_attention, prepared, token_logprobs

pytestmark = pytest.mark.gpu

FREQ = 1e4 ** (-np.arange(0, 128, 2) / 128)


def _prep(d=128):
    import torch
    w = [torch.rand(d, device="cuda") + 0.5 for _ in range(2)]
    return w, B.head_prep(w[0], w[1], 1e-6, torch.tensor(FREQ, dtype=torch.float32, device="cuda"))


@pytest.mark.parametrize("block", [0, 16])
def test_a_request_from_prompt_to_verified_tree(block):
    import torch
    hq, hkv, d, vocab, prompt, nodes = 8, 2, 128, 700, 300, 12
    b = Batch("bf16", hq, hkv, d, [0], [prompt + 40], block, max_nodes=16, max_depth=8, vocab=vocab)
    b.k.fill_(float("nan"))
    b.v.fill_(float("nan"))
    w, prep = _prep()
    ver = b.ver
    heads = b.draw(prompt + 40, (hq + 2 * hkv) * d)
    q, k, v = (x.unflatten(1, (-1, d)) for x in heads.split([hq * d, hkv * d, hkv * d], 1))
    sizes = [1, 130, 64, 1, 104]  # the prompt in pieces
    out = torch.zeros(prompt, hq, d, dtype=torch.bfloat16, device="cuda")
    at = 0
    for n in sizes:
        rows = slice(at, at + n)
        qr = torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda")
        ver.append_kv(q[rows], k[rows], v[rows], prep, b.kv, [at], [0, n], qr)
        ver.chunk_attention(qr, b.kv, [at], [0, n], out[rows])
        at += n
    assert at == prompt
    whole = torch.empty_like(out)
    qr = torch.empty_like(out)
    ver.append_kv(q[:prompt], k[:prompt], v[:prompt], prep, b.kv, [0], [0, prompt], qr)
    ver.chunk_attention(qr, b.kv, [0], [0, prompt], whole)
    torch.cuda.synchronize()
    f = np.float32(FREQ)
    want_q, _ = prepared(to_np(q[:prompt]), to_np(w[0]), 1e-6, f, False, range(prompt))
    b.new = [prompt]
    # (the kernels' own rounded queries and keys: what the attention is given)
    want, size, score = chunk_attention(to_np(qr), b.keys(), b.values(), [0], [0, prompt], 1 / math.sqrt(d))
    assert np.abs(to_np(qr) - want_q).max() <= 2.0 ** -8 * np.abs(want_q).max()
    tol = attention_tolerance("bf16", want, size, score, prompt, d)
    assert (np.abs(to_np(out) - want) <= tol).all() and (np.abs(to_np(whole) - want) <= tol).all()
    # a draft tree behind the prompt: appended at its depths, verified and compacted; then every accepted node's K is what a token at that
    # position would have appended
    parent = np.array([-1, 0, 0, 1, 2, 3, 5, 4, 2, 6, 9, 1], dtype=np.int32)
    rng = np.random.default_rng(0)
    tokens = rng.integers(0, vocab, nodes).astype(np.int32)
    logits = torch.randn(nodes, vocab, device="cuda").to(torch.bfloat16)
    for child, p in ((2, 0), (4, 2), (7, 4)):
        logits[p, int(tokens[child])] = 20.0
    rows = slice(prompt, prompt + nodes)
    tq = torch.empty(nodes, hq, d, dtype=torch.bfloat16, device="cuda")
    ver.append_kv(q[rows], k[rows], v[rows], prep, b.kv, [prompt], [0, nodes], tq, d_parent=torch.tensor(parent, device="cuda"))
    _, acc_len, acc_tok = ver.verify_tree(tq, b.kv, [prompt], [0, nodes], parent, tokens, logits)
    new_len = ver.compact_kv([b.kv], 1)
    path = ver.get_path(1)[0][:4]
    assert acc_len[0] == 3 and path.tolist() == [0, 2, 4, 7] and new_len[0] == prompt + 4
    cache = b.k.clone(), b.v.clone()
    pick = torch.tensor(path, device="cuda").long() + prompt
    ver.append_kv(None, k[pick], v[pick], prep, b.kv, [prompt], [0, 4], None)
    torch.cuda.synchronize()
    where = b.index(0, 0, prompt + 4)
    assert torch.equal(b.k[where], cache[0][where]) and torch.equal(b.v[where], cache[1][where])
    # what the accepted tokens' probabilities were, from the rows that they came out of
    lp, ent, top, tops = ver.token_logprobs(logits, torch.tensor(acc_tok[0][:4], device="cuda"), 3, d_rows=torch.tensor(path, device="cuda"))
    torch.cuda.synchronize()
    assert top[:, 0].tolist() == acc_tok[0][:4].tolist() and torch.equal(lp, tops[:, 0])
    for i, node in enumerate(path):
        assert abs(float(lp[i]) - token_logprobs(to_np(logits[int(node)]), int(acc_tok[0][i]), 3)[0]) < 1e-4
    # and a single token behind them
    one = slice(prompt + nodes, prompt + nodes + 1)
    qr, o = torch.empty(1, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(1, hq, d, dtype=torch.bfloat16, device="cuda")
    ver.append_kv(q[one], k[one], v[one], prep, b.kv, new_len, [0, 1], qr)
    ver.chunk_attention(qr, b.kv, new_len, [0, 1], o)
    torch.cuda.synchronize()
    b.kv_len, b.new = new_len, [1]
    want, size, score = chunk_attention(to_np(qr), b.keys(), b.values(), new_len.tolist(), [0, 1], 1 / math.sqrt(d))
    assert (np.abs(to_np(o) - want) <= attention_tolerance("bf16", want, size, score, prompt + 5, d)).all()


def test_one_root_is_one_token():
    """A tree of a root alone and a chunk of one token are the same question to two kernels."""
    import torch
    b = Batch("bf16", 32, 8, 128, [900, 33, 0], [1, 1, 1], 16, scale=2.0, max_nodes=4, max_depth=3)
    root = torch.full((3,), -1, dtype=torch.int32, device="cuda")
    tree, chunk = torch.empty_like(b.q), torch.empty_like(b.q)
    b.ver.tree_attention_device(b.q, b.kv, b.kv_len, b.off, root, tree)
    b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off, chunk)
    torch.cuda.synchronize()
    want, size, score = chunk_attention(to_np(b.q), b.keys(), b.values(), b.kv_len.tolist(), b.off.tolist(), 1 / math.sqrt(128))
    tol = attention_tolerance("bf16", want, size, score, 901, 128)
    assert (np.abs(to_np(chunk) - want) <= tol).all() and (np.abs(to_np(tree) - to_np(chunk)) <= 2 * tol).all()


@pytest.mark.parametrize("dtype, kv_len, new", [("bf16", [3000, 5], [1, 1]), ("bf16", [100, 64], [70, 3]), ("f32", [700, 64], [20, 3])])
def test_captured_and_replayed(dtype, kv_len, new):
    """Two graphs of one context, replayed in turn with eager calls between them, against eager results, every time."""
    import torch
    print(f"[case] graphs {dtype} {kv_len} {new}", flush=True)
    b = Batch(dtype, 16, 2, 128, kv_len, new, 16, scale=2.0, vocab=50000, nan=False)
    w, prep = _prep()
    n = b.n
    src = [b.draw(n, h, 128) for h in (16, 2, 2)]
    logits = torch.randn(n, 50000, device="cuda").to(b.t)
    tokens = torch.randint(0, 50000, (n,), device="cuda", dtype=torch.int32)
    q, out = torch.empty_like(b.q), torch.empty_like(b.q)
    lp, ent = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ids, tops = torch.empty(n, 5, device="cuda", dtype=torch.int32), torch.empty(n, 5, device="cuda")
    st = torch.cuda.Stream()

    def bound(stream):
        return [b.ver.bind_append_kv(src[0], src[1], src[2], prep, b.kv, b.kv_len, b.off, q, stream=stream),
                b.ver.bind_chunk_attention(q, b.kv, b.kv_len, b.off, out, stream=stream),
                b.ver.bind_token_logprobs(logits, tokens, 5, lp, ent, ids, tops, stream=stream)]
    calls = bound(st)
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=st):
            for c in calls:
                c()
        graphs.append(gr)
    for i in range(6):
        for t in src + [logits]:
            t.copy_(torch.randn(t.shape, device="cuda") * (1 + i))
        for t in (q, out, lp, ent, tops):
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (q, b.k, b.v, out, lp, ent, ids, tops)]
        for c in bound(None):
            c()
        torch.cuda.synchronize()
        for g, e in zip(got, (q, b.k, b.v, out, lp, ent, ids, tops)):
            assert torch.equal(g, e)


def test_calls_between_verifications_leave_their_state():
    import torch
    hq, hkv, d, vocab = 8, 2, 128, 300
    b = Batch("bf16", hq, hkv, d, [50], [6], max_nodes=8, max_depth=5, vocab=vocab)
    parent, tokens = np.array([-1, 0, 0, 2, 3, 3], dtype=np.int32), np.arange(6, dtype=np.int32)
    logits = torch.randn(6, vocab, device="cuda").to(torch.bfloat16)
    for child, p in ((2, 0), (3, 2), (5, 3)):
        logits[p, child] = 30.0
    ver, status = b.ver, None
    _, acc, _ = ver.verify_tree(b.q, b.kv, b.kv_len, b.off, parent, tokens, logits)
    other = torch.cuda.Stream()
    out = torch.empty_like(b.q)
    with torch.cuda.stream(other):  # (a host-form call's launches may still be under way: these wait for them)
        ver.chunk_attention(b.q, b.kv, b.kv_len, b.off, out)
        ver.token_logprobs(logits, torch.tensor(tokens, device="cuda"), 4)
    other.synchronize()
    assert acc[0] == 3 and ver.get_path(1)[0].tolist() == [0, 2, 3, 5, -1, -1]
    k = b.k.clone()
    assert ver.compact_kv([b.kv], 1)[0] == 54
    torch.cuda.synchronize()
    assert torch.equal(b.k[0, 51:54], k[0, [52, 53, 55]])


def test_refusals_reach_python_and_write_nothing():
    import torch
    b = Batch("bf16", 8, 2, 64, [3], [2], max_nodes=4)
    out = torch.full_like(b.q, 9.0)
    with pytest.raises(B.CbError, match="does not fit"):
        b.ver.chunk_attention(b.q, b.kv, [400], b.off, out)
    with pytest.raises(ValueError):
        b.ver.chunk_attention(b.q.float(), b.kv, b.kv_len, b.off, out)
    with pytest.raises(ValueError):
        b.ver.chunk_attention(b.q[:1], b.kv, b.kv_len, b.off, out)
    with pytest.raises(ValueError):
        b.ver.append_kv(b.q, b.q, b.q, B.head_prep(), b.kv, b.kv_len, b.off, out)
    with pytest.raises(ValueError):
        b.ver.token_logprobs(torch.zeros(2, 99, dtype=torch.bfloat16, device="cuda"), None)
    torch.cuda.synchronize()
    assert (out == 9.0).all()
