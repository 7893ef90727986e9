"""Log probabilities (cb_token_logprobs_device) of many rows, of one row in many places, with errors counted from the kernel's own sums."""
import math

import numpy as np
import pytest

from paper_2511_21699_amd import binding as B
from .serving_gpu import to_np
from .serving_reference import token_logprobs

pytestmark = pytest.mark.gpu

F = 2.0 ** -24  # half a step in 32 bits


def _tolerances(x, token, top):
    """What the log probabilities of the token and of the top ones and the entropy may be off by, of one row.

    With d = max - x and weights p: an exponential of d in one or several factors has its argument rounded twice and is off by a step itself, 2 d + 2
    half steps; a lane has at most T = vocab / 64 entries, so that many additions, and for every 16 of them a change of reference (three roundings to Z, six
    to the sum of e d); lanes, wavefronts and parts are joined in fewer than 64 roundings.  A logarithm is off by two steps of its size, and one near 1 by
    a step of the argument."""
    x = np.asarray(x, dtype=np.float64)
    d = x.max() - x
    e = np.exp(-d)
    p, lz = e / e.sum(), math.log(e.sum())
    d = np.where(p > 0, d, 0.0)
    t = -(-len(x) // 64)
    mean = float((p * d).sum())
    z = F * (2 * mean + 2 + t * (1 + 3 / 16) + 64) + 4 * F * lz + 2 * F
    at = lambda i: z + F * (2 * abs(x[i] - x.max()) + lz)  # noqa: E731
    entropy = z + F * (float((p * d * (2 * d + 4)).sum()) + (t * (1 + 6 / 16) + 64) * mean) + mean * (z + 2 * F) + F * (mean + lz)
    return at(token), entropy, np.array([at(i) for i in top])


def _check(x, rows, tokens, top, got):
    """x: float rows by their number."""
    lp, ent, ids, tops = (t.cpu().numpy() for t in got)
    for i, r in rows:
        want = token_logprobs(x[r], int(tokens[i]), top)
        tol = _tolerances(x[r], int(tokens[i]), want[2])
        assert ids[i].tolist() == want[2].tolist(), (i, r)
        assert abs(lp[i] - want[0]) <= tol[0] and abs(ent[i] - want[1]) <= tol[1] and (np.abs(tops[i] - want[3]) <= tol[2]).all(), (
            i, r, abs(lp[i] - want[0]) / tol[0], abs(ent[i] - want[1]) / tol[1])


def _logits(dtype, rows, vocab, seed, extra=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, vocab + extra, generator=g, device="cuda") * 2.5
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)[:, :vocab]


def _ver(dtype, vocab):
    return B.Verifier(B.make_config(8, 8, 64, dtype, dtype, 1, 8, 7, vocab))


MANY = [  # dtype, vocabulary, rows, top: one, two, four wavefronts to a row, and eight
    ("f32", 1000, 2000, 5), ("bf16", 1000, 2000, 32),
    ("f32", 33333, 1100, 1), ("bf16", 33333, 1100, 20), ("f32", 3000, 500, 32), ("f32", 3000, 1030, 0), ("bf16", 128256, 1024, 8),
    ("f32", 40000, 400, 20), ("bf16", 40000, 400, 32), ("f32", 128256, 385, 5), ("bf16", 20000, 1023, 1),
    ("f32", 40000, 300, 8), ("bf16", 128256, 130, 20), ("f32", 128256, 129, 0),
]


@pytest.mark.parametrize("i", range(len(MANY)))
def test_many_rows(i):
    import torch
    dtype, vocab, rows, top = MANY[i]
    print(f"[case] many rows {MANY[i]}", flush=True)
    x = _logits(dtype, rows, vocab, i)
    rng = np.random.default_rng(i)
    tokens = torch.tensor(rng.integers(0, vocab, rows), dtype=torch.int32, device="cuda")
    got = _ver(dtype, vocab).token_logprobs(x, tokens, top)
    torch.cuda.synchronize()
    sample = sorted({0, 1, rows - 1, rows // 2, *rng.integers(0, rows, 20).tolist()})
    host = dict(zip(sample, to_np(x[torch.tensor(sample, device="cuda")])))
    _check(host, [(r, r) for r in sample], tokens.cpu().numpy(), top, got)
    assert all(not t.isnan().any() for t in got)


@pytest.mark.parametrize("dtype, vocab", [("f32", 40000), ("bf16", 128256), ("bf16", 1000)])
@pytest.mark.parametrize("n", [1, 5, 100, 300, 1100])
def test_a_row_gives_the_same_bits_at_every_place_of_a_call(dtype, vocab, n):
    """Rows of one alignment, in calls of one size: wherever the row stands, whatever stands beside it, asked for by number or in order."""
    import torch
    print(f"[case] places {dtype} {vocab} {n}", flush=True)
    x = _logits(dtype, n, vocab, 4)
    places = sorted({0, n // 3, n - 1})
    one = x[0].clone()
    for r in places:
        x[r] = one
    tokens, ver = torch.full((n,), 7, dtype=torch.int32, device="cuda"), _ver(dtype, vocab)
    plain = ver.token_logprobs(x, tokens, 7)
    x2 = _logits(dtype, 3, vocab, 5)
    x2[2] = one
    rows = torch.randint(0, 3, (n,), device="cuda", dtype=torch.int32)
    rows[torch.tensor(places, device="cuda")] = 2
    chosen = ver.token_logprobs(x2, tokens, 7, d_rows=rows)
    torch.cuda.synchronize()
    for t in (*plain, *chosen):
        for r in places:
            assert torch.equal(t[r], t[0])
    for a, b in zip(plain, chosen):
        assert torch.equal(a[0], b[0])
    _check({0: to_np(one)}, [(0, 0)], [7], 7, plain)


@pytest.mark.parametrize("dtype, vocab", [("f32", 5000), ("bf16", 33333)])
def test_alignments_and_sizes_of_a_call_differ_by_roundings(dtype, vocab):
    import torch
    x = _logits(dtype, 9, vocab, 6, extra=1)  # (a row further is an entry further from a 16-byte border)
    x[:] = x[0].clone()
    host, ver = {0: to_np(x[0])}, _ver(dtype, vocab)
    for n in (1, 2, 9):
        got = ver.token_logprobs(x[:n], torch.full((n,), 3, dtype=torch.int32, device="cuda"), 20)
        torch.cuda.synchronize()
        _check(host, [(i, 0) for i in range(n)], [3] * n, 20, got)
    rows = torch.arange(9, device="cuda", dtype=torch.int32).repeat(150)
    got = ver.token_logprobs(x, torch.full((1350,), 3, dtype=torch.int32, device="cuda"), 20, d_rows=rows)
    torch.cuda.synchronize()
    _check(host, [(i, 0) for i in (0, 1, 2, 3, 4, 5, 6, 7, 8, 1349)], [3] * 1350, 20, got)
