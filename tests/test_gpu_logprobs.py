"""Log probabilities, entropies and likeliest tokens of logits rows (cb_token_logprobs_device) against a 64-bit form."""
import numpy as np
import pytest

from paper_2511_21699_amd import binding as B
from .serving_gpu import to_np
from .serving_reference import logprob_tolerance, token_logprobs

pytestmark = pytest.mark.gpu

CASES = [  # dtype, vocabulary, rows, top, elements between rows beyond the vocabulary, selected
    ("bf16", 1, 3, 1, 0, 0),
    ("bf16", 2, 2, 2, 3, 0),
    ("bf16", 31, 5, 31, 0, 0),
    ("bf16", 64, 2, 32, 1, 0),
    ("bf16", 1000, 7, 20, 0, 0),
    ("bf16", 32000, 1, 5, 0, 0),
    ("bf16", 33333, 9, 32, 0, 4),
    ("bf16", 128256, 3, 20, 8, 0),
    ("bf16", 128256, 70, 1, 0, 12),
    ("bf16", 5003, 600, 8, 5, 0),
    ("bf16", 8192, 2, 0, 0, 0),
    ("f32", 1, 1, 1, 0, 0),
    ("f32", 257, 3, 32, 2, 0),
    ("f32", 33333, 4, 20, 1, 0),
    ("f32", 128256, 2, 32, 0, 0),
    ("f32", 4097, 900, 3, 0, 50),
    ("bf16", 300000, 2, 32, 0, 0),
]


def _ver(dtype, vocab):
    return B.Verifier(B.make_config(8, 8, 64, dtype, dtype, 1, 8, 7, vocab))


def _check(x, rows, tokens, top, got):
    import torch
    torch.cuda.synchronize()
    lp, ent, ids, tops = (None if t is None else t.cpu().numpy() for t in got)
    x = to_np(x)
    for i, r in enumerate(rows):
        want = token_logprobs(x[r], int(tokens[i]) if tokens is not None else 0, top)
        assert ids[i].tolist() == want[2].tolist(), (i, r)
        tol = logprob_tolerance(want[3], want[1], x.shape[1])
        same = tops[i] == want[3].astype(np.float32)
        assert (same | (np.abs(tops[i] - np.where(same, 0, want[3])) <= tol)).all(), (i, tops[i], want[3])
        if tokens is not None and not (np.isnan(want[0]) and np.isnan(lp[i])):
            assert lp[i] == want[0] or abs(lp[i] - want[0]) <= logprob_tolerance(want[0], want[1], x.shape[1]), (i, lp[i], want[0])
        # entropy: log Z and a sum of e (max - x) over Z: as a log probability of about its size, twice
        assert abs(ent[i] - want[1]) <= 2 * logprob_tolerance(want[1], want[1], x.shape[1]), (i, ent[i], want[1])


def _logits(dtype, rows, vocab, extra, seed, scale=2.5):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, vocab + extra, generator=g, device="cuda") * scale
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)[:, :vocab]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_logprobs_against_64_bits(i):
    import torch
    dtype, vocab, rows, top, extra, selected = CASES[i]
    print(f"[case] logprobs {CASES[i]}", flush=True)
    x = _logits(dtype, rows, vocab, extra, i)
    rng = np.random.default_rng(i)
    want = rng.integers(0, rows, selected) if selected else np.arange(rows)  # (some rows twice)
    d_rows = torch.tensor(want, dtype=torch.int32, device="cuda") if selected else None
    tokens = torch.tensor(rng.integers(0, vocab, len(want)), dtype=torch.int32, device="cuda")
    got = _ver(dtype, vocab).token_logprobs(x, tokens, top, d_rows=d_rows)
    _check(x, want, tokens.cpu().numpy(), top, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [40, 9000, 40000])
def test_rows_that_select_badly(dtype, vocab):
    """Equal entries, ascending and descending rows, forbidden tokens, few allowed ones, rows of one entry's size, zeros of both signs."""
    import torch
    print(f"[case] odd rows {dtype} {vocab}", flush=True)
    x = _logits(dtype, 12, vocab, 0, 1)
    x[0] = 1.5
    x[1] = torch.arange(vocab, device="cuda") * 1e-3
    x[2] = torch.arange(vocab, 0, -1, device="cuda") * 1e-3
    x[3] = -float("inf")
    x[4] = -float("inf")
    x[4, vocab - 1] = -3.0
    x[5, ::2] = -float("inf")
    x[6] = -float("inf")
    x[6, [3, 17, 21]] = torch.tensor([1.0, 2.0, 1.0], dtype=x.dtype, device="cuda")
    x[7] *= 1000
    x[8] = 0.0
    x[8, ::3] = -0.0
    x[9] = -1e30
    x[10, :vocab // 2] = 9.0
    x[11] = torch.finfo(x.dtype).min
    tokens = torch.tensor([0, 5, 7, 1, vocab - 1, 2, 17, 3, 4, -1, vocab, 6], dtype=torch.int32, device="cuda")
    for top in (0, 1, 32):
        got = _ver(dtype, vocab).token_logprobs(x, tokens, top)
        _check(x, range(12), tokens.cpu().numpy(), top, got)


def test_parts_of_the_results_and_rows_that_do_not_exist():
    import torch
    x = _logits("bf16", 4, 5000, 0, 2)
    ver = _ver("bf16", 5000)
    lp, ent, ids, tops = ver.token_logprobs(x, torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda"), 2, d_rows=torch.tensor([2, -1, 4], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert lp.isnan().tolist() == [False, True, True] and ent.isnan().tolist() == [False, True, True]
    assert ids[1:].tolist() == [[-1, -1], [-1, -1]] and tops[1:].isnan().all()
    only = torch.empty(4, device="cuda")
    ver.bind_token_logprobs(x, None, 0, None, only)()
    torch.cuda.synchronize()
    assert torch.equal(only, ver.token_logprobs(x, None, 3)[1])
    nothing = ver.token_logprobs(x[:0], torch.empty(0, dtype=torch.int32, device="cuda"), 2)
    assert nothing[0].numel() == 0
    # rows that are not numbers: indices stay inside the vocabulary
    x[0, 7], x[1, 9], x[2] = float("nan"), float("inf"), float("nan")
    ids = ver.token_logprobs(x, None, 32)[2]
    torch.cuda.synchronize()
    assert ((ids >= 0) & (ids < 5000)).all()


def test_the_same_row_gives_the_same_bits_wherever_it_stands():
    import torch
    x = _logits("f32", 1, 40000, 0, 4)
    ver = _ver("f32", 40000)
    one = ver.token_logprobs(x, torch.zeros(1, dtype=torch.int32, device="cuda"), 7)
    again = ver.token_logprobs(x, torch.zeros(1, dtype=torch.int32, device="cuda"), 7)
    torch.cuda.synchronize()
    for a, b in zip(one, again):
        assert torch.equal(a, b)
