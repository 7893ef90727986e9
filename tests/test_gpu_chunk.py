"""Attention of a chunk of new tokens over the cache (cb_chunk_attention_device) against a 64-bit form."""
import math

import numpy as np
import pytest

from paper_2511_21699_amd import binding as B
from .serving_gpu import Batch, to_np
from .serving_reference import attention_tolerance, chunk_attention

pytestmark = pytest.mark.gpu

TM, HM = B.CB_LAYOUT_TOKEN_MAJOR, B.CB_LAYOUT_HEAD_MAJOR
CASES = [  # dtype, heads, kv heads, head_dim, prefixes, new tokens, block, layout, scale of the queries
    ("bf16", 32, 8, 128, [0], [1], 0, TM, 1.0),                       # the first token of all
    ("bf16", 32, 8, 128, [1000], [1], 0, TM, 4.0),
    ("bf16", 8, 8, 128, [31, 32, 33], [1, 1, 1], 16, TM, 2.0),
    ("bf16", 32, 8, 128, [0, 700, 0, 5, 64], [1, 1, 0, 2, 1], 16, HM, 2.0),  # one sequence has nothing new
    ("bf16", 8, 1, 128, [4000], [3], 16, TM, 1.0),                    # one kv head: split over the keys
    ("bf16", 4, 4, 128, [0], [257], 0, TM, 2.0),
    ("bf16", 32, 8, 128, [0], [130], 0, HM, 2.0),
    ("bf16", 8, 2, 128, [95, 0, 33], [64, 200, 31], 16, TM, 2.0),
    ("bf16", 10, 2, 128, [77], [103], 0, TM, 2.0),                    # five heads to a kv head: rows of a tile share tokens unevenly
    ("bf16", 6, 3, 128, [129], [300], 1, TM, 2.0),                    # one token to a block
    ("bf16", 8, 8, 64, [500], [1], 16, TM, 2.0),
    ("bf16", 32, 8, 64, [0, 300, 1500], [90, 1, 33], 16, TM, 2.0),
    ("bf16", 4, 2, 64, [10], [520], 0, HM, 2.0),
    ("bf16", 4, 2, 64, [40], [70], 24, TM, 2.0),                      # blocks that are no power of two
    ("bf16", 8, 4, 128, [40, 3], [70, 1], 48, HM, 2.0),
    ("f32", 8, 8, 64, [256], [15], 0, TM, 2.0),
    ("f32", 16, 8, 128, [0, 333, 20], [40, 1, 0], 16, TM, 2.0),
    ("f32", 6, 2, 128, [0], [211], 0, HM, 2.0),
    ("f32", 8, 1, 64, [3000], [2], 12, TM, 1.0),
    ("f32", 4, 4, 128, [17], [150], 64, TM, 2.0),
]


def _check(b, out, first=0):
    d = b.d
    want, size, score = chunk_attention(to_np(b.q), b.keys(), b.values(), b.kv_len.tolist(), b.off.tolist(), 1 / math.sqrt(d))
    tol = attention_tolerance(b.dtype, want, size, score, max(int(a) + c for a, c in zip(b.kv_len, b.new)), d)
    got = to_np(out)[:b.n]
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(), float(np.nanmax(np.abs(got - want) / tol)))


@pytest.mark.parametrize("i", range(len(CASES)))
def test_chunk_attention_against_64_bits(i):
    import torch
    dtype, hq, hkv, d, lens, new, block, layout, scale = CASES[i]
    print(f"[case] chunk {CASES[i]}", flush=True)
    b = Batch(dtype, hq, hkv, d, lens, new, block, layout, seed=i, scale=scale)
    out = torch.full((b.n + 3, hq, d), 55.0, dtype=b.t, device="cuda")
    b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off, out)
    torch.cuda.synchronize()
    _check(b, out)
    assert (out[b.n:] == 55.0).all()
    again = b.q.clone()  # in place, and in another call of the same context
    b.ver.chunk_attention(again, b.kv, b.kv_len, b.off, again)
    torch.cuda.synchronize()
    assert torch.equal(again, out[:b.n])


TILES = [  # the kernels and their split merges, whatever the planner would take: dtype, heads, kv heads, head_dim, prefixes, new tokens, block
    ("bf16", 8, 2, 128, [95, 0, 700], [70, 200, 3], 16),
    ("bf16", 6, 6, 128, [33], [530], 0),
    ("bf16", 10, 2, 64, [0, 1111], [150, 1], 1),
    ("bf16", 4, 4, 64, [64], [400], 0),
    ("f32", 8, 2, 128, [95, 0, 300], [20, 60, 1], 16),
    ("f32", 6, 3, 64, [10], [90], 0),
]


@pytest.mark.parametrize("case", TILES)
@pytest.mark.parametrize("rows", [64, 128, 256])
@pytest.mark.parametrize("splits, coop", [(1, 1), (2, 1), (3, 0), (7, 1), (8, 0)])
def test_every_tile_and_split(case, rows, splits, coop):
    import torch
    print(f"[case] tiles {case} {rows} {splits} {coop}", flush=True)
    dtype, hq, hkv, d, lens, new, block = case
    b = Batch(dtype, hq, hkv, d, lens, new, block, seed=rows + splits, scale=2.0)
    for name, value in (("tile_rows", rows), ("splits", splits), ("coop_merge", coop)):
        b.ver.set_option(name, value)
    out = torch.full((b.n + 1, hq, d), 55.0, dtype=b.t, device="cuda")
    for _ in range(2):
        b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off, out)
        torch.cuda.synchronize()
        _check(b, out)
        assert (out[b.n:] == 55.0).all()
        out[:b.n] = 0
    t = new[0] - 1  # the first sequence's last token holds anything: nobody else sees it
    clean = b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off)
    if t > 0:
        b.put(0, int(lens[0]) + t, torch.full((1, hkv, d), float("nan"), dtype=b.t, device="cuda"), torch.full((1, hkv, d), float("inf"), dtype=b.t, device="cuda"))
        odd = b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off)
        torch.cuda.synchronize()
        assert torch.equal(odd[:t], clean[:t]) and torch.equal(odd[t + 1:], clean[t + 1:])
        assert odd[t].isnan().all()


@pytest.mark.parametrize("dtype, d, hq, hkv, s, n", [("bf16", 128, 8, 2, 20, 90), ("bf16", 64, 4, 4, 3, 300), ("f32", 128, 4, 2, 40, 50), ("bf16", 128, 4, 4, 600, 40)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_what_a_token_must_not_see_can_hold_anything(dtype, d, hq, hkv, s, n, what):
    """Earlier tokens' results do not depend on later tokens' K and V."""
    import torch
    print(f"[case] hidden {dtype} {d} {hq}/{hkv} {s}+{n} {what}", flush=True)
    b = Batch(dtype, hq, hkv, d, [s], [n], seed=3, scale=2.0)
    clean = b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off)
    for t in (n - 1, n // 2, 1):
        b.k[0, s + t, :, ::3] = what
        b.v[0, s + t, :, 1::5] = what
        got = b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off)
        torch.cuda.synchronize()
        assert torch.equal(got[:t], clean[:t])


@pytest.mark.parametrize("dtype, d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_values_that_a_token_sees_come_through(dtype, d):
    """An infinite value of a token reaches that token and later ones, and no others."""
    import torch
    b = Batch(dtype, 4, 2, d, [7], [60], seed=5)
    clean = b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off)
    b.v[0, 7 + 30, 1, 5] = float("inf")
    got = b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off)
    torch.cuda.synchronize()
    assert torch.equal(got[:30], clean[:30])
    assert torch.equal(got[:, :2], clean[:, :2])
    assert (got[30:, 2:, 5] == float("inf")).all()
    rest = [i for i in range(d) if i != 5]
    assert torch.equal(got[:, :, rest], clean[:, :, rest])


def test_scores_far_apart():
    """A row whose largest score comes last, a row of equal scores, and scores that differ by thousands."""
    import torch
    b = Batch("bf16", 4, 4, 128, [500], [40], seed=9, scale=30.0)
    b.k[0, 520] *= 20
    b.k[0, 100:140] = 0
    b.q[3] = 0
    out = b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off)
    torch.cuda.synchronize()
    _check(b, out)


def test_long_caches_and_far_slots():
    """Slots beyond 32-bit offsets: one sequence's slice of a cache of more than 4 GiB."""
    import torch
    heads, d, s = 32, 128, 600000
    k, v = (torch.zeros(1, s + 8, heads, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = torch.Generator().manual_seed(1)
    new = [torch.randn(3, heads, d, generator=g).to(torch.bfloat16).cuda() for _ in range(3)]
    ver = B.Verifier(B.make_config(heads, heads, d, "bf16", "bf16", 1, 8, 7, 10))
    kv = B.kv_layer(k, v)
    out, q = torch.empty_like(new[0]), torch.empty_like(new[0])
    ver.append_kv(new[0], new[1], new[2], B.head_prep(), kv, [s], [0, 3], q)
    ver.chunk_attention(q, kv, [s], [0, 3], out)
    torch.cuda.synchronize()
    assert torch.equal(k[0, s:s + 3], new[1]) and torch.equal(v[0, s:s + 3], new[2])
    # the prefix's keys are zero: they weigh e^0 each
    x = (new[0].float()[:, None] * new[1].float()[None]).sum(-1).cpu().numpy().astype(np.float64) / math.sqrt(d)  # [query, key, head]
    p = np.exp(x) * np.tril(np.ones((3, 3)))[:, :, None]
    want = np.einsum("qkh,khd->qhd", p, to_np(new[2]).astype(np.float64)) / (s + p.sum(1))[:, :, None]
    size = np.einsum("qkh,khd->qhd", p, np.abs(to_np(new[2])).astype(np.float64)) / (s + p.sum(1))[:, :, None]
    # (the denominator's 600000 additions of ones in 32 bits, 16 keys to an accumulation: exact below 2^24)
    assert (np.abs(to_np(out) - want) <= 2 ** -5 * size + 1e-12).all()


@pytest.mark.parametrize("dtype, hq, hkv, d", [("bf16", 8, 2, 128), ("bf16", 8, 4, 64), ("f32", 4, 2, 128)])
@pytest.mark.parametrize("block", [1, 2, 16])
@pytest.mark.parametrize("rows, splits", [(64, 1), (128, 2), (256, 1)])
def test_long_block_tables(dtype, hq, hkv, d, block, rows, splits):
    """More table entries than are kept at a time, and entries behind a sequence's last block that mean nothing."""
    import torch
    print(f"[case] tables {dtype} {hq}/{hkv} d{d} block {block} rows {rows} splits {splits}", flush=True)
    b = Batch(dtype, hq, hkv, d, [5000, 17, 2900], [50, 1, 90], block, seed=block)
    for i in range(3):
        used = (int(b.kv_len[i]) + b.new[i] + block - 1) // block
        b.table[i, used:] = torch.tensor([-7, 2**31 - 1, 2**20], dtype=torch.int32, device="cuda").repeat(b.table.shape[1])[:b.table.shape[1] - used]
    b.ver.set_option("tile_rows", rows)
    b.ver.set_option("splits", splits)
    out = b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off)
    torch.cuda.synchronize()
    _check(b, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_splits", [1, 0])
def test_a_small_workspace_takes_any_chunk(dtype, max_splits):
    """max_nodes 1: chunks of any length all the same; 64 sequences, some with nothing new."""
    import torch
    lens, new = [(97 * i) % 600 for i in range(64)], [(0, 1, 1, 5, 70)[i % 5] for i in range(64)]
    b = Batch(dtype, 8, 2, 64, lens, new, 16, seed=2, max_nodes=1, max_depth=1, max_splits=max_splits)
    out = b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off)
    torch.cuda.synchronize()
    _check(b, out)


def test_two_contexts_on_two_streams():
    """Launches whose tiles' workgroups wait for each other, from two contexts at once."""
    import torch
    bs = [Batch("bf16", 32, 8, 128, [4000], [1], 16, seed=s, scale=2.0) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in bs]
    outs = [torch.empty_like(b.q) for b in bs]
    calls = [b.ver.bind_chunk_attention(b.q, b.kv, b.kv_len, b.off, o, stream=st) for b, o, st in zip(bs, outs, streams)]
    torch.cuda.synchronize()
    for _ in range(20):
        for c in calls:
            c()
    torch.cuda.synchronize()
    for b, o in zip(bs, outs):
        _check(b, o)


@pytest.mark.parametrize("splits", [1, 4])
def test_heads_and_batches_that_fill_no_tile(splits):
    """16 heads to a kv head, and a batch of 64 single tokens beside two longer chunks."""
    import torch
    b = Batch("bf16", 16, 1, 128, [300 + 41 * i for i in range(62)] + [0, 1000], [1] * 62 + [33, 20], 16, seed=4, scale=2.0)
    b.ver.set_option("splits", splits)
    out = b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off)
    torch.cuda.synchronize()
    _check(b, out)
