"""Attention of a chunk over the cache (cb_chunk_attention_device) where inputs are no numbers: who may see it, and who may not."""
import pytest

from .serving_gpu import Batch

pytestmark = pytest.mark.gpu

WHAT = [float("nan"), float("inf"), -float("inf")]


def _options(b, rows=0, splits=0, coop=1):
    for name, value in (("tile_rows", rows), ("splits", splits), ("coop_merge", coop)):
        b.ver.set_option(name, value)


def _attend(b):
    import torch
    out = b.ver.chunk_attention(b.q, b.kv, b.kv_len, b.off)
    torch.cuda.synchronize()
    return out


def _spoil_queries(b, at):
    """One head's query of one token: its own row is no number, and every other row is the same to the bit.  (An infinite entry gives scores of
    both infinities over a few random keys, whose softmax is no number either.)"""
    import torch
    clean, kept = _attend(b), b.q.clone()
    assert not clean.isnan().any()
    for token, head in at:
        for what in WHAT:
            b.q[token, head, 3] = what
            got = _attend(b)
            b.q.copy_(kept)
            assert got[token, head].isnan().all(), (token, head, what)
            got[token, head] = clean[token, head]
            assert torch.equal(got, clean), (token, head, what, (got != clean).any(-1).nonzero()[:4].tolist())


@pytest.mark.parametrize("dtype, d, rows", [("bf16", 128, 64), ("bf16", 128, 128), ("bf16", 128, 256), ("bf16", 64, 64), ("bf16", 64, 128), ("f32", 128, 0)])
@pytest.mark.parametrize("hq, hkv", [(2, 2), (8, 2), (16, 1)])
@pytest.mark.parametrize("splits, coop", [(1, 1), (3, 1), (8, 1), (8, 0)])
def test_a_query_that_is_no_number_spoils_its_own_row_alone(dtype, d, rows, hq, hkv, splits, coop):
    print(f"[case] odd query {dtype} {d} {rows} {hq}/{hkv} {splits} {coop}", flush=True)
    b = Batch(dtype, hq, hkv, d, [700, 90], [45, 1], 16, seed=splits, scale=2.0)
    _options(b, rows, splits, coop)
    _spoil_queries(b, [(44, hq - 1), (21, 0), (45, hq - 1)])


@pytest.mark.parametrize("hq, hkv, d, kv_len, new, block", [(32, 8, 128, [4000], [3], 16), (32, 8, 128, [2500], [1], 0), (32, 32, 128, [0], [300], 0),
                                                            (32, 8, 128, [9000], [256], 16), (32, 8, 64, [3000, 0], [100, 33], 16)])
def test_odd_queries_with_the_plans_own_tiles(hq, hkv, d, kv_len, new, block):
    b = Batch("bf16", hq, hkv, d, kv_len, new, block, seed=1, scale=2.0)
    _spoil_queries(b, [(new[0] - 1, hq - 1), (new[0] // 2, hq // 2)])


TILES = [("bf16", 128, 64), ("bf16", 128, 128), ("bf16", 128, 256), ("bf16", 64, 64), ("bf16", 64, 128), ("f32", 128, 0), ("f32", 64, 0)]


def _spoil_value(b, slot, seen_from, what):
    """One entry of one value, of the sequence's kv head 1: rows from token seen_from on see it, whatever its weight; returns theirs."""
    import torch
    clean = _attend(b)
    kept = b.v[0, slot, 1, 5].clone()
    b.v[0, slot, 1, 5] = what
    got = _attend(b)
    b.v[0, slot, 1, 5] = kept
    g = b.hq // b.hkv
    rows = got[seen_from:b.new[0], g:2 * g, 5].clone()
    got[seen_from:b.new[0], g:2 * g, 5] = clean[seen_from:b.new[0], g:2 * g, 5]
    assert not clean.isnan().any() and torch.equal(got, clean)
    return rows


@pytest.mark.parametrize("dtype, d, rows", TILES)
@pytest.mark.parametrize("splits", [1, 3])
def test_values_come_through_whatever_their_weight(dtype, d, rows, splits):
    """Scores hundreds apart: the weights of most values that a token sees are 0 in 32 bits, and in the formula they are not."""
    print(f"[case] odd weightless value {dtype} {d} {rows} {splits}", flush=True)
    b = Batch(dtype, 8, 2, d, [70], [60], seed=7, scale=100.0)
    _options(b, rows, splits)
    for what in WHAT:
        for t in (0, 20, 59):
            assert not _spoil_value(b, 70 + t, t, what).isfinite().any(), (what, t)


@pytest.mark.parametrize("dtype, d, rows", TILES)
@pytest.mark.parametrize("kv_len, new, splits, slot", [(40, 1, 1, 40), (95, 1, 1, 95), (700, 1, 0, 700), (287, 1, 3, 95), (1000, 2, 2, 511), (70, 60, 3, 33)])
def test_the_last_value_of_a_split_comes_through(dtype, d, rows, kv_len, new, splits, slot):
    """The places behind a split's last key repeat it, with weight 0."""
    print(f"[case] odd last value {dtype} {d} {rows} {kv_len}+{new} {splits} {slot}", flush=True)
    b = Batch(dtype, 8, 2, d, [kv_len], [new], 16, seed=8)
    _options(b, rows, splits)
    b.v = b.v.view(-1, b.hkv, d)  # (a slot of the cache is a row)
    at = int(b.table[0, slot // 16]) * 16 + slot % 16
    import torch
    clean, kept = _attend(b), b.v[at, 1, 5].clone()
    for what in WHAT:
        b.v[at, 1, 5] = what
        got = _attend(b)
        mine = got[max(0, slot - kv_len):, 4:8, 5]
        assert (mine.isnan() if what != what else mine == what).all(), what
        mine.copy_(clean[max(0, slot - kv_len):, 4:8, 5])
        assert torch.equal(got, clean), what
    b.v[at, 1, 5] = kept
