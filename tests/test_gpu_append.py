"""New tokens into the cache (cb_append_kv_device): norm, rotation and slots against a 64-bit form."""
import numpy as np
import pytest

from paper_2511_21699_amd import binding as B
from .serving_gpu import Batch, to_np
from .serving_reference import HALF_STEP, depths, prepared

pytestmark = pytest.mark.gpu

TM, HM = B.CB_LAYOUT_TOKEN_MAJOR, B.CB_LAYOUT_HEAD_MAJOR
CASES = [  # dtype, heads, kv heads, head_dim, prefixes, new tokens, block, layout, norm, rotary, interleaved, tree
    ("bf16", 32, 8, 128, [0], [1], 0, TM, True, 128, False, False),
    ("bf16", 32, 8, 128, [100, 0, 17, 5], [1, 1, 0, 1], 16, TM, True, 128, False, False),
    ("bf16", 32, 8, 128, [15, 31, 2], [40, 1, 17], 16, HM, True, 64, False, False),
    ("bf16", 40, 40, 128, [7], [13], 0, HM, True, 128, True, False),
    ("bf16", 6, 3, 64, [0, 9], [33, 0], 4, TM, True, 32, True, False),
    ("bf16", 8, 8, 64, [1], [5], 0, TM, False, 16, False, False),
    ("bf16", 5, 1, 64, [3], [70], 48, TM, True, 48, False, False),          # blocks that are no power of two
    ("bf16", 32, 8, 128, [2000], [300], 64, TM, True, 112, False, False),
    ("bf16", 8, 2, 128, [10], [21], 0, TM, True, 0, False, False),
    ("f32", 8, 8, 64, [256], [15], 0, TM, False, 64, True, True),
    ("f32", 16, 8, 128, [33, 0, 70000], [40, 3, 9], 16, TM, True, 128, False, False),
    ("f32", 3, 3, 128, [1], [3], 0, HM, True, 96, True, False),
    ("bf16", 32, 8, 128, [60001], [64], 0, TM, True, 64, False, True),
    ("bf16", 16, 4, 64, [5, 100, 0], [256, 1, 63], 16, HM, True, 64, False, True),
    ("f32", 8, 4, 64, [0, 3], [0, 200], 0, TM, True, 32, False, True),
]


def _parents(rng, n, kind):
    if kind == "chain":
        return [i - 1 for i in range(n)]
    return [-1 if i == 0 else int(rng.integers(max(0, i - 9), i)) for i in range(n)]


def _run(i, q_in_place=False, kind="random"):
    import torch
    dtype, hq, hkv, d, lens, new, block, layout, norm, rotary, inter, tree = CASES[i]
    print(f"[case] append {CASES[i]}", flush=True)
    b = Batch(dtype, hq, hkv, d, lens, new, block, layout, seed=i, max_nodes=256, max_depth=255)
    rng = np.random.default_rng(i)
    par = [_parents(rng, n, kind) for n in new]
    parent = torch.tensor([p for x in par for p in x], dtype=torch.int32, device="cuda") if tree else None
    pos = [s + x for s, n, p in zip(lens, new, par) for x in (depths(p) if tree else range(n))]
    qkv = b.draw(b.n + 2, (hq + 2 * hkv) * d)  # (two rows more than there are tokens)
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hkv * d, hkv * d], 1))
    out = torch.full((b.n + 2, hq, d), 77.0, dtype=b.t, device="cuda")
    if q_in_place:
        out[:b.n + 2] = q
        q = out
    w = [torch.randn(d, device="cuda") + 1 if norm else None for _ in range(2)]
    freq = (1e4 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / max(rotary, 1))).float().cuda() if rotary else None
    want_q, size_q = prepared(to_np(q)[:b.n], None if w[0] is None else to_np(w[0]), 1e-5, None if freq is None else freq.cpu().numpy(), inter, pos)
    want_k, size_k = prepared(to_np(k)[:b.n], None if w[1] is None else to_np(w[1]), 1e-5, None if freq is None else freq.cpu().numpy(), inter, pos)
    before, tail = (b.k.clone(), b.v.clone()), to_np(out[b.n:])
    b.ver.append_kv(q, k, v, B.head_prep(w[0], w[1], 1e-5, freq, inter), b.kv, b.kv_len, b.off, out, d_parent=parent)
    torch.cuda.synchronize()
    # A result is the pair's elements times norm and angle factors in 32 bits, some of them off by a few steps each (sum of D squares,
    # root and reciprocal, weight, sine and cosine of a reduced angle: less than 64 half steps of the pair's size), and one rounding.
    far = lambda got, want, size: np.abs(got - want) <= HALF_STEP[dtype] * np.abs(want) + 64 * 2.0 ** -24 * size  # noqa: E731
    assert far(to_np(out)[:b.n], want_q, size_q).all()
    assert np.array_equal(to_np(out[b.n:]), tail)
    for s in range(len(new)):
        at = b.index(s, lens[s], new[s])
        assert far(to_np(b.k[at]), want_k[b.off[s]:b.off[s + 1]], size_k[b.off[s]:b.off[s + 1]]).all()
        assert torch.equal(b.v[at], v[b.off[s]:b.off[s + 1]])
        before[0][at], before[1][at] = b.k[at], b.v[at]
    for got, was in zip((b.k, b.v), before):  # every other slot is as it was
        assert torch.equal(got.view(torch.int16 if dtype == "bf16" else torch.int32), was.view(torch.int16 if dtype == "bf16" else torch.int32))
    assert b.ver.device_status() == 0


@pytest.mark.parametrize("i", range(len(CASES)))
def test_append_against_64_bits(i):
    _run(i)


def test_append_queries_in_place_and_deep_trees():
    _run(2, q_in_place=True)
    _run(13, kind="chain")


def test_append_keys_and_values_only():
    import torch
    b = Batch("bf16", 8, 2, 64, [3], [4], max_nodes=8)
    k, v = b.draw(4, 2, 64), b.draw(4, 2, 64)
    b.ver.append_kv(None, k, v, B.head_prep(), b.kv, b.kv_len, b.off, None)
    torch.cuda.synchronize()
    assert torch.equal(b.k[0, 3:7], k) and torch.equal(b.v[0, 3:7], v)


def test_append_leaves_out_pages_outside_the_pool_and_repairs_trees():
    import torch
    b = Batch("bf16", 8, 2, 64, [14, 14], [4, 4], block=16, max_nodes=8)
    b.table[1, 1] = b.k.shape[0] + 3
    b.table[0, 1] = -2
    b.k.zero_()
    b.v.zero_()
    k, v, out = b.draw(8, 2, 64), b.draw(8, 2, 64), torch.empty_like(b.q)
    b.ver.append_kv(b.q, k, v, B.head_prep(), b.kv, b.kv_len, b.off, out)
    assert b.ver.device_status() == 64
    assert torch.equal(out, b.q)
    for s in range(2):  # slots 14 and 15 are in a good page, 16 and 17 are not
        assert torch.equal(b.k[b.table[s, 0].long(), 14:16], k[4 * s:4 * s + 2])
    assert int((b.k != 0).any(-1).any(-1).sum()) == 4 and int((b.v != 0).any(-1).any(-1).sum()) == 4
    # a parent that is not an earlier node is the root
    b = Batch("f32", 1, 1, 64, [9], [4], max_nodes=8)
    k, out = b.draw(4, 1, 64), torch.empty_like(b.q)
    freq = torch.full((8,), 0.25, device="cuda")
    b.ver.append_kv(b.q, k, k, B.head_prep(inv_freq=freq), b.kv, b.kv_len, b.off, out, d_parent=torch.tensor([-1, 0, 5, 1], dtype=torch.int32, device="cuda"))
    assert b.ver.device_status() == 1
    want, size = prepared(to_np(b.q), None, 0, [0.25] * 8, False, [9, 10, 10, 11])
    assert (np.abs(to_np(out) - want) <= 64 * 2.0 ** -24 * size).all()
