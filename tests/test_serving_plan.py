"""How a chunk's attention is cut up, for batches, without a GPU."""
import ctypes as C

import numpy as np
import pytest

from paper_2511_21699_amd import binding as B


@pytest.mark.parametrize("seed", range(40))
def test_a_batch_has_as_many_workgroups_as_its_tiles_have_splits(seed):
    """A sequence's splits have the longest sequence's keys, or its own where those are fewer; one with nothing new has no workgroups."""
    rng = np.random.default_rng(seed)
    g, hkv, d, dtype = int(rng.choice([1, 4, 7, 16])), int(rng.choice([1, 2, 8])), int(rng.choice([64, 128])), str(rng.choice(["bf16", "f32"]))
    batch = int(rng.integers(2, 65))
    n = [int(rng.choice([0, 1, 1, 5, 70, 300, 2000])) for _ in range(batch)]
    s = [int(rng.choice([0, 1, 100, 3000, 20000])) for _ in range(batch)]
    n[0], s[0] = 1 + int(rng.integers(300)), 20000 + 2000  # the longest
    cfg = B.make_config(g * hkv, hkv, d, dtype, dtype, batch, 64, 8, 100, 16)
    off, lens = np.concatenate([[0], np.cumsum(n)]).astype(np.int32), np.array(s, dtype=np.int32)
    ip = C.POINTER(C.c_int32)
    for rows, splits in ((0, 0), (64, 0), (128, 5), (256, 1), (0, 64)):
        plan = (C.c_int32 * 5)()
        assert B.load().cb_debug_chunk_plan(C.byref(cfg), batch, lens.ctypes.data_as(ip), off.ctypes.data_as(ip), splits, rows, plan) == B.CB_OK
        tile, most, keys, jobs, tiles = plan
        up = lambda x, y: -(-x // y)  # noqa: E731
        of = [up(a + b, min(up(a + b, 32) * 32, keys)) if b else 0 for a, b in zip(s, n)]
        assert most == max(of) and tiles == max(up(x * g, tile) for x in n)
        assert jobs == sum(up(b * g, tile) * hkv * x for b, x in zip(n, of))
