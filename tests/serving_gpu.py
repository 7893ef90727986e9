"""Batches on the GPU for the tests of the calls around the verification."""
import numpy as np

from paper_2511_21699_amd import binding as B


def to_np(t):
    return t.detach().float().cpu().numpy()


class Batch:
    """Sequences of a cache, contiguous (block 0) or paged with shuffled pages, and their new tokens.  Slots that no sequence has hold NaN."""

    def __init__(self, dtype, hq, hkv, d, kv_len, new, block=0, layout=B.CB_LAYOUT_TOKEN_MAJOR, seed=0, spare=5, scale=1.0, max_nodes=64, max_depth=63, vocab=100, nan=True,
                 max_splits=0):
        import torch
        self.dtype, self.hq, self.hkv, self.d, self.block, self.layout = dtype, hq, hkv, d, block, layout
        self.kv_len, self.new = np.array(kv_len, dtype=np.int32), list(new)
        self.off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.n, batch = int(self.off[-1]), len(kv_len)
        self.t = torch.float32 if dtype == "f32" else torch.bfloat16
        g = torch.Generator().manual_seed(seed)
        self.draw = lambda *size, s=1.0: (torch.randn(*size, generator=g) * s).to(self.t).cuda()
        longest = max(int(a) + b for a, b in zip(kv_len, new))
        if block:
            per = (longest + block - 1) // block + 1
            units, tokens = batch * per + spare, block
            self.table = torch.randperm(units, generator=g)[:batch * per].view(batch, per).to(torch.int32).cuda()
        else:
            units, tokens, self.table = batch, longest + spare, None
        size = (units, hkv, tokens, d) if layout == B.CB_LAYOUT_HEAD_MAJOR else (units, tokens, hkv, d)
        fill = float("nan") if nan else 0.0
        self.k, self.v = torch.full(size, fill, dtype=self.t, device="cuda"), torch.full(size, fill, dtype=self.t, device="cuda")
        for b in range(batch):
            n = int(kv_len[b]) + new[b]
            self.put(b, 0, self.draw(n, hkv, d), self.draw(n, hkv, d))
        self.q = self.draw(self.n, hq, d, s=scale)
        self.kv = B.kv_layer(self.k, self.v, self.table, layout, paged=block > 0)
        self.cfg = B.make_config(hq, hkv, d, dtype, dtype, batch, max_nodes, max_depth, vocab, block, max_splits)
        self.ver = B.Verifier(self.cfg)

    def index(self, b, first, n):
        import torch
        slots = torch.arange(first, first + n, device="cuda")
        unit = self.table[b].long()[slots // self.block] if self.block else torch.full((n,), b, device="cuda")
        at = slots % self.block if self.block else slots
        return (unit, slice(None), at) if self.layout == B.CB_LAYOUT_HEAD_MAJOR else (unit, at)

    def put(self, b, first, k, v):
        if len(k):
            self.k[self.index(b, first, len(k))], self.v[self.index(b, first, len(k))] = k, v

    def rows(self, cache, b, n=None):
        """[slots, Hkv, D] of a sequence as float32 on the host."""
        n = int(self.kv_len[b]) + self.new[b] if n is None else n
        return to_np(cache[self.index(b, 0, n)])

    def keys(self):
        return [self.rows(self.k, b) for b in range(len(self.new))]

    def values(self):
        return [self.rows(self.v, b) for b in range(len(self.new))]
