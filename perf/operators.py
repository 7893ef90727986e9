"""What a serving program does around the verification of draft trees, as timed cases: tokens go into the cache with their query and key
heads normalised and rotated ("append"), a chunk of new tokens attends over the cache ("attend"), and tokens get their log
probabilities ("logprob").

A case is a dict of plain values.

  op              "append", "attend" or "logprob"               dtype           "bf16" / "f32" of all tensors
  append and attend:
  hq, hkv, d      query heads, kv heads, head dimension         batch           sequences
  s_lo, s_hi      range of their cached prefixes                n_lo, n_hi      range of their new tokens
  lengths         fixes the lengths (and trees) in the ranges   block           0 contiguous cache, else tokens per block
  head_major      cache layout
  append:
  tree            the tokens are draft trees, not chunks        norm            heads are normalised
  rotary          leading dims that are rotated                 interleaved     neighbouring dims are pairs, not halves
  theta           base of the rotation's frequencies
  logprob:
  rows, vocab     of the logits                                 selected        0, or how many of the rows are asked for
  top             alternatives to each token
"""
import math
import random

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-6

_APPEND = dict(op="append", dtype="bf16", hq=32, hkv=8, d=128, batch=1, s_lo=0, s_hi=0, n_lo=1, n_hi=1, lengths=0, block=0, head_major=False,
               tree=False, norm=True, rotary=128, interleaved=False, theta=1e6)
_ATTEND = dict(op="attend", dtype="bf16", hq=32, hkv=8, d=128, batch=1, s_lo=0, s_hi=0, n_lo=1, n_hi=1, lengths=0, block=0, head_major=False)
_LOGPROB = dict(op="logprob", dtype="bf16", rows=1, vocab=32000, selected=0, top=5)


def listed():
    return [
        # the smallest: a small fp32 model's draft tree, as runs that compare implementations have it; rotation of neighbours, no norm
        dict(_APPEND, name="append_tree_f32", dtype="f32", hq=8, hkv=8, d=64, s_lo=256, s_hi=256, n_lo=15, n_hi=15, tree=True, norm=False, rotary=64,
             interleaved=True, theta=1e4),
        # a serving batch's ordinary step: one token of each sequence into a paged cache
        dict(_APPEND, name="append_step", batch=16, s_lo=100, s_hi=2000, lengths=1, block=16),
        # a draft tree far into a long document, half of every head rotated
        dict(_APPEND, name="append_tree_far", s_lo=60001, s_hi=60001, n_lo=64, n_hi=64, tree=True, rotary=64),
        # a long prompt
        dict(_APPEND, name="append_prompt", hkv=32, n_lo=8192, n_hi=8192),
        # the smallest: fp32, the beginning of a request
        dict(_ATTEND, name="attend_f32", dtype="f32", hq=8, hkv=8, d=64, s_lo=256, s_hi=256, n_lo=15, n_hi=15),
        # a serving batch's ordinary step over a paged cache, lengths spread widely
        dict(_ATTEND, name="attend_step", batch=16, s_lo=512, s_hi=16384, lengths=4, block=16),
        # a batch in which prompts of odd sizes and single tokens meet; small heads
        dict(_ATTEND, name="attend_mixed", d=64, batch=8, s_hi=3000, n_hi=700, lengths=5, block=16),
        # a prompt into an empty cache, every head with K and V of its own
        dict(_ATTEND, name="attend_prompt", hkv=32, n_lo=2048, n_hi=2048),
        # the largest: the last chunk of a long document
        dict(_ATTEND, name="attend_document", s_lo=28672, s_hi=28672, n_lo=4096, n_hi=4096, block=16),
        # one token's alternatives, as an interactive request shows them
        dict(_LOGPROB, name="logprob_token"),
        # the accepted paths of a batch of draft trees, out of all nodes' rows
        dict(_LOGPROB, name="logprob_paths", rows=256, vocab=128256, selected=40, top=20),
        # a prompt's tokens scored; rows that are not 16-byte aligned, fp32
        dict(_LOGPROB, name="logprob_prompt", dtype="f32", rows=2048, vocab=33333, top=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "logprob"])
    if op == "logprob":
        c = dict(_LOGPROB, dtype=rng.choice(["bf16", "f32"]), vocab=rng.choice([1000, 32000, 33333, 128256, _log(rng, 50, 200000)]), top=rng.choice([0, 1, 5, 20, 32]))
        c["rows"] = max(1, min(_log(rng, 1, 4096), int(7e7 / c["vocab"])))
        c["selected"] = rng.choice([0, 0, (c["rows"] + 3) // 4])
        return c
    c = dict(_APPEND if op == "append" else _ATTEND, lengths=rng.randrange(1000), block=rng.choice([0, 16, 64]), head_major=rng.random() < 0.25)
    c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
    c["hq"], c["hkv"], c["d"] = rng.choice([(8, 8, 64), (16, 8, 128), (32, 8, 128), (32, 8, 128), (32, 32, 128), (40, 40, 128), (32, 8, 64)])
    c["batch"] = 1 if rng.random() < 0.5 else _log(rng, 2, 32)
    n = 1 if rng.random() < 0.3 else _log(rng, 2, 4096)
    s = _log(rng, 1, 32768)
    if op == "append":
        c["tree"], c["norm"], c["interleaved"] = rng.random() < 0.4, rng.random() < 0.6, rng.random() < 0.3
        c["rotary"] = rng.choice([c["d"], c["d"], c["d"] // 2, 32])
        c["theta"] = rng.choice([1e4, 5e5, 1e6])
        n = min(n, 256) if c["tree"] else n
    # no more of the cache, of new tokens and of scores than the largest listed cases
    while (c["batch"] * (s + n) * c["hkv"] * c["d"] * (4 if c["dtype"] == "f32" else 2) > 3e8 or c["batch"] * n * (c["hq"] + 2 * c["hkv"]) * c["d"] > 1e8
           or (op == "attend" and c["batch"] * c["hq"] * n * (s + n) > (4e9 if c["dtype"] == "bf16" else 2e8))):
        if c["batch"] > 1:
            c["batch"] //= 2
        else:
            s, n = s * 3 // 4, max(1, n * 3 // 4)
    c["s_hi"], c["n_hi"] = s, n
    c["s_lo"] = s if c["batch"] == 1 else s // rng.choice([1, 4, 32])
    c["n_lo"] = n if c["batch"] == 1 else max(1, n // rng.choice([1, 4, 32]))
    return c


def _shape(case):
    """The sequences' cached prefixes and numbers of new tokens, and the trees' parents (-1 at roots)."""
    rng = random.Random(case["lengths"])
    spread = lambda lo, hi: lo if lo == hi else rng.choice([lo, hi, rng.randint(lo, hi), rng.randint(lo, hi)])  # noqa: E731
    s, n = [], []
    for _ in range(case["batch"]):
        s.append(spread(case["s_lo"], case["s_hi"]))
        n.append(spread(case["n_lo"], case["n_hi"]))
    s[0], n[0] = case["s_hi"], case["n_hi"]
    parent = [-1 if i == 0 else rng.randint(max(0, i - 12), i - 1) for k in n for i in range(k)] if case.get("tree") else None
    return s, n, parent


def _draw_normal(g, *size, scale=1.0):
    return torch.randn(*size, generator=g, device="cuda", dtype=torch.float32) * scale


def _cache(case, g, longest):
    """K and V of a cache that holds anything, and its block table."""
    t, h, d, block = _TYPES[case["dtype"]], case["hkv"], case["d"], case["block"]
    units, tokens, table = case["batch"], longest, None
    if block:
        per_seq = (longest + block - 1) // block
        units, tokens = case["batch"] * per_seq + 3, block
        table = torch.randperm(units, generator=g, device="cuda")[:case["batch"] * per_seq].view(case["batch"], per_seq).to(torch.int32)
    size = (units, h, tokens, d) if case["head_major"] else (units, tokens, h, d)
    k, v = _draw_normal(g, *size).to(t), _draw_normal(g, *size).to(t)
    return k, v, table


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = _TYPES[case["dtype"]]
    if case["op"] == "logprob":
        x = _draw_normal(g, case["rows"], case["vocab"], scale=2.5)
        x += 6.0 * (torch.rand(x.shape, generator=g, device="cuda") < 4.0 / case["vocab"])
        st = dict(case=case, logits=x.to(t))
        n = case["selected"] or case["rows"]
        st["rows"] = torch.randperm(case["rows"], generator=g, device="cuda")[:n].sort()[0].to(torch.int32) if case["selected"] else None
        best = st["logits"][st["rows"].long() if case["selected"] else slice(None)].float().argmax(-1)
        other = torch.randint(0, case["vocab"], (n,), generator=g, device="cuda")
        st["tokens"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.6, best, other).to(torch.int32)
        new = lambda *size, dtype=torch.float32: torch.empty(*size, dtype=dtype, device="cuda")  # noqa: E731
        st["out"] = dict(logprob=new(n), entropy=new(n), top_tokens=new(n, case["top"], dtype=torch.int32), top_logprobs=new(n, case["top"]))
        if own:
            from paper_2511_21699_amd import binding as B
            cfg = B.make_config(8, 8, 64, case["dtype"], case["dtype"], 1, 64, 8, case["vocab"])
            st["call"] = B.Verifier(cfg).bind_token_logprobs(st["logits"], st["tokens"], case["top"], st["out"]["logprob"], st["out"]["entropy"], st["out"]["top_tokens"],
                                                             st["out"]["top_logprobs"], d_rows=st["rows"])
        return st
    s, n, parent = _shape(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    total = int(off[-1])
    st = dict(case=case, kv_len=np.array(s, dtype=np.int32), offsets=off, total=total)
    st["k"], st["v"], st["table"] = _cache(case, g, max(a + b for a, b in zip(s, n)))
    to = lambda x, dtype=torch.int64: torch.tensor(x, dtype=dtype, device="cuda")  # noqa: E731
    st["seq"] = to([b for b, k in enumerate(n) for _ in range(k)])       # of every new token: its sequence,
    st["slot"] = to([a + i for a, k in zip(s, n) for i in range(k)])     # and its slot in the cache
    st["lens"], st["news"], st["parent"] = to(s), to(n), None
    if case["op"] == "attend":
        st["q"] = _draw_normal(g, total, hq, d, scale=2.0).to(t)
        st["out"] = torch.empty_like(st["q"])
    else:
        # (one product of the model gives a token's queries, keys and values side by side)
        qkv = _draw_normal(g, total, (hq + 2 * hkv) * d, scale=1.5).to(t)
        st["q"], st["new_k"], st["new_v"] = (x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hkv * d, hkv * d], 1))
        st["out"] = torch.empty(total, hq, d, dtype=t, device="cuda")
        st["freq"] = (case["theta"] ** (-torch.arange(0, case["rotary"], 2, device="cuda", dtype=torch.float64) / case["rotary"])).float()
        st["wq"], st["wk"] = (1.0 + _draw_normal(g, d, scale=0.2) for _ in range(2)) if case["norm"] else (None, None)
        if parent:
            st["parent"] = to(parent, torch.int32)
            depth, first = [], 0
            for i, p in enumerate(parent):
                first = i if p < 0 else first
                depth.append(0 if p < 0 else depth[first + p] + 1)
            st["depth"] = to(depth)
    if own:
        from paper_2511_21699_amd import binding as B
        cfg = B.make_config(hq, hkv, d, case["dtype"], case["dtype"], case["batch"], min(256, max(n)), 255, 1000, block_size=case["block"])
        ver = B.Verifier(cfg)
        kv = B.kv_layer(st["k"], st["v"], st["table"], B.CB_LAYOUT_HEAD_MAJOR if case["head_major"] else B.CB_LAYOUT_TOKEN_MAJOR, paged=case["block"] > 0)
        if case["op"] == "attend":
            st["call"] = ver.bind_chunk_attention(st["q"], kv, st["kv_len"], off, st["out"])
        else:
            prep = B.head_prep(st["wq"], st["wk"], _EPS, st["freq"], interleaved=case["interleaved"])
            st["call"] = ver.bind_append_kv(st["q"], st["new_k"], st["new_v"], prep, kv, st["kv_len"], off, st["out"], d_parent=st["parent"])
    return st


def _index(st):
    """Where the cache holds the new tokens' rows, as an index of its first dimensions."""
    case, seq, slot = st["case"], st["seq"], st["slot"]
    if case["block"]:
        unit, at = st["table"].long()[seq, slot // case["block"]], slot % case["block"]
    else:
        unit, at = seq, slot
    return (unit, slice(None), at) if case["head_major"] else (unit, at)


def _prepared(x, w, cos, sin, case):
    """Heads normalised and rotated, in 32 bits: x / rms(x) * w, then every pair (a, b) becomes (a cos - b sin, b cos + a sin)."""
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * w
    r = case["rotary"]
    turned, rest = x[..., :r], x[..., r:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if case["interleaved"] else (turned[..., :r // 2], turned[..., r // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, rest], -1)


def _append(st):
    case, t = st["case"], st["k"].dtype
    position = st["slot"] if st["parent"] is None else st["lens"][st["seq"]] + st["depth"]
    angle = (position.double()[:, None] * st["freq"].double())[:, None]
    cos, sin = angle.cos().float(), angle.sin().float()
    st["out"].copy_(_prepared(st["q"], st["wq"], cos, sin, case))
    index = _index(st)
    st["k"][index] = _prepared(st["new_k"], st["wk"], cos, sin, case).to(t)
    st["v"][index] = st["new_v"]
    return dict(q=st["out"], k=st["k"], v=st["v"])


def _attend(st):
    case, batch, hq, hkv, d = st["case"], st["case"]["batch"], st["case"]["hq"], st["case"]["hkv"], st["case"]["d"]
    g = hq // hkv

    def rows(cache):  # [batch, hkv, slots, d] in 32 bits
        if case["block"]:
            cache = cache[st["table"].long()]
            cache = cache.permute(0, 2, 1, 3, 4) if case["head_major"] else cache.permute(0, 3, 1, 2, 4)
            return cache.float().reshape(batch, hkv, -1, d)
        return (cache if case["head_major"] else cache.transpose(1, 2)).float().contiguous()

    k, v = rows(st["k"]), rows(st["v"])
    most = case["n_hi"]
    slots = k.shape[2]
    at = st["slot"] - st["lens"][st["seq"]]
    q = torch.zeros(batch, most, hq, d, dtype=torch.float32, device="cuda")
    q[st["seq"], at] = st["q"].float() * d ** -0.5
    # the query heads of a kv head are rows of one product
    q = q.view(batch, most, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(batch, hkv, most * g, d)
    p = q @ k.transpose(2, 3).contiguous()
    seen = st["lens"][:, None] + torch.arange(most, device="cuda") + 1
    hidden = torch.arange(slots, device="cuda") >= seen.repeat_interleave(g, 1)[:, None, :, None]
    p.masked_fill_(hidden, -math.inf)
    p -= p.amax(-1, keepdim=True)
    p.exp_()
    total = p.sum(-1, keepdim=True)
    # (a cache's slots behind a sequence hold anything: those values are not multiplied, by 0 either)
    v = v.masked_fill((torch.arange(slots, device="cuda") >= (st["lens"] + st["news"])[:, None])[:, None, :, None], 0.0)
    o = (p @ v) / total
    o = o.view(batch, hkv, most, g, d).permute(0, 2, 1, 3, 4).reshape(batch, most, hq, d)
    st["out"].copy_(o[st["seq"], at])
    return st["out"]


def _logprob(st):
    top, out = st["case"]["top"], st["out"]
    x = (st["logits"] if st["rows"] is None else st["logits"][st["rows"].long()]).float()
    shifted = x - x.amax(-1, keepdim=True)
    e = shifted.exp()
    total = e.sum(-1, keepdim=True)
    logs = shifted - total.log()
    out["logprob"].copy_(logs.gather(1, st["tokens"].long()[:, None])[:, 0])
    out["entropy"].copy_(-(e * logs).sum(-1) / total[:, 0])
    if top:
        # whole numbers that order the entries by value and, among equal ones, the lower index first
        bits = (x + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7fffffff) - 1, bits) * 2 ** 20 + (2 ** 20 - 1 - torch.arange(x.shape[1], device="cuda"))
        best = torch.topk(key, top, dim=-1)[0]
        index = 2 ** 20 - 1 - (best & (2 ** 20 - 1))
        out["top_tokens"].copy_(index)
        out["top_logprobs"].copy_(logs.gather(1, index))
    return out


def run(state):
    if own:
        state["call"]()
        return dict(q=state["out"], k=state["k"], v=state["v"]) if state["case"]["op"] == "append" else state["out"]
    return {"append": _append, "attend": _attend, "logprob": _logprob}[state["case"]["op"]](state)


def work(case):
    eb = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "logprob":
        rows = case["selected"] or case["rows"]
        return {"bytes": rows * (case["vocab"] * eb + 12 + 8 * case["top"]), "flops": rows * case["vocab"] * 5}
    s, n, _ = _shape(case)
    new, hq, hkv, d = sum(n), case["hq"], case["hkv"], case["d"]
    if case["op"] == "append":
        return {"bytes": 2 * new * (hq + 2 * hkv) * d * eb, "flops": new * (hq + hkv) * d * (3 + (4 if case["norm"] else 0))}
    keys = sum(a + b for a, b in zip(s, n))
    pairs = sum(b * a + b * (b + 1) // 2 for a, b in zip(s, n))
    return {"bytes": (2 * keys * hkv + 2 * new * hq) * d * eb, "flops": 4 * pairs * hq * d}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "logprob":
        rows = range(case["rows"]) if st["rows"] is None else st["rows"].tolist()
        lp, ent, ids, tops = [], [], [], []
        for r, token in zip(rows, st["tokens"].tolist()):
            x = st["logits"][r].double()
            z = torch.logsumexp(x, 0)
            lp.append(x[token] - z)
            ent.append(z - torch.dot(torch.exp(x - z), x))
            order = torch.sort(x, descending=True, stable=True)[1][:case["top"]]
            ids.append(order.to(torch.int32))
            tops.append(x[order] - z)
        return dict(logprob=torch.stack(lp), entropy=torch.stack(ent), top_tokens=torch.stack(ids), top_logprobs=torch.stack(tops))
    s, n, off = st["kv_len"].tolist(), np.diff(st["offsets"]).tolist(), st["offsets"].tolist()
    d, block = case["d"], case["block"]

    if case["op"] == "append":
        r = case["rotary"]
        parents = st["parent"].tolist() if case["tree"] else None
        pos = []
        for b in range(case["batch"]):
            depth = []
            for i in range(n[b]):
                depth.append(i if parents is None else (0 if i == 0 else depth[parents[off[b] + i]] + 1))
            pos += [s[b] + x for x in depth]
        angle = torch.tensor(pos, dtype=torch.float64, device="cuda")[:, None] * st["freq"].double()
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]

        def heads(x, w):
            x = x.double()
            if w is not None:
                x = x / (x.pow(2).mean(-1, keepdim=True) + _EPS).sqrt() * w.double()
            i = torch.arange(r // 2, device="cuda")
            ia, ib = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + r // 2)
            z = torch.complex(x[..., ia].contiguous(), x[..., ib].contiguous()) * turn
            y = x.clone()
            y[..., ia], y[..., ib] = z.real, z.imag
            return y

        k, v, new_k, new_v = st["k"].double(), st["v"].double(), heads(st["new_k"], st["wk"]), st["new_v"].double()
        units, ats, table = [], [], st["table"].tolist() if block else None
        for b in range(case["batch"]):
            for slot in range(s[b], s[b] + n[b]):
                units.append(table[b][slot // block] if block else b)
                ats.append(slot % block if block else slot)
        units, ats = (torch.tensor(x, device="cuda") for x in (units, ats))
        if case["head_major"]:
            k[units, :, ats], v[units, :, ats] = new_k, new_v
        else:
            k[units, ats], v[units, ats] = new_k, new_v
        return dict(q=heads(st["q"], st["wq"]), k=k, v=v)
    out = torch.empty(st["total"], case["hq"], d, dtype=torch.float64, device="cuda")
    g = case["hq"] // case["hkv"]
    for b in range(case["batch"]):
        length = s[b] + n[b]

        def rows(cache, head):
            if not block:
                return (cache[b, head, :length] if case["head_major"] else cache[b, :length, head]).double()
            units = st["table"][b, :(length + block - 1) // block].long()
            pages = cache[units][:, head] if case["head_major"] else cache[units][:, :, head]
            return pages.reshape(-1, d)[:length].double()

        hidden = torch.arange(length, device="cuda")[None, :] > s[b] + torch.arange(n[b], device="cuda")[:, None]
        for head in range(case["hkv"]):
            k, v = rows(st["k"], head), rows(st["v"], head)
            for j in range(head * g, head * g + g):
                score = (st["q"][off[b]:off[b + 1], j].double() @ k.T) / math.sqrt(d)
                out[off[b]:off[b + 1], j] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ v
    return out

