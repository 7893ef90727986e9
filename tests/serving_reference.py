"""Plain 64-bit forms of the calls around the verification (cb_append_kv_device, cb_chunk_attention_device, cb_token_logprobs_device) on
numpy arrays, and batches to try them on."""
import math

import numpy as np

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # a rounding's relative error at most


def depths(parents):
    out = []
    for p in parents:
        out.append(0 if p < 0 else out[p] + 1)
    return out


def prepared(x, weight, eps, inv_freq, interleaved, positions):
    """Heads [n, H, D] normalised and rotated; and what their rounding errors are relative to (the pairs' sizes)."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    y, size = x.copy(), np.abs(x)
    r = 0 if inv_freq is None else 2 * len(inv_freq)
    for i in range(r // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        angle = np.asarray(positions, dtype=np.float64)[:, None] * float(inv_freq[i])
        c, s = np.cos(angle), np.sin(angle)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = np.hypot(x[..., a], x[..., b])
    return y, size


def chunk_attention(q, keys, values, kv_len, offsets, scale):
    """q [n, Hq, D]; keys, values: per sequence [slots, Hkv, D].  Returns the output, sum p |v| and the largest scale * sum |q k| of each row."""
    q = np.asarray(q, dtype=np.float64)
    n, hq, d = q.shape
    out, size, score = np.zeros_like(q), np.zeros_like(q), np.zeros((n, hq, 1))
    for b, s in enumerate(kv_len):
        t0, t1 = offsets[b], offsets[b + 1]
        if t0 == t1:
            continue
        length = s + t1 - t0
        hidden = np.arange(length)[None, :] > s + np.arange(t1 - t0)[:, None]
        g = hq // np.asarray(keys[b]).shape[1]
        for h in range(hq):
            k, v = (np.asarray(x[b][:length, h // g], dtype=np.float64) for x in (keys, values))
            x = np.where(hidden, -np.inf, q[t0:t1, h] @ k.T * scale)
            p = np.exp(x - x.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[t0:t1, h], size[t0:t1, h] = p @ v, p @ np.abs(v)
            score[t0:t1, h, 0] = np.where(hidden, 0.0, np.abs(q[t0:t1, h]) @ np.abs(k).T).max(-1) * scale
    return out, size, score


def attention_tolerance(dtype, out, size, score, longest, d):
    """What the kernels' arithmetic can be off by.  Scores are sums of d products in 32 bits: each is off by (d + 2) 2^-24 of sum |q k|, and
    so by that much, relatively, each probability (twice: numerator and denominator); sums of n terms in 32 bits add 2^-24 for every
    addition on the way, at most n / 16 with 16 keys to an accumulation; bf16 probabilities half a step each, in numerator and denominator; partial states and
    output are rounded once more each."""
    h, f = HALF_STEP[dtype], 2.0 ** -24
    probability = 2 * ((d + 2) * f * score + 8 * f) + (longest / 16 + 64) * f + (2 * h if dtype == "bf16" else 0.0)
    return probability * size + 2 * h * np.abs(out) + 1e-30


def token_logprobs(x, token, top):
    """One row in 64 bits: (log probability, entropy, the top tokens, their log probabilities)."""
    x = np.asarray(x, dtype=np.float64)
    m = x.max()
    order = np.lexsort((np.arange(len(x)), -x))[:top]
    if m == -np.inf:
        return -np.inf, 0.0, order, np.full(top, -np.inf)
    e = np.exp(x - m)
    z = e.sum()
    logs = x - m - math.log(z)
    entropy = -(e[e > 0] / z * logs[e > 0]).sum()
    return logs[token] if 0 <= token < len(x) else np.nan, entropy, order, logs[order]


def logprob_tolerance(logp, entropy, vocab):
    """A log probability is a difference of (x - max), log Z and nothing else: half a step of each, and Z's relative error -- an exponential off
    by (|x - max| + 2) 2^-24 relatively, weighted by itself: at most (|entropy| + 4) 2^-24 on average; sums of 256 terms and a tree above them."""
    f = 2.0 ** -24
    z = (abs(entropy) + 4 + 256 + 32) * f
    finite = np.where(np.isfinite(logp), np.abs(logp), 0.0)
    return 3 * f * (finite + math.log(vocab + 1)) + z
