"""The operators of several sequences over one paged cache, plainly, in 64 bits on the CPU: one loop per definition."""
import math

import torch

TORCH = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def rotate(x, pos, theta):
    """x [heads, d] at one position: adjacent pairs turned by pos theta^(-2i/d)."""
    d = x.shape[-1]
    x, y = x.double(), torch.empty(x.shape, dtype=torch.float64)
    for i in range(d // 2):
        a = pos * theta ** (-2.0 * i / d)
        c, s = math.cos(a), math.sin(a)
        y[:, 2 * i] = x[:, 2 * i] * c - x[:, 2 * i + 1] * s
        y[:, 2 * i + 1] = x[:, 2 * i] * s + x[:, 2 * i + 1] * c
    return y


def attention(q, K, V, table, shared, length, width):
    """[n_seq, heads, d]; a position on a page out of range does not count."""
    n_seq, heads, d = q.shape
    n_pages, n_kv, page, _ = K.shape
    out = torch.zeros(n_seq, heads, d, dtype=torch.float64)
    for s in range(n_seq):
        lead = s - s % width
        at = [(int(table[lead if p < shared[s // width] else s, p // page]), p % page) for p in range(int(length[s]))]
        at = [(a, b) for a, b in at if 0 <= a < n_pages]
        if not at:
            continue
        a, b = (torch.tensor(x) for x in zip(*at))
        for h in range(heads):
            k, v = (pool[a, h * n_kv // heads, b].double() for pool in (K, V))
            out[s, h] = torch.softmax(k @ q[s, h].double() / math.sqrt(d), 0) @ v
    return out


def select(logits, scores, n_out, tau, ended=None, end_token=-1):
    """[(score, token, parent, ended)] of one group's beams; logits [n_in, vocab]."""
    found = []
    big = torch.finfo(torch.float32).max
    for b in range(len(scores)):
        score = float(scores[b])
        if not score > -math.inf:
            continue
        if ended is not None and ended[b]:
            found.append((score, end_token, b))
            continue
        z = logits[b].double()
        z = torch.where(z.isnan(), -math.inf, z).clamp(max=big)
        logp = z / tau - torch.logsumexp(z / tau, 0)
        best = torch.sort(z, descending=True, stable=True).indices[:n_out].tolist()
        found += [(score + float(logp[v]), v, b) for v in best if z[v] > -math.inf]
    found.sort(key=lambda c: (-c[0], c[2], c[1]))
    out = [(s, v, b, int(v == end_token or (ended is not None and bool(ended[b])))) for s, v, b in found[:n_out]]
    return out + [(-math.inf, 0, j if j < len(scores) else 0, 0) for j in range(len(out), n_out)]


def reorder(K, V, table, parents, length, width):
    """(K, V, table) behind one selection; K, V [layers, pages, heads, page, d]."""
    K, V, out = K.clone(), V.clone(), table.clone()
    page = K.shape[3]
    for g in range(len(parents)):
        n = int(length[g * width])
        e, filled = n // page, n % page
        row = lambda w: g * width + w  # noqa: E731
        spare, seen = [w for w in range(width) if w not in parents[g].tolist()], set()
        for j, p in enumerate(parents[g].tolist()):
            takes = p
            if p in seen:
                takes = spare.pop(0)
                if filled:
                    a, b = int(table[row(p), e]), int(table[row(takes), e])
                    K[:, b, :, :filled], V[:, b, :, :filled] = K[:, a, :, :filled], V[:, a, :, :filled]
            seen.add(p)
            out[row(j), :e], out[row(j), e:] = table[row(p), :e], table[row(takes), e:]
    return K, V, out
