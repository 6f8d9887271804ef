"""The operators of chunks of new tokens over a paged cache, plainly, in 64 bits on the CPU: one loop per definition."""
import math

import torch

from batch_reference import TORCH, rotate  # noqa: F401

BIG = torch.finfo(torch.float32).max


def finite(x):
    return torch.where(x.isnan(), torch.zeros((), dtype=x.dtype), x).clamp(-BIG, BIG)


def quantise(x):
    """Codes and scales of rows x [.., d] in 64 bits."""
    scale = (x.abs().amax(-1) / 127.0).float()
    step = scale.double()
    code = torch.where(step[..., None] > 0, x / step.clamp(min=1e-300)[..., None], 0.0).round().clamp(-127, 127)
    return code.to(torch.int8), scale


def values(pool, scale=None):
    """What a pool stands for."""
    return pool.double() if scale is None else pool.double() * scale.double()[..., None]


def attention(q, K, V, table, first, length, K_scale=None, V_scale=None):
    """(out, sum of p |v|) [tokens, heads, d], NaN for rows that are no sequence's; a position on a page out of range does not count."""
    n_tokens, heads, d = q.shape
    n_pages, n_kv, page, _ = K.shape
    out = torch.full((n_tokens, heads, d), math.nan, dtype=torch.float64)
    size = out.clone()
    first = first.tolist()
    for s, n in enumerate(length.tolist()):
        a, b = first[s], first[s + 1]
        if a == b:
            continue
        at = [(p, int(table[s, p // page]), p % page) for p in range(n)]
        at = [x for x in at if 0 <= x[1] < n_pages]
        out[a:b], size[a:b] = 0.0, 0.0
        if not at:
            continue
        p, pages, rows = (torch.tensor(x) for x in zip(*at))
        k, v = (values(x[pages, :, rows], None if y is None else y[pages, :, rows]) for x, y in ((K, K_scale), (V, V_scale)))
        k, v = k.repeat_interleave(heads // n_kv, 1), v.repeat_interleave(heads // n_kv, 1)
        for t in range(a, b):
            seen = p <= n - (b - a) + t - a
            if not seen.any():
                continue
            w = torch.softmax((k[seen] * q[t].double()).sum(-1) / math.sqrt(d), 0)[..., None]
            out[t], size[t] = (w * v[seen]).sum(0), (w * v[seen].abs()).sum(0)
    return out, size


def probabilities(row, tau):
    z = row.double()
    z = torch.where(z.isnan(), -math.inf, z).clamp(max=BIG) / tau
    top = z.max()
    if top == -math.inf:
        return torch.zeros_like(z)
    e = torch.exp(z - top)
    return e / e.sum()


def verify(logits, tokens, u, tau, draft_logits=None, draft_tau=1.0):
    """One sequence: (drafts that stand, tokens given, their log p, whether something was no token or no row, how near a decision was)."""
    m, V = len(tokens) - 1, logits.shape[1]
    given, logp, err, near, at = [], [], False, 1.0, 0
    rest = None
    for at in range(m + 1):
        p = probabilities(logits[at], tau)
        err |= not p.any()
        if at == m:
            rest = p
            break
        x = int(tokens[at + 1])
        err |= not 0 <= x < V
        q = torch.zeros(V, dtype=torch.float64)
        if draft_logits is not None:
            q = probabilities(draft_logits[at], draft_tau)
        elif 0 <= x < V:
            q[x] = 1.0
        if 0 <= x < V:
            near = min(near, abs(float(u[at] * q[x] - p[x])))
            if float(u[at]) * float(q[x]) < float(p[x]):
                given.append(x)
                logp.append(math.log(float(p[x])))
                continue
        rest = (p - q).clamp(min=0.0)
        if not rest.any():
            rest = p
        break
    total = rest.cumsum(0)
    bound = float(u[m]) * float(total[-1])
    x = int((total <= bound).sum())
    if x >= V:
        x = int(rest.nonzero().max()) if rest.any() else 0
    if rest.any():
        near = min(near, float((total - bound).abs().min() / total[-1]))
    return at, given + [x], logp + [math.log(float(p[x])) if p[x] > 0 else -math.inf], err, near
