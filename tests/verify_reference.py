"""Verification of drafted tokens by its definition in logarithms, in 64 bits on the CPU: nothing of it underflows but the weights that a token is drawn with."""
import math

import torch

BIG = torch.finfo(torch.float32).max


def log2_probabilities(row, tau):
    """log2 p of a row of logits (no number: -inf; +inf: the largest finite number); all -inf where no logit is finite."""
    z = row.double()
    z = torch.where(z.isnan(), -math.inf, z).clamp(max=BIG)
    top = z.max()
    if top == -math.inf:
        return z
    d = (z - top) * (math.log2(math.e) / tau)
    return d - torch.exp2(d).sum().log2()


def verify(logits, tokens, u, tau, draft_logits=None, draft_tau=1.0):
    """One sequence: (drafts that stand, tokens given, their log p, whether something was no token or no row, how near a draft's decision was, relative to p / q, and how near the draw, relative to the sum)."""
    m, V = len(tokens) - 1, logits.shape[1]
    given, logp, err, near, lq, x = [], [], False, math.inf, None, None
    for at in range(m + 1):
        lp = log2_probabilities(logits[at], tau)
        err |= bool(lp.max() == -math.inf)
        if at == m:
            break
        x = int(tokens[at + 1])
        known = 0 <= x < V
        err |= not known
        lq = None if draft_logits is None else log2_probabilities(draft_logits[at], draft_tau)
        stands = known and float(lp[x]) > -math.inf
        if stands and (lq is None or float(lq[x]) > -math.inf):
            ratio = float(lp[x]) - (0.0 if lq is None else float(lq[x]))
            r = 2.0 ** min(ratio, 900.0) if ratio >= -1021.0 else 0.0
            stands = float(u[at]) < r
            near = min(near, abs(float(u[at]) / r - 1.0)) if r else near
        if not stands:
            break
        given.append(x)
        logp.append(float(lp[x]) * math.log(2.0))
    weight = lambda l: torch.where(l - l.max() >= -1021.0, torch.exp2(l), 0.0) if l.max() > -math.inf else torch.zeros_like(l)  # noqa: E731
    w = weight(lp)
    rest = w
    if at < m:
        rest = w.clone()
        if lq is not None:
            rest = (w - weight(lq)).clamp(min=0.0)
        elif 0 <= x < V:
            rest[x] = 0.0
        if not rest.any():
            rest = w
    total = rest.cumsum(0)
    bound = float(u[m]) * float(total[-1])
    some = rest.nonzero()[:, 0]
    past = some[total[some] > bound]
    token = int(past[0]) if len(past) else int(some[-1]) if len(some) else 0
    # how near a border between two tokens is: those behind a token of some weight, but for the last
    far = float((total[some[:-1]] - bound).abs().min() / total[-1]) if len(some) > 1 else math.inf
    return len(given), given + [token], logp + [float(lp[token]) * math.log(2.0)], err, near, far
