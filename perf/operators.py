"""The operators of several sequences that share a prompt, as measurable cases.

k independent passes or a beam search over one prompt are k sequences that agree in their first
positions.  Four operators of `paper_2405_18400_amd` take such a batch through a step:

  append   keys and values of new tokens go into a paged cache, rotated on the way, with the
           queries of the same tokens (`spd_op_append_paged`)
  attend   one query per sequence and head over its positions; a group's shared positions are
           read once for all of its sequences (`spd_op_attention_shared`)
  select   the best continuations of a group's beams over the vocabulary (`spd_op_beam_select`)
  reorder  page tables follow the beams they continue; pages that are still being filled are
           copied (`spd_op_beam_reorder`)

A paged cache is K and V [pages, key/value heads, page size, d_head] and a table [sequences,
entries] of page numbers: position p of sequence s lies in page table[s][p // page size], row
p % page size.  Head layouts are those of the 7B, 13B and 70B shapes of the benchmark.

`own` false: the plain form, elementary operations in 32 bits (64 for angles and for scores that are
ranked).  `own` true: the library.
"""
import math

import torch

own = False

TORCH = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}
THETA = 10000.0


def listed():
    return [
        # one decoding step of four beams of a 7B model: the smallest call, nothing but latency
        {"name": "append-step", "op": "append", "dtype": "fp16", "heads": 32, "kv_heads": 32, "d_head": 128, "page": 16, "seqs": 4, "tokens": 4, "pad": 0, "start": 70},
        # prompts of uneven lengths in one call, padded behind the last, far into their texts: grouped heads of a 70B model
        {"name": "append-prompts", "op": "append", "dtype": "bf16", "heads": 64, "kv_heads": 8, "d_head": 128, "page": 64, "seqs": 7, "tokens": 4099, "pad": 61, "start": 30011},
        # the attention of that step of four beams behind a 64-token prompt
        {"name": "attend-step", "op": "attend", "dtype": "fp16", "heads": 32, "kv_heads": 32, "d_head": 128, "page": 16, "groups": 1, "width": 4, "shared": 64, "own": 10},
        # five beams of a 13B model with the default fp32 cache behind a prompt that ends inside a page
        {"name": "attend-fp32", "op": "attend", "dtype": "fp32", "heads": 40, "kv_heads": 40, "d_head": 128, "page": 32, "groups": 1, "width": 5, "shared": 1027, "own": 20},
        # eight beams, grouped heads, a prompt of eight thousand tokens
        {"name": "attend-beams", "op": "attend", "dtype": "fp16", "heads": 64, "kv_heads": 8, "d_head": 128, "page": 64, "groups": 1, "width": 8, "shared": 8191, "own": 100},
        # a batch of eight prompts with eight sequences each, whose own parts count
        {"name": "attend-batch", "op": "attend", "dtype": "bf16", "heads": 32, "kv_heads": 8, "d_head": 128, "page": 16, "groups": 8, "width": 8, "shared": 2001, "own": 300},
        # sixteen sequences over one very long document
        {"name": "attend-long", "op": "attend", "dtype": "fp16", "heads": 64, "kv_heads": 8, "d_head": 128, "page": 128, "groups": 1, "width": 16, "shared": 65537, "own": 33},
        # the selection of that step of four beams
        {"name": "select-step", "op": "select", "dtype": "fp32", "groups": 1, "n_in": 4, "n_out": 4, "vocab": 32000, "ended": 0, "tau": 1.0},
        # a batch of sixteen prompts, some beams at their end
        {"name": "select-batch", "op": "select", "dtype": "fp32", "groups": 16, "n_in": 8, "n_out": 8, "vocab": 50258, "ended": 1, "tau": 0.7},
        # wide beams over a large vocabulary, logits in 16 bits
        {"name": "select-wide", "op": "select", "dtype": "bf16", "groups": 4, "n_in": 16, "n_out": 16, "vocab": 131072, "ended": 0, "tau": 1.0},
        # the cache of a 7B model after the selection of that step of four beams
        {"name": "reorder-step", "op": "reorder", "dtype": "fp16", "layers": 32, "kv_heads": 32, "d_head": 128, "page": 16, "groups": 1, "width": 4, "alive": 2, "length": 74},
        # grouped heads, a batch of eight prompts, large pages
        {"name": "reorder-batch", "op": "reorder", "dtype": "bf16", "layers": 16, "kv_heads": 8, "d_head": 128, "page": 64, "groups": 8, "width": 8, "alive": 3, "length": 303},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "select", "select", "reorder"])
    if op == "select":
        groups, n_in, vocab = _log(rng, 1, 16), rng.randrange(1, 17), _log(rng, 50, 131072)
        while groups * n_in * vocab > 8_000_000:
            groups, vocab = max(1, groups // 2), max(50, vocab // 2 + 1)
        return {"op": op, "dtype": rng.choice(["fp32", "fp32", "bf16", "fp16"]), "groups": groups, "n_in": n_in, "n_out": rng.randrange(1, min(16, n_in * 8) + 1), "vocab": vocab,
                "ended": rng.randrange(0, (n_in + 1) // 2), "tau": round(rng.uniform(0.3, 1.5), 3)}
    kv = rng.choice([1, 2, 4, 8, 8, 32, 40])
    heads = kv * rng.choice([1, 1, 2, 3, 4, 8] if kv <= 8 else [1])
    case = {"op": op, "dtype": rng.choice(["fp16", "fp16", "bf16", "fp32"]), "heads": heads, "kv_heads": kv, "d_head": rng.choice([64, 128, 128, 256]), "page": rng.choice([8, 16, 32, 64, 128])}
    if op == "append":
        seqs = _log(rng, 1, 40)
        return {**case, "seqs": seqs, "tokens": _log(rng, seqs, 40 + 15_000_000 // (heads * case["d_head"] + 1000)), "pad": rng.choice([0, 0, 1, 77]), "start": _log(rng, 1, 100_000)}
    if op == "attend":
        groups, width = _log(rng, 1, 8), _log(rng, 1, 24)
        shared = _log(rng, 1, 40_000) if rng.random() < 0.9 else 0
        room = 30_000_000 // (kv * case["d_head"])
        shared = min(shared, room // (2 * groups))
        return {**case, "groups": groups, "width": width, "shared": shared, "own": min(_log(rng, 1, 2000), max(1, room // (2 * groups * width)))}
    width = rng.randrange(2, 17)
    layers = _log(rng, 1, 40)
    per = kv * case["d_head"] * case["page"] * width
    layers = min(layers, max(1, 20_000_000 // per))
    del case["heads"]
    return {**case, "layers": layers, "groups": min(_log(rng, 1, 8), max(1, 20_000_000 // (per * layers))), "width": width, "alive": rng.randrange(1, width + 1), "length": _log(rng, 1, 1000)}


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype=torch.float32, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _spread(total, parts):
    """`total` in `parts` uneven shares, each at least one (their sizes are part of the case, not of the seed)."""
    weights = [3 + (5 * i) % 7 for i in range(parts)]
    shares = [1 + (total - parts) * w // sum(weights) for w in weights]
    shares[-1] += total - sum(shares)
    return shares


def _own_lengths(c):
    """Uneven lengths of the sequences' own parts, the longest `own`, the shortest about half of it."""
    return [c["own"] - (5 * i) % (c["own"] // 2 + 1) for i in range(c["groups"] * c["width"])]


def _lengths(c):
    """Text lengths of the groups whose tables are put in order."""
    return [c["length"] + 3 * g for g in range(c["groups"])]


def _pool(g, c, pages):
    shape = (pages, c["kv_heads"], c["page"], c["d_head"])
    return _normal(g, shape, TORCH[c["dtype"]]), _normal(g, shape, TORCH[c["dtype"]])


def _prepare_append(c, g):
    shares, page = _spread(c["tokens"], c["seqs"]), c["page"]
    seq, pos, used = [], [], []
    for s, n in enumerate(shares):
        first = c["start"] + 3 * s
        seq += [s] * n
        pos += range(first, first + n)
        used.append((first // page, (first + n - 1) // page + 1))
    order = torch.randperm(sum(b - a for a, b in used), generator=g, device="cuda").int()
    table = torch.full((c["seqs"], max(b for _, b in used)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, (a, b) in enumerate(used):
        table[s, a:b] = order[at:at + b - a]
        at += b - a
    seq, pos = seq + [-1] * c["pad"], pos + [0] * c["pad"]
    n, h, kv, d = len(seq), c["heads"], c["kv_heads"], c["d_head"]
    K, V = _pool(g, c, at)
    qkv = _normal(g, (n, (h + 2 * kv) * d))   # the rows that one product makes of a token
    q, k, v = qkv.split([h * d, kv * d, kv * d], 1)
    return {"c": c, "K": K, "V": V, "table": table, "q": q.unflatten(1, (h, d)), "k": k.unflatten(1, (kv, d)), "v": v.unflatten(1, (kv, d)),
            "seq": _ints(seq), "pos": _ints(pos), "q_out": torch.zeros(n, h, d, device="cuda")}


def _prepare_attend(c, g):
    G, W, page = c["groups"], c["width"], c["page"]
    n, owns = G * W, _own_lengths(c)
    whole, last = c["shared"] // page, (c["shared"] + c["own"] - 1) // page + 1   # pages of shared positions alone; a row's entries
    pages = G * whole + n * (last - whole)
    order = torch.randperm(pages, generator=g, device="cuda").int()
    common = order[:G * whole].view(G, 1, whole).expand(G, W, whole).reshape(n, whole)
    table = torch.cat([common, order[G * whole:].view(n, last - whole)], 1).contiguous()
    K, V = _pool(g, c, pages)
    shape = (n, c["heads"], c["d_head"])
    return {"c": c, "K": K, "V": V, "table": table, "q": _normal(g, shape), "shared": _ints([c["shared"]] * G), "length": _ints([c["shared"] + o for o in owns]),
            "out": torch.empty(shape, device="cuda")}


def _prepare_select(c, g):
    G, n_in, V = c["groups"], c["n_in"], c["vocab"]
    # logits of a trained model: a few likely tokens above a broad rest; scores of sequences of some tokens
    logits = _normal(g, (G, n_in, V), std=2.5)
    scores = -torch.rand(G, n_in, device="cuda", generator=g) * 5.0 - 1.0
    order = torch.rand(G, n_in, device="cuda", generator=g).argsort(1)
    out = lambda t: torch.empty(G, c["n_out"], dtype=t, device="cuda")  # noqa: E731
    return {"c": c, "logits": logits.to(TORCH[c["dtype"]]), "scores": scores, "ended": (order < c["ended"]).int(), "end": 2 % V, "out_scores": out(torch.float32), "out_tokens": out(torch.int32),
            "out_parents": out(torch.int32), "out_ended": out(torch.int32)}


def _prepare_reorder(c, g):
    G, W, page, L = c["groups"], c["width"], c["page"], c["layers"]
    lengths = _lengths(c)
    entries = max(lengths) // page + 2
    first = min(lengths) // page            # entries before it: full pages, whose contents no call reads
    pages = G * W * (entries - first)
    table = torch.zeros(G * W, entries, dtype=torch.int32, device="cuda")
    table[:, :first] = torch.randint(0, pages, (G * W, first), generator=g, device="cuda").int()
    table[:, first:] = torch.randperm(pages, generator=g, device="cuda").int().view(G * W, entries - first)
    shape = (L, pages, c["kv_heads"], page, c["d_head"])
    alive = torch.rand(G, W, device="cuda", generator=g).argsort(1)[:, :c["alive"]]
    pick = torch.randint(0, c["alive"], (G, W), generator=g, device="cuda")
    pick[:, :c["alive"]] = torch.arange(c["alive"], device="cuda")      # every row that lives on has a child
    parents = alive.gather(1, pick).gather(1, torch.rand(G, W, device="cuda", generator=g).argsort(1)).int()
    return {"c": c, "K": _normal(g, shape, TORCH[c["dtype"]]), "V": _normal(g, shape, TORCH[c["dtype"]]), "table": table, "parents": parents,
            "length": _ints([n for n in lengths for _ in range(W)]), "table_out": torch.empty_like(table)}


def prepare(case, seed):
    make = {"append": _prepare_append, "attend": _prepare_attend, "select": _prepare_select, "reorder": _prepare_reorder}[case["op"]]
    return make(dict(case), _generator(seed))


# ------------------------------------------------------------------ the library's operators
def _own_append(s):
    import paper_2405_18400_amd as pkg
    pkg.spd_op_append_paged(s["c"]["dtype"], s["K"], s["V"], s["table"], s["k"], s["v"], s["seq"], s["pos"], THETA, q=s["q"], q_out=s["q_out"])
    return {"K": s["K"], "V": s["V"], "q": s["q_out"]}


def _own_attend(s):
    import paper_2405_18400_amd as pkg
    c = s["c"]
    pkg.spd_op_attention_shared(c["dtype"], s["q"], s["K"], s["V"], s["table"], s["shared"], s["length"], s["out"], c["width"], c["shared"], c["own"])
    return s["out"]


def _own_select(s):
    import paper_2405_18400_amd as pkg
    c = s["c"]
    pkg.spd_op_beam_select(c["dtype"], s["logits"], s["scores"], s["out_scores"], s["out_tokens"], s["out_parents"], tau=c["tau"], ended=s["ended"], end_token=s["end"],
                           out_ended=s["out_ended"])
    return {"scores": s["out_scores"], "tokens": s["out_tokens"], "parents": s["out_parents"], "ended": s["out_ended"]}


def _own_reorder(s):
    import paper_2405_18400_amd as pkg
    c = s["c"]
    pkg.spd_op_beam_reorder(c["dtype"], s["K"], s["V"], s["table"], s["parents"], s["length"], s["table_out"], c["width"])
    return {"K": s["K"], "V": s["V"], "table": s["table_out"]}


# ------------------------------------------------------------------ the plain forms
def _turned(x, pos, theta):
    d = x.shape[-1]
    angle = pos.double()[:, None] * theta ** (-torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / d)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)


def _plain_append(s):
    n = s["c"]["tokens"]                    # tokens behind them are padding
    seq, pos, page = s["seq"][:n].long(), s["pos"][:n].long(), s["c"]["page"]
    at, row = s["table"][seq, pos // page].long(), pos % page
    s["K"][at, :, row] = _turned(s["k"][:n], pos, THETA).to(s["K"].dtype)
    s["V"][at, :, row] = s["v"][:n].to(s["V"].dtype)
    s["q_out"][:n] = _turned(s["q"][:n], pos, THETA)
    return {"K": s["K"], "V": s["V"], "q": s["q_out"]}


def _gathered(pool, table, first, count):
    """Positions first .. first + count - 1 of every row of `table`: [rows, key/value heads, count, d_head] in 32 bits."""
    p = torch.arange(first, first + count, device=pool.device)
    page = pool.shape[2]
    return pool[table[:, p // page].long(), :, p % page].float().transpose(1, 2)


def _plain_attend(s):
    c = s["c"]
    G, W, kv, d = c["groups"], c["width"], c["kv_heads"], c["d_head"]
    group = c["heads"] // kv
    q = s["q"].view(G, W, kv, group, d)
    # the shared positions: all rows of a group against one copy of its keys
    K, V = (_gathered(x, s["table"][::W], 0, c["shared"]) for x in (s["K"], s["V"]))
    z0 = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(G, kv, W * group, d), K.transpose(2, 3)).view(G, kv, W, group, -1).transpose(1, 2)
    # each sequence's own positions
    Ko, Vo = (_gathered(x, s["table"], c["shared"], c["own"]) for x in (s["K"], s["V"]))
    z1 = torch.matmul(q.reshape(G * W, kv, group, d), Ko.transpose(2, 3)).view(G, W, kv, group, -1)
    there = torch.arange(c["own"], device=q.device) < (s["length"] - c["shared"]).view(G, W, 1, 1, 1)
    z = torch.cat([z0, z1.masked_fill(~there, float("-inf"))], -1) / math.sqrt(d)
    e = torch.exp(z - z.amax(-1, keepdim=True))
    p = e / e.sum(-1, keepdim=True)
    o0 = torch.matmul(p[..., :c["shared"]].transpose(1, 2).reshape(G, kv, W * group, -1), V).view(G, kv, W, group, d).transpose(1, 2)
    o1 = torch.matmul(p[..., c["shared"]:].reshape(G * W, kv, group, -1), Vo).view(G, W, kv, group, d)
    return (o0 + o1).reshape(G * W, c["heads"], d)


def _plain_select(s):
    c = s["c"]
    V = c["vocab"]
    z = s["logits"].double() / c["tau"]     # (continuations of different beams are ranked against one another)
    m = z.amax(-1, keepdim=True)
    total = s["scores"].double()[..., None] + (z - m - torch.log(torch.exp(z - m).sum(-1, keepdim=True)))
    ended = s["ended"][..., None] != 0
    stays = torch.arange(V, device=z.device) == s["end"]
    total = torch.where(ended, torch.where(stays, s["scores"].double()[..., None], float("-inf")), total)
    best, at = torch.sort(total.flatten(1), dim=1, descending=True, stable=True)
    best, at = best[:, :c["n_out"]], at[:, :c["n_out"]]
    tokens, parents = at % V, at // V
    over = (s["ended"].gather(1, parents) != 0) | (tokens == s["end"])
    return {"scores": best.float(), "tokens": tokens.int(), "parents": parents.int(), "ended": over.int()}


def _plain_reorder(s):
    c = s["c"]
    G, W, page = c["groups"], c["width"], c["page"]
    parents, table = s["parents"].long(), s["table"].view(G, W, -1)
    slot = torch.arange(W, device=parents.device)
    same = parents[:, :, None] == parents[:, None, :]
    first = ~(same & (slot[None, :] < slot[:, None])).any(2)                 # a row's first child keeps the row
    free = (~(parents[:, :, None] == slot).any(1)).int().sort(dim=1, descending=True, stable=True).indices
    row = torch.where(first, parents, free.gather(1, (~first).long().cumsum(1).sub(1).clamp(min=0)))   # further children: the rows without a child, in order
    length = s["length"].view(G, W)[:, :1].long()
    at = length // page                                                      # the entry that is being filled
    entry = torch.arange(table.shape[2], device=parents.device)
    of_parent = table.gather(1, parents[..., None].expand_as(table))
    of_row = table.gather(1, row[..., None].expand_as(table))
    out = torch.where(entry < at[..., None], of_parent, of_row)
    source, target = (x.gather(2, at[..., None].expand(G, W, 1))[..., 0].flatten().long() for x in (of_parent, of_row))
    filled = (torch.arange(page, device=parents.device) < (length % page).expand(G, W).reshape(-1, 1))[None, :, None, :, None]
    for pool in (s["K"], s["V"]):
        pool[:, target] = torch.where(filled, pool[:, source], pool[:, target])
    return {"K": s["K"], "V": s["V"], "table": out.view(G * W, -1)}


def run(state):
    op = state["c"]["op"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "select": _own_select, "reorder": _own_reorder}[op](state)
    return {"append": _plain_append, "attend": _plain_attend, "select": _plain_select, "reorder": _plain_reorder}[op](state)


# ------------------------------------------------------------------ bytes and operations
def work(case):
    c = case
    if c["op"] == "select":
        rows = c["groups"] * (c["n_in"] - c["ended"])     # an ended beam's logits are not needed
        return {"bytes": rows * c["vocab"] * BYTES[c["dtype"]] + 8 * c["groups"] * c["n_in"] + 16 * c["groups"] * c["n_out"], "flops": 4 * rows * c["vocab"]}
    el, kv, d = BYTES[c["dtype"]], c["kv_heads"], c["d_head"]
    if c["op"] == "append":
        return {"bytes": c["tokens"] * (d * (8 * c["heads"] + 8 * kv + 2 * kv * el) + 12), "flops": 3 * c["tokens"] * d * (c["heads"] + kv)}
    if c["op"] == "attend":
        owns = _own_lengths(c)
        positions = c["groups"] * c["shared"] + sum(owns)
        return {"bytes": positions * kv * d * 2 * el + 8 * len(owns) * c["heads"] * d, "flops": 4 * c["heads"] * d * sum(c["shared"] + o for o in owns)}
    rows = sum(n % c["page"] for n in _lengths(c)) * (c["width"] - c["alive"])
    entries = max(_lengths(c)) // c["page"] + 2
    return {"bytes": rows * c["layers"] * kv * d * el * 4 + 8 * c["groups"] * c["width"] * (entries + 1), "flops": 0}


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_append(s):
    c = s["c"]
    K, V, q = s["K"].double(), s["V"].double(), s["q_out"].double()
    seq, pos, table = s["seq"].cpu(), s["pos"].cpu(), s["table"].cpu()
    n, half = c["tokens"], c["d_head"] // 2
    freq = torch.tensor([THETA ** (-2.0 * i / c["d_head"]) for i in range(half)], dtype=torch.float64, device="cuda")
    wheel = torch.polar(torch.ones(n, half, dtype=torch.float64, device="cuda"), pos[:n].double().cuda()[:, None] * freq)[:, None]
    turn = lambda x: torch.view_as_real(torch.view_as_complex(x[:n].double().unflatten(2, (half, 2)).contiguous()) * wheel).flatten(2)  # noqa: E731
    flat = torch.tensor([int(table[seq[i], pos[i] // c["page"]]) for i in range(n)], device="cuda")
    row = (pos[:n] % c["page"]).long().cuda()
    K[flat, :, row], V[flat, :, row], q[:n] = turn(s["k"]), s["v"][:n].double(), turn(s["q"])
    return {"K": K, "V": V, "q": q}


def _exact_attend(s):
    c = s["c"]
    group, out = c["heads"] // c["kv_heads"], []
    for i, n in enumerate(s["length"].tolist()):
        lead = s["table"][i - i % c["width"]]
        p = torch.arange(n, device="cuda")
        at = torch.where(p < c["shared"], lead[p // c["page"]], s["table"][i][p // c["page"]]).long()
        heads = []
        for h in range(c["kv_heads"]):
            k, v = (x[at, h, p % c["page"]].double() for x in (s["K"], s["V"]))
            heads.append(torch.softmax(s["q"][i, h * group:(h + 1) * group].double() @ k.T * c["d_head"] ** -0.5, -1) @ v)
        out.append(torch.cat(heads))
    return torch.stack(out)


def _exact_select(s):
    c, out = s["c"], []
    ended = s["ended"].tolist()
    for g in range(c["groups"]):
        found = []
        for b in range(c["n_in"]):
            score = s["scores"][g, b].double()
            if ended[g][b]:
                found.append(score[None])
            else:
                logp = torch.log_softmax(s["logits"][g, b].double() / c["tau"], 0)
                found.append(score + logp.topk(min(c["n_out"], c["vocab"])).values)
        out.append(torch.cat(found).sort(descending=True).values[:c["n_out"]])
    return {"scores": torch.stack(out), "tokens": None, "parents": None, "ended": None}


def _exact_reorder(s):
    c = s["c"]
    K, V = s["K"].double(), s["V"].double()
    parents, table, length = s["parents"].tolist(), s["table"].tolist(), s["length"].tolist()
    for g in range(c["groups"]):
        n = length[g * c["width"]]
        spare, taken = [w for w in range(c["width"]) if w not in parents[g]], set()
        for p in parents[g]:
            if p in taken:
                a, b = (table[g * c["width"] + w][n // c["page"]] for w in (p, spare.pop(0)))
                for pool in (K, V):
                    pool[:, b, :, :n % c["page"]] = pool[:, a, :, :n % c["page"]]
            taken.add(p)
    return {"K": K, "V": V, "table": None}


def exact(case, seed):
    made = {"append": _exact_append, "attend": _exact_attend, "select": _exact_select, "reorder": _exact_reorder}[case["op"]]
    return made(prepare(case, seed))
