"""The operators that take drafted tokens and prompts in chunks through a paged cache, as measurable cases.

A program that runs a model's products itself feeds each sequence a chunk of new tokens per step: a piece
of its prompt, one token, or one token and the drafts behind it.  Four operators of
`paper_2405_18400_amd` take such a batch through a step:

  write    keys and values of new tokens go into an 8-bit paged cache with a scale per position and head,
           rotated on the way, with the queries of the same tokens (`spd_op_append_paged_q8`); what is
           held in 8 bits is then read back (`spd_op_read_paged`)
  read     cached positions come back as rows (`spd_op_read_paged`)
  attend   causal attention of every sequence's new tokens over its cached positions
           (`spd_op_attention_paged`)
  verify   which drafted tokens stand, by the target's and the drafter's probabilities and given random
           numbers, and the token behind them (`spd_op_verify_drafts`)

A paged cache is K and V [pages, key/value heads, page size, d_head] and a table [sequences, entries]
of page numbers; an 8-bit cache ("int8") has scales [pages, key/value heads, page size] besides: a value
is its code times its row's scale.  Sequence s has the new tokens first[s] .. first[s + 1] - 1.  Head
layouts are those of the 7B, 13B and 70B shapes of the benchmark.

`own` false: the plain form, elementary operations in 32 bits (64 for angles, for what is rounded to a
code or compared with a random number).  `own` true: the library.
"""
import math

import torch

own = False

TORCH = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2, "int8": 1}
THETA = 10000.0


def listed():
    return [
        # one decoding step of four sequences of a 7B model: the smallest call, nothing but latency
        {"name": "write-step", "op": "write", "heads": 32, "kv_heads": 32, "d_head": 128, "page": 16, "seqs": 4, "tokens": 4, "pad": 0, "start": 70},
        # prompts of uneven lengths in one call, padded behind the last, far into their texts: grouped heads of a 70B model
        {"name": "write-prompts", "op": "write", "heads": 64, "kv_heads": 8, "d_head": 128, "page": 64, "seqs": 7, "tokens": 4099, "pad": 61, "start": 30011},
        # the newest positions of a few sequences, for a program that looks at what it has cached
        {"name": "read-step", "op": "read", "dtype": "int8", "out": "fp32", "kv_heads": 32, "d_head": 128, "page": 16, "seqs": 4, "tokens": 20, "pad": 0, "start": 70},
        # long documents moved out of an 8-bit cache to 16 bits
        {"name": "read-long", "op": "read", "dtype": "int8", "out": "fp16", "kv_heads": 8, "d_head": 128, "page": 64, "seqs": 3, "tokens": 60001, "pad": 7, "start": 0},
        # one decoding step of four sequences of a 7B model behind a 64-token prompt: latency
        {"name": "attend-step", "op": "attend", "dtype": "fp16", "io": "fp32", "heads": 32, "kv_heads": 32, "d_head": 128, "page": 16, "seqs": 4, "tokens": 4, "past": 73, "ones": 0, "pad": 0},
        # one token and some drafts of eight sequences of a 70B model over an 8-bit cache of four thousand positions
        {"name": "attend-drafts", "op": "attend", "dtype": "int8", "io": "fp32", "heads": 64, "kv_heads": 8, "d_head": 128, "page": 64, "seqs": 8, "tokens": 40, "past": 4001, "ones": 0, "pad": 3},
        # three prompts of a 7B model from their beginnings, in 16 bits throughout
        {"name": "attend-prompts", "op": "attend", "dtype": "bf16", "io": "bf16", "heads": 32, "kv_heads": 32, "d_head": 128, "page": 16, "seqs": 3, "tokens": 2999, "past": 0, "ones": 0, "pad": 0},
        # a chunk of a very long prompt of a 70B model
        {"name": "attend-chunk", "op": "attend", "dtype": "fp16", "io": "fp32", "heads": 64, "kv_heads": 8, "d_head": 128, "page": 128, "seqs": 1, "tokens": 512, "past": 32257, "ones": 0, "pad": 0},
        # eight sequences that decode and one that is still at its prompt, in one call
        {"name": "attend-mixed", "op": "attend", "dtype": "int8", "io": "bf16", "heads": 32, "kv_heads": 8, "d_head": 128, "page": 32, "seqs": 9, "tokens": 708, "past": 2003, "ones": 8, "pad": 60},
        # two prompts of a 13B model with the library's default fp32 cache
        {"name": "attend-fp32", "op": "attend", "dtype": "fp32", "io": "fp32", "heads": 40, "kv_heads": 40, "d_head": 128, "page": 32, "seqs": 2, "tokens": 261, "past": 500, "ones": 0, "pad": 0},
        # four drafts of one sequence, drawn from a drafter's distribution
        {"name": "verify-step", "op": "verify", "dtype": "fp32", "seqs": 1, "tokens": 5, "vocab": 32000, "drawn": 1, "tau": 1.0, "pad": 0},
        # a batch of 32 sequences with uneven numbers of drafts, a large vocabulary, logits in 16 bits
        {"name": "verify-batch", "op": "verify", "dtype": "bf16", "seqs": 32, "tokens": 190, "vocab": 131072, "drawn": 1, "tau": 0.8, "pad": 2},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "read", "attend", "attend", "attend", "attend", "verify", "verify"])
    if op == "verify":
        seqs, vocab = _log(rng, 1, 64), _log(rng, 50, 131072)
        tokens = seqs + rng.randrange(0, 8 * seqs + 1)
        while tokens * vocab > 20_000_000:
            seqs, tokens = max(1, seqs // 2), max(1, seqs // 2, tokens // 2)
        return {"op": op, "dtype": rng.choice(["fp32", "bf16", "bf16", "fp16"]), "seqs": seqs, "tokens": tokens, "vocab": vocab, "drawn": rng.choice([0, 1, 1]),
                "tau": round(rng.uniform(0.3, 1.5), 3), "pad": rng.choice([0, 0, 5])}
    kv = rng.choice([1, 2, 4, 8, 8, 32, 40])
    heads = kv * rng.choice([1, 1, 2, 3, 4, 8] if kv <= 8 else [1])
    d, page = rng.choice([64, 128, 128, 256]), rng.choice([8, 16, 32, 64, 128])
    pad = rng.choice([0, 0, 1, 77])
    if op != "attend":
        seqs = _log(rng, 1, 40)
        tokens = _log(rng, seqs, 40 + 12_000_000 // ((heads + kv) * d + 1000))
        case = {"op": op, "kv_heads": kv, "d_head": d, "page": page, "seqs": seqs, "tokens": tokens, "pad": pad, "start": _log(rng, 1, 100_000)}
        if op == "write":
            return {**case, "heads": heads}
        return {**case, "dtype": rng.choice(["int8", "int8", "fp16", "bf16", "fp32"]), "out": rng.choice(["fp32", "fp16", "bf16"])}
    dtype = rng.choice(["fp16", "bf16", "int8", "int8", "fp32"])
    io = rng.choice({"fp32": ["fp32"], "int8": ["fp32", "fp16", "bf16"]}.get(dtype, ["fp32", dtype]))
    seqs = _log(rng, 1, 24)
    tokens, past = seqs + _log(rng, 1, 2000) - 1, _log(rng, 1, 30_000) if rng.random() < 0.85 else 0
    most = 2e10 if dtype == "fp32" else 1e11
    while (past + tokens) * tokens * heads * d * 4 > most and tokens > seqs:
        tokens = max(seqs, tokens // 2)
    while ((past + tokens) * seqs * kv * d > 60_000_000 or (past + tokens) * tokens * heads * d * 4 > most) and past > 1:
        past = past // 2
    return {"op": op, "dtype": dtype, "io": io, "heads": heads, "kv_heads": kv, "d_head": d, "page": page, "seqs": seqs, "tokens": tokens, "past": past,
            "ones": rng.choice([0, 0, seqs // 2]), "pad": pad}


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


def _news(c):
    """New tokens of each sequence: `ones` sequences have one, the others uneven shares of the rest."""
    ones = c.get("ones", 0)
    return [1] * ones + _spread(c["tokens"] - ones, c["seqs"] - ones)


def _pasts(c):
    """Uneven numbers of positions cached before, the most `past`."""
    return [c["past"] - (5 * i) * (c["past"] // 37 + 1) % (c["past"] // 2 + 1) for i in range(c["seqs"])]


def _firsts(news):
    at = [0]
    for n in news:
        at.append(at[-1] + n)
    return at


def _pool(g, c, pages):
    """Keys and values as a model's; an 8-bit pool has codes and scales that such rows are rounded to."""
    shape = (pages, c["kv_heads"], c["page"], c["d_head"])
    if c["dtype"] != "int8":
        return {"K": _normal(g, shape, TORCH[c["dtype"]]), "V": _normal(g, shape, TORCH[c["dtype"]])}
    out = {}
    for name in ("K", "V"):
        x = _normal(g, shape)
        scale = x.abs().amax(-1) / 127.0
        out[name] = (x / scale[..., None]).round_().to(torch.int8)
        out[name + "_scale"] = scale
    return out


def _table(g, rows, page):
    """Pages in any order for the entries [a, b) that each row needs; the others are none."""
    used = sum(b - a for a, b in rows)
    order = torch.randperm(used, generator=g, device="cuda").int()
    table = torch.full((len(rows), max(b for _, b in rows)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, (a, b) in enumerate(rows):
        table[s, a:b] = order[at:at + b - a]
        at += b - a
    return table, used


def _places(c, g):
    """Sequence and position of each token of a call that names them one by one, and the table."""
    shares, page = _spread(c["tokens"], c["seqs"]), c["page"]
    seq, pos, rows = [], [], []
    for s, n in enumerate(shares):
        first = c["start"] + 3 * s
        seq += [s] * n
        pos += range(first, first + n)
        rows.append((first // page, (first + n - 1) // page + 1))
    table, pages = _table(g, rows, page)
    return _ints(seq + [-1] * c["pad"]), _ints(pos + [0] * c["pad"]), table, pages


def _prepare_write(c, g):
    seq, pos, table, pages = _places(c, g)
    n, h, kv, d = len(seq), c["heads"], c["kv_heads"], c["d_head"]
    qkv = _normal(g, (n, (h + 2 * kv) * d))   # the rows that one product makes of a token
    q, k, v = qkv.split([h * d, kv * d, kv * d], 1)
    zeros = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    return {"c": c, "K": zeros(pages, kv, c["page"], d, dtype=torch.int8), "V": zeros(pages, kv, c["page"], d, dtype=torch.int8), "K_scale": zeros(pages, kv, c["page"]),
            "V_scale": zeros(pages, kv, c["page"]), "table": table, "q": q.unflatten(1, (h, d)), "k": k.unflatten(1, (kv, d)), "v": v.unflatten(1, (kv, d)), "seq": seq, "pos": pos,
            "q_out": zeros(n, h, d), "k_out": zeros(n, kv, d), "v_out": zeros(n, kv, d)}


def _prepare_read(c, g):
    seq, pos, table, pages = _places(c, g)
    shape = (len(seq), c["kv_heads"], c["d_head"])
    return {"c": c, **_pool(g, c, pages), "table": table, "seq": seq, "pos": pos, "k_out": torch.zeros(shape, dtype=TORCH[c["out"]], device="cuda"),
            "v_out": torch.zeros(shape, dtype=TORCH[c["out"]], device="cuda")}


def _prepare_attend(c, g):
    news, pasts = _news(c), _pasts(c)
    lengths = [p + n for p, n in zip(pasts, news)]
    table, pages = _table(g, [(0, (n - 1) // c["page"] + 1) for n in lengths], c["page"])
    shape = (c["tokens"] + c["pad"], c["heads"], c["d_head"])
    return {"c": c, **_pool(g, c, pages), "table": table, "q": _normal(g, shape, TORCH[c["io"]]), "first": _ints(_firsts(news)), "length": _ints(lengths),
            "out": torch.zeros(shape, dtype=TORCH[c["io"]], device="cuda")}


def _prepare_verify(c, g):
    rows, V, kind = c["tokens"] + c["pad"], c["vocab"], TORCH[c["dtype"]]
    # logits of a trained model: a few likely tokens above a broad rest; a drafter that is near to it
    common = _normal(g, (rows, V), std=2.5)
    target = (common + _normal(g, (rows, V), std=0.5)).to(kind)
    drafter = (common + _normal(g, (rows, V), std=0.5)).to(kind)
    u = torch.rand(rows, device="cuda", generator=g)
    # row j of a sequence is what follows its token j, so the draft at j + 1 is drawn from the drafter's row j (or is the drafter's best)
    scores = drafter.float() / c["tau"]
    if c["drawn"]:
        scores -= torch.rand(rows, V, device="cuda", generator=g).clamp_(1e-7, 1.0 - 1e-7).log_().neg_().log_()
    drafts = scores.argmax(-1).int()
    tokens = torch.cat([torch.randint(0, V, (1,), device="cuda", generator=g).int(), drafts[:-1]])
    return {"c": c, "logits": target, "draft_logits": drafter if c["drawn"] else None, "tokens": tokens, "first": _ints(_firsts(_news(c))), "u": u,
            "out_tokens": torch.zeros(rows, dtype=torch.int32, device="cuda"), "out_logprobs": torch.zeros(rows, device="cuda"),
            "out_accepted": torch.zeros(c["seqs"], dtype=torch.int32, device="cuda")}


def prepare(case, seed):
    make = {"write": _prepare_write, "read": _prepare_read, "attend": _prepare_attend, "verify": _prepare_verify}[case["op"]]
    return make(dict(case), _generator(seed))


# ------------------------------------------------------------------ the library's operators
def _own_write(s):
    import paper_2405_18400_amd as pkg
    pkg.spd_op_append_paged_q8(s["K"], s["V"], s["K_scale"], s["V_scale"], s["table"], s["k"], s["v"], s["seq"], s["pos"], THETA, q=s["q"], q_out=s["q_out"])
    pkg.spd_op_read_paged("int8", s["K"], s["V"], s["table"], s["seq"], s["pos"], s["k_out"], s["v_out"], K_scale=s["K_scale"], V_scale=s["V_scale"])
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _own_read(s):
    import paper_2405_18400_amd as pkg
    pkg.spd_op_read_paged(s["c"]["dtype"], s["K"], s["V"], s["table"], s["seq"], s["pos"], s["k_out"], s["v_out"], K_scale=s.get("K_scale"), V_scale=s.get("V_scale"))
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_attend(s):
    import paper_2405_18400_amd as pkg
    c = s["c"]
    news = _news(c)
    pkg.spd_op_attention_paged(c["dtype"], s["q"], s["K"], s["V"], s["table"], s["first"], s["length"], s["out"], max(news), max(p + n for p, n in zip(_pasts(c), news)),
                               K_scale=s.get("K_scale"), V_scale=s.get("V_scale"))
    return s["out"]


def _own_verify(s):
    import paper_2405_18400_amd as pkg
    c = s["c"]
    pkg.spd_op_verify_drafts(c["dtype"], s["logits"], s["tokens"], s["first"], s["u"], s["out_tokens"], s["out_logprobs"], s["out_accepted"], tau=c["tau"],
                             draft_logits=s["draft_logits"], draft_tau=c["tau"])
    return {"tokens": s["out_tokens"], "logprobs": s["out_logprobs"], "accepted": s["out_accepted"]}


# ------------------------------------------------------------------ the plain forms
def _turned(x, pos):
    d = x.shape[-1]
    angle = pos.double()[:, None] * THETA ** (-torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / d)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x[..., 0::2].double(), x[..., 1::2].double()
    return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)


def _codes(x):
    """Codes and scales of rows (in 64 bits: a value half-way between two codes)."""
    scale = (x.abs().amax(-1) / 127.0).float()
    code = (x / torch.where(scale > 0, scale, 1.0).double()[..., None]).round().clamp(-127, 127)
    return code.to(torch.int8), scale


def _at(s, n):
    seq, pos, page = s["seq"][:n].long(), s["pos"][:n].long(), s["c"]["page"]
    return s["table"][seq, pos // page].long(), pos % page


def _plain_write(s):
    n = s["c"]["tokens"]                    # tokens behind them are padding
    at, row = _at(s, n)
    for name, x in (("K", _turned(s["k"][:n], s["pos"][:n])), ("V", s["v"][:n].double())):
        code, scale = _codes(x)
        s[name][at, :, row] = code
        s[name + "_scale"][at, :, row] = scale
        s[name.lower() + "_out"][:n] = s[name][at, :, row].float() * s[name + "_scale"][at, :, row][..., None]
    s["q_out"][:n] = _turned(s["q"][:n], s["pos"][:n]).float()
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _plain_read(s):
    n = s["c"]["tokens"]
    at, row = _at(s, n)
    for name in ("K", "V"):
        x = s[name][at, :, row].float()
        if name + "_scale" in s:
            x = x * s[name + "_scale"][at, :, row][..., None]
        s[name.lower() + "_out"][:n] = x.to(s["k_out"].dtype)
    return {"k": s["k_out"], "v": s["v_out"]}


def _cached(s, name, row, count):
    """Positions 0 .. count - 1 of a sequence: [key/value heads, count, d_head] in 32 bits."""
    p, page = torch.arange(count, device="cuda"), s["c"]["page"]
    at = s["table"][row][p // page].long()
    x = s[name][at, :, p % page].float()
    if name + "_scale" in s:
        x = x * s[name + "_scale"][at, :, p % page][..., None]
    return x.transpose(0, 1)


def _plain_attend(s):
    c = s["c"]
    kv, d = c["kv_heads"], c["d_head"]
    group, at = c["heads"] // kv, 0
    for i, (n, past) in enumerate(zip(_news(c), _pasts(c))):
        K, V = _cached(s, "K", i, past + n), _cached(s, "V", i, past + n)
        q = s["q"][at:at + n].float().view(n, kv, group, d).permute(1, 2, 0, 3).reshape(kv, group * n, d)
        z = torch.matmul(q, K.transpose(1, 2)).div_(math.sqrt(d)).view(kv, group, n, past + n)
        hidden = torch.arange(past + n, device="cuda") > torch.arange(past, past + n, device="cuda")[:, None]
        z.masked_fill_(hidden, float("-inf"))
        e = z.sub_(z.amax(-1, keepdim=True)).exp_()
        p = e.div_(e.sum(-1, keepdim=True)).view(kv, group * n, past + n)
        o = torch.matmul(p, V).view(kv, group, n, d).permute(2, 0, 1, 3).reshape(n, c["heads"], d)
        s["out"][at:at + n] = o.to(s["out"].dtype)
        at += n
    return s["out"]


def _softmax(logits, tau):
    z = logits.double() / tau
    e = torch.exp(z - z.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _plain_verify(s):
    c = s["c"]
    n, V = c["tokens"], c["vocab"]
    news = torch.tensor(_news(c), device="cuda")
    first, last = s["first"][:-1].long(), s["first"][1:].long() - 1
    place = torch.arange(n, device="cuda")
    seq = torch.repeat_interleave(torch.arange(c["seqs"], device="cuda"), news, output_size=n)
    step = place - first[seq]
    p = _softmax(s["logits"][:n], c["tau"])             # (64 bits: probabilities next to a random number)
    draft = torch.cat([s["tokens"][1:n], s["tokens"][:1]]).long()                       # the draft that row j is asked about: the token behind it
    of_p = p.gather(1, draft[:, None])[:, 0]
    of_q = torch.ones_like(of_p)
    if s["draft_logits"] is not None:
        q = _softmax(s["draft_logits"][:n], c["tau"])
        of_q = q.gather(1, draft[:, None])[:, 0]
    stands = (s["u"][:n].double() * of_q < of_p) & (place < last[seq])
    refused = torch.where(stands, n, step)              # a sequence's first row whose draft does not stand (its last row has none)
    accepted = torch.full((c["seqs"],), n, device="cuda").scatter_reduce(0, seq, refused, "amin")
    stop = first + accepted
    w, all_stand = p[stop], stop == last
    if s["draft_logits"] is not None:
        rest = (w - q[stop]).clamp(min=0.0)
    else:
        rest = w.scatter(1, draft[stop][:, None], 0.0)
    w = torch.where(all_stand[:, None] | (rest.sum(-1, keepdim=True) == 0), w, rest)
    total = w.cumsum(-1)
    bound = s["u"][last].double() * total[:, -1]
    chosen = (total <= bound[:, None]).sum(-1).clamp(max=V - 1)
    emitted = torch.where(place < stop[seq], draft, chosen[seq])
    given = step <= accepted[seq]
    s["out_tokens"][:n] = torch.where(given, emitted, -1).int()
    s["out_logprobs"][:n] = torch.where(given, p.gather(1, emitted[:, None])[:, 0].log(), 0.0).float()
    s["out_accepted"].copy_(accepted)
    return {"tokens": s["out_tokens"], "logprobs": s["out_logprobs"], "accepted": s["out_accepted"]}


def run(state):
    op = state["c"]["op"]
    if own:
        return {"write": _own_write, "read": _own_read, "attend": _own_attend, "verify": _own_verify}[op](state)
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend, "verify": _plain_verify}[op](state)


# ------------------------------------------------------------------ bytes and operations
def work(case):
    c = case
    if c["op"] == "verify":
        rows = c["tokens"] + (c["tokens"] - c["seqs"]) * c["drawn"]
        return {"bytes": rows * c["vocab"] * BYTES[c["dtype"]] + 16 * c["tokens"] + 8 * c["seqs"], "flops": 4 * rows * c["vocab"]}
    kv, d = c["kv_heads"], c["d_head"]
    if c["op"] == "write":                  # rows in and rotated, codes and scales out; codes and scales in again and rows out
        return {"bytes": c["tokens"] * (8 * d * c["heads"] + 8 * d * kv + 4 * kv * (d + 4) + 8 * d * kv + 12), "flops": c["tokens"] * d * (3 * c["heads"] + 9 * kv)}
    el = BYTES[c["dtype"]]
    row = kv * (d * el + (4 if c["dtype"] == "int8" else 0))
    if c["op"] == "read":
        return {"bytes": c["tokens"] * (2 * row + 2 * kv * d * BYTES[c["out"]] + 12), "flops": c["tokens"] * kv * d * 2}
    news, pasts = _news(c), _pasts(c)
    return {"bytes": sum(p + n for p, n in zip(pasts, news)) * 2 * row + 2 * c["tokens"] * c["heads"] * d * BYTES[c["io"]],
            "flops": 4 * c["heads"] * d * sum(n * p + n * (n + 1) // 2 for p, n in zip(pasts, news))}


# ------------------------------------------------------------------ the definition in 64 bits
def _flat_rows(s):
    c = s["c"]
    seq, pos, table = s["seq"].tolist(), s["pos"].tolist(), s["table"].tolist()
    return torch.tensor([table[seq[i]][pos[i] // c["page"]] * c["page"] + pos[i] % c["page"] for i in range(c["tokens"])], device="cuda")


def _exact_write(s):
    c = s["c"]
    n, half = c["tokens"], c["d_head"] // 2
    freq = torch.tensor([THETA ** (-2.0 * i / c["d_head"]) for i in range(half)], dtype=torch.float64, device="cuda")
    wheel = torch.polar(torch.ones(n, half, dtype=torch.float64, device="cuda"), s["pos"][:n].double()[:, None] * freq)[:, None]
    turn = lambda x: torch.view_as_real(torch.view_as_complex(x[:n].double().unflatten(2, (half, 2)).contiguous()) * wheel).flatten(2)  # noqa: E731
    out = {"q": s["q_out"].double(), "k": s["k_out"].double(), "v": s["v_out"].double()}
    out["q"][:n] = turn(s["q"])
    for name, x in (("k", turn(s["k"])), ("v", s["v"][:n].double())):
        step = torch.linalg.vector_norm(x, ord=float("inf"), dim=2, keepdim=True).div(127).float().double()
        out[name][:n] = torch.round(x / step) * step
    return out


def _exact_read(s):
    at, out = _flat_rows(s), {}
    for name in ("K", "V"):
        x = s[name].transpose(1, 2).flatten(0, 1).index_select(0, at).double()
        if s["c"]["dtype"] == "int8":
            x *= s[name + "_scale"].transpose(1, 2).flatten(0, 1).index_select(0, at).double().unsqueeze(2)
        whole = s[name.lower() + "_out"].double()
        whole[:len(at)] = x
        out[name.lower()] = whole
    return out


def _exact_attend(s):
    c = s["c"]
    group, page, out, first, table = c["heads"] // c["kv_heads"], c["page"], s["out"].double(), s["first"].tolist(), s["table"].cpu()
    for i, n in enumerate(s["length"].tolist()):
        at = (table[i, torch.arange(n) // page].long() * page + torch.arange(n) % page).cuda()
        rows = slice(first[i], first[i + 1])
        new = first[i + 1] - first[i]
        for h in range(c["kv_heads"]):
            k, v = (s[x][:, h].reshape(-1, c["d_head"]).index_select(0, at).double() for x in ("K", "V"))
            if c["dtype"] == "int8":
                k, v = (y * s[x][:, h].reshape(-1).index_select(0, at).double()[:, None] for y, x in ((k, "K_scale"), (v, "V_scale")))
            for g in range(h * group, (h + 1) * group):
                scores = s["q"][rows, g].double() @ k.T * c["d_head"] ** -0.5
                out[rows, g] = torch.softmax(scores + torch.full_like(scores, -math.inf).triu_(n - new + 1), -1) @ v
    return out


def _exact_verify(s):
    c = s["c"]
    first, tokens, u = s["first"].tolist(), s["tokens"].tolist(), s["u"].tolist()
    out = s["out_logprobs"].double()
    for i in range(c["seqs"]):
        at, end = first[i], first[i + 1] - 1
        while True:
            logp = torch.log_softmax(s["logits"][at].double() / c["tau"], 0)
            logq = None if s["draft_logits"] is None or at == end else torch.log_softmax(s["draft_logits"][at].double() / c["tau"], 0)
            if at < end:
                x = tokens[at + 1]
                if u[at] < math.exp(min(0.0, float(logp[x] - (logq[x] if logq is not None else 0.0)))):
                    out[at] = logp[x]
                    at += 1
                    continue
            weight = logp.exp()
            if at < end and logq is not None:
                weight = torch.relu(weight - logq.exp())
            elif at < end:
                weight[tokens[at + 1]] = 0.0
            total = weight.cumsum(0)
            out[at] = logp[min(int(torch.searchsorted(total, total[-1:] * u[end], right=True)), c["vocab"] - 1)]
            break
    return {"tokens": None, "logprobs": out, "accepted": None}


def exact(case, seed):
    made = {"write": _exact_write, "read": _exact_read, "attend": _exact_attend, "verify": _exact_verify}[case["op"]]
    return made(prepare(case, seed))
