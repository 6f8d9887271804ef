"""The operators of chunks of new tokens over a paged cache against their definitions in 64 bits (chunk_reference.py)."""
import math

import pytest
import torch

import chunk_reference as R

pytestmark = pytest.mark.gpu

THETA = 10000.0
HALF_STEP = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


def P():
    import paper_2405_18400_amd as pkg
    return pkg


def say(*what):
    print(*what, flush=True)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def ints(x):
    return torch.as_tensor(x, dtype=torch.int32)


def zero():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def split(rows, heads, kv, d):
    q, k, v = rows.split([heads * d, kv * d, kv * d], 1)
    return q.unflatten(1, (heads, d)), k.unflatten(1, (kv, d)), v.unflatten(1, (kv, d))


def places(page, lengths, start, seed, pad=()):
    """A permuted table with entries that are no pages, and the tokens of `lengths` from `start` on, padding at the places `pad`: (pages, table, seq, pos)."""
    g = gen(seed)
    first = [start + 5 * s for s in range(len(lengths))]
    entries = max(a + n - 1 for a, n in zip(first, lengths)) // page + 1
    used = [(s, e) for s, (a, n) in enumerate(zip(first, lengths)) for e in range(a // page, (a + n - 1) // page + 1)]
    order = torch.randperm(len(used) + 2, generator=g)
    table = torch.full((len(lengths), entries), -7, dtype=torch.int32)
    for (s, e), p in zip(used, order):
        table[s, e] = int(p)
    tokens = [(s, p) for s, (a, n) in enumerate(zip(first, lengths)) for p in range(a, a + n)]
    for at in pad:
        tokens.insert(at, (-1, -1))
    return len(used) + 2, table, ints([s for s, _ in tokens]), ints([p for _, p in tokens])


def page_of(table, s, p, page, pages):
    at = int(table[s, p // page]) if 0 <= s < len(table) and 0 <= p < page * table.shape[1] else -1
    return at if 0 <= at < pages else -1


# ------------------------------------------------------------------ writing to 8 bits
def write(pages, table, seq, pos, rows, heads, kv, d, page, theta=THETA, stride=True):
    q, k, v = split(rows.cuda(), heads, kv, d)
    if not stride:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    K, V = (torch.full((pages, kv, page, d), x, dtype=torch.int8, device="cuda") for x in (77, -78))
    Ks, Vs = (torch.full((pages, kv, page), x, device="cuda") for x in (3.0, 4.0))
    q_out, err = (torch.full((len(seq), heads, d), 9.0, device="cuda") if heads else None), zero()
    P().spd_op_append_paged_q8(K, V, Ks, Vs, table.cuda(), k, v, seq.cuda(), pos.cuda(), theta, q=q if heads else None, q_out=q_out, err=err)
    return K.cpu(), V.cpu(), Ks.cpu(), Vs.cpu(), q_out.cpu() if heads else None, int(err)


def check_write(pages, table, seq, pos, rows, heads, kv, d, page, theta=THETA):
    K, V, Ks, Vs, q_out, err = write(pages, table, seq, pos, rows, heads, kv, d, page, theta)
    q, k, v = split(rows, heads, kv, d)
    wK, wV = torch.full_like(K, 77), torch.full_like(V, -78)
    wKs, wVs = torch.full_like(Ks, 3.0), torch.full_like(Vs, 4.0)
    bad = 0
    for t, (s, p) in enumerate(zip(seq.tolist(), pos.tolist())):
        at = page_of(table, s, p, page, pages)
        bad += s >= 0 and at < 0
        if at < 0:
            assert heads == 0 or (q_out[t] == 9.0).all(), t
            continue
        # Rotation in 64 bits, rounded once to fp32; the angle's own rounding, 2^-53 of up to 2^31, turns values by 2^-22 of themselves at most, at usual positions far less.
        turned = abs(p) * 2.0 ** -50
        if heads:
            want = R.rotate(q[t], p, theta)
            pair = q[t].unflatten(1, (d // 2, 2)).abs().sum(2).double().repeat_interleave(2, 1)
            assert ((q_out[t] - want).abs() <= want.abs() * 2.0 ** -24 + pair * turned + 2.0 ** -149).all(), t
        for got, scale, x, w, ws in ((K, Ks, R.rotate(R.finite(k[t]), p, theta), wK, wKs), (V, Vs, R.finite(v[t]).double(), wV, wVs)):
            code, step = R.quantise(x)
            c, st = got[at, :, p % page], scale[at, :, p % page]
            # (a scale next to a rounding border of fp32, or a code next to one between two codes, may go the other way: by a place, and by one where x / scale is nearer to the border than the angle's error)
            assert ((st - step).abs() <= step * 2.0 ** -23).all(), t
            slack = 127 * (turned + 2.0 ** -40)
            ratio = torch.where(step[:, None] > 0, x / step.double().clamp(min=1e-300)[:, None], 0.0)
            border = ((ratio - ratio.floor() - 0.5).abs() < slack) | ((st != step)[:, None] & ((ratio - ratio.floor() - 0.5).abs() < 127 * 2.0 ** -22))
            assert (((c.int() - code.int()).abs() == 0) | (border & ((c.int() - code.int()).abs() == 1))).all(), t
            w[at, :, p % page], ws[at, :, p % page] = c, st
    assert torch.equal(K, wK) and torch.equal(V, wV) and torch.equal(Ks, wKs) and torch.equal(Vs, wVs)     # everything else as it was
    assert err == int(bad > 0)
    return K, V, Ks, Vs


@pytest.mark.parametrize("heads,kv,d,page,lengths,start", [
    (4, 4, 128, 16, [1, 1, 1], 70), (8, 2, 64, 32, [5, 1, 40], 0), (3, 1, 256, 8, [17, 2], 30), (1, 1, 8, 4, [3], 2), (6, 3, 16, 1024, [9, 1], 1020), (40, 40, 128, 64, [3, 2], 63),
    (5, 5, 32, 4, [1], 0), (64, 8, 128, 16, [300], 1), (0, 2, 64, 16, [7, 5], 9)])
def test_write(heads, kv, d, page, lengths, start):
    say("write", heads, kv, d, page, lengths, start)
    pages, table, seq, pos = places(page, lengths, start, seed=d + page)
    check_write(pages, table, seq, pos, torch.randn(len(seq), (heads + 2 * kv) * d, generator=gen(d)), heads, kv, d, page)


def test_write_of_many_tokens_with_padding_between_and_behind():
    pages, table, seq, pos = places(16, [400, 1, 333], 11, seed=1, pad=(0, 17, 18, 500, 738, 739))
    check_write(pages, table, seq, pos, torch.randn(len(seq), 48 * 128, generator=gen(2)), 32, 8, 128, 16)


@pytest.mark.parametrize("start,theta", [(0, 1e4), (65535, 1e4), (1_000_003, 5e5)])
def test_write_far_positions(start, theta):
    pages, table, seq, pos = places(1024, [3, 2], start, seed=3)
    check_write(pages, table, seq, pos, torch.randn(5, 4 * 128, generator=gen(3)), 2, 1, 128, 1024, theta)


def test_write_the_farthest_positions():
    table = torch.full((1, 2 ** 31 // 1024), -1, dtype=torch.int32)
    table[0, -1] = 1
    check_write(3, table, ints([0, 0, 0]), ints([2 ** 31 - 1, 2 ** 31 - 1024, 2 ** 31 - 70]), torch.randn(3, 4 * 64, generator=gen(4)), 2, 1, 64, 1024)


def test_write_out_of_range():
    """Sequences, positions and pages out of range: those tokens are left out whole, the others are written."""
    pages, table, seq, pos = places(16, [6, 5], 30, seed=5)
    seq[1], seq[4], pos[6], pos[8] = 2, 2 ** 31 - 1, -1, 16 * table.shape[1]
    table[0, 2] = pages
    check_write(pages, table, seq, pos, torch.randn(11, 6 * 64, generator=gen(5)), 2, 2, 64, 16)


def test_write_of_what_is_no_number_and_of_what_is_very_small_or_large():
    """NaN counts as zero, an infinity as the largest number; rows of zeros, of numbers next to fp32's ends."""
    pages, table, seq, pos = places(16, [8], 0, seed=6)
    rows = torch.randn(8, 3 * 64, generator=gen(6))
    rows[0, 70], rows[1, 130], rows[2, 64:128], rows[3, 131] = math.nan, math.inf, 0.0, -math.inf
    rows[4, 64:] *= 1e-42
    rows[5, 64:] = 0.0
    rows[5, 190] = 1e-45
    rows[6, 64:] *= 1e37
    rows[7, 128:] = torch.arange(64) * 3.0 - 81.0       # codes half-way between two: steps of 3 / 2 ...
    rows[7, 191] = 127 * 6.0
    pos[:8] = ints([0, 1, 2, 3, 4, 5, 6, 7])
    K, V, Ks, Vs = check_write(pages, table, seq, pos, rows, 1, 1, 64, 16)
    at = int(table[0, 0])
    assert Ks[at, 0, 2] == 0 and (K[at, 0, 2] == 0).all() and (K[at, 0, 5] == 0).all() and Vs[at, 0, 7] == 6.0
    assert V[at, 0, 7, :4].tolist() == [-14, -13, -12, -12]                 # -13.5, -13, -12.5, -12: to even
    assert Vs[at, 0, 1] == torch.tensor(R.BIG / 127.0).float() and V[at, 0, 1, 2] == 127 and V[at, 0, 3, 3] == -127


def test_write_in_place_and_from_rows_of_their_own():
    pages, table, seq, pos = places(16, [9], 3, seed=7)
    rows = torch.randn(9, 8 * 64, generator=gen(7))
    want = write(pages, table, seq, pos, rows, 4, 2, 64, 16)
    got = write(pages, table, seq, pos, rows, 4, 2, 64, 16, stride=False)
    assert all(torch.equal(a, b) for a, b in zip(want[:5], got[:5]))
    q, k, v = (x.contiguous() for x in split(rows.cuda(), 4, 2, 64))
    K, V = (torch.zeros(pages, 2, 16, 64, dtype=torch.int8, device="cuda") for _ in range(2))
    Ks, Vs = (torch.zeros(pages, 2, 16, device="cuda") for _ in range(2))
    P().spd_op_append_paged_q8(K, V, Ks, Vs, table.cuda(), k, v, seq.cuda(), pos.cuda(), THETA, q=q, q_out=q)
    assert torch.equal(q.cpu(), want[4])


# ------------------------------------------------------------------ reading back
def pool(dtype, pages, kv, page, d, seed):
    g = gen(seed)
    if dtype == "int8":
        K, V = (torch.randint(-128, 128, (pages, kv, page, d), generator=g).to(torch.int8) for _ in range(2))
        return K, V, *(torch.rand(pages, kv, page, generator=g) + 0.01 for _ in range(2))
    K, V = (torch.randn(pages, kv, page, d, generator=g).to(R.TORCH[dtype]) for _ in range(2))
    return K, V, None, None


def dev(x):
    return None if x is None else x.cuda()


@pytest.mark.parametrize("dtype", ["int8", "fp16", "bf16", "fp32"])
@pytest.mark.parametrize("out", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("kv,d,page,lengths,start,pad", [(2, 64, 16, [5, 1, 40], 7, (0, 9, 48)), (3, 8, 4, [3], 0, ()), (1, 256, 64, [65], 63, (66,) * 0), (40, 128, 8, [9, 30], 3, (2,)),
                                                         (5, 16, 1024, [20], 1015, ())])
def test_read(dtype, out, kv, d, page, lengths, start, pad):
    say("read", dtype, out, kv, d, page, lengths, start, pad)
    pages, table, seq, pos = places(page, lengths, start, seed=page, pad=pad)
    table[0, start // page] = pages                        # out of range
    seq[-1], pos[-1] = seq[len(seq) // 2], pos[len(seq) // 2]     # a position named twice
    K, V, Ks, Vs = pool(dtype, pages, kv, page, d, seed=d)
    k_out, v_out = (torch.full((len(seq), kv, d), 5.0, dtype=R.TORCH[out], device="cuda") for _ in range(2))
    err, bad = zero(), 0
    P().spd_op_read_paged(dtype, K.cuda(), V.cuda(), table.cuda(), seq.cuda(), pos.cuda(), k_out, v_out, K_scale=dev(Ks), V_scale=dev(Vs), err=err)
    for t, (s, p) in enumerate(zip(seq.tolist(), pos.tolist())):
        at = page_of(table, s, p, page, pages)
        bad += s >= 0 and at < 0
        for got, x, scale in ((k_out, K, Ks), (v_out, V, Vs)):
            if at < 0:
                assert (got[t] == 5.0).all(), t
            else:                                         # (code x scale in 64 bits is exact: rounded to fp32, then to 16 bits, as the library does)
                y = x[at, :, p % page].float()
                y = y if scale is None else y * scale[at, :, p % page, None]
                assert torch.equal(got[t].cpu(), y.to(R.TORCH[out])), t
    assert int(err) == int(bad > 0) == 1


def test_read_out_of_range_and_nothing():
    pages, table, seq, pos = places(16, [4], 0, seed=1)
    K, V, Ks, Vs = pool("int8", pages, 2, 16, 64, seed=2)
    seq, pos = ints([1, 0, 0, -1, 0]), ints([0, -1, 16 * table.shape[1], 0, 2])
    outs = [torch.full((5, 2, 64), 5.0, device="cuda") for _ in range(2)]
    err = zero()
    P().spd_op_read_paged("int8", K.cuda(), V.cuda(), table.cuda(), seq.cuda(), pos.cuda(), *outs, K_scale=Ks.cuda(), V_scale=Vs.cuda(), err=err)
    assert int(err) == 1 and all((o[:4] == 5.0).all() for o in outs)
    assert torch.equal(outs[0][4].cpu(), K[table[0, 0], :, 2].float() * Ks[table[0, 0], :, 2, None])
    P().spd_op_read_paged("int8", K.cuda(), V.cuda(), table.cuda(), seq[:0].cuda(), pos[:0].cuda(), outs[0][:0], outs[1][:0], K_scale=Ks.cuda(), V_scale=Vs.cuda())


# ------------------------------------------------------------------ attention
def attention_case(dtype, io, heads, kv, d, page, news, pasts, seed, pad=0, std=1.0):
    """Pools of NaN (8 bits: of NaN scales) but for the positions that count; entries that no position needs are no pages."""
    g = gen(seed)
    lengths = [a + b for a, b in zip(news, pasts)]
    entries = (max(lengths + [1]) - 1) // page + 2
    n_seq = len(news)
    pages = n_seq * entries + 1
    order = torch.randperm(pages, generator=g)[:n_seq * entries].int().view(n_seq, entries)
    table = torch.full((n_seq, entries), -1, dtype=torch.int32)
    K, V = (torch.full((pages, kv, page, d), math.nan) for _ in range(2))
    for s, n in enumerate(lengths):
        used = (n - 1) // page + 1
        table[s, :used] = order[s, :used]
        for e in range(used):
            rows = min(page, n - e * page)
            K[order[s, e], :, :rows] = torch.randn(kv, rows, d, generator=g) * std
            V[order[s, e], :, :rows] = torch.randn(kv, rows, d, generator=g)
    scales = [None, None]
    if dtype == "int8":
        (K, ks), (V, vs) = (R.quantise(x.double().nan_to_num(0.0)) for x in (K, V))
        scales = [torch.where(x == 0, math.nan, x) for x in (ks, vs)]
        K, V = (torch.where(x.isnan()[..., None], torch.randint(-128, 128, y.shape, generator=g).to(torch.int8), y) for x, y in zip(scales, (K, V)))
    else:
        K, V = K.to(R.TORCH[dtype]), V.to(R.TORCH[dtype])
    q = torch.randn(sum(news) + pad, heads, d, generator=g).to(R.TORCH[io])
    first = [0]
    for n in news:
        first.append(first[-1] + n)
    return dict(q=q, K=K, V=V, table=table, first=ints(first), length=ints(lengths), K_scale=scales[0], V_scale=scales[1])


def attend(dtype, case, max_new=None, max_len=None, q=None):
    c = case
    out, err = torch.full(c["q"].shape, 7.0, dtype=c["q"].dtype, device="cuda"), zero()
    news = c["first"].diff().clamp(min=0)
    P().spd_op_attention_paged(dtype, c["q"].cuda() if q is None else q, c["K"].cuda(), c["V"].cuda(), c["table"].cuda(), c["first"].cuda(), c["length"].cuda(), out,
                               int(news.max()) if max_new is None else max_new, int(c["length"].max()) if max_len is None else max_len, K_scale=dev(c["K_scale"]), V_scale=dev(c["V_scale"]), err=err)
    return out.cpu(), int(err)


def check(dtype, case, bound=1e-5, **kw):
    """Rows of fp32: the difference against the largest of sum p |v| of the row.  fp32 sums of d_head products and of up to some thousand probabilities, about sqrt(terms) 2^-24 of the scale, scores of a
    few units: below 1e-5.  Rows of 16 bits: the probabilities are rounded to the type (int8: to fp16), half a step each, which is at most half a step of sum p |v| in all, and the
    result half a step of itself."""
    got, err = attend(dtype, case, **kw)
    assert err == 0
    want, size = R.attention(**case)
    mine = ~want[..., 0].isnan()
    assert (got[~mine] == 7.0).all()                            # rows that are no sequence's
    half = 0.0 if got.dtype is torch.float32 else torch.finfo(got.dtype).eps / 2
    got, want, size = got[mine].double(), want[mine], size[mine]
    if got.numel():
        worst = float(((got - want).abs() / (2 * half * size + bound * size.amax(-1, keepdim=True)).clamp(min=1e-30)).max())
        assert worst < 1


KINDS = [("fp16", "fp32"), ("fp16", "fp16"), ("bf16", "fp32"), ("bf16", "bf16"), ("int8", "fp32"), ("int8", "fp16"), ("int8", "bf16"), ("fp32", "fp32")]


@pytest.mark.parametrize("dtype,io", KINDS)
@pytest.mark.parametrize("heads,kv,d,page,news,pasts,pad", [
    (4, 4, 128, 16, [1, 1, 1, 1], [73, 69, 65, 64], 0),             # a step of four sequences
    (1, 1, 8, 4, [1], [0], 0),                                      # one position
    (8, 1, 64, 8, [2, 1, 7], [0, 0, 1], 2),                         # prompts from their beginnings
    (6, 2, 64, 16, [5, 0, 3, 1], [37, 16, 0, 100], 1),              # a sequence without new tokens; ends inside pages
    (16, 2, 128, 64, [4, 6], [200, 231], 0),                        # one tile of rows and a part
    (3, 3, 256, 16, [33, 2], [51, 83], 3), (10, 2, 16, 4, [12, 30], [9, 0], 0), (4, 2, 32, 8, [40], [3], 5), (2, 1, 32, 1024, [10, 3], [1020, 0], 0),
    (5, 5, 128, 32, [150], [129], 0), (34, 1, 128, 16, [3], [40], 0), (1, 1, 256, 128, [70], [300], 0), (8, 8, 64, 4, [1, 70], [500, 30], 0)])
def test_attention(dtype, io, heads, kv, d, page, news, pasts, pad):
    say("attention", dtype, io, heads, kv, d, page, news, pasts, pad)
    check(dtype, attention_case(dtype, io, heads, kv, d, page, news, pasts, seed=d + page, pad=pad))


@pytest.mark.parametrize("dtype,io", KINDS)
@pytest.mark.parametrize("heads,kv,d,page,news,pasts", [
    (8, 1, 128, 16, [1, 4], [1500, 2100]), (4, 2, 64, 32, [130, 1, 1], [700, 300, 1200]), (2, 2, 128, 128, [300], [400]), (4, 1, 256, 16, [6], [900]), (16, 2, 128, 64, [17, 40], [1301, 5]),
    (1, 1, 64, 4, [1], [5000]), (6, 3, 32, 1024, [1, 20], [2100, 1000])])
def test_attention_of_long_parts_and_many_rows(dtype, io, heads, kv, d, page, news, pasts):
    """Positions cut into several chunks, rows of queries past one tile, and both."""
    say("attention", dtype, io, heads, kv, d, page, news, pasts)
    check(dtype, attention_case(dtype, io, heads, kv, d, page, news, pasts, seed=news[0]))


@pytest.mark.parametrize("dtype,io", KINDS)
@pytest.mark.parametrize("page", [4, 8, 16])
@pytest.mark.parametrize("heads,kv,d,news,pasts", [(4, 2, 64, [3, 40], [70, 21]), (2, 2, 128, [5, 150], [601, 9]), (4, 1, 128, [2], [130]), (2, 1, 256, [90, 1], [33, 75]), (2, 2, 256, [2, 3], [61, 700])])
def test_attention_over_pages_shorter_than_a_waves_part_of_a_stage(dtype, io, page, heads, kv, d, news, pasts):
    """A wave brings 8 or 16 keys of a stage: on one page, on several, or several pages to one of its loads; tiles of 64 and 128 rows."""
    say("attention", dtype, io, page, heads, kv, d, news, pasts)
    check(dtype, attention_case(dtype, io, heads, kv, d, page, news, pasts, seed=d + page + 1, pad=1))


@pytest.mark.parametrize("dtype,io", KINDS)
@pytest.mark.parametrize("max_new,max_len", [(0, 1024), (1, 200), (1000, 173)])
def test_attention_bounds_size_the_launch_alone(dtype, io, max_new, max_len):
    """Too small or too large a max_new, more room in max_len than there is: the same up to the order of sums."""
    case = attention_case(dtype, io, 4, 2, 64, 16, [9, 60], [100, 113], seed=3)
    case["table"] = torch.cat([case["table"], torch.full((2, 64), -1, dtype=torch.int32)], 1)
    check(dtype, case, max_new=max_new, max_len=max_len)


@pytest.mark.parametrize("dtype,io,heads,kv,d,page", [("fp16", "fp32", 2, 1, 64, 16), ("int8", "bf16", 8, 2, 128, 16), ("bf16", "bf16", 3, 3, 32, 8), ("fp32", "fp32", 4, 2, 64, 64)])
@pytest.mark.parametrize("n_seq,long", [(64, 0), (65, 0), (130, 300), (200, 1700)])
def test_attention_of_many_sequences(dtype, io, heads, kv, d, page, n_seq, long):
    """One past what a wave looks at in one go, and many; no new tokens, one, a few and more than a tile of rows; long ones next to short ones."""
    say("attention", dtype, io, heads, kv, d, page, n_seq, long)
    g = gen(n_seq)
    news = [int(x) for x in torch.randint(0, 4, (n_seq,), generator=g)]
    pasts = [int(x) for x in torch.randint(0, 60, (n_seq,), generator=g)]
    news[0], news[-1], news[n_seq // 2], pasts[3] = 0, 2, 90, long
    check(dtype, attention_case(dtype, io, heads, kv, d, page, news, pasts, seed=n_seq, pad=3))


@pytest.mark.parametrize("dtype,io", [("fp16", "fp16"), ("int8", "fp32")])
def test_attention_of_many_sequences_with_firsts_and_lengths_out_of_range(dtype, io):
    case = attention_case(dtype, io, 2, 2, 64, 16, [2] * 80, [30] * 80, seed=9, pad=1)
    want, _ = attend(dtype, case)
    for where, what, value, rows, left in [("first", 70, 100, slice(0, 161), 7.0), ("length", 75, 1, slice(150, 152), 0.0), ("length", 3, 33, slice(6, 8), 0.0), ("first", 80, 162, slice(158, 161), 0.0),
                                           ("first", 0, -1, slice(0, 2), 0.0)]:
        changed = case[where].clone()
        changed[what] = value
        got, err = attend(dtype, {**case, where: changed}, max_new=2, max_len=32)
        keep = torch.ones(161, dtype=torch.bool)
        keep[rows] = False
        assert err == 1 and torch.equal(got[keep], want[keep]) and (got[rows] == left).all(), (where, what)


def test_attention_of_nothing():
    out = torch.full((3, 4, 64), 7.0, device="cuda")
    pools = (torch.zeros(1, 2, 16, 64, dtype=torch.float16, device="cuda"),) * 2
    P().spd_op_attention_paged("fp16", torch.zeros_like(out), *pools, ints([]).view(0, 1).cuda(), ints([0]).cuda(), ints([]).cuda(), out, 0, 0)
    P().spd_op_attention_paged("fp16", out[:0], *pools, ints([[0]]).cuda(), ints([0, 0]).cuda(), ints([5]).cuda(), out[:0].clone(), 0, 16)
    P().spd_op_attention_paged("fp16", torch.zeros_like(out), *pools, ints([[0]]).cuda(), ints([1, 1]).cuda(), ints([0]).cuda(), out, 0, 0)
    assert (out == 7.0).all()


@pytest.mark.parametrize("dtype,io", KINDS)
def test_attention_weights_add_up_to_one(dtype, io):
    """One key far above twenty thousand others, at weights near 2^-20: values of one come out as one (16 bits: to half a step of the largest weight and half a step of the result)."""
    n, d = 20_000, 64
    q = torch.zeros(8, 4, d)
    q[..., 0] = 8.0
    K = torch.zeros(n // 16, 1, 16, d)
    K[..., 0] = 0.25 * torch.rand(n // 16, 1, 16, generator=gen(14))
    K[700, 0, 3, 0] = 14.0                                   # 8 x 14 / 8 = 14 = 20.2 log 2
    V = torch.ones(n // 16, 1, 16, d)
    scales = (None, None)
    if dtype == "int8":
        (K, ks), (V, vs) = R.quantise(K.double()), R.quantise(V.double())
        scales = (ks, vs)
        one = vs.max() * 127
    else:
        K, V, one = K.to(R.TORCH[dtype]), V.to(R.TORCH[dtype]), 1.0
    case = dict(q=q.to(R.TORCH[io]), K=K, V=V, table=torch.arange(n // 16, dtype=torch.int32)[None], first=ints([0, 8]), length=ints([n]), K_scale=scales[0], V_scale=scales[1])
    got, err = attend(dtype, case)
    off = float((got.double() - one).abs().max())
    assert err == 0 and off <= (1e-6 if io == "fp32" else 2 * HALF_STEP[io])


@pytest.mark.parametrize("dtype,io", KINDS)
def test_attention_large_and_small_values(dtype, io):
    """Queries and keys far from one: scores of some hundreds (one key takes all), of 1e-6 (all alike), queries of very different sizes in one call."""
    case = attention_case(dtype, io, 4, 2, 64, 16, [7, 70], [80, 5], seed=6, std=3.0)
    sizes = [1e-3, 1.0, 40.0, 1e-4] if io == "fp16" else [1e-7, 1.0, 40.0, 1e-30]
    case["q"] = (case["q"].float() * torch.tensor(sizes).view(1, 4, 1)).to(R.TORCH[io])
    got, err = attend(dtype, case)
    want, size = R.attention(**case)
    half = 0.0 if io == "fp32" else HALF_STEP[io]
    assert err == 0
    for h, bound in ((0, 3e-5), (1, 3e-5), (3, 3e-5), (2, 2e-3)):        # (a score's fp32 sum is off by sqrt(64) 2^-24 of q k / 8, 1000 at the largest: 5e-4 in an exponent)
        off = (got[:, h].double() - want[:, h]).abs()
        assert (off <= 2 * half * size[:, h] + bound * size[:, h].amax(-1, keepdim=True)).all(), h


@pytest.mark.parametrize("dtype", ["int8", "fp16", "bf16", "fp32"])
def test_attention_over_values_and_scales_of_any_size(dtype):
    """Values next to the type's ends, rows of an 8-bit cache whose scales differ by 2^60: as near as the largest that counts."""
    case = attention_case(dtype, "fp32", 2, 1, 64, 16, [3, 40], [90, 20], seed=8)
    if dtype == "int8":
        for s in ("K_scale", "V_scale"):
            power = torch.randint(-40, 21, case["V_scale"].shape, generator=gen(9)) if s == "V_scale" else torch.randint(-6, 1, case["V_scale"].shape, generator=gen(10))
            case[s] = case[s] * 2.0 ** power
    else:
        case["V"] = (case["V"].float() * {"fp16": 12000.0, "bf16": 2.0 ** 125, "fp32": 2.0 ** 125}[dtype]).to(case["V"].dtype)
    check(dtype, case)


@pytest.mark.parametrize("dtype,io", KINDS)
def test_attention_sees_what_is_no_number_only_where_it_counts(dtype, io):
    """A NaN or an infinity in a value, a key or a scale: the rows at and behind its position alone, a value's in its feature; an infinite query: its own row."""
    news, pasts, past = [40, 6, 3], [50, 20, 9], 50
    case = attention_case(dtype, io, 4, 2, 128, 16, news, pasts, seed=7)
    clean, err = attend(dtype, case)
    page = lambda s, p: (int(case["table"][s, p // 16]), p % 16)  # noqa: E731
    spoilt = torch.zeros(clean.shape, dtype=torch.bool)
    if dtype == "int8":
        a, b = page(0, past + 21)
        case["V_scale"][a, 1, b] = math.nan
        spoilt[21:40, 2:] = True
        a, b = page(1, 22)
        case["V_scale"][a, 0, b] = math.inf
        spoilt[42:46, :2] = True
    else:
        a, b = page(0, past + 21)
        case["V"][a, 1, b, 5] = math.nan
        spoilt[21:40, 2:, 5] = True
        a, b = page(1, 22)
        case["V"][a, 0, b, 77] = math.inf
        spoilt[42:46, :2, 77] = True
    a, b = page(0, past + 30)
    (case["K"] if dtype != "int8" else case["K_scale"])[(a, 0, b, 3) if dtype != "int8" else (a, 0, b)] = math.nan
    spoilt[30:40, :2] = True
    case["q"][47, 1, 3] = math.inf
    spoilt[47, 1] = True
    got, err = attend(dtype, case)
    same, fine = bool(torch.equal(got[~spoilt], clean[~spoilt])), torch.isfinite(got)
    assert err == 0 and same
    seen = [bool(fine[21:40, 2:, 5].any()), bool(fine[42:46, :2, 77].any()), bool(fine[30:40, :2].any()), bool(fine[47, 1].all())]
    assert seen == [False] * 4


@pytest.mark.parametrize("dtype,io", [("fp16", "fp32"), ("int8", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("heads,past", [(2, 40), (16, 40), (2, 1500)])
def test_attention_with_lengths_firsts_and_pages_out_of_range(dtype, io, heads, past):
    case = attention_case(dtype, io, heads, 2, 64, 16, [3, 5, 2, 4], [past, past - 7, past // 2, 0], seed=4)
    want, _ = attend(dtype, case)
    longest = int(case["length"].max())

    def differs(rows, zero_rows=None, **changed):
        c = {**case, **changed}
        got, err = attend(dtype, c, max_new=5, max_len=longest)
        keep = torch.ones(14, dtype=torch.bool)
        keep[rows] = False
        assert err == 1 and torch.equal(got[keep], want[keep])
        if zero_rows is not None:
            assert (got[zero_rows] == 0).all()
        return got

    length = case["length"].clone()
    for bad in (4, -1, longest + 1, 2 ** 31 - 1):                # below its new tokens, negative, past the bound
        length[1] = bad
        differs(slice(3, 8), slice(3, 8), length=length)
    first = case["first"].clone()
    first[4] = 15                                               # passes n_tokens
    differs(slice(10, 14), first=first)
    first = case["first"].clone()
    first[2] = 2                                                # descends: there is no telling whose rows are whose, none is written
    assert (differs(slice(0, 14), first=first) == 7.0).all()
    first = case["first"].clone()
    first[0] = -1
    differs(slice(0, 3), first=first)
    for bad in (-1, len(case["K"]), 2 ** 31 - 1, -2 ** 31):
        table = case["table"].clone()
        table[0, 1] = bad
        got = differs(slice(0, 3), table=table)
        hole, size = R.attention(**{**case, "table": table})
        off = (got[:3].double() - hole[:3]).abs()
        assert (off <= (0 if io == "fp32" else 2 * HALF_STEP[io]) * size[:3] + 1e-5 * size[:3].amax(-1, keepdim=True)).all()
    table = case["table"].clone()
    table[3] = -1                                                # no position at all: zeros
    differs(slice(10, 14), slice(10, 14), table=table)


@pytest.mark.parametrize("io", ["fp32", "fp16"])
def test_attention_of_query_rows_that_lie_apart(io):
    case = attention_case("fp16", io, 4, 2, 64, 16, [9, 30], [20, 0], seed=5)
    want, _ = attend("fp16", case)
    rows = torch.full((39, 4 * 64 + 24), math.nan, dtype=R.TORCH[io], device="cuda")
    rows[:, :256] = case["q"].flatten(1).cuda()
    got, _ = attend("fp16", case, q=rows[:, :256].unflatten(1, (4, 64)))
    assert torch.equal(got, want)


def test_attention_offsets_past_32_bits():
    """Pools of more than 2^32 bytes, positions on their last pages."""
    pages, kv, page, d = 70_000, 4, 64, 128
    K, V = (torch.zeros(pages, kv, page, d, dtype=torch.float16, device="cuda") for _ in range(2))
    g = gen(2)
    last = [pages - 1, pages - 3, 2]
    rows = torch.randn(2, 3, kv, page, d, generator=g).half()
    for i, p in enumerate(last):
        K[p], V[p] = rows[0, i].cuda(), rows[1, i].cuda()
    q, out = torch.randn(40, 8, d, generator=g).cuda(), torch.empty(40, 8, d, device="cuda")
    P().spd_op_attention_paged("fp16", q, K, V, ints([last]).cuda(), ints([0, 40]).cuda(), ints([150]).cuda(), out, 40, 150)
    want, size = R.attention(q.cpu(), rows[0], rows[1], ints([[0, 1, 2]]), ints([0, 40]), ints([150]))
    assert ((out.cpu().double() - want).abs() <= 1e-5 * size.amax(-1, keepdim=True)).all()
    codes = torch.randint(-127, 128, (pages, 8, page, d), dtype=torch.int8, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    scale = torch.rand(pages, 8, page, device="cuda", generator=torch.Generator("cuda").manual_seed(4))
    outs = [torch.empty(3, 8, d, device="cuda") for _ in range(2)]
    P().spd_op_read_paged("int8", codes, codes, ints([last]).cuda(), ints([0, 0, 0]).cuda(), ints([5, 70, 140]).cuda(), *outs, K_scale=scale, V_scale=scale)
    for i, p in enumerate((5, 70, 140)):
        assert torch.equal(outs[1][i], codes[last[i], :, p % 64].float() * scale[last[i], :, p % 64, None])


# ------------------------------------------------------------------ verification
def verify_case(dtype, counts, vocab, seed, drawn=True, pad=0, noise=0.5):
    g = gen(seed)
    n = sum(counts) + pad
    common = torch.randn(n, vocab, generator=g) * 2.5
    target, drafter = (((common + noise * torch.randn(n, vocab, generator=g)).to(R.TORCH[dtype])) for _ in range(2))
    gumbel = -torch.log(-torch.log(torch.rand(n, vocab, generator=g).clamp(1e-7, 1 - 1e-7)))
    tokens = torch.cat([ints([0]), (drafter.float() + (gumbel if drawn else 0.0)).argmax(1)[:-1].int()])
    first = [0]
    for c in counts:
        first.append(first[-1] + c)
    return dict(logits=target, tokens=tokens, first=ints(first), u=torch.rand(n, generator=g), draft_logits=drafter if drawn else None)


def run_verify(dtype, case, tau=1.0, draft_tau=1.0):
    c = case
    n, n_seq = len(c["tokens"]), len(c["first"]) - 1
    out_t, out_l, out_a, err = torch.full((n,), -5, dtype=torch.int32, device="cuda"), torch.full((n,), 9.0, device="cuda"), torch.full((n_seq,), -5, dtype=torch.int32, device="cuda"), zero()
    P().spd_op_verify_drafts(dtype, c["logits"].cuda(), c["tokens"].cuda(), c["first"].cuda(), c["u"].cuda(), out_t, out_l, out_a, tau=tau, draft_logits=dev(c["draft_logits"]),
                             draft_tau=draft_tau, err=err)
    return out_t.cpu(), out_l.cpu(), out_a.cpu(), int(err)


def check_verify(dtype, case, tau=1.0, draft_tau=1.0, at_border=False):
    """Decisions are those of 64 bits, unless one is nearer to its random number than sums of fp32 exponentials may be off, 2^-18 (acceptance), or 2^-44 (the drawn token); there are none such in these
    cases but where `at_border` says so.  A logarithm of a probability is off by 2^-22 and half a step of itself."""
    out_t, out_l, out_a, err = run_verify(dtype, case, tau, draft_tau)
    first = case["first"].tolist()
    seen, bad = set(), False
    for s in range(len(first) - 1):
        a, b = first[s], first[s + 1]
        if a == b:
            assert out_a[s] == 0
            continue
        seen |= set(range(a, b))
        m, given, logp, wrong, near = R.verify(case["logits"][a:b], case["tokens"][a:b], case["u"][a:b], tau, None if case["draft_logits"] is None else case["draft_logits"][a:b], draft_tau)
        bad |= wrong
        assert at_border or near > 2.0 ** -44
        assert int(out_a[s]) == m and out_t[a:a + m + 1].tolist() == given, (s, out_a[s], m, out_t[a:b], given)
        assert (out_t[a + m + 1:b] == -1).all() and (out_l[a + m + 1:b] == 0).all()
        for i, w in enumerate(logp):
            got = float(out_l[a + i])
            assert got == w or abs(got - w) <= 2.0 ** -22 + abs(w) * 2.0 ** -24, (s, i, got, w)
    rest = [i for i in range(len(out_t)) if i not in seen]
    assert (out_t[rest] == -5).all() and (out_l[rest] == 9.0).all()
    assert err == int(bad)
    return out_t, out_l, out_a


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("counts,vocab,drawn,tau,draft_tau,pad", [
    ([5], 32000, True, 1.0, 1.0, 0), ([1, 1, 1], 1000, True, 0.7, 1.0, 0), ([4, 1, 0, 9, 2], 50258, True, 0.9, 1.3, 3), ([6, 3], 777, False, 1.0, 1.0, 0), ([3] * 40, 51, True, 1.2, 0.8, 0),
    ([2, 17], 1, True, 1.0, 1.0, 0), ([9] * 5, 2, False, 1.0, 1.0, 1), ([3, 5], 131072, False, 0.5, 1.0, 0), ([2] * 70, 4099, True, 1.0, 1.0, 2), ([65], 257, True, 1.0, 1.0, 0)])
def test_verify(dtype, counts, vocab, drawn, tau, draft_tau, pad):
    say("verify", dtype, counts, vocab, drawn, tau, draft_tau, pad)
    check_verify(dtype, verify_case(dtype, counts, vocab, seed=vocab, drawn=drawn, pad=pad), tau, draft_tau)


@pytest.mark.parametrize("drawn", [True, False])
def test_verify_all_stand_none_stands_and_the_ends_of_u(drawn):
    """A drafter that is the target (every draft stands if u < 1), u of 0 and next to 1, drafts that the target excludes."""
    case = verify_case("fp32", [6, 6, 6, 6], 500, seed=1, drawn=drawn, noise=0.0)
    case["u"][6:12] = 0.0
    case["u"][12:18] = 1.0 - 2.0 ** -24
    case["logits"][18, case["tokens"][19]] = -math.inf
    _, _, out_a = check_verify("fp32", case, at_border=True)
    if drawn:
        assert out_a.tolist() == [5, 5, 5, 0]
    else:
        assert out_a[1] == 5 and out_a[3] == 0


def test_verify_what_is_no_number():
    """NaN is excluded, +inf the largest number, rows without a finite logit, a drafter's row likewise."""
    case = verify_case("fp32", [4, 4, 4, 4, 3], 300, seed=2)
    case["logits"][0, ::3] = math.nan
    case["logits"][4, 7] = math.inf
    case["logits"][5, [7, 11]] = math.inf
    case["tokens"][5], case["u"][7] = 7, 0.3
    case["tokens"][6], case["u"][5] = 11, 0.1
    case["logits"][9] = -math.inf
    case["draft_logits"][12] = -math.inf
    case["draft_logits"][16, ::2] = math.nan
    check_verify("fp32", case)


def test_verify_drafts_that_are_no_tokens():
    case = verify_case("fp16", [4, 4, 4], 300, seed=3)
    case["u"][:] = 0.0
    case["tokens"][2], case["tokens"][5], case["tokens"][8] = 300, -1, 2 ** 31 - 1     # (the last: a sequence's first token, which nothing asks about)
    _, _, out_a = check_verify("fp16", case, at_border=True)
    assert out_a.tolist()[:2] == [1, 0]


def test_verify_firsts_out_of_range():
    case = verify_case("fp32", [3, 3, 3, 3], 200, seed=4)
    want = run_verify("fp32", case)
    for at, bad, lost in ((4, 13, [3]), (0, -1, [0]), (2, 2, [0, 1, 2, 3])):      # (where it descends there is no telling whose rows are whose: none is written)
        c = dict(case, first=case["first"].clone())
        c["first"][at] = bad
        out_t, out_l, out_a, err = run_verify("fp32", c)
        assert err == 1 and (out_a[lost] == 0).all()
        for s in range(4):
            rows = slice(3 * s, 3 * s + 3)
            if s not in lost:
                assert torch.equal(out_t[rows], want[0][rows]) and out_a[s] == want[2][s]
            else:
                assert (out_t[rows] == -5).all() and (out_l[rows] == 9.0).all()


@pytest.mark.parametrize("dtype,stride,shift", [("fp32", 1003, 1), ("bf16", 1001, 3), ("fp16", 1000, 0)])
def test_verify_rows_off_the_grid_of_16_bytes(dtype, stride, shift):
    case = verify_case(dtype, [5, 4], 999, seed=5)
    want = check_verify(dtype, case)
    kind = R.TORCH[dtype]
    apart = []
    for name in ("logits", "draft_logits"):
        wide = torch.full((9 * stride + 8,), math.nan, dtype=kind)
        view = wide[shift:shift + 9 * stride].view(9, stride)[:, :999]
        view.copy_(case[name])
        whole = wide.cuda()
        apart.append(whole[shift:shift + 9 * stride].view(9, stride)[:, :999])
    out_t, out_l, out_a = torch.full((9,), -5, dtype=torch.int32, device="cuda"), torch.full((9,), 9.0, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    P().spd_op_verify_drafts(dtype, apart[0], case["tokens"].cuda(), case["first"].cuda(), case["u"].cuda(), out_t, out_l, out_a, draft_logits=apart[1])
    assert torch.equal(out_t.cpu(), want[0]) and torch.equal(out_a.cpu(), want[2]) and (out_l.cpu() - want[1]).abs().max() < 1e-6


def test_verified_texts_have_the_targets_distribution():
    """Twenty thousand sequences of one draft over a small vocabulary, all with the same rows: how often each token comes first, against p (five standard deviations)."""
    n, V = 20_000, 13
    g = gen(6)
    target, drafter = torch.randn(V, generator=g) * 1.5, torch.randn(V, generator=g) * 1.5
    q = drafter.softmax(0)
    drafts = torch.multinomial(q, n, replacement=True, generator=g).int()
    tokens = torch.stack([torch.zeros(n, dtype=torch.int32), drafts], 1).flatten()
    case = dict(logits=target.expand(2 * n, V).contiguous(), draft_logits=drafter.expand(2 * n, V).contiguous(), tokens=tokens, first=ints(range(0, 2 * n + 1, 2)), u=torch.rand(2 * n, generator=g))
    out_t, _, out_a, err = run_verify("fp32", case)
    p = target.double().softmax(0)
    seen = torch.bincount(out_t.view(n, 2)[:, 0].long(), minlength=V).double()
    assert err == 0 and ((seen - n * p).abs() <= 5 * (n * p * (1 - p)).sqrt()).all()
    stands = float(torch.minimum(p, q.double()).sum())
    assert abs(float(out_a.double().mean()) - stands) <= 5 * math.sqrt(stands * (1 - stands) / n)


# ------------------------------------------------------------------ together
class Model:
    """A little decoder whose projections torch runs, everything else by the operators: every call takes a chunk of each sequence."""
    layers, heads, kv, d, vocab, page = 2, 4, 2, 32, 61, 8

    def __init__(self, dtype, n_seq, seed, like=None, noise=0.0):
        g = gen(seed)
        self.dtype, self.dm = dtype, self.heads * self.d
        draw = lambda *shape, by: torch.randn(*shape, generator=g) * by  # noqa: E731
        self.w = {"embed": draw(self.vocab, self.dm, by=1.0), "head": draw(self.vocab, self.dm, by=2.0 / self.dm ** 0.5)}
        for l in range(self.layers):
            self.w[f"qkv{l}"] = draw((self.heads + 2 * self.kv) * self.d, self.dm, by=self.dm ** -0.5)
            self.w[f"o{l}"] = draw(self.dm, self.dm, by=self.dm ** -0.5)
        if like is not None:
            self.w = {k: like.w[k] + noise * self.w[k] for k in self.w}
        self.on_gpu = {k: v.cuda() for k, v in self.w.items()}
        self.entries = 10
        self.table = torch.randperm(n_seq * self.entries, generator=g).int().view(n_seq, self.entries).cuda()
        shape = (self.layers, n_seq * self.entries, self.kv, self.page, self.d)
        if dtype == "int8":
            self.K, self.V = (torch.zeros(shape, dtype=torch.int8, device="cuda") for _ in range(2))
            self.scales = [torch.full(shape[:4], math.nan, device="cuda") for _ in range(2)]
        else:
            self.K, self.V = (torch.full(shape, math.nan, device="cuda").to(R.TORCH[dtype]) for _ in range(2))
            self.scales = [None, None]
        self.err = zero()

    def forward(self, tokens, seq, pos, first, length, max_new, max_len):
        x = self.on_gpu["embed"][tokens.long()]
        for l in range(self.layers):
            q, k, v = split(x @ self.on_gpu[f"qkv{l}"].T, self.heads, self.kv, self.d)
            turned = torch.zeros(len(tokens), self.heads, self.d, device="cuda")
            scales = {}
            if self.dtype == "int8":
                scales = {"K_scale": self.scales[0][l], "V_scale": self.scales[1][l]}
                P().spd_op_append_paged_q8(self.K[l], self.V[l], *scales.values(), self.table, k, v, seq, pos, THETA, q=q, q_out=turned, err=self.err)
            else:
                P().spd_op_append_paged(self.dtype, self.K[l], self.V[l], self.table, k, v, seq, pos, THETA, q=q, q_out=turned, err=self.err)
            o = torch.zeros_like(turned)
            P().spd_op_attention_paged(self.dtype, turned, self.K[l], self.V[l], self.table, first, length, o, max_new, max_len, **scales, err=self.err)
            x = x + o.flatten(1) @ self.on_gpu[f"o{l}"].T
        return x @ self.on_gpu["head"].T

    def chunk(self, texts, cached):
        """Sequence s's texts[s] from position cached[s] on, in one call; the logits of all its tokens."""
        news = [t[c:] for t, c in zip(texts, cached)]
        first = [0]
        for n in news:
            first.append(first[-1] + len(n))
        tokens = ints([x for n in news for x in n]).cuda()
        seq, pos = ints([s for s, n in enumerate(news) for _ in n]).cuda(), ints([c + i for n, c in zip(news, cached) for i in range(len(n))]).cuda()
        z = self.forward(tokens, seq, pos, ints(first).cuda(), ints([len(t) for t in texts]).cuda(), max(map(len, news)), max(map(len, texts)))
        return z, tokens, ints(first).cuda()

    def logits64(self, text):
        """All tokens' logits of a text, nothing cached, in 64 bits; an 8-bit cache's keys and values as their codes."""
        x = self.w["embed"][text].double()
        for l in range(self.layers):
            q, k, v = split(x @ self.w[f"qkv{l}"].double().T, self.heads, self.kv, self.d)
            turn = lambda y: torch.stack([R.rotate(y[p], p, THETA) for p in range(len(text))])  # noqa: E731
            q, k = turn(q), turn(k)
            if self.dtype == "int8":
                k, v = (R.values(*R.quantise(y)) for y in (k, v.float().double()))
            else:
                k, v = (y.float().to(R.TORCH[self.dtype]).double() for y in (k, v))
            k, v = k.repeat_interleave(self.heads // self.kv, 1), v.repeat_interleave(self.heads // self.kv, 1)
            z = torch.einsum("qhd,khd->hqk", q, k) / math.sqrt(self.d)
            z = z.masked_fill(torch.ones(len(text), len(text)).triu(1).bool(), -math.inf)
            x = x + torch.einsum("hqk,khd->qhd", z.softmax(-1), v).flatten(1) @ self.w[f"o{l}"].double().T
        return x @ self.w["head"].double().T


@pytest.mark.parametrize("dtype,bound", [("fp32", 1e-4), ("fp16", 5e-3), ("bf16", 4e-2), ("int8", 2e-2)])
def test_speculative_decoding(dtype, bound):
    """A drafter proposes up to four tokens per sequence, one by one; the target takes them with its own newest token in one chunk, and what stands goes on.  Every chunk's logits are those of the texts so far,
    computed from scratch in 64 bits, and every verification is that of the chunk's logits.  Bound: fp32 sums (1e-4 of the logits' scale is ample for two layers); a cache of 16 or 8 bits may round a
    key the other way than the reference where the two differ in their last bits: some steps of the type (8 bits: 1 / 127 of a row's largest value)."""
    prompts = [[5, 17, 40, 3, 9], [11], [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13]]
    n = len(prompts)
    target = Model(dtype, n, seed=11)
    drafter = Model(dtype, n, seed=12, like=target, noise=0.15)
    texts, cached, drafted = [list(p) for p in prompts], [0] * n, [0] * n       # cached positions of the target and of the drafter
    g, stood = gen(13), 0
    for step in range(7):
        counts = [(step + s) % 5 for s in range(n)]             # drafts of this step, none among them
        drafts, rows = [[] for _ in range(n)], [[] for _ in range(n)]
        for i in range(max(counts)):
            on = [s for s in range(n) if i < counts[s]]
            whole = [texts[s] + drafts[s] for s in range(n)]
            upto = [whole[s] if s in on else whole[s][:drafted[s]] for s in range(n)]     # (others: no new token)
            z, _, first = drafter.chunk(upto, drafted)
            for s in on:
                row = z[int(first[s + 1]) - 1].cpu()
                drafts[s].append(int(torch.multinomial(row.softmax(0), 1, generator=g)))
                rows[s].append(row)
                drafted[s] = len(whole[s])
        whole = [t + x for t, x in zip(texts, drafts)]
        z, tokens, first = target.chunk(whole, cached)
        for s in range(n):
            want = target.logits64(whole[s])[cached[s]:]
            off = (z[int(first[s]):int(first[s + 1])].cpu().double() - want).abs().max() / want.abs().max()
            assert off < bound, (step, s, off)
        # verification looks at the last token of a text and the drafts behind it
        keep = [i for s in range(n) for i in range(int(first[s + 1]) - counts[s] - 1, int(first[s + 1]))]
        at = [0]
        for c in counts:
            at.append(at[-1] + c + 1)
        blank = torch.zeros(drafter.vocab)
        case = dict(logits=z[keep].contiguous(), tokens=tokens[keep].contiguous(), first=ints(at), u=torch.rand(len(keep), generator=g),
                    draft_logits=torch.stack([r for s in range(n) for r in rows[s] + [blank]]))
        case = {k: v.cpu() for k, v in case.items()}
        out_t, _, out_a = check_verify("fp32", case)
        for s in range(n):
            a = int(out_a[s])
            stood += a
            texts[s] = texts[s] + out_t[at[s]:at[s] + a + 1].tolist()
            cached[s] = len(texts[s]) - 1                       # positions behind those that stand are written again
            drafted[s] = min(drafted[s], cached[s])
    assert int(target.err) == 0 and int(drafter.err) == 0 and stood > 0


# ------------------------------------------------------------------ streams and graphs
@pytest.mark.parametrize("heads,io,max_len,vocab", [(2, "fp32", 190, 900), (32, "fp32", 700, 33000), (16, "bf16", 1600, 5000)])
def test_operators_in_a_graph_and_on_another_stream(heads, io, max_len, vocab):
    """A step of all four captured once and replayed with other lengths, numbers of new tokens, positions and draws (they are on the device), between eager work; a second graph of the same operators has
    scratch of its own.  Every replay equals the eager calls."""
    g = gen(12)
    kv, d, page, n_pages, n_seq, n = 2, 64, 16, 420, 4, 24
    table = torch.randperm(n_pages, generator=g).int()[:n_seq * 100].view(n_seq, 100).cuda()
    qkv = torch.randn(n, (heads + 2 * kv) * d, generator=g).cuda()
    rows = [torch.randn(n, vocab, generator=g).cuda() for _ in range(2)]
    K0, V0 = (torch.randint(-127, 128, (n_pages, kv, page, d), generator=g).to(torch.int8).cuda() for _ in range(2))
    s0 = torch.rand(n_pages, kv, page, generator=g).cuda() / 50

    class Step:
        def __init__(self):
            i = lambda k: torch.zeros(k, dtype=torch.int32, device="cuda")  # noqa: E731
            self.K, self.V, self.Ks, self.Vs = K0.clone(), V0.clone(), s0.clone(), s0.clone()
            self.seq, self.pos, self.first, self.length, self.tokens, self.u = i(n), i(n), i(n_seq + 1), i(n_seq), i(n), torch.zeros(n, device="cuda")
            self.q, self.out = torch.zeros(n, heads, d, device="cuda"), torch.zeros(n, heads, d, device="cuda", dtype=R.TORCH[io])
            self.k, self.v = (torch.zeros(n, kv, d, device="cuda") for _ in range(2))
            self.t, self.a, self.l = i(n), i(n_seq), torch.zeros(n, device="cuda")

        def load(self, i):
            counts, lengths = [[5, 1, 0, 9], [6, 6, 6, 6], [1, 1, 1, 1], [0, 24, 0, 0]][i], [max_len - 31 * i - 3 * s for s in range(n_seq)]
            for x, y in ((self.K, K0), (self.V, V0), (self.Ks, s0), (self.Vs, s0)):
                x.copy_(y)
            first = torch.tensor([0] + counts).cumsum(0)
            seq = [s for s, c in enumerate(counts) for _ in range(c)]
            pos = [lengths[s] - c + j for s, c in enumerate(counts) for j in range(c)]
            pad = n - len(seq)
            self.first.copy_(first), self.length.copy_(ints(lengths)), self.seq.copy_(ints(seq + [-1] * pad)), self.pos.copy_(ints(pos + [0] * pad))
            self.tokens.copy_(torch.randint(0, vocab, (n,), generator=gen(50 + i)))
            self.u.copy_(torch.rand(n, generator=gen(60 + i)) * 0.1)
            for x in (self.q, self.out, self.k, self.v, self.t, self.a, self.l):
                x.zero_()

        def run(self):
            pkg = P()
            q, k, v = split(qkv, heads, kv, d)
            pkg.spd_op_append_paged_q8(self.K, self.V, self.Ks, self.Vs, table, k, v, self.seq, self.pos, THETA, q=q, q_out=self.q)
            pkg.spd_op_read_paged("int8", self.K, self.V, table, self.seq, self.pos, self.k, self.v, K_scale=self.Ks, V_scale=self.Vs)
            pkg.spd_op_attention_paged("int8", self.q.to(R.TORCH[io]), self.K, self.V, table, self.first, self.length, self.out, 9, max_len, K_scale=self.Ks, V_scale=self.Vs)
            pkg.spd_op_verify_drafts("fp32", rows[0], self.tokens, self.first, self.u, self.t, self.l, self.a, draft_logits=rows[1])

        def results(self):
            return [x.clone() for x in (self.K, self.V, self.Ks, self.Vs, self.q, self.k, self.v, self.out, self.t, self.l, self.a)]

    eager, steps, graphs, want = Step(), [Step(), Step()], [], []
    for i in range(4):
        eager.load(i)
        eager.run()
        want.append(eager.results())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for st in steps:
        st.load(0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            st.run()                                            # on a stream that is not the default
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(st.results(), want[0]))
        st.load(0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            st.run()
        graphs.append(graph)
    for i in (1, 3, 0, 2):
        for st in steps:
            st.load(i)
        eager.load(i)
        eager.run()
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for graph, stream in zip(graphs, streams):              # both at once
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for st in steps + [eager]:
            assert all(torch.equal(a, b) for a, b in zip(st.results(), want[i])), i
