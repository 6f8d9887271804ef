"""The operators of several sequences over one paged cache against their definitions in 64 bits (batch_reference.py)."""
import itertools
import math

import pytest
import torch

import batch_reference as R

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


# ------------------------------------------------------------------ append
def append_case(dtype, heads, kv, d, page, lengths, start, seed, pad=()):
    """Pools of a recognisable filling, a permuted table, the tokens of `lengths` from `start` on; padding tokens at the places `pad`."""
    g = gen(seed)
    first = [start + 5 * s for s in range(len(lengths))]
    entries = max(a + n - 1 for a, n in zip(first, lengths)) // page + 1
    used = [(s, e) for s, (a, n) in enumerate(zip(first, lengths)) for e in range(a // page, (a + n - 1) // page + 1)]
    order = torch.randperm(len(used) + 2, generator=g)
    table = torch.full((len(lengths), entries), -7, dtype=torch.int32)
    for (s, e), p in zip(used, order):
        table[s, e] = int(p)
    K, V = (torch.full((len(used) + 2, kv, page, d), x).to(R.TORCH[dtype]) for x in (3.25, -1.5))
    tokens = [(s, p) for s, (a, n) in enumerate(zip(first, lengths)) for p in range(a, a + n)]
    for at in pad:
        tokens.insert(at, (-1, -1))
    n = len(tokens)
    rows = torch.randn(n, (heads + 2 * kv) * d, generator=g)
    return K, V, table, rows, ints([s for s, _ in tokens]), ints([p for _, p in tokens])


def split(rows, heads, kv, d):
    q, k, v = rows.split([heads * d, kv * d, kv * d], 1)
    return q.unflatten(1, (heads, d)), k.unflatten(1, (kv, d)), v.unflatten(1, (kv, d))


def check_append(dtype, heads, kv, d, K, V, table, rows, seq, pos, theta=THETA):
    page = K.shape[2]
    q, k, v = split(rows.cuda(), heads, kv, d)
    Kd, Vd, q_out, err = K.cuda(), V.cuda(), torch.full((len(seq), heads, d), 9.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    P().spd_op_append_paged(dtype, Kd, Vd, table.cuda(), k, v, seq.cuda(), pos.cuda(), theta, q=q, q_out=q_out, err=err)
    Kd, Vd, q_out = Kd.cpu(), Vd.cpu(), q_out.cpu()
    wantK, wantV, bad = K.clone(), V.clone(), 0
    seen = torch.zeros(K.shape[:3], dtype=torch.bool)
    q, k, v = split(rows, heads, kv, d)
    for t, (s, p) in enumerate(zip(seq.tolist(), pos.tolist())):
        at = int(table[s, p // page]) if 0 <= s < len(table) and 0 <= p < page * table.shape[1] else -1
        bad += s >= 0 and not 0 <= at < len(K)
        if not 0 <= at < len(K):
            assert (q_out[t] == 9.0).all(), t
            continue
        # A rotated value is a c - b s.  c and s: the angle, below pi / 4 after its reduction, rounded to fp32 (2^-25), the function to 2 units in the last
        # place (2^-23); two products and a difference in fp32 (2^-24 of |a| + |b| each): below 2^-22 (|a| + |b|).  Then half a step of the cache's type.
        spread = lambda x: (x.unflatten(1, (d // 2, 2)).abs().sum(2) * 2.0 ** -22).double().repeat_interleave(2, 1)  # noqa: E731
        want, off = R.rotate(q[t], p, theta), spread(q[t])
        assert ((q_out[t] - want).abs() <= off).all(), (t, (q_out[t] - want).abs().max())
        want, off = R.rotate(k[t], p, theta), spread(k[t])
        got = Kd[at, :, p % page].double()
        assert ((got - want).abs() <= off + (want.abs() + off) * HALF_STEP[dtype] + 2.0 ** -25).all(), (t, (got - want).abs().max())
        wantK[at, :, p % page], wantV[at, :, p % page] = Kd[at, :, p % page], v[t].to(V.dtype)
        seen[at, :, p % page] = True
    assert torch.equal(Kd[~seen], wantK[~seen]) and torch.equal(Vd, wantV)      # values as torch rounds them, everything else as it was
    assert int(err) == int(bad > 0)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("heads,kv,d,page,lengths,start", [
    (4, 4, 128, 16, [1, 1, 1], 70), (8, 2, 64, 32, [5, 1, 40], 0), (3, 1, 256, 8, [17, 2], 30), (1, 1, 8, 4, [3], 2), (6, 3, 16, 1024, [9, 1], 1020), (40, 40, 128, 64, [3, 2], 63),
    (5, 5, 32, 4, [1], 0), (64, 8, 128, 16, [300], 1)])
def test_append(dtype, heads, kv, d, page, lengths, start):
    say("append", dtype, heads, kv, d, page, lengths, start)
    check_append(dtype, heads, kv, d, *append_case(dtype, heads, kv, d, page, lengths, start, seed=d + page))


@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
def test_append_of_many_tokens_with_padding_between_and_behind(dtype):
    """More pieces than one per thread; padding in front, inside and behind."""
    check_append(dtype, 32, 8, 128, *append_case(dtype, 32, 8, 128, 16, [400, 1, 333], 11, seed=1, pad=(0, 17, 18, 500, 738, 739)))


@pytest.mark.parametrize("start,theta", [(0, 1e4), (65535, 1e4), (1_000_003, 5e5), (2_000_000_000, 1e4)])
def test_append_far_positions(start, theta):
    """The definition's own angle in 64 bits is off by 2^-53 of itself, 2e-7 at two thousand million: within the bound up to there with a page of 1024."""
    if start > 1_000_000_000:   # (a table row for so far a position would be large: one entry per 1024 positions)
        K, V, table, rows, seq, pos = append_case("fp32", 2, 1, 64, 1024, [2], 0, seed=2)
        table = torch.full((1, start // 1024 + 1), -1, dtype=torch.int32)
        table[0, start // 1024] = 1
        pos = ints([start + 1, start + 2])
        q, k, v = split(rows.cuda(), 2, 1, 64)
        q_out = torch.empty(2, 2, 64, device="cuda")
        P().spd_op_append_paged("fp32", K.cuda(), V.cuda(), table.cuda(), k, v, seq.cuda(), pos.cuda(), theta, q=q, q_out=q_out)
        want = torch.stack([R.rotate(split(rows, 2, 1, 64)[0][t], start + 1 + t, theta) for t in range(2)])
        # angle and reduction: a few roundings of 2^-53 of 2e9 and of the frequency, 1e-6 in all, times |a| + |b| < 8
        assert (q_out.cpu() - want).abs().max() < 8e-6
        return
    check_append("fp32", 2, 1, 64, *append_case("fp32", 2, 1, 64, 128, [3, 2], start, seed=2), theta=theta)


def test_append_leaves_out_what_is_out_of_range():
    """Pages outside the pool, positions behind the table, sequences that are none: the other tokens arrive, nothing else changes."""
    K, V, table, rows, seq, pos = append_case("fp16", 2, 2, 64, 16, [20, 20], 0, seed=3)
    table[0, 1], table[1, 0] = len(K), -1
    pos[3], pos[5], seq[7] = 16 * table.shape[1], -4, 2
    check_append("fp16", 2, 2, 64, K, V, table, rows, seq, pos)


def test_append_without_queries_and_in_place():
    K, V, table, rows, seq, pos = append_case("bf16", 4, 2, 64, 16, [3, 4], 9, seed=4)
    q, k, v = (x.contiguous().cuda() for x in split(rows, 4, 2, 64))
    outs = []
    for in_place in (False, True):
        Kd, Vd, qd = K.cuda(), V.cuda(), q.clone()
        out = qd if in_place else torch.empty_like(qd)
        P().spd_op_append_paged("bf16", Kd, Vd, table.cuda(), k, v, seq.cuda(), pos.cuda(), THETA, q=qd, q_out=out)
        outs.append((Kd, Vd, out))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    Kd, Vd = K.cuda(), V.cuda()
    P().spd_op_append_paged("bf16", Kd, Vd, table.cuda(), k, v, seq.cuda(), pos.cuda(), THETA)
    assert torch.equal(Kd, outs[0][0]) and torch.equal(Vd, outs[0][1])
    P().spd_op_append_paged("bf16", Kd, Vd, table.cuda(), k[:0], v[:0], seq[:0].cuda(), pos[:0].cuda(), THETA)


def test_append_keeps_what_is_no_number():
    """Infinities and NaN of one value row stay where they are (a NaN whose payload would round up stays one)."""
    K, V, table, rows, seq, pos = append_case("bf16", 1, 1, 8, 4, [2], 1, seed=5)
    v = torch.tensor([math.inf, -math.inf, math.nan, 1.0, 0.0, -0.0, 3e38, -3e38])
    nan = torch.tensor([0x7FFFFFFF, -1], dtype=torch.int32).view(torch.float32)
    rows[0, -8:], rows[1, -8:-6] = v, nan
    q, k, vv = split(rows.cuda(), 1, 1, 8)
    Vd = V.cuda()
    P().spd_op_append_paged("bf16", K.cuda(), Vd, table.cuda(), k, vv, seq.cuda(), pos.cuda(), THETA)
    got = Vd.cpu()[table[0, 0], 0, 1]
    assert torch.equal(got[3:], v[3:].bfloat16()) and got[0] == math.inf and got[1] == -math.inf and got[2].isnan()
    assert Vd.cpu()[table[0, 0], 0, 2, :2].isnan().all()


# ------------------------------------------------------------------ attention
def attention_case(dtype, heads, kv, d, page, shared, lengths, width, seed, std=1.0):
    """Pools of NaN but for the positions that count, those of a group on pages of its first sequence; entries that no position needs are no pages."""
    g = gen(seed)
    n_seq = len(lengths)
    entries = max([max(n, shared[s // width]) for s, n in enumerate(lengths)] + [1]) // page + 2
    pages = n_seq * entries
    order = torch.randperm(pages, generator=g).int().view(n_seq, entries)
    table = torch.full((n_seq, entries), -1, dtype=torch.int32)
    K, V = (torch.full((pages, kv, page, d), math.nan) for _ in range(2))
    for s, n in enumerate(lengths):
        common, lead = shared[s // width], s - s % width
        for p in range(max(n, common if s == lead else 0)):
            owner = lead if p < common else s
            # (own positions on the page where the shared ones end are on a page of the sequence itself)
            table[owner, p // page] = order[owner, p // page]
            K[order[owner, p // page], :, p % page] = torch.randn(kv, d, generator=g) * std
            V[order[owner, p // page], :, p % page] = torch.randn(kv, d, generator=g)
    q = torch.randn(n_seq, heads, d, generator=g)
    return q, K.to(R.TORCH[dtype]), V.to(R.TORCH[dtype]), table, ints(shared), ints(lengths)


def attend(dtype, q, K, V, table, shared, length, width, max_shared=None, max_own=None):
    out, err = torch.full(q.shape, math.nan, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    own = max(n - int(shared[s // width]) for s, n in enumerate(length.tolist()))
    P().spd_op_attention_shared(dtype, q.cuda(), K.cuda(), V.cuda(), table.cuda(), shared.cuda(), length.cuda(), out, width,
                                int(shared.max()) if max_shared is None else max_shared, max(own, 0) if max_own is None else max_own, err=err)
    return out.cpu(), int(err)


def close(got, want, bound=1e-5):
    """Per query and head: the difference against the largest value.  fp32 sums of d_head products and of up to some thousand probabilities, about
    sqrt(terms) 2^-24 of the scale, scores of a few units: below 1e-5."""
    scale = want.abs().amax(-1, keepdim=True)
    assert torch.isfinite(got).all()
    off = ((got.double() - want).abs() / scale.clamp(min=1e-30)).masked_fill(scale == 0, 0.0)
    assert (got[want == 0] == 0).all() and off.max() < bound, off.max()


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("heads,kv,d,page,shared,lengths,width", [
    (4, 4, 128, 16, [64], [74, 70, 66, 65], 4),                      # a step of four beams
    (8, 1, 64, 8, [1], [1, 2], 2), (8, 2, 128, 32, [0, 40], [1, 0, 45, 40], 2),    # one position, none, none of its own
    (6, 2, 64, 16, [37, 16], [20, 37, 38, 0, 100, 17], 3),           # shorter than the shared part; ends inside pages
    (16, 1, 128, 64, [200], [231, 263], 2), (3, 3, 256, 16, [50], [51, 83, 90], 3),
    (10, 2, 8, 4, [9], [12, 30], 2), (4, 2, 16, 4, [3], [4, 9], 2), (2, 1, 32, 1024, [700], [701, 1030], 2),
    (1, 1, 128, 16, [], [], 1)])
def test_attention(dtype, heads, kv, d, page, shared, lengths, width):
    if not lengths:
        out = torch.empty(0, heads, d, device="cuda")
        P().spd_op_attention_shared(dtype, out, *(torch.zeros(1, kv, page, d, dtype=R.TORCH[dtype], device="cuda"),) * 2, ints([]).view(0, 1).cuda(), ints([]).cuda(), ints([]).cuda(), out,
                                    width, 0, 0)
        return
    say("attention", dtype, heads, kv, d, page, shared, lengths, width)
    case = attention_case(dtype, heads, kv, d, page, shared, lengths, width, seed=d + page)
    got, err = attend(dtype, *case, width)
    assert err == 0
    close(got, R.attention(*case, width))


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("heads,kv,d,shared,own,width,page", [
    (8, 1, 128, 1500, 7, 3, 16), (32, 2, 64, 700, 300, 5, 16), (2, 2, 128, 2100, 0, 1, 16), (16, 2, 128, 400, 33, 17, 16), (4, 1, 256, 900, 90, 6, 16), (5, 5, 128, 1024, 512, 2, 16),
    (24, 3, 128, 513, 1, 9, 16),
    # more query heads per key/value head than a tile has rows, alone and in groups; several tiles of d_head 256; small and large pages on the LDS path
    (34, 1, 128, 700, 60, 1, 16), (40, 2, 64, 600, 100, 3, 8), (16, 1, 256, 600, 10, 6, 16), (16, 2, 128, 1301, 40, 4, 4), (8, 1, 64, 1100, 40, 8, 1024)])
def test_attention_of_long_parts_and_many_rows(dtype, heads, kv, d, shared, own, width, page):
    """Parts cut into several chunks, rows of queries past one tile, groups of heads that do not divide a tile."""
    say("attention", dtype, heads, kv, d, shared, own, width, page)
    lengths = [shared + max(0, own - 3 * w) for w in range(width)] + [shared + own // 2] * width
    case = attention_case(dtype, heads, kv, d, page, [shared, shared - 1], lengths, width, seed=own)
    got, err = attend(dtype, *case, width)
    assert err == 0
    close(got, R.attention(*case, width))


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("width", [1, 8])
def test_attention_weights_add_up_to_one(dtype, width):
    """One key far above twenty thousand others, at weights near 2^-20: values of one come out as one.  A weight is cut to 2^-36 of the largest (2^-24 in bf16 and fp32
    of itself), so the many lose at most 20000 x 2^-36 = 3e-7; fp32 sums of 20000 terms in the waves' and chunks' order some 2^-22."""
    n, d = 20_000, 64
    q = torch.zeros(width, 4, d)
    q[..., 0] = 8.0
    K = torch.zeros(n // 16, 1, 16, d)
    K[..., 0] = 0.25 * torch.rand(n // 16, 1, 16, generator=gen(14))
    K[700, 0, 3, 0] = 14.0                                   # 8 x 14 / 8 = 14 = 20.2 log 2
    V = torch.ones(n // 16, 1, 16, d)
    table = torch.arange(n // 16, dtype=torch.int32).expand(width, -1).contiguous()
    got, err = attend(dtype, q, K.to(R.TORCH[dtype]), V.to(R.TORCH[dtype]), table, ints([n]), ints([n] * width), width)
    assert err == 0 and (got - 1.0).abs().max() < 1e-6, (got - 1.0).abs().max()


@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
def test_attention_of_a_long_sequence_that_ends_inside_the_shared_positions(dtype):
    """Its block takes more positions than a chunk has, on pages of four."""
    case = attention_case(dtype, 2, 1, 32, 4, [9001], [9003, 8999, 4097, 9001], 4, seed=13)
    got, err = attend(dtype, *case, 4)
    assert err == 0
    close(got, R.attention(*case, 4))


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_attention_large_and_small_values(dtype):
    """Queries and keys far from one: scores of some hundreds (one key takes all), of 1e-6 (all alike), queries of very different sizes in one call."""
    case = list(attention_case(dtype, 4, 2, 64, 16, [70], [80, 75], 2, seed=6, std=3.0))
    case[0] = case[0] * torch.tensor([1e-7, 1.0, 40.0, 1e-30]).view(1, 4, 1)
    got, _ = attend(dtype, *case, 2)
    want = R.attention(*case, 2)
    # a score is off by its fp32 sum's rounding, sqrt(64) 2^-24 of q k / 8 ~ 3 x 40 x sqrt(64) = 1000 at the largest: 5e-4 in an exponent
    close(got[:, [0, 1, 3]], want[:, [0, 1, 3]], 3e-5)
    close(got[:, 2:3], want[:, 2:3], 2e-3)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_attention_sees_what_is_no_number_only_where_it_counts(dtype):
    """A NaN in one sequence's own value, an infinite query: those rows alone."""
    q, K, V, table, shared, length = attention_case(dtype, 4, 2, 128, 16, [40], [45, 50, 47], 3, seed=7)
    clean, _ = attend(dtype, q, K, V, table, shared, length, 3)
    V[table[1, 48 // 16], 1, 48 % 16, 5] = math.nan
    q[2, 0, 3] = math.inf
    got, _ = attend(dtype, q, K, V, table, shared, length, 3)
    assert got[1, 2:, 5].isnan().all() and not torch.isfinite(got[2, 0]).all()
    spoilt = torch.zeros(got.shape, dtype=torch.bool)
    spoilt[1, 2:, 5], spoilt[2, 0] = True, True
    assert torch.equal(got[~spoilt], clean[~spoilt])


@pytest.mark.parametrize("d", [64, 32])
def test_attention_with_lengths_and_pages_out_of_range(d):
    q, K, V, table, shared, length = attention_case("fp16", 4, 2, d, 16, [40, 30], [45, 50, 36, 47], 2, seed=8)
    args = (q, K, V, table)
    assert attend("fp16", *args, shared, length, 2, max_shared=64, max_own=17)[1] == 0
    # sequences that do not fit their bounds: zeros, the others as before
    for bad_shared, bad_length, gone in (([40, 30], [45, -1, 36, 47], [1]), ([40, 30], [45, 58, 36, 47], [1]), ([40, 65], [45, 50, 36, 47], [2, 3]), ([-1, 30], [45, 50, 36, 47], [0, 1]),
                                         ([40, 30], [45, 50, 36, 2_000_000_000], [3])):
        got, err = attend("fp16", *args, ints(bad_shared), ints(bad_length), 2, max_shared=64, max_own=17)
        here = [s for s in range(4) if s not in gone]
        assert err == 1 and (got[gone] == 0).all()
        close(got[here], R.attention(*args, shared, length, 2)[here])
    # pages that are none: their positions do not count
    for s, e, page in ((0, 1, -1), (3, 2, len(K)), (2, 0, 2_000_000_000)):
        bad = table.clone()
        bad[s, e] = page
        got, err = attend("fp16", q, K, V, bad, shared, length, 2)
        assert err == 1
        close(got, R.attention(q, K, V, bad, shared, length, 2))
    got, err = attend("fp16", q, K, V, torch.full_like(table, -1), shared, length, 2)
    assert err == 1 and (got == 0).all()


@pytest.mark.parametrize("dtype,heads", [("fp16", 4), ("fp16", 16), ("bf16", 16), ("fp32", 16)])
def test_attention_cut_into_chunks_with_lengths_and_pages_out_of_range(dtype, heads):
    """The same where shared positions have blocks of their own, a tile of 8 rows and one of 32; a sequence that ends inside them beside one that is empty."""
    q, K, V, table, shared, length = attention_case(dtype, heads, 2, 64, 16, [700, 650], [705, 690, 0, 720, 651, 700, 650, 1], 4, seed=15)
    got, err = attend(dtype, q, K, V, table, shared, length, 4, max_shared=704, max_own=60)
    assert err == 0
    close(got, R.attention(q, K, V, table, shared, length, 4))
    for bad_shared, bad_length, gone in (([700, 650], [705, -1, 0, 720, 651, 700, 650, 1], [1, 2]), ([700, 650], [705, 690, 0, 761, 651, 700, 650, 1], [2, 3]),
                                         ([705, 650], [705, 690, 0, 720, 651, 700, 650, 1], [0, 1, 2, 3]), ([700, -1], [705, 690, 0, 720, 651, 700, 650, 1], [2, 4, 5, 6, 7])):
        got, err = attend(dtype, q, K, V, table, ints(bad_shared), ints(bad_length), 4, max_shared=704, max_own=60)
        here = [s for s in range(8) if s not in gone]
        assert err == 1 and (got[gone] == 0).all()
        close(got[here], R.attention(q, K, V, table, shared, length, 4)[here])
    for s, e, page in ((0, 3, -1), (4, 40, len(K)), (3, 44, -2_000_000_000)):
        bad = table.clone()
        bad[s, e] = page
        got, err = attend(dtype, q, K, V, bad, shared, length, 4)
        assert err == 1
        close(got, R.attention(q, K, V, bad, shared, length, 4))


def test_attention_offsets_past_32_bits():
    """A pool of more than 2^32 bytes per tensor whose last page counts."""
    n_pages, page, kv, d = 8193, 1024, 2, 128
    K, V = (torch.zeros(n_pages, kv, page, d, dtype=torch.float16, device="cuda") for _ in range(2))
    assert K.numel() * 2 > 2 ** 32
    g = gen(9)
    k, v, q = torch.randn(kv, 3, d, generator=g).half(), torch.randn(kv, 3, d, generator=g).half(), torch.randn(1, 4, d, generator=g)
    K[-1, :, 5:8], V[-1, :, 5:8] = k.cuda(), v.cuda()
    table = ints([[n_pages - 1]])
    small = [torch.zeros(1, kv, page, d, dtype=torch.float16) for _ in range(2)]
    small[0][0, :, 5:8], small[1][0, :, 5:8] = k, v
    out = torch.empty(1, 4, d, device="cuda")
    P().spd_op_attention_shared("fp16", q.cuda(), K, V, table.cuda(), ints([2]).cuda(), ints([8]).cuda(), out, 1, 2, 6)
    close(out.cpu(), R.attention(q, *small, ints([[0]]), [2], [8], 1))
    kk = torch.randn(1, kv, d, generator=g)
    P().spd_op_append_paged("fp16", K, V, table.cuda(), kk.cuda(), kk.cuda(), ints([0]).cuda(), ints([1023]).cuda(), THETA)
    assert torch.equal(V[-1, :, 1023].cpu(), kk[0].half())


# ------------------------------------------------------------------ selection
def run_select(dtype, logits, scores, n_out, tau=1.0, ended=None, end_token=-1):
    groups, n_in = scores.shape
    out = lambda t: torch.full((groups, n_out), -3, dtype=t, device="cuda")  # noqa: E731
    s, t, p, e = out(torch.float32), out(torch.int32), out(torch.int32), out(torch.int32)
    P().spd_op_beam_select(dtype, logits if logits.is_cuda else logits.cuda(), scores.cuda(), s, t, p, tau=tau, ended=None if ended is None else ints(ended).cuda(), end_token=end_token,
                           out_ended=e)
    return s.cpu(), t.cpu(), p.cpu(), e.cpu()


def check_select(dtype, logits, scores, n_out, tau=1.0, ended=None, end_token=-1, on_gpu=None):
    s, t, p, e = run_select(dtype, logits if on_gpu is None else on_gpu, scores, n_out, tau, ended, end_token)
    for g in range(len(scores)):
        want = R.select(logits[g].float(), scores[g], n_out, tau, None if ended is None else ended[g], end_token)
        assert t[g].tolist() == [c[1] for c in want] and p[g].tolist() == [c[2] for c in want] and e[g].tolist() == [c[3] for c in want], (g, want)
        score = torch.tensor([c[0] for c in want], dtype=torch.float64)
        here = score > -math.inf
        assert (s[g][~here] == -math.inf).all()
        # the sum of exponentials in fp32 (1e-6 of it at 131072 terms, arguments of up to 30 / tau rounded at 2^-23), one rounding of the score
        assert ((s[g][here] - score[here]).abs() <= 5e-6 + score[here].abs() * 2.0 ** -24).all(), (s[g], score)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("groups,n_in,n_out,vocab,tau", [
    (1, 4, 4, 32000, 1.0), (3, 1, 5, 1000, 0.7), (2, 16, 16, 4097, 1.3), (1, 2, 16, 9, 1.0), (2, 8, 3, 4096, 0.4), (1, 16, 16, 1, 1.0), (1, 3, 1, 131074, 1.0), (5, 5, 10, 257, 2.0),
    (1, 2, 2, 300_001, 1.0), (2, 3, 16, 2049, 1.0), (1, 16, 16, 2048, 0.9), (30, 16, 16, 20_000, 1.0), (70, 16, 2, 9000, 1.0), (16, 16, 16, 33_000, 1.0)])
def test_select(dtype, groups, n_in, n_out, vocab, tau):
    say("select", dtype, groups, n_in, n_out, vocab)
    g = gen(vocab)
    logits = (torch.randn(groups, n_in, vocab, generator=g) * 3).to(R.TORCH[dtype])
    check_select(dtype, logits, -torch.rand(groups, n_in, generator=g) * 4, n_out, tau)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_select_ties_go_to_the_lower_beam_and_token(dtype):
    """All logits alike; two values; a plateau across slices; equal beams."""
    t = R.TORCH[dtype]
    check_select(dtype, torch.zeros(1, 2, 10_000, dtype=t), torch.zeros(1, 2), 7)
    z = torch.zeros(2, 3, 9000, dtype=t)
    z[:, :, ::7] = 1.0
    check_select(dtype, z, torch.tensor([[-1.0, -1.0, -1.0], [-2.0, -1.0, -1.5]]), 16)
    z = torch.randn(1, 1, 20_000, generator=gen(1)).to(t)
    z[0, 0, 3000:15_000] = 9.0
    z[0, 0, [100, 16_000]] = 10.0
    check_select(dtype, z, torch.zeros(1, 1), 16)
    for vocab in (5000, 3000):
        z = torch.zeros(1, 1, vocab, dtype=t)
        z[0, 0, 1::2] = -0.0
        check_select(dtype, z, torch.zeros(1, 1), 5)
        check_select(dtype, z - 1.0, torch.zeros(1, 1), 16)
        z = torch.full((1, 2, vocab), -1e4, dtype=t)         # a few live among masked ones, fewer than asked for; one lane's entries hold all large values
        z[0, 0, [7, vocab - 1, 1200]] = torch.tensor([1.0, 2.0, 1.0], dtype=t)
        z[0, 1, 5:vocab:64] = torch.randn(len(range(5, vocab, 64)), generator=gen(2)).to(t)
        check_select(dtype, z, torch.tensor([[-1.0, -1.0]]), 9)
        z = torch.randn(1, 3, vocab, generator=gen(3)).to(t)
        z[0, 1] = z[0, 0]
        z[0, 2] = z[0, 0]
        check_select(dtype, z, torch.tensor([[-1.0, -1.0, -1.0]]), 16)


def test_select_values_that_are_excluded_or_no_numbers():
    inf, big = math.inf, torch.finfo(torch.float32).max
    z = torch.randn(6, 2, 5000, generator=gen(2))
    z[0, 0] = -inf                                   # a row without a continuation
    z[1, :, 3:] = -inf                               # six continuations for eight places
    z[2, 0, ::2], z[2, 1] = math.nan, math.nan
    z[3, 0, [5, 4000]], z[3, 1, 7] = inf, -big       # two certain tokens
    z[4, 0] = -big                                   # masked with the lowest value, all of it and all but one
    z[4, 1], z[4, 1, 17] = -big, 1.0
    z[5] = -inf
    z[0, 1, 100:200] = torch.tensor([0x7F800001, 0x7FBFFFFF, -4194305, 0x7FC00000], dtype=torch.int32).view(torch.float32).repeat(25)   # signalling NaN too
    s = -torch.rand(6, 2, generator=gen(3))
    check_select("fp32", z, s, 8)
    check_select("fp32", z[..., :2500].contiguous(), s, 8)
    # the lowest values of fp16 and bf16 as masks
    for dtype in ("fp16", "bf16"):
        h = torch.randn(1, 2, 700, generator=gen(4)).to(R.TORCH[dtype])
        h[0, 0, 5:] = torch.finfo(R.TORCH[dtype]).min
        check_select(dtype, h, torch.zeros(1, 2), 9)


def test_select_absent_and_ended_beams():
    g = gen(5)
    z = torch.randn(5, 4, 3000, generator=g)
    s = torch.tensor([[0.0, -math.inf, -math.inf, -math.inf], [-1.0, -2.0, math.nan, -0.5], [-1.0, -1.5, -2.0, -9.0], [-3.0, -0.1, -0.2, -0.3], [-math.inf] * 4])
    ended = torch.tensor([[0, 0, 0, 0], [0, 1, 1, 0], [1, 1, 1, 1], [0, 1, 0, 1], [1, 0, 0, 1]], dtype=torch.int32)
    z[3, 2, 2] = 20.0                                # the end token as an ordinary continuation
    z[2], z[1, 1] = math.nan, math.nan               # rows of ended beams are not read
    z[ended != 0] = math.nan
    for n_out in (1, 4, 11):
        check_select("fp32", z, s, n_out, tau=0.8, ended=ended, end_token=2)
    check_select("fp32", torch.nan_to_num(z), s, 6, end_token=2)     # an end token without ended beams


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab,stride,shift", [(1003, 1005, 0), (1003, 1024, 1), (4100, 4104, 0), (50, 50, 3)])
def test_select_rows_off_the_grid_of_16_bytes(dtype, vocab, stride, shift):
    g = gen(stride)
    store = torch.full((6 * stride + 8,), 50.0)
    rows = store[shift:shift + 6 * stride].view(2, 3, stride)
    rows[..., :vocab] = torch.randn(2, 3, vocab, generator=g) * 2
    on_gpu = store.to(R.TORCH[dtype]).cuda()[shift:shift + 6 * stride].view(2, 3, stride)[..., :vocab]
    check_select(dtype, on_gpu.cpu(), -torch.rand(2, 3, generator=g), 6, on_gpu=on_gpu)


def test_select_into_its_inputs():
    g = gen(6)
    z, s, e = torch.randn(3, 5, 800, generator=g).cuda(), -torch.rand(3, 5, generator=g).cuda(), (torch.rand(3, 5, generator=g) < 0.3).int().cuda()
    want = run_select("fp32", z, s.cpu(), 5, 0.9, e.cpu(), 4)
    t, p = (torch.empty(3, 5, dtype=torch.int32, device="cuda") for _ in range(2))
    P().spd_op_beam_select("fp32", z, s, s, t, p, tau=0.9, ended=e, end_token=4, out_ended=e)
    assert all(torch.equal(a.cpu(), b) for a, b in zip((s, t, p, e), want))


# ------------------------------------------------------------------ reorder
def reorder_case(dtype, layers, kv, d, page, lengths, width, seed):
    g = gen(seed)
    groups, entries = len(lengths), max(lengths) // page + 2
    pages = groups * width * entries
    table = torch.randperm(pages, generator=g).int().view(groups * width, entries)
    K, V = (torch.randn(layers, pages, kv, page, d, generator=g).to(R.TORCH[dtype]) for _ in range(2))
    return K, V, table, ints([n for n in lengths for _ in range(width)])


def check_reorder(dtype, K, V, table, length, parents, width, want=None, want_err=0):
    Kd, Vd, out, err = K.cuda(), V.cuda(), torch.full_like(table, -9).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    P().spd_op_beam_reorder(dtype, Kd, Vd, table.cuda(), parents.cuda(), length.cuda(), out, width, err=err)
    a, b, c = R.reorder(K, V, table, parents, length, width) if want is None else want
    assert torch.equal(out.cpu(), c) and torch.equal(Kd.cpu(), a) and torch.equal(Vd.cpu(), b) and int(err) == want_err


@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
@pytest.mark.parametrize("layers,kv,d,page,lengths,width", [(3, 2, 64, 16, [37, 10], 4), (1, 1, 8, 4, [7], 2), (2, 40, 128, 16, [31], 5), (2, 3, 16, 4, [5, 2], 3), (1, 2, 256, 64, [63, 65, 1], 16),
                                                            (2, 1, 32, 8, [16, 0, 8], 4), (1, 1, 16, 8, [20, 20], 1)])
def test_reorder(dtype, layers, kv, d, page, lengths, width):
    K, V, table, length = reorder_case(dtype, layers, kv, d, page, lengths, width, seed=width)
    g = gen(page)
    for parents in (torch.randint(0, width, (len(lengths), width), generator=g), torch.arange(width).expand(len(lengths), width), torch.zeros(len(lengths), width),
                    torch.full((len(lengths), width), width - 1), torch.arange(width - 1, -1, -1).expand(len(lengths), width)):
        check_reorder(dtype, K, V, table, length, ints(parents).contiguous(), width)


def test_reorder_every_choice_of_three_parents():
    K, V, table, length = reorder_case("bf16", 1, 1, 16, 4, [6] * 27, 3, seed=1)
    check_reorder("bf16", K, V, table, length, ints(list(itertools.product(range(3), repeat=3))), 3)


def test_reorder_leaves_a_group_that_makes_no_sense_as_it_was():
    """Parents that are none, unequal lengths, a length behind the table, pages out of the pool or shared where they are written: the first group
    stays, the second is put in order."""
    K, V, table, length = reorder_case("fp16", 2, 2, 64, 16, [37, 40], 3, seed=2)
    good = ints([[2, 2, 0], [1, 1, 1]])
    e = 37 // 16

    def case(parents=good, length=length, table=table):
        a, b, c = R.reorder(K, V, table, ints([[0, 1, 2], [1, 1, 1]]), ints([37, 37, 37, 40, 40, 40]), 3)
        check_reorder("fp16", K, V, table, length, parents, 3, want=(a, b, c), want_err=1)

    case(parents=ints([[2, 3, 0], [1, 1, 1]]))
    case(parents=ints([[-1, 0, 0], [1, 1, 1]]))
    case(length=ints([37, 37, 38, 40, 40, 40]))
    case(length=ints([-1, -1, -1, 40, 40, 40]))
    case(length=ints([2_000_000_000] * 3 + [40] * 3))
    for at, page in (((0, e), -1), ((2, e), len(K[0])), ((1, e), int(table[2, e]))):
        bad = table.clone()
        bad[at] = page
        case(table=bad)
    # where nothing is copied, pages do not matter; a full table has nothing behind it
    full = table.clone()
    full[0, e] = -1
    check_reorder("fp16", K, V, full, length, ints([[0, 2, 1], [0, 1, 2]]), 3)
    check_reorder("fp16", K, V, table, ints([16 * table.shape[1]] * 6), good, 3)


# ------------------------------------------------------------------ together
class Beams:
    """A little decoder of several prompts with beams, its projections by torch, everything else by the operators; texts kept on the host."""
    layers, heads, kv, d, vocab, page, width = 2, 4, 2, 32, 97, 4, 3

    def __init__(self, dtype, prompts, seed):
        g = gen(seed)
        self.dtype, self.dm, G = dtype, self.heads * self.d, len(prompts)
        self.embed = torch.randn(self.vocab, self.dm, generator=g)
        self.wqkv = [torch.randn((self.heads + 2 * self.kv) * self.d, self.dm, generator=g) / self.dm ** 0.5 for _ in range(self.layers)]
        self.wo = [torch.randn(self.dm, self.dm, generator=g) / self.dm ** 0.5 for _ in range(self.layers)]
        self.head = torch.randn(self.vocab, self.dm, generator=g) / self.dm ** 0.5 * 2
        self.entries, n = 12, G * self.width
        self.prompts, self.texts = prompts, [[list(p)] for p in prompts]
        whole = [(len(p) - 1) // self.page for p in prompts]    # the pages in front of the one in which a prompt ends are common to its group
        table = torch.arange(n * self.entries, dtype=torch.int32).view(n, self.entries).flip(1)
        for s in range(n):
            table[s, :whole[s // self.width]] = table[s - s % self.width, :whole[s // self.width]]
        self.table, self.spare = table.cuda(), torch.empty_like(table).cuda()
        self.K, self.V = (torch.full((self.layers, n * self.entries, self.kv, self.page, self.d), math.nan, device="cuda").to(R.TORCH[dtype]) for _ in range(2))
        self.shared, self.err = ints([len(p) - 1 for p in prompts]).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
        self.dev = {k: [w.cuda() for w in v] if isinstance(v, list) else v.cuda() for k, v in {"embed": self.embed, "wqkv": self.wqkv, "wo": self.wo, "head": self.head}.items()}

    def forward(self, tokens, seq, pos, width, table, shared, length, max_shared, max_own, attend=True):
        """Rows of new tokens through the layers; (attend: one per sequence) their logits."""
        x = self.dev["embed"][tokens.long()]
        for l in range(self.layers):
            q, k, v = split(x @ self.dev["wqkv"][l].T, self.heads, self.kv, self.d)
            turned = torch.empty(len(tokens), self.heads, self.d, device="cuda")
            P().spd_op_append_paged(self.dtype, self.K[l], self.V[l], table, k, v, seq, pos, THETA, q=q, q_out=turned, err=self.err)
            o = torch.empty_like(turned)
            P().spd_op_attention_shared(self.dtype, turned, self.K[l], self.V[l], table, shared, length, o, width, max_shared, max_own, err=self.err)
            x = x + o.flatten(1) @ self.dev["wo"][l].T
        return x @ self.dev["head"].T

    def start(self):
        """Prompts token by token into every row's pages, logits of each group's first row."""
        n, logits = len(self.prompts) * self.width, None
        for t in range(max(map(len, self.prompts))):
            on = [s for s in range(n) if t < len(self.prompts[s // self.width])]
            tokens = torch.tensor([self.prompts[s // self.width][min(t, len(self.prompts[s // self.width]) - 1)] for s in range(n)]).cuda()
            seq, pos = ints([s if s in on else -1 for s in range(n)]).cuda(), ints([t] * n).cuda()
            length = ints([t + 1 if s in on else 0 for s in range(n)]).cuda()
            z = self.forward(tokens, seq, pos, 1, self.table, torch.zeros(n, dtype=torch.int32, device="cuda"), length, 0, t + 1)
            logits = z if logits is None else torch.where((length > 0)[:, None], z, logits)
        self.length = ints([len(self.prompts[s // self.width]) for s in range(n)]).cuda()
        return logits.view(len(self.prompts), self.width, -1)

    def logits64(self, text):
        """The last token's logits of a text, nothing cached, in 64 bits."""
        x = self.embed[text].double()
        for l in range(self.layers):
            q, k, v = split(x @ self.wqkv[l].double().T, self.heads, self.kv, self.d)
            turn = lambda y: torch.stack([R.rotate(y[p], p, THETA) for p in range(len(text))])  # noqa: E731
            q, k = turn(q), turn(k)
            rounded = lambda y: y.to(R.TORCH[self.dtype]).double()  # noqa: E731
            k, v = rounded(k.float()).repeat_interleave(self.heads // self.kv, 1), rounded(v.float()).repeat_interleave(self.heads // self.kv, 1)
            z = torch.einsum("qhd,khd->hqk", q, k) / math.sqrt(self.d)
            z = z.masked_fill(torch.ones(len(text), len(text)).triu(1).bool(), -math.inf)
            x = x + torch.einsum("hqk,khd->qhd", z.softmax(-1), v).flatten(1) @ self.wo[l].double().T
        return (x @ self.head.double().T)[-1]


@pytest.mark.parametrize("dtype,bound", [("fp32", 1e-4), ("fp16", 5e-3), ("bf16", 4e-2)])
def test_a_beam_search(dtype, bound):
    """Append, attention, selection and reordering over nine steps: every step's logits are those of the texts so far, computed from scratch in 64 bits, and every
    selection that of the step's logits.  Bound: fp32 sums (1e-4 of the logits' scale is ample for two layers); a cache of 16 bits may round a key the other way
    than the reference does where the two differ in their last bits, half a step of 2^-10 (fp16), 2^-7 (bf16) of values next to the rounding border, over
    d_head keys and two layers: some steps of the type."""
    B = Beams(dtype, [[5, 17, 80, 3, 9], [11], [1, 2, 3, 4, 5, 6, 7, 8]], seed=11)
    G, W = len(B.prompts), B.width
    out = lambda t: torch.empty(G, W, dtype=t, device="cuda")  # noqa: E731
    z = B.start()[:, :1]
    scores, ended = torch.zeros(G, 1, device="cuda"), torch.zeros(G, 1, dtype=torch.int32, device="cuda")
    for step in range(9):
        for g, texts in enumerate(B.texts):
            for b, text in enumerate(texts):
                want = B.logits64(text)
                off = (z[g, b].cpu().double() - want).abs().max() / want.abs().max()
                assert off < bound, (step, g, b, off)
        s, t, p, e = out(torch.float32), out(torch.int32), out(torch.int32), out(torch.int32)
        P().spd_op_beam_select("fp32", z, scores, s, t, p, ended=ended, end_token=13, out_ended=e)
        for g in range(G):
            chosen = R.select(z[g].cpu(), scores[g].cpu(), W, 1.0, ended[g].cpu(), 13)
            assert [(v, b) for _, v, b, _ in chosen] == list(zip(t[g].tolist(), p[g].tolist())), step
        B.texts = [[B.texts[g][b] + [v] for b, v in zip(p[g].tolist(), t[g].tolist())] for g in range(G)]
        P().spd_op_beam_reorder(dtype, B.K, B.V, B.table, p, B.length, B.spare, W, err=B.err)
        B.table, B.spare, scores, ended = B.spare, B.table, s, e
        pos, B.length = B.length, B.length + 1
        z = B.forward(t.flatten(), ints(range(G * W)).cuda(), pos, W, B.table, B.shared, B.length, 7, 20).view(G, W, -1)
    assert int(B.err) == 0


# ------------------------------------------------------------------ streams and graphs
@pytest.mark.parametrize("heads,max_own,vocab", [(8, 250, 5000), (16, 700, 3000), (8, 700, 5000)])
def test_operators_in_a_graph_and_on_another_stream(heads, max_own, vocab):
    """A step of all four captured once and replayed with other lengths, positions and scores (they are on the device), between eager work; a second graph of the same
    operators has scratch of its own.  Every replay equals the eager calls.  One block per sequence and head, and shared positions cut into chunks, a tile of 32 rows
    through LDS and one of 16; the selection in one launch and in two."""
    g = gen(12)
    W, kv, d, page, n_pages = 4, 2, 128, 16, 420
    n = 2 * W
    K0, V0 = (torch.randn(1, n_pages, kv, page, d, generator=g).half().cuda() for _ in range(2))
    table = torch.randperm(n_pages, generator=g).int()[:n * 50].view(n, 50).cuda()
    qkv, logits = torch.randn(n, (heads + 2 * kv) * d, generator=g).cuda(), torch.randn(2, W, vocab, generator=g).cuda()
    seq = ints(range(n)).cuda()

    class Step:
        def __init__(self):
            self.K, self.V, self.length, self.pos = K0.clone(), V0.clone(), torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
            self.shared, self.scores = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, W, device="cuda")
            self.q, self.out = (torch.empty(n, heads, d, device="cuda") for _ in range(2))
            self.s, self.t, self.p = torch.empty(2, W, device="cuda"), *(torch.empty(2, W, dtype=torch.int32, device="cuda") for _ in range(2))
            self.table = torch.empty_like(table)

        def load(self, i):
            self.K.copy_(K0), self.V.copy_(V0)
            self.shared.fill_(40 + 7 * i)
            self.length.copy_(ints([200 + 9 * i + 1] * n))
            self.pos.copy_(self.length - 1)
            self.scores.copy_(-torch.rand(2, W, generator=gen(100 + i)))

        def run(self):
            q, k, v = split(qkv, heads, kv, d)
            pkg = P()
            pkg.spd_op_append_paged("fp16", self.K[0], self.V[0], table, k, v, seq, self.pos, THETA, q=q, q_out=self.q)
            pkg.spd_op_attention_shared("fp16", self.q, self.K[0], self.V[0], table, self.shared, self.length, self.out, W, 100, max_own)
            pkg.spd_op_beam_select("fp32", logits, self.scores, self.s, self.t, self.p)
            pkg.spd_op_beam_reorder("fp16", self.K, self.V, table, self.p, self.length, self.table, W)

        def results(self):
            return [x.clone() for x in (self.K, self.V, self.out, self.s, self.t, self.p, self.table)]

    eager, steps, graphs = Step(), [Step(), Step()], []
    want = []
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
