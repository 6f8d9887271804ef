"""The operators of several sequences over one paged cache at the limits of what their arguments may hold."""
import itertools
import math

import pytest
import torch

import batch_reference as R
from test_batch_ops_limits_host import RINGS, SELECTIONS
from test_gpu_batch_ops import Beams, P, attend, attention_case, close, gen, ints, reorder_case, say

pytestmark = pytest.mark.gpu

# dtype, heads, kv, shared, lengths, width: one block per sequence and head; cut into chunks, up to 16 query rows and more
PATHS = [("short", 4, 2, [37, 30], [45, 50, 36, 47], 2), ("few", 4, 2, [700], [705, 720, 690], 3), ("many", 16, 2, [700], [705, 720, 690], 3)]


def by_path(f):
    return pytest.mark.parametrize("heads,kv,shared,lengths,width", [p[1:] for p in PATHS], ids=[p[0] for p in PATHS])(f)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@by_path
def test_attention_of_values_as_large_as_the_type_holds(dtype, heads, kv, shared, lengths, width):
    """Weights add up to one, so no result passes the largest value.  Values of some 2^122 (2^13 in fp16), all of them nearly the largest number, and small ones."""
    q, K, V, table, *rest = attention_case(dtype, heads, kv, 64, 16, shared, lengths, width, seed=21)
    for scale in (2.0 ** 13,) if dtype == "fp16" else (2.0 ** 122, 2.0 ** -80):
        case = (q, K, (V.float() * scale).to(V.dtype), table, *rest)
        got, err = attend(dtype, *case, width)
        assert err == 0
        close(got, R.attention(*case, width))
    # all alike: 1 - 2^-8 of 2^128 (65504 in fp16), fp32 sums of some hundred weights, above and below: 1e-6 of it
    most = 65504.0 if dtype == "fp16" else 2.0 ** 128 * (1 - 2.0 ** -8)
    got, _ = attend(dtype, q, K, torch.where(V.isnan(), V, torch.full_like(V, most)), table, *rest, width)
    assert ((got.double() / most - 1.0).abs() < 1e-6).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@by_path
def test_attention_of_scores_far_from_zero(dtype, heads, kv, shared, lengths, width):
    """Scores of 2^19 to 2^37, all of them exact numbers whose next neighbours are 2^12 and more away: the best key takes all, equal best ones share."""
    q, K, V, table, *rest = attention_case(dtype, heads, kv, 64, 16, shared, lengths, width, seed=22)
    g = gen(23)
    K = torch.where(K.isnan(), K, torch.randint(-100, 101, K.shape, generator=g).to(K.dtype))
    q = torch.zeros_like(q)
    q[..., 0] = torch.tensor([2.0 ** 15, 2.0 ** 22, -(2.0 ** 26), 2.0 ** 33]).repeat(heads // 4)     # over sqrt(64): steps of 2^12 and more
    got, err = attend(dtype, q, K, V, table, *rest, width)
    assert err == 0
    close(got, R.attention(q, K, V, table, *rest, width), 1e-6)             # a handful of equal weights: some 2^-22
    # all scores far below zero, and near one another: the definition's weights to a few steps of the scores (2^-3 at 2^21: compared where they are exact)
    K[..., 0] = torch.where(K[..., 0].isnan(), K[..., 0], -120.0 - (K[..., 0] > 0).to(K.dtype) * 8)
    q[..., 0] = 2.0 ** 20
    got, err = attend(dtype, q, K, V, table, *rest, width)
    assert err == 0
    close(got, R.attention(q, K, V, table, *rest, width), 1e-5)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("heads", [4, 16])
def test_attention_reports_pages_that_a_sequence_needs_alone(dtype, heads):
    """Shared positions with blocks of their own: entries behind every sequence of a group may hold anything, also where shared[g] reaches over them."""
    q, K, V, table, shared, length = attention_case(dtype, heads, 2, 64, 16, [700, 650, 700], [300, 17, 0, 290, 651, 700, 650, 20, 0, 0, 0, 0], 4, seed=24)
    want = R.attention(q, K, V, table, shared, length, 4)
    table[0, 300 // 16 + 1:], table[8] = -5, 1 << 30
    for max_shared, max_own in ((700, 50), (704, 300)):
        got, err = attend(dtype, q, K, V, table, shared, length, 4, max_shared=max_shared, max_own=max_own)
        assert err == 0
        close(got, want)
    table[0, 300 // 16] = -5                                                # the last one that is needed
    got, err = attend(dtype, q, K, V, table, shared, length, 4, max_shared=700, max_own=50)
    assert err == 1
    close(got, R.attention(q, K, V, table, shared, length, 4))


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_attention_weights_of_many_small_ones_add_up_to_one(dtype):
    """Where a wave keeps one reference over many keys: a sequence of 60000 positions that ends inside a longer shared part, the first key 2^20 above the others.
    Values of one come out as one: a weight is off by 2^-37 of the largest at most, to either side, and the many together by 60000 x 2^-37 = 4e-7.  The sums: a
    lane adds 3750 weights and a wave's product 1875 partial sums to what the first key left there, each rounded to 2^-24 of it at most, a uniform error:
    sqrt(3750 + 1875) 2^-24 / sqrt(3) = 2.6e-6 as one standard deviation."""
    n, d = 60_000, 64
    q = torch.zeros(2, 4, d)
    q[..., 0] = 8.0
    pages = (n + 200) // 16 + 1
    K = torch.zeros(pages, 1, 16, d)
    K[..., 0] = 0.25 * torch.rand(pages, 1, 16, generator=gen(25))
    K[0, 0, 0, 0] = 14.0                                     # 8 x 14 / 8 = 14 = 20.2 log 2
    V = torch.ones(pages, 1, 16, d)
    table = torch.arange(pages, dtype=torch.int32).expand(2, -1).contiguous()
    got, err = attend(dtype, q, K.to(R.TORCH[dtype]), V.to(R.TORCH[dtype]), table, ints([n + 100]), ints([n, n - 1]), 2, max_own=1)
    assert err == 0 and (got - 1.0).abs().max() < 8e-6, (got - 1.0).abs().max()       # three standard deviations


def balanced(dtype, g, rows, d=128):
    """Queries of some units with all 24 bits in use, and two keys for each whose scores differ by little, but come about from quite different products."""
    q = torch.randn(rows, d, generator=g, dtype=torch.float64) * 4
    q = q.float().double()
    k = torch.randn(rows, 2, d, generator=g, dtype=torch.float64) * 4
    k -= (k @ q[:, :, None]) / (q * q).sum(-1)[:, None, None] * q[:, None]
    return q.float(), k.to(R.TORCH[dtype])


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("heads,width,bound", [(4, 1, 0), (64, 1, 0), (4, 2, 600), (64, 2, 600)], ids=["alone", "alone-many", "few", "many"])
def test_attention_uses_all_bits_of_its_queries(dtype, heads, width, bound):
    """Of two keys the first has the value one, the other's is zero: the result is a weight p, off by p (1 - p) <= 1/4 of the scores' error.  A score of 128 products of
    some 16 / sqrt(128): twelve steps of 32 products, each rounded to 2^-25 of a partial sum (at most some 16 in all), 6e-6 at worst, 2e-6 of the weight, and the
    exponential's 2^-22.  A query without its last eight bits (2^-16 of 4, over 128 keys of 4, / sqrt(128), random signs) moves a score by some 1e-4."""
    g = gen(26)
    n_kv, n_seq, page = 2, 16, 4
    q, K = torch.zeros(n_seq, heads, 128), torch.zeros(n_seq, n_kv, page, 128, dtype=R.TORCH[dtype])
    V = torch.zeros_like(K)
    for s in range(0, n_seq, width):
        qq, kk = balanced(dtype, g, n_kv)
        q[s:s + width], K[s, :, :2] = qq.repeat_interleave(heads // n_kv, 0), kk
    V[:, :, 0] = 1.0
    table = torch.full((n_seq, 150), -1, dtype=torch.int32)
    table[:, 0] = torch.arange(n_seq)
    rest = (K, V, table, ints([2] * (n_seq // width)), ints([2] * n_seq))
    got, err = attend(dtype, q, *rest, width, max_shared=max(bound, 2))     # (a bound of 600: blocks of their own for the shared positions)
    want = R.attention(q, *rest, width)
    assert err == 0 and 0.2 < want[..., 0].mean() < 0.8 and (got - want).abs().max() < 4e-6, (got - want).abs().max()
    if dtype != "fp32":                                      # what the bound has to see: queries of fewer bits, in the oracle
        cut = (q.view(torch.int32) & ~(0xFF if dtype == "bf16" else 0x1FFF)).view(torch.float32)
        assert (R.attention(cut, *rest, width) - want).abs().max() > 8e-6


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("groups,n_in,vocab", [shape for shape, _ in SELECTIONS])
def test_select_with_slices_of_every_length(dtype, groups, n_in, vocab):
    """Ties inside and across slices, a last slice that is not full, in every instance of the first kernel."""
    say("select", dtype, groups, n_in, vocab)
    g = gen(vocab + groups)
    logits = (torch.randn(groups, n_in, vocab, generator=g) * 3).to(R.TORCH[dtype])
    top = logits[:, :, :512].float().amax(-1, keepdim=True).to(logits.dtype) + 2
    for at in (0, 511, 513, 1023, 4097, vocab - 1, vocab - 2):              # equal logits here and there, the last entries among them
        logits[:, ::2, at] = top[:, ::2, 0]
    logits[0, 1], logits[-1, 2] = 0.5, logits[-1, 0]                        # a row all alike; two equal rows
    scores = -torch.rand(groups, n_in, generator=g) * 4
    scores[-1, 2] = scores[-1, 0]
    few = sorted({0, groups // 2, groups - 1})
    out = [torch.empty(groups, 16, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]
    P().spd_op_beam_select(dtype, logits.cuda(), scores.cuda(), *out, tau=0.9)
    s, t, p = (x.cpu() for x in out)
    for i in few:
        want = R.select(logits[i].float(), scores[i], 16, 0.9)
        assert t[i].tolist() == [c[1] for c in want] and p[i].tolist() == [c[2] for c in want], i
        score = torch.tensor([c[0] for c in want], dtype=torch.float64)
        # as in the test of random logits: the sum of exponentials 1e-6 of itself, arguments of up to 30 / tau rounded at 2^-23
        assert ((s[i] - score).abs() <= 5e-6 + score.abs() * 2.0 ** -24).all()


def positions(K, V, table, shared, length, width):
    """What each sequence's positions hold, [layers, kv, positions, 2 d] per sequence, read as the attention reads them."""
    page = K.shape[3]
    rows = []
    for s, n in enumerate(length.tolist()):
        p = torch.arange(n)
        at = torch.where(p < shared[s // width], table[s - s % width, p // page], table[s, p // page]).long()
        assert ((at >= 0) & (at < K.shape[1])).all()
        rows.append(torch.cat([K[:, at, :, p % page], V[:, at, :, p % page]], -1))
    return rows


@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
@pytest.mark.parametrize("page,shared,length", [(16, 37, 45), (16, 37, 61), (16, 37, 37), (16, 32, 40), (4, 3, 2), (8, 0, 9), (16, 37, 48), (4, 6, 7), (64, 33, 100)])
def test_reorder_keeps_shared_positions_that_the_first_row_alone_holds(dtype, page, shared, length):
    """All choices of three parents, on caches filled as for the attention: pages of NaN but for what counts, entries that no call needs out of range.  Every beam holds
    its parent's positions, as the attention reads them, bit by bit; three times in a row, with the parents of another group each time."""
    say("reorder", dtype, page, shared, length)
    choices = list(itertools.product(range(3), repeat=3))
    n = 3 * len(choices)
    cases = [attention_case(dtype, 1, 2, 16, page, [shared] * len(choices), [length] * n, 3, seed=31 + l) for l in range(2)]
    table = cases[0][3].clone()
    order = torch.randperm(n * table.shape[1], generator=gen(31)).int().view(n, -1)     # (attention_case's own pages: rows have one to write on, filled or not)
    e = length // page
    K, V = (torch.full((2, n * table.shape[1], 2, page, 16), math.nan).to(R.TORCH[dtype]) for _ in range(2))
    for s in range(n):
        for i in range(table.shape[1]):
            if table[s, i] >= 0:
                for l, c in enumerate(cases):
                    K[l, order[s, i]], V[l, order[s, i]] = c[1][cases[l][3][s, i]], c[2][cases[l][3][s, i]]
                table[s, i] = order[s, i]
            elif i >= min(e, min(shared, length) // page):
                table[s, i] = order[s, i]
    sh, ln = ints([shared] * len(choices)), ints([length] * n)
    Kd, Vd, td = K.cuda(), V.cuda(), table.cuda()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    for step in range(3):
        before = positions(Kd.cpu(), Vd.cpu(), td.cpu(), sh, ln, 3)
        parents = ints(choices[step:] + choices[:step])
        out = torch.full_like(td, -9)
        P().spd_op_beam_reorder(dtype, Kd, Vd, td, parents.cuda(), ln.cuda(), out, 3, err=err, shared=sh.cuda())
        assert int(err) == 0
        after = positions(Kd.cpu(), Vd.cpu(), out.cpu(), sh, ln, 3)
        for s in range(n):
            was = before[s - s % 3 + int(parents[s // 3, s % 3])]
            assert not was.isnan().any() and torch.equal(after[s], was), (step, s, parents[s // 3].tolist())
        pages = out.cpu()[:, e:].sort().values if length < page * out.shape[1] else out.cpu()[:, :0]
        assert len(set(pages.flatten().tolist())) == pages.numel()           # every beam has pages of its own to go on with
        td = out


def test_reorder_leaves_a_group_whose_shared_positions_make_no_sense_as_it_was():
    K, V, table, length = reorder_case("fp16", 2, 2, 64, 16, [37, 40], 3, seed=32)
    parents = ints([[2, 2, 0], [0, 1, 1]])
    a, b, c = R.reorder(K, V, table, ints([[0, 1, 2], [0, 1, 1]]), length, 3)
    for shared, entry, page in ((-1, None, 0), (16 * table.shape[1] + 1, None, 0), (20, (0, 1), -1), (20, (2, 1), len(K[0])), (35, (0, 2), 1 << 30), (35, (2, 2), -7)):
        bad, want = table.clone(), c.clone()
        if entry:
            bad[entry] = page
            want[entry] = page
        Kd, Vd, out, err = K.cuda(), V.cuda(), torch.full_like(table, -9).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
        P().spd_op_beam_reorder("fp16", Kd, Vd, bad.cuda(), parents.cuda(), length.cuda(), out, 3, err=err, shared=ints([shared, 0]).cuda())
        assert torch.equal(out.cpu(), want) and torch.equal(Kd.cpu(), a) and torch.equal(Vd.cpu(), b) and int(err) == 1, (shared, entry)


class FirstRows(Beams):
    """Prompts in each group's first row alone; the other rows' pages hold NaN there, and their entries in front of the page where a prompt ends are no pages."""

    def start(self):
        W = self.width
        for s in range(len(self.prompts) * W):
            if s % W:
                self.table[s, :len(self.prompts[s // W]) // self.page] = -1
        self.shared = ints([len(p) for p in self.prompts]).cuda()
        prompts, self.prompts = self.prompts, [p if s % W == 0 else [] for p in self.prompts for s in range(W)]
        self.width = 1                                          # (each row by itself, those without a prompt as padding)
        n, logits = len(self.prompts), None
        for t in range(max(map(len, self.prompts))):
            on = [t < len(p) for p in self.prompts]
            tokens = torch.tensor([p[t] if o else 0 for p, o in zip(self.prompts, on)]).cuda()
            length = ints([t + 1 if o else 0 for o in on]).cuda()
            z = self.forward(tokens, ints([s if o else -1 for s, o in enumerate(on)]).cuda(), ints([t] * n).cuda(), 1, self.table, torch.zeros(n, dtype=torch.int32, device="cuda"), length, 0,
                             t + 1)
            logits = z if logits is None else torch.where((length > 0)[:, None], z, logits)
        self.prompts, self.width = prompts, W
        self.length = ints([len(prompts[s // W]) for s in range(n)]).cuda()
        return logits.view(len(prompts), W, -1)


@pytest.mark.parametrize("dtype,bound", [("fp32", 1e-4), ("fp16", 5e-3), ("bf16", 4e-2)])
def test_a_beam_search_over_prompts_that_the_first_rows_hold(dtype, bound):
    """As test_a_beam_search, its bounds too, with prompts that end inside pages, at their ends and in front of the first page's."""
    B = FirstRows(dtype, [[5, 17, 80, 3, 9, 2], [11], [1, 2, 3, 4, 5, 6, 7, 8]], seed=11)
    G, W = len(B.prompts), B.width
    z = B.start()[:, :1]
    scores, ended = torch.zeros(G, 1, device="cuda"), torch.zeros(G, 1, dtype=torch.int32, device="cuda")
    moved = 0
    for step in range(9):
        for g, texts in enumerate(B.texts):
            for b, text in enumerate(texts):
                want = B.logits64(text)
                off = (z[g, b].cpu().double() - want).abs().max() / want.abs().max()
                assert off < bound, (step, g, b, off)
        s, t, p, e = (torch.empty(G, W, dtype=x, device="cuda") for x in (torch.float32, torch.int32, torch.int32, torch.int32))
        P().spd_op_beam_select("fp32", z, scores, s, t, p, ended=ended, end_token=13, out_ended=e)
        B.texts = [[B.texts[g][b] + [v] for b, v in zip(p[g].tolist(), t[g].tolist())] for g in range(G)]
        moved += int((p[:, 0] != 0).sum())
        P().spd_op_beam_reorder(dtype, B.K, B.V, B.table, p, B.length, B.spare, W, err=B.err, shared=B.shared)
        B.table, B.spare, scores, ended = B.spare, B.table, s, e
        pos, B.length = B.length, B.length + 1
        z = B.forward(t.flatten(), ints(range(G * W)).cuda(), pos, W, B.table, B.shared, B.length, 8, 20).view(G, W, -1)
    assert int(B.err) == 0 and moved > 0                        # (a first beam that goes on from another row)


def on_gpu(dtype, heads, kv, d, page, groups, width, shared, own, seed):
    """A larger case, made on the GPU: every row has pages of its own in random order, those of shared positions count in a group's first row alone.  Lengths behind the shared
    positions, at their end, inside them and none."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = groups * width
    shareds = [shared - 3 * i for i in range(groups)]
    lengths = [shareds[s // width] + own - s % (own + 1) for s in range(n)]
    lengths[1], lengths[width], lengths[-1] = shareds[0] - 5, shareds[1], 0
    entries = (max(max(lengths), shared) - 1) // page + 1
    table = torch.randperm(n * entries, generator=g, device="cuda").int().view(n, entries)
    K, V = (torch.empty(n * entries, kv, page, d, device="cuda", dtype=R.TORCH[dtype]).normal_(generator=g) for _ in range(2))
    q = torch.empty(n, heads, d, device="cuda").normal_(generator=g)
    return q, K, V, table, ints(shareds).cuda(), ints(lengths).cuda()


def in_64_bits(q, K, V, table, shared, length, width):
    """batch_reference.attention with a sequence's heads at once, on the GPU."""
    n, heads, d = q.shape
    pages, kv, page, _ = K.shape
    out = torch.zeros(n, heads, d, dtype=torch.float64, device="cuda")
    for s, m in enumerate(length.tolist()):
        p = torch.arange(m, device="cuda")
        at = torch.where(p < shared[s // width], table[s - s % width, p // page], table[s, p // page]).long()
        there = (at >= 0) & (at < pages)
        at, p = at[there], p[there]
        if len(p):
            k, v = (x[at, :, p % page].double().transpose(0, 1).contiguous() for x in (K, V))
            z = torch.matmul(q[s].double().view(kv, heads // kv, d), k.transpose(1, 2).contiguous()) / math.sqrt(d)
            out[s] = torch.matmul(z.softmax(-1), v).view(heads, d)
    return out


def attend_on_gpu(dtype, q, K, V, table, shared, length, width, max_own):
    out, err = torch.full_like(q, math.nan), torch.zeros(1, dtype=torch.int32, device="cuda")
    P().spd_op_attention_shared(dtype, q, K, V, table, shared, length, out, width, int(shared.max()), max_own, err=err)
    return out, int(err)


@pytest.mark.parametrize("case", [c for c, _ in RINGS], ids=lambda c: "-".join(map(str, c)))
def test_attention_through_stages_that_are_filled_again(case):
    """Blocks whose waves share out rows, over chunks of more than twice the stages that LDS holds; then with a page that is none late in a chunk."""
    say("ring", *case)
    dtype, heads, kv, d, page, groups, width, shared, own = case
    q, K, V, table, *rest = on_gpu(*case, seed=d + width)
    got, err = attend_on_gpu(dtype, q, K, V, table, *rest, width, own)
    assert err == 0
    close(got, in_64_bits(q, K, V, table, *rest, width))
    chunk = P().spd_test_attention_shared_cut(dtype, groups * width, width, heads, kv, d, shared, own)[1]
    table[width, (2 * chunk - 40) // page] = -1              # of the second group, in the last stages of the second chunk
    table[0, (chunk - 70) // page] = len(K)
    got, err = attend_on_gpu(dtype, q, K, V, table, *rest, width, own)
    assert err == 1
    close(got, in_64_bits(q, K, V, table, *rest, width))


@pytest.mark.parametrize("heads", [4, 16])
def test_shared_positions_in_a_graph(heads):
    """Attention cut into chunks and a reordering that keeps shared positions, captured once and replayed with other lengths, shared parts and parents: sequences that end before
    the shared positions do, groups without any, none at all.  Every replay equals the eager calls; err is set by the one that has a reason."""
    g = gen(41)
    W, G, kv, d, page, entries = 3, 3, 2, 64, 16, 50
    n = W * G
    K0, V0 = (torch.randn(2, n * entries, kv, page, d, generator=g).half().cuda() for _ in range(2))
    table = torch.randperm(n * entries, generator=g).int().view(n, entries).cuda()
    q = torch.randn(n, heads, d, generator=g).cuda()
    # shared, lengths (the same within a group: they are reordered), parents, err
    runs = [([600, 40, 700], [640, 50, 655], [[1, 1, 0], [0, 1, 2], [2, 0, 2]], 0), ([600, 700, 0], [599, 0, 33], [[2, 2, 2], [1, 0, 2], [0, 0, 0]], 0),
            ([0, 0, 0], [0, 0, 0], [[1, 2, 0]] * 3, 0), ([-1, 650, 700], [640, 650, 703], [[1, 1, 0], [2, 1, 1], [0, 1, 2]], 1), ([597, 33, 700], [640, 50, 701], [[2, 1, 0], [1, 1, 1], [2, 2, 1]], 0)]

    class Step:
        def __init__(self):
            self.K, self.V, self.out, self.table = K0.clone(), V0.clone(), torch.empty_like(q), torch.empty_like(table)
            self.shared, self.length, self.parents = ints([0] * G).cuda(), ints([0] * n).cuda(), torch.zeros(G, W, dtype=torch.int32, device="cuda")
            self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

        def load(self, run):
            self.K.copy_(K0), self.V.copy_(V0), self.err.zero_()
            self.shared.copy_(ints(run[0])), self.length.copy_(ints([x for x in run[1] for _ in range(W)])), self.parents.copy_(ints(run[2]))

        def run(self):
            P().spd_op_attention_shared("fp16", q, self.K[0], self.V[0], table, self.shared, self.length, self.out, W, 700, 60, err=self.err)
            P().spd_op_beam_reorder("fp16", self.K, self.V, table, self.parents, self.length, self.table, W, err=self.err, shared=self.shared)

        def results(self):
            return [x.clone() for x in (self.K, self.V, self.out, self.table, self.err)]

    eager, step = Step(), Step()
    step.load(runs[0])
    step.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    for i in (0, 1, 2, 3, 4, 1, 0):
        eager.load(runs[i])
        eager.run()
        want = eager.results()
        step.load(runs[i])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(step.results(), want)), i
        assert int(want[4]) == runs[i][3], i
        if not runs[i][3]:
            close(want[2], in_64_bits(q, K0[0], V0[0], table, eager.shared, eager.length, W))


def test_reorder_of_layers_that_lie_in_turn():
    """A layer's keys, its values and room for something else, then the next layer's: the C entry takes the distance between layers; the tables lie in that room."""
    K, V, table, length = reorder_case("fp16", 3, 2, 64, 16, [37, 10], 4, seed=51)
    parents = ints([[2, 2, 0, 2], [1, 0, 0, 3]])
    one = K[0].numel()
    store = torch.full((3, 3, one), 7.0, dtype=torch.float16, device="cuda")
    store[:, 0], store[:, 2] = K.flatten(1).cuda(), V.flatten(1).cuda()
    room = store[1, 1].view(torch.int32)
    sizes = [table.numel(), table.numel(), parents.numel(), length.numel()]
    t, out, p, n = room[:sum(sizes)].split(sizes)
    t.copy_(table.flatten()), p.copy_(parents.flatten()), n.copy_(length)
    rc = P().lib().spd_op_beam_reorder(2, store[0, 0].data_ptr(), store[0, 2].data_ptr(), t.data_ptr(), K.shape[1], 2, 16, 64, 8, table.shape[1], 3, 3 * one, 4, p.data_ptr(), n.data_ptr(),
                                       out.data_ptr(), None, torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    a, b, c = R.reorder(K, V, table, parents, length, 4)
    assert torch.equal(out.cpu().view(table.shape), c) and torch.equal(store[:, 0].cpu().view(K.shape), a) and torch.equal(store[:, 2].cpu().view(V.shape), b)
    assert (store[0, 1] == 7.0).all() and (store[2, 1] == 7.0).all()
