"""The operators of chunks of new tokens where no other test goes: sequences outside of a call's rows, the forms that large calls take."""
import pytest
import torch

import chunk_reference as R
from test_gpu_chunk_ops import P, attend, attention_case, check, dev, gen, ints, places, pool, say, zero  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ sequences outside of the rows
@pytest.mark.parametrize("dtype,io", [("fp16", "fp32"), ("int8", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("n_seq", [4, 64, 65, 80])
@pytest.mark.parametrize("past", [20, 700])
def test_sequences_without_a_row_whose_numbers_do_not_fit(dtype, io, n_seq, past):
    """Wholly in front of the call's rows, wholly behind them, or without new tokens and of a length that cannot be: *err is set, and every other sequence's rows are what they are without them."""
    say("outside", dtype, io, n_seq, past)
    case = attention_case(dtype, io, 4, 2, 64, 16, [2] * n_seq, [past] * n_seq, seed=n_seq)
    n, longest = 2 * n_seq, past + 2
    run = lambda **changed: attend(dtype, {**case, **changed}, max_new=4, max_len=longest)  # noqa: E731
    want, err = run()
    assert err == 0
    first = case["first"].clone()                            # the first sequence in front of row 0
    first[0], first[1] = -3, 0
    got, err = run(first=first)
    assert err == 1 and torch.equal(got[4:], want[4:])       # (sequence 1 has four new tokens then: rows of its own)
    first = case["first"].clone()                            # the last one behind the last row: the rows in front of it are the last but one's
    first[n_seq - 1], first[n_seq] = n, n + 4
    got, err = run(first=first)
    assert err == 1 and torch.equal(got[:n - 4], want[:n - 4])
    first = case["first"].clone()                            # nothing new at a place behind all rows
    first[n_seq - 1], first[n_seq] = n + 1, n + 1
    _, err = run(first=first)
    assert err == 1
    for at in (0, n_seq // 2, n_seq - 1):                    # no new tokens
        for bad in (-1, longest + 1, 2 ** 31 - 1, -2 ** 31):
            first, length = case["first"].clone(), case["length"].clone()
            if at + 1 < n_seq:
                first[at + 1] = first[at]                    # (the next one has its rows then)
                length[at + 1] = longest
            else:
                first[at] = first[at + 1]
            length[at] = bad
            got, err = run(first=first, length=length)
            keep = torch.ones(n, dtype=torch.bool)
            keep[max(0, 2 * at - 2):2 * at + 4] = False
            assert err == 1 and torch.equal(got[keep], want[keep]), (at, bad)
            length[at] = 0
            assert run(first=first, length=length)[1] == 0, at


# ------------------------------------------------------------------ 8-bit values of very different scales
def eight_bits(io, heads, kv, d, page, news, pasts, seed):
    return attention_case("int8", io, heads, kv, d, page, news, pasts, seed=seed)


@pytest.mark.parametrize("io", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("heads,kv,d,news,pasts", [(2, 1, 64, [3, 40], [90, 20]), (4, 2, 128, [150, 2], [30, 700]), (2, 2, 256, [70], [0]), (8, 1, 32, [30, 9], [100, 0]), (2, 2, 128, [1, 1, 5], [600, 64, 2000])])
@pytest.mark.parametrize("grows", [0.6, -0.6])
def test_attention_over_scales_that_grow_or_fall_along_the_text(io, heads, kv, d, news, pasts, grows):
    """Values a 64th of 2^40 apart from position to position, so that what lies a stage behind a row, which it does not see, is up to 2^39 larger than all that it sees (and, falling, what it sees last 2^39 smaller): every row is
    as near as its own largest that counts, see check()."""
    case = eight_bits(io, heads, kv, d, 16, news, pasts, seed=d)
    table, length = case["table"], case["length"].tolist()
    for s, n in enumerate(length):
        for p in range(n):
            at = (int(table[s, p // 16]), slice(None), p % 16)
            case["V_scale"][at] *= 2.0 ** round(grows * ((p - n) % 64 if grows > 0 else -((n - p) % 64)))
    if io == "fp16":
        case["V_scale"] *= 2.0 ** -22            # (results from the smallest fp16 numbers to past the largest)
    check_all_rows("int8", case)


def io_of(case):
    return case["q"].dtype


def check_all_rows(dtype, case):
    """check(), whose bounds hang on the row's own sum of p |v|; results below fp16's normal numbers are off by half of their step, 2^-25, besides."""
    got, err = attend(dtype, case)
    assert err == 0
    want, size = R.attention(**case)
    half, least = (0.0, 0.0) if got.dtype is torch.float32 else (torch.finfo(got.dtype).eps / 2, 2.0 ** -25 if got.dtype is torch.float16 else 0.0)
    got = got.double()
    allowed = 2 * half * size + 1e-5 * size.amax(-1, keepdim=True) + least
    past = got.isinf()                       # past the largest fp16 number: by what may be off, at least
    assert io_of(case) is torch.float16 or not past.any()
    assert (want.abs() + allowed)[past].ge(65520.0).all() and torch.equal(got[past].sign(), want[past].sign())
    assert float(((got - want).abs() / allowed)[~past].max()) < 1


@pytest.mark.parametrize("io", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("heads,d,news,past", [(2, 64, 3, 90), (4, 128, 2, 800), (1, 256, 70, 200), (32, 128, 5, 400), (2, 128, 140, 60)])
@pytest.mark.parametrize("far", [20, 45, 70])
def test_attention_over_large_scales_that_hardly_count(io, heads, d, news, past, far):
    """A few keys with values 2^far times as large as the others' and scores so far below them that their weights are e^-90 = 2^-130: the others' values are what comes out."""
    case = eight_bits(io, heads, 1, d, 16, [news], [past], seed=far)
    case["q"][..., 0] = 8.0 * d ** 0.5 / 8.0
    table, n = case["table"], int(case["length"][0])
    for p in range(0, n, 37):
        at = (int(table[0, p // 16]), 0, p % 16)
        case["K"][at] = 0
        case["K"][at][0] = -127
        case["K_scale"][at] = 90.0 / 127.0
        case["V_scale"][at] *= 2.0 ** far
    for p in range(n):
        if p % 37:
            case["K"][int(table[0, p // 16]), 0, p % 16, 0] = 0
    check_all_rows("int8", case)


# ------------------------------------------------------------------ the forms that large calls take
@pytest.mark.parametrize("dtype,io", [("fp16", "fp32"), ("fp16", "fp16"), ("bf16", "fp32"), ("bf16", "bf16"), ("int8", "fp32"), ("int8", "fp16"), ("int8", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("heads,kv,d,news,past", [(40, 2, 64, [7, 0, 13, 1, 183, 2, 5], 1500), (33, 3, 32, [3, 250, 1], 700), (43, 1, 128, [1, 1, 200, 1], 900)])
def test_chunks_of_many_rows_are_put_together_two_at_a_time(dtype, io, heads, kv, d, news, past):
    """More than 8192 rows with several chunks of positions, odd in number: pairs of rows of one wave that lie in two tokens, in two sequences, and the last one alone."""
    say("joined", dtype, io, heads, kv, d, news, past)
    n = sum(news) * heads
    assert n > 8192
    check(dtype, attention_case(dtype, io, heads, kv, d, 16, news, [past - 37 * s for s in range(len(news))], seed=d, pad=1))


@pytest.mark.parametrize("dtype", ["int8", "fp16", "bf16", "fp32"])
@pytest.mark.parametrize("out", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("kv,d,lengths", [(8, 128, [4100, 1, 4900]), (3, 64, [20011, 5003]), (5, 256, [3500])])
def test_many_rows_are_read_four_pieces_at_a_time(dtype, out, kv, d, lengths):
    """More than 2^20 pieces of eight elements, with a last block that is not full, padding and pages out of range between them."""
    say("read", dtype, out, kv, d, lengths)
    pages, table, seq, pos = places(16, lengths, 3, seed=d, pad=(0, 1000, 1001, 3333))
    bad = table.clone()
    bad[0, 2:2000:97] = torch.tensor([-1, pages, 2 ** 31 - 1], dtype=torch.int32).repeat(8)[:len(bad[0, 2:2000:97])]
    n = len(seq)
    assert n * 2 * kv * d // 8 >= 1 << 20
    K, V, Ks, Vs = pool(dtype, pages, kv, 16, d, seed=d)
    for which, expected in ((table, 0), (bad, 1)):
        k_out, v_out = (torch.full((n, kv, d), 5.0, dtype=R.TORCH[out], device="cuda") for _ in range(2))
        err = zero()
        P().spd_op_read_paged(dtype, K.cuda(), V.cuda(), which.cuda(), seq.cuda(), pos.cuda(), k_out, v_out, K_scale=dev(Ks), V_scale=dev(Vs), err=err)
        at = torch.where(seq >= 0, which[seq.clamp(min=0).long(), (pos // 16).clamp(min=0).long()], -1)
        ok = (at >= 0) & (at < pages)
        assert int(err) == expected == int(bool((~ok & (seq >= 0)).any()))
        for got, x, scale in ((k_out, K, Ks), (v_out, V, Vs)):
            want = torch.full((n, kv, d), 5.0, dtype=R.TORCH[out])
            y = x.transpose(1, 2)[at[ok].long(), (pos[ok] % 16).long()].float()
            if scale is not None:
                y = y * scale.transpose(1, 2)[at[ok].long(), (pos[ok] % 16).long()][..., None]
            want[ok] = y.to(R.TORCH[out])
            assert torch.equal(got.cpu(), want)


# ------------------------------------------------------------------ what is no number in a chunk that weighs nothing
@pytest.mark.parametrize("dtype,io", [("fp16", "fp32"), ("fp16", "fp16"), ("bf16", "fp32"), ("bf16", "bf16"), ("int8", "fp32"), ("int8", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("heads,news,past", [(2, 3, 1500), (2, 60, 1500), (40, 230, 900)])
def test_a_value_that_is_no_number_counts_in_a_chunk_that_weighs_nothing(dtype, io, heads, news, past):
    """Scores of later chunks are 400 above those of the first, whose weight is 0 in 32 bits: a NaN in it is in the result all the same, as it is where positions are not cut."""
    case = attention_case(dtype, io, heads, 1, 64, 16, [news], [past], seed=heads)
    n = past + news
    case["q"][..., 0] = 80.0
    table = case["table"][0].long()
    for p in range(n):
        at = (table[p // 16], 0, p % 16)
        if dtype == "int8":
            case["K"][at][0] = 0 if p < n - 300 else 127
            case["K_scale"][at] = 40.0 / 127.0 if p >= n - 300 else case["K_scale"][at]
            case["K"][at][1:] = 0 if p >= n - 300 else case["K"][at][1:]
        else:
            case["K"][at][0] = 0.0 if p < n - 300 else 40.0
    clean, err = attend(dtype, case)
    assert err == 0 and bool(clean.isfinite().all())
    at = (table[2], 0, 5)
    if dtype == "int8":
        case["V_scale"][at] = float("nan")
    else:
        case["V"][at][7] = float("nan")
    got, err = attend(dtype, case)
    assert err == 0
    if dtype == "int8":
        assert not got.isfinite().any()
    else:
        assert not got[..., 7].isfinite().any()
        rest = [i for i in range(64) if i != 7]
        assert torch.equal(got[..., rest], clean[..., rest])
