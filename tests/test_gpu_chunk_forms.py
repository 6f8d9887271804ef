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
