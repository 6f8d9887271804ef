"""Decisions and draws of spd_op_verify_drafts where they are hard: numbers next to a border, probabilities next to nothing, the forms that large calls take.

The definition here, apart from the kernels': everything in logarithms, in 64 bits (Python's whole and decimal numbers where that is not enough)."""
import math

import pytest
import torch

import chunk_reference as R
import verify_reference as V
from test_gpu_chunk_ops import P, dev, gen, ints, run_verify, say, verify_case, zero  # noqa: F401

pytestmark = pytest.mark.gpu


def between(a, b):
    """An fp32 number strictly between two 64-bit numbers, as far from both as one can be."""
    u = torch.tensor((a + b) / 2, dtype=torch.float32)
    assert min(a, b) < float(u) < max(a, b)
    return float(u)


# ------------------------------------------------------------------ temperatures
@pytest.mark.parametrize("tau", [0.7, 1.1, 0.3])
def test_a_draw_goes_by_tau_in_64_bits(tau):
    """Two tokens, the first with p = exp(-30) / (1 + exp(-30)), u between that and the same for tau rounded to fp32.  (They are 30 (2^-26 .. 2^-25) = 4e-7 .. 9e-7 of themselves apart, u's steps 2^-24 = 6e-8.)"""
    z = torch.tensor([[-30.0 * tau, 0.0]])
    of = lambda t: 1.0 / (1.0 + math.exp(-float(z[0, 0]) / t))  # noqa: E731
    tau32 = float(torch.tensor(tau, dtype=torch.float32))
    u = between(of(tau), of(tau32))
    case = dict(logits=z, tokens=ints([0]), first=ints([0, 1]), u=torch.tensor([u]), draft_logits=None)
    out_t, _, _, err = run_verify("fp32", case, tau=tau)
    assert err == 0 and int(out_t[0]) == (0 if u < of(tau) else 1)


@pytest.mark.parametrize("drawn", [False, True])
def test_a_draft_is_decided_by_tau_in_64_bits(drawn):
    """The draft has p = exp(-30) / (1 + exp(-30)) (drawn: q = 1/2, and the drafter's temperature is what is rounded: q = exp(-30) .. beside p = 1/2 that of u q < p)."""
    tau = 0.7
    tau32 = float(torch.tensor(tau, dtype=torch.float32))
    z = torch.tensor([[-30.0 * tau, 0.0], [0.0, 0.0]])
    of = lambda t: 1.0 / (1.0 + math.exp(-float(z[0, 0]) / t))  # noqa: E731
    if not drawn:                            # stands for u < p
        u = between(of(tau), of(tau32))
        want = u < of(tau)
        case = dict(logits=z, tokens=ints([0, 0]), first=ints([0, 2]), u=torch.tensor([u, 0.5]), draft_logits=None)
        _, _, out_a, _ = run_verify("fp32", case, tau=tau)
    else:                                    # p = of(1.0) with a logit that makes it about half of q: stands for u < p / q
        p_row = torch.tensor([[-30.0 - math.log(2.0), 0.0], [0.0, 0.0]])
        p = 1.0 / (1.0 + math.exp(-float(p_row[0, 0])))
        u = between(p / of(tau), p / of(tau32))
        want = u < p / of(tau)
        case = dict(logits=p_row, tokens=ints([0, 0]), first=ints([0, 2]), u=torch.tensor([u, 0.5]), draft_logits=z)
        _, _, out_a, _ = run_verify("fp32", case, tau=1.0, draft_tau=tau)
    assert int(out_a[0]) == int(want)


# ------------------------------------------------------------------ decisions and draws against the definition
def check64(dtype, case, tau=1.0, draft_tau=1.0, sure=2.0 ** -40, got=None):
    """All outputs are the definition's.  Exponentials of 64 bits are off by 2e-13, a quotient of two sums by 6e-13 < 2^-40 = 9e-13: it and the random number are further apart than `sure`, relative to the quotient; the draw is
    2^-40 of the sum from the nearest border, or u is 0 (which is exact).  A logarithm of a probability is off by 2^-22 and half a step of itself."""
    out_t, out_l, out_a, err = got or run_verify(dtype, case, tau, draft_tau)
    first, bad, seen = case["first"].tolist(), False, torch.zeros(len(out_t), dtype=torch.bool)
    for s, (a, b) in enumerate(zip(first, first[1:])):
        if a == b:
            assert out_a[s] == 0
            continue
        seen[a:b] = True
        m, given, logp, wrong, near, far = V.verify(case["logits"][a:b], case["tokens"][a:b], case["u"][a:b], tau, None if case["draft_logits"] is None else case["draft_logits"][a:b], draft_tau)
        assert near > sure and (far > 2.0 ** -40 or float(case["u"][b - 1]) == 0.0), (s, near, far)
        bad |= wrong
        assert int(out_a[s]) == m and out_t[a:a + m + 1].tolist() == given, (s, out_a[s], m, out_t[a:b].tolist(), given)
        assert (out_t[a + m + 1:b] == -1).all() and (out_l[a + m + 1:b] == 0).all()
        for i, w in enumerate(logp):
            assert float(out_l[a + i]) == w or abs(float(out_l[a + i]) - w) <= 2.0 ** -22 + abs(w) * 2.0 ** -24, (s, i, out_l[a + i], w)
    assert (out_t[~seen] == -5).all() and (out_l[~seen] == 9.0).all() and err == int(bad)
    return out_t, out_l, out_a


def one_draft(target, drafter, u, draft=1, last=0.5):
    """One sequence per random number: its newest token and one draft, every row `target` and `drafter`."""
    n = len(u)
    rows = lambda x: None if x is None else torch.as_tensor(x).expand(2 * n, -1).contiguous()  # noqa: E731
    return dict(logits=rows(target), draft_logits=rows(drafter), tokens=ints([0, draft] * n), first=ints(range(0, 2 * n + 1, 2)), u=torch.tensor([[x, last] for x in u]).flatten())


@pytest.mark.parametrize("tau,z,y,u,stands", [
    (1.0, -640.0, -630.0, [0.525, 1e-3, 4e-5, 3.5e-5], [0, 0, 0, 1]),        # p / q = e^-10 (1 + e^-2) / (1 + e^-1) = 3.8e-5
    (1.0, -1072.0, -676.0, [0.525, 1e-30, 0.0], [0, 0, 1]),         # 1e-172
    (0.05, -40.0, -32.0, [0.525, 1e-30, 0.0], [0, 0, 1]),           # 3e-70
    (0.01, -12.0, -7.0, [0.525, 1e-30, 0.0], [0, 0, 1]),            # 7e-218
    (0.01, -12.0, -3.0, [0.525, 0.0], [0, 0]),                      # 1e-391: a quotient that counts as 0
    (0.01, -7.0, -12.0, [0.525, 1.0 - 2.0 ** -24], [1, 1]),         # more than one
    (0.01, -12.0, -11.99, [0.3, 0.42], [1, 0]),                     # e^-1 or so (0.37: the logits are rounded)
    (1.0, -1e9, -1e9, [0.525, 1.0 - 2.0 ** -24], [1, 0]),           # masked alike in both: p / q = (1 + e^-2) / (1 + e^-1) = 0.83
    (1.0, -1e9, -5.0, [0.525, 0.0], [0, 0]),                        # masked in the target alone
    (1.0, -5.0, -1e9, [0.525, 0.0], [1, 1]),                        # in the drafter alone
    (1.0, -math.inf, -math.inf, [0.525, 0.0], [0, 0]),
    (1.0, -5.0, -math.inf, [0.525, 0.0], [1, 1])])
def test_drafts_whose_probabilities_64_bits_do_not_hold(tau, z, y, u, stands):
    say("tiny", tau, z, y)
    case = one_draft([0.0, z, -1.0], [0.0, y, -2.0], u)
    _, _, out_a = check64("fp32", case, tau, tau)
    assert out_a.tolist() == stands


@pytest.mark.parametrize("dtype,mask", [("fp32", -1e9), ("fp32", -3.4028234663852886e38), ("bf16", -1e9), ("bf16", -3.3895313892515355e38), ("fp16", -65504.0), ("fp16", -30000.0)])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("u", [0.0, 0.3, 1.0 - 2.0 ** -24])
def test_finite_masks(dtype, mask, drawn, u):
    """Every second token is masked with a finite number, in both models, the first among them: none of these stands (but where the drafter drew it) or is drawn, whatever u."""
    case = verify_case(dtype, [5, 1, 4, 3], 50, seed=31, drawn=drawn)
    for name in ("logits", "draft_logits"):
        if case[name] is not None:
            case[name][:, ::2] = mask
    case["u"][:] = u
    odd = torch.randint(0, 25, case["tokens"].shape, generator=gen(32)).int() * 2 + 1
    case["tokens"] = torch.where(case["tokens"] % 2 == 1, case["tokens"], odd)
    case["tokens"][8] = 12                       # a masked draft
    if drawn:
        case["draft_logits"][7, 12] = 1.0        # that the drafter did not mask
    out_t, _, _ = check64(dtype, case)
    given = out_t[out_t >= 0]
    assert (given % 2 == 1).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("tau,draft_tau", [(0.01, 0.01), (0.003, 0.02), (2.0 ** -100, 2.0 ** -100), (2.0 ** 100, 2.0 ** 100), (1.0, 2.0 ** -100), (40.0, 0.01)])
def test_temperatures_far_from_one(dtype, drawn, tau, draft_tau):
    case = verify_case(dtype, [4, 1, 0, 9, 2, 3, 3, 3], 1037, seed=33, drawn=drawn, noise=0.05)
    check64(dtype, case, tau, draft_tau)


# ------------------------------------------------------------------ next to the border
def neighbours(r):
    """The fp32 numbers on either side of r."""
    x = torch.tensor(r, dtype=torch.float64).float()
    other = torch.nextafter(x, torch.tensor(0.0 if float(x) > r else 2.0))
    return sorted([float(x), float(other)])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("rows,vocab,tau,draft_tau", [(24, 4099, 1.0, 1.0), (140, 4099, 0.7, 1.3), (7, 50258, 0.8, 0.8), (70, 20011, 0.6, 0.7), (700, 4099, 0.9, 0.8)])
def test_random_numbers_next_to_a_quotient(dtype, drawn, rows, vocab, tau, draft_tau):
    """Every row twice, with the fp32 numbers in front of and behind p / q, which sums of fp32 exponentials cannot tell apart: the draft stands with the one and not with the other."""
    say("border", dtype, drawn, rows, vocab)
    case = verify_case(dtype, [1] * rows, vocab, seed=rows, drawn=drawn)
    z, y, tokens, u = case["logits"], case["draft_logits"], [], []
    for r in range(rows):
        ratio = V.log2_probabilities(z[r], tau) - (0.0 if y is None else V.log2_probabilities(y[r], draft_tau))
        x = int(((ratio > -14.0) & (ratio < -0.2)).nonzero()[r % 5])
        for v in neighbours(2.0 ** float(ratio[x])):
            tokens += [0, x]
            u += [v, 0.37]
    four = lambda t: None if t is None else t.repeat_interleave(4, 0)  # noqa: E731
    case = dict(logits=four(z), draft_logits=four(y), tokens=ints(tokens), first=ints(range(0, 4 * rows + 1, 2)), u=torch.tensor(u))
    _, _, out_a = check64(dtype, case, tau, draft_tau)
    assert out_a.tolist() == [1, 0] * rows


def test_many_random_numbers_next_to_quotients_in_one_sequence():
    """Forty drafts that all stand, but the last, each by the smallest step of its random number."""
    z, y = (torch.randn(41, 3001, generator=gen(s)) * 2.5 for s in (41, 42))
    tokens, u = [0], []
    for r in range(40):
        ratio = V.log2_probabilities(z[r], 1.0) - V.log2_probabilities(y[r], 1.0)
        x = int(((ratio > -14.0) & (ratio < -0.2)).nonzero()[r])
        tokens.append(x)
        u.append(neighbours(2.0 ** float(ratio[x]))[r == 39])
    case = dict(logits=z, draft_logits=y, tokens=ints(tokens), first=ints([0, 41]), u=torch.tensor(u + [0.6]))
    _, _, out_a = check64("fp32", case)
    assert out_a.tolist() == [39]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab,gap,ties", [(5, 8.0, 1), (5, 8.0, 2)] + [(v, g, n) for v, g in ((300, 12.0), (33000, 20.0), (131, 3.0)) for n in (1, 2, 7)])
def test_log_probabilities_next_to_nothing(dtype, vocab, gap, ties):
    """A likely token's log p is the logarithm of 1 and what the other tokens weigh.  Sums of those are off by at most 2^-24 (4.2 log2(vocab) + 41 + 8) < 2^-16 of themselves, and so is the logarithm."""
    z = torch.randn(3, vocab, generator=gen(vocab)) - gap
    for i in range(ties):
        z[:, (vocab // 2 + 3 * i) % vocab] = 4.0     # (in the last row one of as many)
    z[:2, [(vocab // 2 + 3 * i) % vocab for i in range(1, ties)]] = -gap
    z = z.to(R.TORCH[dtype])
    case = dict(logits=z, draft_logits=None, tokens=ints([0, vocab // 2, vocab // 2]), first=ints([0, 3]), u=torch.tensor([0.1, 0.1, 0.0]))
    out_t, out_l, out_a = check64(dtype, case)
    want = [float(V.log2_probabilities(z[i], 1.0)[int(out_t[i])]) * math.log(2.0) for i in range(3)]
    assert out_a.tolist() == [2] and -0.2 < want[0] < 0.0
    assert all(abs(float(g) - w) <= abs(w) * 2.0 ** -16 for g, w in zip(out_l, want))


# ------------------------------------------------------------------ slices of 32 logits per thread
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("counts,vocab,tau,draft_tau,pad", [
    ([1 + (5 * i) % 9 for i in range(60)], 50258, 0.8, 1.0, 3), ([1 + (3 * i) % 7 for i in range(33)], 131071, 0.9, 0.9, 0), ([2] * 520, 8193, 1.3, 0.7, 1), ([5, 0] * 420, 8192, 1.0, 1.0, 0), ([3] * 700, 2049, 1.0, 1.1, 2)])
def test_verify_calls_of_many_logits(dtype, drawn, counts, vocab, tau, draft_tau, pad):
    say("verify", dtype, drawn, len(counts), vocab)
    n = sum(counts) + pad
    assert n * 2 * -(-vocab // 8192) >= 4096
    case = verify_case(dtype, counts, vocab, seed=vocab, drawn=drawn, pad=pad)
    _, _, out_a = check64(dtype, case, tau, draft_tau)
    some = torch.tensor(counts) > 1
    if drawn:
        assert 0 < int(out_a.sum()) < int((torch.tensor(counts) - 1).clamp(min=0).sum()) and some.any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_verify_calls_of_many_logits_that_are_no_numbers(dtype):
    """NaN, infinite and masked logits in every slice, rows of nothing else, rows that start on no grid of 16 bytes."""
    counts, vocab = [4] * 103, 33333
    case = verify_case(dtype, counts, vocab, seed=55)
    z, y = case["logits"], case["draft_logits"]
    z[:, 5::7] = math.nan
    y[:, 3::5] = -math.inf
    z[8, 20000] = y[9, 32000] = math.inf
    z[12] = -math.inf
    y[17] = math.nan
    case["tokens"][case["tokens"] % 7 == 5] += 1
    check64(dtype, case)


@pytest.mark.parametrize("first,lost", [([0, 4, 8, 1200], 2), ([-4, 4, 8, 1028], 0)])
def test_verify_calls_of_many_logits_with_firsts_out_of_range(first, lost):
    case = verify_case("bf16", [4, 4, 1020], 8300, seed=56)
    want = run_verify("bf16", case)
    out_t, out_l, out_a, err = run_verify("bf16", dict(case, first=ints(first)))
    assert err == 1 and int(out_a[lost]) == 0
    for s in range(3):
        rows = slice(*case["first"][s:s + 2].tolist())
        if s == lost or (lost == 0 and s == 0):
            assert (out_t[rows] == -5).all() and (out_l[rows] == 9.0).all()
        else:
            assert torch.equal(out_t[rows], want[0][rows]) and torch.equal(out_l[rows], want[1][rows]) and out_a[s] == want[2][s]
