"""Decisions and draws of spd_op_verify_drafts where they are hard: numbers next to a border, probabilities next to nothing, the forms that large calls take.

The definition here, apart from the kernels': everything in logarithms, in 64 bits (Python's whole and decimal numbers where that is not enough)."""
import math

import pytest
import torch

import chunk_reference as R
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
