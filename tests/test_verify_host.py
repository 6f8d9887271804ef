"""Temperatures of a verification of drafts, seen without a GPU (every status is returned before anything is enqueued)."""
import pytest
import torch

import verify_reference as V
from test_chunk_ops_host import EINVAL, VERIFY, call, pkg  # noqa: F401


@pytest.mark.parametrize("name", ["tau", "draft_tau"])
@pytest.mark.parametrize("value", [2.0 ** -100 * (1 - 2.0 ** -40), 2.0 ** 100 * (1 + 2.0 ** -40)])
def test_temperatures_cross_the_interface_in_64_bits(pkg, name, value):  # noqa: F811
    """Numbers that 32 bits round to the bounds, which are allowed."""
    assert call(pkg, "spd_op_verify_drafts", VERIFY, **{name: value}) == EINVAL
    assert call(pkg, "spd_op_verify_drafts", VERIFY, n_seq=0, **{name: 2.0 ** -100 if value < 1 else 2.0 ** 100}) == 0


# ------------------------------------------------------------------ the reference that the GPU tests go by
def test_reference_verification_in_logarithms():
    """p = (1/2, 1/4, 1/4), q = (1/4, 1/2, 1/4): token 0 always stands, token 1 for u < 1/2, what is left of its row is all at token 0."""
    z, y = torch.tensor([0.5, 0.25, 0.25]).log().expand(2, 3), torch.tensor([0.25, 0.5, 0.25]).log().expand(2, 3)
    go = lambda draft, u: V.verify(z, torch.tensor([0, draft]), torch.tensor(u), 1.0, y)[:2]  # noqa: E731
    assert go(0, [0.99, 0.6]) == (1, [0, 1]) and go(1, [0.4, 0.8]) == (1, [1, 2]) and go(1, [0.6, 0.99]) == (0, [0])
    assert V.verify(z, torch.tensor([0, 1]), torch.tensor([0.3, 0.7]), 1.0)[:2] == (0, [2])        # chosen, not drawn: stands for u < 1/4; else 0 or 2, two to one


def test_reference_verification_of_what_64_bits_do_not_hold():
    """p(x) = e^-1200 and q(x) = e^-700, or the other way round; a mask in both; u = 0."""
    z, y = torch.tensor([[0.0, -12.0]]).expand(2, 2), torch.tensor([[0.0, -7.0]]).expand(2, 2)
    go = lambda a, b, u, tau=0.01: V.verify(a, torch.tensor([0, 1]), torch.tensor(u), tau, b, tau)[:3]  # noqa: E731
    assert go(z, y, [0.525, 0.5])[0] == 0 and go(y, z, [0.999, 0.5])[0] == 1
    assert abs(go(y, z, [0.5, 0.5])[2][0] + 700.0) < 1e-3
    mask = torch.tensor([[0.0, -1e9]]).expand(2, 2)
    assert go(mask, mask, [0.5, 0.0]) [0] == 1 and go(mask, z, [0.0, 0.0])[0] == 0 and V.verify(mask, torch.tensor([0, 1]), torch.tensor([0.0, 0.0]), 1.0)[:2] == (0, [0])
    flipped = mask.flip(1)
    assert V.verify(flipped[:1], torch.tensor([0]), torch.tensor([0.0]), 1.0)[1] == [1]             # the masked token comes first, and is not drawn


# ------------------------------------------------------------------ how a call is cut
@pytest.mark.parametrize("n_seq,n_tokens,vocab,each", [
    (1, 5, 32000, 8), (16, 128, 131072, 32), (16, 127, 131072, 8), (32, 192, 131072, 32), (4, 16, 131072, 8), (64, 600, 32000, 32), (64, 400, 32000, 8), (1000, 6000, 2048, 8), (1000, 6000, 2049, 32),
    (1 << 16, 15, 1 << 20, 32), (3, 0, 5000, 8)])
def test_logits_per_thread(pkg, n_seq, n_tokens, vocab, each):  # noqa: F811
    """The scratch tells: slices of 256 threads of 8 or 32 logits, sums and largest logits of two rows per token and slice, four numbers per piece at most.  Many sequences without tokens count as well: their blocks of
    small slices would pass a grid's end."""
    up = lambda x: (x + 255) // 256 * 256  # noqa: E731
    slices = -(-vocab // (256 * each))
    pieces = slices * each // 4
    need = 2 * up(2 * n_tokens * slices * 4) + up(2 * n_seq * pieces * 8) + up(n_seq * pieces * 8) + up(n_seq * 20)
    assert pkg.lib().spd_op_verify_drafts_scratch_bytes(n_seq, n_tokens, vocab) == need
    assert max(2 * n_tokens, n_seq) * slices * 256 < 1 << 32
