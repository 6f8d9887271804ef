"""Temperatures of a verification of drafts, seen without a GPU (every status is returned before anything is enqueued)."""
import pytest

from test_chunk_ops_host import EINVAL, VERIFY, call, pkg  # noqa: F401


@pytest.mark.parametrize("name", ["tau", "draft_tau"])
@pytest.mark.parametrize("value", [2.0 ** -100 * (1 - 2.0 ** -40), 2.0 ** 100 * (1 + 2.0 ** -40)])
def test_temperatures_cross_the_interface_in_64_bits(pkg, name, value):  # noqa: F811
    """Numbers that 32 bits round to the bounds, which are allowed."""
    assert call(pkg, "spd_op_verify_drafts", VERIFY, **{name: value}) == EINVAL
    assert call(pkg, "spd_op_verify_drafts", VERIFY, n_seq=0, **{name: 2.0 ** -100 if value < 1 else 2.0 ** 100}) == 0
