"""The operators of several sequences over one paged cache at the limits of what their arguments may hold."""

import pytest
import torch

import batch_reference as R
from test_gpu_batch_ops import attend, attention_case, close, gen

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
