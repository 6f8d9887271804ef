"""What the operators of several sequences over one paged cache refuse, seen without a GPU: every status below is returned before
anything is enqueued (the pointers are addresses that nothing may follow)."""
import ctypes as C
import math

import pytest
import torch

import batch_reference as R

EINVAL, EWORKSPACE = -1, -4
A = 1 << 20          # an aligned address


@pytest.fixture(scope="module")
def pkg():
    import os

    import paper_2405_18400_amd as P
    if not os.path.exists(P.library_path()):
        from paper_2405_18400_amd.build import build_library
        build_library()
    return P


CACHE = dict(dtype=2, K=A, V=2 * A, table=3 * A, n_pages=40, n_kv_heads=2, page_size=16, d_head=64, n_seq=6, table_stride=9)
APPEND = dict(CACHE, q=4 * A, q_stride=256, k=5 * A, v=6 * A, kv_stride=128, seq=7 * A, pos=8 * A, n_tokens=6, n_heads=4, rope_theta=1e4, q_out=9 * A, err=None, stream=None)
ATTEND = dict(dtype=2, q=4 * A, K=A, V=2 * A, table=3 * A, n_pages=40, n_kv_heads=2, page_size=16, d_head=64, n_seq=6, table_stride=60, shared=5 * A, len=6 * A, width=3, n_heads=4,
              max_shared=700, max_own=20, out=7 * A, scratch=8 * A, scratch_bytes=1 << 30, err=None, stream=None)
SELECT = dict(dtype=0, logits=A, row_stride=5000, n_groups=2, n_in=3, n_out=4, vocab=5000, scores=2 * A, ended=3 * A, end_token=2, tau=1.0, out_scores=4 * A, out_tokens=5 * A,
              out_parents=6 * A, out_ended=7 * A, scratch=8 * A, scratch_bytes=1 << 30, stream=None)
REORDER = dict(CACHE, n_layers=2, layer_stride=40 * 2 * 16 * 64, width=3, parents=4 * A, len=5 * A, table_out=6 * A, err=None, stream=None)

BAD_CACHE = [("dtype", 3), ("dtype", -1), ("K", None), ("V", None), ("table", None), ("K", A + 8), ("V", A + 4), ("table", A + 2), ("n_pages", 0), ("n_kv_heads", 0),
             ("page_size", 0), ("page_size", 2), ("page_size", 24), ("page_size", 2048), ("page_size", -16), ("d_head", 4), ("d_head", 96), ("d_head", 512), ("d_head", 0), ("n_seq", -1),
             ("table_stride", 0)]


def call(pkg, name, base, **changed):
    assert set(changed) <= set(base)
    return getattr(pkg.lib(), name)(*{**base, **changed}.values())


@pytest.mark.parametrize("what,value", BAD_CACHE + [("n_tokens", -1), ("k", None), ("v", None), ("seq", None), ("pos", None), ("kv_stride", 127), ("kv_stride", 130), ("k", A + 4),
                                                    ("v", A + 8), ("q", None), ("q_out", None), ("n_heads", 0), ("q_stride", 252), ("q_stride", 258), ("q", A + 4),
                                                    ("q_out", A + 4), ("rope_theta", 0.0), ("rope_theta", -1.0), ("rope_theta", math.inf), ("rope_theta", math.nan),
                                                    ("n_heads", -1), ("n_heads", 1 << 20)])
def test_append_refuses(pkg, what, value):
    assert call(pkg, "spd_op_append_paged", APPEND, **{what: value}) == EINVAL


@pytest.mark.parametrize("out", [4 * A + 16, 4 * A - 16, 4 * A + 5 * 256 * 4, 5 * A, 5 * A + 5 * 128 * 4, 5 * A - 16, 6 * A - 6 * 256 * 4 + 16, 6 * A + 128 * 4])
def test_append_refuses_results_over_what_other_blocks_read(pkg, out):
    assert call(pkg, "spd_op_append_paged", APPEND, q_out=out) == EINVAL


@pytest.mark.parametrize("out", [4 * A, 4 * A + 16, 4 * A - 16, 4 * A + 6 * 4 * 64 * 4 - 16, 4 * A - 6 * 4 * 64 * 4 + 16])
def test_attention_refuses_results_over_its_queries(pkg, out):
    assert call(pkg, "spd_op_attention_shared", ATTEND, out=out) == EINVAL


@pytest.mark.parametrize("n_in,n_out,name,at", [(3, 4, "out_scores", 2 * A), (3, 4, "out_ended", 3 * A), (3, 3, "out_scores", 2 * A + 4), (3, 3, "out_ended", 3 * A - 4),
                                                (4, 3, "out_tokens", 2 * A + 2 * 4 * 4 - 4), (4, 3, "out_parents", 3 * A - 2 * 3 * 4 + 4)])
def test_select_refuses_results_over_another_groups_inputs(pkg, n_in, n_out, name, at):
    assert call(pkg, "spd_op_beam_select", SELECT, n_in=n_in, n_out=n_out, **{name: at}) == EINVAL


def test_append_in_place_wants_whole_rows(pkg):
    assert call(pkg, "spd_op_append_paged", APPEND, q_out=APPEND["q"], q_stride=512) == EINVAL
    assert call(pkg, "spd_op_append_paged", APPEND, n_tokens=0) == 0                       # nothing to do, nothing enqueued
    assert call(pkg, "spd_op_append_paged", APPEND, n_tokens=0, k=None, v=None, q=None, q_out=None, n_heads=0) == 0


@pytest.mark.parametrize("what,value", BAD_CACHE + [("width", 0), ("width", 4), ("n_heads", 0), ("n_heads", 3), ("max_shared", -1), ("max_own", -1), ("max_shared", 961), ("max_own", 961),
                                                    ("max_own", (1 << 31) - 1), ("q", None), ("q", A + 4), ("out", None), ("out", A + 8), ("shared", None), ("len", None),
                                                    ("scratch", None), ("scratch", A + 64)])
def test_attention_refuses(pkg, what, value):
    assert call(pkg, "spd_op_attention_shared", ATTEND, **{what: value}) == EINVAL


def test_attention_scratch(pkg):
    f = pkg.lib().spd_op_attention_shared_scratch_bytes
    need = f(6, 3, 4, 2, 64, 700, 20)
    assert need > 0 and need % 256 == 0
    assert call(pkg, "spd_op_attention_shared", ATTEND, scratch_bytes=need - 1) == EWORKSPACE
    assert f(6, 3, 4, 2, 64, 4000, 20) >= need
    assert f(6, 3, 4, 2, 64, 100, 20) == 0                    # one block per sequence and head: nothing to join
    for i, bad in enumerate([0, 0, 0, 0, 0, -1, -1]):
        args = [6, 3, 4, 2, 64, 700, 20]
        args[i] = bad
        assert f(*args) == 0
    assert call(pkg, "spd_op_attention_shared", ATTEND, n_seq=0) == 0


@pytest.mark.parametrize("what,value", [("dtype", 3), ("logits", None), ("logits", A + 2), ("row_stride", 4999), ("n_groups", -1), ("n_in", 0), ("n_in", 17), ("n_out", 0), ("n_out", 17),
                                        ("vocab", 0), ("vocab", -5), ("scores", None), ("end_token", -1), ("end_token", 5000), ("tau", 0.0), ("tau", -1.0), ("tau", math.nan),
                                        ("tau", math.inf), ("tau", 1e-40), ("out_scores", None), ("out_tokens", None), ("out_parents", None), ("scratch", None), ("scratch", A + 8)])
def test_select_refuses(pkg, what, value):
    assert call(pkg, "spd_op_beam_select", SELECT, **{what: value}) == EINVAL


def test_select_scratch(pkg):
    need = pkg.lib().spd_op_beam_select_scratch_bytes(2, 3, 4, 5000)
    assert need > 0 and need % 256 == 0
    assert call(pkg, "spd_op_beam_select", SELECT, scratch_bytes=need - 1) == EWORKSPACE
    assert pkg.lib().spd_op_beam_select_scratch_bytes(2, 3, 4, 0) == 0
    assert pkg.lib().spd_op_beam_select_scratch_bytes(2, 3, 4, 4096) == 0    # one launch
    assert call(pkg, "spd_op_beam_select", SELECT, n_groups=0) == 0


@pytest.mark.parametrize("what,value", BAD_CACHE + [("width", 0), ("width", 17), ("width", 4), ("n_layers", 0), ("layer_stride", 40 * 2 * 16 * 64 - 8), ("layer_stride", 40 * 2 * 16 * 64 + 4),
                                                    ("parents", None), ("len", None), ("table_out", None), ("table_out", 3 * A), ("table_out", 3 * A + 6 * 9 * 4 - 4),
                                                    ("table_out", 3 * A - 6 * 9 * 4 + 4)])
def test_reorder_refuses(pkg, what, value):
    assert call(pkg, "spd_op_beam_reorder", REORDER, **{what: value}) == EINVAL


def test_reorder_of_nothing(pkg):
    assert call(pkg, "spd_op_beam_reorder", REORDER, n_seq=0, table_out=None, parents=None, len=None) == 0


def test_python_refuses_tensors_that_are_not_what_they_should_be(pkg, monkeypatch):
    """Shapes, types and devices, before the library is asked (a stand-in says which device is the current one)."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)          # (that of a CPU tensor)
    K, i = torch.zeros(4, 2, 8, 16), lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    k = torch.zeros(3, 2, 16)
    ok = lambda **c: {**dict(K=K, V=K, table=i(2, 2), k=k, v=k, seq=i(3), pos=i(3)), **c}  # noqa: E731
    for bad in (dict(K=K.half()), dict(V=K[:2]), dict(table=torch.zeros(2, 2)), dict(seq=i(2)), dict(pos=i(3).long()), dict(k=k[:2]), dict(v=k.half()),
                dict(k=torch.zeros(3, 16, 2).transpose(1, 2)), dict(K=K.transpose(1, 2)), dict(v=torch.zeros(3, 3, 16)[:, :2]), dict(q=torch.zeros(3, 4, 16)),
                dict(q=torch.zeros(3, 4, 8), q_out=torch.zeros(3, 4, 8)), dict(q=torch.zeros(3, 4, 16), q_out=torch.zeros(3, 4, 16).half()), dict(err=i(2))):
        a = ok(**bad)
        with pytest.raises(ValueError):
            pkg.spd_op_append_paged("fp32", a.pop("K"), a.pop("V"), a.pop("table"), a.pop("k"), a.pop("v"), a.pop("seq"), a.pop("pos"), 1e4, **a)
    q = torch.zeros(4, 2, 16)
    for bad in (dict(q=q[:3]), dict(table=i(3, 2)), dict(shared=i(4)), dict(length=i(2)), dict(out=q.half()), dict(width=0), dict(width=3), dict(dtype="fp8")):
        a = {**dict(dtype="fp32", q=q, K=K, V=K, table=i(4, 2), shared=i(2), length=i(4), out=q, width=2, max_shared=3, max_own=3), **bad}
        with pytest.raises(ValueError):
            pkg.spd_op_attention_shared(**a)
    z, s = torch.zeros(2, 3, 50), torch.zeros(2, 3)
    for bad in (dict(logits=z.half()), dict(logits=torch.zeros(2, 50, 3).transpose(1, 2)), dict(logits=torch.zeros(3, 2, 50).transpose(0, 1)), dict(scores=s[:1]), dict(out_tokens=s),
                dict(out_parents=i(2, 3)), dict(ended=i(2, 4), end_token=1), dict(out_ended=i(2, 3))):
        a = {**dict(dtype="fp32", logits=z, scores=s, out_scores=torch.zeros(2, 4), out_tokens=i(2, 4), out_parents=i(2, 4)), **bad}
        with pytest.raises(ValueError):
            pkg.spd_op_beam_select(**a)
    for bad in (dict(parents=i(1, 2)), dict(length=i(2)), dict(table_out=i(4, 3)), dict(width=3), dict(V=K[:2]), dict(K=K.half())):
        a = {**dict(dtype="fp32", K=K, V=K, table=i(4, 2), parents=i(2, 2), length=i(4), table_out=i(4, 2), width=2), **bad}
        with pytest.raises(ValueError):
            pkg.spd_op_beam_reorder(**a)
    other = K.reshape(4, 8, 2, 16)                                         # as many elements in another order
    with pytest.raises(ValueError):
        pkg.spd_op_append_paged("fp32", K, other, i(2, 2), k, k, i(3), i(3), 1e4)
    with pytest.raises(ValueError):
        pkg.spd_op_attention_shared("fp32", q, K, other, i(4, 2), i(2), i(4), torch.empty_like(q), 2, 3, 3)
    with pytest.raises(ValueError):
        pkg.spd_op_beam_reorder("fp32", K, other, i(4, 2), i(2, 2), i(4), i(4, 2), 2)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)           # tensors of another device
    with pytest.raises(ValueError):
        pkg.spd_op_append_paged("fp32", K, K, i(2, 2), k, k, i(3), i(3), 1e4)


# ---- the references themselves, where they can be seen to be right
def test_reference_rotation_keeps_lengths_and_adds_angles():
    x = torch.randn(2, 16, dtype=torch.float64)
    y = R.rotate(x, 5, 1e4)
    torch.testing.assert_close(R.rotate(y, 7, 1e4), R.rotate(x, 12, 1e4))
    torch.testing.assert_close(y.norm(dim=1), x.norm(dim=1))
    assert torch.equal(R.rotate(x, 0, 1e4), x)


def test_reference_selection_is_that_of_all_continuations():
    g = torch.Generator().manual_seed(3)
    z, s = torch.randn(3, 11, generator=g), torch.tensor([-1.0, -0.5, -2.0])
    every = sorted(((float(s[b]) + float(torch.log_softmax(z[b].double() / 0.7, 0)[v]), -b, -v) for b in range(3) for v in range(11)), reverse=True)[:5]
    got = R.select(z, s, 5, 0.7)
    assert [(b, v) for _, v, b, _ in got] == [(-b, -v) for _, b, v in every]
    assert [c[0] for c in got] == pytest.approx([c[0] for c in every], abs=1e-12)


def test_reference_attention_of_shared_positions_is_that_of_whole_sequences():
    g = torch.Generator().manual_seed(4)
    K, V = (torch.randn(12, 2, 4, 8, generator=g) for _ in range(2))
    table = torch.tensor([[0, 1, 2], [0, 1, 3]])
    q = torch.randn(2, 4, 8, generator=g)
    assert torch.equal(R.attention(q, K, V, table, [8], [11, 9], 2), R.attention(q, K, V, table, [0], [11, 9], 2))
