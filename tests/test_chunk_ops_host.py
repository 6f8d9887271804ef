"""What the operators of chunks of new tokens over a paged cache refuse, seen without a GPU: every status below is returned before
anything is enqueued (the pointers are addresses that nothing may follow)."""
import math

import pytest
import torch

import chunk_reference as R
from test_batch_ops_host import APPEND, REORDER
from test_batch_ops_host import ATTEND as SHARED

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


POOLS = dict(K=A, V=2 * A, K_scale=3 * A, V_scale=4 * A, table=5 * A)
SIZES = dict(n_pages=40, n_kv_heads=2, page_size=16, d_head=64, n_seq=6, table_stride=60)
WRITE = dict(POOLS, **SIZES, q=6 * A, q_stride=256, k=7 * A, v=8 * A, kv_stride=128, seq=9 * A, pos=10 * A, n_tokens=6, n_heads=4, rope_theta=1e4, q_out=11 * A, err=None, stream=None)
READ = dict(dtype=3, **POOLS, **SIZES, seq=6 * A, pos=7 * A, n_tokens=6, out_dtype=0, k_out=8 * A, v_out=9 * A, err=None, stream=None)
ATTEND = dict(dtype=3, io_dtype=0, q=6 * A, q_stride=256, **POOLS, **SIZES, first=7 * A, len=8 * A, n_tokens=30, n_heads=4, max_new=9, max_len=960, out=9 * A, scratch=16 * A, scratch_bytes=1 << 40,
              err=None, stream=None)
VERIFY = dict(dtype=0, logits=A, row_stride=5000, draft_logits=2 * A, draft_stride=5000, tokens=3 * A, first=4 * A, u=5 * A, n_seq=3, n_tokens=7, vocab=5000, tau=1.0, draft_tau=1.0, out_tokens=6 * A,
              out_logprobs=7 * A, out_accepted=8 * A, scratch=9 * A, scratch_bytes=1 << 30, err=None, stream=None)

BAD_POOLS = [("K", None), ("V", None), ("table", None), ("K_scale", None), ("V_scale", None), ("K", A + 8), ("V", 2 * A + 4), ("K_scale", 3 * A + 4), ("V_scale", 4 * A + 8), ("table", 5 * A + 2), ("n_pages", 0),
             ("n_kv_heads", 0), ("page_size", 0), ("page_size", 2), ("page_size", 24), ("page_size", 2048), ("page_size", -16), ("d_head", 4), ("d_head", 96), ("d_head", 512), ("d_head", 0),
             ("n_seq", -1), ("table_stride", 0)]


def call(pkg, name, base, **changed):
    assert set(changed) <= set(base)
    return getattr(pkg.lib(), name)(*{**base, **changed}.values())


@pytest.mark.parametrize("what,value", BAD_POOLS + [("n_tokens", -1), ("k", None), ("v", None), ("seq", None), ("pos", None), ("kv_stride", 127), ("kv_stride", 130), ("k", 7 * A + 4), ("v", 8 * A + 8),
                                                    ("q", None), ("q_out", None), ("n_heads", 0), ("q_stride", 252), ("q_stride", 258), ("q", 6 * A + 4), ("q_out", 11 * A + 4), ("rope_theta", 0.0),
                                                    ("rope_theta", -1.0), ("rope_theta", math.inf), ("rope_theta", math.nan), ("n_heads", -1), ("n_heads", 1 << 20)])
def test_write_refuses(pkg, what, value):
    assert call(pkg, "spd_op_append_paged_q8", WRITE, **{what: value}) == EINVAL


@pytest.mark.parametrize("changed", [dict(q_out=6 * A + 16), dict(q_out=7 * A), dict(q_out=3 * A), dict(q_out=4 * A - 16), dict(K_scale=A + 4096), dict(V_scale=3 * A + 16), dict(V=A + 4096), dict(K_scale=7 * A),
                                     dict(V_scale=5 * A), dict(K=8 * A), dict(err=3 * A + 4), dict(q_out=6 * A, q_stride=512)])
def test_write_refuses_results_over_what_other_blocks_read_or_write(pkg, changed):
    assert call(pkg, "spd_op_append_paged_q8", WRITE, **changed) == EINVAL


def test_write_of_nothing(pkg):
    assert call(pkg, "spd_op_append_paged_q8", WRITE, n_tokens=0) == 0
    assert call(pkg, "spd_op_append_paged_q8", WRITE, n_tokens=0, k=None, v=None, q=None, q_out=None, n_heads=0) == 0


@pytest.mark.parametrize("what,value", BAD_POOLS + [("dtype", 4), ("dtype", -1), ("dtype", 2), ("out_dtype", 3), ("out_dtype", -1), ("n_tokens", -1), ("seq", None), ("pos", None), ("k_out", None), ("v_out", None),
                                                    ("k_out", 8 * A + 4), ("v_out", 9 * A + 8), ("n_kv_heads", 1 << 20), ("k_out", 9 * A), ("k_out", 9 * A + 16), ("v_out", 2 * A), ("k_out", 3 * A),
                                                    ("v_out", 6 * A), ("k_out", 5 * A), ("err", 8 * A + 16)])
def test_read_refuses(pkg, what, value):
    assert call(pkg, "spd_op_read_paged", READ, **{what: value}) == EINVAL


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_scales_come_with_8_bits_alone(pkg, dtype):
    assert call(pkg, "spd_op_read_paged", READ, dtype=dtype) == EINVAL
    assert call(pkg, "spd_op_read_paged", READ, dtype=dtype, K_scale=None) == EINVAL
    assert call(pkg, "spd_op_read_paged", READ, dtype=dtype, K_scale=None, V_scale=None, n_tokens=0) == 0
    assert call(pkg, "spd_op_attention_paged", ATTEND, dtype=dtype) == EINVAL
    assert call(pkg, "spd_op_attention_paged", ATTEND, dtype=dtype, K_scale=None, V_scale=None, n_tokens=0) == 0


@pytest.mark.parametrize("what,value", BAD_POOLS + [("dtype", 4), ("dtype", -1), ("io_dtype", 3), ("io_dtype", -1), ("n_heads", 0), ("n_heads", 3), ("n_heads", -2), ("max_new", -1), ("max_len", -1), ("max_len", 961),
                                                    ("max_len", (1 << 31) - 1), ("n_tokens", -1), ("q", None), ("q", 6 * A + 8), ("out", None), ("out", 9 * A + 4), ("first", None), ("len", None), ("q_stride", 252),
                                                    ("q_stride", 260), ("q_stride", 255), ("scratch", 16 * A + 64), ("n_tokens", 1 << 24), ("out", 6 * A), ("out", 6 * A + 16), ("out", 6 * A + 29 * 1024),
                                                    ("out", A), ("out", 3 * A), ("out", 5 * A), ("out", 7 * A), ("out", 8 * A), ("err", 9 * A + 4),
                                                    ("n_seq", (1 << 16) + 1), ("n_pages", 1 << 30)])
def test_attention_refuses(pkg, what, value):
    if what == "scratch" and not pkg.lib().spd_op_attention_paged_scratch_bytes(3, 0, 6, 30, 4, 2, 64, 9, 960):
        pytest.skip("this call takes no scratch")
    assert call(pkg, "spd_op_attention_paged", ATTEND, **{what: value}) == EINVAL


@pytest.mark.parametrize("dtype,io,fits", [(0, 0, True), (0, 1, False), (0, 2, False), (1, 0, True), (1, 1, True), (1, 2, False), (2, 0, True), (2, 1, False), (2, 2, True), (3, 0, True), (3, 1, True), (3, 2, True)])
def test_attention_types(pkg, dtype, io, fits):
    scales = {} if dtype == 3 else dict(K_scale=None, V_scale=None)
    assert call(pkg, "spd_op_attention_paged", ATTEND, dtype=dtype, io_dtype=io, n_tokens=0, **scales) == (0 if fits else EINVAL)


def test_attention_scratch(pkg):
    size = lambda *a: pkg.lib().spd_op_attention_paged_scratch_bytes(*a)  # noqa: E731
    for bad in ((9, 0, 1, 4, 4, 2, 64, 4, 4000), (2, 0, 0, 4, 4, 2, 64, 4, 4000), (2, 0, 1, 0, 4, 2, 64, 4, 4000), (2, 0, 1, 4, 3, 2, 64, 4, 4000), (2, 0, 1, 4, 4, 0, 64, 4, 4000), (2, 0, 1, 4, 4, 2, 0, 4, 4000),
                (2, 0, 1, 4, 4, 2, 64, -1, 4000), (2, 0, 1, 4, 4, 2, 64, 4, -1), (2, 1, 1, 4, 4, 2, 64, 4, 4000)):
        assert size(*bad) == 0
    need = size(3, 0, 6, 30, 4, 2, 64, 9, 960)
    assert need % 256 == 0
    if need:
        assert call(pkg, "spd_op_attention_paged", ATTEND, scratch_bytes=need - 1) == EWORKSPACE
        assert call(pkg, "spd_op_attention_paged", ATTEND, scratch=None) == EINVAL
        assert call(pkg, "spd_op_attention_paged", ATTEND, scratch=9 * A) == EINVAL


@pytest.mark.parametrize("what,value", [("dtype", 3), ("dtype", -1), ("logits", None), ("logits", A + 2), ("draft_logits", 2 * A + 2), ("row_stride", 4999), ("draft_stride", 4999), ("tokens", None), ("first", None),
                                        ("u", None), ("n_seq", -1), ("n_tokens", -1), ("vocab", 0), ("vocab", -1), ("vocab", (1 << 24) + 1), ("tau", 0.0), ("tau", -1.0), ("tau", math.inf), ("tau", math.nan),
                                        ("draft_tau", 0.0), ("draft_tau", math.nan), ("out_tokens", None), ("out_logprobs", None), ("out_accepted", None), ("out_tokens", 3 * A), ("out_tokens", A + 4), ("out_logprobs", 5 * A),
                                        ("out_logprobs", 6 * A + 4), ("out_accepted", 4 * A), ("out_accepted", 7 * A + 24), ("err", 8 * A + 8), ("out_tokens", 2 * A + 6 * 20000 + 19996), ("n_seq", (1 << 16) + 1), ("n_tokens", (1 << 20) + 1), ("tau", 2.0 ** -101), ("tau", 2.0 ** 101),
                                        ("draft_tau", 2.0 ** -101), ("draft_tau", 2.0 ** 101)])
def test_verify_refuses(pkg, what, value):
    assert call(pkg, "spd_op_verify_drafts", VERIFY, **{what: value}) == EINVAL


def test_verify_of_nothing_and_scratch(pkg):
    assert call(pkg, "spd_op_verify_drafts", VERIFY, n_seq=0) == 0
    size = lambda *a: pkg.lib().spd_op_verify_drafts_scratch_bytes(*a)  # noqa: E731
    assert size(0, 5, 100) == size(2, -1, 100) == size(2, 5, 0) == size(-1, 5, 100) == 0
    need = size(3, 7, 5000)
    assert need % 256 == 0
    if need:
        assert call(pkg, "spd_op_verify_drafts", VERIFY, scratch_bytes=need - 1) == EWORKSPACE
        assert call(pkg, "spd_op_verify_drafts", VERIFY, scratch=None) == EINVAL
        assert call(pkg, "spd_op_verify_drafts", VERIFY, scratch=9 * A + 64) == EINVAL
        assert call(pkg, "spd_op_verify_drafts", VERIFY, scratch=A) == EINVAL


def test_grids_past_32_bits_are_refused(pkg):
    """Calls whose threads pass 32 bits; nothing is launched."""
    assert call(pkg, "spd_op_verify_drafts", VERIFY, logits=1 << 50, draft_logits=1 << 51, tokens=1 << 52, first=1 << 53, u=1 << 54, out_tokens=1 << 55, out_logprobs=1 << 56, out_accepted=1 << 57, scratch=1 << 58,
                n_tokens=1 << 20, vocab=1 << 18, row_stride=1 << 18, draft_stride=1 << 18, scratch_bytes=1 << 50) == EINVAL
    wide = dict(zip(("K", "V", "K_scale", "V_scale", "table", "q", "first", "len", "out"), (1 << n for n in range(48, 57))), scratch=1 << 58)
    assert call(pkg, "spd_op_attention_paged", ATTEND, **wide, n_pages=1, n_kv_heads=1 << 10, n_heads=1 << 10, n_seq=1 << 16, n_tokens=1 << 14, q_stride=1 << 16) == EINVAL
    wide = dict(zip(("K", "V", "K_scale", "V_scale", "table", "q", "k", "v", "seq", "pos", "q_out"), (1 << n for n in range(48, 59))))
    assert call(pkg, "spd_op_append_paged_q8", WRITE, **wide, n_heads=1 << 14, q_stride=1 << 20, n_tokens=1 << 20) == EINVAL


@pytest.mark.parametrize("name", ["spd_op_append_paged", "spd_op_attention_shared", "spd_op_beam_reorder"])
def test_operators_without_scales_take_no_8_bit_cache(pkg, name):
    base = {"spd_op_append_paged": APPEND, "spd_op_attention_shared": SHARED, "spd_op_beam_reorder": REORDER}[name]
    assert call(pkg, name, base, dtype=3) == EINVAL


def test_python_refuses_tensors_that_are_not_what_they_should_be(pkg, monkeypatch):
    """Shapes, types, strides and devices, before the library is asked; a good call gets there (stand-ins say which device is the current one, and that the library was asked)."""
    from paper_2405_18400_amd import binding

    class Enqueued(Exception):
        pass

    class Library:
        spd_op_attention_paged_scratch_bytes = spd_op_verify_drafts_scratch_bytes = staticmethod(lambda *a: 0)

        def __getattr__(self, name):
            def enqueue(*args):
                raise Enqueued(name)
            return enqueue

    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)          # (that of a CPU tensor)
    monkeypatch.setattr(binding, "_stream_ptr", lambda device=None: None)
    monkeypatch.setattr(binding, "lib", Library)
    i, f = lambda *s: torch.zeros(*s, dtype=torch.int32), torch.zeros  # noqa: E731
    codes, scale, half, rows = f(4, 2, 8, 16, dtype=torch.int8), f(4, 2, 8), f(4, 2, 8, 16, dtype=torch.float16), f(3, 2, 16)
    write = dict(K=codes, V=codes, K_scale=scale, V_scale=scale, table=i(2, 2), k=rows, v=rows, seq=i(3), pos=i(3), rope_theta=1e4)
    read = dict(dtype="int8", K=codes, V=codes, table=i(2, 2), seq=i(3), pos=i(3), k_out=rows, v_out=rows, K_scale=scale, V_scale=scale)
    attend = dict(dtype="int8", q=f(5, 4, 16), K=codes, V=codes, table=i(2, 2), first=i(3), length=i(2), out=f(5, 4, 16), max_new=3, max_len=9, K_scale=scale, V_scale=scale)
    verify = dict(dtype="fp16", logits=f(5, 50).half(), tokens=i(5), first=i(3), u=f(5), out_tokens=i(5), out_logprobs=f(5), out_accepted=i(2), draft_logits=f(5, 50).half())
    pools = [dict(K=codes[:2]), dict(V=codes.transpose(1, 2)), dict(K=half), dict(table=f(2, 2)), dict(table=i(2, 4)[:, ::2]), dict(K_scale=None), dict(V_scale=None), dict(K_scale=scale[:3]),
             dict(V_scale=scale.double()), dict(K_scale=f(4, 8, 2).transpose(1, 2)), dict(err=i(2)), dict(err=f(1))]
    for name, good, others, bad in [
            ("spd_op_append_paged_q8", write, [dict(q=f(3, 4, 16), q_out=f(3, 4, 16)), dict(k=f(3, 6, 16)[:, :2], v=f(3, 6, 16)[:, 2:4])],
             [dict(k=rows[:2]), dict(v=rows.half()), dict(q=f(3, 4, 16)), dict(q_out=f(3, 4, 16)), dict(k=f(3, 4, 16)[:, ::2], v=f(3, 4, 16)[:, ::2]), dict(seq=i(2)), dict(pos=i(3).long()),
              dict(k=f(3, 6, 16)[:, :2]), dict(q=f(3, 4, 8), q_out=f(3, 4, 8)), dict(q=f(3, 4, 16), q_out=f(3, 4, 16).half())]),
            ("spd_op_read_paged", read, [dict(k_out=rows.half(), v_out=rows.half()), dict(dtype="fp16", K=half, V=half, K_scale=None, V_scale=None)],
             [dict(dtype="fp16"), dict(dtype="fp16", K=half, V=half), dict(dtype="fp8"), dict(k_out=rows.half()), dict(k_out=rows.double(), v_out=rows.double()), dict(k_out=rows[:2]), dict(seq=i(4)),
              dict(v_out=f(3, 16, 2).transpose(1, 2))]),
            ("spd_op_attention_paged", attend, [dict(q=f(5, 4, 16).half(), out=f(5, 4, 16).half()), dict(q=f(5, 9, 16)[:, :4]), dict(dtype="fp16", K=half, V=half, K_scale=None, V_scale=None)],
             [dict(q=f(5, 4, 16).half()), dict(out=f(4, 4, 16)), dict(q=f(5, 4, 8)), dict(q=f(5, 16, 4).transpose(1, 2)), dict(q=f(5, 8, 16)[:, ::2]), dict(q=f(5, 4, 16).double(), out=f(5, 4, 16).double()),
              dict(first=i(2)), dict(length=i(3)), dict(first=i(3).long()), dict(max_new=1 << 31), dict(max_len=1 << 32), dict(dtype="fp8"), dict(dtype="fp16")]),
            ("spd_op_verify_drafts", verify, [dict(draft_logits=None), dict(logits=f(5, 60).half()[:, :50])],
             [dict(logits=f(5, 50)), dict(draft_logits=f(5, 49).half()), dict(logits=f(50, 5).half().t()), dict(tokens=i(4)), dict(first=i(0)), dict(first=i(4)), dict(u=f(5).double()), dict(out_tokens=f(5)),
              dict(out_logprobs=f(6)), dict(out_accepted=i(3)), dict(dtype="int8"), dict(err=i(2))])]:
        for more in [{}, dict(err=i(1))] + others:
            with pytest.raises(Enqueued, match=name):
                getattr(pkg, name)(**{**good, **more})
        for wrong in bad + (pools if "K" in good else []):
            with pytest.raises(ValueError):
                getattr(pkg, name)(**{**good, **wrong})
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)           # tensors of another device
    for name, good in (("spd_op_append_paged_q8", write), ("spd_op_read_paged", read), ("spd_op_attention_paged", attend), ("spd_op_verify_drafts", verify)):
        with pytest.raises(ValueError):
            getattr(pkg, name)(**good)


# ------------------------------------------------------------------ the references that the GPU tests go by
def test_reference_quantisation():
    x = torch.tensor([[1.0, -2.0, 0.5, 127.0], [0.0, 0.0, 0.0, 0.0], [381.0, 1.5, 4.5, -7.5]], dtype=torch.float64)
    code, scale = R.quantise(x)
    assert code.tolist() == [[1, -2, 0, 127], [0, 0, 0, 0], [127, 0, 2, -2]] and scale.tolist() == [1.0, 0.0, 3.0]


def test_reference_attention_over_pages():
    """One token over three positions on two pages, then two tokens: the first does not see the last position."""
    K = torch.zeros(2, 1, 2, 2)
    V = torch.tensor([[[[1.0, 2.0], [3.0, 4.0]]], [[[5.0, 6.0], [math.nan, math.nan]]]])
    table = torch.tensor([[0, 1]], dtype=torch.int32)
    out, _ = R.attention(torch.zeros(1, 1, 2), K, V, table, torch.tensor([0, 1]), torch.tensor([3]))
    assert torch.allclose(out, torch.tensor([[[3.0, 4.0]]], dtype=torch.float64))
    out, _ = R.attention(torch.zeros(2, 1, 2), K, V, table, torch.tensor([0, 2]), torch.tensor([3]))
    assert torch.allclose(out[0], torch.tensor([[2.0, 3.0]], dtype=torch.float64))


def test_reference_verification():
    """p = (1/2, 1/4, 1/4), q = (1/4, 1/2, 1/4): token 0 always stands, token 1 for u < 1/2, what is left of its row is all at token 0."""
    z, y = torch.tensor([0.5, 0.25, 0.25]).log().expand(2, 3), torch.tensor([0.25, 0.5, 0.25]).log().expand(2, 3)
    go = lambda draft, u: R.verify(z, torch.tensor([0, draft]), torch.tensor(u), 1.0, y)[:2]  # noqa: E731
    assert go(0, [0.99, 0.6]) == (1, [0, 1]) and go(1, [0.4, 0.8]) == (1, [1, 2]) and go(1, [0.6, 0.99]) == (0, [0])
    given = R.verify(z, torch.tensor([0, 1]), torch.tensor([0.3, 0.7]), 1.0)       # chosen, not drawn: stands for u < 1/4; else 0 or 2, two to one
    assert given[:2] == (0, [2])
