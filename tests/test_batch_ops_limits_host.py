"""What the operators of several sequences over one paged cache refuse and how they cut their work, seen without a GPU (no status below follows a pointer)."""
import pytest

from test_batch_ops_host import A, APPEND, ATTEND, BAD_CACHE, EINVAL, REORDER, SELECT, call, pkg  # noqa: F401


def over(base, what, size, *others):
    """Places of `what` (`size` bytes) over the beginning and the end of each of `others` (their bytes)."""
    return [pytest.param(what, base[o] + at, id=f"{what}-{o}-{at}") for o, n in others for at in {4 - size, n - 4}]


def aligned(places, by):
    """The same, towards the middle, where an address has to be a multiple of `by`."""
    return [pytest.param(p.values[0], (p.values[1] + (by - 1 if p.id.rsplit("-", 2)[1] == "" else 0)) // by * by, id=p.id) for p in places]


POOL, TABLE = 40 * 2 * 16 * 64 * 2, 6 * 9 * 4
LOGITS = (5 * 5000 + 5000) * 4


@pytest.mark.parametrize("what,at", aligned(over(APPEND, "q_out", 6 * 256 * 4, ("table", TABLE), ("seq", 24), ("pos", 24), ("K", POOL), ("V", POOL)), 16)
                         + aligned(over(APPEND, "K", POOL, ("V", POOL), ("q", 6 * 256 * 4), ("k", 6 * 128 * 4), ("v", 6 * 128 * 4), ("table", TABLE), ("seq", 24), ("pos", 24)), 16)
                         + aligned(over(APPEND, "V", POOL, ("q", 6 * 256 * 4), ("k", 6 * 128 * 4), ("v", 6 * 128 * 4), ("table", TABLE), ("seq", 24), ("pos", 24)), 16))
def test_append_refuses_what_it_writes_over_what_it_reads(pkg, what, at):  # noqa: F811
    assert call(pkg, "spd_op_append_paged", APPEND, **{what: at}) == EINVAL


@pytest.mark.parametrize("what,at", aligned(over(ATTEND, "out", 6 * 4 * 64 * 4, ("K", POOL), ("V", POOL), ("table", 6 * 60 * 4), ("shared", 8), ("len", 24), ("scratch", 256)), 16)
                         + aligned(over(ATTEND, "scratch", 256, ("K", POOL), ("V", POOL), ("q", 6 * 4 * 64 * 4), ("table", 6 * 60 * 4), ("shared", 8), ("len", 24)), 256))
def test_attention_refuses_what_it_writes_over_what_it_reads(pkg, what, at):  # noqa: F811
    assert call(pkg, "spd_op_attention_shared", ATTEND, **{what: at}) == EINVAL


@pytest.mark.parametrize("what,at", [p for o in ("out_scores", "out_tokens", "out_parents", "out_ended") for p in over(SELECT, o, 32, ("logits", LOGITS), ("scratch", 256))]
                         + over(SELECT, "out_tokens", 32, ("out_scores", 32)) + over(SELECT, "out_parents", 32, ("out_scores", 32), ("out_tokens", 32))
                         + over(SELECT, "out_ended", 32, ("out_scores", 32), ("out_tokens", 32), ("out_parents", 32))
                         + aligned(over(SELECT, "scratch", 256, ("logits", LOGITS), ("scores", 24), ("ended", 24)), 256))
def test_select_refuses_what_it_writes_over_what_it_reads(pkg, what, at):  # noqa: F811
    assert call(pkg, "spd_op_beam_select", SELECT, **{what: at}) == EINVAL


@pytest.mark.parametrize("what,at", over(REORDER, "table_out", TABLE, ("parents", 24), ("len", 24), ("K", 2 * POOL), ("V", 2 * POOL))
                         + aligned(over(REORDER, "K", 2 * POOL, ("V", 2 * POOL), ("table", TABLE), ("parents", 24), ("len", 24)), 16)
                         + aligned(over(REORDER, "V", 2 * POOL, ("table", TABLE), ("parents", 24), ("len", 24)), 16))
def test_reorder_refuses_what_it_writes_over_what_it_reads(pkg, what, at):  # noqa: F811
    assert call(pkg, "spd_op_beam_reorder", REORDER, **{what: at}) == EINVAL


REORDER_SHARED = {**{k: v for k, v in REORDER.items() if k not in ("table_out", "err", "stream")}, "shared": 7 * A, "table_out": 6 * A, "err": None, "stream": None}


@pytest.mark.parametrize("what,at", BAD_CACHE + [("width", 0), ("width", 17), ("width", 4), ("n_layers", 0), ("layer_stride", 40 * 2 * 16 * 64 - 8), ("parents", None), ("len", None),
                                                 ("table_out", None), ("table_out", 3 * A), ("shared", None)]
                         + over(REORDER_SHARED, "table_out", TABLE, ("parents", 24), ("shared", 8)) + aligned(over(REORDER_SHARED, "K", 2 * POOL, ("shared", 8)), 16))
def test_reorder_with_shared_positions_refuses(pkg, what, at):  # noqa: F811
    assert call(pkg, "spd_op_beam_reorder_shared", REORDER_SHARED, **{what: at}) == EINVAL
    assert call(pkg, "spd_op_beam_reorder_shared", REORDER_SHARED, n_seq=0, shared=None) == 0


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
def test_attention_plans_the_blocks_that_it_launches(pkg, dtype, d):  # noqa: F811
    """Shared blocks: two per compute unit at most each a chunk of 128 positions or more (and 4096 at most), also for a sequence on its own with more query heads per
    key/value head than a tile has rows."""
    for group in (1, 4, 16, 17, 34, 64):
        for width in (1, 2, 8, 33):
            for positions in (600, 5000, 40_000):
                chunks, chunk, own, rows, blocks, keys, stages = pkg.spd_test_attention_shared_cut(dtype, 2 * width, width, 2 * group, 2, d, positions, 100)
                tiles = -(-width * group // rows)
                assert blocks == chunks * 4 * tiles and chunks * chunk >= positions + 100 * (width == 1)
                assert chunk == 4096 or (blocks <= 512 + 4 * tiles and (chunk <= 128 or blocks >= 128)), (group, width, positions, blocks)
                assert (keys > 0) == (rows >= 64) and (rows < 64 or width > 1)


# Selections of 16 (groups, beams, vocabulary) and the logits per lane that each takes: every instance of the first kernel, rows on the grid of 16 bytes and off it, last slices
# that are not full.  (The GPU tests run these.)
SELECTIONS = [((16, 16, 9001), 8), ((1, 16, 16_002), 8), ((16, 16, 50_258), 16), ((40, 16, 33_003), 16), ((1, 16, 50_000), 32), ((4, 16, 5003), 32), ((4, 16, 131_072), 64),
              ((4, 16, 131_070), 64), ((2, 16, 100_003), 64)]


@pytest.mark.parametrize("shape,entries", SELECTIONS)
def test_select_slices(pkg, shape, entries):  # noqa: F811
    assert pkg.spd_test_beam_select_cut(*shape[:2], 16, shape[2]) == (entries, -(-shape[2] // (64 * entries)))


def test_select_slices_follow_what_the_gpu_holds(pkg):  # noqa: F811
    """As many entries per lane as make for the least of rounds of waves and turns of the second kernel; a vocabulary of one launch has no slices."""
    assert pkg.spd_test_beam_select_cut(3, 2, 4, 4096) == (0, 1)
    places = {8: 1024 * 8, 16: 1024 * 8, 32: 1024 * 3, 64: 1024 * 2}       # SIMDs and the waves that each holds

    def cost(rows, n_out, vocab, ne):
        slices = -(-vocab // (64 * ne))
        halves = n_out > 8 and slices * n_out > 64 and slices <= n_out
        return -(-rows * slices // places[ne]) * (32 + ne) + -(-slices * n_out // 512) * 96 + 200 * halves

    for rows in (1, 7, 64, 200, 3000):
        for n_out in (1, 5, 16):
            for vocab in (4097, 10_000, 50_258, 131_072, 1_000_001):
                entries, slices = pkg.spd_test_beam_select_cut(rows, 1, n_out, vocab)
                assert slices == -(-vocab // (64 * entries)) and cost(rows, n_out, vocab, entries) == min(cost(rows, n_out, vocab, ne) for ne in places)


class Enqueued(Exception):
    pass


def test_python_looks_arguments_over_once_with_err_as_without(pkg, monkeypatch):  # noqa: F811
    """A good call reaches the library without the check of each tensor that says what is wrong with one; a bad err or shared is still refused."""
    import torch

    from paper_2405_18400_amd import binding
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(binding, "_stream_ptr", lambda device=None: None)

    class Library:
        spd_op_attention_shared_scratch_bytes = spd_op_beam_select_scratch_bytes = staticmethod(lambda *a: 0)

        def __getattr__(self, name):
            def enqueue(*args):
                raise Enqueued(name)
            return enqueue

    monkeypatch.setattr(binding, "lib", Library)
    refused = []
    says = binding._refuse
    monkeypatch.setattr(binding, "_refuse", lambda *a, **k: (refused.append(a), says(*a, **k)))
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    K, V, q, k = torch.zeros(4, 2, 8, 16), torch.zeros(4, 2, 8, 16), torch.zeros(4, 2, 16), torch.zeros(3, 2, 16)
    calls = [lambda **c: pkg.spd_op_append_paged("fp32", K, V, i(2, 2), k, k, i(3), i(3), 1e4, **c),
             lambda **c: pkg.spd_op_attention_shared("fp32", q, K, V, i(4, 2), i(2), i(4), torch.empty_like(q), 2, 3, 3, **c),
             lambda **c: pkg.spd_op_beam_reorder("fp32", K, V, i(4, 2), i(2, 2), i(4), i(4, 2), 2, **c)]
    for f in calls:
        for good in ({}, {"err": i(1)}):
            with pytest.raises(Enqueued):
                f(**good)
        assert not refused
        for bad in (i(2), i(1).long(), torch.zeros(1)):
            with pytest.raises(ValueError):
                f(err=bad)
        refused.clear()
    with pytest.raises(Enqueued, match="spd_op_beam_reorder_shared"):
        calls[2](shared=i(2), err=i(1))
    assert not refused
    for bad in (i(3), i(2).long(), torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            calls[2](shared=bad)


def test_python_refuses_numbers_and_pools_that_would_be_cut_off(pkg, monkeypatch):  # noqa: F811
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    K, V, q = torch.zeros(4, 2, 8, 16), torch.zeros(4, 2, 8, 16), torch.zeros(4, 2, 16)
    for bounds in ((1 << 32, 3), (3, 1 << 31), ((1 << 32) + 3, 3)):
        with pytest.raises(ValueError):
            pkg.spd_op_attention_shared("fp32", q, K, V, i(4, 2), i(2), i(4), torch.empty_like(q), 2, *bounds)
    for end in (1 << 32, (1 << 32) + 2, -(1 << 32)):
        with pytest.raises(ValueError):
            pkg.spd_op_beam_select("fp32", torch.zeros(2, 3, 50), torch.zeros(2, 3), torch.zeros(2, 4), i(2, 4), i(2, 4), ended=i(2, 3), end_token=end)
    with pytest.raises(ValueError):
        pkg.spd_op_beam_reorder("fp32", K[None, None], V[None, None], i(4, 2), i(2, 2), i(4), i(4, 2), 2)


# Calls whose shared blocks share out rows and go through their stages in LDS more than twice over: (dtype, heads, kv, d_head, page, groups, width, shared, own), then keys of a stage,
# stages and rows of a block.  (The GPU tests run these.)
RINGS = [(("fp16", 16, 2, 64, 16, 16, 4, 6001, 40), (64, 4, 64)), (("bf16", 16, 2, 64, 16, 16, 10, 6001, 40), (64, 4, 64)), (("fp16", 16, 2, 64, 16, 16, 10, 6001, 40), (64, 4, 128)),
         (("fp16", 8, 2, 128, 32, 8, 5, 6007, 33), (64, 2, 64)), (("bf16", 32, 2, 128, 16, 8, 6, 5003, 33), (64, 2, 64)), (("fp16", 32, 2, 128, 16, 8, 6, 5003, 33), (32, 4, 128)),
         (("fp16", 8, 2, 256, 16, 8, 5, 4100, 9), (32, 3, 64)), (("bf16", 16, 1, 256, 8, 8, 5, 9001, 9), (32, 3, 64)),
         (("fp16", 32, 4, 64, 4, 16, 3, 5003, 21), (64, 4, 64)),            # more page numbers of a chunk than a block has threads
         (("fp16", 16, 2, 128, 16, 8, 17, 5001, 33), (32, 4, 128))]         # 136 rows: a second tile of eight


@pytest.mark.parametrize("case,cut", RINGS)
def test_rings_go_round(pkg, case, cut):  # noqa: F811
    dtype, heads, kv, d, page, groups, width, shared, own = case
    chunks, chunk, _, rows, _, keys, stages = pkg.spd_test_attention_shared_cut(dtype, groups * width, width, heads, kv, d, shared, own)
    assert (keys, stages, rows) == cut and chunks > 1 and chunk > 2 * stages * keys
    if page == 4:
        assert chunk // page > 256


@pytest.mark.parametrize("layers,stride,off", [(2, POOL, POOL - 16), (2, POOL, 16), (4, 2 * POOL, POOL - 16), (4, 2 * POOL, POOL + 16), (4, 2 * POOL, 7 * POOL - 16), (4, 2 * POOL, 5 * POOL + 16),
                                               (4, 3 * POOL, 2 * POOL + 16), (3, POOL + 16, POOL)])
@pytest.mark.parametrize("first", ["K", "V"])
def test_reorder_refuses_pools_whose_layers_meet(pkg, layers, stride, off, first):  # noqa: F811
    other = "V" if first == "K" else "K"
    assert call(pkg, "spd_op_beam_reorder", REORDER, n_layers=layers, layer_stride=stride // 2, **{first: 64 * A, other: 64 * A + off}) == EINVAL


@pytest.mark.parametrize("at", [-16, POOL - 16, 2 * POOL - 16, 3 * POOL - 16, 7 * POOL - 16])
def test_reorder_refuses_tables_over_a_layer(pkg, at):  # noqa: F811
    """Keys and values in turn, a pool's room between them."""
    pools = dict(K=64 * A, V=64 * A + 2 * POOL, n_layers=3, layer_stride=4 * POOL // 2)
    for what in ("table_out", "table", "parents", "len"):
        assert call(pkg, "spd_op_beam_reorder", REORDER, **pools, **{what: 64 * A + at}) == EINVAL
