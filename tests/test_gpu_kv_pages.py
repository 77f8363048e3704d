"""ivf_kv_fork, ivf_kv_compact and ivf_kv_copy against their sequential forms: whole numbers and copied bits are compared for equality."""
import math

import numpy as np
import pytest
import torch

import kv_reference as R
import kv_whole_reference as W
from paper_2608_08751_b200 import binding as B
from test_gpu_kv import TYPES, _cache, _gen, _i32, _np

pytestmark = pytest.mark.gpu


def _rows(rng, n, most, page, beams=1, spare=40, columns_over=2):
    """(table, lengths, pages): rows of up to `most` tokens; the rows of a group of `beams` share the filled blocks of a first part."""
    lens = rng.integers(0, most + 1, n)
    blocks = [R.ceil_div(int(x), page) for x in lens]
    pages = sum(blocks) + spare
    order = rng.permutation(pages)
    table = rng.integers(0, pages + 500, (n, max(blocks + [1]) + columns_over))  # what lies past the held pages is stale
    at = 0
    for b, k in enumerate(blocks):
        table[b, :k] = order[at: at + k]
        at += k
    for b in range(n):
        first = b // beams * beams
        share = min(lens[b], lens[first]) // 2 // page
        table[b, :share] = table[first, :share]
    return table, lens, pages


def _fork(table, lens, parent, keep, pages, page, **more):
    return B.ivf_kv_fork(_i32(table), _i32(lens), _i32(parent), None if keep is None else _i32(keep), pages, page, **more)


def _same(got, want):
    for name, value in want.items():
        assert (_np(getattr(got, name)) == value).all(), name


SIZES = [  # rows, most tokens, page, beams: small ones go by one block of threads, the others by several launches
    (1, 1, 16, 1), (4, 100, 16, 4), (32, 500, 64, 4), (7, 0, 32, 1), (1024, 200, 16, 2), (1025, 100, 16, 5), (60, 20000, 16, 3), (300, 9000, 128, 8),
    (2100, 1500, 32, 2), (5, 300000, 16, 5),
]


@pytest.mark.parametrize("rows,most,page,beams", SIZES)
@pytest.mark.parametrize("kept", [False, True])
def test_fork_equals_the_sequential_form(rows, most, page, beams, kept):
    rng = np.random.default_rng(rows + most)
    table, lens, pages = _rows(rng, rows, most, page, beams, spare=2 * rows + 40)
    n = max(1, rows + int(rng.integers(-2, 3)))
    first = np.minimum(np.arange(n), rows - 1) // beams * beams
    parent = np.where(rng.random(n) < 0.1, -1, np.minimum(first + rng.integers(0, beams, n), rows - 1))
    keep = None
    if kept:  # cut back by a little, to a block's edge, to nothing, into what is shared
        length = np.where(parent >= 0, lens[parent], 0)
        keep = np.select([rng.random(n) < 0.3, rng.random(n) < 0.2, rng.random(n) < 0.1], [length - rng.integers(0, 9, n), length // page * page, length // 3], length).clip(0)
    want = W.fork(table, lens, parent, keep, pages, page)
    got = _fork(table, lens, parent, keep, pages, page)
    B.ivf_check()
    _same(got, want)
    # into the tensors of an earlier call, the table a view of a wider one
    wide = torch.full((n, table.shape[1] + 3), 77, dtype=torch.int32, device="cuda")
    again = B.KvFork(wide[:, : table.shape[1]], *(torch.full_like(t, 5) for t in got[1:]))
    assert _fork(table, lens, parent, keep, pages, page, fork=again) is again
    B.ivf_check()
    _same(again, want)
    assert (wide[:, table.shape[1]:] == 77).all()


@pytest.mark.parametrize("rows", [6, 1500])
def test_who_keeps_a_partly_filled_page(rows):
    page, columns = 16, 4
    table = np.arange(rows * columns).reshape(rows, columns)
    lens = np.full(rows, 40)
    pages = rows * columns + 20
    cases = [
        ([0, 0, 0], [40, 40, 40]),           # the lowest row keeps it, two copies
        ([0, 0], [40, 20]),                  # the second row ends in a block that the first one fills: a copy of it
        ([0, 0], [20, 40]),                  # the same the other way round
        ([0, 0], [20, 24]),                  # both end in block 1, the longer one second
        ([0, 0, 0], [32, 16, 48 - 8]),       # edges: nothing partly filled but the last
        ([1, 0, 1, -1, 0], [5, 7, 16, 0, 0]),
        ([0], [33]),
    ]
    for parent, keep in cases:
        _same(_fork(table, lens, parent, keep, pages, page), W.fork(table, lens, np.array(parent), np.array(keep), pages, page))
    # a page that another row shares as filled is not written into when this row is cut back into it
    table[1, 0] = table[0, 0]
    got = _fork(table, lens, [0, 1], [8, 40], pages, page)
    _same(got, W.fork(table, lens, np.array([0, 1]), np.array([8, 40]), pages, page))
    assert int(got.copy_from[0]) == table[0, 0] and int(got.table[0, 0]) != table[0, 0] and int(got.table[1, 0]) == table[0, 0]
    B.ivf_check()


@pytest.mark.parametrize("rows", [20, 1300])
@pytest.mark.parametrize("what", ["parent", "keep", "length", "page", "columns"])
def test_fork_flags_and_skips_what_is_out_of_range(rows, what):
    rng = np.random.default_rng(1)
    table, lens, pages = _rows(rng, rows, 200, 32, spare=50)
    lens[:6] = np.maximum(lens[:6], 10)
    table[:6, 0] = np.arange(6)
    parent, keep = np.arange(rows), lens.copy()
    if what == "parent":
        parent[3] = rows
    elif what == "keep":
        keep[2], keep[4] = lens[2] + 1, -1
    elif what == "length":
        lens[1], keep = -5, None
    elif what == "page":
        table[0, 0], table[5, lens[5] // 32 if lens[5] % 32 else 0] = pages, pages + 3
        table[2, 0] = -1  # a missing one is nothing to speak of
    else:
        lens[1] = keep[1] = table.shape[1] * 32 + 1
    got = _fork(table, lens, parent, keep, pages, 32)
    with pytest.raises(B.IvfError) as e:
        B.ivf_check()
    assert e.value.code == B.IVF_ERR_BAD_ID and "ivf_kv_fork" in str(e.value)
    _same(got, W.fork(table, lens, parent, keep, pages, 32))


@pytest.mark.parametrize("rows,spare", [(8, 3), (8, 0), (1200, 100)])
def test_fork_without_pages_enough(rows, spare):
    table, lens = np.arange(rows)[:, None].repeat(2, 1), np.full(rows, 5)
    table[:, 1] = -1
    parent = np.arange(rows) // 4 * 4
    pages = rows // 4 * 4 if spare == 0 else rows // 4 + spare  # (row 4 i holds page 4 i; numbers past the cache are missing pages)
    table[::4, 0] = np.arange(rows // 4)
    got = _fork(table, lens, parent, None, pages if spare else rows // 4, 16)
    with pytest.raises(B.IvfError) as e:
        B.ivf_check()
    assert e.value.code == B.IVF_ERR_NO_PAGES and "ivf_kv_fork" in str(e.value)
    _same(got, W.fork(table, lens, parent, None, pages if spare else rows // 4, 16))


def test_fork_of_nothing():
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    got = B.ivf_kv_fork(torch.zeros(0, 3, dtype=torch.int32, device="cuda"), none, none, None, 70, 16)
    assert _np(got.free_pages).tolist() == list(range(70)) and int(got.n_free) == 70 and got.table.shape == (0, 3)
    got = B.ivf_kv_fork(torch.zeros(0, 3, dtype=torch.int32, device="cuda"), none, _i32([-1, -1]), None, 0, 16)
    assert int(got.n_free) == 0 and (got.table == -1).all() and (got.copy_from == -1).all()
    got = B.ivf_kv_fork(torch.zeros(0, 3, dtype=torch.int32, device="cuda"), none, none, None, 40000, 16)
    assert _np(got.free_pages).tolist() == list(range(40000))
    B.ivf_check()


@pytest.mark.parametrize("rows,most,page,beams", SIZES)
@pytest.mark.parametrize("moves", [None, 0, 7, 10 ** 6])
def test_compact_equals_the_sequential_form(rows, most, page, beams, moves):
    rng = np.random.default_rng(rows + most + 1)
    table, lens, pages = _rows(rng, rows, most, page, beams)
    lens = np.where(rng.random(rows) < 0.4, 0, lens)
    want = W.compact(table, lens, pages, page, pages if moves is None else moves)
    out = torch.full(table.shape, 9, dtype=torch.int32, device="cuda")
    got = B.ivf_kv_compact(_i32(table), _i32(lens), pages, page, max_moves=moves, out=out)
    B.ivf_check()
    assert got.table is out
    _same(got, want)
    # in place, in a view; and nothing is left to move after all moves
    wide = torch.full((rows, table.shape[1] + 5), 77, dtype=torch.int32, device="cuda")
    wide[:, : table.shape[1]] = _i32(table)
    got = B.ivf_kv_compact(wide[:, : table.shape[1]], _i32(lens), pages, page, max_moves=moves)
    _same(got, want)
    assert (wide[:, table.shape[1]:] == 77).all()
    if moves is None:
        more = B.ivf_kv_compact(got.table, _i32(lens), pages, page)
        assert (more.copy_from == -1).all() and (_np(more.table) == want["table"]).all()
    B.ivf_check()


@pytest.mark.parametrize("rows", [20, 1300])
def test_compact_flags_and_skips_what_is_out_of_range(rows):
    rng = np.random.default_rng(2)
    for what in ("length", "long", "page"):
        table, lens, pages = _rows(rng, rows, 200, 32)
        if what == "length":
            lens[2] = -4
        elif what == "long":
            table[1] = np.where(table[1] >= pages, -1, table[1])
            lens[1] = table.shape[1] * 32 + 5
        else:
            lens[3], table[3, 0] = 40, pages
        got = B.ivf_kv_compact(_i32(table), _i32(lens), pages, 32, out=torch.empty_like(_i32(table)))
        with pytest.raises(B.IvfError) as e:
            B.ivf_check()
        assert e.value.code == B.IVF_ERR_BAD_ID and "ivf_kv_compact" in str(e.value)
        _same(got, W.compact(table, lens, pages, 32, pages))


@pytest.mark.parametrize("kv,dim,page,kind,layout", [(1, 16, 16, "bf16", "head"), (4, 96, 32, "fp16", "token"), (8, 128, 64, "bf16", "both"), (3, 256, 128, "fp16", "head"),
                                                     (2, 80, 64, "bf16", "token")])
@pytest.mark.parametrize("filled", [False, True])
def test_copy_moves_bits(kv, dim, page, kind, layout, filled):
    g = _gen(dim)
    n, pages = 23, 60
    caches = [_cache(pages, kv, page, dim, kind, layout, 0.0) for _ in range(2)]
    for c in caches:
        c.copy_(torch.randn(c.shape, device="cuda", generator=g).to(TYPES[kind]))
        c[5] = math.nan
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    source, to = order[:n].clone(), order[n: 2 * n].clone()
    source[2], to[4], source[6], to[6] = -1, -1, -1, -1
    source[9] = source[8]  # one page may be copied twice
    fill = torch.randint(-1, page + 1, (n,), device="cuda", generator=g).to(torch.int32) if filled else None
    codes = torch.randint(-127, 128, (pages, kv, dim), device="cuda", generator=g).to(torch.int8)
    scales = torch.rand(pages, kv, device="cuda", generator=g)
    want = [c.clone() for c in caches]
    want_codes, want_scales = codes.clone(), scales.clone()
    for i, (a, b) in enumerate(zip(source.tolist(), to.tolist())):
        f = page if fill is None else int(fill[i])
        if a < 0 or b < 0 or f <= 0:
            continue
        for w in want:
            w[b, :, :f] = w[a, :, :f]
        want_codes[b], want_scales[b] = codes[a], scales[a]
    B.ivf_kv_copy(*caches, source, to, fill, codes, scales)
    B.ivf_check()
    for w, c in zip(want, caches):
        assert torch.equal(w.contiguous().view(torch.int16), c.contiguous().view(torch.int16))
    assert torch.equal(codes, want_codes) and torch.equal(scales, want_scales)
    B.ivf_kv_copy(*caches, source[:0], to[:0])


def test_copy_flags_and_skips_what_is_out_of_range():
    for what in ("from", "to", "fill"):
        k, v = (torch.randn(6, 2, 16, 32, device="cuda").half() for _ in range(2))
        was = k.clone()
        source, to, fill = _i32([0, 1]), _i32([2, 3]), _i32([16, 16])
        {"from": source, "to": to, "fill": fill}[what][0] = 17
        B.ivf_kv_copy(k, v, source, to, fill)
        with pytest.raises(B.IvfError) as e:
            B.ivf_check()
        assert e.value.code == B.IVF_ERR_BAD_ID and "ivf_kv_copy" in str(e.value)
        assert torch.equal(k[2], was[2]) and torch.equal(k[3], was[1])


def test_far_pages():
    pages, stride = 1100, 2_000_000
    big = torch.zeros(pages, stride, dtype=torch.float16, device="cuda")
    k, v = (big.as_strided((pages, 2, 64, 64), (stride, 4096, 64, 1), off) for off in (0, 8192))
    k[1099], v[1098] = 1.5, 2.5
    B.ivf_kv_copy(k, v, _i32([1099, 1098]), _i32([1090, 1]))
    B.ivf_check()
    assert (k[1090] == 1.5).all() and (v[1] == 2.5).all() and (v[1090] == 0).all() and (k[1] == 0).all()


@pytest.mark.parametrize("rows,most", [(16, 300), (900, 3000)])
def test_fork_attend_and_compact_as_a_server_does(rows, most):
    """Rows branch, end and are cut back; what a row reads through its table stays what it was, copies and moves included."""
    rng = np.random.default_rng(rows)
    page, kv, dim = 16, 1, 16
    table, lens, pages = _rows(rng, rows, most, page, beams=2, spare=4 * rows, columns_over=4)
    k = torch.randn(pages, kv, page, dim, device="cuda").half()
    v = torch.randn(pages, kv, page, dim, device="cuda").half()

    def read(c, table, lens):
        c, table = _np(c), _np(table)
        return [c[table[b, np.arange(int(n)) // page], 0, np.arange(int(n)) % page] for b, n in enumerate(_np(lens))]
    held = _i32(table), _i32(lens)
    for step in range(3):
        n = rows
        parent = np.where(rng.random(n) < 0.2, -1, rng.integers(0, n, n))
        length = np.where(parent >= 0, _np(held[1])[parent], 0)
        keep = np.where(rng.random(n) < 0.3, length - rng.integers(0, 20, n), length).clip(0)
        before = [read(c, *held) for c in (k, v)]
        fork = B.ivf_kv_fork(*held, _i32(parent), _i32(keep), pages, page)
        B.ivf_kv_copy(k, v, fork.copy_from, fork.copy_to, fork.copy_fill)
        for c, was in zip((k, v), before):
            for row, p, f in zip(read(c, fork.table, fork.kv_lens), parent, keep):
                assert p < 0 or (row == was[p][: int(f)]).all()
        # new tokens go to pages that nobody else writes
        plan = B.ivf_kv_tables(fork.kv_lens, torch.ones_like(fork.kv_lens), fork.free_pages[: int(fork.n_free)], fork.table, page, n)
        slots = _np(plan.token_slot)
        assert (slots >= 0).all() and len(set(slots.tolist())) == n
        holders = np.zeros(pages, np.int64)
        for b, length in enumerate(_np(fork.kv_lens)):
            np.add.at(holders, _np(fork.table)[b, : int(length) // page], 1)
        assert (holders[slots // page] == 0).all()
        B.ivf_kv_append(torch.randn(n, 1, dim, device="cuda").half(), torch.randn(n, kv, dim, device="cuda").half(), torch.randn(n, kv, dim, device="cuda").half(),
                        k, v, plan.token_pos, plan.token_slot)
        lens_now = plan.kv_lens.clone()
        q = torch.randn(n, 2, dim, device="cuda").half()
        out = B.ivf_kv_attend_chunk(q, k, v, fork.table, plan.token_start, lens_now, 0.25)[0]
        before = [read(c, fork.table, lens_now) for c in (k, v)]
        moved = B.ivf_kv_compact(fork.table, lens_now, pages, page)
        B.ivf_kv_copy(k, v, moved.copy_from, moved.copy_to)
        for c, was in zip((k, v), before):
            assert all((a == b).all() for a, b in zip(read(c, moved.table, lens_now), was))
        assert int(moved.table.max()) < int(moved.n_held)
        assert torch.equal(out, B.ivf_kv_attend_chunk(q, k, v, moved.table, plan.token_start, lens_now, 0.25)[0])
        held = moved.table, lens_now
    B.ivf_check()


def test_captured_plans_do_not_share_scratch_memory():
    rng = np.random.default_rng(3)
    calls = []
    for seed in range(2):
        table, lens, pages = _rows(rng, 1500, 300, 16, beams=2, spare=3100)
        parent = np.arange(1500) // 2 * 2
        ints = _i32(table), _i32(lens), _i32(parent)
        graph = torch.cuda.CUDAGraph()
        _fork(table, lens, parent, None, pages, 16)
        with torch.cuda.graph(graph):
            fork = B.ivf_kv_fork(*ints, None, pages, 16)
            moved = B.ivf_kv_compact(fork.table, fork.kv_lens, pages, 16, out=torch.empty_like(fork.table))
        calls.append((graph, fork, moved, W.fork(table, lens, parent, None, pages, 16), pages, ints))
    for i in (0, 1, 1, 0):
        graph, fork, moved, want, pages, _ = calls[i]
        for t in (*fork, *moved):
            t.fill_(3)
        graph.replay()
        B.ivf_check()
        _same(fork, want)
        _same(moved, W.compact(want["table"], want["kv_lens"], pages, 16, pages))
