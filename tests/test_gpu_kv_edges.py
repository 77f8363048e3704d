"""Block-cache operators at their edges, against the plain 64-bit forms; tolerances as in test_gpu_kv.py."""
import math
import subprocess
import sys

import numpy as np
import pytest
import torch

import kv_reference as R
from paper_2608_08751_b200 import binding as B
from test_gpu_kv import _attend_case, _cache, _check_attend, _gen, _i32, _np, kernel, select_kernel  # noqa: F401
from test_gpu_kv import test_append_matches_the_formula as check_append

pytestmark = pytest.mark.gpu


def _against_plain(case, scale, kind, dim):
    kc, vc, table, req, pos, q, sel = case
    got, lse = B.ivf_kv_attend(q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), scale, want_lse=True)
    B.ivf_check()
    _check_attend(got, lse, R.attend(_np(q), np.nan_to_num(_np(kc)), np.nan_to_num(_np(vc)), table, req, pos, sel, scale), kind, dim)
    return got


# ---------------------------------------------------------------------------------------------- requests that share a window

# A page of 128 is two boxes of a window's plan, and a last one that nobody sees is given back: the box of the request
# that has it, not of one before it.
@pytest.mark.parametrize("dim,kind", [(64, "fp16"), (128, "bf16"), (256, "bf16")])
@pytest.mark.parametrize("contexts,group,empty", [
    ([501, 8], 8, [1]), ([8, 501], 8, [0]), ([501, 9, 8], 4, [1, 2]), ([8, 501, 9], 4, [0, 2]), ([700, 8, 501], 4, [1]), ([9, 8], 8, [0, 1]),
])
def test_a_request_with_no_block_leaves_its_neighbours_alone(kernel, contexts, group, empty, dim, kind):  # noqa: F811
    case = _attend_case(contexts, 8, 1, group, dim, 128, 4, kind, "head", seed=len(contexts) + dim)
    req, sel = case[3], case[6]
    for b, c in enumerate(contexts):
        sel[req == b] = -1 if b in empty else [0, (c - 1) // 128, -1, -1] if c > 128 else [0, -1, -1, -1]
    got = _against_plain(case, 1 / math.sqrt(dim), kind, dim)
    assert (got[torch.from_numpy(np.isin(req, empty)).cuda()] == 0).all()


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("contexts,empty", [([501, 8], 1), ([8, 501], 0)])
def test_a_request_without_pages_leaves_its_neighbours_alone(kernel, contexts, empty, page):  # noqa: F811
    kc, vc, table, req, pos, q, _ = _attend_case(contexts, 8, 2, 8, 64, page, 4, "bf16", "head", seed=page)
    table[empty] = -1  # it found no free page
    codes = torch.randint(-127, 128, (kc.shape[0], 2, 64), device="cuda", generator=_gen(1)).to(torch.int8)
    sel = _np(B.ivf_kv_select(q, codes, torch.ones(kc.shape[0], 2, device="cuda"), _i32(table), _i32(req), _i32(pos), page, 4))
    assert (sel[req == empty] == -1).all() and (sel[req != empty][:, :, 0] == 0).all()
    _against_plain((kc, vc, table, req, pos, q, sel), 0.125, "bf16", 64)


# ---------------------------------------------------------------------------------------------- padding inside a window

# A token is padding by its request or by its position; either way the window's other tokens keep their places.
@pytest.mark.parametrize("page", [32, 128])
@pytest.mark.parametrize("group,fresh", [(8, 8), (2, 32), (1, 60)])
@pytest.mark.parametrize("by_pos,by_req", [([3], []), ([3], [5]), ([0, 9], [12]), ([15], [])])
def test_padding_by_position_inside_a_shared_window(kernel, by_pos, by_req, group, fresh, page):  # noqa: F811
    case = _attend_case([400, 260], fresh, 2, group, 64, page, 3, "bf16", "head", seed=fresh + page)
    req, pos = case[3], case[4]
    pos[by_pos], req[by_req] = -1, -1
    got = _against_plain(case, 0.125, "bf16", 64)
    assert (got[by_pos + by_req] == 0).all()


# ---------------------------------------------------------------------------------------------- output over the queries

@pytest.mark.parametrize("group,fresh", [(4, 64), (20, 40), (8, 1)])
def test_output_in_place_of_the_queries(kernel, group, fresh):  # noqa: F811
    kc, vc, table, req, pos, q, sel = _attend_case([640, 300], fresh, 2, group, 128, 64, 4, "bf16", "head", seed=group)
    n = len(req)
    for h in range(2):  # one block that the odd tokens of the first request do not see
        for t in np.flatnonzero(req == 0):
            sel[t, h] = [0, 2, 5, 9] if t % 2 else [0, 3, 5, 9]
    vc[int(table[0, 3]), :, 7] = math.inf
    want = R.attend(_np(q), np.nan_to_num(_np(kc)), np.nan_to_num(_np(vc), posinf=1e30), table, req, pos, sel, 0.1)
    clean = [t for t in range(n) if req[t] == 1 or t % 2]
    got, lse = B.ivf_kv_attend(q.clone(), kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), 0.1, want_lse=True)
    over = q.clone()
    same, lse2 = B.ivf_kv_attend(over, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), 0.1, out=over, want_lse=True)
    B.ivf_check()
    assert same.data_ptr() == over.data_ptr()
    for x, y in ((got, lse), (same, lse2)):
        _check_attend(x[clean], y[clean], tuple(w[clean] for w in want), "bf16", 128)


def test_output_beside_the_queries(kernel):  # noqa: F811
    # rows of one buffer in turn: the same numbers as apart
    kc, vc, table, req, pos, q, sel = _attend_case([640, 300], 64, 2, 4, 128, 64, 4, "bf16", "head", seed=8)
    both = torch.zeros(len(req), 2, 8, 128, dtype=q.dtype, device="cuda")
    both[:, 0] = q
    args = (kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), 0.1)
    want, _ = B.ivf_kv_attend(q, *args)
    got, _ = B.ivf_kv_attend(both[:, 0], *args, out=both[:, 1])
    B.ivf_check()
    assert torch.equal(got, want) and torch.equal(both[:, 0], q)


# ---------------------------------------------------------------------------------------------- weights of single tokens

# For up to 8 query heads to a kv head a weight w (the largest is 1) meets the values as two 16-bit parts.  With u = 2^-8 or 2^-11 the first is within u w of it, the
# second within u of that rest, or within 2^-25 where float16 has no finer steps: u^2 w + 2^-25 in all, which is
# u^2 + 2^-25 / (smallest weight) of the weighted mean of |v|.  Each product of 16 tokens joins the sums in 32 bits with an
# error of 2^-22 of them at most; a warp takes every fourth piece of 16 tokens, two products each.  The rest as in
# test_gpu_kv.py: the output's own rounding, the logits', 2^-20.  (Weights of one part miss this by far.)
@pytest.mark.parametrize("contexts,fresh,kv,group,dim,page,take,kind", [
    ([20], 1, 2, 8, 128, 64, 2, "bf16"), ([33, 7], 2, 2, 7, 64, 16, 3, "fp16"), ([18] * 40, 1, 4, 4, 256, 32, 2, "bf16"),
    ([50], 3, 1, 3, 96, 128, 1, "fp16"), ([16] * 70, 1, 8, 2, 128, 64, 1, "bf16"), ([900], 1, 2, 8, 128, 64, 12, "bf16"),
])
def test_weights_of_single_tokens_keep_their_bits(contexts, fresh, kv, group, dim, page, take, kind):
    kc, vc, table, req, pos, q, sel = _attend_case(contexts, fresh, kv, group, dim, page, take, kind, "head", seed=take)
    scale = 0.3 / math.sqrt(dim)  # many weights of much the same size
    B.ivf_debug_set_kv_attend(1)
    try:
        got, _ = B.ivf_kv_attend(q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), scale)
    finally:
        B.ivf_debug_set_kv_attend(0)
    B.ivf_check()
    keys = np.nan_to_num(_np(kc))
    out, _, size, unit = R.attend(_np(q), keys, np.nan_to_num(_np(vc)), table, req, pos, sel, scale)
    least = np.ones(q.shape[:2])
    for t in range(len(req)):
        for h in range(kv):
            k = np.concatenate([keys[table[req[t], b], h, : max(0, min(page, pos[t] + 1 - b * page))] for b in sel[t, h] if b >= 0])
            z = _np(q)[t, h * group: (h + 1) * group] @ k.T * scale
            least[t, h * group: (h + 1) * group] = np.exp(z.min(1) - z.max(1))
    u = R.UNIT[kind]
    parts = u * u + (2.0 ** -25 / least if kind == "fp16" else 0 * least) + 2 * R.ceil_div(take * page, 64) * 2.0 ** -22
    tol = u * np.abs(out) + (parts + 2 * dim * 2.0 ** -24 * unit + 2.0 ** -20)[..., None] * size + R.TINY[kind]
    d = np.abs(_np(got) - out)
    assert (d <= tol).all(), (d / tol).max()


@pytest.mark.parametrize("group", [3, 8, 9, 20])
@pytest.mark.parametrize("dim,kind", [(64, "fp16"), (128, "bf16"), (256, "bf16")])
@pytest.mark.parametrize("fresh", [1, 40])
def test_infinite_values_of_tokens_that_are_seen(kernel, fresh, group, dim, kind):  # noqa: F811
    kc, vc, table, req, pos, q, sel = _attend_case([200], fresh, 1, group, dim, 32, 7, kind, "head", seed=group)
    vc[int(table[0, 1]), 0, 3, :16] = math.inf
    vc[int(table[0, 1]), 0, 4, 16:32] = -math.inf
    scale = 0.1 / math.sqrt(dim)
    got = _np(B.ivf_kv_attend(q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), scale)[0])
    B.ivf_check()
    seen = (sel[:, 0] == 1).any(1)
    assert seen.any()
    assert (got[seen, :, :16] == math.inf).all() and (got[seen, :, 16:32] == -math.inf).all()
    want = R.attend(_np(q), np.nan_to_num(_np(kc)), np.nan_to_num(_np(vc), posinf=0, neginf=0), table, req, pos, sel, scale)
    got[seen, :, :32] = want[0][seen, :, :32]
    _check_attend(torch.from_numpy(got), None, want, kind, dim)


# ---------------------------------------------------------------------------------------------- graphs and streams

def _mixed_windows(seed, requests, fresh, group=8, page=64):
    """Prompt chunks of which some windows are finished and some left: several requests, a value that is not finite."""
    case = _attend_case([700 + 13 * i for i in range(requests)], fresh, 2, group, 128, page, 4, "bf16", "head", seed=seed, shared=True)
    table, vc = case[2], case[1]
    vc[int(table[0, 3]), :, 5] = math.inf
    kc, vc, table, req, pos, q, sel = case
    return (q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), 0.1)


def _same(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_a_graph_outlives_larger_calls(kernel):  # noqa: F811
    small, large = _mixed_windows(1, 9, 24), _mixed_windows(2, 6, 400)
    first = B.ivf_kv_attend(*small)[0]
    want = first.clone()
    assert want.isfinite().any() and not want.isfinite().all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, _ = B.ivf_kv_attend(*small)
    B.ivf_kv_attend(*large)
    B.ivf_release_workspace()
    spoil = torch.full((1 << 22,), 1, dtype=torch.uint8, device="cuda")  # takes over what may have been given back
    for fill in (0, 1, 255):
        out.view(torch.uint8).fill_(fill)
        spoil.fill_(fill)
        graph.replay()
        torch.cuda.synchronize()
        assert _same(out, want)
    B.ivf_check()


def test_two_streams_without_order(kernel):  # noqa: F811
    cases = [_mixed_windows(3, 12, 20), _mixed_windows(4, 2, 300)]
    want = [B.ivf_kv_attend(*c)[0].clone() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[torch.empty_like(w) for _ in range(20)] for w in want]
    torch.cuda.synchronize()
    for i in range(20):
        for c, s, o in zip(cases, streams, outs):
            with torch.cuda.stream(s):
                B.ivf_kv_attend(*c, out=o[i])
    torch.cuda.synchronize()
    B.ivf_check()
    for w, o in zip(want, outs):
        assert all(_same(x, w) for x in o)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_stale_outputs_are_not_taken_for_marks(kernel, kind):  # noqa: F811
    # an output buffer full of the bytes that mark a row, of a call that finishes every window
    case = _attend_case([640], 128, 2, 20, 64, 64, 4, kind, "head", seed=6, shared=True)
    kc, vc, table, req, pos, q, sel = case
    out = torch.full_like(q, math.nan)
    out.view(torch.int16).fill_(-1)
    got, _ = B.ivf_kv_attend(q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), 0.1, out=out)
    want, _ = B.ivf_kv_attend(q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), 0.1)
    B.ivf_check()
    assert _same(got, want) and got.isfinite().all()


def test_more_rows_left_than_one_look():
    # nearly every window is left (requests of four tokens): several rounds of looking, and the same arithmetic as by themselves
    n_req, kv, dim = 330, 40, 64
    g = _gen(7)
    kc, vc = (torch.randn(n_req, kv, 16, dim, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    req, pos = np.repeat(np.arange(n_req), 4), np.tile(np.arange(4), n_req)
    req[500:540], pos[500:540] = 3, np.arange(4).repeat(10)  # and some that are not
    q = torch.randn(len(req), kv * 2, dim, device="cuda", generator=g).to(torch.bfloat16)
    sel = torch.zeros(len(req), kv, 2, dtype=torch.int32, device="cuda")
    sel[:, :, 1] = -1
    args = (q, kc, vc, _i32(np.arange(n_req)).view(-1, 1), _i32(req), _i32(pos), sel, 0.1)
    got = []
    try:
        for forced in (1, 2):
            B.ivf_debug_set_kv_attend(forced)
            got.append(B.ivf_kv_attend(*args)[0])
    finally:
        B.ivf_debug_set_kv_attend(0)
    B.ivf_check()
    assert torch.equal(got[0][:448], got[1][:448]) and torch.equal(got[0][640:], got[1][640:])
    assert got[1].isfinite().all() and (got[0] - got[1]).abs().max() < 0.1


# ---------------------------------------------------------------------------------------------- tables: no room

def test_tables_without_room_for_tokens_or_blocks():
    # nothing but the table, the lengths and the counts to write
    table = torch.full((1, 4), 9, dtype=torch.int32, device="cuda")
    plan = B.ivf_kv_tables(_i32([20]), _i32([0]), _i32([5, 6]), table, 16, 0, max_touched=0)
    B.ivf_check()
    assert _np(plan.kv_lens).tolist() == [20] and _np(plan.token_start).tolist() == [0, 0] and int(plan.used) == 0
    assert _np(table).tolist() == [[9, 9, -1, -1]]
    plan = B.ivf_kv_tables(_i32([20]), _i32([30]), _i32([5, 6]), table, 16, 0, max_touched=0)
    with pytest.raises(B.IvfError) as e:
        B.ivf_check()
    assert e.value.code == B.IVF_ERR_NO_PAGES
    assert _np(table).tolist() == [[9, 9, 5, 6]] and int(plan.used) == 2 and _np(plan.token_start).tolist() == [0, 30]


# ---------------------------------------------------------------------------------------------- tables: long sums

def test_tables_of_lengths_whose_sum_passes_31_bits():
    # each length is fine by itself; the sums are not, and nothing is read or written by a sum that went round
    page, most = 16, 2 ** 31 - 1
    lengths = [(0, 1_500_000_000), (40, 1_500_000_000), (17, 1_500_000_000), (5, 3)]
    table = torch.full((4, 6), 77, dtype=torch.int32, device="cuda")
    plan = B.ivf_kv_tables(_i32([c for c, _ in lengths]), _i32([f for _, f in lengths]), _i32([3, 4]), table, page, 40, max_touched=5)
    with pytest.raises(B.IvfError) as e:
        B.ivf_check()
    assert e.value.code == B.IVF_ERR_NO_PAGES and "ivf_kv_tables" in str(e.value)
    assert _np(plan.token_start).tolist() == [0, 1_500_000_000, most, most, most]
    assert int(plan.used) == sum(R.ceil_div(c + f, page) - R.ceil_div(c, page) for c, f in lengths)
    assert _np(plan.kv_lens).tolist() == [c + f for c, f in lengths]
    assert _np(plan.token_req).tolist() == [0] * 40 and _np(plan.token_pos).tolist() == list(range(40))
    assert _np(plan.token_slot).tolist() == [48 + i for i in range(16)] + [64 + i for i in range(16)] + [-1] * 8
    assert _np(plan.touched_page).tolist() == [3, 4, -1, -1, -1] and _np(plan.touched_fill).tolist() == [16, 16, 0, 0, 0]
    assert _np(table).tolist() == [[3, 4, -1, -1, -1, -1], [77, 77, 77, -1, -1, -1], [77, 77, -1, -1, -1, -1], [77, -1, -1, -1, -1, -1]]


@pytest.mark.parametrize("n", [2, 3, 1500])
def test_tables_of_sums_that_come_round_to_a_small_number(n):
    # 32-bit sums of these are 0, 1 and so on again: still too few tokens
    long = 2 ** 31 - 200
    cached, fresh = [5] * n, [long] * n
    table = torch.full((n, 3), 8, dtype=torch.int32, device="cuda")
    plan = B.ivf_kv_tables(_i32(cached), _i32(fresh), _i32([1]), table, 128, 600)
    with pytest.raises(B.IvfError) as e:
        B.ivf_check()
    assert e.value.code == B.IVF_ERR_NO_PAGES
    assert (plan.token_req == 0).all() and _np(plan.token_pos).tolist() == list(range(5, 605))
    assert _np(plan.token_start)[:3].tolist() == [0, long, 2 ** 31 - 1]
    assert int(plan.used) == min(2 ** 31 - 1, n * (R.ceil_div(long + 5, 128) - 1))
    assert _np(plan.token_slot).tolist() == [8 * 128 + i for i in range(5, 128)] + [128 + i for i in range(128)] + [-1] * (600 - 251)


# ---------------------------------------------------------------------------------------------- threads

_THREADS = """
import ctypes, sys, threading
import torch
from paper_2608_08751_b200 import binding as B
L = B.lib()
i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
stream = torch.cuda.current_stream().cuda_stream
s64 = lambda *v: (ctypes.c_int64 * len(v))(*v)
failed = []
zero = torch.zeros(1 << 16, dtype=torch.int32, device="cuda")
for dtype in (B.IVF_F16, B.IVF_BF16):
    for kernel in (1, 2):
        B.ivf_debug_set_kv_select(kernel)
        for dim in ((64, 128, 256) if kernel == 1 else range(32, 257, 32)):
            q = torch.zeros(1, 1, dim, dtype=torch.float16, device="cuda")
            codes, scales = torch.zeros(1, 1, dim, dtype=torch.int8, device="cuda"), torch.zeros(1, 1, device="cuda")
            def call(blocks):
                table, out = zero[:blocks], torch.empty(1, dtype=torch.int32, device="cuda")
                rc = L.ivf_kv_select(q.data_ptr(), s64(dim, dim), dtype, 1, 1, 1, dim, codes.data_ptr(), scales.data_ptr(), 1, table.data_ptr(), blocks, 1,
                                     blocks, 16, zero.data_ptr(), zero.data_ptr(), 1, 0, 1, out.data_ptr(), stream)
                if rc:
                    failed.append((dtype, kernel, dim, blocks, L.ivf_last_error()))
            small, large = (12000, 49152) if kernel == 1 else (700, 2688)
            gate = threading.Barrier(4)
            def first(blocks):
                gate.wait()
                call(blocks)
            threads = [threading.Thread(target=first, args=(b,)) for b in (small, large, small, large)]
            [t.start() for t in threads]
            [t.join() for t in threads]
            for b in (large, small, large):
                call(b)
torch.cuda.synchronize()
B.ivf_check()
print(len(failed), failed[:3])
sys.exit(1 if failed else 0)
"""


def test_first_calls_of_several_host_threads():
    # each thread's first launch of a kernel asks for another amount of shared memory
    run = subprocess.run([sys.executable, "-c", _THREADS], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout + run.stderr


# ---------------------------------------------------------------------------------------------- summaries and queries that are not finite

@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_a_block_without_a_finite_mean_has_no_summary(what):
    kc = _cache(3, 2, 16, 64, "bf16", fill=1.0)
    kc[1, 0, 4, 17] = what
    codes, scales = torch.full((3, 2, 64), 99, dtype=torch.int8, device="cuda"), torch.full((3, 2), 5.0, device="cuda")
    B.ivf_kv_summarize(kc, _i32([0, 1, 2]), _i32([16, 9, 4]), codes, scales)
    B.ivf_check()
    assert (codes[1, 0] == 0).all() and float(scales[1, 0]) == 0.0
    codes[1, 0], scales[1, 0] = codes[1, 1], scales[1, 1]
    assert (codes == 127).all() and (scales == scales[0, 0]).all() and float(scales[0, 0]) > 0


@pytest.mark.parametrize("what", [math.nan, math.inf])
@pytest.mark.parametrize("fresh", [1, 40])
def test_a_query_that_is_not_finite_prefers_no_block(select_kernel, fresh, what):  # noqa: F811
    n_blocks, dim = 300, 96
    g = _gen(3)
    codes = torch.randint(-127, 128, (n_blocks, 2, dim), device="cuda", generator=g).to(torch.int8)
    q = torch.randn(fresh, 6, dim, device="cuda", generator=g).to(torch.bfloat16)
    q[0, 1, 40] = what  # a head of the first group
    pos = np.arange(n_blocks * 16 - fresh, n_blocks * 16)
    table = np.arange(n_blocks)[None]
    scales = torch.rand(n_blocks, 2, device="cuda", generator=g) + 0.1
    got = _np(B.ivf_kv_select(q, codes, scales, _i32(table), _i32([0] * fresh), _i32(pos), 16, 8, n_first=1, n_last=2))
    B.ivf_check()
    assert got[0, 0].tolist() == [0, 1, 2, 3, 4, 5, pos[0] // 16 - 1, pos[0] // 16]
    q[0, :3] = 0  # no preference either, and a number for the plain form
    want = R.select(_np(q), _np(codes), scales.cpu().numpy(), table, np.zeros(fresh, np.int64), pos, 16, 8, 1, 2)
    assert (got == want).all()


# ---------------------------------------------------------------------------------------------- append

@pytest.mark.parametrize("n,kv,group,dim,rot,pairs,page,kind,layout,weights", [
    # from 592 tokens on a block of threads takes a whole token, several rows to a lane group
    (640, 8, 4, 128, 128, False, 64, "bf16", "head", True), (640, 8, 4, 128, 64, True, 32, "fp16", "token", True),
    (601, 8, 2, 256, 256, False, 16, "fp16", "both", True), (593, 12, 1, 256, 128, True, 64, "bf16", "token", True),
    (700, 5, 7, 96, 96, True, 128, "bf16", "head", False), (1000, 3, 20, 80, 32, False, 32, "fp16", "head", True),
    (592, 1, 64, 64, 64, True, 16, "bf16", "head", True), (591, 8, 4, 128, 128, True, 64, "bf16", "head", True),
    (600, 16, 1, 16, 16, True, 16, "fp16", "both", True), (800, 40, 1, 48, 0, False, 16, "bf16", "token", True),
])
def test_append_of_prompts(n, kv, group, dim, rot, pairs, page, kind, layout, weights):
    check_append(n, kv, group, dim, rot, pairs, page, kind, layout, weights)


def test_append_rotates_the_query_of_a_token_without_a_place():
    # a slot past the cache is one that writes nothing, as a negative slot is; a position past the angles is padding
    x = torch.randn(4, 2, 64, device="cuda", generator=_gen(2)).to(torch.bfloat16)
    kc, vc = _cache(2, 2, 16, 64, "bf16", fill=0.0), _cache(2, 2, 16, 64, "bf16", fill=0.0)
    rotary = torch.randn(4, 32, device="cuda", generator=_gen(3))
    places = [torch.tensor(s, device="cuda") for s in ([0, 1, 2, 3], [0, 32, -1, 3])]
    good = B.ivf_kv_append(x, x, x, kc, vc, _i32([0, 1, 2, 3]), places[0], rotary=rotary)
    B.ivf_check()
    got = B.ivf_kv_append(x, x, x, kc, vc, _i32([0, 1, 2, 4]), places[1], rotary=rotary)
    with pytest.raises(B.IvfError):
        B.ivf_check()
    assert torch.equal(got[:3], good[:3]) and (got[3] == 0).all()


# ---------------------------------------------------------------------------------------------- autograd

def test_forward_mode_tangents_are_refused():
    import torch.autograd.forward_ad as fwad
    kc, vc, table, req, pos, q, sel = _attend_case([40], 1, 1, 2, 64, 16, 2, "bf16", "head", seed=1)
    with fwad.dual_level():
        dual = fwad.make_dual(q, torch.ones_like(q))
        with pytest.raises(ValueError, match="gradient"):
            B.ivf_kv_attend(dual, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), 0.1)
        with pytest.raises(ValueError, match="gradient"):
            B.ivf_kv_summarize(fwad.make_dual(kc, torch.ones_like(kc)), _i32([0]), _i32([1]), torch.zeros(kc.shape[0], 1, 64, dtype=torch.int8, device="cuda"),
                               torch.zeros(kc.shape[0], 1, device="cuda"))


def test_tensors_written_in_place_count_a_version():
    kc, vc = _cache(4, 1, 16, 64, "bf16", fill=0.0), _cache(4, 1, 16, 64, "bf16", fill=0.0)
    table, x = torch.full((1, 4), -1, dtype=torch.int32, device="cuda"), torch.ones(3, 1, 64, device="cuda", dtype=torch.bfloat16)
    codes, scales = torch.zeros(4, 1, 64, dtype=torch.int8, device="cuda"), torch.zeros(4, 1, device="cuda")
    before = table._version
    plan = B.ivf_kv_tables(_i32([0]), _i32([3]), _i32([0, 1]), table, 16, 3)
    assert table._version > before
    old = [t._version for t in plan]
    B.ivf_kv_tables(_i32([0]), _i32([3]), _i32([0, 1]), table, 16, 3, plan=plan)
    assert all(t._version > v for t, v in zip(plan, old))
    q, old = torch.empty_like(x), (kc._version, vc._version)
    old_q = q._version
    B.ivf_kv_append(x, x, x, kc, vc, plan.token_pos, plan.token_slot, q_out=q)
    assert kc._version > old[0] and vc._version > old[1] and q._version > old_q
    old = (codes._version, scales._version, kc._version)
    B.ivf_kv_summarize(kc, plan.touched_page, plan.touched_fill, codes, scales)
    assert codes._version > old[0] and scales._version > old[1] and kc._version == old[2]
    sel = torch.empty(3, 1, 2, dtype=torch.int32, device="cuda")
    old = sel._version
    B.ivf_kv_select(q, codes, scales, table, plan.token_req, plan.token_pos, 16, 2, out=sel)
    assert sel._version > old
    out, old = torch.empty_like(q), q._version
    old_out = out._version
    B.ivf_kv_attend(q, kc, vc, table, plan.token_req, plan.token_pos, sel, 0.1, out=out)
    assert out._version > old_out and q._version == old
    B.ivf_check()
    with torch.inference_mode():  # its tensors count no versions
        y = torch.ones(3, 1, 64, device="cuda", dtype=torch.bfloat16)
        z = torch.empty_like(y)
    B.ivf_kv_append(y, y, y, kc, vc, plan.token_pos, plan.token_slot, q_out=z)
    B.ivf_check()


# ---------------------------------------------------------------------------------------------- axes of one element

def test_axes_of_one_element_may_carry_any_stride():
    # a table of one column cut out of a wider tensor crosswise, caches and queries of one head or token likewise
    n, dim = 5, 64
    kc, vc, table, req, pos, q, sel = _attend_case([16] * n, 1, 1, 1, dim, 16, 1, "bf16", "head", seed=4)
    one = _i32(table[:, :1])
    want, _ = B.ivf_kv_attend(q, kc, vc, one, _i32(req), _i32(pos), _i32(sel), 0.1)
    for odd in (torch.as_strided(one, (n, 1), (1, 7)), torch.as_strided(one, (n, 1), (1, 0))):
        got, _ = B.ivf_kv_attend(q, kc, vc, odd, _i32(req), _i32(pos), _i32(sel), 0.1)
        assert torch.equal(got, want)
        codes = torch.ones(kc.shape[0], 1, dim, dtype=torch.int8, device="cuda")
        ids = B.ivf_kv_select(q, codes, torch.ones(kc.shape[0], 1, device="cuda"), odd, _i32(req), _i32(pos), 16, 2)
        assert _np(ids)[:, 0].tolist() == [[0, -1]] * n
        plan = B.ivf_kv_tables(_i32([1] * n), _i32([1] * n), _i32([0]), odd, 16, n)
        assert _np(plan.token_slot).tolist() == [int(p) * 16 + 1 for p in table[:, 0]]
    wide = torch.zeros(n, 3, dim, dtype=q.dtype, device="cuda")
    wide[:, :1] = q
    got, _ = B.ivf_kv_attend(torch.as_strided(wide, (n, 1, dim), (3 * dim, 5, 1)), kc, vc, one, _i32(req), _i32(pos), _i32(sel), 0.1)
    assert torch.equal(got, want)
    B.ivf_check()


# ---------------------------------------------------------------------------------------------- the longest requests

@pytest.mark.parametrize("dim,fresh", [(64, 1), (128, 40)])
def test_positions_up_to_the_last_number(kernel, dim, fresh):  # noqa: F811
    # a request whose last token has position 2^31 - 1, in a table of 2^24 columns
    page, columns = 128, 1 << 24
    g = _gen(dim)
    kc, vc = (torch.randn(5, 1, page, dim, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    table = np.full((1, columns), -1, np.int32)
    blocks = [0, 7, columns // 2, columns - 2, columns - 1]
    table[0, blocks] = [3, 1, 4, 0, 2]
    pos = np.arange(2 ** 31 - fresh, 2 ** 31)
    req = np.zeros(fresh, np.int64)
    sel = np.tile(np.array(blocks)[None, None], (fresh, 1, 1))
    sel[::3, 0] = [0, 7, columns // 2, columns - 1, -1]
    q = torch.randn(fresh, 4, dim, device="cuda", generator=g).to(torch.bfloat16)
    _against_plain((kc, vc, table, req, pos, q, sel), 0.125, "bf16", dim)


# ---------------------------------------------------------------------------------------------- axes that are too long

def test_axes_past_32_bits_are_refused():
    # expanded, so that they cost no memory; cut to 32 bits the head count would be 4
    q = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda").expand(1, 2 ** 32 + 4, 64)
    codes, scales = torch.zeros(1, 4, 64, dtype=torch.int8, device="cuda"), torch.zeros(1, 4, device="cuda")
    with pytest.raises(ValueError, match="axis 1"):
        B.ivf_kv_select(q, codes, scales, _i32([[0]]), _i32([0]), _i32([0]), 16, 1)
    kc = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16, device="cuda").expand(1, 1, 2 ** 32 + 16, 64)
    with pytest.raises(ValueError, match="axis 2"):
        B.ivf_kv_summarize(kc, _i32([0]), _i32([1]), codes[:, :1].contiguous(), scales[:, :1].contiguous())
    B.ivf_check()
