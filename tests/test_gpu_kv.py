"""The block-cache operators against their plain 64-bit forms, through the binding.

Tolerances.  Outputs in a 16-bit type carry one rounding, u = 2^-8 (bf16) or 2^-11 (fp16) of the value.  append:
32-bit arithmetic before it, a few 2^-24 of the magnitudes that meet in an output: 2^-20 of them is allowed.
attend: the exponentials are rounded to the same type before the second product, at most u of the weighted mean
of |v|; a logit sums d exact products in 32 bits, at most d 2^-24 of their magnitudes, and moves its weight by as
much; 2^-20 covers exp2 and the final division.  Whole numbers are compared for equality."""
import math

import numpy as np
import pytest
import torch

import kv_reference as R
from paper_2608_08751_b200 import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _np(t):
    return t.detach().cpu().double().numpy() if t.is_floating_point() else t.detach().cpu().numpy().astype(np.int64)


def _i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ---------------------------------------------------------------------------------------------- tables

def _tables_case(lengths, page, columns, spare=5, seed=0, pad=3):
    cached, fresh = np.array(lengths, np.int64).T
    rng = np.random.default_rng(seed)
    held = [R.ceil_div(max(0, int(c)), page) for c in cached]
    need = sum(R.ceil_div(int(c + f), page) - R.ceil_div(int(c), page) for c, f in zip(cached, fresh) if c >= 0 and f >= 0)
    pages = rng.permutation(sum(held) + max(0, need) + max(0, spare)).astype(np.int64)
    table = rng.integers(0, 1000, (len(held), columns))  # what lies past the held pages is stale
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = pages[at: at + n][:columns]
        at += n
    free = pages[at: at + need + spare]
    tokens = int(max(0, fresh.clip(min=0).sum() + pad))
    return cached, fresh, free, table, tokens


def _run_tables(cached, fresh, free, table, tokens, page, touched=None, stride=0):
    t = _i32(table)
    if stride:
        wide = torch.full((t.shape[0], t.shape[1] + stride), 77, dtype=torch.int32, device="cuda")
        wide[:, : t.shape[1]] = t
        t = wide[:, : t.shape[1]]
    plan = B.ivf_kv_tables(_i32(cached), _i32(fresh), _i32(free), t, page, tokens, max_touched=touched)
    if stride:
        assert (wide[:, t.shape[1]:] == 77).all()
    return t, plan


def _same_tables(t, plan, want):
    assert (_np(t) == want["table"]).all()
    for name in ("kv_lens", "token_start", "token_req", "token_pos", "token_slot", "touched_page", "touched_fill"):
        assert (_np(getattr(plan, name)) == np.array(want[name])).all(), name
    assert int(plan.used) == want["used"]


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("lengths", [
    [(0, 1)], [(0, 0)], [(5, 0), (0, 0), (7, 1)], [(63, 1), (64, 1), (65, 1), (127, 2), (128, 0)],
    [(0, 300), (15, 17), (16, 16), (31, 1), (100, 1)], [(1, 1)] * 33, [(i * 13 % 200, i % 5) for i in range(700)],
])
def test_tables_equal_the_sequential_form(page, lengths):
    case = _tables_case(lengths, page, columns=24, seed=len(lengths) + page)
    cached, fresh, free, table, tokens = case
    touched = tokens // page + 2 * len(lengths)
    t, plan = _run_tables(*case, page, stride=len(lengths) % 3)
    B.ivf_check()
    want = R.tables(cached, fresh, page, free, table, tokens, touched)
    _same_tables(t, plan, want)
    # once more on the same arrays: the held entries were left alone, so nothing changes
    t2 = B.ivf_kv_tables(_i32(cached), _i32(fresh), _i32(free), t, page, tokens, plan=plan)
    _same_tables(t, t2, want)


@pytest.mark.parametrize("n", [4097, 16384])
def test_tables_of_many_requests(n):
    rng = np.random.default_rng(n)
    lengths = np.stack([rng.integers(0, 400, n), rng.integers(0, 3, n)], 1)
    case = _tables_case(lengths, 32, columns=13, seed=1)
    t, plan = _run_tables(*case, 32)
    B.ivf_check()
    _same_tables(t, plan, R.tables(case[0], case[1], 32, case[2], case[3], case[4], case[4] // 32 + 2 * n))


@pytest.mark.parametrize("what", ["pages", "columns", "tokens", "touched", "negative"])
def test_tables_shortages_are_cut_and_flagged(what):
    lengths = [(60, 10), (0, 200), (130, 3), (5, 64)]
    cached, fresh, free, table, tokens = _tables_case(lengths, 64, columns=6, spare=2)
    touched = tokens // 64 + 8
    code = B.IVF_ERR_NO_PAGES
    if what == "pages":
        free = free[:3]
    elif what == "columns":
        table = table[:, :3]
    elif what == "tokens":
        tokens = 150
    elif what == "touched":
        touched = 3
    else:
        cached[2], fresh[3], code = -4, -1, B.IVF_ERR_BAD_ID
    t, plan = _run_tables(cached, fresh, free, table, tokens, 64, touched=touched)
    with pytest.raises(B.IvfError) as e:
        B.ivf_check()
    assert e.value.code == code and "ivf_kv_tables" in str(e.value)
    _same_tables(t, plan, R.tables(cached, fresh, 64, free, table, tokens, touched))


def test_tables_of_no_request():
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    plan = B.ivf_kv_tables(none, none, none, torch.zeros(0, 4, dtype=torch.int32, device="cuda"), 16, 3)
    B.ivf_check()
    assert _np(plan.token_start).tolist() == [0] and int(plan.used) == 0 and (plan.token_slot == -1).all() and (plan.token_req == -1).all()


# ---------------------------------------------------------------------------------------------- append

def _cache(pages, heads, page, dim, kind, layout="head", fill=math.nan):
    if layout == "token":  # [pages, page, heads, d] in memory
        return torch.full((pages, page, heads, dim), fill, dtype=TYPES[kind], device="cuda").transpose(1, 2)
    if layout == "both":  # keys and values of a page side by side, rows with a gap
        return torch.full((pages, 2, heads, page, dim + 8), fill, dtype=TYPES[kind], device="cuda")[:, 1, :, :, :dim]
    return torch.full((pages, heads, page, dim), fill, dtype=TYPES[kind], device="cuda")


APPEND = [
    # tokens, kv_heads, group, dim, rot, interleaved, page, type, layout, weights
    (1, 1, 1, 16, 16, False, 16, "bf16", "head", True), (3, 2, 4, 64, 64, False, 16, "fp16", "token", True),
    (37, 4, 7, 96, 64, True, 32, "fp16", "head", True), (130, 8, 4, 128, 128, False, 64, "bf16", "both", True),
    (5, 3, 5, 80, 32, True, 128, "bf16", "token", False), (9, 1, 16, 256, 128, False, 64, "fp16", "both", True),
    (17, 2, 3, 48, 48, False, 16, "bf16", "head", True), (6, 2, 1, 112, 0, False, 32, "fp16", "head", True),
    (4, 1, 2, 256, 256, True, 16, "bf16", "token", False), (600, 2, 2, 32, 32, False, 128, "fp16", "head", True),
]


@pytest.mark.parametrize("n,kv,group,dim,rot,pairs,page,kind,layout,weights", APPEND)
def test_append_matches_the_formula(n, kv, group, dim, rot, pairs, page, kind, layout, weights):
    g = _gen(n + dim)
    heads = kv * group
    qkv = (torch.randn(n, (heads + 2 * kv) * dim + 8, device="cuda", generator=g) * 3).to(TYPES[kind])
    q, k, v = (x.view(n, -1, dim) for x in qkv[:, : (heads + 2 * kv) * dim].split([heads * dim, kv * dim, kv * dim], 1))
    pages = R.ceil_div(n, page) + 2
    kc, vc = _cache(pages, kv, page, dim, kind, layout), _cache(pages, kv, page, dim, kind, layout)
    slots = torch.randperm(pages * page, device="cuda", generator=g)[:n]
    pos = torch.randint(0, 50, (n,), device="cuda", generator=g).to(torch.int32)
    if n > 4:
        pos[2], slots[3] = -1, -1  # a padded token; one that is not written
    rotary = torch.randn(50, rot, device="cuda", generator=g) if rot else None
    qw, kw = (1 + 0.2 * torch.randn(dim, device="cuda", generator=g) if weights else None for _ in range(2))
    got = B.ivf_kv_append(q, k, v, kc, vc, pos, slots, rotary=rotary, interleaved=pairs, q_weight=qw, k_weight=kw, eps=1e-5)
    B.ivf_check()
    npos, nslot = _np(pos).clip(min=0), _np(slots)
    w = (None, None) if not weights else (_np(qw), _np(kw))
    rt = None if rotary is None else _np(rotary)
    live = _np(pos) >= 0
    want, mag = R.turned(_np(q), w[0], 1e-5, rt, npos, pairs)
    want[~live], mag[~live] = 0, 0
    assert (np.abs(_np(got) - want) <= R.UNIT[kind] * np.abs(want) + 2.0 ** -20 * mag + R.TINY[kind]).all()
    wk, mk = R.turned(_np(k), w[1], 1e-5, rt, npos, pairs)
    ck, cv = _np(kc), _np(vc)
    written = np.zeros((pages, page), bool)
    for t in range(n):
        if live[t] and nslot[t] >= 0:
            at, off = divmod(int(nslot[t]), page)
            written[at, off] = True
            assert (np.abs(ck[at, :, off] - wk[t]) <= R.UNIT[kind] * np.abs(wk[t]) + 2.0 ** -20 * mk[t] + R.TINY[kind]).all()
            assert (cv[at, :, off] == _np(v)[t]).all()
    assert np.isnan(ck.transpose(0, 2, 1, 3)[~written]).all() and np.isnan(cv.transpose(0, 2, 1, 3)[~written]).all()
    # in place: the same numbers
    again = qkv.clone()
    q2, k2, v2 = (x.view(n, -1, dim) for x in again[:, : (heads + 2 * kv) * dim].split([heads * dim, kv * dim, kv * dim], 1))
    same = B.ivf_kv_append(q2, k2, v2, kc, vc, pos, slots, rotary=rotary, interleaved=pairs, q_weight=qw, k_weight=kw, eps=1e-5, q_out=q2)
    assert same.data_ptr() == q2.data_ptr() and torch.equal(same, got)


def test_append_zero_rows_infinities_and_bad_places():
    n, d = 6, 64
    x = torch.zeros(n, 1, d, device="cuda", dtype=torch.bfloat16)
    x[1, 0, 40] = math.inf  # past the rotated part: stays where it is
    kc, vc = _cache(2, 1, 16, d, "bf16", fill=0.0), _cache(2, 1, 16, d, "bf16", fill=0.0)
    rotary = torch.ones(4, 32, device="cuda")
    out = B.ivf_kv_append(x, x, x, kc, vc, _i32([0, 1, 2, 3, 0, 1]), torch.arange(n, device="cuda"), rotary=rotary)
    B.ivf_check()
    assert torch.equal(out, x) and torch.equal(kc[0, 0, :n], x[:, 0])
    w = torch.ones(d, device="cuda")
    out = B.ivf_kv_append(x[:1], x[:1], x[:1], kc, vc, _i32([0]), torch.zeros(1, device="cuda", dtype=torch.int64), rotary=rotary, q_weight=w, k_weight=w)
    B.ivf_check()
    assert (out == 0).all()  # a zero row has the norm sqrt(eps)
    x[:] = 1
    before = kc.clone()
    out = B.ivf_kv_append(x, x, x, kc, vc, _i32([4, 0, 0, -2, 9, 1]), torch.tensor([0, 32, 1 << 40, 3, 4, -5], device="cuda"), rotary=rotary)
    with pytest.raises(B.IvfError) as e:
        B.ivf_check()
    assert e.value.code == B.IVF_ERR_BAD_ID and "ivf_kv_append" in str(e.value)
    assert torch.equal(kc, before)  # positions and slots past their ranges write nothing
    assert (out[[0, 3, 4]] == 0).all() and (out[[1, 2, 5]] != 0).any()


# ---------------------------------------------------------------------------------------------- summarize

@pytest.mark.parametrize("kv,dim,page,kind,layout", [
    (1, 16, 16, "bf16", "head"), (2, 32, 32, "fp16", "token"), (3, 64, 128, "bf16", "both"), (8, 128, 64, "bf16", "head"),
    (4, 96, 16, "fp16", "head"), (2, 80, 32, "bf16", "token"), (1, 256, 128, "fp16", "head"), (5, 192, 64, "bf16", "both"),
])
def test_summaries_are_the_same_whole_numbers(kv, dim, page, kind, layout):
    g = _gen(dim + page)
    n = 40
    kc = _cache(n, kv, page, dim, kind, layout)
    fills = [1, page, page - 1, 2, page // 2 + 1] * 7
    pages = np.random.default_rng(dim).permutation(n)[: len(fills)].copy()
    for p, f in zip(pages, fills):  # what lies past the fill stays NaN
        kc[int(p), :, :f] = (torch.randn(kv, f, dim, device="cuda", generator=g) * 2).to(TYPES[kind])
    kc[int(pages[1])] = 0  # a page of zeros
    if kind == "bf16":
        kc[int(pages[6])] = 1e-38  # a scale below the normal numbers
    codes = torch.full((n, kv, dim), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((n, kv), 5.0, device="cuda")
    B.ivf_kv_summarize(kc, _i32(list(pages) + [-1, 3]), _i32(fills + [7, 0]), codes, scales)  # two padded entries
    B.ivf_check()
    c, s, keys = _np(codes), scales.cpu().numpy(), _np(kc)
    for p, f in zip(pages, fills):
        want, unit, mean = R.summary(keys[p], f)
        assert (c[p] == want).all() and (s[p] == unit).all()
        # against 64 bits: half a step and the 32-bit sum's rounding
        assert (np.abs(c[p] * s[p].astype(np.float64)[:, None] - mean) <= (0.5 + 1e-4) * s[p].astype(np.float64)[:, None] + 2e-38).all()
    rest = np.setdiff1d(np.arange(n), pages)
    assert (c[rest] == 99).all() and (s[rest] == 5).all()


def test_summaries_refuse_pages_and_fills_out_of_range():
    kc = _cache(4, 2, 16, 32, "bf16", fill=1.0)
    codes, scales = torch.zeros(4, 2, 32, dtype=torch.int8, device="cuda"), torch.zeros(4, 2, device="cuda")
    for pages, fills in (([4, 1], [3, 2]), ([-2, 1], [3, 2]), ([0, 1], [17, 2]), ([0, 1], [-1, 2])):
        codes.zero_()
        B.ivf_kv_summarize(kc, _i32(pages), _i32(fills), codes, scales)
        with pytest.raises(B.IvfError) as e:
            B.ivf_check()
        assert e.value.code == B.IVF_ERR_BAD_ID and "ivf_kv_summarize" in str(e.value)
        assert (codes[1] == 127).all() and (codes[[0, 2, 3]] == 0).all()


# ---------------------------------------------------------------------------------------------- select

def _request_table(blocks, pages, seed, columns=None):
    rng = np.random.default_rng(seed)
    order = rng.permutation(pages)
    columns = columns or max(blocks) + 2
    table, at = np.full((len(blocks), columns), -1, np.int64), 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at: at + n]
        at += n
    return table


@pytest.fixture(params=["by size", "single tokens", "windows"])
def select_kernel(request):
    """Every selection test runs with the kernel chosen by the sizes and with either forced."""
    B.ivf_debug_set_kv_select(["by size", "single tokens", "windows"].index(request.param))
    yield request.param
    B.ivf_debug_set_kv_select(0)


SELECT = [
    # contexts, fresh, kv, group, dim, page, take, first, last, type
    ([1], 1, 1, 1, 16, 16, 1, 0, 1, "bf16"), ([17], 3, 2, 3, 64, 16, 2, 0, 1, "fp16"), ([1000, 1, 64, 65], 1, 2, 4, 128, 16, 8, 1, 2, "bf16"),
    ([900, 500], 40, 2, 2, 96, 32, 5, 1, 1, "fp16"), ([5000], 70, 1, 8, 80, 16, 64, 2, 3, "bf16"), ([4096, 4000], 7, 1, 16, 256, 128, 17, 0, 2, "bf16"),
    ([2000], 33, 3, 5, 48, 16, 31, 31, 1, "fp16"), ([40000], 2, 1, 7, 128, 16, 1024, 1, 1, "bf16"), ([700, 30, 3, 900], 20, 4, 1, 64, 64, 4, 1, 3, "bf16"),
    ([3000] * 3, 16, 1, 64, 32, 32, 12, 0, 1, "fp16"), ([300], 130, 1, 20, 128, 64, 3, 0, 3, "bf16"),
]


def _step(contexts, fresh):
    req = np.concatenate([np.full(min(fresh, c), b) for b, c in enumerate(contexts)])
    pos = np.concatenate([np.arange(c - min(fresh, c), c) for c in contexts])
    return req, pos


@pytest.mark.parametrize("contexts,fresh,kv,group,dim,page,take,first,last,kind", SELECT)
def test_selection_equals_the_plain_form(select_kernel, contexts, fresh, kv, group, dim, page, take, first, last, kind):
    if first + last > take:
        first = take - last
    g = _gen(dim + take)
    blocks = [R.ceil_div(c, page) for c in contexts]
    pages = sum(blocks) + 3
    table = _request_table(blocks, pages, take)
    req, pos = _step(contexts, fresh)
    n = len(req)
    wide = torch.randn(n, kv * group + 1, dim, device="cuda", generator=g).to(TYPES[kind])
    q = wide[:, 1:]
    codes = torch.randint(-127, 128, (pages, kv, dim), device="cuda", generator=g).to(torch.int8)
    scales = torch.rand(pages, kv, device="cuda", generator=g) + 0.1
    if n > 2:
        req[1] = -1
    if blocks[0] > 6:
        table[0, 4] = -1  # a missing page is not visible
    got = B.ivf_kv_select(q, codes, scales, _i32(table), _i32(req), _i32(pos), page, take, n_first=first, n_last=last)
    B.ivf_check()
    want = R.select(_np(q), _np(codes), scales.cpu().numpy(), table, req, pos, page, take, first, last)
    assert (_np(got) == want).all()
    again = B.ivf_kv_select(q, codes, scales, _i32(table), _i32(req), _i32(pos), page, take, n_first=first, n_last=last)
    assert torch.equal(got, again)


@pytest.mark.parametrize("n_blocks,take", [(50, 8), (700, 64), (5000, 33), (20000, 1000)])
@pytest.mark.parametrize("fresh", [1, 20])
def test_ties_go_to_the_lower_block(select_kernel, n_blocks, take, fresh):
    # few distinct scores: nearly every place in the list is decided by the tie rule; zero scales of both signs too
    g = _gen(n_blocks)
    page, dim = 16, 32
    table = _request_table([n_blocks], n_blocks, 5)
    codes = torch.randint(-1, 2, (n_blocks, 1, dim), device="cuda", generator=g).to(torch.int8)
    codes[:, :, 4:] = 0
    scales = torch.ones(n_blocks, 1, device="cuda")
    scales[::7] = 0.0
    scales[3::7] = -0.0
    q = torch.randint(-2, 3, (fresh, 1, dim), device="cuda", generator=g).to(torch.bfloat16)
    q[0] = 0  # no preference at all
    req, pos = np.zeros(fresh, np.int64), np.arange(n_blocks * page - fresh, n_blocks * page)
    got = B.ivf_kv_select(q, codes, scales, _i32(table), _i32(req), _i32(pos), page, take, n_first=0, n_last=1)
    B.ivf_check()
    want = R.select(_np(q), _np(codes), scales.cpu().numpy(), table, req, pos, page, take, 0, 1)
    assert (_np(got) == want).all()
    assert (_np(got)[0, 0] == list(range(take - 1)) + [pos[0] // page]).all()


def test_selection_skips_what_is_out_of_range(select_kernel):
    codes, scales = torch.ones(8, 1, 32, dtype=torch.int8, device="cuda"), torch.ones(8, 1, device="cuda")
    q = torch.ones(4, 1, 32, device="cuda", dtype=torch.bfloat16)
    table = np.array([[0, 1, 2, 8, 3], [4, 5, -1, -1, -1]])
    got = B.ivf_kv_select(q, codes, scales, _i32(table), _i32([0, 2, 1, 0]), _i32([79, 5, 31, 80]), 16, 4, n_first=1, n_last=1)
    with pytest.raises(B.IvfError) as e:
        B.ivf_check()
    assert e.value.code == B.IVF_ERR_BAD_ID and "ivf_kv_select" in str(e.value)
    assert _np(got)[:, 0].tolist() == [[0, 1, 2, 4], [-1] * 4, [0, 1, -1, -1], [-1] * 4]
    scales[:] = math.nan  # scores without a value: some choice, in range and ascending
    got = _np(B.ivf_kv_select(q[:1], codes, scales, _i32(np.ascontiguousarray(table[:, [0, 1, 2, 4, 4]])), _i32([0]), _i32([79]), 16, 3))
    assert (np.diff(got[0, 0]) > 0).all() and got.min() >= 0 and got.max() <= 4
    B.ivf_check()


# ---------------------------------------------------------------------------------------------- attend

@pytest.fixture(params=["by size", "single tokens", "windows"])
def kernel(request):
    """Every attention test runs with the kernel chosen by the sizes and with either forced."""
    B.ivf_debug_set_kv_attend(["by size", "single tokens", "windows"].index(request.param))
    yield request.param
    B.ivf_debug_set_kv_attend(0)


def _attend_case(contexts, fresh, kv, group, dim, page, take, kind, layout, seed, forced_last=True, shared=False):
    """Caches whose places past a request's end hold NaN, and a random ascending selection for each token."""
    g = _gen(seed)
    rng = np.random.default_rng(seed)
    blocks = [R.ceil_div(c, page) for c in contexts]
    pages = sum(blocks) + 2
    table = _request_table(blocks, pages, seed)
    kc, vc = _cache(pages, kv, page, dim, kind, layout), _cache(pages, kv, page, dim, kind, layout)
    for b, c in enumerate(contexts):
        for j in range(blocks[b]):
            fill = min(page, c - j * page)
            for plane in (kc, vc):
                plane[int(table[b, j]), :, :fill] = torch.randn(kv, fill, dim, device="cuda", generator=g).to(TYPES[kind])
    req, pos = _step(contexts, fresh)
    n = len(req)
    q = (torch.randn(n, kv * group, dim, device="cuda", generator=g) * 2).to(TYPES[kind])
    sel = np.full((n, kv, take), -1, np.int64)
    for t in range(n):
        last = pos[t] // page
        for h in range(kv):
            pool = np.arange(last + 1)
            if shared and len(pool) > take:  # neighbours want much the same
                pool = np.unique(np.concatenate([pool[: take], rng.choice(pool, 2), [last]]))
            pick = rng.choice(pool, min(take, len(pool)), replace=False)
            if forced_last and last not in pick:
                pick[0] = last
            sel[t, h, : len(pick)] = np.sort(pick)
    return kc, vc, table, req, pos, q, sel


def _check_attend(got, lse, want, kind, dim):
    out, wl, size, unit = want
    u = R.UNIT[kind]
    near = dim * 2.0 ** -24 * unit
    tol = u * (np.abs(out) + size) + (2 * near[..., None] + 2.0 ** -20) * size + R.TINY[kind]
    d = np.abs(_np(got) - out)
    assert np.isfinite(d).all() and (d <= tol).all(), (d / tol).max()
    if lse is not None:
        x = _np(lse)
        none = np.isinf(wl)
        assert (x[none] == -np.inf).all() and np.isfinite(x[~none]).all()
        assert (np.abs(x[~none] - wl[~none]) <= near[~none] + 2.0 ** -20 * (1 + np.abs(wl[~none]))).all()


ATTEND = [
    # contexts, fresh, kv, group, dim, page, take, type, layout
    ([1], 1, 1, 1, 16, 16, 1, "bf16", "head"), ([1, 16, 17, 15], 1, 2, 2, 64, 16, 3, "fp16", "token"), ([700], 1, 1, 7, 96, 64, 5, "fp16", "head"),
    ([2000, 3, 900, 64], 1, 8, 4, 128, 64, 9, "bf16", "head"), ([130, 257], 5, 2, 16, 80, 32, 4, "bf16", "both"), ([500], 3, 1, 20, 128, 16, 12, "fp16", "token"),
    ([300, 40], 2, 2, 3, 256, 32, 6, "bf16", "head"), ([260], 4, 1, 64, 192, 128, 2, "fp16", "both"), ([4000], 1, 1, 5, 48, 16, 100, "bf16", "head"),
    ([600], 1, 2, 8, 112, 128, 3, "bf16", "token"), ([20000], 1, 1, 4, 128, 16, 1024, "bf16", "head"),
]


@pytest.mark.parametrize("contexts,fresh,kv,group,dim,page,take,kind,layout", ATTEND)
def test_attention_of_single_and_drafted_tokens(kernel, contexts, fresh, kv, group, dim, page, take, kind, layout):
    kc, vc, table, req, pos, q, sel = _attend_case(contexts, fresh, kv, group, dim, page, take, kind, layout, seed=dim + take)
    scale = 1 / math.sqrt(dim)
    got, lse = B.ivf_kv_attend(q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), scale, want_lse=True)
    B.ivf_check()
    want = R.attend(_np(q), np.nan_to_num(_np(kc)), np.nan_to_num(_np(vc)), table, req, pos, sel, scale)
    _check_attend(got, lse, want, kind, dim)
    again, _ = B.ivf_kv_attend(q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), scale)
    assert torch.equal(got, again)


PROMPT = [
    # contexts, fresh, kv, group, dim, page, take, type, layout, shared
    ([300], 300, 1, 4, 128, 64, 3, "bf16", "head", False), ([900, 50], 120, 2, 8, 128, 64, 4, "bf16", "head", True),
    ([500], 200, 1, 1, 64, 16, 6, "fp16", "token", True), ([333, 77, 260], 77, 2, 3, 96, 32, 4, "fp16", "both", False),
    ([1500], 90, 1, 16, 128, 128, 3, "bf16", "head", True), ([400, 401], 129, 1, 5, 80, 64, 3, "bf16", "token", False),
    ([300], 64, 1, 7, 256, 32, 4, "bf16", "head", True), ([260], 80, 1, 20, 64, 16, 5, "fp16", "head", False),
    ([700] * 9, 17, 1, 8, 128, 64, 5, "bf16", "head", True), ([200], 40, 1, 64, 128, 64, 2, "bf16", "head", False),
    ([150], 150, 1, 2, 16, 16, 4, "fp16", "head", False),
    # several requests in a window, pages of two boxes whose last half is empty
    ([704, 190, 333], 61, 2, 7, 64, 128, 4, "fp16", "head", True), ([300, 420, 1000], 50, 1, 1, 128, 128, 3, "bf16", "token", True),
    ([130, 270], 40, 1, 4, 256, 128, 2, "bf16", "both", False),
]


@pytest.mark.parametrize("contexts,fresh,kv,group,dim,page,take,kind,layout,shared", PROMPT)
def test_attention_of_prompt_chunks(kernel, contexts, fresh, kv, group, dim, page, take, kind, layout, shared):
    kc, vc, table, req, pos, q, sel = _attend_case(contexts, fresh, kv, group, dim, page, take, kind, layout, seed=dim + take + 1, shared=shared)
    scale = 1 / math.sqrt(dim)
    got, lse = B.ivf_kv_attend(q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), scale, want_lse=True)
    B.ivf_check()
    want = R.attend(_np(q), np.nan_to_num(_np(kc)), np.nan_to_num(_np(vc)), table, req, pos, sel, scale)
    _check_attend(got, lse, want, kind, dim)
    again, _ = B.ivf_kv_attend(q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), scale)
    assert torch.equal(got, again)


@pytest.mark.parametrize("fresh", [1, 70])
@pytest.mark.parametrize("dim,kind", [(64, "fp16"), (128, "bf16"), (256, "bf16")])
def test_attention_rows_that_see_nothing_and_odd_selections(kernel, fresh, dim, kind):
    kc, vc, table, req, pos, q, sel = _attend_case([600, 333, 90], fresh, 2, 4, dim, 32, 5, kind, "head", seed=fresh)
    n = len(req)
    sel[0] = -1                     # nothing selected
    if n > 4:
        sel[1, 0] = -1              # ... for one kv head
        req[2] = -1                 # padding
        pos[3] = -1
        sel[n - 1] = np.array([0, 1, 40, 41, 50])  # blocks past the token's own are ignored
        sel[4] = np.array([0, -1, -1, -1, -1])
    scale = 0.3
    got, lse = B.ivf_kv_attend(q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), scale, want_lse=True)
    B.ivf_check()
    seen = np.where(sel * 32 <= pos[:, None, None], sel, -1)
    want = R.attend(_np(q), np.nan_to_num(_np(kc)), np.nan_to_num(_np(vc)), table, req, pos, seen, scale)
    _check_attend(got, lse, want, kind, dim)
    assert (got[0] == 0).all()


@pytest.mark.parametrize("fresh", [1, 48])
def test_attention_with_large_and_equal_logits(kernel, fresh):
    # logits of several hundred (one key takes all), then all equal (the mean of the values): no overflow, no drift
    kc, vc, table, req, pos, q, sel = _attend_case([900], fresh, 1, 8, 128, 64, 6, "bf16", "head", seed=9)
    for scale in (30.0, -30.0, 0.0):
        got, lse = B.ivf_kv_attend(q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), scale, want_lse=True)
        B.ivf_check()
        want = R.attend(_np(q), np.nan_to_num(_np(kc)), np.nan_to_num(_np(vc)), table, req, pos, sel, scale)
        _check_attend(got, lse, want, "bf16", 128)


@pytest.mark.parametrize("fresh", [1, 64])
def test_values_of_tokens_that_are_not_seen_may_be_anything(kernel, fresh):
    # infinities and NaN in blocks that a token did not select, and at positions after its own: other tokens of
    # the same tile read those blocks, this one must not notice
    kc, vc, table, req, pos, q, sel = _attend_case([640], fresh, 1, 4, 128, 64, 4, "bf16", "head", seed=31)
    n = len(req)
    sel[:, 0] = np.array([0, 3, 5, 9])
    if n > 1:
        sel[1::2, 0] = np.array([0, 2, 5, 9])
    bad = int(table[0, 9])
    k0, v0 = kc.clone(), vc.clone()
    vc[bad, 0, 63] = math.nan  # the last token's own value: earlier tokens do not see it
    kc[bad, 0, 62] = math.inf
    vc[int(table[0, 3]), 0, 7] = math.inf  # only even tokens selected it
    got, _ = B.ivf_kv_attend(q, kc, vc, _i32(table), _i32(req), _i32(pos), _i32(sel), 0.1)
    clean, _ = B.ivf_kv_attend(q, k0, v0, _i32(table), _i32(req), _i32(pos), _i32(sel), 0.1)
    B.ivf_check()
    untouched = [t for t in range(n) if t % 2 == 1 and pos[t] < 638]
    if untouched:
        want = R.attend(_np(q), np.nan_to_num(_np(k0)), np.nan_to_num(_np(v0)), table, req, pos, sel, 0.1)
        part = tuple(w[untouched] for w in want)
        _check_attend(got[untouched], None, part, "bf16", 128)
        _check_attend(clean[untouched], None, part, "bf16", 128)


def test_attention_refuses_what_is_out_of_range(kernel):
    kc, vc, table, req, pos, q, sel = _attend_case([100, 100], 1, 1, 2, 64, 16, 3, "bf16", "head", seed=2)
    bad = table.copy()
    bad[0, sel[0, 0, 0]] = 10000  # a page past the cache: its block is left out
    got, _ = B.ivf_kv_attend(q, kc, vc, _i32(bad), _i32(req), _i32(pos), _i32(sel), 0.2)
    with pytest.raises(B.IvfError) as e:
        B.ivf_check()
    assert e.value.code == B.IVF_ERR_BAD_ID and "ivf_kv_attend" in str(e.value)
    less = sel.copy()
    less[0, 0] = [less[0, 0, 1], less[0, 0, 2], -1]
    want = R.attend(_np(q), np.nan_to_num(_np(kc)), np.nan_to_num(_np(vc)), table, req, pos, less, 0.2)
    _check_attend(got, None, want, "bf16", 64)
    got, _ = B.ivf_kv_attend(q, kc, vc, _i32(table), _i32([0, 2]), _i32(pos), _i32(sel), 0.2)
    with pytest.raises(B.IvfError):
        B.ivf_check()
    assert (got[1] == 0).all()


def test_offsets_past_32_bits(kernel):
    # pages that start 2^31 elements into the cache and further
    page, dim, kv = 128, 128, 1
    pages = (1 << 31) // (page * dim) + 8
    kc = torch.empty(pages, kv, page, dim, dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    far = [pages - 1, pages - 5, 1, pages - 3]
    g = _gen(4)
    n = 400
    q, k, v = (torch.randn(n, h, dim, device="cuda", generator=g).to(torch.bfloat16) for h in (4, 1, 1))
    plan = B.ivf_kv_tables(_i32([0]), _i32([n]), _i32(far), torch.empty(1, 4, dtype=torch.int32, device="cuda"), page, n)
    table = _i32([far])
    qr = B.ivf_kv_append(q, k, v, kc, vc, plan.token_pos, plan.token_slot)
    codes, scales = torch.empty(pages, kv, dim, dtype=torch.int8, device="cuda"), torch.empty(pages, kv, device="cuda")
    B.ivf_kv_summarize(kc, plan.touched_page, plan.touched_fill, codes, scales)
    sel = B.ivf_kv_select(qr, codes, scales, table, plan.token_req, plan.token_pos, page, 3)
    out, lse = B.ivf_kv_attend(qr, kc, vc, table, plan.token_req, plan.token_pos, sel, 0.1, want_lse=True)
    B.ivf_check()
    small_k, small_v = (np.zeros((4, 1, page, dim)) for _ in range(2))
    small_k.transpose(0, 2, 1, 3).reshape(-1, 1, dim)[:n], small_v.transpose(0, 2, 1, 3).reshape(-1, 1, dim)[:n] = _np(k), _np(v)
    req, pos, tab = np.zeros(n, np.int64), np.arange(n), np.arange(4)[None]
    c, s = np.zeros((4, 1, dim), np.int64), np.zeros((4, 1), np.float32)
    for j in range(4):
        c[j], s[j], _ = R.summary(small_k[j], min(page, n - j * page))
    want_sel = R.select(_np(q), c, s, tab, req, pos, page, 3, 1, 1)
    assert (_np(sel) == want_sel).all()
    _check_attend(out, lse, R.attend(_np(q), small_k, small_v, tab, req, pos, want_sel, 0.1), "bf16", dim)


# ---------------------------------------------------------------------------------------------- the step as a whole

def _whole_step(stream_device, q, k, v, state):
    cached, fresh, free, table, kc, vc, codes, scales, rotary, w, tokens = state
    plan = B.ivf_kv_tables(cached, fresh, free, table, 32, tokens)
    qr = B.ivf_kv_append(q, k, v, kc, vc, plan.token_pos, plan.token_slot, rotary=rotary, q_weight=w, k_weight=w)
    B.ivf_kv_summarize(kc, plan.touched_page, plan.touched_fill, codes, scales)
    sel = B.ivf_kv_select(qr, codes, scales, table, plan.token_req, plan.token_pos, 32, 4)
    out, lse = B.ivf_kv_attend(qr, kc, vc, table, plan.token_req, plan.token_pos, sel, 0.125, want_lse=True)
    return plan, qr, sel, out, lse


def _whole_state(seed, lengths, tokens, dim=64, kv=2, heads=6):
    g = _gen(seed)
    pages = 64
    table = torch.full((len(lengths), 16), -1, dtype=torch.int32, device="cuda")
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    at = 0
    for b, (c, _) in enumerate(lengths):
        n = R.ceil_div(c, 32)
        table[b, :n] = order[at: at + n]
        at += n
    kc = torch.randn(pages, kv, 32, dim, device="cuda", generator=g).to(torch.bfloat16)
    vc = torch.randn(pages, kv, 32, dim, device="cuda", generator=g).to(torch.bfloat16)
    codes, scales = torch.empty(pages, kv, dim, dtype=torch.int8, device="cuda"), torch.empty(pages, kv, device="cuda")
    B.ivf_kv_summarize(kc, _i32(range(pages)), _i32([32] * pages), codes, scales)
    qkv = [torch.randn(tokens, h, dim, device="cuda", generator=g).to(torch.bfloat16) for h in (heads, kv, kv)]
    state = (_i32([c for c, _ in lengths]), _i32([f for _, f in lengths]), order[at:].contiguous(), table, kc, vc, codes, scales,
             torch.randn(512, dim, device="cuda", generator=g), 1 + 0.1 * torch.randn(dim, device="cuda", generator=g), tokens)
    return qkv, state


LENGTHS = [(100, 1), (31, 1), (32, 1), (0, 20), (333, 1), (64, 0)]


def test_the_five_calls_as_one_step(kernel):
    qkv, state = _whole_state(1, LENGTHS, 27)  # 24 tokens and padding
    plan, qr, sel, out, lse = _whole_step(None, *qkv, state)
    B.ivf_check()
    req, pos, table = _np(plan.token_req), _np(plan.token_pos), _np(state[3])
    kc, vc = _np(state[4]), _np(state[5])
    want_sel = R.select(_np(qr), _np(state[6]), state[7].cpu().numpy(), table, req, pos, 32, 4, 1, 1)
    assert (_np(sel) == want_sel).all() and (req[24:] == -1).all()
    _check_attend(out, lse, R.attend(_np(qr), kc, vc, table, req, pos, want_sel, 0.125), "bf16", 64)
    for p, f in zip(_np(plan.touched_page), _np(plan.touched_fill)):
        if p >= 0:
            c, s, _ = R.summary(kc[p], f)
            assert (c == _np(state[6])[p]).all() and (s == state[7].cpu().numpy()[p]).all()


def test_another_stream_and_a_captured_graph_give_the_same(kernel):
    qkv, state = _whole_state(2, LENGTHS, 27)
    first = [t.clone() for t in _whole_step(None, *qkv, state)[1:]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = _whole_step(None, *qkv, state)[1:]
    side.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = _whole_step(None, *qkv, state)[1:]
    for t in third:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(first, third):
        assert torch.equal(a, b)
    # new lengths and queries in the same arrays: what the graph computes follows
    qkv[0].mul_(-1)
    state[0][0] = 40
    graph.replay()
    want = _whole_step(None, *qkv, state)[1:]
    for a, b in zip(want, third):
        assert torch.equal(a, b)
    B.ivf_check()


def test_binding_refuses_mismatched_tensors():
    qkv, state = _whole_state(3, LENGTHS, 27)
    kc, vc = state[4], state[5]
    pos, slot = _i32([0] * 27), torch.zeros(27, dtype=torch.int64, device="cuda")
    q, k, v = qkv
    with pytest.raises(ValueError):
        B.ivf_kv_append(q, k[:, :1], v, kc, vc, pos, slot)
    with pytest.raises(ValueError):
        B.ivf_kv_append(q, k, v, kc, vc.half(), pos, slot)
    with pytest.raises(ValueError):
        B.ivf_kv_append(q, k, v, kc, vc, pos.long(), slot)
    with pytest.raises(ValueError):
        B.ivf_kv_append(q.cpu(), k, v, kc, vc, pos, slot)
    with pytest.raises(TypeError):
        B.ivf_kv_append(q.float(), k.float(), v.float(), kc.float(), vc.float(), pos, slot)
    with pytest.raises(ValueError):
        B.ivf_kv_summarize(kc, pos, pos, state[6][:3], state[7])
    with pytest.raises(ValueError):
        B.ivf_kv_attend(q, kc, vc, state[3], pos, pos, torch.zeros(27, 1, 4, dtype=torch.int32, device="cuda"), 1.0)
    with pytest.raises(ValueError):
        B.ivf_kv_attend(q.transpose(1, 2), kc, vc, state[3], pos, pos, torch.zeros(27, 2, 4, dtype=torch.int32, device="cuda"), 1.0)
    with pytest.raises(B.IvfError):  # strides that are no multiple of 16 bytes
        wide = torch.zeros(27, 6, 65, dtype=torch.bfloat16, device="cuda")[..., :64]
        B.ivf_kv_attend(wide, kc, vc, state[3], pos, pos, torch.zeros(27, 2, 4, dtype=torch.int32, device="cuda"), 1.0)
    with pytest.raises(B.IvfError):
        B.ivf_kv_attend(q, kc, vc, state[3], pos, pos, torch.zeros(27, 2, 4, dtype=torch.int32, device="cuda"), math.nan)
    with pytest.raises(ValueError):  # no gradients are computed: said, not dropped
        B.ivf_kv_attend(q.clone().requires_grad_(), kc, vc, state[3], pos, pos, torch.zeros(27, 2, 4, dtype=torch.int32, device="cuda"), 1.0)
    with pytest.raises(TypeError):
        B.ivf_kv_summarize(kc, [1], pos, state[6], state[7])
    empty = B.ivf_kv_attend(q[:0], kc, vc, state[3], pos[:0], pos[:0], torch.zeros(0, 2, 4, dtype=torch.int32, device="cuda"), 1.0)
    assert empty[0].shape == (0, 6, 64)
