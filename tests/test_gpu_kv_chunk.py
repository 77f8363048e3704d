"""ivf_kv_attend_chunk against its plain 64-bit form, through the binding.

Tolerances.  The output carries one rounding, u = 2^-8 (bf16) or 2^-11 (fp16) of the value, and the rounding of the exponentials to the
same type, at most u of the weighted mean of |v|.  A logit sums d exact products in 32 bits, is scaled, capped and biased: at most
(d + 16) 2^-24 of the magnitudes that meet in it (of the cap beside: tanh as 1 - 2 / (1 + exp(2 x)) is off by 8 2^-24), and moves its
weight, the sum and so the output by as much, twice.  2^-20 covers exp2, the joins and the final division."""
import itertools
import math

import numpy as np
import pytest
import torch

import kv_reference as R
import kv_whole_reference as W
from paper_2608_08751_b200 import binding as B
from test_gpu_kv import TYPES, _cache, _gen, _i32, _np

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[0, 1, 2], ids=["auto", "rows", "tiles"])
def kernel(request):
    B.ivf_debug_set_kv_chunk(request.param)
    yield request.param
    B.ivf_debug_set_kv_chunk(0)


def _case(requests, kv, group, dim, page, kind, layout="head", seed=0, spare=3, q_scale=1.5, junk=math.nan):
    """requests: (tokens before, new tokens).  What no token may look at holds `junk`."""
    g = _gen(seed)
    lens = np.array([c + f for c, f in requests], np.int64)
    start = np.concatenate([[0], np.cumsum([f for _, f in requests])]).astype(np.int64)
    blocks = [R.ceil_div(int(n), page) for n in lens]
    pages = sum(blocks) + spare
    order = np.random.default_rng(seed).permutation(pages)
    table = np.full((len(requests), max(blocks + [1]) + 2), -1, np.int64)
    at = 0
    kc, vc = _cache(pages, kv, page, dim, kind, layout, junk), _cache(pages, kv, page, dim, kind, layout, junk)
    for b, n in enumerate(blocks):
        table[b, :n] = order[at: at + n]
        at += n
        for j in range(n):
            fill = min(page, int(lens[b]) - j * page)
            for c, s in ((kc, 1.0), (vc, 1.0)):
                c[table[b, j], :, :fill] = (torch.randn(kv, fill, dim, device="cuda", generator=g) * s).to(TYPES[kind])
    q = (torch.randn(int(start[-1]), kv * group, dim, device="cuda", generator=g) * q_scale).to(TYPES[kind])
    return {"q": q, "kc": kc, "vc": vc, "table": table, "start": start, "lens": lens, "scale": dim ** -0.5, "kind": kind}


def _run(c, out=None, **more):
    return B.ivf_kv_attend_chunk(c["q"], c["kc"], c["vc"], _i32(c["table"]), _i32(c["start"]), _i32(c["lens"]), c["scale"], out=out, want_lse=True, **more)


def _finite(x):
    return np.where(np.isfinite(x), x, 0.0)  # (only what no token sees is not finite)


def _check(c, out, lse, cap=0.0, slopes=None, window=0, prefix=None):
    want, want_lse, size, unit = W.attend_chunk(_np(c["q"]), _finite(_np(c["kc"])), _finite(_np(c["vc"])), c["table"], c["start"], c["lens"], c["scale"], cap,
                                                slopes, window, prefix)
    u, dim = R.UNIT[c["kind"]], c["q"].shape[2]
    move = (dim + 16) * 2.0 ** -24 * unit + 8 * 2.0 ** -24 * cap + 2.0 ** -20
    tol = u * np.abs(want) + (u + 2 * move[..., None]) * size + R.TINY[c["kind"]]
    assert (np.abs(_np(out) - want) <= tol).all()
    seen = np.isfinite(want_lse)
    got = _np(lse)
    assert (np.isneginf(got) == ~seen).all()
    assert (np.abs(got - want_lse)[seen] <= (move + 2.0 ** -22 * np.abs(want_lse))[seen]).all()


def _more(c, cap=0.0, bias=False, window=0, prefix=None):
    heads = c["q"].shape[1]
    slopes = (2.0 ** (-8.0 * (np.arange(heads) + 1) / heads)).astype(np.float32) if bias else None
    call = {"cap": cap, "window": window, "slopes": torch.tensor(slopes, device="cuda") if bias else None, "prefix": _i32(prefix) if prefix is not None else None}
    return call, {"cap": cap, "slopes": slopes.astype(np.float64) if bias else None, "window": window, "prefix": prefix}


SHAPES = [
    # requests, kv_heads, group, dim, page, type, layout
    ([(0, 1)], 1, 1, 16, 16, "bf16", "head"), ([(15, 1), (16, 1), (17, 1), (63, 1), (64, 1), (0, 0), (300, 1)], 2, 4, 64, 16, "fp16", "token"),
    ([(200, 5), (0, 5), (31, 2), (7, 0)], 4, 7, 96, 32, "bf16", "head"), ([(0, 130)], 1, 8, 128, 64, "fp16", "both"),
    ([(700, 70), (3, 33)], 2, 4, 128, 64, "bf16", "head"), ([(129, 64), (0, 300)], 1, 16, 80, 128, "fp16", "token"),
    ([(40, 40), (500, 1)], 2, 2, 256, 128, "bf16", "head"), ([(100, 3)], 1, 20, 112, 32, "fp16", "both"), ([(260, 2)], 1, 64, 128, 16, "bf16", "head"),
    ([(0, 257), (1000, 20)], 2, 1, 64, 16, "bf16", "token"), ([(50, 9)], 3, 5, 48, 64, "fp16", "head"), ([(333, 77)], 2, 3, 224, 64, "fp16", "both"),
]


@pytest.mark.parametrize("requests,kv,group,dim,page,kind,layout", SHAPES)
def test_matches_the_formula(kernel, requests, kv, group, dim, page, kind, layout):
    c = _case(requests, kv, group, dim, page, kind, layout, seed=dim + len(requests))
    out, lse = _run(c)
    B.ivf_check()
    _check(c, out, lse)


MORE = [dict(cap=5.0), dict(bias=True), dict(window=1), dict(window=37), dict(prefix=True), dict(cap=2.0, bias=True, window=100, prefix=True),
        dict(cap=30.0, window=64), dict(bias=True, prefix=True), dict(window=2 ** 31 - 1)]


@pytest.mark.parametrize("more", MORE, ids=["-".join(m) for m in MORE])
@pytest.mark.parametrize("shape", [2, 4, 5, 6, 9], ids=str)
def test_caps_biases_windows_and_prefixes(kernel, shape, more):
    requests, kv, group, dim, page, kind, layout = SHAPES[shape]
    more = dict(more)
    if "prefix" in more:
        more["prefix"] = [(90, 0, 2000, -3)[i % 4] for i in range(len(requests))]
    c = _case(requests, kv, group, dim, page, kind, layout, seed=shape, q_scale=4.0)
    call, ref = _more(c, **more)
    out, lse = _run(c, **call)
    B.ivf_check()
    _check(c, out, lse, **ref)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("context,n", [(5000, 1), (5000, 3), (9000, 40), (2, 1)])
def test_long_contexts_are_shared_out(kernel, context, n, kind):
    c = _case([(context, n), (context // 7, 1)], 2, 4, 128, 64, kind, seed=context + n)
    out, lse = _run(c)
    B.ivf_check()
    _check(c, out, lse)


def test_many_requests_of_all_lengths(kernel):
    rng = np.random.default_rng(5)
    c = _case([(int(rng.integers(0, 150)), int(rng.integers(0, 4))) for _ in range(300)], 2, 2, 64, 16, "bf16", seed=5)
    out, lse = _run(c)
    B.ivf_check()
    _check(c, out, lse)


def test_padding_rows_are_zeros_and_rows_past_the_tensor_are_left(kernel):
    c = _case([(70, 5), (0, 12), (9, 3)], 2, 4, 64, 32, "bf16")
    n = c["q"].shape[0]
    wide = torch.full((n + 9, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    padded = dict(c, q=torch.cat([c["q"], torch.full((4, 8, 64), math.nan, dtype=torch.bfloat16, device="cuda")]))
    out, lse = _run(padded, out=wide[: n + 4])
    B.ivf_check()
    assert (out[n:] == 0).all() and torch.isneginf(lse[n:]).all() and (wide[n + 4:] == 7).all()
    _check(c, out[:n], lse[:n])
    # fewer rows than token_start speaks of: the rest does not exist
    short = dict(c, q=c["q"][:14].contiguous())
    got, got_lse = _run(short)
    B.ivf_check()
    assert torch.equal(got, out[:14]) or (got.float() - out[:14].float()).abs().max() < 0.05
    whole = W.attend_chunk(_np(c["q"]), _finite(_np(c["kc"])), _finite(_np(c["vc"])), c["table"], c["start"], c["lens"], c["scale"])
    assert np.abs(_np(got) - whole[0][:14]).max() < 0.05 and np.abs(_np(got_lse) - whole[1][:14]).max() < 1e-3


def test_strided_queries_outputs_and_expanded_keys(kernel):
    c = _case([(33, 9), (140, 30)], 2, 4, 64, 16, "fp16")
    n = c["q"].shape[0]
    qkv = torch.zeros(n, 8 * 64 + 256, dtype=torch.float16, device="cuda")
    qkv[:, 128: 128 + 512] = c["q"].reshape(n, 512)
    c["q"] = qkv[:, 128: 128 + 512].view(n, 8, 64)
    heads_first = torch.zeros(8, n, 72, dtype=torch.float16, device="cuda")
    out, lse = _run(c, out=heads_first[:, :, :64].transpose(0, 1))
    B.ivf_check()
    _check(c, out, lse)
    assert (heads_first[:, :, 64:] == 0).all()
    one = c["kc"][:, :1].expand(-1, 2, -1, -1)  # both kv heads read the same keys
    same = dict(c, kc=one)
    out, lse = _run(same)
    B.ivf_check()
    _check(same, out, lse)


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_values_that_are_not_finite_reach_only_those_who_see_them(kernel, kind, value):
    c = _case([(100, 40), (4, 30)], 2, 4, 64, 32, kind, seed=3)
    clean, clean_lse = _run(c, window=90, prefix=_i32([0, 20]))
    bad = [(0, 120), (0, 135), (0, 60), (1, 25), (1, 10)]  # (request, key): in front of, inside and behind the new tokens
    v = c["vc"].clone() if c["vc"].is_contiguous() else c["vc"]
    c["vc"] = v
    for b, key in bad:
        v[c["table"][b, key // 32], 0, key % 32, 5] = value
    out, lse = _run(c, window=90, prefix=_i32([0, 20]))
    B.ivf_check()
    got, was = _np(out), _np(clean)
    for b in range(2):
        given = int(c["start"][b + 1] - c["start"][b])
        for t in range(given):
            row, pos = int(c["start"][b]) + t, int(c["lens"][b]) - given + t
            sees = any(r == b and (key <= pos or key < (0, 20)[b]) and pos - key < 90 for r, key in bad)
            for head in range(8):
                hit = sees and head < 4
                assert np.isfinite(got[row, head, 5]) != hit, (row, head)
                if hit and not math.isnan(value) and kind == "bf16":
                    assert got[row, head, 5] == value or math.isnan(got[row, head, 5])
                rest = np.delete(got[row, head], 5)
                assert np.isfinite(rest).all() and np.abs(rest - np.delete(was[row, head], 5)).max() <= 2 * R.UNIT[kind] * 8
    assert torch.equal(lse, clean_lse)


def test_keys_and_queries_that_are_not_finite(kernel):
    c = _case([(40, 20)], 1, 4, 64, 16, "bf16", seed=4)
    clean, _ = _run(c)
    key = 50  # seen by the tokens from position 50 on
    c["kc"][c["table"][0, key // 16], 0, key % 16, 3] = math.nan
    c["q"][2, 1, 0] = math.inf
    out, lse = _run(c)
    B.ivf_check()
    for t in range(20):
        for head in range(4):
            broken = 40 + t >= key or (t, head) == (2, 1)
            assert bool(torch.isnan(out[t, head]).any()) == broken, (t, head)
            if not broken:
                assert (out[t, head].float() - clean[t, head].float()).abs().max() <= 2 * R.UNIT["bf16"] * 8


def test_missing_pages_and_a_window_whose_old_pages_are_gone(kernel):
    c = _case([(500, 20), (90, 2)], 2, 4, 64, 32, "bf16", seed=6)
    c["table"][0, 3] = -1
    c["table"][0, 14] = -1
    out, lse = _run(c)
    B.ivf_check()
    _check(c, out, lse)
    c["table"][0, :12] = -1  # keys before 384; the window begins at 401
    out, lse = _run(c, window=100)
    B.ivf_check()
    _check(c, out, lse, window=100)
    c["table"][1, :] = -1    # nothing at all
    out, lse = _run(c)
    B.ivf_check()
    _check(c, out, lse)
    assert (out[20:] == 0).all()


@pytest.mark.parametrize("what", ["page", "length", "columns", "descending"])
def test_what_is_out_of_range_is_flagged_and_skipped(kernel, what):
    c = _case([(100, 10), (200, 6), (60, 3)], 2, 2, 64, 32, "fp16", seed=7)
    if what == "page":
        c["table"][0, 1] = c["kc"].shape[0]
    elif what == "length":
        c["lens"][1] = 4
    elif what == "columns":
        c["table"] = c["table"][:, :5]
    else:
        c["start"] = np.array([0, 10, 8, 19])
    out, lse = _run(c)
    with pytest.raises(B.IvfError) as e:
        B.ivf_check()
    assert e.value.code == B.IVF_ERR_BAD_ID and "ivf_kv_attend_chunk" in str(e.value)
    if what != "descending":
        _check(c, out, lse)


def test_a_call_gives_the_same_bits_each_time(kernel):
    c = _case([(3000, 60), (777, 1), (12, 50)], 2, 4, 128, 64, "bf16", seed=8)
    first = _run(c)
    for _ in range(3):
        again = _run(c)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_no_request_and_no_token():
    c = _case([(3, 2)], 1, 2, 64, 16, "bf16")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    out, lse = B.ivf_kv_attend_chunk(c["q"], c["kc"], c["vc"], torch.zeros(0, 4, dtype=torch.int32, device="cuda"), _i32([0]), none, 1.0, want_lse=True)
    B.ivf_check()
    assert (out == 0).all() and torch.isneginf(lse).all()
    out, lse = B.ivf_kv_attend_chunk(c["q"][:0], c["kc"], c["vc"], _i32(c["table"]), _i32([0, 0]), _i32([0]), 1.0, want_lse=True)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)


@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0])
def test_scales(kernel, scale):
    c = _case([(100, 33)], 2, 4, 64, 32, "fp16", seed=9)
    c["scale"] = scale
    for cap in (0.0, 4.0):
        out, lse = _run(c, cap=cap)
        B.ivf_check()
        _check(c, out, lse, cap=cap)


def test_far_offsets_of_a_large_cache(kernel):
    # pages past 2^31 elements: 1,100 pages of 16 x 64 x 2,048 elements' stride
    pages, kv, page, dim = 1100, 1, 64, 128
    big = torch.empty(pages, 2_000_000, dtype=torch.bfloat16, device="cuda")
    kc = big.as_strided((pages, kv, page, dim), (2_000_000, 16384, 256, 1))
    vc = big.as_strided((pages, kv, page, dim), (2_000_000, 16384, 256, 1), 128)
    c = _case([(300, 20)], kv, 4, dim, page, "bf16", seed=10)
    table = c["table"].copy()
    for j in range(5):
        src, dst = c["table"][0, j], 1095 + j
        kc[dst], vc[dst] = c["kc"][src], c["vc"][src]
        table[0, j] = dst
    out, lse = _run(dict(c, kc=kc, vc=vc, table=table))
    B.ivf_check()
    _check(c, out, lse)


def test_streams_and_captured_graphs(kernel):
    cases = [_case([(2000, 9), (40, 1)], 2, 4, 128, 64, "bf16", seed=s) for s in (11, 12)]
    want = [_run(c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = []
    for _ in range(5):
        got = []
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                got.append(B.ivf_kv_attend_chunk(c["q"], c["kc"], c["vc"], _i32(c["table"]), _i32(c["start"]), _i32(c["lens"]), c["scale"], want_lse=True))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    graphs, outs, held = [], [], []
    for c in cases:
        ints = [_i32(c[k]) for k in ("table", "start", "lens")]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(B.ivf_kv_attend_chunk(c["q"], c["kc"], c["vc"], *ints, c["scale"], want_lse=True))
        graphs.append(graph)
        held.append(ints)
    for order in itertools.permutations(range(2)):
        for i in order:
            outs[i][0].zero_()
            graphs[i].replay()
        _run(_case([(5000, 64)], 2, 4, 128, 64, "bf16", seed=13))  # another call in between
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i][0], want[i][0]) and torch.equal(outs[i][1], want[i][1])
    # the lengths are the device's: a captured call follows them
    held[0][2][0] -= 500
    graphs[0].replay()
    B.ivf_check()
    shorter = dict(cases[0], lens=cases[0]["lens"] - np.array([500, 0]))
    _check(shorter, *outs[0])


def test_a_plan_of_tables_is_what_it_takes(kernel):
    """A prompt in two chunks and three single tokens through ivf_kv_tables and ivf_kv_append, against the formula over all keys."""
    kv, group, dim, page = 2, 4, 64, 16
    pages = 40
    kc, vc = _cache(pages, kv, page, dim, "bf16"), _cache(pages, kv, page, dim, "bf16")
    g = _gen(14)
    free = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table, cached, taken = _i32(np.full((2, 12), -1)), _i32([0, 0]), 0
    for fresh in ([50, 3], [21, 0], [1, 1], [1, 1], [1, 1]):
        tokens = sum(fresh) + 2
        plan = B.ivf_kv_tables(cached, _i32(fresh), free[taken:], table, page, tokens)
        q, k, v = (torch.randn(tokens, n, dim, device="cuda", generator=g).to(torch.bfloat16) for n in (kv * group, kv, kv))
        q = B.ivf_kv_append(q, k, v, kc, vc, plan.token_pos, plan.token_slot)
        out, lse = B.ivf_kv_attend_chunk(q, kc, vc, table, plan.token_start, plan.kv_lens, dim ** -0.5, want_lse=True)
        B.ivf_check()
        c = {"q": q, "kc": kc, "vc": vc, "table": _np(table), "start": _np(plan.token_start), "lens": _np(plan.kv_lens), "scale": dim ** -0.5, "kind": "bf16"}
        _check(c, out, lse)
        cached = plan.kv_lens.clone()
        taken += int(plan.used)
