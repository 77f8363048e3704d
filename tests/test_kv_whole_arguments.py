"""No-GPU checks of the operators on whole paged caches: arguments are refused before any CUDA call."""
import ctypes

import pytest
import torch

from paper_2608_08751_b200 import binding as B

INV, UNS, OK = B.IVF_ERR_INVALID_ARG, B.IVF_ERR_UNSUPPORTED, B.IVF_OK
_buf = (ctypes.c_char * (1 << 16))()
P = (ctypes.addressof(_buf) + 255) & ~255
PLACES = {name: P + 2048 * i for i, name in enumerate(
    ("table", "lens", "parent", "keep", "out", "out_lens", "from", "to", "fill", "free", "count", "ws"))}


def _s(*v):
    return (ctypes.c_int64 * len(v))(*v)


def _cache(k=P, v=P, ks=(4096, 1024, 64), vs=(4096, 1024, 64), pages=10, page=16, kv=2, dim=64, dtype=B.IVF_BF16):
    return ctypes.byref(B._KvCache(k, v, _s(*ks), _s(*vs), pages, page, kv, dim, dtype))


def _error():
    return B.lib().ivf_last_error()


def test_attend_chunk():
    def call(n=4, heads=4, cache=None, q=P, qs=(256, 64), table=P, stride=8, n_req=2, blocks=8, start=P, lens=P, scale=1.0, cap=0.0, window=0, out=P + 8192,
             os=(256, 64), ws=P, bytes=1 << 40):
        return B.lib().ivf_kv_attend_chunk(q, _s(*qs), n, heads, cache or _cache(), table, stride, n_req, blocks, start, lens, scale, cap, None, window, None, out,
                                           _s(*os), None, ws, bytes, None)
    nan, inf = float("nan"), float("inf")
    assert call(n=-1) == INV and call(n_req=-1) == INV and call(n=1 << 28) == UNS and call(n_req=16385) == UNS
    assert call(heads=3) == INV and call(heads=130) == UNS and call(cache=_cache(kv=0)) == INV
    assert call(scale=nan) == INV and call(scale=inf) == INV
    assert call(cap=-1.0) == INV and call(cap=nan) == INV and call(cap=inf) == INV and call(window=-1) == INV
    assert call(stride=7) == INV and call(blocks=0) == INV
    assert call(start=None) == INV and call(lens=None) == INV and call(table=None) == INV
    assert call(q=None) == INV and call(q=P + 8) == INV and call(qs=(250, 64)) == INV and call(out=None) == INV and call(os=(256, 60)) == INV
    assert call(cache=_cache(dim=72)) == UNS and call(cache=_cache(page=48)) == UNS and call(cache=_cache(dtype=B.IVF_F32)) == INV
    assert call(cache=_cache(v=None)) == INV and call(cache=_cache(ks=(4096, 1024, 60))) == INV
    for os in ((0, 64), (256, 0), (248, 64)):
        assert call(os=os) == INV and b"is written" in _error()
    assert call(out=P) == INV and b"must not share" in _error()
    assert call(out=P + 2048 - 128) == INV and b"must not share" in _error()
    assert call(ws=None) == INV and call(bytes=1000) == INV and call(ws=P + 8) == INV and b"workspace" in _error()
    assert call(n=0, q=None, table=None, start=None, ws=None) == OK


def test_attend_chunk_workspace():
    def call(n=4, heads=4, n_req=2, cache=None, out=True):
        got = ctypes.c_int64(-1)
        return B.lib().ivf_kv_attend_chunk_workspace(n, heads, cache or _cache(), n_req, ctypes.byref(got) if out else None), got.value
    assert call()[0] == OK and call()[1] > 0 and call()[1] % 16 == 0 and call(n=0) == (OK, 0)
    assert call(n=-1)[0] == INV and call(n_req=-1)[0] == INV and call(heads=3)[0] == INV and call(out=False)[0] == INV and call(cache=_cache(dim=8))[0] == UNS
    assert B.lib().ivf_debug_set_kv_chunk(3) == INV and B.lib().ivf_debug_set_kv_chunk(-1) == INV


def _fork(n_old=4, n_new=4, blocks=8, stride=8, out_stride=8, pages=40, page=16, bytes=0, **at):
    p = {**PLACES, **at}
    return B.lib().ivf_kv_fork(p["table"], stride, p["lens"], n_old, blocks, p["parent"], p["keep"], n_new, pages, page, p["out"], out_stride, p["out_lens"],
                               p["from"], p["to"], p["fill"], p["free"], p["count"], p["ws"], bytes, None)


def _compact(n=4, blocks=8, stride=8, out_stride=8, pages=40, page=16, moves=10, bytes=0, **at):
    p = {**PLACES, **at}
    return B.lib().ivf_kv_compact(p["table"], stride, p["lens"], n, blocks, pages, page, p["out"], out_stride, p["from"], p["to"], moves, p["count"], p["ws"],
                                  bytes, None)


def test_fork():
    assert _fork(n_old=-1) == INV and _fork(n_new=-1) == INV and _fork(n_old=16385) == UNS and _fork(n_new=16385) == UNS
    assert _fork(page=24) == UNS and _fork(pages=-1) == INV and _fork(pages=1 << 31) == INV
    assert _fork(blocks=0) == INV and _fork(stride=7) == INV and _fork(out_stride=7) == INV
    for name in ("table", "lens", "parent", "out", "out_lens", "from", "to", "fill", "free", "count"):
        assert _fork(**{name: None}) == INV and b"null pointer" in _error(), name
    for out in ("out", "out_lens", "from", "to", "fill", "free", "count"):
        for src in ("table", "lens", "parent", "keep"):
            assert _fork(**{out: PLACES[src]}) == INV and b"must not lie over" in _error(), (out, src)
    for a in ("out", "out_lens", "from", "to", "fill", "free", "count"):
        for b in ("out", "out_lens", "from", "to", "fill", "free", "count"):
            assert a == b or (_fork(**{a: PLACES[b]}) == INV and b"each other" in _error()), (a, b)
    assert _fork(table=PLACES["out"] + 96) == INV and b"must not lie over" in _error()
    assert _fork(pages=1 << 20, free=P + 30000) == INV and b"workspace" in _error()


def test_compact():
    assert _compact(n=-1) == INV and _compact(n=16385) == UNS and _compact(page=1) == UNS and _compact(pages=-1) == INV
    assert _compact(moves=-1) == INV and _compact(moves=1 << 31) == INV and _compact(blocks=0) == INV and _compact(stride=7) == INV
    for name in ("table", "lens", "out", "from", "to", "count"):
        assert _compact(**{name: None}) == INV and b"null pointer" in _error(), name
    for out in ("from", "to", "count"):
        for src in ("table", "lens", "out"):
            assert _compact(**{out: PLACES[src]}) == INV and b"must not lie over" in _error(), (out, src)
    assert _compact(to=PLACES["from"]) == INV and _compact(count=PLACES["to"] + 8) == INV and _compact(count=PLACES["from"]) == INV
    assert _compact(out=PLACES["lens"]) == INV and _compact(out=PLACES["table"] + 4) == INV and _compact(out=PLACES["table"], out_stride=9) == INV
    assert _compact(pages=1 << 20) == INV and b"workspace" in _error()
    got = ctypes.c_int64(-1)
    assert B.lib().ivf_kv_pages_workspace(4, 8, 40, ctypes.byref(got)) == OK and got.value == 0
    assert B.lib().ivf_kv_pages_workspace(4, 8, 1 << 20, ctypes.byref(got)) == OK and got.value > 4 << 20
    assert B.lib().ivf_kv_pages_workspace(-1, 8, 40, ctypes.byref(got)) == INV and B.lib().ivf_kv_pages_workspace(4, 0, 40, ctypes.byref(got)) == INV
    assert B.lib().ivf_kv_pages_workspace(4, 8, 40, None) == INV


def test_copy():
    def call(n=4, cache=None, source=P, to=P, codes=None, scales=None):
        return B.lib().ivf_kv_copy(cache or _cache(), source, to, None, n, codes, scales, None)
    assert call(n=-1) == INV and call(n=1 << 31) == UNS and call(source=None) == INV and call(to=None) == INV
    assert call(codes=P) == INV and call(scales=P) == INV and call(codes=P + 4, scales=P) == INV
    assert call(cache=_cache(dim=8)) == UNS and call(cache=_cache(k=None)) == INV and call(cache=_cache(dtype=B.IVF_F32)) == INV and call(cache=_cache(kv=0)) == INV
    for bad in ((0, 1024, 64), (4096, 0, 64), (4096, 1024, 0)):
        assert call(cache=_cache(ks=bad)) == INV and b"is written" in _error()
        assert call(cache=_cache(vs=bad)) == INV and b"is written" in _error()
    assert call(n=0, source=None, to=None) == OK


def test_neighbours_are_not_refused():
    if torch.cuda.is_available():
        return  # (these are host addresses)
    # what follows the argument checks needs a device, so "not refused" is any other answer
    def refused(rc):
        return rc == INV
    assert not refused(_fork()) and not refused(_fork(keep=None)) and not refused(_fork(n_old=0, table=None, lens=None)) and not refused(_fork(pages=0, free=None))
    assert not refused(_fork(n_new=1, out_stride=0)) and not refused(_fork(table=PLACES["out"] + 32, stride=16, out_stride=16))
    def attend(q, out, n=4):
        return B.lib().ivf_kv_attend_chunk(q, _s(1024, 64), n, 4, _cache(), P, 8, 2, 8, P, P, 1.0, 0.0, None, 0, None, out, _s(1024, 64), None, P, 1 << 40, None)
    # an output that shares rows of one buffer with the queries, but no element
    assert not refused(attend(P, P + 512)) and not refused(attend(P + 1024, P)) and refused(attend(P, P + 256)) and refused(attend(P + 256, P))
    assert not refused(_compact()) and not refused(_compact(out=PLACES["table"])) and not refused(_compact(moves=0, **{"from": None, "to": None}))


def test_tensors_are_refused_in_python():
    i32 = torch.zeros(4, dtype=torch.int32)
    table = torch.zeros(4, 4, dtype=torch.int32)
    half = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
    q = torch.zeros(4, 2, 64, dtype=torch.float16)
    for call in (lambda: B.ivf_kv_attend_chunk(q, half, half, table, i32, i32, 1.0), lambda: B.ivf_kv_fork(table, i32, i32, None, 10, 16),
                 lambda: B.ivf_kv_compact(table, i32, 10, 16), lambda: B.ivf_kv_copy(half, half, i32, i32)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(TypeError, match="float16 or bfloat16"):
        B.ivf_kv_copy(half.float(), half.float(), i32, i32)
    with pytest.raises(TypeError, match="torch.Tensor"):
        B.ivf_kv_fork([[0]], i32, i32, None, 10, 16)
    with pytest.raises(TypeError):
        B.ivf_kv_attend_chunk(q, half, half, table, i32)


def test_scales_and_caps_that_base_2_cannot_hold():
    """The kernels take scale * log2(e), cap * log2(e) and scale / cap: out of the range of a float they gave NaN without a word, and scale / cap below the
    normal numbers a logit with few digits."""
    def call(scale, cap):
        return B.lib().ivf_kv_attend_chunk(None, _s(256, 64), 0, 4, _cache(), None, 8, 2, 8, None, None, scale, cap, None, 0, None, None, _s(256, 64), None, None, 0, None)
    for scale, cap in ((3e38, 0.0), (-3e38, 0.0), (1.0, 3.4e38), (1.0, 1e-39), (0.1, 1e38), (-0.1, 1e38), (1e-30, 1e20), (3e38, 3e38)):
        assert call(scale, cap) == INV and b"scale" in _error() and b"cap" in _error(), (scale, cap)
    for scale, cap in ((2e38, 0.0), (-0.125, 50.0), (0.0, 2e38), (1.0, 1e37), (1e-40, 0.0), (0.0, 0.0), (1e30, 1e-5)):
        assert call(scale, cap) == OK, (scale, cap)


@pytest.mark.skipif(torch.cuda.is_available(), reason="these are host addresses: what is not refused here would run")
def test_outputs_in_the_gaps_of_the_queries_are_not_refused():
    """Views of one buffer with the same strides, in any order of its axes, are told apart exactly."""
    def refused(gap, q_stride, n, heads, out_stride=None):
        out_stride = out_stride or q_stride
        kv = 2 if heads % 2 == 0 else 1
        rc = B.lib().ivf_kv_attend_chunk(P, _s(*q_stride), n, heads, _cache(kv=kv), P, 8, 2, 8, P, P, 1.0, 0.0, None, 0, None, P + 2 * gap, _s(*out_stride), None, P,
                                         1 << 40, None)
        return rc == INV and b"must not share" in _error()
    n, heads = 7, 4
    # heads first, [heads, 2, n, 64]: queries and outputs of a head in turn
    assert not refused(n * 64, (64, 2 * n * 64), n, heads) and refused((n - 1) * 64, (64, 2 * n * 64), n, heads) and refused(0, (64, 2 * n * 64), n, heads)
    # [heads, n, 2, 64] and [n, heads, 2, 64]: rows in turn
    for strides in ((128, n * 128), (heads * 128, 128)):
        assert not refused(64, strides, n, heads) and refused(56, strides, n, heads) and refused(128, strides, n, heads) and refused(72, strides, n, heads)
    # [n, 2, heads, 64]: tokens in turn
    assert not refused(heads * 64, (2 * heads * 64, 64), n, heads) and refused(heads * 64 - 8, (2 * heads * 64, 64), n, heads)
    # behind the last row of one order and among the rows of the next
    assert not refused(n * 64, (64, 2 * n * 64), n, 1) and refused(8, (64, 64), 1, 1) and not refused(64, (0, 0), 1, 1)
    # strides that differ, ranges that meet: refused, whatever the elements
    assert refused(64, (256, 1024), n, heads, (512, 4096))
    # brute force
    rng = torch.Generator().manual_seed(0)
    pick = lambda *v: v[int(torch.randint(0, len(v), (1,), generator=rng))]  # noqa: E731
    seen = set()
    for _ in range(400):
        n, heads = pick(1, 2, 3, 5), pick(1, 2, 4)
        st, sh = pick(64, 128, 192, 320, 448, 1024), pick(64, 128, 256, 640, 1088)
        if (n > 1 and heads > 1 and (max(st, sh) < 64 + ((n - 1) * st if st < sh else (heads - 1) * sh))) or (n > 1 and heads > 1 and st == sh):
            continue  # (an output with two elements in one place is another refusal)
        gap = pick(0, 8, 56, 64, 72, 128, 192, 256, 320, 640, 1024)
        rows = {t * st + h * sh + x for t in range(n) for h in range(heads) for x in range(64)}
        share = any(r + gap in rows for r in rows)
        assert refused(gap, (st, sh), n, heads) == share, (gap, st, sh, n, heads)
        seen.add(share)
    assert seen == {False, True}
