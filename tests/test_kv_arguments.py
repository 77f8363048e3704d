"""No-GPU checks of the block-cache entry points: arguments are refused before any CUDA call."""
import ctypes

from paper_2608_08751_b200 import binding as B

INV, UNS, OK = B.IVF_ERR_INVALID_ARG, B.IVF_ERR_UNSUPPORTED, B.IVF_OK
_buf = (ctypes.c_char * 4096)()
P = (ctypes.addressof(_buf) + 255) & ~255


def _s(*v):
    return (ctypes.c_int64 * len(v))(*v)


def _cache(k=P, v=P, ks=(4096, 1024, 64), vs=(4096, 1024, 64), pages=10, page=16, kv=2, dim=64, dtype=B.IVF_BF16):
    return ctypes.byref(B._KvCache(k, v, _s(*ks), _s(*vs), pages, page, kv, dim, dtype))


def test_tables():
    def call(n=4, page=16, free=P, nf=3, table=P, stride=8, blocks=8, tokens=5, touched=9, cached=P, slot=P, used=P):
        return B.lib().ivf_kv_tables(cached, P, n, page, free, nf, table, stride, blocks, P, P, P, P, slot, tokens, P, P, touched, used, None)
    assert call(n=-1) == INV and call(nf=-1) == INV and call(tokens=-1) == INV and call(touched=-1) == INV
    assert call(page=0) == UNS and call(page=48) == UNS and call(page=256) == UNS
    assert call(n=16385) == UNS and call(tokens=1 << 31) == UNS
    assert call(stride=7) == INV and call(blocks=0) == INV
    assert call(cached=None) == INV and call(table=None) == INV and call(used=None) == INV and call(slot=None) == INV and call(free=None) == INV
    assert call(n=0, cached=None, table=None) == OK


def test_append():
    def call(n=4, heads=4, cache=None, rot=64, n_pos=10, rotary=P, eps=1e-6, q=P, qs=(256, 64), pos=P, out=P, w=P, ks=(128, 64)):
        return B.lib().ivf_kv_append(q, _s(*qs), P, _s(*ks), P, _s(128, 64), n, heads, cache or _cache(), pos, P, rotary, n_pos, rot, 0, w, w, eps,
                                     out, _s(256, 64), None)
    assert call(n=-1) == INV and call(n=1 << 31) == UNS
    assert call(heads=5) == INV and call(heads=1) == INV and call(heads=130) == UNS
    assert call(rot=24) == UNS and call(rot=80) == UNS and call(rot=-16) == UNS
    assert call(n_pos=0) == INV and call(rotary=None) == INV and call(eps=-1.0) == INV and call(eps=float("nan")) == INV
    assert call(q=None) == INV and call(q=P + 2) == INV and call(qs=(250, 64)) == INV and call(qs=(-256, 64)) == INV and call(ks=(128, 60)) == INV
    assert call(pos=None) == INV and call(out=None) == INV and call(w=P + 4) == INV
    assert call(cache=_cache(dtype=B.IVF_F32)) == INV and call(cache=_cache(dtype=9)) == INV
    assert call(cache=_cache(dim=72)) == UNS and call(cache=_cache(dim=272)) == UNS and call(cache=_cache(dim=0)) == UNS
    assert call(cache=_cache(page=24)) == UNS and call(cache=_cache(pages=-1)) == INV
    assert call(cache=_cache(k=None)) == INV and call(cache=_cache(v=P + 8)) == INV and call(cache=_cache(ks=(4096, 1024, 60))) == INV
    assert call(cache=_cache(kv=0)) == INV
    assert B.lib().ivf_kv_append(P, _s(0, 0), P, _s(0, 0), P, _s(0, 0), 4, 4, None, P, P, None, 0, 0, 0, None, None, 0.0, P, _s(0, 0), None) == INV
    assert call(n=0, q=None, pos=None, out=None) == OK


def test_summarize():
    def call(n=4, cache=None, pages=P, codes=P, scales=P):
        return B.lib().ivf_kv_summarize(cache or _cache(), pages, P, n, codes, scales, None)
    assert call(n=-1) == INV and call(n=1 << 31) == UNS
    assert call(pages=None) == INV and call(codes=None) == INV and call(scales=None) == INV and call(codes=P + 4) == INV
    assert call(cache=_cache(dtype=B.IVF_U8)) == INV and call(cache=_cache(page=8)) == UNS and call(cache=_cache(kv=0)) == INV
    assert call(n=0, pages=None) == OK


def test_select():
    def call(n=4, q=P, qs=(256, 64), dtype=B.IVF_BF16, heads=4, kv=2, dim=64, codes=P, pages=10, table=P, stride=8, n_req=2, blocks=8, page=16, req=P,
             take=4, first=1, last=1, out=P):
        return B.lib().ivf_kv_select(q, _s(*qs), dtype, n, heads, kv, dim, codes, P, pages, table, stride, n_req, blocks, page, req, P, take, first, last,
                                     out, None)
    assert call(n=-1) == INV and call(dtype=B.IVF_I8) == INV and call(page=17) == UNS and call(dim=8) == UNS
    assert call(heads=3) == INV and call(kv=0) == INV and call(heads=260) == UNS
    assert call(take=0) == UNS and call(take=1025) == UNS
    assert call(first=-1) == INV and call(last=0) == INV and call(first=4) == INV and call(last=5) == INV and call(first=2, last=3) == INV
    assert call(stride=7) == INV and call(n_req=0) == INV and call(blocks=0) == INV and call(stride=50000, blocks=50000) == UNS
    assert call(q=None) == INV and call(q=P + 8) == INV and call(qs=(256, 63)) == INV and call(codes=None) == INV and call(codes=P + 8) == INV
    assert call(table=None) == INV and call(req=None) == INV and call(out=None) == INV and call(pages=-1) == INV
    assert call(n=0, q=None, table=None) == OK


def test_attend():
    def call(n=4, q=P, qs=(256, 64), heads=4, cache=None, table=P, stride=8, n_req=2, blocks=8, req=P, sel=P, take=4, scale=1.0, out=P, os=(256, 64)):
        return B.lib().ivf_kv_attend(q, _s(*qs), n, heads, cache or _cache(), table, stride, n_req, blocks, req, P, sel, take, scale, out, _s(*os), None,
                                     None)
    assert call(n=-1) == INV and call(heads=7) == INV and call(heads=256) == UNS
    assert call(take=0) == UNS and call(take=1025) == UNS
    assert call(scale=float("inf")) == INV and call(scale=float("nan")) == INV
    assert call(q=None) == INV and call(q=P + 4) == INV and call(qs=(256, 4)) == INV and call(out=None) == INV and call(os=(256, 62)) == INV
    assert call(sel=None) == INV and call(table=None) == INV and call(req=None) == INV and call(stride=4) == INV and call(n_req=0) == INV
    assert call(cache=_cache(v=None)) == INV and call(cache=_cache(vs=(4096, 1024, 68))) == INV and call(cache=_cache(page=64, dim=264)) == UNS
    assert call(n=0, q=None, sel=None) == OK
    assert b"" != B.lib().ivf_last_error()
