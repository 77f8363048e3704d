"""No-GPU checks: block-cache calls whose outputs lie over what the call still reads are refused before any CUDA call."""
import ctypes

from paper_2608_08751_b200 import binding as B

_buf = (ctypes.c_char * (1 << 16))()
P = (ctypes.addressof(_buf) + 255) & ~255
PLACES = {name: P + 2048 * i for i, name in enumerate(
    ("cached", "fresh", "free", "table", "lens", "start", "req", "pos", "slot", "page", "fill", "used"))}


def _tables(n=4, blocks=8, stride=8, nf=16, tokens=5, touched=9, **at):
    p = {**PLACES, **at}
    return B.lib().ivf_kv_tables(p["cached"], p["fresh"], n, 16, p["free"], nf, p["table"], stride, blocks, p["lens"], p["start"], p["req"], p["pos"],
                                 p["slot"], tokens, p["page"], p["fill"], touched, p["used"], None)


def test_tables_outputs_over_the_lengths_or_the_free_list():
    for out in ("lens", "start", "req", "pos", "slot", "page", "fill", "used", "table"):
        for src in ("cached", "fresh", "free"):
            assert _tables(**{out: PLACES[src]}) == B.IVF_ERR_INVALID_ARG, (out, src)
            assert b"must not lie over" in B.lib().ivf_last_error()
    assert _tables(cached=PLACES["lens"]) == B.IVF_ERR_INVALID_ARG  # a plan's lengths as the next step's, in the same plan
    assert _tables(lens=PLACES["cached"] + 12) == B.IVF_ERR_INVALID_ARG and _tables(used=PLACES["free"] + 60) == B.IVF_ERR_INVALID_ARG
    assert _tables(stride=512, free=PLACES["table"] + 2048 + 28, nf=1) == B.IVF_ERR_INVALID_ARG  # inside the second row


def test_tables_neighbours_are_not_refused():
    # what follows the argument checks needs a device, so "not refused" is any other answer (there is none at no request)
    def refused(**kw):
        return _tables(**kw) == B.IVF_ERR_INVALID_ARG and b"must not lie over" in B.lib().ivf_last_error()
    import torch
    if torch.cuda.is_available():
        return  # (these are host addresses)
    assert not refused() and not refused(lens=PLACES["cached"] + 16) and not refused(used=PLACES["cached"] - 4)
    assert not refused(tokens=0, req=PLACES["cached"], pos=PLACES["cached"], slot=PLACES["cached"])
    assert not refused(stride=512, free=PLACES["table"] + 32, nf=16)  # between two rows
    assert not refused(stride=512, n=2, free=PLACES["table"] + 2048 + 32, nf=100, lens=P + 40000, start=P + 41000)  # behind the last one


def _s(*v):
    return (ctypes.c_int64 * len(v))(*v)


def _cache(ks=(4096, 1024, 64), vs=(4096, 1024, 64), pages=10, kv=2):
    return ctypes.byref(B._KvCache(P, P, _s(*ks), _s(*vs), pages, 16, kv, 64, B.IVF_BF16))


def _append(n=4, heads=4, out=(256, 64), cache=None):
    return B.lib().ivf_kv_append(P, _s(0, 0), P, _s(0, 0), P, _s(0, 0), n, heads, cache or _cache(), P, P, None, 0, 0, 0, None, None, 1e-6, P, _s(*out), None)


def _attend(n=4, heads=4, out=(256, 64), cache=None):
    return B.lib().ivf_kv_attend(P, _s(0, 0), n, heads, cache or _cache(), P, 8, 2, 8, P, P, P, 4, 1.0, P, _s(*out), None, None)


def _written(rc):
    return rc == B.IVF_ERR_INVALID_ARG and b"is written" in B.lib().ivf_last_error()


def test_written_tensors_with_two_elements_in_one_place():
    for call in (_append, _attend):
        for out in ((0, 64), (256, 0), (248, 64), (256, 56), (64, 192)):
            assert _written(call(out=out)), (call, out)
    for bad in ((0, 1024, 64), (4096, 0, 64), (4096, 1024, 0), (4096, 1016, 64), (2040, 1024, 64)):
        assert _written(_append(cache=_cache(ks=bad))) and _written(_append(cache=_cache(vs=bad))), bad


def test_what_is_only_read_may_be_expanded():
    import torch
    if torch.cuda.is_available():
        return  # (these are host addresses)
    # what follows the argument checks needs a device: any other answer will do.  Axes of one element, heads outside of
    # tokens, and a token axis outside of pages are fine
    assert not _written(_attend(cache=_cache(ks=(0, 0, 0), vs=(0, 0, 0))))
    for call in (_append, _attend):
        assert not _written(call()) and not _written(call(n=1, out=(0, 64))) and not _written(call(n=4, heads=2, out=(64, 256)))
    assert not _written(_append(cache=_cache(ks=(2048, 64, 128), vs=(128, 64, 1280))))
    assert not _written(_append(cache=_cache(ks=(0, 1024, 64), vs=(0, 1024, 64), pages=1)))
