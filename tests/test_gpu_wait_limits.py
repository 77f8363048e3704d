"""Device-side waits that run out in the middle of a call: the kernel returns, the status word says so, and the next call is right.

The limit of a wait is taken down from two seconds to what waits last in ordinary use (a few microseconds) and below, so that they end at many
places: with copies and products in flight, and behind warps that have left in good order.  A call may come through; then its
results count."""
import pytest
import torch

from paper_2608_08751_b200 import binding as B
from test_gpu_kv_chunk import _case, _check, _run

pytestmark = pytest.mark.gpu

LIMITS = [1] * 8 + [1000, 2000, 4000, 6000, 8000, 10000, 12000, 15000, 20000, 30000, 50000] * 2


def _ran_out(call, right, limit):
    """Whether a wait of the call ran out; if none did its result has to be right."""
    B.ivf_debug_set_wait_limit_ns(limit)
    try:
        got = call()
        B.ivf_check()
    except B.IvfError as e:
        assert e.code == B.IVF_ERR_DEVICE_TIMEOUT, e
        return True
    finally:
        B.ivf_debug_set_wait_limit_ns(0)
    assert right(got)
    return False


def _sweep(call, right):
    ends = []
    for limit in LIMITS:
        ends.append(_ran_out(call, right, limit))
        assert right(call())
        B.ivf_check()
    print("ran out:", "".join("x" if e else "." for e in ends))
    assert any(ends[:8])  # (no wait for memory is over within a few looks)


@pytest.mark.parametrize("dim,more", [(64, {}), (128, {}), (256, {}), (128, {"cap": 5.0}), (96, {"window": 100})], ids=str)
def test_attend_chunk_large_tiles(dim, more):
    c = _case([(900, 300), (40, 200), (5, 1)], 2, 4, dim, 32, "bf16", seed=dim)
    B.ivf_debug_set_kv_chunk(2)
    try:
        want = _run(c, **more)
        B.ivf_check()
        _check(c, *want, **more)
        _sweep(lambda: _run(c, **more), lambda got: torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]))
    finally:
        B.ivf_debug_set_kv_chunk(0)
