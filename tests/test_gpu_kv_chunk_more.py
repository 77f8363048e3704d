"""Further calls of ivf_kv_attend_chunk: batches that are not in order, short tensors, and the bits that single tokens keep.  Tolerances as in the tests of
the formula."""
import numpy as np
import pytest
import torch

import kv_reference as R
import kv_whole_reference as W
from paper_2608_08751_b200 import binding as B
from test_gpu_kv import _np
from test_gpu_kv_chunk import _case, _check, _finite, _run, kernel  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("start", [[0, 10, 8, 19], [0, 5, 3, 8], [5, 3, 9, 12], [0, 30, 0, 30], [-3, 4, 9, 11], [0, 0, 7, 2]], ids=str)
@pytest.mark.parametrize("padding", [0, 6])
def test_a_descending_token_start_counts_as_its_running_maximum(kernel, start, padding):  # noqa: F811
    c = _case([(100, 10), (200, 6), (60, 3)], 2, 2, 64, 32, "fp16", seed=7)
    n = max(start) + padding
    c["q"] = torch.randn(n, 4, 64, device="cuda").half()
    out, lse = _run(dict(c, start=np.array(start)), out=torch.full_like(c["q"], 7.0))
    with pytest.raises(B.IvfError) as e:
        B.ivf_check()
    assert e.value.code == B.IVF_ERR_BAD_ID and "ivf_kv_attend_chunk" in str(e.value)
    _check(dict(c, start=np.maximum(np.maximum.accumulate(start), 0)), out, lse)


def test_a_descending_token_start_of_many_requests(kernel):  # noqa: F811
    rng = np.random.default_rng(1)
    c = _case([(int(rng.integers(0, 60)), int(rng.integers(0, 4))) for _ in range(700)], 1, 4, 64, 16, "bf16", seed=1)
    start = c["start"].copy()
    for b in (3, 150, 400, 401, 699):
        start[b] = max(0, start[b] - 5)
    start[300] += 40
    lens = c["lens"]
    lens = np.maximum(lens, np.diff(start).clip(0))  # (no request with fewer tokens in the cache than new ones)
    c["table"] = np.where(c["table"] < 0, 0, c["table"])
    c["kc"], c["vc"] = torch.nan_to_num(c["kc"]), torch.nan_to_num(c["vc"])
    out, lse = _run(dict(c, start=start, lens=lens))
    with pytest.raises(B.IvfError):
        B.ivf_check()
    _check(dict(c, start=np.maximum.accumulate(start), lens=lens), out, lse)


@pytest.mark.parametrize("requests,group,dim,kind", [
    ([(700, 1), (90, 1), (0, 1)], 4, 128, "bf16"), ([(700, 1), (31, 1)], 7, 96, "fp16"), ([(3000, 1)], 8, 64, "bf16"), ([(400, 1)] * 5, 1, 112, "fp16"),
    ([(500, 2), (60, 2)], 4, 64, "bf16"), ([(300, 5)], 1, 64, "fp16"), ([(20000, 1)], 2, 128, "bf16"), ([(900, 3), (40, 1)], 2, 16, "bf16"),
], ids=str)
def test_weights_of_few_rows_keep_their_bits(requests, group, dim, kind):
    """Up to 8 rows of a request and kv head: the weights come in two parts, so beside the output's own rounding, u of the value, and the logits'
    own error an output is off by u^2 of the weighted mean of |v|, not u; and by half a step of the type's least number for each key, against a largest
    weight of one."""
    c = _case(requests, 2, group, dim, 32, kind, seed=dim + group)
    out, lse = _run(c)
    B.ivf_check()
    want, _, size, unit = W.attend_chunk(_np(c["q"]), _finite(_np(c["kc"])), _finite(_np(c["vc"])), c["table"], c["start"], c["lens"], c["scale"])
    u = R.UNIT[kind]
    move = (dim + 16) * 2.0 ** -24 * unit + 2.0 ** -20
    least = {"bf16": 2.0 ** -134, "fp16": 2.0 ** -25}[kind] * max(c["lens"]) * np.abs(_finite(_np(c["vc"]))).max()
    tol = u * np.abs(want) + (u * u + 2 * move[..., None]) * size + least + R.TINY[kind]
    off = np.abs(_np(out) - want)
    assert (off <= tol).all(), (off / tol).max()


def test_queries_and_outputs_of_a_head_in_turn(kernel):  # noqa: F811
    c = _case([(50, 20), (7, 9)], 2, 2, 64, 16, "bf16", seed=7)
    both = torch.zeros(4, 2, 29, 64, dtype=torch.bfloat16, device="cuda")
    both[:, 0] = c["q"].transpose(0, 1)
    q, out = both[:, 0].transpose(0, 1), both[:, 1].transpose(0, 1)
    _, lse = _run(dict(c, q=q), out=out)
    B.ivf_check()
    _check(c, out, lse)
    assert torch.equal(q, c["q"])
    with pytest.raises(B.IvfError, match="share memory"):
        _run(dict(c, q=q), out=both[:, 0].transpose(0, 1))


def test_fewer_rows_than_token_start_speaks_of(kernel):  # noqa: F811
    c = _case([(70, 5), (0, 12), (9, 3)], 2, 4, 64, 32, "bf16")
    for n in (1, 5, 14, 19):
        short = dict(c, q=c["q"][:n].contiguous())
        out, lse = _run(short)
        B.ivf_check()
        _check(short, out, lse)
