"""Calls of ivf_kv_attend_chunk, ivf_kv_fork, ivf_kv_compact and ivf_kv_copy that the documentation allows and ordinary use seldom makes.  Tolerances as
in the tests of the formula."""
import math

import numpy as np
import pytest
import torch

import kv_whole_reference as W
from paper_2608_08751_b200 import binding as B
from test_gpu_kv import _gen, _i32, _np
from test_gpu_kv_chunk import _case, _check, _finite, _more, _run, kernel  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 80, 96, 112, 128, 144, 160, 192, 208, 256])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_every_width_of_heads(kernel, dim, kind):  # noqa: F811
    c = _case([(150, 35), (20, 3)], 2, 4, dim, 32, kind, seed=dim)
    for more in ({}, {"cap": 3.0, "bias": True}):
        call, ref = _more(c, **more)
        out, lse = _run(c, **call)
        B.ivf_check()
        _check(c, out, lse, **ref)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 6, 7, 9, 11, 13, 17, 31, 33, 48, 63, 64])
def test_every_size_of_groups(kernel, group):  # noqa: F811
    c = _case([(90, 140 // group + 2), (130, 1)], 2, group, 64, 16, "bf16", seed=group)
    out, lse = _run(c)
    B.ivf_check()
    _check(c, out, lse)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_new_tokens_at_every_place_in_a_page(kernel, page):  # noqa: F811
    c = _case([(page - 1, 1), (page, 1), (page + 1, 1), (2 * page - 3, 5), (0, page), (0, page + 1), (3 * page, 2 * page), (0, 1), (5 * page - 1, 3)], 1, 4, 64, page, "fp16",
              seed=page)
    out, lse = _run(c)
    B.ivf_check()
    _check(c, out, lse)


@pytest.mark.parametrize("slope", [8.0, -0.01, 0.0])
def test_steep_flat_and_rising_biases(kernel, slope):  # noqa: F811
    # a steep one leaves the near keys alone, a rising one weighs the far ones most: the maximum then grows with every tile
    c = _case([(700, 40)], 2, 4, 64, 64, "bf16", seed=3)
    slopes = np.full(8, slope, np.float32)
    out, lse = _run(c, slopes=torch.tensor(slopes, device="cuda"))
    B.ivf_check()
    _check(c, out, lse, slopes=slopes.astype(np.float64))


@pytest.mark.parametrize("size", [60.0, 600.0])
def test_logits_far_apart(kernel, size):  # noqa: F811
    # a few keys far above the others, at both ends: references that are left behind by more than any exponent
    c = _case([(600, 30)], 1, 4, 64, 32, "bf16", seed=4)
    for key in (3, 300, 598):
        c["kc"][c["table"][0, key // 32], 0, key % 32] = (c["q"][5, 0].float() * size / 64).to(torch.bfloat16)
    out, lse = _run(c)
    B.ivf_check()
    _check(c, out, lse)


def test_a_saturated_cap(kernel):  # noqa: F811
    c = _case([(200, 30)], 2, 4, 64, 32, "fp16", seed=5, q_scale=200.0)
    out, lse = _run(c, cap=2.0)
    B.ivf_check()
    _check(c, out, lse, cap=2.0)


def test_small_capped_logits_keep_their_digits(kernel):  # noqa: F811
    """One key to a token and one number to a query, so that the product is exact and lse is the logit: tanh, the cap, and the way to base 2 and
    back are a dozen roundings of 2^-24 of the logit, 2^-20 at most; nothing of the cap's own size."""
    c = _case([(90, 40)], 1, 4, 64, 32, "fp16", seed=11)
    c["q"][:, :, 1:] = 0
    for cap in (50.0, 1000.0):
        out, lse = _run(c, cap=cap, window=1)
        B.ivf_check()
        want = W.attend_chunk(_np(c["q"]), _finite(_np(c["kc"])), _finite(_np(c["vc"])), c["table"], c["start"], c["lens"], c["scale"], cap, window=1)[1]
        assert (np.abs(_np(lse) - want) <= 2.0 ** -20 * np.abs(want) + 1e-30).all()


def test_prefixes_in_front_of_inside_and_behind_the_new_tokens(kernel):  # noqa: F811
    c = _case([(100, 60)] * 6, 1, 4, 64, 32, "bf16", seed=6)
    prefix = np.array([50, 100, 101, 130, 160, 10 ** 6])
    for window in (0, 1, 40, 130):
        out, lse = _run(c, prefix=_i32(prefix), window=window)
        B.ivf_check()
        _check(c, out, lse, prefix=prefix, window=window)


def test_an_output_between_the_queries_of_one_buffer(kernel):  # noqa: F811
    c = _case([(50, 20)], 2, 2, 64, 16, "bf16", seed=7)
    both = torch.zeros(20, 2, 4, 64, dtype=torch.bfloat16, device="cuda")
    both[:, 0] = c["q"]
    out, lse = _run(dict(c, q=both[:, 0]), out=both[:, 1])
    B.ivf_check()
    _check(c, both[:, 1], lse)
    assert torch.equal(both[:, 0], c["q"])
    with pytest.raises(B.IvfError, match="share memory"):
        _run(c, out=c["q"])


def test_tensors_that_carry_gradients_are_refused():
    c = _case([(10, 4)], 1, 2, 64, 16, "fp16")
    ints = _i32(c["table"]), _i32(c["start"]), _i32(c["lens"])
    slopes = torch.ones(2, device="cuda", requires_grad=True)
    for q, more in ((c["q"].clone().requires_grad_(), {}), (c["q"], {"slopes": slopes})):
        with pytest.raises(ValueError, match="gradients"):
            B.ivf_kv_attend_chunk(q, c["kc"], c["vc"], *ints, 1.0, **more)
        with torch.no_grad():
            B.ivf_kv_attend_chunk(q, c["kc"], c["vc"], *ints, 1.0, **more)
    with pytest.raises(ValueError, match="gradients"):
        B.ivf_kv_copy(c["kc"].clone().requires_grad_(), c["vc"], _i32([0]), _i32([1]))


def test_written_tensors_count_a_version():
    c = _case([(10, 4)], 1, 2, 64, 16, "fp16")
    table, lens = _i32(c["table"]), _i32(c["lens"])
    out = torch.empty_like(c["q"])
    was = out._version, c["kc"]._version, table._version
    _run(c, out=out)
    B.ivf_kv_copy(c["kc"], c["vc"], _i32([0]), _i32([1]))
    B.ivf_kv_compact(table, lens, 4, 16)
    assert out._version > was[0] and c["kc"]._version > was[1] and table._version > was[2]
    with torch.inference_mode():
        B.ivf_kv_copy(c["kc"].clone(), c["vc"].clone(), _i32([0]), _i32([1]))


def test_shapes_that_do_not_fit_are_refused():
    c = _case([(10, 4)], 1, 2, 64, 16, "fp16")
    table, start, lens = _i32(c["table"]), _i32(c["start"]), _i32(c["lens"])
    call = lambda **k: B.ivf_kv_attend_chunk(*[{**dict(q=c["q"], kc=c["kc"], vc=c["vc"], t=table, s=start, n=lens), **k}[x] for x in ("q", "kc", "vc", "t", "s", "n")], 1.0)  # noqa: E731
    for bad in ({"s": start[:1]}, {"n": torch.cat([lens, lens])}, {"s": start.long()}, {"vc": c["vc"][1:]}, {"q": c["q"].float()}, {"q": c["q"][:, :, :48]}, {"t": table[0]}):
        with pytest.raises((ValueError, TypeError)):
            call(**bad)
    for more in ({"slopes": torch.ones(3, device="cuda")}, {"prefix": _i32([1, 2])}, {"out": c["q"][:2].clone()}):
        with pytest.raises(ValueError):
            B.ivf_kv_attend_chunk(c["q"], c["kc"], c["vc"], table, start, lens, 1.0, **more)
    with pytest.raises(ValueError):
        B.ivf_kv_fork(table, lens, lens, lens[:0], 10, 16)
    with pytest.raises(ValueError):
        B.ivf_kv_compact(table, lens, 10, 16, out=table[:, :1])
    with pytest.raises(ValueError, match="both or neither"):
        B.ivf_kv_copy(c["kc"], c["vc"], lens, lens, codes=torch.zeros(c["kc"].shape[0], 1, 64, dtype=torch.int8, device="cuda"))


def test_many_items_and_few_keys_to_a_span(kernel):  # noqa: F811
    # more items than blocks of threads, and requests without new tokens in between
    lengths = [(int(a), int(b)) for a, b in np.stack([np.arange(500) * 7 % 60, np.arange(500) % 3], 1)]
    c = _case(lengths, 2, 4, 64, 16, "bf16", seed=8)
    out, lse = _run(c)
    B.ivf_check()
    _check(c, out, lse)


def test_one_long_request_among_many_short_ones(kernel):  # noqa: F811
    c = _case([(3, 1)] * 40 + [(20000, 2)] + [(9, 2)] * 30, 1, 4, 64, 64, "fp16", seed=9)
    out, lse = _run(c)
    B.ivf_check()
    _check(c, out, lse)


def test_forked_rows_attend_to_shared_pages(kernel):  # noqa: F811
    """Rows of the table that name the same pages are read like any others."""
    c = _case([(200, 0), (0, 0), (0, 0)], 2, 2, 64, 16, "bf16", seed=10, spare=8)
    pages = c["kc"].shape[0]
    fork = B.ivf_kv_fork(_i32(c["table"]), _i32(c["lens"]), _i32([0, 0, 0]), _i32([200, 200, 96]), pages, 16)
    B.ivf_kv_copy(c["kc"], c["vc"], fork.copy_from, fork.copy_to, fork.copy_fill)
    q = torch.randn(6, 4, 64, device="cuda", generator=_gen(1)).to(torch.bfloat16)
    out, lse = B.ivf_kv_attend_chunk(q, c["kc"], c["vc"], fork.table, _i32([0, 2, 4, 6]), fork.kv_lens, 0.125, want_lse=True)
    B.ivf_check()
    now = dict(c, q=q, table=_np(fork.table), start=np.array([0, 2, 4, 6]), lens=_np(fork.kv_lens), scale=0.125)
    _check(now, out, lse)
    first = W.attend_chunk(_np(q)[:2], _finite(_np(c["kc"])), _finite(_np(c["vc"])), c["table"][:1], [0, 2], [200], 0.125)[0]
    assert np.abs(_np(out)[:2] - first).max() < 0.05


def test_a_fork_that_ends_in_a_missing_block():
    table = _i32([[3, -1, 2], [5, 6, -1]])
    got = B.ivf_kv_fork(table, _i32([40, 20]), _i32([0, 1, 0]), _i32([20, 20, 40]), 9, 16)
    want = W.fork(_np(table), np.array([40, 20]), np.array([0, 1, 0]), np.array([20, 20, 40]), 9, 16)
    for name, value in want.items():
        assert (_np(getattr(got, name)) == value).all(), name
    B.ivf_check()
    assert not math.isnan(float(got.n_free))
