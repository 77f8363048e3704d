"""How ivf_kv_attend_chunk shares its work out, on the host: every tile of tokens of every kv head is taken, each of its keys once, by neighbouring
blocks of threads that know of each other, and what a tile reads is what its tokens see."""
import ctypes

import numpy as np
import pytest

from paper_2608_08751_b200 import binding as B

ROWS = ("cta", "b", "hv", "token", "tokens", "pos", "k0", "k1", "first", "last", "parts")


def _spans(start, lens, n_tokens=None, heads=4, kv=1, dim=64, page=16, blocks=None, window=0, prefix=None, tiles=0, sms=148):
    i32 = lambda a: np.ascontiguousarray(a, np.int32)  # noqa: E731
    start, lens = i32(start), i32(lens)
    prefix = None if prefix is None else i32(prefix)
    blocks = blocks or max(1, -(-int(max(lens.max(initial=1), 1)) // page))
    at = lambda a: None if a is None else a.ctypes.data  # noqa: E731
    cache = ctypes.byref(B._KvCache(None, None, (ctypes.c_int64 * 3)(), (ctypes.c_int64 * 3)(), 1, page, kv, dim, B.IVF_BF16))
    info = np.zeros(4, np.int64)
    out = np.zeros((0, 11), np.int64)
    while True:
        rc = B.lib().ivf_debug_kv_chunk_spans(int(start[-1]) if n_tokens is None else n_tokens, heads, cache, len(lens), blocks, at(start), at(lens), window,
                                              at(prefix), tiles, sms, at(out), len(out), at(info))
        assert rc == B.IVF_OK, B.lib().ivf_last_error()
        if info[0] <= len(out):
            return dict(zip(ROWS, out[: info[0]].T)), {"ctas": int(info[1]), "tile": int(info[2]), "line": int(info[3])}
        out = np.zeros((info[0], 11), np.int64)


def _seen(pos, n, window, prefix, room):
    """One token's keys, as the definition has them: k < n, k <= pos or k < prefix, pos - k < window, and columns that exist."""
    k = np.arange(min(n, room))
    see = (k <= pos) | (k < prefix)
    if window:
        see &= pos - k < window
    return k[see]


def _check(start, lens, n_tokens=None, heads=4, kv=1, page=16, blocks=None, window=0, prefix=None, tiles=0, brute=True, **more):
    got, info = _spans(start, lens, n_tokens, heads, kv, page=page, blocks=blocks, window=window, prefix=prefix, tiles=tiles, **more)
    n_tokens = int(start[-1]) if n_tokens is None else n_tokens
    room = (blocks or max(1, -(-int(max(max(lens), 1)) // page))) * page
    group, rows = heads // kv, 128 if tiles else 16
    hvs = kv * -(-group // rows)
    assert (np.diff(got["cta"]) >= 0).all()
    # a block's list: whole items but for its first and last on the line; with large tiles the end of a cut one comes last
    n = len(got["cta"])
    opens, ends = np.ones(n, bool), np.ones(n, bool)
    opens[1:] = got["cta"][1:] != got["cta"][:-1]
    ends[:-1] = opens[1:]
    assert (got["first"].astype(bool) | opens | (ends if tiles else False)).all()
    if not tiles:
        assert (got["last"].astype(bool) | ends).all()
    # items in order of the line, their parts by blocks
    order = np.lexsort((got["cta"], got["token"], got["hv"], got["b"]))
    g = {k: v[order] for k, v in got.items()}
    new = np.ones(n, bool)
    new[1:] = (g["b"][1:] != g["b"][:-1]) | (g["hv"][1:] != g["hv"][:-1]) | (g["token"][1:] != g["token"][:-1])
    assert (g["first"].astype(bool) == new).all() and (g["last"][:-1].astype(bool) == new[1:]).all() and (n == 0 or g["last"][-1] == 1)
    assert (~new[1:] <= ((g["cta"][1:] == g["cta"][:-1] + 1) & (g["k0"][1:] == g["k1"][:-1]))).all() and (g["k1"] >= g["k0"]).all()
    where = np.flatnonzero(new)
    count = np.diff(np.append(where, n))
    assert (g["parts"][where] == np.where(count > 1, count, 0)).all()
    # every tile of every request, and the keys it has
    want = []
    for b in range(len(lens)):
        s0, s1, length = int(start[b]), int(start[b + 1]), int(lens[b])
        if s1 <= s0:
            continue
        end = min(s1, n_tokens)
        for hv in range(hvs):
            for t in range(s0, end, info["tile"]):
                want.append((b, hv, t, min(info["tile"], end - t), length - (s1 - s0) + t - s0))
    have = np.stack([g[k][where] for k in ("b", "hv", "token", "tokens", "pos")], 1) if n else np.zeros((0, 5), int)
    want = np.array(want, np.int64).reshape(-1, 5)
    seeing = lens[want[:, 0]] >= (np.array(start)[1:] - np.array(start)[:-1])[want[:, 0]] if len(want) else np.zeros(0, bool)
    assert have.shape == want.shape and (have[:, :4] == want[:, :4]).all() and (have[seeing, 4] == want[seeing, 4]).all()
    lo, hi = g["k0"][where], g["k1"][where + count - 1]
    assert (hi[~seeing] <= lo[~seeing]).all()
    for i in np.flatnonzero(seeing):
        b, _, _, tokens, pos = want[i]
        p = 0 if prefix is None else max(0, int(prefix[b]))
        if brute:
            keys = np.concatenate([_seen(pos + t, int(lens[b]), window, p, room) for t in range(tokens)])
            assert (lo[i], hi[i]) == (keys.min(), keys.max() + 1) if len(keys) else hi[i] <= lo[i]
        else:
            top = min(max(pos + tokens, min(p, int(lens[b]))), room)
            assert hi[i] == top and lo[i] == min(top, max(0, pos - window + 1) if window else 0)
    return info


@pytest.mark.parametrize("tiles", [0, 1], ids=["rows", "tiles"])
def test_random_batches(tiles):
    rng = np.random.default_rng(tiles)
    for _ in range(250):
        n = int(rng.integers(1, 60 if rng.random() < 0.1 else 7))
        most = int(rng.choice([2, 20, 600]))
        fresh = np.where(rng.random(n) < 0.12, 0, rng.integers(1, most + 1, n))
        lens = fresh + rng.integers(0, int(rng.choice([60, 3000])), n)
        lens = np.where(rng.random(n) < 0.04, fresh - 1, lens)  # (fewer tokens in the cache than new ones)
        start = np.concatenate([[int(rng.integers(0, 3))], fresh]).cumsum()
        page = int(rng.choice([16, 32, 64, 128]))
        blocks = max(1, -(-int(max(lens.max(), 1)) // page) - (int(rng.integers(1, 4)) if rng.random() < 0.2 else 0))
        kv = int(rng.integers(1, 4))
        _check(start, lens, int(start[-1]) - (int(rng.integers(0, min(5, start[-1] + 1))) if rng.random() < 0.2 else 0), kv * int(rng.integers(1, 24)), kv, page, blocks,
               int(rng.choice([0, 0, 1, 40, 2000])), rng.integers(-2, lens.max() + 5, n) if rng.random() < 0.5 else None, tiles,
               dim=int(rng.choice([64, 128, 256])), sms=int(rng.choice([1, 7, 148])))


@pytest.mark.parametrize("tiles", [0, 1], ids=["rows", "tiles"])
@pytest.mark.parametrize("window,prefix", [(0, False), (5000, False), (0, True)])
def test_lines_past_32_bits(tiles, window, prefix):
    rng = np.random.default_rng(7)
    lens = np.concatenate([[2 ** 31 - 1, 2 ** 31 - 1, 1], rng.integers(1 << 20, 1 << 30, 60)])
    fresh = np.minimum(rng.integers(1, 3000, 63), lens)
    info = _check(np.concatenate([[0], fresh]).cumsum(), lens, heads=8, kv=2, page=128, window=window, prefix=lens // 3 * 2 if prefix else None, tiles=tiles, brute=False)
    assert info["line"] > 2 ** 32 or window
    assert info["ctas"] == 148 * (1 if tiles else 3)


@pytest.mark.parametrize("tiles", [0, 1], ids=["rows", "tiles"])
def test_as_many_requests_as_there_may_be(tiles):
    rng = np.random.default_rng(8)
    fresh = np.where(rng.random(16384) < 0.7, 1, rng.integers(0, 4, 16384))
    lens = fresh + rng.integers(0, 500000, 16384)
    info = _check(np.concatenate([[0], fresh]).cumsum(), lens, heads=4, kv=1, page=16, tiles=tiles, brute=False)
    assert info["line"] > 2 ** 31
    info = _check(np.zeros(16385, np.int64), lens, tiles=tiles)
    assert info["ctas"] == 1 and info["line"] == 0


@pytest.mark.parametrize("tiles", [0, 1], ids=["rows", "tiles"])
@pytest.mark.parametrize("start", [[0, 10, 8, 19], [0, 5, 3], [5, 3, 9], [4, 4, 2, 2, 9, 1, 30], [-3, 4, 9], [0, 40, 0, 40, 0, 40, 12, 90], [7, -2 ** 31, 5]], ids=str)
def test_a_row_belongs_to_one_request_where_token_start_descends(tiles, start):
    """The first request whose rows reach a row has it, at the position that it has there."""
    n = len(start) - 1
    lens = np.array([60 + 7 * b for b in range(n)])
    n_tokens = max(start) + 3
    got, info = _spans(start, lens, n_tokens, heads=6, kv=2, tiles=tiles)
    owner, pos = {}, {}
    for b in range(n):
        for t in range(max(start[b], 0), start[b + 1]):
            if t >= start[0] and t not in owner:
                owner[t], pos[t] = b, lens[b] - (start[b + 1] - start[b]) + t - start[b]
    for hv in range(2):
        seen = {}
        for i in np.flatnonzero((got["hv"] == hv) & (got["first"] == 1)):
            for t in range(got["tokens"][i]):
                row = int(got["token"][i]) + t
                assert row not in seen, (row, "has two requests")
                seen[row] = int(got["b"][i])
                assert seen[row] == owner[row] and got["pos"][i] + t == pos[row]
        assert seen.keys() == owner.keys()


def test_refusals():
    cache = ctypes.byref(B._KvCache(None, None, (ctypes.c_int64 * 3)(), (ctypes.c_int64 * 3)(), 1, 16, 1, 64, B.IVF_BF16))
    a = np.zeros(8, np.int64)
    call = lambda n=1, heads=1, req=1, blocks=1, start=a.ctypes.data, window=0, sms=1, most=0: B.lib().ivf_debug_kv_chunk_spans(  # noqa: E731
        n, heads, cache, req, blocks, start, a.ctypes.data, window, None, 0, sms, None, most, a.ctypes.data)
    assert call() == B.IVF_OK
    for bad in ({"n": -1}, {"heads": 0}, {"req": -1}, {"blocks": 0}, {"start": None}, {"window": -1}, {"sms": 0}, {"most": 1}):
        assert call(**bad) == B.IVF_ERR_INVALID_ARG, bad
