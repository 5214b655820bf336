"""The paged 8-bit cache on the GPU against its definition: page tables and slots
exactly, stored values and scales exactly, read-back exactly."""
import math

import numpy as np
import pytest
import torch

import _q8_ref as R
from paper_2602_07397_amd import binding as sw

pytestmark = pytest.mark.gpu

U = pytest.importorskip("_gpu_util")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=U.DEV)


# --------------------------------------------------------------------------- tables


class _Requests:
    """A pool and its requests, on the device and as lists."""

    def __init__(self, n, B, b_max, n_pages, seed):
        self.B, self.b_max, self.n_pages = B, b_max, n_pages
        self.rng = np.random.default_rng(seed)
        self.stack = self.rng.permutation(n_pages).tolist()
        self.tables = [[-1] * b_max for _ in range(n)]
        self.lens = [0] * n
        self.d_tables = torch.full((n, b_max), -1, dtype=torch.int32, device=U.DEV)
        self.d_free, self.d_n = _i32(self.stack), _i32([n_pages])

    def call(self, new, rows=0, extra=0, **kw):
        n_slots = len(new) * rows if rows else sum(max(0, b - a) for a, b in zip(self.lens, new)) + extra
        out = sw.block_tables(_i32(self.lens), _i32(new), self.B, self.d_tables, self.d_free, self.d_n,
                              n_slots, rows=rows, **kw)
        return out, n_slots

    def check(self, new, rows=0, extra=0):
        out, n_slots = self.call(new, rows, extra)
        slots, cu, pos = R.allocate(self.lens, new, self.B, self.tables, self.stack, rows, n_slots)
        assert int(out["status"]) == 0
        assert out["slots"].tolist() == slots
        assert out["cu"].tolist() == cu and out["pos"].tolist() == pos
        assert self.d_tables.tolist() == self.tables
        assert self.d_n.tolist() == [len(self.stack)]
        assert self.d_free[:len(self.stack)].tolist() == self.stack
        self.lens = list(new)
        return out


@pytest.mark.parametrize("n,B,rows", [(1, 64, 0), (5, 16, 0), (64, 64, 1), (63, 80, 3), (1030, 16, 0),
                                      (2100, 128, 1), (2100, 16, 3), (1500, 64, 4)])
def test_tables_over_many_calls(n, B, rows):
    b_max = 12
    r = _Requests(n, B, b_max, n * 8, seed=n + B)
    for step in range(6):
        cap = r.rng.integers(0, 6 * B + 1, size=n)
        if rows:
            new = [int(x + r.rng.integers(0, rows + 1)) if x < 6 * B else 0 for x in r.lens]
            if step % 3 == 2:
                new = [x if k % 3 else 0 for k, x in enumerate(r.lens)]
        else:
            new = [int(c) if r.rng.uniform() < 0.5 else x for c, x in zip(cap, r.lens)]
        r.check(new, rows, extra=7 * (step % 2))


def test_tables_with_many_slots():
    r = _Requests(9, 64, 300, 2000, seed=4)
    r.check([0, 17000, 1, 64, 0, 63, 4000, 65, 128], extra=3)
    r.check([5, 17001, 0, 64, 9000, 64, 4000, 0, 129])
    p = _Requests(3, 16, 400, 1000, seed=5)          # padded rows, many of them
    p.check([5000, 0, 17], rows=5000)
    p.check([1, 5000, 5000], rows=5000)
    r.check([0] * 9, extra=9000)                     # everything back


def test_tables_with_many_slots_that_cannot_be_served():
    r = _Requests(2, 16, 1000, 600, seed=10)
    r.check([100, 0])
    state = (r.d_tables.clone(), r.d_free.clone(), r.d_n.clone())
    for new, n_slots, status in (([9000, 1000], 9900, 1), ([9000, 100], 8000, 2)):
        out = sw.block_tables(_i32(r.lens), _i32(new), 16, r.d_tables, r.d_free, r.d_n, n_slots)
        assert int(out["status"]) == status and out["cu"].tolist() == [0, 0, 0] and out["pos"].tolist() == [99, -1]
        assert torch.all(out["slots"] == -1)
        for a, b in zip(state, (r.d_tables, r.d_free, r.d_n)):
            assert torch.equal(a, b)


def test_a_step_back_restores_tables_and_stack():
    r = _Requests(40, 16, 20, 400, seed=6)
    r.check([int(x) for x in r.rng.integers(0, 150, size=40)])
    before = (list(r.stack), [list(t) for t in r.tables], list(r.lens))
    r.check([x + 1 + k % 30 for k, x in enumerate(r.lens)])
    r.check(before[2])
    assert (r.stack, r.tables, r.lens) == before


@pytest.mark.parametrize("what,status", [("pages", 1), ("long", 2), ("negative", 2), ("slots", 2), ("rows", 2),
                                         ("old", 2)])
def test_tables_calls_that_cannot_be_served_change_nothing(what, status):
    r = _Requests(4, 16, 10, 20, seed=7)
    r.check([30, 0, 16, 50])                         # 7 pages of 20
    state = (r.d_tables.clone(), r.d_free.clone(), r.d_n.clone())
    new, rows, n_slots, old = [31, 5, 20, 50], 0, 10, list(r.lens)
    if what == "pages":
        new, n_slots = [31, 160, 20, 160], 400       # 10 + 1 + 6 pages more than the 13 left
    elif what == "long":
        new = [161, 0, 16, 50]
        n_slots = 200
    elif what == "negative":
        new = [31, -1, 16, 50]
    elif what == "slots":
        n_slots = 9                                  # 10 new tokens
    elif what == "rows":
        rows, n_slots = 4, 16                        # 5 new tokens of request 1
    else:
        old[3] = 161
    out = sw.block_tables(_i32(old), _i32(new), 16, r.d_tables, r.d_free, r.d_n, n_slots, rows=rows)
    assert int(out["status"]) == status
    assert out["slots"].tolist() == [-1] * n_slots and out["cu"].tolist() == [0] * 5
    assert out["pos"].tolist() == [x - 1 for x in old]
    for a, b in zip(state, (r.d_tables, r.d_free, r.d_n)):
        assert torch.equal(a, b)


def test_tables_pages_released_in_a_call_serve_that_call():
    r = _Requests(2, 16, 10, 4, seed=8)
    r.check([64, 0])                                 # all four pages
    r.check([0, 64])
    r.check([32, 32])


def test_tables_captured_replays():
    r = _Requests(8, 16, 40, 300, seed=9)
    r.check([20 * k for k in range(8)])
    lens = [_i32(r.lens), _i32([x + 16 for x in r.lens])]
    out = {"slots": _i32([0] * 128), "cu": _i32([0] * 9), "pos": _i32([0] * 8), "status": _i32([5])}
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        sw.block_tables(lens[0], lens[0], 16, r.d_tables, r.d_free, r.d_n, 128, out=dict(out))   # warm
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sw.block_tables(lens[0], lens[1], 16, r.d_tables, r.d_free, r.d_n, 128, out=dict(out))
    for _ in range(4):                               # each replay grows by 16 and is taken along
        g.replay()
        slots, cu, pos = R.allocate(r.lens, [x + 16 for x in r.lens], 16, r.tables, r.stack, 0, 128)
        assert int(out["status"]) == 0 and out["slots"].tolist() == slots
        assert r.d_tables.tolist() == r.tables and r.d_n.tolist() == [len(r.stack)]
        r.lens = [x + 16 for x in r.lens]
        lens[0].copy_(_i32(r.lens))
        lens[1].copy_(_i32([x + 16 for x in r.lens]))


# --------------------------------------------------------------------------- append


def _rand(rng, h, n, d, dtype, spread=1.0):
    x = rng.normal(size=(h, n, d)) * np.exp2(np.round(rng.normal(size=(h, n, 1)) * spread))
    t = torch.from_numpy(x).to(dtype)
    return t, t.double().numpy()


def _same_cache(cache, pool, pages=None):
    x, e = R.cache_values(cache)
    for n in "kv":
        want_e, want = pool.e[n], pool.x[n]
        if pages is not None:
            assert np.array_equal(e[n][pages], want_e[pages]), n
            np.testing.assert_array_equal(x[n][pages], want[pages])
        else:
            assert np.array_equal(e[n], want_e), n
            np.testing.assert_array_equal(x[n], want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("h,B,d", [(1, 16, 64), (3, 64, 128), (2, 80, 64), (2, 1024, 128), (8, 128, 128)])
def test_append_in_pieces(dtype, h, B, d):
    """Sequences that grow by prompts, ragged pieces and single tokens, each piece
    larger than the one before now and then: every stored value and scale exactly."""
    rng = np.random.default_rng(B + d)
    n, b_max = 3, max(2, 300 // B + 1)
    r = _Requests(n, B, b_max, n * b_max + 4, seed=B)
    cache = sw.new_cache_q8(r.n_pages, h, B, d, U.DEV)
    pool = R.Pool(r.n_pages, h, B, d)
    steps = [[B // 2 + 3, 2 * B if B < 200 else 150, 1], [B // 2 + 4, 2 * B if B < 200 else 150, 2],
             [B + 5, 2 * B + 1 if B < 200 else 180, 0], [B + 21, 2 * B + 2 if B < 200 else 181, 17]]
    for i, new in enumerate(steps):
        N = sum(max(0, b - a) for a, b in zip(r.lens, new))
        out = r.check(new)
        k, k64 = _rand(rng, h, N, d, dtype)
        v, v64 = _rand(rng, h, N, d, dtype)
        k, v = k * 2.0 ** (2 * i), v * 2.0 ** (-3 * i)
        sw.kv_append_q8(k.to(U.DEV), v.to(U.DEV), out["slots"], cache, cu=out["cu"])
        pool.append(k64 * 2.0 ** (2 * i), v64 * 2.0 ** (-3 * i), out["slots"].tolist())
        _same_cache(cache, pool)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_tokens_without_sequences(dtype):
    """Decode: a token per sequence, idle ones, several tokens of one page in one call,
    one slot twice (the later stays), slots outside the pool."""
    rng = np.random.default_rng(3)
    h, B, d, P = 4, 32, 128, 12
    cache = sw.new_cache_q8(P, h, B, d, U.DEV)
    pool = R.Pool(P, h, B, d)
    calls = [[0, 32, 64, -1, 5 * 32, 330], [1, 33, -1, -1, 5 * 32 + 1, 331], [2, 3, 4, 36, 35, 34, 34, -1, 12 * 32, 1 << 30],
             [383, 95, 7], [6 * 32 + 5, 6 * 32, 6 * 32 + 9]]
    for i, slots in enumerate(calls):
        k, k64 = _rand(rng, h, len(slots), d, dtype, 2.0)
        v, v64 = _rand(rng, h, len(slots), d, dtype, 2.0)
        sw.kv_append_q8(k.to(U.DEV), v.to(U.DEV), _i32(slots), cache)
        pool.append(k64, v64, slots)
        _same_cache(cache, pool)


def test_append_takes_strided_rows_and_many_tokens():
    rng = np.random.default_rng(5)
    h, B, d, N = 4, 64, 64, 4096                     # the most that goes without sequences
    P = N // B + 3
    slots = rng.permutation(P * B)[:N].astype(np.int32)
    qkv = torch.from_numpy(rng.normal(size=(N, 3, h, d))).to(torch.bfloat16).to(U.DEV)
    k, v = qkv[:, 1].transpose(0, 1), qkv[:, 2].transpose(0, 1)
    assert not k.is_contiguous()
    cache = sw.new_cache_q8(P, h, B, d, U.DEV)
    sw.kv_append_q8(k, v, torch.from_numpy(slots).to(U.DEV), cache)
    pool = R.Pool(P, h, B, d)
    pool.append(k.cpu().double().numpy(), v.cpu().double().numpy(), slots.tolist())
    _same_cache(cache, pool)


def test_append_of_one_token_or_head_in_any_stride():
    rng = np.random.default_rng(15)
    B, d, P = 16, 64, 3
    for h, N, shape, stride in ((1, 5, (1, 5, d), (3, d, 1)), (3, 1, (3, 1, d), (d, 5, 1))):
        base = torch.from_numpy(rng.normal(size=h * N * d)).float().to(U.DEV)
        k = torch.as_strided(base, shape, stride)
        v = torch.as_strided(base, shape, stride)
        slots = [20 + i for i in range(N)]
        cache, pool = sw.new_cache_q8(P, h, B, d, U.DEV), R.Pool(P, h, B, d)
        sw.kv_append_q8(k, v, _i32(slots), cache)
        pool.append(k.cpu().double().numpy(), v.cpu().double().numpy(), slots)
        _same_cache(cache, pool)


def test_append_sequences_that_are_skipped_or_empty():
    rng = np.random.default_rng(6)
    h, B, d, P = 2, 16, 64, 30
    cache, pool = sw.new_cache_q8(P, h, B, d, U.DEV), R.Pool(P, h, B, d)
    lens = [0, 40, 0, 1, 17, 0, 33]
    cu = np.concatenate([[0], np.cumsum(lens)])
    starts = [0, 5, 0, 15, -1, 0, 0]                 # the fifth sequence has no page
    slots, page = [], 0
    for n, a in zip(lens, starts):
        slots += [-1] * n if a < 0 else [page * B + a + i for i in range(n)]
        page += 0 if a < 0 or n == 0 else -(-(a + n) // B)
    extra = 5                                        # rows behind the last sequence
    k, k64 = _rand(rng, h, len(slots) + extra, d, torch.bfloat16)
    v, v64 = _rand(rng, h, len(slots) + extra, d, torch.bfloat16)
    sw.kv_append_q8(k.to(U.DEV), v.to(U.DEV), _i32(slots + [0] * extra), cache, cu=_i32(cu.tolist()))
    pool.append(k64[:, :len(slots)], v64[:, :len(slots)], slots)
    _same_cache(cache, pool)
    before = {n: t.clone() for n, t in cache.items()}
    empty = torch.zeros((h, 0, d), dtype=torch.bfloat16, device=U.DEV)
    sw.kv_append_q8(empty, empty, _i32([]), cache, cu=_i32([0, 0]))
    sw.kv_append_q8(empty, empty, _i32([]), cache)
    for n in cache:
        assert torch.equal(before[n].view(torch.uint8), cache[n].view(torch.uint8))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_of_extreme_values(dtype):
    """Values at every code and tie, zeros, the ends of the range, infinities and NaN;
    a scale that grows by more than the codes' range."""
    h, B, d, P = 1, 16, 64, 9
    cache, pool = sw.new_cache_q8(P, h, B, d, U.DEV), R.Pool(P, h, B, d)
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    codes = np.sort(codes[np.isfinite(codes)])
    ties = (codes[1:] + codes[:-1]) / 2
    big = float(torch.finfo(dtype).max)
    tiny = float(torch.finfo(dtype).tiny)

    def page(vals):
        x = np.zeros(B * d)
        x[:len(vals)] = vals
        return x.reshape(1, B, d)

    rows = [(page(codes), list(range(0, 16))), (page(ties), list(range(16, 32))),
            (page(np.concatenate([ties * 2.0 ** -100, [448 * 2.0 ** -100]])), list(range(32, 48))),
            (page([]), list(range(48, 64))), (page([big, -big, 1.0, tiny]), list(range(64, 80))),
            (page([np.inf, -np.inf, np.nan, 3.0, -0.0]), list(range(80, 96))),
            (page([tiny, -tiny, 3 * tiny]), list(range(96, 112))),
            # below the smallest normal number, where the smallest scale still has codes
            (page(tiny * np.exp2(-np.arange(9.0)) * 1.5), list(range(128, 144)))]
    for x, slots in rows:
        t = torch.from_numpy(x).to(dtype)
        t64 = t.double().numpy()
        sw.kv_append_q8(t.to(U.DEV), (-t).to(U.DEV), _i32(slots), cache)
        pool.append(t64, -t64, slots)
        _same_cache(cache, pool)
    # a page of small values, then one token 2^60 times as large, then a small one again
    for i, (m, slots) in enumerate(((2.0 ** -40, list(range(112, 120))), (2.0 ** 20, [120]), (2.0 ** 12, [121]))):
        x = np.random.default_rng(i).normal(size=(1, len(slots), d)) * m
        t = torch.from_numpy(x).to(dtype)
        sw.kv_append_q8(t.to(U.DEV), t.to(U.DEV), _i32(slots), cache)
        pool.append(t.double().numpy(), t.double().numpy(), slots)
        _same_cache(cache, pool)


def test_begun_page_leaves_its_other_places():
    h, B, d = 1, 16, 64
    cache = sw.new_cache_q8(2, h, B, d, U.DEV)
    cache["k"].view(torch.uint8).random_(0, 256)
    cache["v"].view(torch.uint8).random_(0, 256)
    before = {n: t.clone().view(torch.uint8) for n, t in cache.items()}
    x = torch.randn((h, 3, d), device=U.DEV)
    sw.kv_append_q8(x, x, _i32([16, 17, 18]), cache)
    k, v = cache["k"].view(torch.uint8), cache["v"].view(torch.uint8)
    assert torch.equal(k[0], before["k"][0]) and torch.equal(v[0], before["v"][0])
    assert torch.equal(k[1, :, 3:], before["k"][1, :, 3:]) and torch.equal(v[1, :, :, 3:], before["v"][1, :, :, 3:])
    assert not torch.equal(k[1, :, :3], before["k"][1, :, :3])


# --------------------------------------------------------------------------- fetch


def _filled(rng, P, h, B, d):
    cache = sw.new_cache_q8(P, h, B, d, U.DEV)
    for n in "kv":
        cache[n].copy_(torch.from_numpy(rng.normal(size=cache[n].shape) * 50).clamp(-448, 448).to(torch.float8_e4m3fn))
        cache[n + "_scale"].copy_(torch.from_numpy(rng.integers(100, 140, size=(P, h))).to(torch.uint8))
    return cache


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("h,B,d", [(2, 16, 64), (4, 64, 128), (3, 80, 128), (1, 1024, 64)])
def test_fetch(dtype, h, B, d):
    rng = np.random.default_rng(B)
    lens, first = [2 * B + 7, 0, 1, B, 33], [B - 1, 4, 2 * B, 0, B // 2]
    b_max = max(-(-(a + n) // B) for a, n in zip(first, lens))
    P = 40
    cache = _filled(rng, P, h, B, d)
    tables = rng.permutation(P)[:5 * b_max].reshape(5, b_max).astype(np.int32)
    tables[0, 1] = -1                                # blocks without a page, and behind the pool
    tables[4, b_max - 1] = P
    cu = [0] + np.cumsum(lens).tolist()
    N = cu[-1] + 9
    out = tuple(torch.full((h, N, d), 7.0, dtype=dtype, device=U.DEV) for _ in range(2))
    K, V = sw.kv_fetch_q8(cache, torch.from_numpy(tables).to(U.DEV), _i32(first), _i32(cu), N, out=out)
    x, e = R.cache_values(cache)
    pool = R.Pool(P, h, B, d)
    pool.x = x
    for got, n in ((K, "k"), (V, "v")):
        got = got.cpu().double().numpy()
        for s, (a, m) in enumerate(zip(first, lens)):
            np.testing.assert_array_equal(got[:, cu[s]:cu[s + 1]], pool.tokens(n, tables[s], list(range(a, a + m))))
        assert np.all(got[:, cu[-1]:] == 7.0)        # rows behind the last sequence stay
    K0, _ = sw.kv_fetch_q8(cache, torch.from_numpy(tables).to(U.DEV), None, _i32([0, 1, 1, 1, 1, 1]), 1, dtype=dtype)
    np.testing.assert_array_equal(K0.cpu().double().numpy(), pool.tokens("k", tables[0], [0]))


@pytest.mark.parametrize("n", [63, 65, 129, 4097, 5000])
def test_many_sequences(n):
    """Append and fetch over more sequences than a wavefront looks at once, most of them short or empty."""
    rng = np.random.default_rng(n)
    h, B, d = 1, 16, 64
    lens = rng.choice([0, 0, 1, 2, 17, 40], size=n)
    lens[[0, -1]] = [0, 33]
    starts = rng.integers(0, B, size=n)
    blocks = -(-(starts + lens) // B) * (lens > 0)
    cu = np.concatenate([[0], np.cumsum(lens)])
    first = np.concatenate([[0], np.cumsum(blocks)])
    P, N = int(first[-1]), int(cu[-1])
    pages = rng.permutation(P)
    tables = np.full((n, 4), -1, dtype=np.int32)
    slots = []
    for s in range(n):
        tables[s, :blocks[s]] = pages[first[s]:first[s + 1]]
        slots += [int(tables[s, p // B]) * B + p % B for p in range(starts[s], starts[s] + lens[s])]
    cache, pool = sw.new_cache_q8(P, h, B, d, U.DEV), R.Pool(P, h, B, d)
    k, k64 = _rand(rng, h, N, d, torch.bfloat16)
    v, v64 = _rand(rng, h, N, d, torch.bfloat16)
    d_cu = _i32(cu.tolist())
    sw.kv_append_q8(k.to(U.DEV), v.to(U.DEV), _i32(slots), cache, cu=d_cu)
    pool.append(k64, v64, slots)
    _same_cache(cache, pool)
    K, V = sw.kv_fetch_q8(cache, U.to_dev(tables), _i32(starts.tolist()), d_cu, N, dtype=torch.float32)
    x, _ = R.cache_values(cache)
    pg, o = np.array(slots) // B, np.array(slots) % B
    assert np.array_equal(K.cpu().double().numpy(), x["k"][pg, :, o].transpose(1, 0, 2))
    assert np.array_equal(V.cpu().double().numpy(), x["v"][pg, :, o].transpose(1, 0, 2))


def test_fetch_of_every_scale():
    """Codes times the smallest and the largest scales: exact in fp32; in bf16 exact from
    2^-133 on, its smallest number (below, rounded to a multiple of it)."""
    P, h, B, d = 254, 1, 16, 64
    cache = sw.new_cache_q8(P, h, B, d, U.DEV)
    codes = torch.arange(256, dtype=torch.uint8)
    codes[[127, 255]] = 0                            # NaN
    for n in "kv":
        cache[n].view(torch.uint8).copy_(codes.repeat(P * B * d // 256).reshape(cache[n].shape))
        cache[n + "_scale"].copy_(torch.arange(1, 255, dtype=torch.uint8)[:, None])
    x, _ = R.cache_values(cache)
    tables, cu = torch.arange(P, dtype=torch.int32, device=U.DEV)[None], _i32([0, P * B])
    top = float(torch.finfo(torch.float32).max)
    for dtype, step in ((torch.float32, 2.0 ** -149), (torch.bfloat16, 2.0 ** -133)):
        K, V = sw.kv_fetch_q8(cache, tables, None, cu, P * B, dtype=dtype)
        for got, n in ((K, "k"), (V, "v")):
            want = x[n].transpose(1, 0, 2, 3).reshape(h, P * B, d)
            want = np.where(np.abs(want) < 2.0 ** -118, np.rint(want / step) * step, want)
            want = np.where(np.abs(want) > top, np.sign(want) * np.inf, want)
            np.testing.assert_array_equal(got.cpu().double().numpy(), want)


def test_append_then_fetch_on_another_stream():
    rng = np.random.default_rng(11)
    h, B, d, N = 8, 64, 128, 1000
    P = N // B + 1
    k, k64 = _rand(rng, h, N, d, torch.bfloat16)
    v, v64 = _rand(rng, h, N, d, torch.bfloat16)
    kd, vd = k.to(U.DEV), v.to(U.DEV)
    cache, pool = sw.new_cache_q8(P, h, B, d, U.DEV), R.Pool(P, h, B, d)
    pool.append(k64, v64, list(range(N)))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        sw.kv_append_q8(kd, vd, torch.arange(N, dtype=torch.int32, device=U.DEV), cache, cu=_i32([0, N]))
        K, V = sw.kv_fetch_q8(cache, torch.arange(P, dtype=torch.int32, device=U.DEV)[None], None, _i32([0, N]), N)
    torch.cuda.current_stream().wait_stream(s)
    np.testing.assert_array_equal(K.cpu().double().numpy(), pool.tokens("k", list(range(P)), list(range(N))))
    np.testing.assert_array_equal(V.cpu().double().numpy(), pool.tokens("v", list(range(P)), list(range(N))))
    # a stored value is off by at most half a step of its code
    e = pool.e["k"][np.arange(N) // B].T[..., None].astype(np.float64)
    assert np.all(np.abs(K.cpu().double().numpy() - k64) <= np.maximum(np.abs(k64) * 2.0 ** -4, np.exp2(e - 10)))


def test_binding_refuses_tensors_that_do_not_fit():
    h, B, d, P, N = 2, 16, 64, 4, 8
    cache = sw.new_cache_q8(P, h, B, d, U.DEV)
    x = torch.zeros((h, N, d), device=U.DEV)
    slots = torch.arange(N, dtype=torch.int32, device=U.DEV)
    tables, cu = _i32([[0, 1]]), _i32([0, N])
    for what, call in {
        "dtype": lambda: sw.kv_append_q8(x.half(), x.half(), slots, cache),
        "share": lambda: sw.kv_append_q8(x, x.bfloat16(), slots, cache),
        "shape": lambda: sw.kv_append_q8(x[:, :4], x, slots, cache),
        "last dimension": lambda: sw.kv_append_q8(x.transpose(1, 2).contiguous().transpose(1, 2), x, slots, cache),
        "stride": lambda: sw.kv_append_q8(torch.zeros((h, N, d + 1), device=U.DEV)[..., :d], x, slots, cache),
        "slots": lambda: sw.kv_append_q8(x, x, slots.long(), cache),
        "on cpu": lambda: sw.kv_append_q8(x.cpu(), x, slots, cache),
        "cache k": lambda: sw.kv_append_q8(x, x, slots, {**cache, "k": cache["k"].view(torch.uint8)}),
        "n_pages": lambda: sw.kv_append_q8(x, x, slots, {**cache, "v": cache["v"][:3]}),
        "cu": lambda: sw.kv_fetch_q8(cache, tables, None, cu[:1], N),
        "first": lambda: sw.kv_fetch_q8(cache, tables, _i32([0, 0]), cu, N),
        "of shape": lambda: sw.kv_fetch_q8(cache, tables, None, cu, N, out=(x[:1], x)),
        "V must": lambda: sw.kv_fetch_q8(cache, tables, None, cu, N, out=(x, x.bfloat16())),
        "N=": lambda: sw.kv_fetch_q8(cache, tables, None, cu, -1),
        "new_len": lambda: sw.block_tables(_i32([0]), _i32([0, 0]), B, tables, _i32([2, 3]), _i32([2]), 4),
        "contiguous": lambda: sw.block_tables(_i32([0]), _i32([3]), B, _i32([[0, 1], [2, 3]]).t()[:1], _i32([2, 3]),
                                              _i32([2]), 4),
    }.items():
        with pytest.raises(sw.SketchWalkError, match=what):
            call()
    q = torch.zeros((1, 4, d), device=U.DEV)
    args = dict(tables=tables, pos=_i32([5]), idx=_i32([[0]]), cnt=_i32([1]), kmax=1)
    ok = sw.sparse_attn_decode_q8(q, cache, **args)
    assert torch.equal(ok, q)                        # an empty cache: zero values
    for what, change in {"idx": dict(idx=_i32([[0, 1]])), "pos": dict(pos=_i32([5, 5])), "kmax": dict(kmax="1"),
                         "tables": dict(tables=_i32([0, 1])), "workspace": dict(workspace=torch.zeros(1 << 20, device=U.DEV)),
                         "O of": dict(O=torch.zeros((1, 2, d), device=U.DEV)),
                         "O must": dict(O=torch.zeros((1, 4, d), dtype=torch.bfloat16, device=U.DEV)),
                         "cnt": dict(cnt=torch.ones(1, device=U.DEV))}.items():
        with pytest.raises(sw.SketchWalkError, match=what):
            sw.sparse_attn_decode_q8(q, cache, **{**args, **change})
    with pytest.raises(sw.SketchWalkError, match="q of"):
        sw.sparse_attn_decode_q8(q[:, :, :32], cache, **args)


@pytest.mark.parametrize("n_slots", [40, 9000])
@pytest.mark.parametrize("entry", [-1, 600, 1 << 30])
def test_blocks_given_back_need_a_page(n_slots, entry):
    """A request that gives back a block without a page (in one launch, and with slots over many
    workgroups; its block among the first and among the last ones): nothing changes, and no such
    entry gets onto the stack. Blocks that stay may be without one."""
    for n, at in ((2, (0, 3)), (3, (1, 90)), (1500, (1499, 0)), (1500, (700, 2))):
        r = _Requests(n, 16, 100, 600 + n, seed=11)
        lens = [0] * n
        lens[at[0]] = 1599 if n < 10 else 40
        lens[0] = max(lens[0], 70)
        r.check(lens)
        page = int(r.d_tables[at])
        r.d_tables[at] = entry if entry < 600 else entry + n
        state = (r.d_tables.clone(), r.d_free.clone(), r.d_n.clone())
        gone = [0 if s == at[0] else x + 1 for s, x in enumerate(lens)]
        gone = [x if x <= 1600 else 1600 for x in gone]
        out = sw.block_tables(_i32(lens), _i32(gone), 16, r.d_tables, r.d_free, r.d_n, max(n_slots, n))
        assert int(out["status"]) == 2
        assert torch.all(out["slots"] == -1) and torch.all(out["cu"] == 0) and out["pos"].tolist() == [x - 1 for x in lens]
        for a, b in zip(state, (r.d_tables, r.d_free, r.d_n)):
            assert torch.equal(a, b)
        # the request keeps the block: served
        if at[1] > 0:
            keep = list(lens)
            keep[at[0]] = 16 * (at[1] + 1)
            out = sw.block_tables(_i32(lens), _i32(keep), 16, r.d_tables, r.d_free, r.d_n, max(n_slots, n))
            assert int(out["status"]) == 0
            r.lens, r.d_tables[at] = keep, page
            R.allocate(lens, keep, 16, r.tables, r.stack)
        else:
            r.d_tables[at] = page
        r.check([0] * n, extra=n_slots)              # with its page back, everything goes back


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_stored_values_after_their_scale_has_grown(dtype):
    """A page begun with one of 448 and small ones, then larger tokens one by one: each growth
    rounds the codes again, and all of them together stay within 2^-4 of the value or 2^-9 of
    the last scale; within 2^-10 of it while the scale is the first."""
    h, B, d = 1, 32, 128
    cache, pool = sw.new_cache_q8(1, h, B, d, U.DEV), R.Pool(1, h, B, d)
    rng = np.random.default_rng(16)
    x = np.exp2(rng.uniform(-12, 0, size=(h, 16, d))) * np.sign(rng.normal(size=(h, 16, d)))
    x[0, 0, 0], x[0, 0, 1] = 448.0, 2.501 * 2.0 ** -9
    told = torch.from_numpy(x).to(dtype).double().numpy()
    worst = []
    for step in range(7):
        new = told if step == 0 else np.full((h, 1, d), 448.0 * 2.0 ** step)
        slots = list(range(16)) if step == 0 else [15 + step]
        t = torch.from_numpy(new).to(dtype).to(U.DEV)
        sw.kv_append_q8(t, -t, _i32(slots), cache)
        pool.append(new, -new, slots)
        _same_cache(cache, pool)
        scale = 2.0 ** step
        for n, sign in (("k", 1.0), ("v", -1.0)):
            err = np.abs(R.cache_values(cache)[0][n][0, :, :16] - sign * told)
            bound = np.maximum(np.abs(told) * 2.0 ** -4, scale * 2.0 ** (-10 if step == 0 else -9))
            assert np.all(err <= bound), (step, n)
            worst.append(float((err / np.maximum(np.abs(told) * 2.0 ** -4, scale * 2.0 ** -10)).max()))
    assert max(worst[:2]) <= 1.0 < max(worst[2:])    # the second rounding is there


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_largest_finite_values(dtype):
    """Below 1.9375 * 2^127 they are stored as finite ones, from there on as 2^128, which reads
    back as infinity."""
    h, B, d = 1, 16, 64
    cache = sw.new_cache_q8(1, h, B, d, U.DEV)
    edge = 1.9375 * 2.0 ** 127
    step = 2.0 ** 127 * torch.finfo(dtype).eps
    vals = [1.0 * 2.0 ** 127, 1.875 * 2.0 ** 127, edge - step, edge, float(torch.finfo(dtype).max)]
    x = torch.zeros((h, B, d), dtype=torch.float64)
    x[0, 0, :5] = torch.tensor(vals, dtype=torch.float64)
    x[0, 1, :5] = -x[0, 0, :5]
    t = x.to(dtype)
    assert torch.equal(t.double(), x)
    sw.kv_append_q8(t.to(U.DEV), t.to(U.DEV), torch.arange(B, dtype=torch.int32, device=U.DEV), cache)
    for out in sw.kv_fetch_q8(cache, _i32([[0]]), None, _i32([0, B]), B, dtype=dtype):
        want = torch.tensor([vals[0], vals[1], vals[1], math.inf, math.inf], dtype=torch.float64)
        assert torch.equal(out[0, 0, :5].double().cpu(), want) and torch.equal(out[0, 1, :5].double().cpu(), -want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_fetch_from_before_the_first_position(dtype):
    """Negative positions have no page: their rows are zero, those behind them keep their places."""
    rng = np.random.default_rng(17)
    h, B, d, P = 2, 16, 64, 30
    cache = _filled(rng, P, h, B, d)
    first, lens = [-1, -70, -64, -200, -(1 << 31), 3], [40, 150, 64, 100, 70, 5]
    tables = rng.permutation(P).reshape(6, 5).astype(np.int32)
    cu = [0] + np.cumsum(lens).tolist()
    K, V = sw.kv_fetch_q8(cache, U.to_dev(tables), _i32(first), _i32(cu), cu[-1], dtype=dtype)
    pool = R.Pool(P, h, B, d)
    pool.x, _ = R.cache_values(cache)
    for got, n in ((K, "k"), (V, "v")):
        got = got.cpu().double().numpy()
        for s, (a, m) in enumerate(zip(first, lens)):
            want = np.zeros((h, m, d))
            at = [i for i in range(m) if a + i >= 0]
            if at:
                want[:, at] = pool.tokens(n, tables[s], [a + i for i in at])
            np.testing.assert_array_equal(got[:, cu[s]:cu[s + 1]], want)


def test_fetch_into_tensors_of_another_type_is_refused():
    cache = sw.new_cache_q8(2, 1, 16, 64, U.DEV)
    args = (cache, _i32([[0]]), None, _i32([0, 4]), 4)
    for own, other in ((torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)):
        out = tuple(torch.ones((1, 4, 64), dtype=own, device=U.DEV) for _ in range(2))
        with pytest.raises(sw.SketchWalkError, match="dtype"):
            sw.kv_fetch_q8(*args, dtype=other, out=out)
        for kw in ({}, {"dtype": own}):              # out's own type, named or not
            K, V = sw.kv_fetch_q8(*args, out=out, **kw)
            assert K.dtype is own and torch.all(K == 0) and torch.all(V == 0)
            K.fill_(1)
            V.fill_(1)
    assert sw.kv_fetch_q8(*args)[0].dtype is torch.bfloat16


def test_tables_with_many_slots_captured_and_refused_in_between():
    """A captured call of two launches: served, refused for a block without a page, served again."""
    r = _Requests(3, 16, 400, 1500, seed=12)
    r.check([5000, 16, 0])
    old, new = _i32(r.lens), _i32(r.lens)
    out = {"slots": _i32([0] * 9000), "cu": _i32([0] * 4), "pos": _i32([0] * 3), "status": _i32([5])}
    ws = torch.full((sw.load().sw_block_tables_workspace_bytes(3, 9000),), 255, dtype=torch.uint8, device=U.DEV)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sw.block_tables(old, new, 16, r.d_tables, r.d_free, r.d_n, 9000, out=dict(out), workspace=ws)
    for target in ([100, 6400, 6], [6400, 0, 2000], [0, 0, 0], [6400, 17, 1]):
        old.copy_(_i32(r.lens))
        new.copy_(_i32(target))
        shrinks = [s for s in range(3) if target[s] // 16 + 1 < r.lens[s] // 16]
        if shrinks:
            at = (shrinks[0], r.lens[shrinks[0]] // 16 - 1)
            page = int(r.d_tables[at])
            r.d_tables[at] = -1
            state = (r.d_tables.clone(), r.d_free.clone(), r.d_n.clone())
            g.replay()
            assert int(out["status"]) == 2 and torch.all(out["slots"] == -1) and torch.all(out["cu"] == 0)
            assert out["pos"].tolist() == [x - 1 for x in r.lens]
            for a, b in zip(state, (r.d_tables, r.d_free, r.d_n)):
                assert torch.equal(a, b)
            r.d_tables[at] = page
        g.replay()
        slots, cu, pos = R.allocate(r.lens, target, 16, r.tables, r.stack, 0, 9000)
        assert int(out["status"]) == 0 and out["slots"].tolist() == slots and out["cu"].tolist() == cu
        assert out["pos"].tolist() == pos and r.d_tables.tolist() == r.tables and r.d_n.tolist() == [len(r.stack)]
        assert r.d_free[:len(r.stack)].tolist() == r.stack
        r.lens = list(target)
        torch.cuda.synchronize()
