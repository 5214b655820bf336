"""Decode attention over the paged 8-bit cache, and the one-call step over it."""
import math

import numpy as np
import pytest
import torch

import _q8_ref as R
import oracle as O
import synth
from paper_2602_07397_amd import binding as sw

pytestmark = pytest.mark.gpu

U = pytest.importorskip("_gpu_util")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=U.DEV)


def _cache(seed, P, h, B, d, big=1.0):
    """Random codes, scales that differ from page to page; unused places hold any byte,
    NaN codes among them (the test that calls for it overwrites the used ones)."""
    g = torch.Generator(device=U.DEV).manual_seed(seed)
    cache = sw.new_cache_q8(P, h, B, d, U.DEV)
    for n in "kv":
        x = torch.randn(cache[n].shape, generator=g, device=U.DEV) * 64
        cache[n].copy_(x.clamp_(-448, 448).to(torch.float8_e4m3fn))
        e = torch.randint(-1, 2, (P, h), generator=g, device=U.DEV) - 6 + (int(math.log2(big)) if n == "k" else 0)
        cache[n + "_scale"].copy_((e + 127).to(torch.uint8))
    return cache


def _case(seed, batch, h_q, h_kv, d, B, ctx, dtype, density=0.3, big=1.0):
    rng = np.random.default_rng(seed)
    pos = [int(rng.integers(0, ctx)) for _ in range(batch)]
    pos[0] = ctx - 1
    b_max = -(-ctx // B)
    P = batch * b_max + 3
    tables = rng.permutation(P)[:batch * b_max].reshape(batch, b_max).astype(np.int32)
    sels = [sorted({0, p // B} | {j for j in range(p // B) if rng.uniform() < density}) if p >= 0 else [0]
            for p in pos]
    kmax = max(len(s) for s in sels) + 1
    idx = np.full((batch, kmax), -1, dtype=np.int32)
    for b, s in enumerate(sels):
        idx[b, :len(s)] = s
    q = torch.from_numpy(rng.normal(size=(batch, h_q, d))).to(dtype)
    return dict(q=q, cache=_cache(seed, P, h_kv, B, d, big), tables=tables, pos=pos, idx=idx,
                cnt=np.array([len(s) for s in sels], dtype=np.int32), kmax=kmax, B=B, P=P)


def _run(c, **kw):
    return sw.sparse_attn_decode_q8(U.to_dev(c["q"]), c["cache"], U.to_dev(c["tables"]), _i32(c["pos"]),
                                    U.to_dev(c["idx"]), U.to_dev(c["cnt"]), c["kmax"], **kw)


def _selected(c, b):
    """Pages and places of the tokens that count for sequence b, in list order."""
    p, B = c["pos"][b], c["B"]
    b_max = c["tables"].shape[1]
    if p < 0 or p // B >= b_max:
        return [], []
    pages, places = [], []
    for j in c["idx"][b, :max(0, min(int(c["cnt"][b]), c["kmax"]))]:
        if j < 0 or j > p // B or not 0 <= c["tables"][b, j] < c["P"]:
            continue
        for o in range(min(B, p + 1 - j * B)):
            pages.append(int(c["tables"][b, j]))
            places.append(o)
    return pages, places


def _check(c, got, scale=None):
    x, _ = R.cache_values(c["cache"])
    d = c["q"].shape[2]
    scale = scale or 1.0 / math.sqrt(d)
    got = got.double().cpu().numpy()
    for b in range(len(c["pos"])):
        pages, places = _selected(c, b)
        if not pages:
            assert np.all(got[b] == 0.0), b
            continue
        K = x["k"][pages, :, places].transpose(1, 0, 2)
        V = x["v"][pages, :, places].transpose(1, 0, 2)
        o, a, top = R.attention(c["q"][b].double().numpy(), K, V, scale)
        err = np.abs(got[b] - o)
        bound = R.attention_bound(c["q"].dtype, o, a, top, d, len(pages))
        assert np.all(err <= bound), (b, float((err / bound).max()), float(err.max()))


DT = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("batch,h_q,h_kv,d,B,ctx", [
    (1, 1, 1, 64, 16, 1), (1, 4, 4, 128, 64, 5000), (3, 8, 2, 128, 64, 700), (2, 28, 4, 128, 128, 1500),
    (4, 16, 1, 64, 16, 333), (2, 6, 2, 64, 48, 1000), (5, 12, 4, 128, 80, 777), (1, 32, 8, 128, 1024, 9000),
    (70, 8, 8, 64, 32, 200), (2, 10, 2, 128, 64, 64), (3, 18, 2, 64, 16, 17)])
def test_attention(dtype, batch, h_q, h_kv, d, B, ctx):
    c = _case(batch * 1000 + ctx, batch, h_q, h_kv, d, B, ctx, dtype)
    got = _run(c)
    _check(c, got)
    assert torch.equal(got, _run(c))                 # same inputs, same bits


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("ctx", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 257])
def test_attention_at_group_edges(dtype, ctx):
    c = _case(ctx, 2, 8, 2, 128, 64, ctx, dtype, density=1.0)
    _check(c, _run(c))
    c = _case(ctx + 7, 2, 4, 1, 64, 16, ctx, dtype, density=0.5)
    _check(c, _run(c))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("batch,h_q,h_kv,d", [(255, 2, 2, 64), (256, 4, 1, 128), (257, 2, 2, 64), (300, 3, 1, 128)])
def test_large_batches_of_unlike_lengths(dtype, batch, h_q, h_kv, d):
    """On both sides of the 256 sequences up to which the work is shared out: one long
    sequence among short ones and idle ones."""
    c = _case(batch, batch, h_q, h_kv, d, 16, 1200, dtype, density=0.6)
    rng = np.random.default_rng(batch)
    short = rng.integers(-1, 40, size=batch)
    c["pos"] = [c["pos"][0]] + [int(x) for x in short[1:]]
    got = _run(c)
    _check(c, got)
    assert torch.equal(got, _run(c))


@pytest.mark.parametrize("dtype", DT)
def test_unused_places_may_hold_anything(dtype):
    """Behind a sequence's end, in unlisted pages: NaN codes and the largest values."""
    c = _case(21, 3, 8, 2, 64, 64, 400, dtype)
    clean = _run(c)
    used = {}
    for b in range(3):
        for pg, o in zip(*_selected(c, b)):
            used.setdefault(pg, set()).add(o)
    k, v = c["cache"]["k"].view(torch.uint8), c["cache"]["v"].view(torch.uint8)
    for pg in range(c["P"]):
        rest = [o for o in range(64) if o not in used.get(pg, ())]
        if rest:
            k[pg, :, rest] = 0x7f
            v[pg, :, :, rest] = 0xff
    assert torch.equal(clean, _run(c))


@pytest.mark.parametrize("dtype", DT)
def test_rows_without_a_token_and_pages_that_are_none(dtype):
    c = _case(22, 7, 8, 4, 128, 32, 500, dtype)
    c["pos"][1] = -1                                 # idle
    c["pos"][2] = 32 * c["tables"].shape[1]          # behind the table
    c["cnt"][3] = 0                                  # nothing selected
    c["tables"][4] = -1                              # no page at all
    c["tables"][5, :] = c["P"] + np.arange(c["tables"].shape[1])
    c["cnt"][6] = -5
    c["cnt"][0] = c["kmax"] + 100                    # clamped
    c["idx"][0, 1] = -7                              # entries to skip
    c["idx"][0, 2] = 1 << 30
    c["tables"][0, 0] = -2
    _check(c, _run(c))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("big", [16.0, 256.0])
def test_large_logits(dtype, big):
    c = _case(23, 2, 8, 2, 128, 64, 600, dtype, big=big)
    got = _run(c)
    assert torch.isfinite(got.float()).all()
    _check(c, got)
    _check(c, _run(c, scale=0.003), scale=0.003)


def test_nan_of_a_token_that_counts_shows():
    c = _case(24, 2, 4, 2, 64, 16, 100, torch.float32)
    pg = int(c["tables"][0, 0])
    c["cache"]["k"].view(torch.uint8)[pg, 1, 3, 5] = 0x7f
    got = _run(c)
    assert torch.isnan(got[0, 2:]).all() and torch.isfinite(got[0, :2]).all() and torch.isfinite(got[1]).all()


@pytest.mark.parametrize("dtype", DT)
def test_long_lists(dtype):
    """More chunks than are listed at a time, blocks in any order and one of them twice."""
    c = _case(25, 1, 8, 1, 64, 16, 16 * 33000, dtype, density=1.0)
    n = int(c["cnt"][0])
    c["idx"][0, :n] = c["idx"][0, :n][np.random.default_rng(1).permutation(n)]
    _check(c, _run(c))
    c = _case(26, 1, 4, 2, 128, 64, 1000, dtype)
    n = int(c["cnt"][0])
    c["idx"][0, n] = c["idx"][0, 0]
    c["cnt"][0] = n + 1
    _check(c, _run(c))


def test_pool_behind_4_gib():
    """Pages whose offset passes 32 bits."""
    h, B, d = 8, 64, 128
    P = (1 << 32) // (h * B * d) + 40
    cache = {"k": torch.empty((P, h, B, d), dtype=torch.float8_e4m3fn, device=U.DEV),
             "v": torch.empty((P, h, d, B), dtype=torch.float8_e4m3fn, device=U.DEV),
             "k_scale": torch.full((P, h), 121, dtype=torch.uint8, device=U.DEV),
             "v_scale": torch.full((P, h), 121, dtype=torch.uint8, device=U.DEV)}
    tail = slice(P - 20, P)
    for n in "kv":
        cache[n][tail].copy_((torch.randn(cache[n][tail].shape, device=U.DEV) * 60).clamp(-448, 448).to(torch.float8_e4m3fn))
    tables = np.arange(P - 1, P - 17, -1).astype(np.int32).reshape(2, 8)
    small = {n: t[tail].contiguous() for n, t in cache.items()}
    rng = np.random.default_rng(2)
    q = U.to_dev(torch.from_numpy(rng.normal(size=(2, 32, d))).to(torch.bfloat16))
    args = (_i32([511, 400]), _i32([[0, 2, 5, 7], [0, 1, 3, 6]]), _i32([4, 4]), 4)
    new = torch.randn((2, h, d), device=U.DEV, dtype=torch.bfloat16).transpose(0, 1)
    outs = []
    for c, base in ((cache, 0), (small, P - 20)):
        t = U.to_dev(tables - base)
        slots = _i32([int((tables[0, 7] - base) * B + 63), int((tables[1, 6] - base) * B + 16)])
        sw.kv_append_q8(new, new, slots, c)
        K, V = sw.kv_fetch_q8(c, t, _i32([440, 380]), _i32([0, 72, 93]), 93)
        outs.append((sw.sparse_attn_decode_q8(q, c, t, *args), K, V))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_attention_in_two_streams_and_captured():
    c1, c2 = (_case(s, 4, 32, 8, 128, 64, 3000, torch.bfloat16) for s in (31, 32))
    want = [_run(c1), _run(c2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for c, s in zip((c1, c2), streams):
        with torch.cuda.stream(s):
            got.append([_run(c) for _ in range(3)])
    torch.cuda.synchronize()
    for w, many in zip(want, got):
        assert all(torch.equal(w, g) for g in many)
    dev = {n: U.to_dev(c1[n]) for n in ("q", "tables", "idx", "cnt")}
    pos = _i32(c1["pos"])
    out = torch.empty_like(dev["q"])
    ws = torch.empty((sw.decode_attn_q8_workspace_bytes(4, 32, 8, 128),), dtype=torch.uint8, device=U.DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sw.sparse_attn_decode_q8(dev["q"], c1["cache"], dev["tables"], pos, dev["idx"], dev["cnt"], c1["kmax"],
                                 O=out, workspace=ws)
    for i in range(4):
        out.zero_()
        g.replay()
        assert torch.equal(out, want[0])
        dev["q"].mul_(1.0)                           # the program's own work in between
        torch.cuda.synchronize()


# --------------------------------------------------------------------------- one-call step


def _step_setup(dtype, h_q, h_kv, d, B, L, prompts, steps, seed):
    w = synth.Workload("q8_step", 70 + seed, layers=L, h_q=h_q, h_kv=h_kv, d=d, B=B,
                       dtype="bf16" if dtype == torch.bfloat16 else "f32", pct=30, needles=1,
                       batch=len(prompts), kv_len=max(prompts), steps=steps)
    signs, cols = synth.srht_params(w.d, w.r, w.seed)
    ts, tc = U.to_dev(signs), U.to_dev(cols)
    n = len(prompts)
    b_max = -(-(max(prompts) + steps) // B)
    P = sum(-(-(p + steps) // B) for p in prompts) + 2
    pool = dict(tables=torch.full((n, b_max), -1, dtype=torch.int32, device=U.DEV),
                free=torch.arange(P, dtype=torch.int32, device=U.DEV), n_free=_i32([P]))
    cache = sw.new_cache_q8(P, h_kv, B, d, U.DEV, layers=L)
    state = torch.zeros((L, sw.decode_state_bytes(n, d, w.r, b_max)), dtype=torch.uint8, device=U.DEV)
    N = sum(prompts)
    out = sw.block_tables(_i32([0] * n), _i32(prompts), B, pool["tables"], pool["free"], pool["n_free"], N)
    assert int(out["status"]) == 0
    for l in range(L):
        layer = {k: t[l] for k, t in cache.items()}
        Ks, Vs = [], []
        for s, p in enumerate(prompts):
            Q, K, V = (U.to_dev(x) for x in synth.decode_prefix_inputs(w, l, s, kv_len=p))
            sk = sw.sketch_scores(Q, K, [0, p], B, ts, tc, want_means=True)
            sw.decode_state_init(state[l], n, d, w.r, b_max, s, p, B, sk)
            Ks.append(K)
            Vs.append(V)
        sw.kv_append_q8(torch.cat(Ks, 1), torch.cat(Vs, 1), out["slots"], layer, cu=out["cu"])
    return w, ts, tc, pool, cache, state, b_max


@pytest.mark.parametrize("dtype,h_q,h_kv,d,B,per_ws", [
    (torch.bfloat16, 8, 2, 128, 64, None), (torch.float32, 4, 4, 64, 16, 1), (torch.bfloat16, 14, 2, 64, 32, 2)])
def test_step_is_the_per_layer_calls(dtype, h_q, h_kv, d, B, per_ws):
    """Steps across block borders, pages taken as they come, one sequence idle for a
    step: bit for bit the per-layer calls, and the attention against 64 bits."""
    L, prompts, steps = 3, [2 * B - 2, 1, 3 * B + 5], 5
    w, ts, tc, pool, cache, state, b_max = _step_setup(dtype, h_q, h_kv, d, B, L, prompts, steps, h_q)
    cache2 = {k: t.clone() for k, t in cache.items()}
    state2 = state.clone()
    n, lens = len(prompts), list(prompts)
    kmax = sw.select_max_count_decode(b_max, density_pct=30)
    ws = None
    if per_ws:
        ws = torch.empty((256 + per_ws * sw.decode_attn_q8_workspace_bytes(n, h_q, h_kv, d),), dtype=torch.uint8, device=U.DEV)
    for t in range(steps):
        new = [x + 1 for x in lens]
        if t == 2:
            new[1] = lens[1]
        tok = [synth.decode_step_inputs(w, t, l, batch=n) for l in range(L)]
        q, k, v = (torch.stack([x[i] for x in tok]).to(U.DEV) for i in range(3))
        bt = sw.block_tables(_i32(lens), _i32(new), B, pool["tables"], pool["free"], pool["n_free"], n, rows=1)
        pos = torch.where(bt["slots"] < 0, -1, bt["pos"])           # an idle sequence is skipped
        out = sw.decode_step_q8(q, k, v, cache, pool["tables"], bt["slots"], state, pos, ts, tc, density_pct=30,
                                workspace=ws)
        row = None
        for l in range(L):
            layer = {m: x[l] for m, x in cache2.items()}
            sw.kv_append_q8(k[l].transpose(0, 1), v[l].transpose(0, 1), bt["slots"], layer)
            sw.sketch_scores_decode(q[l], k[l], B, pos, ts, tc, b_max, state2[l])
            row = sw.walk_update_decode(state2[l], n, d, w.r, b_max, B, pos, 8, row)
            idx, cnt, _ = sw.select_topk_blocks_decode(row, B, pos, density_pct=30, kmax=kmax)
            o = sw.sparse_attn_decode_q8(q[l], layer, pool["tables"], pos, idx, cnt, kmax)
            on = [s for s in range(n) if pos[s] >= 0]
            assert torch.equal(out["rows"][l][on], row[on]) and torch.equal(out["cnt"][l][on], cnt[on])
            assert torch.equal(out["idx"][l][on], idx[on]) and torch.equal(out["O"][l], o)
            c = dict(q=q[l].cpu(), cache=layer, tables=pool["tables"].cpu().numpy(), pos=pos.tolist(),
                     idx=idx.cpu().numpy(), cnt=cnt.cpu().numpy(), kmax=kmax, B=B, P=cache["k"].shape[1])
            _check(c, o)
        for m in cache:
            assert torch.equal(cache[m].view(torch.uint8), cache2[m].view(torch.uint8)), m
        assert torch.equal(state, state2)
        lens = new


@pytest.mark.parametrize("what", ["one", "slot", "pages"])
def test_step_leaves_sequences_without_a_place_alone(what):
    """A sequence that did not grow, one whose slot is behind the pool, and a step that the
    pool could not serve at all: as idle ones, in the cache, the state and the outputs."""
    L, B, d, h_q, h_kv, prompts = 2, 32, 64, 4, 2, [64, 31, 64]
    w, ts, tc, pool, cache, state, b_max = _step_setup(torch.float32, h_q, h_kv, d, B, L, prompts, 4, 6)
    n, P = 3, cache["k"].shape[1]
    tok = [synth.decode_step_inputs(w, 0, l, batch=n) for l in range(L)]
    q, k, v = (torch.stack([x[i] for x in tok]).to(U.DEV) for i in range(3))
    if what == "pages":
        pool["n_free"].fill_(1)                      # two are needed
    new = [65, 31 + (what != "one"), 65]
    bt = sw.block_tables(_i32(prompts), _i32(new), B, pool["tables"], pool["free"], pool["n_free"], n, rows=1)
    assert int(bt["status"]) == (1 if what == "pages" else 0)
    if what == "slot":
        bt["slots"][1] = P * B + 3
    idle = [0, 1, 2] if what == "pages" else [1]
    pos = bt["pos"].clone()
    assert pos[1] >= 0
    pos[idle] = -1
    cache2, state2 = {m: t.clone() for m, t in cache.items()}, state.clone()
    before = state.clone()
    out = sw.decode_step_q8(q, k, v, cache, pool["tables"], bt["slots"], state, bt["pos"], ts, tc, density_pct=30)
    slots = bt["slots"].clone()
    slots[idle] = -1
    ref = sw.decode_step_q8(q, k, v, cache2, pool["tables"], slots, state2, pos, ts, tc, density_pct=30)
    assert torch.equal(out["O"], ref["O"]) and torch.all(out["O"][:, idle] == 0)
    assert torch.equal(state, state2)
    for m in cache:
        assert torch.equal(cache[m].view(torch.uint8), cache2[m].view(torch.uint8)), m
    on = [s for s in range(n) if s not in idle]
    for m in ("rows", "idx", "cnt"):
        assert torch.equal(out[m][:, on], ref[m][:, on]), m
    if not on:
        assert torch.equal(state, before)


def test_step_follows_the_step_over_a_contiguous_cache():
    """The same tokens through sw_decode_step (exact cache) and the 8-bit one: the sketch,
    walk and selection are the same bits, the attention is that of the stored values."""
    L, B, d, h_q, h_kv, prompts, steps = 2, 64, 128, 8, 2, [200, 130], 3
    w, ts, tc, pool, cache, state, b_max = _step_setup(torch.bfloat16, h_q, h_kv, d, B, L, prompts, steps, 3)
    n, T = 2, b_max * B
    Kc = torch.zeros((L, n, h_kv, T, d), dtype=torch.bfloat16, device=U.DEV)
    Vc = torch.zeros_like(Kc)
    state2, lens = state.clone(), list(prompts)
    for t in range(steps):
        new = [x + 1 for x in lens]
        tok = [synth.decode_step_inputs(w, t, l, batch=n) for l in range(L)]
        q, k, v = (torch.stack([x[i] for x in tok]).to(U.DEV) for i in range(3))
        bt = sw.block_tables(_i32(lens), _i32(new), B, pool["tables"], pool["free"], pool["n_free"], n, rows=1)
        out = sw.decode_step_q8(q, k, v, cache, pool["tables"], bt["slots"], state, bt["pos"], ts, tc, density_pct=30)
        # the contiguous cache holds the stored values, the new token's among them
        for l in range(L):
            layer = {m: x[l] for m, x in cache.items()}
            for s in range(n):
                K, V = sw.kv_fetch_q8(layer, pool["tables"][s:s + 1], None, _i32([0, new[s]]), new[s])
                Kc[l, s, :, :new[s]], Vc[l, s, :, :new[s]] = K, V
        ref = sw.decode_step(q, k, v, Kc.clone(), Vc.clone(), state2, bt["pos"], ts, tc, B, b_max, density_pct=30)
        for m in ("rows", "idx", "cnt"):
            assert torch.equal(out[m], ref[m]), m
        assert torch.equal(state, state2)
        for l in range(L):
            got = sw.sparse_attn_decode(q[l], Kc[l], Vc[l], B, bt["pos"], out["idx"][l], out["cnt"][l], out["idx"].shape[2])
            a = out["O"][l].float().abs().max()
            # both round weights and outputs to bf16: each within 2^-8 of the weighted mean of |v|, and of itself
            assert (out["O"][l].float() - got.float()).abs().max() <= 4 * 2.0 ** -8 * max(float(Vc.float().abs().max()), float(a))
        lens = new


def test_step_captured_replays():
    L, B, d, h_q, h_kv, prompts = 2, 32, 64, 4, 2, [100, 31]
    w, ts, tc, pool, cache, state, b_max = _step_setup(torch.bfloat16, h_q, h_kv, d, B, L, prompts, 8, 5)
    n = 2
    tok = [synth.decode_step_inputs(w, 0, l, batch=n) for l in range(L)]
    q, k, v = (torch.stack([x[i] for x in tok]).to(U.DEV) for i in range(3))
    old, new = _i32(prompts), _i32([x + 1 for x in prompts])
    kmax = sw.select_max_count_decode(b_max, density_pct=30)
    out = {"rows": torch.zeros((L, n, b_max), dtype=torch.float64, device=U.DEV),
           "idx": torch.zeros((L, n, kmax), dtype=torch.int32, device=U.DEV),
           "cnt": torch.zeros((L, n), dtype=torch.int32, device=U.DEV), "O": torch.zeros_like(q)}
    bt = {"slots": _i32([0, 0]), "cu": _i32([0] * 3), "pos": _i32([0, 0]), "status": _i32([0])}
    ws = torch.empty((sw.load().sw_decode_step_q8_workspace_bytes(n, h_q, h_kv, d),), dtype=torch.uint8, device=U.DEV)

    def step():
        sw.block_tables(old, new, B, pool["tables"], pool["free"], pool["n_free"], n, rows=1, out=bt)
        sw.decode_step_q8(q, k, v, cache, pool["tables"], bt["slots"], state, bt["pos"], ts, tc, density_pct=30,
                          kmax=kmax, out=out, workspace=ws)

    saved = [t.clone() for t in (state, *pool.values(), *(x.view(torch.uint8) for x in cache.values()))]

    def reset():
        for t, s in zip((state, *pool.values(), *(x.view(torch.uint8) for x in cache.values())), saved):
            t.copy_(s)
        old.copy_(_i32(prompts))
        new.copy_(_i32([x + 1 for x in prompts]))

    wants = []
    for _ in range(4):                               # eager: four tokens
        step()
        wants.append({m: x.clone() for m, x in out.items()})
        old.add_(1)
        new.add_(1)
    reset()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    reset()
    for want in wants:
        g.replay()
        for m in out:
            assert torch.equal(out[m], want[m]), m
        old.add_(1)
        new.add_(1)
        torch.cuda.synchronize()


# --------------------------------------------------------------------------- weights


def _fine_bound(c, o, a, top, d, T):
    """R.attention_bound for weights in two bf16 numbers: the first is off by at most 2^-8
    of the weight, the second by 2^-8 of what that leaves, so 2^-16 of the weighted mean of
    |v|; sums and logits as in 32 bits; then the output's own rounding, 2^-8 of it."""
    return (R.attention_bound(torch.float32, o, a, top, d, T) + 2.0 ** -16 * a) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(o)


@pytest.mark.parametrize("batch,h_q,h_kv,d,B,ctx", [
    (2, 8, 2, 128, 64, 50), (3, 8, 2, 64, 16, 700), (2, 16, 1, 128, 128, 9000), (260, 4, 2, 64, 16, 40)])
def test_bf16_weights_keep_16_bits(batch, h_q, h_kv, d, B, ctx):
    """Outputs that are small against the values they are made of show what the weights lose."""
    c = _case(batch + ctx, batch, h_q, h_kv, d, B, ctx, torch.bfloat16)
    got = _run(c).double().cpu().numpy()
    x, _ = R.cache_values(c["cache"])
    for b in range(batch):
        pages, places = _selected(c, b)
        K = x["k"][pages, :, places].transpose(1, 0, 2)
        V = x["v"][pages, :, places].transpose(1, 0, 2)
        o, a, top = R.attention(c["q"][b].double().numpy(), K, V, 1.0 / math.sqrt(d))
        err = np.abs(got[b] - o)
        bound = _fine_bound(c, o, a, top, d, len(pages))
        assert np.all(err <= bound), (b, float((err / bound).max()))


# --------------------------------------------------------------------------- NaN and rows without a token


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("batch,ctx", [(1, 9000), (3, 40), (260, 70)])
def test_a_query_that_is_not_finite_shows(batch, ctx, dtype):
    """Over split work, one workgroup, and batches that are not shared out: a NaN in a query
    makes its head NaN, other heads keep their bits; rows without a token stay zero."""
    c = _case(41, batch, 8, 2, 64, 16, ctx, dtype)
    if batch > 1:
        c["pos"][1] = -1
    clean = _run(c)
    assert torch.isfinite(clean).all()
    c["q"] = c["q"].clone()
    c["q"][:, 3, 7] = math.nan
    got = _run(c)
    live = [b for b in range(batch) if c["pos"][b] >= 0]
    assert torch.isnan(got[live, 3]).all()
    rest = [u for u in range(8) if u != 3]
    assert torch.equal(got[:, rest], clean[:, rest])
    if batch > 1:
        assert torch.all(got[1] == 0)


@pytest.mark.parametrize("dtype", DT)
def test_tokens_that_are_all_nan_show(dtype):
    """A first token whose key was infinite (stored as NaN), and contexts of such keys."""
    h, B, d = 2, 16, 64
    cache = sw.new_cache_q8(40, h, B, d, U.DEV)
    n = 33 * B
    k = torch.full((h, n, d), math.inf, dtype=dtype, device=U.DEV)
    v = torch.ones((h, n, d), dtype=dtype, device=U.DEV)
    sw.kv_append_q8(k, v, torch.arange(n, dtype=torch.int32, device=U.DEV), cache, cu=_i32([0, n]))
    tables = torch.arange(33, dtype=torch.int32, device=U.DEV).repeat(2, 1)
    idx = tables.clone()
    q = torch.ones((2, 4, d), dtype=dtype, device=U.DEV)
    for pos in ([0, -1], [n - 1, 5], [-1, n - 1]):
        got = sw.sparse_attn_decode_q8(q, cache, tables, _i32(pos), idx, _i32([33, 33]), 33)
        for b in range(2):
            assert (torch.isnan(got[b]) if pos[b] >= 0 else got[b] == 0).all(), pos


@pytest.mark.parametrize("dtype", DT)
def test_logits_that_are_all_minus_infinity(dtype):
    """The softmax of such a row has no value; of one with a finite logit beside them it has."""
    h, B, d = 1, 16, 64
    cache = sw.new_cache_q8(40, h, B, d, U.DEV)
    n = 33 * B
    k = torch.ones((h, n, d), dtype=dtype, device=U.DEV)
    v = torch.randn((h, n, d), dtype=dtype, device=U.DEV)
    sw.kv_append_q8(k, v, torch.arange(n, dtype=torch.int32, device=U.DEV), cache, cu=_i32([0, n]))
    tables = torch.arange(33, dtype=torch.int32, device=U.DEV)[None]
    q = torch.ones((1, 4, d), dtype=dtype, device=U.DEV)
    q[0, 1, 3] = -math.inf
    for pos in (0, 16, n - 1):
        got = sw.sparse_attn_decode_q8(q, cache, tables, _i32([pos]), tables, _i32([33]), 33)
        assert torch.isnan(got[0, 1]).all() and torch.isfinite(got[0, [0, 2, 3]]).all(), pos


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("batch", [3, 260])
def test_unlisted_pages_may_have_any_scale(batch, dtype):
    """Pages of no listed block were never begun: their scales, page 0's among them, hold any byte."""
    c = _case(28, batch, 8, 2, 64, 64, 400, dtype)
    c["pos"][1] = -1
    c["cnt"][2] = 1                                  # one group, not full
    c["pos"][2] = 9
    c["tables"][c["tables"] == 0] = c["P"] - 1       # page 0 is nobody's
    clean = _run(c)
    _check(c, clean)
    used = sorted({pg for b in range(batch) for pg in _selected(c, b)[0]})
    rest = sorted(set(range(c["P"])) - set(used))
    assert rest[0] == 0
    for byte in (255, 254, 0):
        for n in "kv":
            c["cache"][n + "_scale"][rest] = byte
        assert torch.equal(clean, _run(c)), byte


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("q_exp,v_exp", [(-80, 0), (90, 0), (0, -80), (0, 90), (90, 90)])
def test_queries_and_values_at_the_ends_of_the_range(dtype, q_exp, v_exp):
    """Magnitudes of 2^-80 and 2^90, with keys that bring the logits back to ordinary ones."""
    c = _case(29, 2, 8, 2, 128, 64, 600, dtype)
    c["q"] = (torch.sign(c["q"].float()) * torch.clamp(c["q"].float().abs(), 1.0, 1.99) * 2.0 ** q_exp).to(dtype)
    c["cache"]["k_scale"] = (c["cache"]["k_scale"].int() - q_exp).to(torch.uint8)
    if v_exp:
        # codes of at least 32, so that every value is of the magnitude
        v = c["cache"]["v"].float()
        c["cache"]["v"].copy_((torch.sign(v + 0.1) * v.abs().clamp(32, 60)).to(torch.float8_e4m3fn))
        c["cache"]["v_scale"].fill_(127 + v_exp - 5)
    got = _run(c)
    assert torch.isfinite(got).all()
    _check(c, got)
