"""CPU checks of the paged 8-bit cache: the 64-bit reference against torch's e4m3,
and every refusal of the entry points (nothing is launched)."""
import ctypes

import numpy as np
import pytest
import torch

import _q8_ref as R
from paper_2602_07397_amd import binding as sw

FAKE = 1 << 20   # 256-byte aligned non-null address; never dereferenced


def test_reference_rounds_as_e4m3():
    rng = np.random.default_rng(1)
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    vals = np.sort(codes[torch.isfinite(codes)].double().numpy())
    assert np.array_equal(R.round_e4m3(vals), vals)
    mid = (vals[1:] + vals[:-1]) / 2
    y = np.concatenate([mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20),
                        rng.uniform(-448, 448, 4000), rng.normal(0, 0.01, 4000)]).astype(np.float32)
    y = y[np.abs(y) <= 448]
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(R.round_e4m3(y), want)


def test_reference_exponent():
    for e in (-126, -10, 0, 3, 119):
        assert R.exponent(448 * 2.0 ** e) == e
        assert R.exponent(449 * 2.0 ** e) == e + 1
    assert R.exponent(0.0) == -126 and R.exponent(1e-40) == -126
    assert R.exponent(float(torch.finfo(torch.float32).max)) == 120


def test_reference_allocation_by_hand():
    tables = [[4, 5, -1], [-1, -1, -1], [6, -1, -1]]
    stack = [9, 8, 7]                                # 7 on top
    slots, cu, pos = R.allocate([20, 0, 16], [0, 17, 18], 16, tables, stack)
    # request 0 gives back 4 and 5 (4 on top), request 1 takes 4 and 5, request 2 takes 7
    assert tables == [[-1, -1, -1], [4, 5, -1], [6, 7, -1]] and stack == [9, 8]
    assert slots == [64 + i for i in range(16)] + [80] + [112, 113]
    assert cu == [0, 0, 17, 19] and pos == [-1, 16, 17]


def _err(fn, args):
    lib = sw.load()
    return getattr(lib, fn)(*args), lib.sw_last_error().decode()


def _refused(fn, base, cases):
    for name, (changes, code, text) in cases.items():
        args = list(base)
        for at, val in changes.items():
            args[at] = val
        rc, msg = _err(fn, args)
        assert rc == code and text in msg, (name, rc, msg)


def test_block_tables_refusals():
    base = [3, 64, 10, FAKE, FAKE, FAKE, FAKE, FAKE, 30, 0, 100, FAKE, FAKE, FAKE, FAKE, None, 0, None]
    _refused("sw_block_tables", base, {
        "n_seqs": ({0: 0}, 1, "n_seqs"), "many": ({0: 65537}, 1, "n_seqs"), "B": ({1: 24}, 1, "B="),
        "B large": ({1: 1040}, 1, "B="), "b_max": ({2: 0}, 1, "b_max"), "b_max B": ({2: 1 << 25}, 1, "b_max"),
        "pages": ({8: 0}, 1, "n_pages"), "pages B": ({8: 1 << 25}, 1, "n_pages"), "rows": ({9: -1}, 1, "rows"),
        "rows and slots": ({9: 2}, 1, "n_slots"), "slots": ({10: -1}, 1, "n_slots"),
        "slots large": ({10: 1 << 31}, 1, "n_slots"), "old": ({3: None}, 1, "old_len"),
        "new": ({4: None}, 1, "new_len"), "tables": ({5: FAKE + 2}, 1, "tables"), "free": ({6: None}, 1, "free"),
        "n_free": ({7: None}, 1, "n_free"), "slot list": ({11: None}, 1, "slots"),
        "cu": ({12: None}, 1, "cu_seqlens"), "pos": ({13: None}, 1, "pos"), "status": ({14: None}, 1, "status"),
        "workspace": ({10: 100000}, 1, "workspace"), "small": ({10: 100000, 15: FAKE, 16: 32}, 1, "workspace_bytes")})
    assert sw.load().sw_block_tables_workspace_bytes(0, 5) == -1
    assert sw.load().sw_block_tables_workspace_bytes(3, 100) == 0


def test_append_refusals():
    base = [sw.SW_BF16, FAKE, FAKE, 128, 1024, 128, 1024, 100, 3, FAKE, FAKE, 30, 8, 128, 64, FAKE, FAKE,
            FAKE, FAKE, None]
    _refused("sw_kv_append_q8", base, {
        "dtype": ({0: 2}, 1, "dtype"), "k": ({1: FAKE + 8}, 1, "k is not"), "v": ({2: None}, 1, "v is NULL"),
        "stride": ({3: 100}, 1, "stride"), "negative": ({4: -1024}, 1, "stride"), "N": ({7: -1}, 1, "N="),
        "many": ({7: 4097, 9: None}, 2, "4096"), "launch": ({7: 1 << 30, 14: 16}, 2, "too many"),
        # 131072 x 2 x 16 workgroups of 1024 threads, 2^32
        "threads": ({8: 65536, 12: 16, 14: 256}, 2, "too many"), "n_seqs": ({8: 0}, 1, "n_seqs"), "slots": ({10: None}, 1, "slots"),
        "cu": ({9: FAKE + 1}, 1, "cu_seqlens"), "pages": ({11: 0}, 1, "n_pages"), "heads": ({12: 0}, 1, "h_kv"),
        "d": ({13: 96}, 2, "d=96"), "B": ({14: 8}, 1, "B="), "k pages": ({15: FAKE + 4}, 1, "k_pages"),
        "v pages": ({16: None}, 1, "v_pages"), "k scale": ({17: None}, 1, "k_scale"),
        "v scale": ({18: None}, 1, "v_scale"), "fp32 stride": ({0: sw.SW_F32, 3: 130}, 1, "stride")})
    empty = list(base)
    empty[7] = 0
    empty[1] = empty[2] = empty[10] = None           # no token: nothing to do
    assert _err("sw_kv_append_q8", empty)[0] == 0


def test_fetch_refusals():
    base = [sw.SW_BF16, FAKE, FAKE, FAKE, FAKE, 30, 8, 128, 64, 3, 10, FAKE, FAKE, FAKE, 100, FAKE, FAKE, None]
    _refused("sw_kv_fetch_q8", base, {
        "dtype": ({0: 5}, 1, "dtype"), "k pages": ({1: None}, 1, "k_pages"), "pages": ({5: -1}, 1, "n_pages"),
        "d": ({7: 256}, 2, "d=256"), "B": ({8: 1040}, 1, "B="), "n_seqs": ({9: 0}, 1, "n_seqs"),
        "b_max": ({10: 0}, 1, "b_max"), "tables": ({11: None}, 1, "tables"), "first": ({12: FAKE + 1}, 1, "first"),
        "cu": ({13: None}, 1, "cu_seqlens"), "N": ({14: -3}, 1, "N="), "K": ({15: FAKE + 4}, 1, "K is not"),
        "V": ({16: None}, 1, "V is NULL")})


def test_attention_refusals():
    base = [sw.SW_BF16, FAKE, FAKE, FAKE, FAKE, FAKE, 4, 32, 8, 128, 30, FAKE, 10, 64, FAKE, FAKE, FAKE, 5,
            ctypes.c_float(0.0), FAKE, FAKE, 1 << 40, None]
    _refused("sw_sparse_attn_decode_q8", base, {
        "dtype": ({0: -1}, 1, "dtype"), "q": ({1: FAKE + 2}, 1, "q is not"), "batch": ({6: 0}, 1, "batch"),
        "heads": ({8: 5}, 1, "h_q"), "group": ({7: 34, 8: 2}, 2, "h_q/h_kv"), "d": ({9: 32}, 2, "d=32"),
        "too many": ({6: 65536, 7: 256, 8: 64}, 2, "2^24"), "pages": ({10: 0}, 1, "n_pages"),
        "tables": ({11: None}, 1, "tables"), "b_max": ({12: 0}, 1, "b_max"), "B": ({13: 40}, 1, "B="),
        "pos": ({14: None}, 1, "pos"), "idx": ({15: None}, 1, "idx"), "cnt": ({16: None}, 1, "cnt"),
        "kmax": ({17: 0}, 1, "kmax"), "O": ({19: FAKE + 4}, 1, "O is not"), "ws": ({20: FAKE + 16}, 1, "workspace"),
        "ws bytes": ({21: 100}, 1, "workspace_bytes")})


def test_step_refusals():
    base = [sw.SW_BF16, 2, 4, 32, 8, 128, 64, 30, 64, 10, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE,
            FAKE, FAKE, FAKE, FAKE, 8, 0, 0, 20, 3, 10, ctypes.c_float(0.0), FAKE, FAKE, FAKE, FAKE, FAKE,
            1 << 40, None]
    _refused("sw_decode_step_q8", base, {
        "dtype": ({0: 2}, 1, "dtype"), "layers": ({1: 0}, 1, "layers"), "batch": ({2: 4097}, 2, "4096"),
        "group": ({3: 136}, 2, "h_q/h_kv"), "d": ({5: 256, 6: 64}, 2, "d=256"), "r": ({6: 129}, 1, "r="),
        "pages": ({7: 0}, 1, "n_pages"), "B": ({8: 24}, 1, "B="), "b_max": ({9: 5000}, 1, "b_max"),
        "variant": ({24: 3}, 2, "variant"), "unknown": ({24: 9}, 1, "variant"), "s": ({23: 0}, 1, "s="),
        "threads": ({2: 4096, 3: 512, 4: 512, 8: 256}, 2, "too many"),
        "budget": ({26: 0}, 1, "density"), "kmax": ({28: 1}, 1, "kmax"), "slots": ({18: None}, 1, "slots"),
        "tables": ({17: None}, 1, "tables"), "state": ({19: FAKE + 8}, 1, "state"),
        "workspace": ({34: None, 35: 0}, 1, "workspace"),
        "ws for the parts alone": ({35: sw.decode_attn_q8_workspace_bytes(4, 32, 8, 128)}, 1, "workspace_bytes"),
        "ws bytes": ({35: 100}, 1, "workspace_bytes")})


def test_binding_refuses_what_does_not_fit():
    cache = sw.new_cache_q8(4, 2, 16, 64, "cpu")
    assert cache["k"].shape == (4, 2, 16, 64) and cache["v"].shape == (4, 2, 64, 16)
    assert cache["k"].dtype == torch.float8_e4m3fn and cache["k_scale"].shape == (4, 2)
    i32 = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros((2, 4, 64))
    with pytest.raises(sw.SketchWalkError):
        sw.kv_append_q8(x, x, i32, cache)            # not on a GPU
    with pytest.raises(sw.SketchWalkError):
        sw.kv_fetch_q8(cache, i32[None], None, i32[:2], 4)
    with pytest.raises(sw.SketchWalkError):
        sw.sparse_attn_decode_q8(torch.zeros((1, 4, 64)), cache, i32[None], i32[:1], i32[None], i32[:1], 4)
    with pytest.raises(sw.SketchWalkError):
        sw.block_tables(i32, i32, 16, torch.zeros((4, 2), dtype=torch.int32), i32, i32[:1], 4)
    with pytest.raises(sw.SketchWalkError, match="d, B"):
        sw.kv_append_q8(x, x, i32, {**cache, "v": cache["k"]})
    with pytest.raises(sw.SketchWalkError, match="k_scale"):
        sw.kv_append_q8(x, x, i32, {**cache, "k_scale": cache["k_scale"][:1]})
    with pytest.raises(sw.SketchWalkError, match="CUDA"):
        sw.kv_append_q8("k", x, i32, cache)          # no tensor
    with pytest.raises(sw.SketchWalkError, match="integer"):
        sw.block_tables(i32, i32, 16, torch.zeros((4, 2), dtype=torch.int32), i32, i32[:1], 4.5)
    with pytest.raises(sw.SketchWalkError, match="dtype"):
        sw.kv_fetch_q8(cache, i32[None], None, i32[:2], 4, dtype=torch.float16)


def test_binding_refuses_sizes_that_do_not_fit_in_32_bits():
    """They are not cut to 32 bits (views of one entry; refused before anything else is looked at)."""
    cache = sw.new_cache_q8(4, 2, 16, 64, "cpu")
    i32 = torch.zeros(4, dtype=torch.int32)
    one = torch.zeros((1, 1), dtype=torch.int32)
    far = (1 << 32) + 5                              # 5 in the lower 32 bits
    tables = torch.zeros((4, 2), dtype=torch.int32)
    for args in ((i32, i32, 16, tables, one[0].expand(far), i32[:1], 4),
                 (i32, i32, 16, one.expand(4, far), i32, i32[:1], 4),
                 (one[0].expand(far), one[0].expand(far), 16, one.expand(far, 2), i32, i32[:1], 4)):
        with pytest.raises(sw.SketchWalkError, match="32 bits"):
            sw.block_tables(*args)
    for t in (one.expand(far, 2), one.expand(4, far)):
        with pytest.raises(sw.SketchWalkError, match="32 bits"):
            sw.kv_fetch_q8(cache, t, None, i32, 4)
    with pytest.raises(sw.SketchWalkError, match="32 bits"):
        sw.sparse_attn_decode_q8(torch.zeros((1, 4, 64)), cache, one.expand(1, far), i32[:1], i32[None], i32[:1], 4)
    with pytest.raises(sw.SketchWalkError, match="32 bits"):
        sw.kv_append_q8(torch.zeros((2, 4, 64)), torch.zeros((2, 4, 64)), i32, {
            **cache, "k": cache["k"][:, :1].expand(4, far, 16, 64), "v": cache["v"][:, :1].expand(4, far, 64, 16),
            "k_scale": cache["k_scale"][:, :1].expand(4, far), "v_scale": cache["v_scale"][:, :1].expand(4, far)})
