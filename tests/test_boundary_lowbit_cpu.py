"""The low-bit operators refuse bad arguments before they launch anything, and the definitions they are tested against agree with
brute force (no GPU needed)."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest

from oracle import lowbit as lb
from workloads import gen


@pytest.fixture(scope="module")
def bt():
    import paper_2406_02657_b200 as bt
    return bt


OK, ODD, ODD4 = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008), ctypes.c_void_p(0x10002)
BIG = 1 << 40
ref = ctypes.byref


def caches(bt):
    mk = bt.binding.bt_block_cache_kv4
    return mk(0x1000, 0x2000), mk(0, 0x2000), mk(0x1000, 0), mk(0x1008, 0x2000), mk(0x1000, 0x2002)


def test_cache_refusals(bt):
    L = bt.lib()
    cfg, wide = bt.make_config(4, 8, 64, 4, 1, 64, 2), bt.make_config(1, 1, 64, 4, 1, 2 ** 30 + 1, 1)
    good, no_kv, no_len, odd_kv, odd_len = caches(bt)

    def append(cfg=cfg, c=good, layer=0, k=OK, v=OK, n=3, stride=3, st=None):
        return L.bt_block_kv4_append(ref(cfg), ref(c) if c else None, layer, k, v, n, stride, 0, st, None)

    def read(cfg=cfg, c=good, layer=0, first=0, n=3, k=OK, v=OK, stride=3):
        return L.bt_block_kv4_read(ref(cfg), ref(c) if c else None, layer, first, n, k, v, stride, None)

    for go in (append, read):
        for bad in (dict(c=None), dict(c=no_kv), dict(c=no_len), dict(k=None), dict(v=None)):
            assert go(**bad) == bt.BT_ERR_NULL, bad
        for bad in (dict(layer=2), dict(layer=-1), dict(n=0), dict(n=-1), dict(stride=2), dict(cfg=bt.make_config(0, 8, 64, 4, 1, 64, 2))):
            assert go(**bad) == bt.BT_ERR_SHAPE, bad
        assert go(n=65, stride=65) == go(n=2 ** 31 - 1, stride=2 ** 31) == bt.BT_ERR_CAPACITY
        for bad in (dict(c=odd_kv), dict(c=odd_len), dict(k=ODD), dict(v=ODD), dict(cfg=wide), dict(cfg=bt.make_config(4, 8, 48, 4, 1, 64, 2)),
                    dict(cfg=bt.make_config(4, 40, 64, 4, 1, 64, 2))):
            assert go(**bad) == bt.BT_ERR_UNSUPPORTED, bad
    assert append(st=ODD4) == bt.BT_ERR_UNSUPPORTED
    assert read(first=-1) == bt.BT_ERR_SHAPE
    assert read(first=62) == read(first=64, n=1) == read(first=2 ** 31 - 1) == bt.BT_ERR_CAPACITY
    assert L.bt_block_kv4_append(None, ref(good), 0, OK, OK, 1, 1, 0, None, None) == bt.BT_ERR_NULL


def test_decode_refusals(bt):
    L = bt.lib()
    cfg, wide = bt.make_config(4, 8, 64, 4, 1, 4000, 2), bt.make_config(1, 1, 64, 4, 1, 2 ** 30 + 1, 1)
    good, no_kv, no_len, odd_kv, odd_len = caches(bt)
    need = bt.bt_workspace_bytes_kv4(cfg)
    assert need > bt.bt_workspace_bytes(cfg) and bt.bt_workspace_bytes_kv4(bt.make_config(4, 8, 48, 4, 1, 64, 2)) == 0
    # the arrival counters that bt_workspace_init zeroes are there even where nothing is split
    one = bt.make_config(4, 8, 64, 4, 1, 4000, 2, decode_splits=1)
    assert bt.bt_workspace_bytes_kv4(one) >= bt.bt_workspace_bytes(one) > 0

    def go(step, cfg=cfg, c=good, layer=0, q=OK, k=OK, v=OK, out=OK, ws=OK, size=need, st=None):
        c = ref(c) if c else None
        if step:
            return L.bt_block_decode_step_kv4(ref(cfg), c, layer, q, k, v, out, ws, size, st, None)
        return L.bt_block_decode_attn_kv4(ref(cfg), c, layer, q, out, ws, size, st, None)

    for step in (False, True):
        for bad in (dict(c=None), dict(c=no_kv), dict(c=no_len), dict(q=None), dict(out=None)) + ((dict(k=None), dict(v=None)) if step else ()):
            assert go(step, **bad) == bt.BT_ERR_NULL, bad
        assert go(step, layer=2) == bt.BT_ERR_SHAPE
        assert go(step, ws=None) == go(step, size=need - 1) == bt.BT_ERR_WORKSPACE
        for bad in (dict(c=odd_kv), dict(c=odd_len), dict(q=ODD), dict(out=ODD), dict(ws=ODD), dict(st=ODD4), dict(cfg=wide, size=BIG)) + \
                ((dict(k=ODD), dict(v=ODD)) if step else ()):
            assert go(step, **bad) == bt.BT_ERR_UNSUPPORTED, bad


def test_projection_refusals(bt):
    L = bt.lib()
    cfg = bt.make_config(4, 8, 64, 4, 2, 64, 2)
    good, no_kv, no_len, odd_kv, odd_len = caches(bt)
    bc, lc = bt.binding.bt_block_cache(0x1000, 0x1000, 0x1000), bt.binding.bt_local_cache(0x1000, 0x1000)

    def prefix(x=OK, xs=OK, w=OK, ws=OK, bias=None, out=OK, st=None):
        return L.bt_prefix_project_i8(ref(cfg), x, xs, w, ws, bias, out, st, None)

    def block(x=OK, xs=OK, w=OK, ws=OK, bias=None, out=OK, st=None, n=2, layer=0, c=bc):
        return L.bt_block_qkv_project_append_i8(ref(cfg), ref(c) if c else None, layer, x, xs, n, w, ws, bias, out, st, None)

    def local(x=OK, xs=OK, w=OK, ws=OK, bias=None, out=OK, st=None, n=2, layer=0, c=lc):
        return L.bt_local_qkv_project_append_i8(ref(cfg), ref(c) if c else None, layer, x, xs, n, w, ws, bias, 0, None, out, st, None)

    def kv4(x=OK, xs=OK, w=OK, ws=OK, bias=None, out=OK, st=None, n=2, layer=0, c=good):
        return L.bt_block_qkv_project_append_i8_kv4(ref(cfg), ref(c) if c else None, layer, x, xs, n, w, ws, bias, out, st, None)

    def kv4_bf16(x=OK, w=OK, bias=None, out=OK, st=None, n=2, layer=0, c=good):
        return L.bt_block_qkv_project_append_kv4(ref(cfg), ref(c) if c else None, layer, x, n, w, bias, out, st, None)

    for go in (prefix, block, local, kv4, kv4_bf16):
        steps = () if go is kv4_bf16 else ("xs", "ws")
        for name in ("x", "w", "out") + steps:
            assert go(**{name: None}) == bt.BT_ERR_NULL, name
            assert go(**{name: ODD}) == bt.BT_ERR_UNSUPPORTED, name
        assert go(bias=ODD) == go(st=ODD4) == bt.BT_ERR_UNSUPPORTED
        if go is prefix:
            continue
        assert go(c=None) == bt.BT_ERR_NULL
        assert go(n=0) == go(n=-3) == go(layer=2) == bt.BT_ERR_SHAPE
        assert go(n=65) == bt.BT_ERR_CAPACITY
    for go in (kv4, kv4_bf16):
        assert go(c=no_kv) == go(c=no_len) == bt.BT_ERR_NULL
        assert go(c=odd_kv) == go(c=odd_len) == bt.BT_ERR_UNSUPPORTED


def test_quantise_refusals(bt):
    go = bt.lib().bt_rows_quantize_i8
    assert go(None, 4, 64, OK, OK, None) == go(OK, 4, 64, None, OK, None) == go(OK, 4, 64, OK, None, None) == bt.BT_ERR_NULL
    assert go(OK, 0, 64, OK, OK, None) == go(OK, 4, 0, OK, OK, None) == go(OK, -1, 64, OK, OK, None) == bt.BT_ERR_SHAPE
    for rows, cols in ((4, 24), (4, 2064), (2 ** 31, 64)):
        assert go(OK, rows, cols, OK, OK, None) == bt.BT_ERR_UNSUPPORTED
    assert go(ODD, 4, 64, OK, OK, None) == go(OK, 4, 64, ODD, OK, None) == go(OK, 4, 64, OK, ODD4, None) == bt.BT_ERR_UNSUPPORTED


def test_cache_tensor(bt):
    cfg = bt.make_config(3, 2, 128, 4, 1, 33, 2)
    cache = bt.BlockCacheKV4(cfg, device="cpu")
    assert cache.kv.shape == (2, 3, 2, 3, 2, 1152) and cache.len.shape == (2, 3) and bt.KV4_TILE_BYTES == 1152
    with pytest.raises(AssertionError):
        bt.BlockCacheKV4(cfg, device="cpu", kv=cache.kv[:1])


@pytest.mark.parametrize("most", [7, 127])
def test_definition_is_the_nearest_code(most):
    """In exact arithmetic: every code is the nearest one, halves away from zero, and the largest value reaches the last code."""
    rng = np.random.default_rng(most)
    x = lb.to_bf16(rng.normal(size=(60, 32)) * 2.0 ** rng.integers(-40, 40, (60, 1)))
    x[0], x[1, :] = 0.0, np.arange(32) / 2.0
    codes, steps = lb.quantised(x, most)
    assert (codes[0] == 0).all() and steps[0] == 0 and np.abs(codes[1:]).max(1).min() == most
    for r in range(1, 60):
        for j in range(32):
            q = abs(Fraction(float(x[r, j]))) / Fraction(float(steps[r]))
            assert abs(codes[r, j]) == (q + Fraction(1, 2)).__floor__()
            assert codes[r, j] * x[r, j] >= 0


@pytest.mark.parametrize("most", [7, 127])
def test_fp32_product_rounds_like_the_exact_quotient(most):
    """The kernels multiply with (1 + 2^-19) / s in fp32 and round to even; every quotient of two 8-bit significands up to the last
    code gives the exact quotient's code, halves away from zero."""
    f = np.float32
    s = np.arange(128, 256, dtype=np.int64)
    for a in range(-2, 9):                                     # x = X 2^a against s in [128, 256)
        X = np.arange(128, 256, dtype=np.int64)[:, None]
        num, den = (X << max(a, 0)), (s << max(-a, 0))[None]
        seen = num * 2 < (2 * most + 1) * den                  # below most + 1/2
        exact = (2 * num + den) // (2 * den)
        inv = (f(1.0) / s.astype(f)) * f(1.0 + 2.0 ** -19)
        got = np.rint((X.astype(f) * f(2.0 ** a)).astype(np.float64) * inv.astype(np.float64)[None])   # the fused sum rounds once
        assert (got == exact)[seen].all()


def test_tiles_hold_the_rows():
    rng = np.random.default_rng(3)
    k, v = lb.to_bf16(rng.normal(size=(20, 128))), lb.to_bf16(rng.normal(size=(20, 128)))
    tiles = np.zeros((2, 2, lb.TILE_BYTES), np.uint8)
    lb.write_tiles(tiles, 0, k, v)
    for part, x in ((0, k), (1, v)):
        for r in (0, 15, 16, 19):
            for d in (0, 1, 31, 32, 63, 64, 127):
                tile, p = tiles[r // 16, d // 64], d % 64
                i = p // 2                                       # the layout again, written out
                at = (r % 16 // 2) * 64 + (i // 8) * 16 + (r % 2) * 8 + i % 8 if part == 0 else \
                    512 + (r % 16 // 4) * 128 + ((i // 4) ^ (2 * (r % 16 // 4))) * 16 + (i % 4) * 4 + r % 4
                byte = tile[at]
                code = int(byte >> 4 if p % 2 else byte & 15) - 8
                at = 1024 + part * 64 + (r % 16) * 4 + (p // 32) * 2
                step = gen.bf16_bits_to_f32(tile[at:at + 2].view(np.uint16))[0]
                assert code * float(step) == lb.held(x)[r, d]


def test_integer_projection_agrees_with_brute_force():
    rng = np.random.default_rng(5)
    x8, w8 = rng.integers(-128, 128, (3, 16)).astype(np.int8), rng.integers(-128, 128, (4, 16)).astype(np.int8)
    xs, ws, bias = rng.uniform(size=3), rng.uniform(size=4), rng.normal(size=4)
    y, tol = lb.project(x8, xs, w8, ws, bias)
    for m in range(3):
        for n in range(4):
            want = sum(int(x8[m, i]) * int(w8[n, i]) for i in range(16)) * xs[m] * ws[n] + bias[n]
            assert abs(y[m, n] - want) < 1e-9 and tol[m, n] > 2.0 ** -9 * abs(want)


def test_host_tensors_are_refused(bt):
    """Memory of the host, or of another device than the current one, does not reach a kernel."""
    import torch

    cfg = bt.make_config(2, 2, 64, 4, 1, 16, 1)
    cache, ws = bt.BlockCacheKV4(cfg, device="cpu"), torch.zeros(bt.bt_workspace_bytes_kv4(cfg), dtype=torch.uint8)
    q, rows = torch.zeros((2, 2, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 3, 64), dtype=torch.bfloat16)
    x8, xs = torch.zeros((2, 1, 128), dtype=torch.int8), torch.zeros((2, 1))
    x, w8 = torch.zeros((2, 1, 128), dtype=torch.bfloat16), torch.zeros((384, 128), dtype=torch.int8)
    for call in (lambda: bt.bt_block_kv4_append(cfg, cache, 0, rows, rows), lambda: bt.bt_block_kv4_read(cfg, cache, 0, rows, rows),
                 lambda: bt.bt_block_decode_attn_kv4(cfg, cache, 0, q, q, ws), lambda: bt.bt_block_decode_step_kv4(cfg, cache, 0, q, q, q, q, ws),
                 lambda: bt.bt_rows_quantize_i8(x, x8, xs), lambda: bt.bt_prefix_project_i8(cfg, x8, xs, w8, xs, None, q),
                 lambda: bt.bt_block_qkv_project_append_kv4(cfg, cache, 0, x, x, None, q),
                 lambda: bt.bt_block_qkv_project_append_i8_kv4(cfg, cache, 0, x8, xs, w8, xs, None, q)):
        with pytest.raises(bt.BtError) as e:
            call()
        assert e.value.code == bt.BT_ERR_UNSUPPORTED


def test_rows_without_their_axis_are_refused(bt):
    """[B,H,hd], as the decode step takes a row: its last axis is not taken for a number of rows."""
    import torch

    cfg = bt.make_config(2, 2, 64, 4, 1, 16, 1)
    cache, row = bt.BlockCacheKV4(cfg, device="cpu"), torch.zeros((2, 2, 64), dtype=torch.bfloat16)
    for call in (lambda k: bt.bt_block_kv4_append(cfg, cache, 0, k, k), lambda k: bt.bt_block_kv4_append(cfg, cache, 0, k, k, n_new=1),
                 lambda k: bt.bt_block_kv4_read(cfg, cache, 0, k, k), lambda k: bt.bt_block_kv4_read(cfg, cache, 0, k, k, n_rows=1)):
        for k in (row, row.transpose(0, 1)):
            with pytest.raises(bt.BtError) as e:
                call(k)
            assert e.value.code == bt.BT_ERR_SHAPE
