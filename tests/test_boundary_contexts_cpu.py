"""The operators for long and shared contexts refuse bad arguments before they launch anything, and the definitions they are
tested against agree with brute force (no GPU needed)."""
import ctypes

import numpy as np
import pytest

from oracle import contexts as ctx


@pytest.fixture(scope="module")
def bt():
    import paper_2406_02657_b200 as bt
    return bt


OK, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008)
BIG = 1 << 30
ref = ctypes.byref


def test_window_refusals(bt):
    L = bt.lib()
    cfg, one = bt.make_config(4, 8, 64, 4, 1, 64, 2), bt.make_config(4, 8, 64, 4, 1, 64, 2, decode_splits=1)
    plain = bt.make_config(4, 8, 64, 4, 1, 64, 2, prefill_plain=1)
    bc, nullc = bt.binding.bt_block_cache(0x1000, 0x1000, 0x1000), bt.binding.bt_block_cache(0x1000, 0, 0x1000)
    attn, step, pre = L.bt_block_decode_attn_window, L.bt_block_decode_step_window, L.bt_block_prefill_attn_window
    for w, s in ((0, 0), (-1, 4), (4, -1)):
        assert attn(ref(one), ref(bc), 0, OK, w, s, OK, None, 0, None, None) == bt.BT_ERR_SHAPE
        assert step(ref(cfg), ref(bc), 0, OK, OK, OK, w, s, OK, OK, BIG, None, None) == bt.BT_ERR_SHAPE
        assert pre(ref(cfg), OK, OK, OK, 8, 8, w, s, OK, None, None) == bt.BT_ERR_SHAPE
    assert attn(None, ref(bc), 0, OK, 4, 0, OK, OK, BIG, None, None) == bt.BT_ERR_NULL
    assert attn(ref(one), ref(nullc), 0, OK, 4, 0, OK, None, 0, None, None) == bt.BT_ERR_NULL
    assert attn(ref(one), ref(bc), 2, OK, 4, 0, OK, None, 0, None, None) == bt.BT_ERR_SHAPE
    assert attn(ref(cfg), ref(bc), 0, OK, 4, 0, OK, OK, 16, None, None) == bt.BT_ERR_WORKSPACE
    assert attn(ref(one), ref(bc), 0, ODD, 4, 0, OK, None, 0, None, None) == bt.BT_ERR_UNSUPPORTED
    assert step(ref(cfg), ref(bc), 0, OK, None, OK, 4, 0, OK, OK, BIG, None, None) == bt.BT_ERR_NULL
    assert step(ref(cfg), ref(bc), 0, OK, OK, OK, 4, 0, OK, None, 0, None, None) == bt.BT_ERR_WORKSPACE
    assert step(ref(cfg), ref(bc), 0, OK, OK, ODD, 4, 0, OK, OK, BIG, None, None) == bt.BT_ERR_UNSUPPORTED
    assert pre(ref(cfg), OK, OK, OK, 16, 8, 4, 0, OK, None, None) == bt.BT_ERR_SHAPE
    assert pre(ref(cfg), OK, None, OK, 8, 8, 4, 0, OK, None, None) == bt.BT_ERR_NULL
    assert pre(ref(cfg), OK, OK, OK, 8, 8, 4, 0, ODD, None, None) == bt.BT_ERR_UNSUPPORTED
    assert pre(ref(plain), OK, OK, OK, 8, 8, 4, 0, OK, None, None) == bt.BT_ERR_UNSUPPORTED


def test_shared_refusals(bt):
    L = bt.lib()
    cfg = bt.make_config(4, 8, 64, 4, 1, 64, 2)
    mk = bt.binding.bt_block_cache
    bc, pc = mk(0x1000, 0x1000, 0x1000), mk(0x2000, 0x2000, 0x2000)
    attn, step = L.bt_block_decode_attn_shared, L.bt_block_decode_step_shared
    need = bt.bt_workspace_bytes_shared(cfg, 100)
    assert need > bt.bt_workspace_bytes(cfg) and need % 4 == 0
    assert bt.bt_workspace_bytes_shared(cfg, 0) == 0 and bt.bt_workspace_bytes_shared(bt.make_config(4, 8, 48, 4, 1, 64, 2), 8) == 0
    go = lambda **k: attn(ref(k.get("cfg", cfg)), k.get("p", ref(pc)), k.get("cap", 100), k.get("c", ref(bc)), k.get("layer", 0),   # noqa: E731
                          k.get("q", OK), k.get("out", OK), k.get("ws", OK), k.get("bytes", need), None, None)
    assert go(p=None) == bt.BT_ERR_NULL and go(c=None) == bt.BT_ERR_NULL and go(q=None) == bt.BT_ERR_NULL
    assert go(p=ref(mk(0, 0x1000, 0x1000))) == bt.BT_ERR_NULL and go(p=ref(mk(0x1000, 0x1000, 0))) == bt.BT_ERR_NULL
    assert go(cap=0) == bt.BT_ERR_SHAPE and go(cap=-5) == bt.BT_ERR_SHAPE and go(layer=2) == bt.BT_ERR_SHAPE
    assert go(ws=None) == bt.BT_ERR_WORKSPACE and go(bytes=need - 1) == bt.BT_ERR_WORKSPACE and go(cap=5000) == bt.BT_ERR_WORKSPACE
    assert go(ws=ODD) == bt.BT_ERR_UNSUPPORTED and go(q=ODD) == bt.BT_ERR_UNSUPPORTED and go(out=ODD) == bt.BT_ERR_UNSUPPORTED
    assert go(p=ref(mk(0x1008, 0x1000, 0x1000))) == bt.BT_ERR_UNSUPPORTED and go(p=ref(mk(0x1000, 0x1000, 0x1002))) == bt.BT_ERR_UNSUPPORTED
    assert step(ref(cfg), ref(pc), 100, ref(bc), 0, OK, None, OK, OK, OK, need, None, None) == bt.BT_ERR_NULL
    assert step(ref(cfg), ref(pc), 100, ref(bc), 0, OK, ODD, OK, OK, OK, need, None, None) == bt.BT_ERR_UNSUPPORTED
    # the prefix a step reads must not be the cache it appends to
    for same in (mk(0x1000, 0x2000, 0x2000), mk(0x2000, 0x1000, 0x2000), mk(0x2000, 0x2000, 0x1000)):
        assert step(ref(cfg), ref(same), 100, ref(bc), 0, OK, OK, OK, OK, OK, need, None, None) == bt.BT_ERR_UNSUPPORTED


def test_weights_refusals(bt):
    L = bt.lib()
    short, split = bt.make_config(4, 8, 64, 4, 1, 64, 2, decode_splits=1), bt.make_config(4, 8, 64, 4, 1, 64, 2)
    long = bt.make_config(64, 8, 64, 4, 1, 5000, 1, decode_splits=1)
    assert bt.bt_workspace_bytes_weights(short) == bt.bt_workspace_bytes(short)
    for cfg in (split, long):
        assert bt.bt_workspace_bytes_weights(cfg) >= bt.bt_workspace_bytes(cfg) + 4 * cfg.batch * cfg.heads * cfg.max_blocks
    assert bt.bt_workspace_bytes_weights(bt.make_config(4, 8, 48, 4, 1, 64, 2)) == 0
    bc = bt.binding.bt_block_cache(0x1000, 0x1000, 0x1000)
    attn, step = L.bt_block_decode_attn_weights, L.bt_block_decode_step_weights
    assert attn(ref(short), ref(bc), 0, OK, OK, OK, None, None, 0, None, None) == bt.BT_ERR_NULL
    assert attn(ref(short), ref(bc), 0, OK, None, OK, OK, None, 0, None, None) == bt.BT_ERR_NULL
    assert attn(ref(short), ref(bc), 0, OK, OK, ODD, OK, None, 0, None, None) == bt.BT_ERR_UNSUPPORTED
    assert attn(ref(short), ref(bc), 0, OK, OK, None, ODD, None, 0, None, None) == bt.BT_ERR_UNSUPPORTED
    assert attn(ref(short), ref(bc), 3, OK, OK, OK, OK, None, 0, None, None) == bt.BT_ERR_SHAPE
    for cfg in (split, long):
        assert attn(ref(cfg), ref(bc), 0, OK, OK, OK, OK, None, 0, None, None) == bt.BT_ERR_WORKSPACE
        assert attn(ref(cfg), ref(bc), 0, OK, OK, OK, OK, OK, bt.bt_workspace_bytes_weights(cfg) - 1, None, None) == bt.BT_ERR_WORKSPACE
        assert attn(ref(cfg), ref(bc), 0, OK, OK, OK, OK, ODD, BIG, None, None) == bt.BT_ERR_UNSUPPORTED
    assert step(ref(short), ref(bc), 0, OK, OK, OK, OK, OK, OK, None, 0, None, None) == bt.BT_ERR_WORKSPACE
    assert step(ref(short), ref(bc), 0, OK, OK, None, OK, OK, OK, OK, BIG, None, None) == bt.BT_ERR_NULL


def test_evict_refusals(bt):
    L = bt.lib()
    cfg = bt.make_config(4, 8, 64, 4, 1, 64, 2)
    mk = bt.binding.bt_block_cache
    bc = mk(0x1000, 0x2000, 0x3000)
    other = mk(0x4000, 0x5000, 0x6000)
    W, DW = ctypes.c_void_p(0x7000), ctypes.c_void_p(0x8000)

    def go(keep=10, trig=0, sinks=1, recent=2, dst=None, dw=None, cap=0, kept=OK, ws=OK, size=BIG, w=W, c=ref(bc), layer=0):
        return L.bt_block_kv_evict(ref(cfg), c, w, layer, keep, trig, sinks, recent, dst, dw, cap, kept, ws, size, None, None)

    assert go(c=None) == go(w=None) == go(kept=None) == bt.BT_ERR_NULL
    assert go(dst=ref(other), dw=None, cap=64) == bt.BT_ERR_NULL and go(dst=ref(mk(0x4000, 0, 0x6000)), dw=DW, cap=64) == bt.BT_ERR_NULL
    assert go(dw=DW) == bt.BT_ERR_NULL
    for bad in (dict(keep=0), dict(keep=-1), dict(sinks=-1), dict(recent=-1), dict(trig=-1), dict(sinks=9), dict(sinks=11, recent=0),
                dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), dict(layer=2), dict(dst=ref(other), dw=DW, cap=0)):
        assert go(**bad) == bt.BT_ERR_SHAPE, bad
    assert go(ws=None) == go(size=16) == bt.BT_ERR_WORKSPACE
    assert go(dst=ref(other), dw=DW, cap=9) == bt.BT_ERR_CAPACITY
    assert go(dst=ref(other), dw=DW, cap=39, trig=41) == bt.BT_ERR_CAPACITY
    for same in (mk(0x1000, 0x5000, 0x6000), mk(0x4000, 0x2000, 0x6000), mk(0x4000, 0x5000, 0x3000)):
        assert go(dst=ref(same), dw=DW, cap=64) == bt.BT_ERR_UNSUPPORTED
    assert go(dst=ref(other), dw=W, cap=64) == bt.BT_ERR_UNSUPPORTED
    assert go(w=ODD) == go(ws=ODD) == go(kept=ctypes.c_void_p(0x1002)) == bt.BT_ERR_UNSUPPORTED
    assert go(dst=ref(mk(0x4008, 0x5000, 0x6000)), dw=DW, cap=64) == bt.BT_ERR_UNSUPPORTED
    assert go(dst=ref(other), dw=ODD, cap=64) == bt.BT_ERR_UNSUPPORTED


@pytest.mark.parametrize("keep", [2 ** 30 + 1, 2 ** 31 - 1])
def test_evict_refuses_more_rows_than_it_can_count(bt, keep):
    cfg, bc = bt.make_config(1, 1, 64, 4, 1, 64, 1), bt.binding.bt_block_cache(0x1000, 0x2000, 0x3000)
    assert bt.lib().bt_block_kv_evict(ref(cfg), ref(bc), OK, 0, keep, 0, 0, 0, None, None, 0, OK, OK, 16, None, None) == bt.BT_ERR_SHAPE


def test_definitions_agree_with_brute_force():
    rng = np.random.default_rng(0)
    q, K, V = rng.normal(size=16), rng.normal(size=(9, 16)), rng.normal(size=(9, 16))
    out, p, tol, _ = ctx.attend(q, K, V)
    e = [np.exp(sum(q * K[j]) / 4.0) for j in range(9)]
    assert np.allclose(p, np.array(e) / sum(e)) and np.allclose(out, sum(e[j] * V[j] for j in range(9)) / sum(e))
    assert (tol > 0).all() and (tol < 0.1).all()
    assert ctx.window_rows(10, 3, 2) == [0, 1, 7, 8, 9] and ctx.window_rows(4, 3, 2) == [0, 1, 2, 3] and ctx.window_rows(0, 3, 2) == []
    # a prefix and own rows are one row range
    a, _ = ctx.decode_shared(q[None, None], K[None, :6], V[None, :6], 4, K[None, None], V[None, None], [3])
    b, *_ = ctx.attend(q, np.concatenate([K[:4], K[:3]]), np.concatenate([V[:4], V[:3]]))
    assert np.allclose(a[0, 0], b)
    # weights of one step add up to one per (sequence, head)
    _, _, new, _ = ctx.decode_weights(q[None, None], K[None, None], V[None, None], [9], np.zeros((1, 1, 9)))
    assert np.isclose(new.sum(), 1.0)
    # eviction: the ends stay, then the heaviest, ties by index, NaN last
    sums = np.array([0, 5, 1, 1, np.nan, -np.inf, 7, 0, 9, 2], np.float32)
    assert ctx.evicted(sums, 10, 5, 1, 2) == [0, 1, 6, 8, 9]
    assert ctx.evicted(sums, 10, 4, 0, 0) == [1, 6, 8, 9]
    assert ctx.evicted(sums, 10, 9, 0, 0) == [0, 1, 2, 3, 5, 6, 7, 8, 9]
    assert ctx.evicted(np.zeros(6, np.float32), 6, 3, 0, 1) == [0, 1, 5]


@pytest.mark.parametrize("counts", [(2 ** 31 - 1, 0, 0), (2 ** 32 + 5, 1, 1), (5, 2 ** 32 + 1, 0), (5, 0, 2 ** 32), (-2 ** 32 + 5, 0, 0)])
def test_evict_refuses_counts_that_no_int_holds(bt, counts):
    """Through the binding, `kept` left to it: refused, not taken modulo 2^32 and not answered with an allocation of that many rows."""
    import torch

    cfg = bt.make_config(64, 16, 64, 4, 1, 8, 1)
    cache = bt.BlockCache(cfg, device="cpu")
    keep, sinks, recent = counts
    with pytest.raises(bt.BtError) as e:
        bt.bt_block_kv_evict(cfg, cache, torch.zeros(1, 64, 16, 8), 0, keep, sinks, recent, torch.zeros(1 << 16), stream=0)
    assert e.value.code == bt.BT_ERR_SHAPE
