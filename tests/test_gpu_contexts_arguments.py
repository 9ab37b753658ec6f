"""GPU tests of arguments of the operators for long and shared contexts that the other tests leave at their usual values."""
import numpy as np
import pytest
import torch

from oracle import contexts as ctx
from workloads import gen

from test_gpu_contexts import check, f64, make_cache, rnd, shared_case
from util import status_word, to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bt():
    import paper_2406_02657_b200 as bt
    assert torch.cuda.is_available()
    return bt


@pytest.mark.parametrize("window,sinks", [(2 ** 32 + 1, 0), (2 ** 63 - 1, 2 ** 63 - 1), (2, 2 ** 32)])
def test_window_of_more_rows_than_an_int_holds_is_all_rows(bt, window, sinks):
    B, H, hd, N = 70, 16, 64, 150
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    x, k, v = (gen.normal_bf16_device(70, i, (B, H, N, hd), device="cuda") for i in range(3))
    a, b = torch.empty_like(x), torch.empty_like(x)
    bt.bt_block_prefill_attn(cfg, x, k, v, a)
    bt.bt_block_prefill_attn_window(cfg, x, k, v, window, sinks, b)
    assert torch.equal(a, b)
    ws = bt.alloc_workspace(cfg)
    q, kn, vn = (gen.normal_bf16_device(71, i, (B, H, hd), device="cuda") for i in range(3))
    outs = []
    for step in (bt.bt_block_decode_step_window, bt.bt_block_decode_attn_window):
        cache = bt.BlockCache(cfg, k=k[None].clone(), v=v[None].clone())
        cache.len.fill_(N - 1)
        wide, plain = torch.empty_like(q), torch.empty_like(q)
        if step is bt.bt_block_decode_step_window:
            step(cfg, cache, 0, q, kn, vn, window, sinks, wide, ws)
            cache.len.fill_(N - 1)
            bt.bt_block_decode_step(cfg, cache, 0, q, kn, vn, plain, ws)
        else:
            step(cfg, cache, 0, q, window, sinks, wide, ws)
            bt.bt_block_decode_attn(cfg, cache, 0, q, plain, ws)
        assert torch.equal(wide, plain)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("scale", [0.02, 0.4])
def test_softmax_scale_of_the_config(bt, hd, scale):
    """cfg->softmax_scale instead of 1 / sqrt(head_dim): every call against its definition, whose scale is the usual one, with the
    queries (in 64 bits) multiplied by what is between the two."""
    lens = [0, 1, 40, 99, 128, 129]
    B, H, N, cap, S, T = len(lens), 4, 130, 140, 133, 130
    _, cache, prefix, k, v, pk, pv = shared_case(bt, B, H, hd, cap, S, N, lens, seed=72)
    q, kn, vn = (rnd(73, i, (B, H, hd)) for i in range(3))
    factor = scale * hd ** 0.5
    for splits in (1, 3):
        cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits, softmax_scale=scale)
        out, st = torch.zeros((B, H, hd), dtype=torch.bfloat16, device="cuda"), status_word()
        K, V, Q = f64(k), f64(v), f64(q) * factor
        bt.bt_block_decode_attn_window(cfg, cache, 0, to_dev(q), 50, 3, out, bt.alloc_workspace(cfg), dev_status=st)
        check(out, *ctx.decode_window(Q, K, V, lens, 50, 3), "window")
        bt.bt_block_decode_attn_shared(cfg, prefix, cache, 0, to_dev(q), out, bt.alloc_workspace_shared(cfg, cap), dev_status=st)
        check(out, *ctx.decode_shared(Q, f64(pk), f64(pv), S, K, V, lens), "shared")
        sums = torch.zeros((1, B, H, N), device="cuda")
        bt.bt_block_decode_attn_weights(cfg, cache, 0, to_dev(q), out, None, sums, bt.alloc_workspace_weights(cfg), dev_status=st)
        o, tol, new, new_tol = ctx.decode_weights(Q, K, V, lens, np.zeros((B, H, N)))
        check(out, o, tol, "weights")
        assert (np.abs(sums[0].double().cpu().numpy() - new) <= new_tol).all()
        # appended rows
        for b, n in enumerate(lens):
            K[b, :, n], V[b, :, n] = f64(kn[b]), f64(vn[b])
        one = [n + 1 for n in lens]
        for call in ("window", "shared", "weights"):
            mine = make_cache(bt, cfg, k, v, lens)
            if call == "window":
                bt.bt_block_decode_step_window(cfg, mine, 0, to_dev(q), to_dev(kn), to_dev(vn), 50, 3, out, bt.alloc_workspace(cfg))
                ref = ctx.decode_window(Q, K, V, one, 50, 3)
            elif call == "shared":
                bt.bt_block_decode_step_shared(cfg, prefix, mine, 0, to_dev(q), to_dev(kn), to_dev(vn), out, bt.alloc_workspace_shared(cfg, cap))
                ref = ctx.decode_shared(Q, f64(pk), f64(pv), S, K, V, one)
            else:
                bt.bt_block_decode_step_weights(cfg, mine, 0, to_dev(q), to_dev(kn), to_dev(vn), out, None, sums, bt.alloc_workspace_weights(cfg))
                ref = ctx.decode_weights(Q, K, V, one, np.zeros((B, H, N)))[:2]
            check(out, *ref, f"{call} step")
    x, y, z = (rnd(74, i, (2, H, T, hd)) for i in range(3))
    cfg = bt.make_config(2, H, hd, 4, 1, T, 1, softmax_scale=scale)
    o = torch.zeros((2, H, T, hd), dtype=torch.bfloat16, device="cuda")
    bt.bt_block_prefill_attn_window(cfg, to_dev(x), to_dev(y), to_dev(z), 30, 5, o)
    for b in range(2):
        for h in range(H):
            check(o[b, h], *ctx.prefill_window(f64(x[b, h]) * factor, f64(y[b, h]), f64(z[b, h]), 30, 5), "prefill")
    y[0, 0, 50, 3] = 0x7FC0                    # ... and rows that are worked out again: those that share a tile with this one
    z[0, 1, 50, 3] = 0x7FC0
    bt.bt_block_prefill_attn_window(cfg, to_dev(x), to_dev(y), to_dev(z), 30, 5, o)
    for h in range(2):
        some = [t for t in range(T) if not 50 <= t < 80]
        check(o[0, h, some], *ctx.prefill_window(f64(x[0, h]) * factor, np.nan_to_num(f64(y[0, h])), np.nan_to_num(f64(z[0, h])), 30, 5, some), "again")
