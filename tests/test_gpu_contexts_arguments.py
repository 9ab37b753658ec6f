"""GPU tests of arguments of the operators for long and shared contexts that the other tests leave at their usual values."""
import pytest
import torch

from workloads import gen

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
