"""The workspace of the decode calls over the 4-bit cache: its arrival counters are at zero after every call."""
import pytest
import torch

from test_gpu_lowbit import filled, rnd
from util import status_word, to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bt():
    import paper_2406_02657_b200 as bt
    assert torch.cuda.is_available()
    return bt


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [0, 1, 5, 64])
def test_counters_are_left_at_zero(bt, hd, splits):
    """Attention and steps, with sequences that are empty or full among them; the counters are the last B * H + B words of bt_workspace_bytes."""
    lens = [0, 63, 64, 200, 299, 300, 300]
    B, H, N = len(lens), 3, 300
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    k, v = rnd(34, 1, (B, H, N, hd)), rnd(34, 2, (B, H, N, hd))
    cache, ws, st = filled(bt, cfg, k, v, lens), bt.alloc_workspace_kv4(cfg), status_word()
    words = bt.bt_workspace_bytes(cfg) // 4
    counters = ws.view(torch.int32)[words - B * H - B:words]
    assert counters.numel() == B * H + B and not counters.any()
    q, kn, vn = (to_dev(rnd(35, i, (B, H, hd))) for i in range(3))
    out = torch.empty_like(q)
    for _ in range(3):
        bt.bt_block_decode_attn_kv4(cfg, cache, 0, q, out, ws, dev_status=st)
        assert not counters.any()
        bt.bt_block_decode_step_kv4(cfg, cache, 0, q, kn, vn, out, ws, dev_status=st)
        assert not counters.any()
    assert cache.len[0].tolist() == [min(N, n + 3) for n in lens] and st.item() == bt.BT_DEV_EMPTY | bt.BT_DEV_OVERFLOW
