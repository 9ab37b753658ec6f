"""Attention over the 4-bit cache where values are as large as bf16 goes or of unlike size in groups of dimensions, against its float64 definition."""
import numpy as np
import pytest
import torch

from oracle import contexts as ctx
from oracle import lowbit as lb

from test_gpu_lowbit import bits, check, f64, filled, rnd
from util import status_word, to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bt():
    import paper_2406_02657_b200 as bt
    assert torch.cuda.is_available()
    return bt


def keys_of(levels, hd):
    """Rows K [..., hd] that a query with 8 in its first dimension scores with `levels` (base 2), under the usual scale."""
    k = np.zeros((*levels.shape, hd))
    k[..., 0] = levels * np.log(2.0) * np.sqrt(hd) / 8.0
    return k


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rise", [0.9, 1.9, 2.6, 3.6, 7.0])
def test_values_near_the_end_of_bf16(bt, hd, rise):
    """V of 1e38 to 3.3e38 under scores that rise from 128 rows to the next 128, more or less than weights may before all become relative to
    something else: a weight above one times such a step has to stay a number."""
    B, H, N = 3, 2, 700
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=1)
    rng = np.random.default_rng(int(10 * rise))
    q = f64(rnd(31, 3, (B, H, hd)))
    q[..., 0] = 8.0
    k = keys_of(np.broadcast_to(rise * (np.arange(N) // 128), (B, H, N)), hd)
    v = rng.uniform(1e38, 3.3e38, (B, H, N, hd))
    v[1] *= rng.choice([-1.0, 1.0], (H, N, hd))
    v[2, :, :300] *= 1e-30                       # the huge ones come late
    q, k, v = bits(q), bits(k), bits(v)
    lens = [N, 517, 400]
    cache, st = filled(bt, cfg, k, v, lens), status_word()
    out, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), bt.alloc_workspace_kv4(cfg)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(q), out, ws, dev_status=st)
    ref, tol = lb.decode(f64(q), lb.held(f64(k)), lb.held(f64(v)), lens)
    check(out, ref, tol, f"rise {rise}")
    assert st.item() == 0


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [2, 3, 40])
@pytest.mark.parametrize("rise", [0.0, 1.9, 3.6])
def test_parts_near_the_end_of_bf16_are_joined(bt, hd, splits, rise):
    """Parts whose results are 1e38 to 3.3e38 each: their weighted sum is no larger than the largest of them."""
    B, H, N = 2, 2, 2600
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    rng = np.random.default_rng(splits)
    q = f64(rnd(32, 3, (B, H, hd)))
    q[..., 0] = 8.0
    k = keys_of(np.broadcast_to(rise * (np.arange(N) // 900), (B, H, N)), hd)
    v = rng.uniform(1e38, 3.3e38, (B, H, N, hd))
    v[1] *= -1.0
    q, k, v = bits(q), bits(k), bits(v)
    lens = [N, 1111]
    cache, st = filled(bt, cfg, k, v, lens), status_word()
    out, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), bt.alloc_workspace_kv4(cfg)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(q), out, ws, dev_status=st)
    ref, tol = lb.decode(f64(q), lb.held(f64(k)), lb.held(f64(v)), lens)
    check(out, ref, tol, f"{splits} parts, rise {rise}")
    assert st.item() == 0


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("apart", [10, 20, 30, 60])
def test_groups_of_unlike_size_keep_their_own_precision(bt, hd, splits, apart):
    """V whose groups of 32 dimensions are 2^apart and more from each other, within a plane of 64 dimensions and across the two, and change
    places along the rows of one sequence: each has the bound of its own size."""
    B, H, N = 3, 4, 600
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    q, k, v = f64(rnd(33, 3, (B, H, hd))), f64(rnd(33, 1, (B, H, N, hd))), f64(rnd(33, 2, (B, H, N, hd)))
    groups = hd // 32
    for h in range(H):
        size = np.repeat(2.0 ** -(apart * ((np.arange(groups) + h) % groups)), 32)
        v[:, h] *= size
        v[1, h, 300:] = v[1, h, 300:] / size * size[::-1]
    v[2, :, :, :32] = 0.0                        # a group without any size
    q, k, v = bits(q), bits(k), bits(v)
    lens = [N, 587, 130]
    cache = filled(bt, cfg, k, v, lens)
    out, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), bt.alloc_workspace_kv4(cfg)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(q), out, ws)
    held = lb.held(f64(v))
    ref, tol = lb.decode(f64(q), lb.held(f64(k)), held, lens)
    check(out, ref, tol, f"{apart} apart")
    # what the bound itself is worth: a hundredth of the largest value of the group, at most
    for b, n in enumerate(lens):
        largest = np.abs(held[b, :, :n]).max(1).reshape(H, groups, 32).max(2)
        assert (tol[b].reshape(H, groups, 32) <= 0.01 * largest[..., None] + 2e-30).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("apart", [10, 18, 30])
def test_groups_of_a_query_keep_their_own_precision(bt, hd, splits, apart):
    """Queries whose groups of 32 dimensions are 2^apart and more from each other, and keys that are so the other way round: every group
    has its part in the scores."""
    B, H, N = 2, 4, 300
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    q, k, v = f64(rnd(36, 3, (B, H, hd))), f64(rnd(36, 1, (B, H, N, hd))), rnd(36, 2, (B, H, N, hd))
    for h in range(H):
        size = np.repeat(2.0 ** -(apart * ((np.arange(hd // 32) + h) % (hd // 32))), 32)
        q[:, h] *= size
        k[:, h] /= size
    q, k = bits(q), bits(k)
    lens = [N, 177]
    cache = filled(bt, cfg, k, v, lens)
    out, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), bt.alloc_workspace_kv4(cfg)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(q), out, ws)
    ref, tol = lb.decode(f64(q), lb.held(f64(k)), lb.held(f64(v)), lens)
    check(out, ref, tol, f"{apart} apart")
    assert tol.max() < 0.03                      # what the bound itself is worth


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("where", ["another group", "the same group"])
def test_huge_queries_and_keys_that_do_not_meet(bt, hd, where):
    """A query and keys of 2^80 in different dimensions, of the same group of 32 or not: their products are zeros, and the scores come from the rest."""
    B, H, N = 2, 2, 150
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    q, k, v = np.zeros((B, H, hd)), np.zeros((B, H, N, hd)), rnd(37, 2, (B, H, N, hd))
    q[..., 3], q[..., 40] = 2.0 ** 80, 2.0
    k[..., 40] = f64(rnd(37, 1, (B, H, N)))
    k[..., 20 if where == "the same group" else 50] = 2.0 ** 80
    if where == "another group":
        q[..., 40], q[..., 5], k[..., 40] = 0.0, 2.0, 0.0
        k[..., 3] = f64(rnd(37, 1, (B, H, N))) * 2.0 ** -80
    q, k = bits(q), bits(k)
    lens = [N, 99]
    cache = filled(bt, cfg, k, v, lens)
    out, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), bt.alloc_workspace_kv4(cfg)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(q), out, ws)
    q, K, V = f64(q), lb.held(f64(k)), lb.held(f64(v))
    assert np.ptp((K * q[:, :, None]).sum(-1)) > 4.0 / np.sqrt(hd)
    # the definition over what meets: the query's rounding leaves powers of two and zeros what they are, so that it adds nothing here
    for b, n in enumerate(lens):
        for h in range(H):
            ref, _, tol, _ = ctx.attend(q[b, h], np.where(q[b, h] != 0, K[b, h, :n], 0.0), V[b, h, :n])
            check(out[b, h], ref, tol + n * 2.0 ** -29 * 1.01 * np.abs(V[b, h, :n]).max(), where)
