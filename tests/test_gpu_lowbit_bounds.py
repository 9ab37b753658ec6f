"""The low-bit operators at their edges: nothing outside the rows that a call may write changes, caches of more than 2^32 bytes, captured
graphs that share a workspace, calls behind one another without a pause, and random configurations against the definitions."""
import numpy as np
import pytest
import torch

from oracle import lowbit as lb
from workloads import gen

from test_gpu_lowbit import FILL, check, cuda, f64, filled, operands, rnd, tiles_of
from util import status_word, to_dev, to_f64

pytestmark = pytest.mark.gpu

GUARD, PATTERN = 4096, 0x5A


@pytest.fixture(scope="module")
def bt():
    import paper_2406_02657_b200 as bt
    assert torch.cuda.is_available()
    return bt


class Guarded:
    """A device tensor carved out of a larger byte buffer with guard bytes on both sides."""

    def __init__(self, shape, dtype, fill=None):
        n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        self.raw = torch.full((GUARD + n + (-n) % 256 + GUARD,), PATTERN, dtype=torch.uint8, device="cuda")
        self.t, self.n = self.raw[GUARD:GUARD + n].view(dtype).view(shape), n
        if fill is not None:
            self.t.copy_(fill)

    def intact(self):
        return bool((self.raw[:GUARD] == PATTERN).all()) and bool((self.raw[GUARD + self.n:] == PATTERN).all())


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_cache_calls_touch_nothing_else(bt, hd, splits):
    rng = np.random.default_rng(splits)
    B, H, N = 21, 5, 100                       # the last tile is there in part
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    lens = rng.integers(0, N + 1, B).astype(np.int32)
    lens[0], lens[1], lens[2] = 0, N, N - 1
    k, v = rnd(70 + splits, 0, (B, H, N, hd)), rnd(70 + splits, 1, (B, H, N, hd))
    source = filled(bt, cfg, k, v, lens)
    kv, ln = Guarded(source.kv.shape, torch.uint8, source.kv), Guarded((1, B), torch.int32, source.len)
    cache = bt.BlockCacheKV4(cfg, kv=kv.t, length=ln.t)
    ws = Guarded((bt.bt_workspace_bytes_kv4(cfg),), torch.uint8)
    bt.bt_workspace_init(cfg, ws.t)
    q, kn, vn = (Guarded((B, H, hd), torch.bfloat16, to_dev(rnd(70 + splits, 2 + i, (B, H, hd)))) for i in range(3))
    out, ko, vo = Guarded((B, H, hd), torch.bfloat16), Guarded((B, H, 37, hd), torch.bfloat16), Guarded((B, H, 37, hd), torch.bfloat16)
    everything = (kv, ln, ws, q, kn, vn, out, ko, vo)
    before = cache.kv.clone()
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, q.t, out.t, ws.t)
    bt.bt_block_kv4_read(cfg, cache, 0, ko.t, vo.t, first=33)
    assert torch.equal(cache.kv, before) and all(g.intact() for g in everything)
    bt.bt_block_decode_step_kv4(cfg, cache, 0, q.t, kn.t, vn.t, out.t, ws.t)
    bt.bt_block_kv4_append(cfg, cache, 0, kn.t.view(B, H, 1, hd), vn.t.view(B, H, 1, hd))
    torch.cuda.synchronize()
    assert all(g.intact() for g in everything)
    tiles = before[0].cpu().numpy()            # the definition's rows written behind what was there, byte for byte
    for b in range(B):
        for h in range(H):
            for r in range(int(lens[b]), min(N, int(lens[b]) + 2)):
                lb.write_tiles(tiles[b, h], r, f64(kn_bits(kn, b, h)), f64(kn_bits(vn, b, h)))
    assert np.array_equal(cache.kv[0].cpu().numpy(), tiles)
    assert cache.len[0].tolist() == [min(N, int(n) + 2) for n in lens]


def kn_bits(g, b, h):
    return gen.torch_to_bits(g.t[b, h].contiguous())[None]


@pytest.mark.parametrize("n", [1, 5])
def test_projections_touch_nothing_else(bt, n):
    B, H, hd, N = 37, 3, 64, 41
    D = H * hd
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    lens = [(b * 11) % (N + 1) for b in range(B)]
    x8, xs, w8, ws, bias = operands(91, B * n, 3 * D, D)
    kv = Guarded((1, B, H, 3, 1, lb.TILE_BYTES), torch.uint8, torch.full((1,), FILL, dtype=torch.uint8))
    ln = Guarded((1, B), torch.int32, torch.tensor([lens], dtype=torch.int32))
    cache, q = bt.BlockCacheKV4(cfg, kv=kv.t, length=ln.t), Guarded((B, H, n, hd), torch.bfloat16)
    steps, feats = Guarded((B * n,), torch.float32, torch.from_numpy(xs)), Guarded((3 * D,), torch.float32, torch.from_numpy(ws))
    xg, wg = Guarded((B, n, D), torch.int8, torch.from_numpy(x8).view(B, n, D)), Guarded((3 * D, D), torch.int8, torch.from_numpy(w8))
    bt.bt_block_qkv_project_append_i8_kv4(cfg, cache, 0, xg.t, steps.t, wg.t, feats.t, to_dev(bias), q.t)
    assert all(g.intact() for g in (kv, ln, q, steps, feats, xg, wg))
    # the rows appended are the two calls' (see the parity tests); here: that no other byte of the cache has changed
    want = tiles_of(cfg)
    touched = np.zeros_like(want, bool)
    for b, m in enumerate(lens):
        for r in range(m, m + n if m + n <= N else m):
            for j in range(32):
                touched[b, :, r // 16, 0, [lb.k_byte(r % 16, j), lb.v_byte(r % 16, j)]] = True
            for part in (1024, 1088):
                touched[b, :, r // 16, 0, part + r % 16 * 4: part + r % 16 * 4 + 4] = True
    got = cache.kv[0].cpu().numpy()
    assert (got[~touched] == FILL).all() and (got[touched] != FILL).any()
    # rows quantised into a buffer between guards, and read from one
    x = Guarded((B * n, D), torch.bfloat16, to_dev(rnd(92, 0, (B * n, D))))
    o8, os = Guarded((B * n, D), torch.int8), Guarded((B * n,), torch.float32)
    bt.bt_rows_quantize_i8(x.t, o8.t, os.t)
    assert all(g.intact() for g in (x, o8, os))


def test_cache_of_more_than_4_gigabytes(bt):
    """Rows behind 2^32 bytes: appended, read back and attended over."""
    B, H, hd, N = 5, 16, 64, 800_000           # 57.6 MB a (sequence, head), 4.6 GB
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    kv = torch.randint(0, 256, (1, B, H, N // 16, 1, lb.TILE_BYTES), dtype=torch.uint8, device="cuda", generator=g)
    kv[..., 1024:] = torch.tensor([0x20, 0x3E] * 64, dtype=torch.uint8, device="cuda")    # every step 0.15625
    cache = bt.BlockCacheKV4(cfg, kv=kv)
    assert kv.numel() > 2 ** 32
    n = N - 3
    cache.len.fill_(n)
    k, v, q = (to_dev(rnd(93, i, (B, H, 1, hd))) for i in range(3))
    out, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), bt.alloc_workspace_kv4(cfg)
    bt.bt_block_decode_step_kv4(cfg, cache, 0, q, k, v, out, ws)
    bt.bt_block_kv4_append(cfg, cache, 0, k, v)
    ko, vo = (torch.empty((B, H, 70, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bt.bt_block_kv4_read(cfg, cache, 0, ko, vo, first=N - 71)
    held = torch.from_numpy(lb.to_bf16(lb.held(to_f64(k)))).cuda()
    for row in (n, n + 1):
        assert torch.equal(ko[:, :, row - (N - 71)].double(), held[:, :, 0])
    assert (cache.len == n + 2).all()
    # the last (sequence, head) against its own rows: codes times 0.15625 have five bits, so that reading them back rounds nothing
    one = bt.make_config(1, 1, hd, 4, 1, N, 1)
    last = bt.BlockCacheKV4(one, kv=kv[:, -1:, -1:].contiguous(), length=torch.full((1, 1), n, dtype=torch.int32, device="cuda"))
    K, V = (torch.zeros((1, 1, n + 1, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bt.bt_block_kv4_read(one, last, 0, K, V)
    rows = [to_f64(t) for t in (K, V)]
    for t, new in zip(rows, (k, v)):
        t[0, 0, n] = lb.held(to_f64(new)[-1, -1, 0])
    ref, tol = lb.decode(to_f64(q)[-1:, -1:, 0], *rows, [n + 1])
    check(out[-1:, -1:], ref, tol, "the last rows")


def test_graphs_that_share_a_workspace(bt):
    """Two captured graphs over one workspace, replayed in turn; steps of both grow the cache as eager calls would."""
    B, H, hd, N = 7, 4, 128, 600
    cfg = bt.make_config(B, H, hd, 4, 1, N, 2)
    caches, ws = [bt.BlockCacheKV4(cfg) for _ in range(2)], bt.alloc_workspace_kv4(cfg)
    rows = [[to_dev(rnd(94, 10 * layer + i, (B, H, 333, hd))) for i in range(2)] for layer in range(2)]
    for c in caches:
        for layer in range(2):
            bt.bt_block_kv4_append(cfg, c, layer, *rows[layer], reset_first=True)
    q, k, v = (to_dev(rnd(95, i, (B, H, hd))) for i in range(3))
    outs = [torch.empty((2, B, H, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    graphs = []
    for layer in range(2):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            bt.bt_block_decode_step_kv4(cfg, caches[0], layer, q, k, v, outs[0][layer], ws)
        graphs.append(g)
    for step in range(4):
        for layer in range(2):
            graphs[layer].replay()
            bt.bt_block_decode_step_kv4(cfg, caches[1], layer, q, k, v, outs[1][layer], ws)
        assert torch.equal(outs[0], outs[1]), step
    assert torch.equal(caches[0].kv, caches[1].kv) and (caches[0].len == 337).all()


def test_calls_without_a_pause(bt):
    """A chain of dependent launches, each of which may start while the one before it drains: append, step, read and projections in turn,
    against the same calls with the GPU waited for in between."""
    B, H, hd, N = 64, 16, 64, 200
    D = H * hd // 2                            # 8 heads for the projection
    cfg, pcfg = bt.make_config(B, H, hd, 4, 1, N, 1), bt.make_config(B, H // 2, hd, 4, 1, N, 1)
    x8, xs, w8, ws8, bias = operands(96, B, 3 * D, D)
    x8, xs, w8, ws8, bias = cuda(x8).view(B, 1, D), cuda(xs), cuda(w8), cuda(ws8), to_dev(bias)
    k, v = (to_dev(rnd(97, i, (B, H, 30, hd))) for i in range(2))
    q = to_dev(rnd(97, 5, (B, H, hd)))
    results = []
    for pause in (False, True):
        cache, small = bt.BlockCacheKV4(cfg), bt.BlockCacheKV4(pcfg)
        ws, small_ws = bt.alloc_workspace_kv4(cfg), bt.alloc_workspace_kv4(pcfg)
        wait = torch.cuda.synchronize if pause else (lambda: None)
        outs = []
        torch.cuda.synchronize()
        for i in range(5):
            out, qp = torch.empty_like(q), torch.empty((B, H // 2, 1, hd), dtype=torch.bfloat16, device="cuda")
            bt.bt_block_kv4_append(cfg, cache, 0, k, v, reset_first=i == 0)
            wait()
            bt.bt_block_decode_step_kv4(cfg, cache, 0, q, k[:, :, i].contiguous(), v[:, :, i].contiguous(), out, ws)
            wait()
            bt.bt_block_qkv_project_append_i8_kv4(pcfg, small, 0, x8, xs, w8, ws8, bias, qp)
            wait()
            so = torch.empty_like(qp)
            bt.bt_block_decode_attn_kv4(pcfg, small, 0, qp, so, small_ws)
            wait()
            ko, vo = (torch.zeros((B, H, 31 * (i + 1), hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            bt.bt_block_kv4_read(cfg, cache, 0, ko, vo)
            wait()
            outs += [out, qp, so, ko, vo, cache.len.clone(), small.len.clone()]
        torch.cuda.synchronize()
        results.append(outs)
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("seed", range(24))
def test_random_configurations(bt, seed):
    rng = np.random.default_rng(1000 + seed)
    hd = int(rng.choice([64, 128]))
    H, B = int(rng.integers(1, 17 if hd == 64 else 9)), int(rng.integers(1, 12))
    N = int(np.exp(rng.uniform(0, np.log(900))))
    N, layers = max(1, N), int(rng.integers(1, 3))
    cfg = bt.make_config(B, H, hd, 4, 1, N, layers, decode_splits=int(rng.choice([0, 0, 1, 2, 5, 33])))
    layer = layers - 1
    lens = [int(rng.integers(0, N + 1)) for _ in range(B)]
    scale_k, scale_v = 2.0 ** rng.uniform(-6, 3), 2.0 ** rng.uniform(-40, 40)
    from_bits = lambda x: gen.f32_to_bf16_bits(np.asarray(x, np.float32))   # noqa: E731
    k, v = from_bits(f64(rnd(seed, 1, (B, H, N, hd))) * scale_k), from_bits(f64(rnd(seed, 2, (B, H, N, hd))) * scale_v)
    q, kn, vn = rnd(seed, 3, (B, H, hd)), from_bits(f64(rnd(seed, 4, (B, H, hd))) * scale_k), from_bits(f64(rnd(seed, 5, (B, H, hd))) * scale_v)
    cache, st, ws = filled(bt, cfg, k, v, lens, layer=layer), status_word(), bt.alloc_workspace_kv4(cfg)
    out = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda")
    bt.bt_block_decode_step_kv4(cfg, cache, layer, to_dev(q), to_dev(kn), to_dev(vn), out, ws, dev_status=st)
    n = [min(N, m + 1) for m in lens]
    for b in range(B):
        if lens[b] < N:
            k[b, :, lens[b]], v[b, :, lens[b]] = kn[b], vn[b]
    ref, tol = lb.decode(f64(q), lb.held(f64(k)), lb.held(f64(v)), n)
    check(out, ref, tol, f"B {B} H {H} hd {hd} N {N}")
    assert cache.len[layer].tolist() == n and st.item() == (bt.BT_DEV_OVERFLOW if N in lens else 0)
