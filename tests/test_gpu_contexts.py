"""GPU parity of the operators for long and shared contexts (window with sinks, shared prefix, summed weights, eviction)
against their float64 definitions.  Bounds on the rounding error come with the definitions; rows, lengths, kept indices
and everything that only moves are compared bit for bit."""
import numpy as np
import pytest
import torch

from oracle import contexts as ctx
from workloads import gen

from util import status_word, to_dev, to_f64

pytestmark = pytest.mark.gpu

NAN = 0x7FC0


@pytest.fixture(scope="module")
def bt():
    import paper_2406_02657_b200 as bt
    assert torch.cuda.is_available()
    return bt


def rnd(seed, tid, shape):
    return gen.normal_bf16_bits(seed, tid, shape)


def f64(bits):
    return gen.bf16_bits_to_f32(bits).astype(np.float64)


def check(got, ref, tol, what):
    g = to_f64(got).reshape(ref.shape)
    assert np.isfinite(g).all(), f"{what}: non-finite output"
    over = np.abs(g - ref) - tol
    assert (over <= 0).all(), f"{what}: {over.max():.3e} beyond the bound at {np.unravel_index(over.argmax(), over.shape)}"


def make_cache(bt, cfg, k, v, lens, layer=0):
    """A cache whose rows at and past each length hold NaN."""
    k, v = k.copy(), v.copy()
    for b, n in enumerate(lens):
        k[b, :, n:] = NAN
        v[b, :, n:] = NAN
    cache = bt.BlockCache(cfg)
    cache.k[layer].copy_(to_dev(k))
    cache.v[layer].copy_(to_dev(v))
    cache.len[layer].copy_(torch.tensor(lens, dtype=torch.int32))
    return cache


# ------------------------------------------------------------------------------------------------ window, decode

LENS = [0, 1, 31, 32, 33, 127, 258, 260, 261]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [0, 1, 3, 7])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 4), (32, 0), (100, 33), (64, 200), (300, 5), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_window_decode(bt, hd, splits, window, sinks):
    B, H, N = len(LENS), 3, 261
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    k, v, q = rnd(1, 1, (B, H, N, hd)), rnd(1, 2, (B, H, N, hd)), rnd(1, 3, (B, H, hd))
    kp, vp = k.copy(), v.copy()
    for b, n in enumerate(LENS):   # a row that is not seen may hold anything
        hidden = sorted(set(range(n)) - set(ctx.window_rows(n, window, sinks)))
        kp[b, :, hidden] = NAN
        vp[b, :, hidden] = 0x7F80 if b % 2 else NAN
    cache = make_cache(bt, cfg, kp, vp, LENS)
    out, st, ws = torch.full((B, H, hd), 7.0, dtype=torch.bfloat16, device="cuda"), status_word(), bt.alloc_workspace(cfg)
    for _ in range(2):
        bt.bt_block_decode_attn_window(cfg, cache, 0, to_dev(q), window, sinks, out, ws, dev_status=st)
        ref, tol = ctx.decode_window(f64(q), f64(k), f64(v), LENS, window, sinks)
        check(out, ref, tol, f"window {window} sinks {sinks}")
    assert st.item() == bt.BT_DEV_EMPTY and (out[0] == 0).all()
    assert not ws.view(torch.int32)[-(B * H + B):].any()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [1, 4])
def test_window_step(bt, hd, splits):
    """Three steps: the appended row is always seen, a full cache overflows and is attended as it is."""
    B, H, N, window, sinks = len(LENS), 2, 261, 40, 3
    cfg = bt.make_config(B, H, hd, 4, 1, N, 2, decode_splits=splits)
    k, v = rnd(2, 1, (B, H, N, hd)), rnd(2, 2, (B, H, N, hd))
    cache = make_cache(bt, cfg, k, v, LENS, layer=1)
    n, ws = list(LENS), bt.alloc_workspace(cfg)
    out = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda")
    for step in range(3):
        q, kn, vn = (rnd(3, 3 * step + i, (B, H, hd)) for i in range(3))
        st = status_word()
        bt.bt_block_decode_step_window(cfg, cache, 1, to_dev(q), to_dev(kn), to_dev(vn), window, sinks, out, ws, dev_status=st)
        for b in range(B):
            if n[b] < N:
                k[b, :, n[b]], v[b, :, n[b]] = kn[b], vn[b]
                n[b] += 1
        ref, tol = ctx.decode_window(f64(q), f64(k), f64(v), n, window, sinks)
        check(out, ref, tol, f"step {step}")
        assert cache.len[1].tolist() == n and cache.len[0].tolist() == [0] * B
        assert st.item() == bt.BT_DEV_OVERFLOW
        gk = gen.torch_to_bits(cache.k[1])
        for b in range(B):
            assert np.array_equal(gk[b, :, :n[b]], k[b, :, :n[b]]) and (gk[b, :, n[b]:] == NAN).all()


def test_window_as_wide_as_the_cache_is_the_plain_attention(bt):
    B, H, hd, N = 70, 16, 64, 200
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    k, v = (gen.normal_bf16_device(4, i, (1, B, H, N, hd), device="cuda") for i in range(2))
    cache = bt.BlockCache(cfg, k=k, v=v)
    cache.len[0].copy_(torch.arange(B, dtype=torch.int32) * 2 + 1)
    q = gen.normal_bf16_device(4, 3, (B, H, hd), device="cuda")
    a, b, ws = torch.empty_like(q), torch.empty_like(q), bt.alloc_workspace(cfg)
    bt.bt_block_decode_attn(cfg, cache, 0, q, a, ws)
    bt.bt_block_decode_attn_window(cfg, cache, 0, q, N, 0, b, ws)
    assert torch.equal(a, b)


@pytest.mark.parametrize("hd,H,N,window,sinks", [(64, 16, 150, 100, 4), (128, 8, 400, 37, 70), (64, 16, 20, 7, 0)])
def test_window_decode_many_items(bt, hd, H, N, window, sinks):
    """Several items per warp: appended rows, lengths around the window's edges, a third of the sequences checked."""
    B = 130
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    k, v = rnd(21, 1, (B, H, N, hd)), rnd(21, 2, (B, H, N, hd))
    lens = [(b * 13) % (N + 1) for b in range(B)]
    cache = make_cache(bt, cfg, k, v, lens)
    q, kn, vn = (rnd(22, i, (B, H, hd)) for i in range(3))
    out, st, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), status_word(), bt.alloc_workspace(cfg)
    bt.bt_block_decode_step_window(cfg, cache, 0, to_dev(q), to_dev(kn), to_dev(vn), window, sinks, out, ws, dev_status=st)
    n = [min(x + 1, N) for x in lens]
    for b in range(B):
        if lens[b] < N:
            k[b, :, lens[b]], v[b, :, lens[b]] = kn[b], vn[b]
    some = list(range(0, B, 3))
    ref, tol = ctx.decode_window(f64(q[some]), f64(k[some]), f64(v[some]), [n[b] for b in some], window, sinks)
    check(out[some], ref, tol, "many items")
    assert cache.len[0].tolist() == n and st.item() == (bt.BT_DEV_OVERFLOW if N in lens else 0)


# ------------------------------------------------------------------------------------------------ window, prefill

@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 127, 128, 129, 257, 300, 513])
def test_window_prefill(bt, hd, T):
    B, H, stride = 2, 3, T + 5
    q = rnd(5, 1, (B, H, T, hd))
    k, v = rnd(5, 2, (B, H, stride, hd)), rnd(5, 3, (B, H, stride, hd))
    kp, vp = k.copy(), v.copy()
    kp[:, :, T:] = NAN
    vp[:, :, T:] = NAN
    dq, dk, dv = to_dev(q), to_dev(kp), to_dev(vp)
    cfg = bt.make_config(B, H, hd, 4, 1, stride, 1)
    rng = np.random.default_rng(T)
    for window, sinks in [(1, 0), (1, 1), (2, 64), (63, 0), (64, 4), (65, 65), (128, 130), (129, 1), (200, 16), (T, 0), (2 ** 31 - 1, 0),
                          (7, T + 5), (190, 70)]:
        out, st = torch.full_like(dq, 7.0), status_word()
        bt.bt_block_prefill_attn_window(cfg, dq, dk, dv, window, sinks, out, kv_seq_stride=stride, dev_status=st)
        assert st.item() == 0
        some = sorted(set([0, T - 1, T // 2] + [t for t in (62, 63, 64, 65, 126, 127, 128, 129, 191, 192, 255, 256, 257) if t < T] +
                          rng.integers(0, T, 6).tolist()))
        for b, h in ((0, 0), (1, 2)):
            ref, tol = ctx.prefill_window(f64(q[b, h]), f64(k[b, h, :T]), f64(v[b, h, :T]), window, sinks, some)
            check(out[b, h, some], ref, tol, f"T {T} window {window} sinks {sinks} ({b},{h})")
        assert torch.isfinite(out).all()


def test_window_prefill_against_the_plain_prefill_when_all_is_visible(bt):
    B, H, hd, T = 2, 4, 64, 700
    cfg = bt.make_config(B, H, hd, 4, 1, T, 1)
    q, k, v = (gen.normal_bf16_device(6, i, (B, H, T, hd), device="cuda") for i in range(3))
    a, b, c = (torch.empty_like(q) for _ in range(3))
    bt.bt_block_prefill_attn(cfg, q, k, v, a)
    bt.bt_block_prefill_attn_window(cfg, q, k, v, T, 0, b)
    bt.bt_block_prefill_attn_window(cfg, q, k, v, 3, T, c)
    assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("B,H,T,window,sinks", [(40, 16, 300, 70, 4), (3, 2, 2100, 200, 20), (1, 1, 8191, 1000, 3), (330, 16, 130, 5, 1)])
def test_window_prefill_many_items(bt, B, H, T, window, sinks):
    """Several items per CTA, with the host-made table of items and without it: every (sequence, head) must come out."""
    hd = 64
    cfg = bt.make_config(B, H, hd, 4, 1, T, 1)
    q, k, v = (gen.normal_bf16_device(7, i, (B, H, T, hd), device="cuda") for i in range(3))
    out = torch.full_like(q, 7.0)
    bt.bt_block_prefill_attn_window(cfg, q, k, v, window, sinks, out)
    i = torch.arange(T, device="cuda")
    seen = (i[None] <= i[:, None]) & ((i[None] > i[:, None] - window) | (i[None] < sinks))
    for b in sorted({0, 1, B // 2, B - 1} & set(range(B))):
        for h in range(H):
            s = (q[b, h].double() @ k[b, h].double().T / 8.0).masked_fill(~seen, float("-inf"))
            p = torch.softmax(s, -1)
            ref, mass = p @ v[b, h].double(), p @ v[b, h].double().abs()
            # 2^-8 for the weights, 2^-8 for the result, 2^-10 for the scores (|s| < 64 in fp32, 64 products)
            tol = (2.0 ** -8 + 2.0 ** -10) * mass * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs()
            assert ((out[b, h].double() - ref).abs() <= tol).all(), (b, h)
        assert torch.isfinite(out[b]).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("B,T,window,sinks", [(64, 600, 64, 4), (128, 100, 3, 0), (40, 1300, 300, 100), (96, 257, 300, 0)])
def test_window_prefill_odd_tiles_many_items(bt, hd, B, T, window, sinks):
    """An odd number of query tiles and many items per CTA: items of one query tile, whose key/value tiles the other issuing
    warp leaves out, between items of two.  Three calls, the same bits, and within the tolerance of the test above."""
    H = 16
    cfg = bt.make_config(B, H, hd, 4, 1, T, 1)
    q, k, v = (gen.normal_bf16_device(17, i, (B, H, T, hd), device="cuda") for i in range(3))
    outs, st = [], status_word()
    for _ in range(3):
        outs.append(torch.full_like(q, 7.0))
        bt.bt_block_prefill_attn_window(cfg, q, k, v, window, sinks, outs[-1], dev_status=st)
    assert st.item() == 0 and torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    i = torch.arange(T, device="cuda")
    seen = (i[None] <= i[:, None]) & ((i[None] > i[:, None] - window) | (i[None] < sinks))
    for b in range(0, B, 3):
        s = (q[b].double() @ k[b].double().transpose(1, 2) / hd ** 0.5).masked_fill(~seen, float("-inf"))
        p = torch.softmax(s, -1)
        ref, mass = p @ v[b].double(), p @ v[b].double().abs()
        tol = (2.0 ** -8 + 2.0 ** -10) * mass * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs()
        assert ((outs[0][b].double() - ref).abs() <= tol).all(), b
    # all visible: the plain prefill's bits
    whole = torch.empty_like(q)
    bt.bt_block_prefill_attn(cfg, q, k, v, whole)
    bt.bt_block_prefill_attn_window(cfg, q, k, v, T, 0, outs[0])
    assert torch.equal(whole, outs[0])


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_window_prefill_rows_that_are_not_seen_may_hold_anything(bt, hd, bad):
    """A row of V (and one of K) that is not finite reaches the queries that see it and no other."""
    B, H, T, window, sinks = 1, 2, 400, 50, 2
    cfg = bt.make_config(B, H, hd, 4, 1, T, 1)
    q, k, v = (gen.normal_bf16_device(8, i, (B, H, T, hd), device="cuda") for i in range(3))
    clean = torch.empty_like(q)
    bt.bt_block_prefill_attn_window(cfg, q, k, v, window, sinks, clean)
    v[0, 0, 150, 5] = bad
    k[0, 1, 260, 3] = float("nan")
    out = torch.empty_like(q)
    bt.bt_block_prefill_attn_window(cfg, q, k, v, window, sinks, out)
    t = torch.arange(T, device="cuda")
    hit0, hit1 = (t >= 150) & (t < 150 + window), (t >= 260) & (t < 260 + window)
    assert not torch.isfinite(out[0, 0, hit0, 5]).any() and not torch.isfinite(out[0, 1, hit1]).any()
    # a row that is worked out again keeps its weights in fp32: it may differ from the tiled one by their rounding, 2^-8
    # of the weighted |v| (below 4 for these values), and by one rounding of the result
    for h, hit in ((0, hit0), (1, hit1)):
        a, b = out[0, h, ~hit].double(), clean[0, h, ~hit].double()
        assert torch.isfinite(a).all()
        assert ((a - b).abs() <= 2.0 ** -8 * 4 + 2.0 ** -7 * b.abs()).all()
    others = [i for i in range(hd) if i != 5]
    assert torch.isfinite(out[0, 0][:, others]).all()


# ------------------------------------------------------------------------------------------------ shared prefix

def shared_case(bt, B, H, hd, cap, S, N, lens, splits=0, seed=9, layer=0, layers=1):
    cfg = bt.make_config(B, H, hd, 4, 1, N, layers, decode_splits=splits)
    k, v = rnd(seed, 1, (B, H, N, hd)), rnd(seed, 2, (B, H, N, hd))
    pk, pv = rnd(seed, 3, (H, cap, hd)), rnd(seed, 4, (H, cap, hd))
    cache = make_cache(bt, cfg, k, v, lens, layer)
    prefix = make_cache(bt, bt.make_config(1, H, hd, 4, 1, cap, layers), pk[None], pv[None], [S], layer)
    return cfg, cache, prefix, k, v, pk, pv


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("cap,S", [(1, 1), (64, 0), (64, 1), (70, 63), (70, 64), (70, 65), (130, 128), (700, 129), (700, 513), (700, 700)])
def test_shared_prefix(bt, hd, cap, S):
    for B, H, splits in ((1, 1, 0), (3, 2, 0), (130, 3, 0), (5, 4, 3), (9, 16, 1), (40, 128 * 16 // hd, 0)):
        N = 70
        lens = [(b * 37) % (N + 1) for b in range(B)]
        cfg, cache, prefix, k, v, pk, pv = shared_case(bt, B, H, hd, cap, S, N, lens, splits)
        q = rnd(10, B, (B, H, hd))
        out, st, ws = torch.full((B, H, hd), 7.0, dtype=torch.bfloat16, device="cuda"), status_word(), bt.alloc_workspace_shared(cfg, cap)
        ref, tol = ctx.decode_shared(f64(q), f64(pk), f64(pv), S, f64(k), f64(v), lens)
        for _ in range(2):
            bt.bt_block_decode_attn_shared(cfg, prefix, cache, 0, to_dev(q), out, ws, dev_status=st)
            check(out, ref, tol, f"B {B} H {H} cap {cap} S {S}")
        assert st.item() == (bt.BT_DEV_EMPTY if S == 0 else 0)      # sequence 0 has nothing of its own
        assert cache.len[0].tolist() == lens and prefix.len[0].tolist() == [S]


@pytest.mark.parametrize("hd", [64, 128])
def test_shared_prefix_step(bt, hd):
    B, H, cap, S, N = 150, 3, 200, 177, 20
    lens = [b % (N + 1) for b in range(B)]
    cfg, cache, prefix, k, v, pk, pv = shared_case(bt, B, H, hd, cap, S, N, lens, layer=1, layers=2)
    n, ws = list(lens), bt.alloc_workspace_shared(cfg, cap)
    out = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda")
    for step in range(3):
        q, kn, vn = (rnd(11, 3 * step + i, (B, H, hd)) for i in range(3))
        st = status_word()
        bt.bt_block_decode_step_shared(cfg, prefix, cache, 1, to_dev(q), to_dev(kn), to_dev(vn), out, ws, dev_status=st)
        for b in range(B):
            if n[b] < N:
                k[b, :, n[b]], v[b, :, n[b]] = kn[b], vn[b]
                n[b] += 1
        ref, tol = ctx.decode_shared(f64(q), f64(pk), f64(pv), S, f64(k), f64(v), n)
        check(out, ref, tol, f"step {step}")
        assert cache.len[1].tolist() == n and st.item() == bt.BT_DEV_OVERFLOW


def test_shared_prefix_at_size_with_back_to_back_calls(bt):
    """Layers one after the other without a wait between them: the two launches of a call overlap with each other, and
    what a call reads was written by the one before it (its output is the next one's query)."""
    B, H, hd, cap, S, N, L = 256, 16, 64, 2048, 2000, 64, 4
    cfg = bt.make_config(B, H, hd, 4, 1, N, L)
    pcfg = bt.make_config(1, H, hd, 4, 1, cap, L)
    cache = bt.BlockCache(cfg, k=gen.normal_bf16_device(12, 0, (L, B, H, N, hd), device="cuda"), v=gen.normal_bf16_device(12, 1, (L, B, H, N, hd), device="cuda"))
    prefix = bt.BlockCache(pcfg, k=gen.normal_bf16_device(12, 2, (L, 1, H, cap, hd), device="cuda"), v=gen.normal_bf16_device(12, 3, (L, 1, H, cap, hd), device="cuda"))
    cache.len.copy_(torch.randint(0, N + 1, (L, B), generator=torch.Generator().manual_seed(1), dtype=torch.int32))
    prefix.len.fill_(S)
    x = [gen.normal_bf16_device(12, 4, (B, H, hd), device="cuda")] + [torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda") for _ in range(L)]
    ws, st = bt.alloc_workspace_shared(cfg, cap), status_word()
    first = None
    for _ in range(60):
        for l in range(L):
            bt.bt_block_decode_attn_shared(cfg, prefix, cache, l, x[l], x[l + 1], ws, dev_status=st)
        torch.cuda.synchronize()
        assert first is None or torch.equal(first, x[L])      # the same inputs, the same result, every time
        first = x[L].clone()
    assert st.item() == 0
    for l in range(L):
        scores = torch.cat([torch.einsum("bhd,hsd->bhs", x[l].double(), prefix.k[l, 0, :, :S].double()),
                            torch.einsum("bhd,bhnd->bhn", x[l].double(), cache.k[l].double())], -1) / 8.0
        scores[..., S:].masked_fill_((torch.arange(N, device="cuda") >= cache.len[l][:, None])[:, None], float("-inf"))
        p = torch.softmax(scores, -1)
        both = lambda f: torch.einsum("bhs,hsd->bhd", p[..., :S], f(prefix.v[l, 0, :, :S].double())) + \
            torch.einsum("bhn,bhnd->bhd", p[..., S:], f(cache.v[l].double()))
        ref, mass = both(lambda t: t), both(torch.abs)
        tol = (2.0 ** -8 + 2.0 ** -10) * mass * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs()
        assert ((x[l + 1].double() - ref).abs() <= tol).all(), l


@pytest.mark.parametrize("N", [40, 150])   # a warp per (sequence, head), and a CTA
def test_shared_prefix_steps_at_size(bt, N):
    """Many CTAs per sequence read its length and the last one raises it: over a whole cache of steps, lengths, rows and results
    are those of the separate calls."""
    B, H, hd, cap, S = 300, 16, 64, 256, 250
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    fill = lambda i, shape: gen.normal_bf16_device(33, i, shape, device="cuda")   # noqa: E731
    prefix = bt.BlockCache(bt.make_config(1, H, hd, 4, 1, cap, 1), k=fill(0, (1, 1, H, cap, hd)), v=fill(1, (1, 1, H, cap, hd)))
    prefix.len.fill_(S)
    one, two = bt.BlockCache(cfg), bt.BlockCache(cfg)
    start = (torch.arange(B, dtype=torch.int32, device="cuda") % 4)[None]
    one.len.copy_(start)
    two.len.copy_(start)
    ws, st = bt.alloc_workspace_shared(cfg, cap), status_word()
    a, b = (torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for step in range(36):
        q, kn, vn = (fill(10 + 3 * step + i, (B, H, hd)) for i in range(3))
        bt.bt_block_decode_step_shared(cfg, prefix, one, 0, q, kn, vn, a, ws, dev_status=st)
        bt.bt_block_kv_append(cfg, two, 0, kn, vn, n_new=1, dev_status=st)
        bt.bt_block_decode_attn_shared(cfg, prefix, two, 0, q, b, ws, dev_status=st)
        assert torch.equal(one.len, two.len) and torch.equal(one.len, start + step + 1)
        # the appended row joins the sum last instead of in its place: fp32 orders, then at most a step of bf16 (2^-7)
        assert ((a.double() - b.double()).abs() <= 2.0 ** -7 * b.double().abs() + 1e-5).all(), step
    assert torch.equal(one.k, two.k) and torch.equal(one.v, two.v) and st.item() == 0


# ------------------------------------------------------------------------------------------------ summed weights

@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("N,splits", [(261, 1), (264, 1), (261, 4), (264, 7), (2051, 1)])
@pytest.mark.parametrize("mode", ["in_place", "apart", "fresh"])
def test_weights(bt, hd, N, splits, mode):
    lens = LENS if N < 300 else [0, 5, 2050, 2051, 1024, 1025, 33, 2000, 100]
    B, H = len(lens), 3
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    k, v, q = rnd(13, 1, (B, H, N, hd)), rnd(13, 2, (B, H, N, hd)), rnd(13, 3, (B, H, hd))
    cache = make_cache(bt, cfg, k, v, lens)
    w = np.random.default_rng(1).random((B, H, N)).astype(np.float32)
    for b, n in enumerate(lens):
        w[b, :, n:] = np.nan           # never read
    w_in = torch.from_numpy(w).cuda()
    w_out = w_in if mode == "in_place" else torch.full_like(w_in, -3.0)
    out, st, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), status_word(), bt.alloc_workspace_weights(cfg)
    bt.bt_block_decode_attn_weights(cfg, cache, 0, to_dev(q), out, None if mode == "fresh" else w_in, w_out, ws, dev_status=st)
    ref, tol, new, new_tol = ctx.decode_weights(f64(q), f64(k), f64(v), lens, np.zeros_like(w) if mode == "fresh" else w)
    check(out, ref, tol, "out")
    got = w_out.double().cpu().numpy()
    for b, n in enumerate(lens):
        assert (np.abs(got[b, :, :n] - new[b, :, :n]) <= new_tol[b, :, :n]).all(), f"sums of sequence {b}"
        tail = got[b, :, n:]
        assert np.isnan(tail).all() if mode == "in_place" else (tail == -3.0).all()
    assert st.item() == bt.BT_DEV_EMPTY


@pytest.mark.parametrize("N,splits", [(261, 1), (261, 5), (2051, 1)])
def test_weights_step(bt, N, splits):
    """The appended row's sum starts with its own weight; earlier sums grow; a full cache only grows its sums."""
    hd, H = 64, 2
    lens = [0, 1, 31, 32, 130, N - 2, N - 1, N]
    B = len(lens)
    cfg = bt.make_config(B, H, hd, 4, 1, N, 2, decode_splits=splits)
    k, v = rnd(14, 1, (B, H, N, hd)), rnd(14, 2, (B, H, N, hd))
    cache = make_cache(bt, cfg, k, v, lens, layer=1)
    sums = np.random.default_rng(2).random((B, H, N)).astype(np.float32)
    w = torch.zeros((2, B, H, N), device="cuda")
    w[1].copy_(torch.from_numpy(sums))
    n, ws = list(lens), bt.alloc_workspace_weights(cfg)
    out = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda")
    for step in range(3):
        q, kn, vn = (rnd(15, 3 * step + i, (B, H, hd)) for i in range(3))
        st = status_word()
        bt.bt_block_decode_step_weights(cfg, cache, 1, to_dev(q), to_dev(kn), to_dev(vn), out, w, w, ws, dev_status=st)
        fresh = [-1] * B
        for b in range(B):
            if n[b] < N:
                k[b, :, n[b]], v[b, :, n[b]] = kn[b], vn[b]
                fresh[b] = n[b]
                n[b] += 1
        ref, tol, new, new_tol = ctx.decode_weights(f64(q), f64(k), f64(v), n, sums, fresh)
        check(out, ref, tol, f"step {step}")
        got = w[1].cpu().numpy()
        for b in range(B):
            assert (np.abs(got[b, :, :n[b]] - new[b, :, :n[b]]) <= new_tol[b, :, :n[b]]).all(), (step, b)
            assert np.array_equal(got[b, :, n[b]:], sums[b, :, n[b]:])
        sums = got.copy()
        assert st.item() == bt.BT_DEV_OVERFLOW and cache.len[1].tolist() == n and not w[0].any()


# ------------------------------------------------------------------------------------------------ eviction

def sums_for(rng, shape, kind):
    w = (rng.random(shape) ** 8).astype(np.float32)
    if kind == "ties":
        w = np.round(w * 4).astype(np.float32) / 4
    elif kind == "zeros":
        w[:] = 0
    elif kind == "odd":                     # signs, infinities, NaN, both zeros, subnormals
        w = (w - 0.3).astype(np.float32)
        pick = rng.random(shape)
        for lo, x in ((0.0, np.nan), (0.1, np.inf), (0.2, -np.inf), (0.3, 0.0), (0.4, -0.0), (0.5, 1e-42)):
            w[(pick >= lo) & (pick < lo + 0.08)] = x
    return w


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("into", ["in_place", "other"])
@pytest.mark.parametrize("kind", ["plain", "ties", "zeros", "odd"])
@pytest.mark.parametrize("N,n_keep,trigger,sinks,recent", [(261, 100, 0, 4, 20), (261, 1, 0, 0, 0), (261, 1, 0, 0, 1), (261, 64, 200, 30, 34),
                                                           (261, 260, 0, 0, 0), (261, 130, 0, 130, 0), (20, 7, 0, 2, 2), (261, 300, 0, 1, 1)])
def test_evict(bt, hd, into, kind, N, n_keep, trigger, sinks, recent):
    lens = [0, 1, N // 3, n_keep - 1, n_keep, n_keep + 1, N - 1, N, trigger - 1, trigger]
    lens = [min(max(n, 0), N) for n in lens]
    B, H, L, layer = len(lens), 3, 2, 1
    cfg = bt.make_config(B, H, hd, 4, 1, N, L)
    k, v = rnd(16, 1, (B, H, N, hd)), rnd(16, 2, (B, H, N, hd))
    w = sums_for(np.random.default_rng(3), (B, H, N), kind)
    cache = bt.BlockCache(cfg)
    cache.k[layer].copy_(to_dev(k))
    cache.v[layer].copy_(to_dev(v))
    cache.len[layer].copy_(torch.tensor(lens, dtype=torch.int32))
    sums = torch.zeros((L, B, H, N), device="cuda")
    sums[layer].copy_(torch.from_numpy(w))
    st, ws = status_word(), bt.alloc_workspace(cfg)
    if into == "other":
        cap = max(n_keep, max(trigger - 1, 0), 1)
        dst, dsums = bt.BlockCache(bt.make_config(B, H, hd, 4, 1, cap, L)), torch.full((L, B, H, cap), -5.0, device="cuda")
        dst.k.fill_(9.0)
        dst.v.fill_(9.0)
        dst.len.fill_(77)
        kept = bt.bt_block_kv_evict(cfg, cache, sums, layer, n_keep, sinks, recent, n_trigger=trigger, dst=dst, dst_weights=dsums, dev_status=st)
        assert torch.equal(cache.len[layer].cpu(), torch.tensor(lens, dtype=torch.int32))
        assert np.array_equal(gen.torch_to_bits(cache.k[layer]), k) and np.array_equal(gen.torch_to_bits(cache.v[layer]), v)
        assert np.array_equal(sums[layer].cpu().numpy().view(np.uint32), w.view(np.uint32))
        assert (dst.len[0] == 77).all() and (dst.k[0] == 9.0).all() and (dsums[0] == -5.0).all()
    else:
        dst, dsums, cap = cache, sums, N
        kept = bt.bt_block_kv_evict(cfg, cache, sums, layer, n_keep, sinks, recent, ws, n_trigger=trigger, dev_status=st)
        assert not cache.len[0].any() and not cache.k[0].any() and not sums[0].any()
        assert not ws.view(torch.int32)[-(B * H + B):].any()
    gk, gv, gw, got = gen.torch_to_bits(dst.k[layer]), gen.torch_to_bits(dst.v[layer]), dsums[layer].cpu().numpy(), kept.cpu().numpy()
    nine = gen.torch_to_bits(torch.tensor([9.0], dtype=torch.bfloat16))[0]
    bits = lambda x: np.ascontiguousarray(x).view(np.uint32)   # NaN compares by its bits
    for b, n in enumerate(lens):
        cut = n > n_keep and n >= trigger
        m = n_keep if cut else n
        assert dst.len[layer, b].item() == m, b
        for h in range(H):
            rows = ctx.evicted(w[b, h], n, n_keep, sinks, recent) if cut else list(range(n))
            assert got[b, h].tolist() == (rows if cut else [-1] * n_keep), (b, h)
            assert np.array_equal(gk[b, h, :m], k[b, h, rows]) and np.array_equal(gv[b, h, :m], v[b, h, rows])
            assert np.array_equal(bits(gw[b, h, :m]), bits(w[b, h, rows]))
            if into == "other":
                assert (gk[b, h, m:] == nine).all() and (gv[b, h, m:] == nine).all() and (gw[b, h, m:] == -5.0).all()
            else:
                assert np.array_equal(gk[b, h, m:], k[b, h, m:]) and np.array_equal(gv[b, h, m:], v[b, h, m:])
                assert np.array_equal(bits(gw[b, h, m:]), bits(w[b, h, m:]))
    assert st.item() == 0


@pytest.mark.parametrize("into", ["in_place", "other"])
@pytest.mark.parametrize("B,H,N,n_keep", [(2, 2, 9001, 4500), (1, 1, 5000, 4900), (700, 16, 96, 40), (1, 2, 40001, 17000), (1, 1, 16385, 16384),
                                          (40, 16, 3000, 1100), (5, 4, 900, 333)])
def test_evict_long_and_many(bt, into, B, H, N, n_keep):
    hd, sinks, recent = 64, 5, 20
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    k, v = (gen.normal_bf16_device(17, i, (1, B, H, N, hd), device="cuda") for i in range(2))
    w = torch.rand((1, B, H, N), generator=torch.Generator("cuda").manual_seed(1), device="cuda").pow_(6)
    w[w < 0.01] = 0.01                                      # a long run of equal sums around the threshold
    cache = bt.BlockCache(cfg, k=k.clone(), v=v.clone())
    lens = torch.tensor([N - b % 7 for b in range(B)], dtype=torch.int32, device="cuda")
    cache.len[0].copy_(lens)
    sums = w.clone()
    j = torch.arange(N, device="cuda")
    n = lens.long()[:, None, None]
    rank = torch.where((j < sinks) | (j >= n - recent), float("inf"), w[0]).masked_fill(j >= n, float("-inf"))
    rows = rank.sort(dim=-1, descending=True, stable=True).indices[..., :n_keep].sort(-1).values
    at = rows[..., None].expand(-1, -1, -1, hd)
    want_k, want_v, want_w = k[0].gather(2, at), v[0].gather(2, at), w[0].gather(2, rows)
    ws = bt.alloc_workspace(cfg)
    for _ in range(40 if B * H > 1000 else 3):   # many CTAs of a sequence read its length while the first ones are done with it
        cache.k.copy_(k)
        cache.v.copy_(v)
        cache.len[0].copy_(lens)
        sums.copy_(w)
        if into == "other":
            dst, dsums = bt.BlockCache(bt.make_config(B, H, hd, 4, 1, n_keep, 1)), torch.zeros((1, B, H, n_keep), device="cuda")
            kept = bt.bt_block_kv_evict(cfg, cache, sums, 0, n_keep, sinks, recent, dst=dst, dst_weights=dsums)
        else:
            dst, dsums = cache, sums
            kept = bt.bt_block_kv_evict(cfg, cache, sums, 0, n_keep, sinks, recent, ws)
        assert (dst.len == n_keep).all() and torch.equal(kept.long(), rows)
        assert torch.equal(dst.k[0, :, :, :n_keep], want_k) and torch.equal(dst.v[0, :, :, :n_keep], want_v)
        assert torch.equal(dsums[0, :, :, :n_keep], want_w)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("N,n_keep,sinks,recent", [(3000, 1100, 4, 300), (3000, 700, 0, 700), (9000, 2500, 100, 1777), (6000, 5999, 1, 256)])
def test_evict_into_another_cache_with_many_recent_rows(bt, hd, N, n_keep, sinks, recent):
    """Few pairs: the last rows move while the others are selected.  Cut and uncut sequences side by side, second layer."""
    B, H = 4, 2
    cfg = bt.make_config(B, H, hd, 4, 1, N, 2)
    k, v = (gen.normal_bf16_device(50, i, (2, B, H, N, hd), device="cuda") for i in range(2))
    w = torch.rand((2, B, H, N), generator=torch.Generator("cuda").manual_seed(5), device="cuda").pow_(4)
    lens = torch.tensor([[0] * B, [N, n_keep, n_keep + 1, N // 2]], dtype=torch.int32, device="cuda")
    cache = bt.BlockCache(cfg, k=k, v=v, length=lens)
    dst, dw = bt.BlockCache(bt.make_config(B, H, hd, 4, 1, n_keep, 2)), torch.full((2, B, H, n_keep), -1.0, device="cuda")
    kept = bt.bt_block_kv_evict(cfg, cache, w, 1, n_keep, sinks, recent, dst=dst, dst_weights=dw)
    j, n = torch.arange(N, device="cuda"), lens[1].long()[:, None, None]
    rank = torch.where((j < sinks) | (j >= n - recent), float("inf"), w[1]).masked_fill(j >= n, float("-inf"))
    rows = rank.sort(dim=-1, descending=True, stable=True).indices[..., :n_keep].sort(-1).values
    cut = (n > n_keep).expand(-1, H, 1)
    assert torch.equal(kept.long(), torch.where(cut, rows, -1))
    assert torch.equal(dst.len[1], lens[1].clamp(max=n_keep)) and not dst.len[0].any() and not dst.k[0].any()
    for b in range(B):
        m = min(int(lens[1, b]), n_keep)
        for h in range(H):
            r = rows[b, h] if cut[b, h, 0] else torch.arange(m, device="cuda")
            assert torch.equal(dst.k[1, b, h, :m], k[1, b, h, r]) and torch.equal(dst.v[1, b, h, :m], v[1, b, h, r])
            assert torch.equal(dw[1, b, h, :m], w[1, b, h, r]) and not dst.k[1, b, h, m:].any() and (dw[1, b, h, m:] == -1).all()


# ------------------------------------------------------------------------------------------------ together

def test_generation_with_a_bounded_cache(bt):
    """A prompt prefilled under a window and cached, then steps that sum weights and an eviction whenever the cache is full
    - every call captured into one graph per step kind, replayed on a stream that is not the default one, as a serving
    loop would.  A float64 model of the same loop follows it, fed with the sums the GPU chose by."""
    B, H, hd, N, T, n_keep, sinks, recent, window = 3, 2, 64, 24, 16, 14, 2, 4, 6
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    cache, ws = bt.BlockCache(cfg), bt.alloc_workspace_weights(cfg)
    sums = torch.zeros((1, B, H, N), device="cuda")
    q, k, v = (rnd(18, i, (B, H, T, hd)) for i in range(3))
    out = torch.empty((B, H, T, hd), dtype=torch.bfloat16, device="cuda")
    bt.bt_block_prefill_attn_window(cfg, to_dev(q), to_dev(k), to_dev(v), window, sinks, out)
    bt.bt_block_kv_append(cfg, cache, 0, to_dev(k), to_dev(v))
    for b in range(B):
        for h in range(H):
            check(out[b, h], *ctx.prefill_window(f64(q[b, h]), f64(k[b, h]), f64(v[b, h]), window, sinks), what="prompt")
    K, V = np.zeros((B, H, N, hd), np.uint16), np.zeros((B, H, N, hd), np.uint16)
    K[:, :, :T], V[:, :, :T] = k, v
    n = T
    side = torch.cuda.Stream()
    x, kn, vn, o = (torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda") for _ in range(4))
    kept = torch.empty((B, H, n_keep), dtype=torch.int32, device="cuda")
    st = status_word()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            bt.bt_block_kv_evict(cfg, cache, sums, 0, n_keep, sinks, recent, ws, n_trigger=N, kept=kept, dev_status=st, stream=side)
            bt.bt_block_decode_step_weights(cfg, cache, 0, x, kn, vn, o, sums, sums, ws, dev_status=st, stream=side)
        evictions = 0
        for step in range(40):
            before = sums[0].cpu().numpy()
            a, b_, c = (rnd(19, 3 * step + i, (B, H, hd)) for i in range(3))
            x.copy_(to_dev(a))
            kn.copy_(to_dev(b_))
            vn.copy_(to_dev(c))
            graph.replay()
            side.synchronize()
            model = before.copy()
            if n == N:
                evictions += 1
                for b in range(B):
                    for h in range(H):
                        rows = ctx.evicted(before[b, h], n, n_keep, sinks, recent)
                        assert kept[b, h].tolist() == rows
                        K[b, h, :n_keep], V[b, h, :n_keep], model[b, h, :n_keep] = K[b, h, rows], V[b, h, rows], before[b, h, rows]
                n = n_keep
            else:
                assert (kept == -1).all()
            K[:, :, n], V[:, :, n] = b_, c
            n += 1
            ref, tol, new, new_tol = ctx.decode_weights(f64(a), f64(K), f64(V), [n] * B, model, [n - 1] * B)
            check(o, ref, tol, f"step {step}")
            got = sums[0].double().cpu().numpy()
            assert (np.abs(got - new)[:, :, :n] <= new_tol[:, :, :n]).all()
            assert (cache.len == n).all()
        assert evictions >= 3 and st.item() == 0


@pytest.mark.parametrize("B,H,N,n_keep", [(2, 2, 2000, 900), (3, 1, 9000, 1500), (60, 16, 300, 100)])
def test_evict_in_place_in_a_graph(bt, B, H, N, n_keep):
    """Captured before it ever ran on these sizes, replayed on rows that change between replays (clusters of several CTAs in the
    first two cases), equal to a stable selection each time."""
    hd, sinks, recent = 64, 3, 11
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    cache, sums, ws = bt.BlockCache(cfg), torch.zeros((1, B, H, N), device="cuda"), bt.alloc_workspace(cfg)
    kept = torch.empty((B, H, n_keep), dtype=torch.int32, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        bt.bt_block_kv_evict(cfg, cache, sums, 0, n_keep, sinks, recent, ws, kept=kept, stream=side)
    for turn in range(4):
        k, v = gen.normal_bf16_device(40 + turn, 0, (1, B, H, N, hd), device="cuda"), gen.normal_bf16_device(40 + turn, 1, (1, B, H, N, hd), device="cuda")
        w = torch.rand((1, B, H, N), generator=torch.Generator("cuda").manual_seed(turn), device="cuda").pow_(4)
        cache.k.copy_(k)
        cache.v.copy_(v)
        sums.copy_(w)
        n = torch.full((1, B), N - turn, dtype=torch.int32, device="cuda")
        n[0, 0] = n_keep if turn == 2 else N
        cache.len.copy_(n)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        j, m = torch.arange(N, device="cuda"), n[0].long()[:, None, None]
        rank = torch.where((j < sinks) | (j >= m - recent), float("inf"), w[0]).masked_fill(j >= m, float("-inf"))
        rows = rank.sort(dim=-1, descending=True, stable=True).indices[..., :n_keep].sort(-1).values
        cut = (m > n_keep).expand(-1, H, 1)
        assert torch.equal(kept.long(), torch.where(cut, rows, -1)) and (cache.len == n_keep).all()
        rows = torch.where(cut, rows, torch.arange(n_keep, device="cuda"))
        at = rows[..., None].expand(-1, -1, -1, hd)
        assert torch.equal(cache.k[0, :, :, :n_keep], k[0].gather(2, at)) and torch.equal(cache.v[0, :, :, :n_keep], v[0].gather(2, at))
        assert torch.equal(cache.k[0, :, :, n_keep:], k[0, :, :, n_keep:]) and torch.equal(sums[0, :, :, :n_keep], w[0].gather(2, rows))


def test_two_graphs_with_their_own_workspaces_on_two_streams(bt):
    """The same calls captured twice, each with its own workspace and outputs, replayed at the same time."""
    B, H, hd, N, cap, S = 6, 4, 128, 300, 500, 450
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    assert bt.bt_decode_splits(cfg) > 1
    lens = [0, 300, 17, 150, 299, 64]
    _, cache, prefix, k, v, pk, pv = shared_case(bt, B, H, hd, cap, S, N, lens)
    q = to_dev(rnd(20, 1, (B, H, hd)))
    runs = []
    torch.cuda.synchronize()
    for _ in range(2):
        s = torch.cuda.Stream()
        r = dict(stream=s, ws=bt.alloc_workspace_weights(cfg), ws2=bt.alloc_workspace_shared(cfg, cap), sums=torch.zeros((1, B, H, N), device="cuda"),
                 outs=[torch.empty_like(q) for _ in range(3)], graph=torch.cuda.CUDAGraph())
        torch.cuda.synchronize()
        with torch.cuda.graph(r["graph"], stream=s):
            bt.bt_block_decode_attn_window(cfg, cache, 0, q, 50, 3, r["outs"][0], r["ws"], stream=s)
            bt.bt_block_decode_attn_shared(cfg, prefix, cache, 0, q, r["outs"][1], r["ws2"], stream=s)
            bt.bt_block_decode_attn_weights(cfg, cache, 0, q, r["outs"][2], r["sums"], r["sums"], r["ws"], stream=s)
        runs.append(r)
    torch.cuda.synchronize()
    for _ in range(20):
        for r in runs:
            with torch.cuda.stream(r["stream"]):
                r["graph"].replay()
    torch.cuda.synchronize()
    Q, K, V = to_f64(q).reshape(B, H, hd), f64(k), f64(v)
    refs = [ctx.decode_window(Q, K, V, lens, 50, 3), ctx.decode_shared(Q, f64(pk), f64(pv), S, K, V, lens)]
    o, tol, new, new_tol = ctx.decode_weights(Q, K, V, lens, np.zeros((B, H, N)))
    refs.append((o, tol))
    for r in runs:
        for got, (ref, t) in zip(r["outs"], refs):
            check(got, ref, t, "replayed")
        sums = r["sums"][0].double().cpu().numpy()
        for b, n in enumerate(lens):
            assert (np.abs(sums[b, :, :n] - 20 * new[b, :, :n]) <= 20 * new_tol[b, :, :n] + 20 * 20 * 2.0 ** -23 * new[b, :, :n]).all()
            assert not sums[b, :, n:].any()


# ------------------------------------------------------------------------------------------------ nothing else is touched

class Guarded:
    """A device tensor between two guard regions of known bytes."""

    SIDE, PATTERN = 4096, 0x5A

    def __init__(self, shape, dtype, fill=None):
        self.n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        self.raw = torch.full((2 * self.SIDE + self.n + (-self.n) % 256,), self.PATTERN, dtype=torch.uint8, device="cuda")
        self.t = self.raw[self.SIDE:self.SIDE + self.n].view(dtype).view(shape)
        if fill is not None:
            self.t.copy_(fill)
        self.before = self.raw.clone()

    def guards(self):
        return bool((self.raw[:self.SIDE] == self.PATTERN).all() and (self.raw[self.SIDE + self.n:] == self.PATTERN).all())

    def unchanged(self):
        return torch.equal(self.raw, self.before)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("B,H,N,splits", [(37, 5, 97, 0), (3, 2, 700, 0), (5, 3, 130, 4), (90, 8, 33, 1)])
def test_contexts_touch_nothing_outside_their_rows(bt, hd, B, H, N, splits):
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
    lens = torch.tensor([(b * 29) % (N + 1) for b in range(B)], dtype=i32)
    lens[0], lens[-1] = N, 0
    data = lambda seed, shape: gen.normal_bf16_device(30, seed, shape, device="cuda")   # noqa: E731
    q, kn, vn, out = (Guarded((B, H, hd), bf, data(i, (B, H, hd))) for i in range(4))
    cap, S = 90, 77
    pk, pv = Guarded((1, 1, H, cap, hd), bf, data(5, (1, 1, H, cap, hd))), Guarded((1, 1, H, cap, hd), bf, data(6, (1, 1, H, cap, hd)))
    plen = Guarded((1, 1), i32, torch.tensor([[S]], dtype=i32))
    prefix = bt.BlockCache(bt.make_config(1, H, hd, 4, 1, cap, 1), k=pk.t, v=pv.t, length=plen.t)

    def fresh():
        k, v = Guarded((1, B, H, N, hd), bf, data(7, (1, B, H, N, hd))), Guarded((1, B, H, N, hd), bf, data(8, (1, B, H, N, hd)))
        n = Guarded((1, B), i32, lens[None])
        return k, v, n, bt.BlockCache(cfg, k=k.t, v=v.t, length=n.t)

    def workspace(nbytes):
        ws = Guarded((max(nbytes, 4) // 4,), f32)
        bt.bt_workspace_init(cfg, ws.t)
        return ws

    at = torch.arange(N, device="cuda")
    for call in ("window", "shared", "weights"):
        k, v, n, cache = fresh()
        sums = Guarded((1, B, H, N), f32, torch.ones(1, B, H, N))
        ws = workspace({"window": bt.bt_workspace_bytes(cfg), "shared": bt.bt_workspace_bytes_shared(cfg, cap),
                        "weights": bt.bt_workspace_bytes_weights(cfg)}[call])
        k0, v0 = k.t.clone(), v.t.clone()
        if call == "window":
            bt.bt_block_decode_step_window(cfg, cache, 0, q.t, kn.t, vn.t, 20, 3, out.t, ws.t)
        elif call == "shared":
            bt.bt_block_decode_step_shared(cfg, prefix, cache, 0, q.t, kn.t, vn.t, out.t, ws.t)
        else:
            bt.bt_block_decode_step_weights(cfg, cache, 0, q.t, kn.t, vn.t, out.t, sums.t, sums.t, ws.t)
        torch.cuda.synchronize()
        assert all(g.guards() for g in (k, v, n, ws, out, sums)), call
        assert all(g.unchanged() for g in (q, kn, vn, pk, pv, plen)), call
        new = (at[None] == lens.cuda()[:, None])[:, None, :, None]            # the appended rows
        assert torch.equal(k.t[0], torch.where(new, kn.t[:, :, None], k0[0])) and torch.equal(v.t[0], torch.where(new, vn.t[:, :, None], v0[0]))
        assert torch.equal(n.t[0].cpu(), (lens + 1).clamp(max=N))
        past = (at[None] >= n.t[0][:, None])[:, None].expand(-1, H, -1)
        assert (sums.t[0][past] == 1).all()
        assert not ws.t.view(i32)[:bt.bt_workspace_bytes(cfg) // 4][-(B * H + B):].any()   # the counters are back at zero
    keep = max(1, N // 3)
    for into in (False, True):
        k, v, n, cache = fresh()
        sums = Guarded((1, B, H, N), f32, torch.rand((1, B, H, N), device="cuda", generator=torch.Generator("cuda").manual_seed(3)))
        kept, ws = Guarded((B, H, keep), i32), workspace(bt.bt_workspace_bytes(cfg))
        dk, dv, dw, dn = Guarded((1, B, H, keep, hd), bf), Guarded((1, B, H, keep, hd), bf), Guarded((1, B, H, keep), f32), Guarded((1, B), i32)
        if into:
            dst = bt.BlockCache(bt.make_config(B, H, hd, 4, 1, keep, 1), k=dk.t, v=dv.t, length=dn.t)
            bt.bt_block_kv_evict(cfg, cache, sums.t, 0, keep, 0, keep // 2, dst=dst, dst_weights=dw.t, kept=kept.t)
        else:
            bt.bt_block_kv_evict(cfg, cache, sums.t, 0, keep, 0, keep // 2, ws.t, kept=kept.t)
        torch.cuda.synchronize()
        assert all(g.guards() for g in (k, v, n, sums, kept, ws, dk, dv, dw, dn))
        assert all(g.unchanged() for g in ((k, v, n, sums) if into else (dk, dv, dw, dn)))
        assert torch.equal((dn if into else n).t[0].cpu(), lens.clamp(max=keep))
    T = min(N, 300)
    x, y, z, o = (Guarded((2, H, T, hd), bf, data(10 + i, (2, H, T, hd))) for i in range(4))
    bt.bt_block_prefill_attn_window(cfg_of(bt, 2, H, hd, T), x.t, y.t, z.t, 17, 2, o.t)
    torch.cuda.synchronize()
    assert o.guards() and all(g.unchanged() for g in (x, y, z)) and torch.isfinite(o.t).all()


def cfg_of(bt, B, H, hd, N):
    return bt.make_config(B, H, hd, 4, 1, N, 1)
