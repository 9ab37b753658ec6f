"""GPU parity of the low-bit operators (4-bit block cache, attention over it, 8-bit projections) against their float64
definitions.  Codes, steps, lengths and everything that only moves are compared bit for bit; bounds on rounding come with the
definitions."""
import numpy as np
import pytest
import torch

from oracle import lowbit as lb
from workloads import gen

from util import local_kv_split, status_word, to_dev, to_f64

pytestmark = pytest.mark.gpu

FILL = 0xFF   # a cache full of these holds NaN steps


@pytest.fixture(scope="module")
def bt():
    import paper_2406_02657_b200 as bt
    assert torch.cuda.is_available()
    return bt


def rnd(seed, tid, shape):
    return gen.normal_bf16_bits(seed, tid, shape)


def f64(bits):
    return gen.bf16_bits_to_f32(bits).astype(np.float64)


def bits(x):
    return gen.f32_to_bf16_bits(np.asarray(x, np.float32))


def check(got, ref, tol, what):
    g = to_f64(got).reshape(ref.shape)
    assert np.isfinite(g).all(), f"{what}: non-finite output"
    over = np.abs(g - ref) - tol
    assert (over <= 0).all(), f"{what}: {over.max():.3e} beyond the bound at {np.unravel_index(over.argmax(), over.shape)}"


def empty_cache(bt, cfg):
    cache = bt.BlockCacheKV4(cfg)
    cache.kv.fill_(FILL)
    return cache


def tiles_of(cfg):
    return np.full((cfg.batch, cfg.heads, -(-cfg.max_blocks // 16), cfg.head_dim // 64, lb.TILE_BYTES), FILL, np.uint8)


def filled(bt, cfg, k, v, lens, layer=0):
    """A cache of rows k, v [B,H,N,hd] (bits) of which lens[b] are valid, the others NaN; written by the definition."""
    tiles = tiles_of(cfg)
    K, V = f64(k), f64(v)
    for b, n in enumerate(lens):
        for h in range(cfg.heads):
            lb.write_tiles(tiles[b, h], 0, K[b, h, :n], V[b, h, :n])
    cache = empty_cache(bt, cfg)
    cache.kv[layer].copy_(torch.from_numpy(tiles))
    cache.len[layer].copy_(torch.tensor(lens, dtype=torch.int32))
    return cache


def awkward(rows):
    """Rows with what a quantiser can get wrong: zeros, exact halves, one value alone, tiny, huge, infinite and NaN ones."""
    x = f64(rows).copy()
    flat = x.reshape(-1, x.shape[-1])
    n = flat.shape[0]
    flat[0 % n, :32] = 0.0
    flat[1 % n, :32] = np.arange(32) / 2.0 * 7 / 7.5            # many halves once the largest is 7 steps
    flat[1 % n, 31] = 7.0
    flat[2 % n, :32] = 0.0
    flat[2 % n, 5] = -3.0
    flat[3 % n, :32] *= 2.0 ** -122                              # steps around the least one
    flat[4 % n, :32] *= 2.0 ** -130
    flat[5 % n, :32] = 3.3e38 * np.sign(flat[5 % n, :32])
    flat[6 % n, 3] = np.inf
    flat[7 % n, 40] = np.nan
    flat[8 % n, 63] = -np.inf
    flat[9 % n, 32:64] = -0.0
    flat[10 % n, :32] = np.linspace(-7, 7, 32).round() / 2       # halves of a step of one half
    return bits(x)


# ------------------------------------------------------------------------------------------------ writing and reading rows

@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_new,reset", [(1, False), (1, True), (3, False), (15, True), (16, False), (17, True), (40, False), (70, True)])
def test_append_writes_codes_and_steps(bt, hd, n_new, reset):
    lens = [0, 1, 15, 16, 17, 31, 40, 79, 80]
    B, H, N = len(lens), 3, 80
    cfg = bt.make_config(B, H, hd, 4, 1, N, 2)
    cache, st = empty_cache(bt, cfg), status_word()
    cache.len[1].copy_(torch.tensor(lens, dtype=torch.int32))
    k, v = awkward(rnd(1, n_new, (B, H, n_new, hd))), awkward(rnd(2, n_new, (B, H, n_new, hd)))
    bt.bt_block_kv4_append(cfg, cache, 1, to_dev(k), to_dev(v), reset_first=reset, dev_status=st)
    tiles, after = tiles_of(cfg), []
    for b, n in enumerate(lens):
        start = 0 if reset else n
        ok = start + n_new <= N
        after.append(start + n_new if ok else n)
        for h in range(H if ok else 0):
            lb.write_tiles(tiles[b, h], start, f64(k[b, h]), f64(v[b, h]))
    assert np.array_equal(cache.kv[1].cpu().numpy(), tiles)
    assert cache.len[1].tolist() == after and cache.len[0].tolist() == [0] * B and (cache.kv[0] == FILL).all()
    assert st.item() == (0 if reset else bt.BT_DEV_OVERFLOW)


@pytest.mark.parametrize("hd,B,H,n", [(64, 300, 16, 2), (128, 2, 5, 700), (64, 1, 1, 5000)])
def test_append_many_rows(bt, hd, B, H, n):
    cfg = bt.make_config(B, H, hd, 4, 1, n + 37, 1)
    cache = empty_cache(bt, cfg)
    k, v = rnd(3, 0, (B, H, n, hd)), rnd(3, 1, (B, H, n, hd))
    bt.bt_block_kv4_append(cfg, cache, 0, to_dev(k), to_dev(v), reset_first=True)
    bt.bt_block_kv4_append(cfg, cache, 0, to_dev(k), to_dev(v), n_new=min(n, 21))
    assert (cache.len == n + min(n, 21)).all()
    tiles = cache.kv[0].cpu().numpy()
    rng = np.random.default_rng(n)
    for _ in range(6):
        b, h = rng.integers(B), rng.integers(H)
        ref = tiles_of(bt.make_config(1, 1, hd, 4, 1, n + 37, 1))[0, 0]
        lb.write_tiles(ref, 0, f64(k[b, h]), f64(v[b, h]))
        # the second call's rows are the first n_new of each slab of n
        packed_k, packed_v = (x.reshape(-1)[: B * H * n * hd].reshape(B * H, n, hd)[b * H + h, :min(n, 21)] for x in (k, v))
        lb.write_tiles(ref, n, f64(packed_k), f64(packed_v))
        assert np.array_equal(tiles[b, h], ref)


def test_append_takes_rows_of_a_bf16_cache(bt):
    """src_stride: the first rows of every slab of a bf16 block cache."""
    B, H, hd, N, n = 3, 4, 128, 50, 33
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    source = bt.BlockCache(cfg, k=to_dev(rnd(4, 0, (1, B, H, N, hd))), v=to_dev(rnd(4, 1, (1, B, H, N, hd))))
    a, b = empty_cache(bt, cfg), empty_cache(bt, cfg)
    bt.bt_block_kv4_append(cfg, a, 0, source.k[0], source.v[0], n_new=n, src_stride=N, reset_first=True)
    bt.bt_block_kv4_append(cfg, b, 0, source.k[0, :, :, :n].contiguous(), source.v[0, :, :, :n].contiguous())
    assert torch.equal(a.kv, b.kv) and torch.equal(a.len, b.len)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("first,n_rows,extra", [(0, 80, 0), (0, 1, 0), (79, 1, 3), (16, 16, 0), (5, 40, 7), (33, 47, 0)])
def test_read_gives_the_values_held(bt, hd, first, n_rows, extra):
    lens = [0, 1, 6, 17, 33, 79, 80]
    B, H, N = len(lens), 2, 80
    cfg = bt.make_config(B, H, hd, 4, 1, N, 2)
    k, v = awkward(rnd(5, 0, (B, H, N, hd))), awkward(rnd(5, 1, (B, H, N, hd)))
    cache = filled(bt, cfg, k, v, lens, layer=1)
    ko, vo = (torch.full((B, H, n_rows + extra, hd), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bt.bt_block_kv4_read(cfg, cache, 1, ko, vo, first=first, n_rows=n_rows)
    for got, src in ((to_f64(ko), k), (to_f64(vo), v)):
        want = np.full((B, H, n_rows + extra, hd), 7.0)
        for b, n in enumerate(lens):
            m = max(0, min(n, first + n_rows) - first)
            want[b, :, :m] = lb.to_bf16(lb.held(f64(src[b, :, first:first + m])))
        assert np.array_equal(got, want, equal_nan=True)


# ------------------------------------------------------------------------------------------------ attention

LENS = [0, 1, 15, 16, 17, 63, 64, 65, 128, 200, 258, 261]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [0, 1, 2, 3, 7, 64])
@pytest.mark.parametrize("scale", [0.0, 0.7])
def test_decode(bt, hd, splits, scale):
    B, H, N = len(LENS), 3, 261
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits, softmax_scale=scale)
    k, v, q = rnd(11, 1, (B, H, N, hd)), rnd(11, 2, (B, H, N, hd)), rnd(11, 3, (B, H, hd))
    cache = filled(bt, cfg, k, v, LENS)
    out, st, ws = torch.full((B, H, hd), 7.0, dtype=torch.bfloat16, device="cuda"), status_word(), bt.alloc_workspace_kv4(cfg)
    qs = f64(q) * (scale * np.sqrt(hd) if scale else 1.0)
    ref, tol = lb.decode(qs, lb.held(f64(k)), lb.held(f64(v)), LENS)
    for _ in range(2):
        bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(q), out, ws, dev_status=st)
        check(out, ref, tol, f"splits {splits}")
    assert st.item() == bt.BT_DEV_EMPTY and (out[0] == 0).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [0, 1, 4])
def test_step_is_append_and_attention(bt, hd, splits):
    """Steps over lengths that cross tiles and chunks, a full cache among them, against the two calls and the definition."""
    B, H, N = len(LENS), 2, 261
    cfg = bt.make_config(B, H, hd, 4, 1, N, 2, decode_splits=splits)
    k, v = rnd(12, 1, (B, H, N, hd)), rnd(12, 2, (B, H, N, hd))
    one, two = (filled(bt, cfg, k, v, LENS, layer=1) for _ in range(2))
    n, ws = list(LENS), bt.alloc_workspace_kv4(cfg)
    a, b = (torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for step in range(3):
        q, kn, vn = (rnd(13, 3 * step + i, (B, H, 1, hd)) for i in range(3))
        st = status_word()
        bt.bt_block_decode_step_kv4(cfg, one, 1, to_dev(q), to_dev(kn), to_dev(vn), a, ws, dev_status=st)
        bt.bt_block_kv4_append(cfg, two, 1, to_dev(kn), to_dev(vn))
        bt.bt_block_decode_attn_kv4(cfg, two, 1, to_dev(q), b, ws)
        assert torch.equal(a, b) and torch.equal(one.kv, two.kv) and torch.equal(one.len, two.len)
        for i in range(B):
            if n[i] < N:
                k[i, :, n[i]], v[i, :, n[i]] = kn[i, :, 0], vn[i, :, 0]
                n[i] += 1
        ref, tol = lb.decode(f64(q[:, :, 0]), lb.held(f64(k)), lb.held(f64(v)), n)
        check(a, ref, tol, f"step {step}")
        assert one.len[1].tolist() == n and one.len[0].tolist() == [0] * B and st.item() == bt.BT_DEV_OVERFLOW
    assert not ws.view(torch.int32)[:0].any() and (one.kv[0] == FILL).all()


@pytest.mark.parametrize("hd,B,H,N", [(64, 300, 16, 70), (128, 150, 16, 200), (64, 3, 2, 5000), (128, 1, 1, 9000), (128, 2, 7, 1003)])
def test_decode_many_items_and_long_rows(bt, hd, B, H, N):
    """Several items per warp with lengths all over the range, and ranges that are split; a part of the sequences checked."""
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    k, v, q = rnd(14, 1, (B, H, N, hd)), rnd(14, 2, (B, H, N, hd)), rnd(14, 3, (B, H, hd))
    cache = empty_cache(bt, cfg)
    bt.bt_block_kv4_append(cfg, cache, 0, to_dev(k), to_dev(v))
    lens = [N - (b * 13) % (N + 1) for b in range(B)]
    cache.len[0].copy_(torch.tensor(lens, dtype=torch.int32))
    out, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), bt.alloc_workspace_kv4(cfg)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(q), out, ws)
    some = list(range(0, B, max(1, B // 12)))
    ref, tol = lb.decode(f64(q[some]), lb.held(f64(k[some])), lb.held(f64(v[some])), [lens[b] for b in some])
    check(out[some], ref, tol, "many items")
    again = torch.empty_like(out)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(q), again, ws)
    assert torch.equal(out, again)


@pytest.mark.parametrize("hd", [64, 128])
def test_large_scores_keep_their_precision(bt, hd):
    """Queries and keys with one large mean: the sums cancel, what is left decides the weights."""
    B, H, N = 2, 3, 150
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    k, v = bits(f64(rnd(15, 1, (B, H, N, hd))) + 3.0), rnd(15, 2, (B, H, N, hd))
    q = bits(f64(rnd(15, 3, (B, H, hd))) + 8.0 * np.where(np.arange(hd) % 2, 1.0, -1.0))
    cache = filled(bt, cfg, k, v, [N, 77])
    out, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), bt.alloc_workspace_kv4(cfg)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(q), out, ws)
    ref, tol = lb.decode(f64(q), lb.held(f64(k)), lb.held(f64(v)), [N, 77])
    check(out, ref, tol, "large scores")


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [1, 3])
def test_rows_of_unlike_size(bt, hd, splits):
    """V of sizes from 2^-90 to 2^90 under weights that make up for it or not: a huge row that gets next to no weight takes no precision from
    the others, tiny rows alone keep theirs, and the size grows and shrinks along the rows."""
    B, H, N = 4, 2, 330
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    q, k, v = f64(rnd(18, 3, (B, H, hd))), f64(rnd(18, 1, (B, H, N, hd))), f64(rnd(18, 2, (B, H, N, hd)))
    q[..., 0] = 8.0
    k[..., 0] = 0.0
    k[0, :, 17, 0], v[0, :, 17] = -90.0, v[0, :, 17] * 2.0 ** 60      # weight about 2^-100: huge all the same
    k[0, :, 18, 0], v[0, :, 18] = -60.0, v[0, :, 18] * 2.0 ** 30
    v[1] *= 2.0 ** -90
    v[2] *= 2.0 ** np.linspace(-90, 90, N)[None, :, None]             # and the scores fall as the rows grow
    k[2, :, :, 0] = -np.linspace(0, 90, N) / 2
    v[3] *= 2.0 ** np.linspace(40, -40, N)[None, :, None]
    q, k, v = bits(q), bits(k), bits(v)
    lens = [N, N, N, 301]
    cache = filled(bt, cfg, k, v, lens)
    out, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), bt.alloc_workspace_kv4(cfg)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(q), out, ws)
    ref, tol = lb.decode(f64(q), lb.held(f64(k)), lb.held(f64(v)), lens)
    check(out, ref, tol, "unlike rows")


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("up", [-100, 100])
def test_queries_and_keys_of_unlike_size(bt, hd, up):
    """Products of ordinary size of a tiny query and huge keys, and the other way round."""
    B, H, N = 2, 2, 90
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    q, k, v = f64(rnd(19, 3, (B, H, hd))) * 2.0 ** -up, f64(rnd(19, 1, (B, H, N, hd))) * 2.0 ** up, rnd(19, 2, (B, H, N, hd))
    q, k = bits(q), bits(k)
    cache = filled(bt, cfg, k, v, [N, 41])
    out, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), bt.alloc_workspace_kv4(cfg)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(q), out, ws)
    ref, tol = lb.decode(f64(q), lb.held(f64(k)), lb.held(f64(v)), [N, 41])
    check(out, ref, tol, "unlike query and keys")


@pytest.mark.parametrize("hd", [64, 128])
def test_small_values_over_many_rows(bt, hd):
    """Values near 2^-97 under 409200 equal weights: the weights' power of two is at its end there, and with the sum of the weights it would
    be 20.5 times the least number of fp32.  Exact here: all rows are alike, so an output is its value."""
    n = 409200
    cfg = bt.make_config(1, 1, hd, 4, 1, n, 1, decode_splits=1)
    value = np.ldexp(np.tile(np.arange(-7.0, 8.0), hd)[:hd], -100)
    value[::32] = np.ldexp(7.0, -100)     # the step is 2^-100
    row = torch.from_numpy(value).to("cuda", torch.bfloat16)
    rows = row.expand(1, 1, n, hd).contiguous()
    cache, q, out = empty_cache(bt, cfg), torch.zeros((1, 1, hd), dtype=torch.bfloat16, device="cuda"), torch.empty((1, 1, hd), dtype=torch.bfloat16, device="cuda")
    bt.bt_block_kv4_append(cfg, cache, 0, rows, rows)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, q, out, bt.alloc_workspace_kv4(cfg))
    # sums in fp32, flushed n / 64 / 512 = 13 times with four roundings of 2^-24 each, far below the half step of the result, 2^-8
    check(out, value[None, None], 1.01 * 2.0 ** -8 * np.abs(value), "out")


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [1, 4])
def test_values_that_are_not_finite(bt, hd, splits):
    B, H, N = 6, 2, 200
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    k, v, q = rnd(16, 1, (B, H, N, hd)), rnd(16, 2, (B, H, N, hd)), rnd(16, 3, (B, H, hd))
    k[0, 1, 3, 40] = 0x7FC0            # NaN in K: the head's whole output
    v[1, 0, 199, 40] = 0x7F80          # infinity in V: the 32 dimensions of its step
    v[2, 1, 64, 0] = 0x7FC0
    k[3, 0, 130, 5] = 0xFF80           # held as NaN
    k[4, :, 150:] = 0x7FC0             # past the length
    q[5, 1, 7] = 0x7FC0 if splits == 1 else 0xFF80
    lens = [N, N, N, N, 150, N]
    cache = filled(bt, cfg, k, v, lens)
    out, ws = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), bt.alloc_workspace_kv4(cfg)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(q), out, ws)
    bad = torch.isnan(out).cpu().numpy()
    want = np.zeros((B, H, hd), bool)
    want[0, 1] = want[3, 0] = want[5, 1] = True
    want[1, 0, 32:64] = want[2, 1, :32] = True
    assert np.array_equal(bad, want)


def test_scores_of_minus_infinity_have_no_weight(bt):
    """Steps so large that scores overflow: minus infinity drops out, and where all are the output is zeros."""
    B, H, hd, N = 2, 1, 64, 40
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, softmax_scale=1e37)
    k, v = np.full((B, H, N, hd), 0.0), f64(rnd(17, 2, (B, H, N, hd)))
    k[:, :, :, 0] = -7.0
    k[0, :, 11, 0] = 0.0               # the one score that is not minus infinity (0 times the scale)
    q = np.zeros((B, H, hd))
    q[..., 0] = 7.0
    cache = filled(bt, cfg, bits(k), bits(v), [N, N])
    out, st = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda"), status_word()
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, to_dev(bits(q)), out, bt.alloc_workspace_kv4(cfg), dev_status=st)
    assert np.array_equal(to_f64(out)[0, 0], lb.to_bf16(lb.held(v[0, 0, 11]))) and (out[1] == 0).all() and st.item() == 0


# ------------------------------------------------------------------------------------------------ 8-bit projections

@pytest.mark.parametrize("rows,cols", [(1, 16), (7, 512), (33, 528), (2, 1024), (1000, 1040), (5, 2048)])
def test_rows_quantised(bt, rows, cols):
    x = f64(rnd(21, rows, (rows, cols)))
    x[0, :] = np.linspace(-127, 127, cols).round() / 2    # halves
    x[0, 0] = 127.0
    if rows > 4:
        x[1, :], x[2, 3], x[3, cols - 1] = 0.0, np.nan, -np.inf
        x[4, :] *= 2.0 ** -126
    xb = bits(x)
    x8 = torch.full((rows, cols), 99, dtype=torch.int8, device="cuda")
    steps = torch.full((rows,), 99.0, device="cuda")
    bt.bt_rows_quantize_i8(to_dev(xb), x8, steps)
    codes, want = lb.quantised(f64(xb), 127)
    assert np.array_equal(steps.double().cpu().numpy(), want, equal_nan=True)
    assert np.array_equal(x8.cpu().numpy(), codes)


def operands(seed, rows, features, D):
    """int8 x and w over the whole range of codes with steps that make y of unit size, and a bias."""
    rng = np.random.default_rng(seed)
    x8 = rng.integers(-128, 128, (rows, D)).astype(np.int8)
    w8 = rng.integers(-128, 128, (features, D)).astype(np.int8)
    xs = (rng.uniform(0.5, 2.0, rows) / 74).astype(np.float32)
    ws = (rng.uniform(0.5, 2.0, features) / 74 / np.sqrt(D)).astype(np.float32)
    return x8, xs, w8, ws, rnd(seed, 9, (features,))


def cuda(x):
    return torch.from_numpy(x).cuda()


@pytest.mark.parametrize("B,H,hd,P,with_bias", [(1, 1, 64, 1, True), (5, 2, 64, 3, False), (300, 16, 128, 1, True), (131, 5, 128, 2, True),
                                                (4100, 7, 64, 2, False), (700, 16, 64, 8, True)])
def test_prefix_projection_of_integers(bt, B, H, hd, P, with_bias):
    D = H * hd
    cfg = bt.make_config(B, H, hd, 4, P, 8, 1)
    x8, xs, w8, ws, bias = operands(B, B, P * D, D)
    out, st = torch.full((B, P, D), 9.0, dtype=torch.bfloat16, device="cuda"), status_word()
    bt.bt_prefix_project_i8(cfg, cuda(x8), cuda(xs), cuda(w8), cuda(ws), to_dev(bias) if with_bias else None, out, dev_status=st)
    ref, tol = lb.project(x8, xs.astype(np.float64), w8, ws.astype(np.float64), f64(bias) if with_bias else None)
    check(out, ref.reshape(B, P, D), tol.reshape(B, P, D), "prefix")
    assert st.item() == 0


def test_whole_sums_are_exact(bt):
    """The largest sums there are (2048 products of -128 and -128), and sums that fp32 would not hold term by term."""
    B, H, hd = 3, 16, 128
    D = H * hd
    cfg = bt.make_config(B, H, hd, 4, 1, 8, 1)
    x8 = np.full((B, D), -128, np.int8)
    w8 = np.full((D, D), -128, np.int8)
    x8[1, ::2], x8[2] = 127, 1
    w8[1::2, ::2] = 127
    xs, ws = np.ones(B, np.float32), np.ones(D, np.float32)
    out = torch.empty((B, 1, D), dtype=torch.bfloat16, device="cuda")
    bt.bt_prefix_project_i8(cfg, cuda(x8), cuda(xs), cuda(w8), cuda(ws), None, out)
    want = x8.astype(np.int64) @ w8.astype(np.int64).T
    assert want.max() == 2 ** 25 and np.array_equal(to_f64(out)[:, 0], lb.to_bf16(want.astype(np.float64)))


@pytest.mark.parametrize("B,H,hd,n,N", [(5, 2, 64, 1, 9), (3, 9, 64, 4, 20), (130, 3, 128, 1, 3), (2, 16, 128, 150, 170), (260, 12, 64, 2, 8)])
def test_block_qkv_of_integers(bt, B, H, hd, n, N):
    D = H * hd
    cfg = bt.make_config(B, H, hd, 4, 1, N, 2)
    x8, xs, w8, ws, bias = operands(B + n, B * n, 3 * D, D)
    cache, st = bt.BlockCache(cfg), status_word()
    cache.k.fill_(7.0), cache.v.fill_(7.0)
    lens = [(b * 5) % (N + 1) for b in range(B)]
    cache.len[1].copy_(torch.tensor(lens, dtype=torch.int32))
    q = torch.empty((B, H, n, hd), dtype=torch.bfloat16, device="cuda")
    bt.bt_block_qkv_project_append_i8(cfg, cache, 1, cuda(x8).view(B, n, D), cuda(xs), cuda(w8), cuda(ws), to_dev(bias), q, dev_status=st)
    ref, tol = lb.project(x8, xs.astype(np.float64), w8, ws.astype(np.float64), f64(bias))
    part = lambda t, i: t.reshape(B, n, 3, H, hd)[:, :, i].transpose(0, 2, 1, 3)   # noqa: E731
    check(q, part(ref, 0), part(tol, 0), "q")
    k, v = to_f64(cache.k[1]), to_f64(cache.v[1])
    full = False
    for b, m in enumerate(lens):
        ok = m + n <= N
        full |= not ok
        for got, i in ((k, 1), (v, 2)):
            rows = got[b, :, m:m + n] if ok else got[b, :, :0]
            assert (np.abs(rows - part(ref, i)[b, :, :rows.shape[1]]) <= part(tol, i)[b, :, :rows.shape[1]]).all()
            assert (np.delete(got[b], range(m, m + n) if ok else [], axis=1) == 7.0).all()
    assert cache.len[1].tolist() == [m + n if m + n <= N else m for m in lens] and (cache.k[0] == 7.0).all()
    assert st.item() == (bt.BT_DEV_OVERFLOW if full else 0)


@pytest.mark.parametrize("B,H,hd,n", [(6, 2, 64, 1), (140, 5, 128, 3)])
def test_local_qkv_of_integers(bt, B, H, hd, n):
    D, P = H * hd, 3
    cfg = bt.make_config(B, H, hd, 4, P, 1, 1)
    x8, xs, w8, ws, bias = operands(B + 50, B * n, 3 * D, D)
    cache = bt.LocalCache(cfg)
    cache.len[0].copy_(torch.arange(B, dtype=torch.int32) % 4)
    mask = (torch.arange(B, device="cuda") % 3 == 0).to(torch.uint8)
    q = torch.empty((B, H, n, hd), dtype=torch.bfloat16, device="cuda")
    bt.bt_local_qkv_project_append_i8(cfg, cache, 0, cuda(x8).view(B, n, D), cuda(xs), cuda(w8), cuda(ws), to_dev(bias), q, reset_mask=mask)
    ref, tol = lb.project(x8, xs.astype(np.float64), w8, ws.astype(np.float64), f64(bias))
    part = lambda t, i: t.reshape(B, n, 3, H, hd)[:, :, i].transpose(0, 2, 1, 3)   # noqa: E731
    check(q, part(ref, 0), part(tol, 0), "q")
    k, v = (f64(x) for x in local_kv_split(cache.kv[0]))
    for b in range(B):
        m = 0 if b % 3 == 0 else b % 4
        assert cache.len[0, b] == m + n
        for got, i in ((k, 1), (v, 2)):
            assert (np.abs(got[b, :, m:m + n] - part(ref, i)[b]) <= part(tol, i)[b]).all()
            assert (np.delete(got[b], range(m, m + n), axis=1) == 0).all()


@pytest.mark.parametrize("B,H,hd,n", [(1500, 20, 64, 1), (256, 16, 128, 4), (238, 21, 64, 5), (75, 16, 128, 17)])
def test_products_that_end_in_parts_of_tiles(bt, B, H, hd, n):
    """Products of somewhat more tiles than pairs of processors (six rows of 15, four of 24, five of 16 - the last of them three quarters there -
    and five of 24): those of the last round are worked in halves or quarters.  Into the local cache from its first row, into the block cache, in 4 bits."""
    D = H * hd
    x8, xs, w8, ws, bias = operands(B + 90, B * n, 3 * D, D)
    args = (cuda(x8).view(B, n, D), cuda(xs), cuda(w8), cuda(ws), to_dev(bias))
    ref, tol = lb.project(x8, xs.astype(np.float64), w8, ws.astype(np.float64), f64(bias))
    part = lambda t, i: t.reshape(B, n, 3, H, hd)[:, :, i].transpose(0, 2, 1, 3)   # noqa: E731
    cfg = bt.make_config(B, H, hd, 4, n, n + 3, 1)
    local, q, st = bt.LocalCache(cfg), torch.empty((B, H, n, hd), dtype=torch.bfloat16, device="cuda"), status_word()
    local.len.fill_(3)
    bt.bt_local_qkv_project_append_i8(cfg, local, 0, *args, q, reset_first=True, dev_status=st)
    k, v = (f64(x) for x in local_kv_split(local.kv[0]))
    for got, i in ((to_f64(q), 0), (k[:, :, :n], 1), (v[:, :, :n], 2)):
        assert (np.abs(got - part(ref, i)) <= part(tol, i)).all(), i
    assert (local.len == n).all() and st.item() == 0 and not k[:, :, n:].any() and not v[:, :, n:].any()

    block, q2 = bt.BlockCache(cfg), torch.empty_like(q)
    block.len.fill_(2)
    bt.bt_block_qkv_project_append_i8(cfg, block, 0, *args, q2)
    assert torch.equal(q, q2) and (block.len == n + 2).all() and not block.k[0, :, :, :2].any()
    assert np.array_equal(to_f64(block.k[0, :, :, 2:n + 2]), k[:, :, :n]) and np.array_equal(to_f64(block.v[0, :, :, 2:n + 2]), v[:, :, :n])
    one, two = empty_cache(bt, cfg), empty_cache(bt, cfg)
    one.len.fill_(2), two.len.fill_(2)
    bt.bt_block_qkv_project_append_i8_kv4(cfg, one, 0, *args, q2)
    bt.bt_block_kv4_append(cfg, two, 0, block.k[0, :, :, 2:n + 2], block.v[0, :, :, 2:n + 2])
    assert torch.equal(q, q2) and torch.equal(one.kv, two.kv) and torch.equal(one.len, two.len)

    # bf16: powers of two and small whole numbers, so that every sum is exact
    x = f64(rnd(91, 3, (B * n, D))).round()
    w = np.ldexp(np.random.default_rng(B).integers(-1, 2, (3 * D, D)).astype(np.float64), -4)
    want = x @ w.T
    assert np.abs(want).max() < 2 ** 16   # whole numbers of sixteenths below 2^24
    bt.bt_local_qkv_project_append(cfg, local, 0, to_dev(bits(x)).view(B, n, D), to_dev(bits(w)), None, q, reset_first=True)
    k, v = (f64(x) for x in local_kv_split(local.kv[0]))
    for got, i in ((to_f64(q), 0), (k[:, :, :n], 1), (v[:, :, :n], 2)):
        assert np.array_equal(got, lb.to_bf16(part(want, i))), i


def test_steps_that_are_not_finite(bt):
    """A token quantised from a NaN makes its own outputs NaN and no others; so does a feature's step."""
    B, H, hd = 40, 2, 64
    D = H * hd
    cfg = bt.make_config(B, H, hd, 4, 1, 8, 1)
    x = rnd(31, 0, (B, D))
    x[7, 100] = 0x7FC0
    x8, xs = torch.empty((B, D), dtype=torch.int8, device="cuda"), torch.empty(B, device="cuda")
    bt.bt_rows_quantize_i8(to_dev(x), x8, xs)
    _, _, w8, ws, _ = operands(32, B, D, D)
    ws[5] = np.nan
    out = torch.empty((B, 1, D), dtype=torch.bfloat16, device="cuda")
    bt.bt_prefix_project_i8(cfg, x8, xs, cuda(w8), cuda(ws), None, out)
    want = np.zeros((B, D), bool)
    want[7], want[:, 5] = True, True
    assert np.array_equal(torch.isnan(out)[:, 0].cpu().numpy(), want)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("B,H,hd,n,N", [(5, 2, 64, 1, 9), (33, 3, 128, 5, 40), (2, 16, 128, 150, 170), (300, 12, 64, 1, 70)])
def test_projection_into_the_4_bit_cache(bt, int8, B, H, hd, n, N):
    """Bit for bit what the projection into a bf16 cache and an append of its rows give."""
    D = H * hd
    cfg = bt.make_config(B, H, hd, 4, 1, N, 2)
    rows = bt.make_config(B, H, hd, 4, 1, n, 1)      # a bf16 cache of the new rows alone
    lens = torch.tensor([(b * 7) % (N + 1) for b in range(B)], dtype=torch.int32)
    one, two, new = empty_cache(bt, cfg), empty_cache(bt, cfg), bt.BlockCache(rows)
    for cache in (one, two):
        cache.len[1].copy_(lens)
    qa, qb = (torch.empty((B, H, n, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sa, sb = status_word(), status_word()
    if int8:
        x8, xs, w8, ws, bias = operands(B + 70, B * n, 3 * D, D)
        args = (cuda(x8).view(B, n, D), cuda(xs), cuda(w8), cuda(ws), to_dev(bias))
        bt.bt_block_qkv_project_append_i8_kv4(cfg, one, 1, *args, qa, dev_status=sa)
        bt.bt_block_qkv_project_append_i8(rows, new, 0, *args, qb)
    else:
        args = (to_dev(rnd(41, 0, (B, n, D))), to_dev(bits(f64(rnd(41, 1, (3 * D, D))) / np.sqrt(D))), to_dev(rnd(41, 2, (3 * D,))))
        bt.bt_block_qkv_project_append_kv4(cfg, one, 1, *args, qa, dev_status=sa)
        bt.bt_block_qkv_project_append(rows, new, 0, *args, qb)
    bt.bt_block_kv4_append(cfg, two, 1, new.k[0], new.v[0], dev_status=sb)
    assert torch.equal(qa, qb) and torch.equal(one.kv, two.kv) and torch.equal(one.len, two.len) and sa.item() == sb.item()


# ------------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("hd,H", [(64, 3), (128, 2)])
def test_generation_in_few_bits(bt, hd, H):
    """A prompt projected into the 4-bit cache and read back for its own attention, then steps: activations quantised, projected
    into the cache, attended over it - against the definitions over the whole history, two layers, under a captured graph."""
    B, T, steps, layers = 3, 21, 4, 2
    D, N = H * hd, T + steps
    cfg = bt.make_config(B, H, hd, 4, 1, N, layers)
    cache, ws = empty_cache(bt, cfg), bt.alloc_workspace_kv4(cfg)
    w = []
    for layer in range(layers):
        wb = to_dev(bits(f64(rnd(51, layer, (3 * D, D))) / np.sqrt(D)))
        w8, wst = torch.empty((3 * D, D), dtype=torch.int8, device="cuda"), torch.empty(3 * D, device="cuda")
        bt.bt_rows_quantize_i8(wb, w8, wst)
        w.append((w8, wst))
    K, V = np.zeros((layers, B, H, N, hd)), np.zeros((layers, B, H, N, hd))

    def expected(layer, x, n0):
        """Projected rows of x [B,n,D] (bits); q, and K, V of the history as held."""
        n = x.shape[1]
        codes, xs = lb.quantised(f64(x).reshape(B * n, D), 127)
        y, _ = lb.project(codes, xs, w[layer][0].cpu().numpy(), w[layer][1].double().cpu().numpy(), None)
        y = y.reshape(B, n, 3, H, hd).transpose(2, 0, 3, 1, 4)
        return y, n

    def close_rows(got, want):
        # K and V come out of the product within its rounding; a value next to a code's border may take the next code
        want_codes, want_steps = lb.kv4(lb.to_bf16(want))
        off = np.abs(got - lb.kv4_values(want_codes, want_steps)) / np.repeat(want_steps, 32, -1)
        assert off.max() < 1.1 and (off > 0.06).mean() < 0.01

    bufs = dict(x8=torch.empty((B, 1, D), dtype=torch.int8, device="cuda"), xs=torch.empty((B, 1), device="cuda"),
                x=torch.empty((B, 1, D), dtype=torch.bfloat16, device="cuda"),
                q=torch.empty((layers, B, H, 1, hd), dtype=torch.bfloat16, device="cuda"),
                o=torch.empty((layers, B, H, hd), dtype=torch.bfloat16, device="cuda"))
    # the prompt
    for layer in range(layers):
        x = rnd(52, layer, (B, T, D))
        x8, xs = torch.empty((B, T, D), dtype=torch.int8, device="cuda"), torch.empty((B, T), device="cuda")
        q = torch.empty((B, H, T, hd), dtype=torch.bfloat16, device="cuda")
        bt.bt_rows_quantize_i8(to_dev(x), x8, xs)
        bt.bt_block_qkv_project_append_i8_kv4(cfg, cache, layer, x8, xs, *w[layer], None, q)
        k, v, o = (torch.zeros((B, H, T, hd), dtype=torch.bfloat16, device="cuda") for _ in range(3))
        bt.bt_block_kv4_read(cfg, cache, layer, k, v)
        bt.bt_block_prefill_attn(cfg, q, k, v, o)
        y, _ = expected(layer, x, 0)
        close_rows(to_f64(k), y[1])
        close_rows(to_f64(v), y[2])
        K[layer, :, :, :T], V[layer, :, :, :T] = to_f64(k), to_f64(v)
        # the last position of the prompt attends over all of it: the cache's own attention gives the same
        got = torch.empty((B, H, hd), dtype=torch.bfloat16, device="cuda")
        bt.bt_block_decode_attn_kv4(cfg, cache, layer, q[:, :, -1].contiguous(), got, ws)
        assert (got.float() - o[:, :, -1].float()).abs().max() < 0.05

    def step():
        bt.bt_rows_quantize_i8(bufs["x"], bufs["x8"], bufs["xs"])
        for layer in range(layers):
            bt.bt_block_qkv_project_append_i8_kv4(cfg, cache, layer, bufs["x8"], bufs["xs"], *w[layer], None, bufs["q"][layer])
            bt.bt_block_decode_attn_kv4(cfg, cache, layer, bufs["q"][layer], bufs["o"][layer], ws)

    graph = None
    for i in range(steps):
        x = rnd(53, i, (B, 1, D))
        bufs["x"].copy_(to_dev(x))
        if i == 0:
            step()
        elif i == 1:
            stream = torch.cuda.Stream()
            stream.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                step()
        if i > 0:
            graph.replay()
        torch.cuda.synchronize()
        n = T + i + 1
        assert (cache.len == n).all()
        for layer in range(layers):
            k, v = (torch.zeros((B, H, N, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            bt.bt_block_kv4_read(cfg, cache, layer, k, v)
            y, _ = expected(layer, x, n - 1)
            close_rows(to_f64(k)[:, :, n - 1:n], y[1])
            assert np.array_equal(to_f64(k)[:, :, :n - 1], K[layer, :, :, :n - 1])   # the rows before stay as they are
            K[layer], V[layer] = to_f64(k), to_f64(v)
            # against the rows as read back, whose rounding to bf16 moves scores and values by 2^-8 at most
            ref, tol = lb.decode(to_f64(bufs["q"][layer][:, :, 0]), K[layer], V[layer], [n] * B)
            check(bufs["o"][layer], ref, tol + 0.02 + 0.02 * np.abs(ref), f"step {i} layer {layer}")


def test_strided_rows(bt):
    """Views of larger slabs are taken as they lie (append) and written as they lie (read); what no slab stride says is refused."""
    hd, N, n = 64, 40, 21
    for B, H in ((3, 4), (1, 4), (3, 1), (1, 1)):
        cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
        K, V = to_dev(rnd(71, 1, (B, H, N, hd))), to_dev(rnd(71, 2, (B, H, N, hd)))
        a, b = empty_cache(bt, cfg), empty_cache(bt, cfg)
        bt.bt_block_kv4_append(cfg, a, 0, K[:, :, 5:5 + n], V[:, :, 7:7 + n], reset_first=True)
        bt.bt_block_kv4_append(cfg, b, 0, K[:, :, 5:5 + n].contiguous(), V[:, :, 7:7 + n].contiguous(), reset_first=True)
        assert torch.equal(a.kv, b.kv) and torch.equal(a.len, b.len)
        packed = [torch.empty((B, H, n, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        wide = [torch.full((B, H, N, hd), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        bt.bt_block_kv4_read(cfg, a, 0, *packed)
        bt.bt_block_kv4_read(cfg, a, 0, *[x[:, :, 3:3 + n] for x in wide])
        for x, y in zip(packed, wide):
            assert torch.equal(x, y[:, :, 3:3 + n]) and (y[:, :, :3] == 9).all() and (y[:, :, 3 + n:] == 9).all()
    cfg = bt.make_config(3, 4, hd, 4, 1, N, 1)
    K = to_dev(rnd(71, 3, (3, 4, N, hd)))
    cache = empty_cache(bt, cfg)
    by_row = K.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)[:, :, :n]   # [B][n][H][hd] in memory
    for k, v in ((by_row, by_row), (K[:, :, ::2], K[:, :, ::2]), (K[:, :, :n], K[:, :, :n].contiguous()), (K[:, :2, :n], K[:, :2, :n]),
                 (K[:, :1, :n].expand(3, 4, n, hd), K[:, :, :n])):
        with pytest.raises(bt.BtError) as e:
            bt.bt_block_kv4_append(cfg, cache, 0, k, v)
        assert e.value.code == bt.BT_ERR_UNSUPPORTED
    torch.cuda.synchronize()
    assert (cache.len == 0).all()


def test_tensors_elsewhere_and_not_packed_are_refused(bt):
    """Each tensor of a call in turn in the host's memory, or with strides: refused before anything is launched."""
    B, H, hd, N = 2, 2, 64, 8
    cfg, D = bt.make_config(B, H, hd, 4, 1, N, 1), H * hd
    cache, block, local, ws = bt.BlockCacheKV4(cfg), bt.BlockCache(cfg), bt.LocalCache(cfg), bt.alloc_workspace_kv4(cfg)

    def t(*shape, dtype=torch.bfloat16):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    q, x, w, bias, qo = t(B, H, hd), t(B, 1, D), t(3 * D, D), t(3 * D), t(B, H, 1, hd)
    x8, w8, xs, wsteps = t(B, 1, D, dtype=torch.int8), t(3 * D, D, dtype=torch.int8), t(B, 1, dtype=torch.float32), t(3 * D, dtype=torch.float32)
    status, mask = t(1, dtype=torch.int32), t(B, dtype=torch.uint8)
    calls = [
        (lambda *a: bt.bt_block_decode_attn_kv4(cfg, cache, 0, *a), [q, q, ws, status]),
        (lambda *a: bt.bt_block_decode_step_kv4(cfg, cache, 0, *a), [q, q, q, q, ws, status]),
        (lambda a, b, c, d, s: bt.bt_block_qkv_project_append_kv4(cfg, cache, 0, a, b, c, d, dev_status=s), [x, w, bias, qo, status]),
        (bt.bt_rows_quantize_i8, [x, x8, xs]),
        (lambda *a: bt.bt_prefix_project_i8(cfg, *a), [x8, xs, w8[:D], wsteps[:D], bias[:D], x, status]),
        (lambda *a: bt.bt_block_qkv_project_append_i8(cfg, block, 0, *a[:-1], dev_status=a[-1]), [x8, xs, w8, wsteps, bias, qo, status]),
        (lambda *a: bt.bt_local_qkv_project_append_i8(cfg, local, 0, *a[:-2], reset_mask=a[-2], dev_status=a[-1]),
         [x8, xs, w8, wsteps, bias, qo, mask, status]),
        (lambda *a: bt.bt_block_qkv_project_append_i8_kv4(cfg, cache, 0, *a[:-1], dev_status=a[-1]), [x8, xs, w8, wsteps, bias, qo, status]),
    ]
    for call, args in calls:
        for i, arg in enumerate(args):
            bad = [arg.cpu()]
            if arg.numel() > 1:
                bad.append(torch.stack([arg, arg], -1)[..., 0])
            for b in bad:
                with pytest.raises(bt.BtError) as e:
                    call(*args[:i], b, *args[i + 1:])
                assert e.value.code == bt.BT_ERR_UNSUPPORTED
    rows = t(B, H, 1, hd)
    for call in (bt.bt_block_kv4_append, bt.bt_block_kv4_read):
        for k, v in ((rows.cpu(), rows), (rows, rows.cpu())):
            with pytest.raises(bt.BtError) as e:
                call(cfg, cache, 0, k, v)
            assert e.value.code == bt.BT_ERR_UNSUPPORTED
    torch.cuda.synchronize()
    assert (cache.len == 0).all() and (block.len == 0).all() and (local.len == 0).all()


def test_other_streams_and_two_calls_at_once(bt):
    """Two streams at once with a workspace each; results as alone."""
    B, H, hd, N = 16, 4, 128, 700
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1)
    k, v, q = rnd(61, 1, (B, H, N, hd)), rnd(61, 2, (B, H, N, hd)), rnd(61, 3, (B, H, hd))
    cache = empty_cache(bt, cfg)
    bt.bt_block_kv4_append(cfg, cache, 0, to_dev(k), to_dev(v))
    q = to_dev(q)
    alone = torch.empty_like(q)
    bt.bt_block_decode_attn_kv4(cfg, cache, 0, q, alone, bt.alloc_workspace_kv4(cfg))
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(q) for _ in range(2)]
    spaces = [bt.alloc_workspace_kv4(cfg) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, o, w in zip(streams, outs, spaces):
            bt.bt_block_decode_attn_kv4(cfg, cache, 0, q, o, w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, alone) for o in outs)
