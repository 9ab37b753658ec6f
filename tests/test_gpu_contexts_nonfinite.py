"""GPU tests of the operators for long and shared contexts on visible rows that are not finite: a NaN score, or one of plus infinity, makes the
(sequence, head) that sees it NaN wherever the row lies and however the row range is cut; a score of minus infinity is a
weight of zero; if nothing else is visible the output is zeros.  No other (sequence, head) notices."""
import numpy as np
import pytest
import torch

from oracle import contexts as ctx
from workloads import gen

from test_gpu_contexts import f64, make_cache, rnd, shared_case
from util import status_word, to_dev, to_f64

pytestmark = pytest.mark.gpu

NAN, INF, NEG_INF = 0x7FC0, 0x7F80, 0xFF80


@pytest.fixture(scope="module")
def bt():
    import paper_2406_02657_b200 as bt
    assert torch.cuda.is_available()
    return bt


def attend(q, K, V, p_bf16=False):
    """(out, tol, weights, relative tol on them) of one query over its visible rows, which may hold anything."""
    hd = q.shape[0]
    with np.errstate(invalid="ignore", over="ignore"):
        s = K @ q
    if np.isnan(s).any() or (s == np.inf).any():
        return np.full(hd, np.nan), np.zeros(hd), np.full(len(s), np.nan), 0.0
    some = s != -np.inf
    out, p, tol, rel = ctx.attend(q, K[some], np.nan_to_num(V[some]), p_bf16=p_bf16)
    out = np.where(np.isnan(V).any(0), np.nan, out)
    weights = np.zeros(len(s))
    weights[some] = p
    return out, tol, weights, rel


def check(got, ref, tol, what):
    g = to_f64(got).reshape(ref.shape)
    bad = np.isnan(ref)
    assert np.isnan(g[bad]).all(), f"{what}: finite where the definition has a NaN, at {np.argwhere(bad & ~np.isnan(g))[:5].tolist()}"
    assert np.isfinite(g[~bad]).all(), f"{what}: not finite at {np.argwhere(~bad & ~np.isfinite(g))[:5].tolist()}"
    over = (np.abs(g - ref) - tol)[~bad]
    assert (over <= 0).all(), f"{what}: {over.max():.3e} beyond the bound"


def poison(k, v, q, at):
    """One bad row per sequence, at[b]: in K of head 0 a NaN, in V of head 1 a NaN (dimension 5), in K of head 2 an infinity
    (dimension 7: a score of plus or minus infinity by the sign of q there); head 3 stays clean."""
    for b, j in enumerate(at):
        k[b, 0, j, b % 8] = NAN
        v[b, 1, j, 5] = NAN
        k[b, 2, j, 7] = INF if b % 2 else NEG_INF


def one_by_one(q, K, V, rows, p_bf16=False):
    """attend() for every (sequence, head); rows(b, h) are its visible K and V."""
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    weights = {}
    for b in range(q.shape[0]):
        for h in range(q.shape[1]):
            out[b, h], tol[b, h], *weights[b, h] = attend(q[b, h], *rows(b, h), p_bf16=p_bf16)
    return out, tol, weights


# whole chunks, chunk borders, the ragged end (where a row group holds one row), both ends
AT = [0, 1, 31, 32, 63, 64, 130, 255, 256, 257, 259, 260]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [0, 1, 2, 3, 7])
@pytest.mark.parametrize("window,sinks", [(300, 0), (4, 3), (100, 33)])
def test_window_decode_visible(bt, hd, splits, window, sinks):
    B, H, N = len(AT), 4, 261
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    k, v, q = rnd(61, 1, (B, H, N, hd)), rnd(61, 2, (B, H, N, hd)), rnd(61, 3, (B, H, hd))
    poison(k, v, q, AT)
    cache = make_cache(bt, cfg, k, v, [N] * B)
    out, st, ws = torch.zeros((B, H, hd), dtype=torch.bfloat16, device="cuda"), status_word(), bt.alloc_workspace(cfg)
    bt.bt_block_decode_attn_window(cfg, cache, 0, to_dev(q), window, sinks, out, ws, dev_status=st)
    K, V, seen = f64(k), f64(v), ctx.window_rows(N, window, sinks)
    check(out, *one_by_one(f64(q), K, V, lambda b, h: (K[b, h, seen], V[b, h, seen]))[:2], f"window {window} sinks {sinks}")
    assert st.item() == 0
    if window > N:   # all rows: the plain call
        bt.bt_block_decode_attn(cfg, cache, 0, to_dev(q), out, ws, dev_status=st)
        check(out, *one_by_one(f64(q), K, V, lambda b, h: (K[b, h], V[b, h]))[:2], "plain")


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [1, 4])
@pytest.mark.parametrize("call", ["window", "weights", "shared"])
def test_appended_row_visible(bt, hd, splits, call):
    """The appended row is the bad one: alone, behind few rows, behind many."""
    lens = [0, 1, 2, 3, 4, 31, 32, 33, 100, 129]
    B, H, N = len(lens), 4, 130
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    k, v = rnd(62, 1, (B, H, N, hd)), rnd(62, 2, (B, H, N, hd))
    cache = make_cache(bt, cfg, k, v, lens)
    q, kn, vn = (rnd(62, 3 + i, (B, H, hd)) for i in range(3))
    poison(kn[:, :, None], vn[:, :, None], q, [0] * B)
    out, st = torch.zeros((B, H, hd), dtype=torch.bfloat16, device="cuda"), status_word()
    for b, n in enumerate(lens):
        k[b, :, n], v[b, :, n] = kn[b], vn[b]
    K, V = f64(k), f64(v)
    rows = lambda b, h: (K[b, h, :lens[b] + 1], V[b, h, :lens[b] + 1])   # noqa: E731
    if call == "window":
        bt.bt_block_decode_step_window(cfg, cache, 0, to_dev(q), to_dev(kn), to_dev(vn), N, 0, out, bt.alloc_workspace(cfg), dev_status=st)
    elif call == "weights":
        w = torch.zeros((1, B, H, N), device="cuda")
        bt.bt_block_decode_step_weights(cfg, cache, 0, to_dev(q), to_dev(kn), to_dev(vn), out, w, w, bt.alloc_workspace_weights(cfg), dev_status=st)
    else:
        prefix = bt.BlockCache(bt.make_config(1, H, hd, 4, 1, 8, 1))
        bt.bt_block_decode_step_shared(cfg, prefix, cache, 0, to_dev(q), to_dev(kn), to_dev(vn), out, bt.alloc_workspace_shared(cfg, 8), dev_status=st)
    check(out, *one_by_one(f64(q), K, V, rows, p_bf16=call == "shared")[:2], call)
    assert st.item() == 0 and cache.len[0].tolist() == [n + 1 for n in lens]


# few pairs (the own rows' kernel joins), many (a launch of its own joins): a warp per pair, a CTA per pair, parts of own rows; one part of
# the prefix and several
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("B,N,cap,splits", [(12, 70, 700, 0), (12, 70, 64, 0), (12, 261, 700, 3), (200, 60, 700, 0), (200, 60, 60, 0), (200, 140, 700, 0)])
def test_shared_prefix_visible(bt, hd, B, N, cap, splits):
    H, S = 4, cap - 1
    lens = [N if b < 12 else (b * 37) % (N + 1) for b in range(B)]
    lens[-1] = 0
    q = rnd(63, 9, (B, H, hd))
    # the bad row among the sequences' own
    cfg, cache, prefix, k, v, pk, pv = shared_case(bt, B, H, hd, cap, S, N, lens, splits, seed=63)
    at = [a % N for a in AT[:min(B, 12) - 1]]
    poison(k, v, q, at)
    cache = make_cache(bt, cfg, k, v, lens)
    out, st, ws = torch.zeros((B, H, hd), dtype=torch.bfloat16, device="cuda"), status_word(), bt.alloc_workspace_shared(cfg, cap)
    K, V, PK, PV, Q = f64(k), f64(v), f64(pk), f64(pv), f64(q)

    def rows(b, h):
        return np.concatenate([PK[h, :S], K[b, h, :lens[b]]]), np.concatenate([PV[h, :S], V[b, h, :lens[b]]])

    bt.bt_block_decode_attn_shared(cfg, prefix, cache, 0, to_dev(q), out, ws, dev_status=st)
    check(out, *one_by_one(Q, K, V, rows, p_bf16=True)[:2], "own rows")
    # the bad row in the prefix, for all sequences
    for j in sorted({0, 63, 64, 127, 128, 129, 300, S - 2, S - 1}):
        if j >= S:
            continue
        bad_k, bad_v = pk[None].copy(), pv[None].copy()
        poison(bad_k, bad_v, q, [j])
        PK, PV = f64(bad_k[0]), f64(bad_v[0])
        prefix = make_cache(bt, bt.make_config(1, H, hd, 4, 1, cap, 1), bad_k, bad_v, [S])
        bt.bt_block_decode_attn_shared(cfg, prefix, cache, 0, to_dev(q), out, ws, dev_status=st)
        check(out, *one_by_one(Q, K, V, rows, p_bf16=True)[:2], f"prefix row {j}")
    assert st.item() == 0


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("N,splits", [(261, 1), (264, 1), (261, 4), (264, 7), (2051, 1)])   # sums by the same launch, and by a second one
def test_sums_visible(bt, hd, step, N, splits):
    """Sums grow by the definition's weights: NaN throughout where a score is NaN or plus infinity, nothing for a score of minus infinity, and
    nothing at all where every score is.  With the step form the appended row is one of few scores that are finite, or is not either."""
    lens = [260, 33, 260, 4, 1, 130, 255, 64, 31, 200, 260, 97]
    B, H = len(lens), 6
    cfg = bt.make_config(B, H, hd, 4, 1, N, 1, decode_splits=splits)
    k, v, q = rnd(64, 1, (B, H, N, hd)), rnd(64, 2, (B, H, N, hd)), rnd(64, 3, (B, H, hd))
    poison(k, v, q, [min(a, n - 1) for a, n in zip(AT, lens)])
    Q = f64(q)
    for b in range(B):   # minus infinity: head 4 in every row, head 5 in the first half of them
        for h, rows in ((4, slice(None)), (5, slice(0, lens[b] // 2))):
            k[b, h, rows, 9] = NEG_INF if Q[b, h, 9] > 0 else INF
    kn, vn = k[:, :, 0].copy(), rnd(64, 4, (B, H, hd))
    kn[::2, 4] = rnd(64, 5, (B, H, hd))[::2, 4]
    kn[:, 0], kn[:, 2] = rnd(64, 6, (B, H, hd))[:, 0], rnd(64, 7, (B, H, hd))[:, 2]
    cache = make_cache(bt, cfg, k, v, lens)
    old = np.random.default_rng(4).random((B, H, N)).astype(np.float32)
    sums = torch.from_numpy(old)[None].cuda()
    out, st, ws = torch.zeros((B, H, hd), dtype=torch.bfloat16, device="cuda"), status_word(), bt.alloc_workspace_weights(cfg)
    n, base = list(lens), old.astype(np.float64)
    if step:
        bt.bt_block_decode_step_weights(cfg, cache, 0, to_dev(q), to_dev(kn), to_dev(vn), out, sums, sums, ws, dev_status=st)
        for b in range(B):
            k[b, :, n[b]], v[b, :, n[b]], base[b, :, n[b]] = kn[b], vn[b], 0.0
            n[b] += 1
    else:
        bt.bt_block_decode_attn_weights(cfg, cache, 0, to_dev(q), out, sums, sums, ws, dev_status=st)
    K, V = f64(k), f64(v)
    ref, tol, weights = one_by_one(Q, K, V, lambda b, h: (K[b, h, :n[b]], V[b, h, :n[b]]))
    check(out, ref, tol, "out")
    got = sums[0].cpu().numpy()
    for (b, h), (p, rel) in weights.items():
        new, g = base[b, h, :n[b]] + p, got[b, h, :n[b]]
        assert np.array_equal(np.isnan(g), np.isnan(new)), (b, h)
        nothing = p == 0                                                      # bit for bit what was there
        assert np.array_equal(g[nothing], base[b, h, :n[b]][nothing].astype(np.float32)), (b, h)
        assert not (np.abs(g - new) > rel * p + ctx.STEP * np.abs(new) + 1e-30).any(), (b, h)
        assert np.array_equal(got[b, h, n[b]:], old[b, h, n[b]:])
    assert st.item() == 0


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window,sinks", [(400, 0), (50, 2), (70, 90)])
@pytest.mark.parametrize("j", [0, 1, 63, 130, 299])
def test_window_prefill_visible(bt, hd, window, sinks, j):
    """Queries that see a bad row, and those that share a tile with it without seeing it."""
    B, H, T = 2, 5, 300
    cfg = bt.make_config(B, H, hd, 4, 1, T, 1)
    q, k, v = (rnd(65, i, (B, H, T, hd)) for i in range(3))
    poison(k, v, q, [j] * B)
    q[:, 4, :, 9] &= 0x7FFF                   # head 4: every score is minus infinity
    q[:, 4, :, 9] |= 0x3F80
    k[:, 4, :, 9] = NEG_INF
    out, st = torch.zeros((B, H, T, hd), dtype=torch.bfloat16, device="cuda"), status_word()
    bt.bt_block_prefill_attn_window(cfg, to_dev(q), to_dev(k), to_dev(v), window, sinks, out, dev_status=st)
    Q, K, V = f64(q), f64(k), f64(v)
    ref, tol = np.zeros((B, H, T, hd)), np.zeros((B, H, T, hd))
    for t in range(T):
        seen = ctx.window_rows(t + 1, window, sinks)
        for b in range(B):
            for h in range(H):
                ref[b, h, t], tol[b, h, t], *_ = attend(Q[b, h, t], K[b, h, seen], V[b, h, seen], p_bf16=True)
    check(out, ref, tol, f"window {window} sinks {sinks} row {j}")
    assert st.item() == 0


def test_window_prefill_long_and_not_finite(bt):
    """A value that every one of many queries sees: all rows of the head are worked out again over up to 131072 keys, for longer than the
    kernel's waits last, and none of them runs out."""
    H, hd, T = 2, 64, 131072
    cfg = bt.make_config(1, H, hd, 4, 1, T, 1)
    q, k, v = (gen.normal_bf16_device(66, i, (1, H, T, hd), device="cuda") for i in range(3))
    clean, out, st = torch.empty_like(q), torch.full_like(q, 7.0), status_word()
    bt.bt_block_prefill_attn_window(cfg, q, k, v, T, 0, clean, dev_status=st)
    v[0, 0, 0, 3] = float("nan")
    bt.bt_block_prefill_attn_window(cfg, q, k, v, T, 0, out, dev_status=st)
    assert st.item() == 0
    assert torch.isnan(out[0, 0, :, 3]).all() and torch.equal(out[0, 1], clean[0, 1])
    others = [i for i in range(hd) if i != 3]
    a, b = out[0, 0][:, others].double(), clean[0, 0][:, others].double()
    # fp32 weights against bf16 ones: 2^-8 of the weighted |v|, which is below 6 everywhere, and a rounding of each result
    assert ((a - b).abs() <= 2.0 ** -8 * 6 + 2.0 ** -7 * b.abs()).all()
