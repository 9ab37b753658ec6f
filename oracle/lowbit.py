"""Plain float64 definitions of the low-bit operators (numpy only): rows quantised to 4 and to 8 bits, the tiles of the 4-bit block
cache, attention over it and the projections of 8-bit integers, with bounds on the rounding error of an implementation that
computes them in fp32 (see contexts).
"""
import numpy as np

from workloads import gen

from . import contexts as ctx

TILE_ROWS, TILE_BYTES = 16, 1152
LEAST_STEP = 2.0 ** -126


def to_bf16(x):
    """float64 -> the nearest bf16 value, ties to even, as float64."""
    return gen.bf16_bits_to_f32(gen.f32_to_bf16_bits(np.asarray(x, np.float32))).astype(np.float64)


def quantised(x, most):
    """x float64 [..., width] -> codes int [..., width], steps float64 [...] of the groups along the last axis."""
    fine = np.isfinite(x).all(-1)
    top = np.where(fine, np.abs(np.where(np.isfinite(x), x, 0.0)).max(-1, initial=0.0), 0.0)
    steps = to_bf16(top / most)
    steps = np.where(steps < LEAST_STEP, 0.0, steps)
    some = (steps > 0) & fine
    ratio = np.abs(np.where(some[..., None], x, 0.0)) / np.where(some, steps, 1.0)[..., None]
    codes = (np.floor(ratio + 0.5) * np.sign(np.where(some[..., None], x, 0.0))).astype(np.int64)
    assert np.abs(codes).max(initial=0) <= most
    return codes, np.where(fine, steps, np.nan)


def kv4(x):
    """Rows [..., hd] -> codes [..., hd], steps [..., hd/32]."""
    codes, steps = quantised(x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32), 7)
    return codes.reshape(x.shape), steps


def kv4_values(codes, steps):
    with np.errstate(invalid="ignore"):
        return (codes.reshape(*steps.shape, 32) * steps[..., None]).reshape(codes.shape)


def held(x):
    """What rows [..., hd] are in the 4-bit cache."""
    return kv4_values(*kv4(x))


def step_bits(steps):
    bits = gen.f32_to_bf16_bits(np.where(np.isnan(steps), 0.0, steps).astype(np.float32))
    return np.where(np.isnan(steps), 0x7FFF, bits).astype(np.uint16)


def k_byte(row, pair):
    """Where the codes of dimensions 2 pair, 2 pair + 1 of K of a row lie in a tile (row, pair within it)."""
    return row // 2 * 64 + pair // 8 * 16 + row % 2 * 8 + pair % 8


def v_byte(row, pair):
    quad, unit, word = row // 4, pair // 4, pair % 4
    return 512 + quad * 128 + (unit ^ 2 * quad) * 16 + word * 4 + row % 4


def write_tiles(tiles, row0, k, v):
    """Rows k, v [n, hd] (float64) written into the tiles [ceil(N/16), hd/64, 1152] of one (sequence, head), from row0 on."""
    hd = k.shape[1]
    for part, (x, byte) in enumerate(((k, k_byte), (v, v_byte))):
        codes, steps = kv4(x)
        nib = (codes + 8).astype(np.uint8)
        nib = nib[:, 0::2] | (nib[:, 1::2] << 4)
        bits = step_bits(steps)
        for i in range(x.shape[0]):
            t, r = divmod(row0 + i, TILE_ROWS)
            for p in range(hd // 64):
                tiles[t, p, [byte(r, j) for j in range(32)]] = nib[i, p * 32: p * 32 + 32]
                at = 1024 + part * 64 + r * 4
                tiles[t, p, at: at + 4] = bits[i, 2 * p: 2 * p + 2].view(np.uint8)


def decode(q, K, V, n):
    """q [B,H,hd], K, V [B,H,N,hd] as held, n [B]: (out, tol).  Beside what contexts.attend allows: the query is rounded to whole
    numbers, by 2^-18 of the largest value of its group of 32 dimensions at most (a score error of e moves a weight by a factor within exp(+-e), in numerator and
    denominator), and so are the products of a weight and a step of V, by 2^-29 of the largest one of their group of 32 dimensions, for a
    code of up to 7."""
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(q.shape[0]):
        for h in range(q.shape[1]):
            k, v = K[b, h, :n[b]], V[b, h, :n[b]]
            o, p, e, _ = ctx.attend(q[b, h], k, v)
            if n[b]:
                sizes = np.abs(k).reshape(n[b], -1, 32).sum(2) @ np.abs(q[b, h]).reshape(-1, 32).max(1)
                score = sizes.max() * 2.0 ** -18 / np.sqrt(q.shape[2])
                largest = (p[:, None] * np.abs(v)).max(0).reshape(-1, 32).max(1)
                e += 2 * score * (p @ np.abs(v)) + n[b] * 2.0 ** -29 * 1.01 * np.repeat(largest, 32)
            out[b, h], tol[b, h] = o, e
    return out, tol


def project(x8, x_steps, w8, w_steps, bias):
    """x8 [M,K], w8 [N,K]: y [M,N] before its rounding, and a bound on what fp32 and the rounding to bf16 may add."""
    acc = (x8.astype(np.float64) @ w8.astype(np.float64).T)   # whole numbers, exact
    y = acc * (x_steps[:, None] * w_steps[None])
    b = np.zeros(w8.shape[0]) if bias is None else bias
    # the sum to fp32, the steps' product, the product of both, the bias: a half step of fp32 each (2^-24)
    tol = 4 * 2.0 ** -24 * (np.abs(y) + np.abs(b))
    y = y + b
    return y, tol + ctx.BF16 * (np.abs(y) + tol) + 1e-38
