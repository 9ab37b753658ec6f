"""Cases for the block-cache operators of long and shared contexts, with their plain forms.

Five operators over the block KV cache ``[B, H, N_max, hd]`` (bf16, one row per block, ``len[b]`` rows valid):

* ``window_decode``  - one query per (sequence, head) over the first ``sinks`` rows and the last ``window`` rows;
* ``window_prefill`` - all T prompt positions at once under the same rule, counted from each position;
* ``shared_decode``  - one query over a prefix that the whole batch shares, then over the sequence's own rows;
* ``weights_decode`` - one query over the cache, the attention weights added to a running sum per row;
* ``evict``          - keep the first rows, the last rows and those of the largest sums, in order, drop the rest.

With ``own`` false ``run`` computes them with elementary torch operations in fp32; with ``own`` true it calls
the library.
"""
import math

import torch

own = False


# ---------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the smallest call: a few sequences, a 64-row cache; what counts is the latency of one launch
        dict(name="window-tiny", op="window_decode", B=4, H=8, hd=64, N=64, lo=64, hi=64, window=16, sinks=4),
        # ordinary serving: the block-decoder step of a 2048-token context with a quarter of it visible
        dict(name="window-batch", op="window_decode", B=256, H=16, hd=64, N=512, lo=385, hi=512, window=128, sinks=4),
        # a 64K-token context (L_B = 4) on few sequences: the row range of one head has to be split
        dict(name="window-long", op="window_decode", B=16, H=16, hd=128, N=16384, lo=8001, hi=16384, window=4096, sinks=16),
        # prefill of the paper's 2048-token prompts (512 blocks), a quarter of it visible
        dict(name="window-prompt", op="window_prefill", B=32, H=16, hd=128, T=512, window=128, sinks=4),
        # a long prompt of an odd number of blocks
        dict(name="window-prompt-long", op="window_prefill", B=2, H=16, hd=64, T=8191, window=1024, sinks=16),
        # the smallest call: a short system prompt in front of a few short sequences
        dict(name="shared-tiny", op="shared_decode", B=4, H=8, hd=64, S_max=64, S=64, N=64, lo=1, hi=40),
        # many users of one 8K-token instruction, each with a short history
        dict(name="shared-batch", op="shared_decode", B=256, H=16, hd=64, S_max=2048, S=2041, N=128, lo=1, hi=128),
        # the same at a 32K-token document and wide heads; some sequences have nothing of their own yet
        dict(name="shared-long", op="shared_decode", B=512, H=16, hd=128, S_max=8192, S=8000, N=256, lo=0, hi=256),
        # the block-decoder step of a 2048-token context, its weights summed for the eviction below
        dict(name="weights-batch", op="weights_decode", B=256, H=16, hd=64, N=512, lo=385, hi=512),
        # few sequences of a long context: the row range is split, so are the weights
        dict(name="weights-long", op="weights_decode", B=4, H=16, hd=128, N=16384, lo=12001, hi=16384),
        # the cache of the 2048-token context cut to half; the shortest sequences are left whole
        dict(name="evict-batch", op="evict", B=256, H=16, hd=64, N=512, lo=240, hi=512, keep=256, sinks=4, recent=64),
        # a long prompt's cache cut to a quarter, few sequences
        dict(name="evict-long", op="evict", B=4, H=16, hd=128, N=16384, lo=12001, hi=16384, keep=4096, sinks=16, recent=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["window_decode", "window_prefill", "shared_decode", "weights_decode", "evict"])
    hd = rng.choice([64, 128])
    H = rng.randint(1, 16)
    if op == "window_prefill":
        T = _log(rng, 1, 8191)
        most = max(1, min(64, int(2.5e8 // (T * max(T, 64) * H))))
        return dict(op=op, B=_log(rng, 1, most) if most > 1 else 1, H=H if T < 4096 else min(H, 8), hd=hd, T=T,
                    window=_log(rng, 1, T), sinks=rng.choice([0, 1, 4, 16, rng.randint(0, 200)]))
    if op == "shared_decode":
        S_max = _log(rng, 8, 8192)
        N = _log(rng, 1, 512)
        B = max(1, min(_log(rng, 1, 512), int(2.0e9 // (H * N * hd * 4)), int(6.4e7 // (H * S_max))))
        S = S_max - rng.randint(0, min(S_max, 100))
        lo = rng.randint(0, N)
        return dict(op=op, B=B, H=H, hd=hd, S_max=S_max, S=S, N=N, lo=lo, hi=rng.randint(lo, N))
    N = _log(rng, 16, 16384)
    B = max(1, min(_log(rng, 1, 256), int(4.0e8 // (H * N * hd * 4))))
    lo = rng.randint(N // 2, N)
    hi = rng.randint(lo, N)
    if op == "window_decode":
        return dict(op=op, B=B, H=H, hd=hd, N=N, lo=lo, hi=hi, window=_log(rng, 1, N), sinks=rng.choice([0, 1, 4, rng.randint(0, 64)]))
    if op == "weights_decode":
        return dict(op=op, B=B, H=H, hd=hd, N=N, lo=lo, hi=hi)
    keep = rng.randint(max(1, N // 8), max(1, (3 * N) // 4))
    sinks = rng.randint(0, min(16, keep))
    return dict(op=op, B=B, H=H, hd=hd, N=N, lo=lo, hi=N, keep=keep, sinks=sinks, recent=rng.randint(0, keep - sinks))


def _lens(c):
    """The valid rows of each sequence: spread over lo..hi, the longest first."""
    span = c["hi"] - c["lo"] + 1
    return [c["hi"] - (b * 7919) % span for b in range(c["B"])]


# ---------------------------------------------------------------------------------------------- inputs

def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _normal_big(g, *shape):
    """The same, made slab by slab: a cache of gigabytes needs no fp32 copy of itself."""
    t = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    for part in t:
        part.copy_(torch.randn(part.shape, generator=g, device="cuda", dtype=torch.float32))
    return t


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = {"c": c}
    if c["op"] == "window_prefill":
        shape = (c["B"], c["H"], c["T"], c["hd"])
        s["q"], s["k"], s["v"] = _normal(g, *shape), _normal(g, *shape), _normal(g, *shape)
    else:
        s["k"] = _normal_big(g, c["B"], c["H"], c["N"], c["hd"])
        s["v"] = _normal_big(g, c["B"], c["H"], c["N"], c["hd"])
        s["len"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda")
        if c["op"] != "evict":
            s["q"] = _normal(g, c["B"], c["H"], c["hd"])
    if c["op"] == "shared_decode":
        s["pk"], s["pv"] = _normal(g, c["H"], c["S_max"], c["hd"]), _normal(g, c["H"], c["S_max"], c["hd"])
        s["plen"] = torch.full((1,), c["S"], dtype=torch.int32, device="cuda")
    if c["op"] in ("weights_decode", "evict"):
        # sums of many softmax rows: non-negative, a few heavy rows, most of them light; nothing past the length
        w = torch.rand((c["B"], c["H"], c["N"]), generator=g, device="cuda").pow_(8).mul_(20.0)
        s["w"] = w * (torch.arange(c["N"], device="cuda") < s["len"][:, None, None])
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """The handles that a user's program keeps: configuration, cache objects, workspace, output buffers."""
    import paper_2406_02657_b200 as bt

    c = s["c"]
    s["bt"] = bt
    if c["op"] == "window_prefill":
        s["cfg"] = bt.make_config(c["B"], c["H"], c["hd"], 4, 1, c["T"], 1)
        s["out"] = torch.empty_like(s["q"])
        return
    cfg = s["cfg"] = bt.make_config(c["B"], c["H"], c["hd"], 4, 1, c["N"], 1)
    s["cache"] = bt.BlockCache(cfg, k=s["k"][None], v=s["v"][None], length=s["len"][None])
    if c["op"] != "evict":
        s["out"] = torch.empty_like(s["q"])
    if c["op"] == "shared_decode":
        pcfg = bt.make_config(1, c["H"], c["hd"], 4, 1, c["S_max"], 1)
        s["prefix"] = bt.BlockCache(pcfg, k=s["pk"][None, None], v=s["pv"][None, None], length=s["plen"][None])
        s["ws"] = bt.alloc_workspace_shared(cfg, c["S_max"])
    elif c["op"] == "weights_decode":
        s["w_out"] = torch.zeros_like(s["w"])
        s["ws"] = bt.alloc_workspace_weights(cfg)
    elif c["op"] == "evict":
        s["dst"] = bt.BlockCache(bt.make_config(c["B"], c["H"], c["hd"], 4, 1, c["keep"], 1))
        s["dst_w"] = torch.zeros((c["B"], c["H"], c["keep"]), dtype=torch.float32, device="cuda")
        s["kept"] = torch.empty((c["B"], c["H"], c["keep"]), dtype=torch.int32, device="cuda")
        s["ws"] = bt.alloc_workspace(cfg)
    else:
        s["ws"] = bt.alloc_workspace(cfg)


# ---------------------------------------------------------------------------------------------- one pass

def run(s):
    return _run_own(s) if own else _PLAIN[s["c"]["op"]](s)


def _run_own(s):
    bt, c = s["bt"], s["c"]
    op = c["op"]
    if op == "window_prefill":
        bt.bt_block_prefill_attn_window(s["cfg"], s["q"], s["k"], s["v"], c["window"], c["sinks"], s["out"])
        return s["out"]
    if op == "window_decode":
        bt.bt_block_decode_attn_window(s["cfg"], s["cache"], 0, s["q"], c["window"], c["sinks"], s["out"], s["ws"])
        return s["out"]
    if op == "shared_decode":
        bt.bt_block_decode_attn_shared(s["cfg"], s["prefix"], s["cache"], 0, s["q"], s["out"], s["ws"])
        return s["out"]
    if op == "weights_decode":
        bt.bt_block_decode_attn_weights(s["cfg"], s["cache"], 0, s["q"], s["out"], s["w"], s["w_out"], s["ws"])
        return {"out": s["out"], "weights": s["w_out"]}
    bt.bt_block_kv_evict(s["cfg"], s["cache"], s["w"], 0, c["keep"], c["sinks"], c["recent"], s["ws"], dst=s["dst"],
                         dst_weights=s["dst_w"], kept=s["kept"])
    return {"k": s["dst"].k[0], "v": s["dst"].v[0], "weights": s["dst_w"], "len": s["dst"].len[0], "kept": s["kept"]}


def _softmax(scores, visible):
    """exp(s - max) / sum over the visible entries of the last axis, in fp32; a row with none is all zeros."""
    scores = scores.masked_fill(~visible, float("-inf"))
    m = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - m.masked_fill(m == float("-inf"), 0.0))
    total = e.sum(-1, keepdim=True)
    return e / total.masked_fill(total == 0, 1.0)


def _plain_window_decode(s):
    c, q, k, v = s["c"], s["q"].float(), s["k"], s["v"]
    n = s["len"].long()[:, None]
    most = min(c["N"], c["window"] + c["sinks"])
    r = torch.arange(most, device="cuda")[None]
    first = n.clamp(max=c["sinks"])                             # rows visible as sinks
    at = torch.where(r < first, r, r - first + torch.maximum(n - c["window"], first))
    seen = at < n
    at = at.clamp(max=c["N"] - 1)[:, None, :, None].expand(-1, c["H"], -1, c["hd"])
    kk, vv = k.gather(2, at).float(), v.gather(2, at).float()
    p = _softmax(torch.einsum("bhd,bhnd->bhn", q, kk) / math.sqrt(c["hd"]), seen[:, None])
    return torch.einsum("bhn,bhnd->bhd", p, vv).to(torch.bfloat16)


def _plain_window_prefill(s):
    c = s["c"]
    T, hd = c["T"], c["hd"]
    q, k, v = (s[x].reshape(-1, T, hd) for x in "qkv")
    out = torch.empty_like(q)
    slabs = max(1, int(2.5e8 // (T * T)))
    i = torch.arange(T, device="cuda")
    seen = (i[None] <= i[:, None]) & ((i[None] > i[:, None] - c["window"]) | (i[None] < c["sinks"]))
    for a in range(0, q.shape[0], slabs):
        qq, kk, vv = (x[a:a + slabs].float() for x in (q, k, v))
        p = _softmax(torch.einsum("std,sjd->stj", qq, kk) / math.sqrt(hd), seen)
        out[a:a + slabs] = torch.einsum("stj,sjd->std", p, vv).to(torch.bfloat16)
    return out.reshape(s["q"].shape)


def _plain_shared_decode(s):
    c, q = s["c"], s["q"].float()
    scale = 1.0 / math.sqrt(c["hd"])
    B, H, S, N = c["B"], c["H"], c["S_max"], c["N"]
    scores = torch.cat([torch.einsum("bhd,hsd->bhs", q, s["pk"].float()),
                        torch.einsum("bhd,bhnd->bhn", q, s["k"].float())], -1) * scale
    seen = torch.cat([(torch.arange(S, device="cuda") < s["plen"])[None].expand(B, S),
                      torch.arange(N, device="cuda")[None] < s["len"][:, None]], -1)
    p = _softmax(scores, seen[:, None])
    out = torch.einsum("bhs,hsd->bhd", p[..., :S], s["pv"].float()) + torch.einsum("bhn,bhnd->bhd", p[..., S:], s["v"].float())
    return out.to(torch.bfloat16)


def _plain_weights_decode(s):
    c, q = s["c"], s["q"].float()
    seen = torch.arange(c["N"], device="cuda")[None] < s["len"][:, None]
    p = _softmax(torch.einsum("bhd,bhnd->bhn", q, s["k"].float()) / math.sqrt(c["hd"]), seen[:, None])
    out = torch.einsum("bhn,bhnd->bhd", p, s["v"].float()).to(torch.bfloat16)
    return {"out": out, "weights": s["w"] + p}


def _plain_evict(s):
    c = s["c"]
    B, H, N, keep = c["B"], c["H"], c["N"], c["keep"]
    n = s["len"].long()[:, None, None]
    j = torch.arange(N, device="cuda")
    # one number per row to sort by: kept whatever their sum, by their sum, not there
    rank = torch.where((j < c["sinks"]) | (j >= n - c["recent"]), float("inf"), s["w"]).masked_fill(j >= n, float("-inf"))
    best = rank.sort(dim=-1, descending=True, stable=True).indices[..., :keep].sort(dim=-1).values   # ties: the lowest index
    cut = n > keep
    at = torch.where(cut, best, torch.arange(keep, device="cuda"))
    there = torch.arange(keep, device="cuda") < n
    rows = at[..., None].expand(-1, -1, -1, c["hd"])
    k = s["k"].gather(2, rows).masked_fill(~there[..., None], 0)
    v = s["v"].gather(2, rows).masked_fill(~there[..., None], 0)
    w = s["w"].gather(2, at).masked_fill(~there, 0.0)
    kept = torch.where(cut, at, -1).to(torch.int32)
    return {"k": k, "v": v, "weights": w, "len": s["len"].clamp(max=keep), "kept": kept}


_PLAIN = {"window_decode": _plain_window_decode, "window_prefill": _plain_window_prefill, "shared_decode": _plain_shared_decode,
          "weights_decode": _plain_weights_decode, "evict": _plain_evict}


# ---------------------------------------------------------------------------------------------- the definition, in 64 bits

def _attend(q, keys, values):
    """One query per row of q [H, hd] over keys, values [H, n, hd]: outputs and weights."""
    if keys.shape[1] == 0:
        return torch.zeros_like(q), q.new_zeros(q.shape[0], 0)
    a = (keys @ q[:, :, None])[..., 0] / math.sqrt(q.shape[-1])
    a = torch.exp(a - a.max(1, keepdim=True).values)
    a = a / a.sum(1, keepdim=True)
    return (a[:, None, :] @ values)[:, 0], a


def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    if c["op"] == "evict":
        return _exact_evict(c, s)
    if c["op"] == "window_prefill":
        T, hd = c["T"], c["hd"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        step = max(1, int(2e7 // T))                            # query rows at a time
        for b in range(c["B"]):
            for t0 in range(0, T, step):
                t1 = min(T, t0 + step)
                first = max(c["sinks"], t0 - c["window"] + 1)
                cols = torch.cat([torch.arange(min(c["sinks"], t1)), torch.arange(first, t1)]).cuda() if first < t1 else torch.arange(min(c["sinks"], t1)).cuda()
                t = torch.arange(t0, t1, device="cuda")[:, None]
                hidden = (cols > t) | ((cols <= t - c["window"]) & (cols >= c["sinks"]))
                for h in range(c["H"]):
                    a = s["q"][b, h, t0:t1].double() @ s["k"][b, h, cols].double().T / math.sqrt(hd)
                    a[hidden] = -float("inf")
                    a = torch.exp(a - a.max(1, keepdim=True).values)
                    out[b, h, t0:t1] = a @ s["v"][b, h, cols].double() / a.sum(1, keepdim=True)
        return out
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    weights = s["w"].double() if c["op"] == "weights_decode" else None
    if c["op"] == "shared_decode":
        pk, pv = s["pk"][:, :c["S"]].double(), s["pv"][:, :c["S"]].double()
    for b, n in enumerate(_lens(c)):
        k, v = s["k"][b, :, :n].double(), s["v"][b, :, :n].double()
        if c["op"] == "window_decode":
            rows = [j for j in range(n) if j < c["sinks"] or j >= n - c["window"]]
            k, v = k[:, rows], v[:, rows]
        elif c["op"] == "shared_decode":
            k, v = torch.cat([pk, k], 1), torch.cat([pv, v], 1)
        out[b], a = _attend(s["q"][b].double(), k, v)
        if weights is not None:
            weights[b, :, :n] += a
    return out if weights is None else {"out": out, "weights": weights}


def _exact_evict(c, s):
    """By a threshold instead of a sort: every sum above the last one kept, then the first ones equal to it."""
    keep, free = c["keep"], c["keep"] - c["sinks"] - c["recent"]
    k, v = (torch.zeros((c["B"], c["H"], keep, c["hd"]), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = torch.zeros((c["B"], c["H"], keep), device="cuda")
    kept = torch.full((c["B"], c["H"], keep), -1, dtype=torch.int32, device="cuda")
    lens = _lens(c)
    for b, n in enumerate(lens):
        if n <= keep:
            k[b, :, :n], v[b, :, :n], w[b, :, :n] = s["k"][b, :, :n], s["v"][b, :, :n], s["w"][b, :, :n]
            continue
        middle = s["w"][b, :, c["sinks"]:n - c["recent"]]
        take = torch.zeros((c["H"], n), dtype=torch.bool, device="cuda")
        take[:, :c["sinks"]] = True
        take[:, n - c["recent"]:] = True
        if free > 0:
            least = middle.kthvalue(middle.shape[1] - free + 1, dim=1, keepdim=True).values
            above, equal = middle > least, middle == least
            take[:, c["sinks"]:n - c["recent"]] |= above | (equal & (equal.cumsum(1) <= free - above.sum(1, keepdim=True)))
        for h in range(c["H"]):
            rows = take[h].nonzero()[:, 0]
            k[b, h], v[b, h], w[b, h], kept[b, h] = s["k"][b, h, rows], s["v"][b, h, rows], s["w"][b, h, rows], rows.int()
    return {"k": k, "v": v, "weights": w, "len": torch.tensor([min(n, keep) for n in lens], dtype=torch.int32, device="cuda"), "kept": kept}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Bytes: each visible row of K and V once, queries, outputs, sums and lengths once.  Flops: the two products."""
    c = dict(case)
    row = 2 * c["hd"] * 2                                       # one row of K and one of V
    bh = c["B"] * c["H"]
    if c["op"] == "window_prefill":
        T, w, sk = c["T"], c["window"], c["sinks"]
        pairs = sum(min(t + 1, w) + min(sk, max(0, t + 1 - w)) for t in range(T))
        return {"bytes": 4 * bh * T * c["hd"] * 2, "flops": 4 * bh * c["hd"] * pairs}
    lens = _lens(c)
    qo = 2 * bh * c["hd"] * 2
    if c["op"] == "evict":
        rows = sum(min(n, c["keep"]) for n in lens) * c["H"]
        sums = sum(n for n in lens if n > c["keep"]) * c["H"] * 4
        return {"bytes": 2 * rows * row + sums + 4 * rows + 4 * bh * c["keep"] + 8 * c["B"], "flops": 0}
    if c["op"] == "window_decode":
        rows = sum(min(n, c["window"] + c["sinks"]) for n in lens) * c["H"]
        return {"bytes": rows * row + qo + 4 * c["B"], "flops": 4 * rows * c["hd"]}
    rows = sum(lens) * c["H"]
    if c["op"] == "shared_decode":
        return {"bytes": (rows + c["H"] * c["S"]) * row + qo + 4 * c["B"] + 4, "flops": 4 * (rows + bh * c["S"]) * c["hd"]}
    return {"bytes": rows * (row + 8) + qo + 4 * c["B"], "flops": 4 * rows * c["hd"]}
