"""Cases for the block decoder's low-bit operators, with their plain forms.

Three operators:

* ``kv4_write``  - new K,V rows quantised to 4 bits into the block cache, then the valid rows read back as bf16;
* ``kv4_decode`` - one query per (sequence, head) over a block cache held in 4 bits;
* ``project_i8`` - activations quantised to 8 bits (a scale per token), multiplied with 8-bit weights (a scale per output
  channel): the prefix projection, and the QKV projection into the local or the block cache.

The 4-bit form of a row: for every 32 dimensions a step ``s = bf16(max|x| / 7)`` and codes ``u = round(x / s)``, halves away
from zero, ``-7 <= u <= 7``; the value held is ``s u``.  The 8-bit form of a row: ``s = bf16(max|x| / 127)``,
``u = round(x / s)`` likewise.  Both quotients are of numbers of 8 significant bits, so that 32 bits decide every rounding as
64 bits would.

With ``own`` false ``run`` computes them with elementary torch operations in fp32; with ``own`` true it calls the library.
"""
import math

import torch

own = False


# ---------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the smallest call: the first block of a few sequences; what counts is the latency of a launch
        dict(name="write-tiny", op="kv4_write", B=4, H=8, hd=64, N=64, n=1, lo=0, hi=0),
        # prompts of 2048 tokens (512 blocks) cached for a batch, and read back for the prompt's own attention
        dict(name="write-prompt", op="kv4_write", B=32, H=16, hd=128, N=512, n=512, lo=0, hi=0),
        # a second turn of odd length behind histories of different lengths
        dict(name="write-turn", op="kv4_write", B=13, H=7, hd=64, N=1501, n=487, lo=0, hi=1001),
        # the smallest call: a few sequences, a 64-row cache
        dict(name="decode-tiny", op="kv4_decode", B=4, H=8, hd=64, N=64, lo=64, hi=64),
        # ordinary serving: the block-decoder step of a 2048-token context
        dict(name="decode-batch", op="kv4_decode", B=256, H=16, hd=64, N=512, lo=385, hi=512),
        # few sequences of a 64K-token context: the row range of one head has to be split
        dict(name="decode-long", op="kv4_decode", B=4, H=16, hd=128, N=16384, lo=12001, hi=16384),
        # long contexts in a batch: the cache is gigabytes, what counts is the rate at which it is read
        dict(name="decode-large", op="kv4_decode", B=24, H=16, hd=128, N=16000, lo=12001, hi=16000),
        # prefix projection of a few sequences
        dict(name="prefix-tiny", op="project_i8", kind="prefix", B=4, H=8, hd=64, P=1, n=1, N=1, lo=0, hi=0),
        # prefix projection of a full batch of the token decoder
        dict(name="prefix-batch", op="project_i8", kind="prefix", B=4096, H=16, hd=64, P=2, n=1, N=1, lo=0, hi=0),
        # one token step of the token decoder at model dim 2048, at a block boundary
        dict(name="qkv-token", op="project_i8", kind="local", B=4096, H=16, hd=128, P=1, n=1, N=1, lo=0, hi=0),
        # a few rows for every sequence of an odd batch, behind the rows that it has
        dict(name="qkv-rows", op="project_i8", kind="block", B=250, H=9, hd=64, P=1, n=3, N=77, lo=0, hi=74),
        # the QKV projection of prompts of 512 blocks at model dim 2048
        dict(name="qkv-prompt", op="project_i8", kind="block", B=32, H=16, hd=128, P=1, n=512, N=512, lo=0, hi=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) if hi > lo else lo


def draw(rng):
    op = rng.choice(["kv4_write", "kv4_decode", "project_i8"])
    hd = rng.choice([64, 128])
    H = rng.randint(1, 16)
    if op == "kv4_write":
        n = _log(rng, 1, 2048)
        lo = rng.choice([0, rng.randint(0, 700)])
        hi = lo if lo == 0 else rng.randint(lo, lo + 300)
        N = n + hi + rng.randint(0, 40)
        B = max(1, min(_log(rng, 1, 64), 33000000 // (H * N * hd)))
        return dict(op=op, B=B, H=H, hd=hd, N=N, n=n, lo=lo, hi=hi)
    if op == "kv4_decode":
        N = _log(rng, 16, 16384)
        B = max(1, min(_log(rng, 1, 256), 200000000 // (H * N * hd)))
        lo = rng.choice([0, rng.randint(N // 2, N)])
        return dict(op=op, B=B, H=H, hd=hd, N=N, lo=lo, hi=rng.randint(max(lo, N // 2), N))
    kind = rng.choice(["prefix", "local", "block"])
    B = _log(rng, 1, 4096)
    P = rng.randint(1, 4)
    if kind != "block":
        return dict(op=op, kind=kind, B=B, H=H, hd=hd, P=P, n=1 if kind == "prefix" else rng.randint(1, P), N=1, lo=0, hi=0)
    n = _log(rng, 1, max(1, min(512, 16384 // B)))
    hi = rng.choice([0, rng.randint(0, 30)])
    return dict(op=op, kind=kind, B=B, H=H, hd=hd, P=P, n=n, N=n + hi + rng.randint(0, 5), lo=0, hi=hi)


def _lens(c):
    """The rows each sequence has before the call: spread over lo..hi, the longest first."""
    span = c["hi"] - c["lo"] + 1
    return [c["hi"] - (b * 7919) % span for b in range(c["B"])]


# ---------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _channels(g, *shape):
    """Channels of unlike size, as keys and activations have them."""
    return torch.exp(0.5 * _normal(g, *shape))


def _rows(g, c, n, spread):
    """bf16 rows [B,H,n,hd], made sequence by sequence (a long cache needs no fp32 copy of itself)."""
    size = _channels(g, c["H"], 1, c["hd"]) if spread else torch.ones(1, device="cuda")
    t = torch.empty((c["B"], c["H"], n, c["hd"]), dtype=torch.bfloat16, device="cuda")
    for part in t:
        part.copy_(_normal(g, *part.shape) * size)
    return t


def prepare(case, seed):
    c = dict(case)
    g = _generator(seed)
    s = {"c": c, "len0": torch.tensor(_lens(c), dtype=torch.int32, device="cuda")}
    if c["op"] == "project_i8":
        return _prepare_project(s, g)
    if c["op"] == "kv4_write":
        s["k_new"], s["v_new"] = _rows(g, c, c["n"], True), _rows(g, c, c["n"], False)
    else:
        s["q"] = _normal(g, c["B"], c["H"], c["hd"]).to(torch.bfloat16)
    # the rows that the cache already holds
    have = c["hi"]
    k, v = _rows(g, c, have, True), _rows(g, c, have, False)
    if own:
        return _prepare_own_cache(s, k, v)
    s["k"], s["ks"] = _held(k, c["N"])
    s["v"], s["vs"] = _held(v, c["N"])
    return s


def _held(x, N):
    """Rows quantised a sequence at a time: packed codes [B,H,N,hd/2] and steps [B,H,N,hd/32]; rows past x are zeros."""
    B, H, n, hd = x.shape
    codes = torch.zeros((B, H, N, hd // 2), dtype=torch.uint8, device="cuda")
    steps = torch.zeros((B, H, N, hd // 32), dtype=torch.bfloat16, device="cuda")
    for b in range(B if n else 0):
        u, step = _quantise(x[b].reshape(H, n, hd // 32, 32), 7.0)
        codes[b, :, :n] = _pack(u.reshape(H, n, hd))
        steps[b, :, :n] = step[..., 0]
    return codes, steps


def _prepare_own_cache(s, k, v):
    """The library's cache with the same rows, its workspace and output buffers."""
    import paper_2406_02657_b200 as bt

    c = s["c"]
    s["bt"] = bt
    cfg = s["cfg"] = bt.make_config(c["B"], c["H"], c["hd"], 4, 1, c["N"], 1)
    s["cache"] = bt.BlockCacheKV4(cfg)
    if c["hi"]:
        bt.bt_block_kv4_append(cfg, s["cache"], 0, k, v, reset_first=True)
    s["cache"].len[0].copy_(s["len0"])
    if c["op"] == "kv4_decode":
        s["ws"] = bt.alloc_workspace_kv4(cfg)
        s["out"] = torch.empty_like(s["q"])
    else:
        s["k_out"], s["v_out"] = (torch.zeros((c["B"], c["H"], c["N"], c["hd"]), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return s


def _prepare_project(s, g):
    c = s["c"]
    D = c["H"] * c["hd"]
    features = D * (c["P"] if c["kind"] == "prefix" else 3)
    s["x"] = (_normal(g, c["B"], c["n"], D) * _channels(g, D)).to(torch.bfloat16)
    s["w8"], ws = _quantise(_normal(g, features, D) / math.sqrt(D), 127.0)
    s["w8"], s["ws"] = s["w8"].to(torch.int8), ws[:, 0].contiguous()
    s["bias"] = (0.1 * _normal(g, features)).to(torch.bfloat16)
    cap = c["N"] if c["kind"] == "block" else c["P"] + 4
    if own:
        import paper_2406_02657_b200 as bt

        s["bt"] = bt
        cfg = s["cfg"] = bt.make_config(c["B"], c["H"], c["hd"], 4, c["P"], c["N"], 1)
        s["x8"] = torch.empty(s["x"].shape, dtype=torch.int8, device="cuda")
        s["xs"] = torch.empty(s["x"].shape[:2], device="cuda")
        if c["kind"] == "prefix":
            s["out"] = torch.empty((c["B"], c["P"], D), dtype=torch.bfloat16, device="cuda")
            return s
        s["q_out"] = torch.empty((c["B"], c["H"], c["n"], c["hd"]), dtype=torch.bfloat16, device="cuda")
        s["cache"] = bt.LocalCache(cfg) if c["kind"] == "local" else bt.BlockCache(cfg)
    elif c["kind"] == "local":
        s["kv"] = torch.zeros((c["B"], c["H"], cap, 2, c["hd"]), dtype=torch.bfloat16, device="cuda")
    elif c["kind"] == "block":
        s["k"], s["v"] = (torch.zeros((c["B"], c["H"], cap, c["hd"]), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return s


# ---------------------------------------------------------------------------------------------- one pass

def run(s):
    return _OWN[s["c"]["op"]](s) if own else _PLAIN[s["c"]["op"]](s)


def _own_write(s):
    bt, c = s["bt"], s["c"]
    if c["hi"]:                                # every pass appends to the lengths that the state began with
        s["cache"].len[0].copy_(s["len0"])
    bt.bt_block_kv4_append(s["cfg"], s["cache"], 0, s["k_new"], s["v_new"], reset_first=not c["hi"])
    bt.bt_block_kv4_read(s["cfg"], s["cache"], 0, s["k_out"], s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"], "len": s["cache"].len[0]}


def _own_decode(s):
    s["bt"].bt_block_decode_attn_kv4(s["cfg"], s["cache"], 0, s["q"], s["out"], s["ws"])
    return s["out"]


def _own_project(s):
    bt, c, cfg = s["bt"], s["c"], s["cfg"]
    bt.bt_rows_quantize_i8(s["x"], s["x8"], s["xs"])
    if c["kind"] == "prefix":
        bt.bt_prefix_project_i8(cfg, s["x8"], s["xs"], s["w8"], s["ws"], s["bias"], s["out"])
        return s["out"]
    if c["kind"] == "local":
        bt.bt_local_qkv_project_append_i8(cfg, s["cache"], 0, s["x8"], s["xs"], s["w8"], s["ws"], s["bias"], s["q_out"], reset_first=True)
        return {"q": s["q_out"], "kv": s["cache"].kv[0], "len": s["cache"].len[0]}
    s["cache"].len[0].copy_(s["len0"])         # every pass appends to the lengths that the state began with
    bt.bt_block_qkv_project_append_i8(cfg, s["cache"], 0, s["x8"], s["xs"], s["w8"], s["ws"], s["bias"], s["q_out"])
    return {"q": s["q_out"], "k": s["cache"].k[0], "v": s["cache"].v[0], "len": s["cache"].len[0]}


_OWN = {"kv4_write": _own_write, "kv4_decode": _own_decode, "project_i8": _own_project}


def _quantise(x, most):
    """Codes (whole numbers in fp32) and steps (fp32 values of bf16) of the groups along the last axis."""
    x = x.float()
    step = (x.abs().amax(-1, keepdim=True) / most).to(torch.bfloat16).float()
    u = torch.floor(x.abs() / step.masked_fill(step == 0, 1.0) + 0.5).clamp(max=most) * torch.sign(x)
    return u, step


def _pack(u):
    """Codes -7..7 as two to a byte, the even dimension in the low half, 8 added."""
    u = (u + 8).to(torch.uint8)
    return u[..., 0::2] | (u[..., 1::2] << 4)


def _values(codes, steps):
    """The fp32 values of packed codes [..., hd/2] under steps [..., hd/32]."""
    u = torch.stack([codes & 15, codes >> 4], -1).float() - 8.0
    return (u.reshape(*steps.shape, 32) * steps.float()[..., None]).reshape(*codes.shape[:-1], -1)


def _plain_write(s):
    c = s["c"]
    B, H, n, hd = s["k_new"].shape
    at = (s["len0"].long()[:, None] + torch.arange(n, device="cuda"))[:, None, :, None].expand(B, H, n, 1)
    seen = (torch.arange(c["N"], device="cuda") < s["len0"][:, None] + n)[:, None, :, None]
    out = {"len": s["len0"] + n}
    _into(s, "k", at, hd)
    _into(s, "v", at, hd)
    out["k"] = _values(s["k"], s["ks"]).masked_fill(~seen, 0.0).to(torch.bfloat16)
    out["v"] = _values(s["v"], s["vs"]).masked_fill(~seen, 0.0).to(torch.bfloat16)
    return out


def _into(s, name, at, hd):
    u, step = _quantise(s[name + "_new"].unflatten(-1, (hd // 32, 32)), 7.0)
    s[name].scatter_(2, at.expand(-1, -1, -1, hd // 2), _pack(u.flatten(-2)))
    s[name + "s"].scatter_(2, at.expand(-1, -1, -1, hd // 32), step[..., 0].to(torch.bfloat16))


def _plain_decode(s):
    c = s["c"]
    scores = torch.einsum("bhd,bhnd->bhn", s["q"].float(), _values(s["k"], s["ks"])) / math.sqrt(c["hd"])
    seen = (torch.arange(c["N"], device="cuda") < s["len0"][:, None])[:, None]
    scores = scores.masked_fill(~seen, float("-inf"))
    m = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - m.masked_fill(m == float("-inf"), 0.0))
    total = e.sum(-1, keepdim=True)
    p = e / total.masked_fill(total == 0, 1.0)      # a sequence without rows: zeros
    return torch.einsum("bhn,bhnd->bhd", p, _values(s["v"], s["vs"])).to(torch.bfloat16)


def _plain_project(s):
    c = s["c"]
    B, n, D = s["x"].shape
    x, step = _quantise(s["x"], 127.0)
    y = (x.reshape(B * n, D) @ s["w8"].float().T).reshape(B, n, -1) * (step * s["ws"]) + s["bias"].float()
    y = y.to(torch.bfloat16)
    if c["kind"] == "prefix":
        return y.reshape(B, c["P"], D)
    q, k, v = y.reshape(B, n, 3, c["H"], c["hd"]).permute(2, 0, 3, 1, 4)      # each [B,H,n,hd]
    if c["kind"] == "local":
        s["kv"][:, :, :n, 0], s["kv"][:, :, :n, 1] = k, v
        return {"q": q.contiguous(), "kv": s["kv"], "len": torch.full_like(s["len0"], n)}
    at = (s["len0"].long()[:, None] + torch.arange(n, device="cuda"))[:, None, :, None].expand(B, c["H"], n, c["hd"])
    s["k"].scatter_(2, at, k)
    s["v"].scatter_(2, at, v)
    return {"q": q.contiguous(), "k": s["k"], "v": s["v"], "len": s["len0"] + n}


_PLAIN = {"kv4_write": _plain_write, "kv4_decode": _plain_decode, "project_i8": _plain_project}


# ---------------------------------------------------------------------------------------------- the definition, in 64 bits

def _held_values(x, most, width):
    """What a row of x (last axis, groups of `width`) is held as: a search among the codes instead of a quotient."""
    x = x.double()
    g = x.reshape(-1, width)
    step = (g.abs().max(1).values / most).float().to(torch.bfloat16).double()[:, None]
    # the codes' upper borders in magnitude: from (j + 1/2) steps on, the code is j + 1 at least
    borders = (torch.arange(int(most), device=x.device, dtype=torch.float64) + 0.5)[None] * step
    mag = torch.searchsorted(borders.contiguous(), g.abs().contiguous(), right=True).double()
    return (torch.where(step > 0, mag, torch.zeros_like(mag)) * step * torch.where(g < 0, -1.0, 1.0)).reshape(x.shape)


def exact(case, seed):
    c = dict(case)
    g = _generator(seed)
    lens = _lens(c)
    if c["op"] == "project_i8":
        return _exact_project(c, seed, lens)
    if c["op"] == "kv4_write":
        k_new, v_new = _rows(g, c, c["n"], True), _rows(g, c, c["n"], False)
        k, v = _rows(g, c, c["hi"], True), _rows(g, c, c["hi"], False)
        out = {"len": torch.tensor([n + c["n"] for n in lens], dtype=torch.int32, device="cuda")}
        for name, new, old in (("k", k_new, k), ("v", v_new, v)):
            out[name] = torch.zeros((c["B"], c["H"], c["N"], c["hd"]), dtype=torch.float64, device="cuda")
            for b, n in enumerate(lens):
                out[name][b, :, :n + c["n"]] = _held_values(torch.cat([old[b, :, :n], new[b]], 1), 7, 32)
        return out
    q = _normal(g, c["B"], c["H"], c["hd"]).to(torch.bfloat16).double()
    k, v = _rows(g, c, c["hi"], True), _rows(g, c, c["hi"], False)
    out = torch.zeros_like(q)
    for b, n in enumerate(lens):
        for h in range(c["H"] if n else 0):
            a = _held_values(k[b, h, :n], 7, 32) @ q[b, h] / math.sqrt(c["hd"])
            a = torch.exp(a - a.max())
            out[b, h] = a @ _held_values(v[b, h, :n], 7, 32) / a.sum()
    return out


def _exact_project(c, seed, lens):
    s = _inputs_only(c, seed)
    B, n, D = s["x"].shape
    x = _held_values(s["x"], 127, D).reshape(B * n, D)
    y = torch.addmm(s["bias"].double(), x, (s["w8"].double() * s["ws"].double()[:, None]).T)
    if c["kind"] == "prefix":
        return y.reshape(B, c["P"], D)
    rows = y.reshape(B, n, 3 * c["H"], c["hd"]).transpose(1, 2)              # [B, 3H, n, hd]
    q, k, v = rows[:, :c["H"]], rows[:, c["H"]:2 * c["H"]], rows[:, 2 * c["H"]:]
    if c["kind"] == "local":
        kv = torch.zeros((B, c["H"], c["P"] + 4, 2, c["hd"]), dtype=torch.float64, device="cuda")
        kv[:, :, :n] = torch.stack([k, v], 3)
        return {"q": q, "kv": kv, "len": torch.full((B,), n, dtype=torch.int32, device="cuda")}
    out = {"q": q, "len": torch.tensor([m + n for m in lens], dtype=torch.int32, device="cuda")}
    for name, t in (("k", k), ("v", v)):
        out[name] = torch.zeros((B, c["H"], c["N"], c["hd"]), dtype=torch.float64, device="cuda")
        for b, m in enumerate(lens):
            out[name][b, :, m:m + n] = t[b]
    return out


def _inputs_only(c, seed):
    """The inputs of a projection, as prepare() makes them."""
    s = prepare(c, seed)
    return {name: s[name] for name in ("x", "w8", "ws", "bias")}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Bytes: each input once, each output once (a 4-bit row of K and V takes 1.125 hd bytes).  Flops: the products."""
    c = dict(case)
    hd, bh = c["hd"], c["B"] * c["H"]
    lens = _lens(c)
    held = 9 * hd // 8
    if c["op"] == "kv4_decode":
        rows = sum(lens) * c["H"]
        return {"bytes": rows * held + 2 * bh * hd * 2 + 4 * c["B"], "flops": 4 * rows * hd}
    if c["op"] == "kv4_write":
        new = bh * c["n"]
        old = sum(lens) * c["H"]
        # the new rows in, held and read back; the old ones read back
        return {"bytes": new * (4 * hd + held + 4 * hd) + old * (held + 4 * hd) + 8 * c["B"], "flops": 0}
    D, M = c["H"] * hd, c["B"] * c["n"]
    features = D * (c["P"] if c["kind"] == "prefix" else 3)
    return {"bytes": 2 * M * D + features * D + 4 * features + 2 * features + 2 * M * features, "flops": 2 * M * D * features}
