"""The binding refuses tensors that do not hold what a call over the low-bit operators would read or write, before the library is called (no GPU
needed: the tensors are in the host's memory and say that they are on the current device; the library's calls are recorded)."""
import copy

import pytest
import torch


@pytest.fixture(scope="module")
def bt():
    import paper_2406_02657_b200 as bt
    return bt


class OnDevice:
    """A tensor that says it is on the current device."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0


class Recorder:
    def __init__(self, lib):
        self.calls, self.bt_status_string = [], lib.bt_status_string

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


@pytest.fixture
def lib(bt, monkeypatch):
    rec = Recorder(bt.lib())
    monkeypatch.setattr(bt.binding, "_lib", rec)
    monkeypatch.setattr(bt.binding, "_device", lambda: 0)
    monkeypatch.setattr(bt.binding, "_raw_stream", lambda device: 0)
    return rec


def t(*shape, dtype=torch.bfloat16):
    return OnDevice(torch.zeros(shape, dtype=dtype))


def view(shape, f, dtype=torch.bfloat16):
    return OnDevice(f(torch.zeros(shape, dtype=dtype)))


B, H, HD, N = 2, 3, 64, 16


def config(bt, **other):
    size = dict(batch=B, heads=H, head_dim=HD, block_len=4, prefix_len=2, max_blocks=N, n_layers=2)
    return bt.make_config(**{**size, **other})


def kv4(bt, cfg):
    cache = bt.BlockCacheKV4(cfg, device="cpu")
    cache.device = 0
    return cache


def refused(bt, lib, code, call, *args, **kwargs):
    before = len(lib.calls)
    with pytest.raises(bt.BtError) as e:
        call(*args, **kwargs)
    assert e.value.code == code and len(lib.calls) == before, e.value


def passed(lib, call, *args, **kwargs):
    before = len(lib.calls)
    call(*args, **kwargs)
    assert len(lib.calls) == before + 1
    return lib.calls[-1]


def test_rows_of_k_and_v_are_there(bt, lib):
    """Append and read: k and v of one shape, of the config's sizes, with as many rows as the call takes."""
    cfg = config(bt)
    cache, k = kv4(bt, cfg), t(B, H, 5, HD)
    for call, stride, n in ((bt.bt_block_kv4_append, "src_stride", "n_new"), (bt.bt_block_kv4_read, "dst_stride", "n_rows")):
        name, args = passed(lib, call, cfg, cache, 0, k, t(B, H, 5, HD))
        assert name == call.__name__ and 5 in args
        passed(lib, call, cfg, cache, 0, k, k, **{n: 3})
        wide = view((B, H, N, HD), lambda x: x[:, :, 2:7])
        passed(lib, call, cfg, cache, 0, wide, wide)
        # v has fewer rows, no rows' axis, next to nothing; and the other way round
        for other in (t(B, H, 3, HD), t(B, H, HD), t(1), t(B, H, 0, HD), t(B, H - 1, 5, HD), t(B, H, 5, HD // 2), t(B * H, 5, HD)):
            refused(bt, lib, bt.BT_ERR_SHAPE, call, cfg, cache, 0, k, other)
            refused(bt, lib, bt.BT_ERR_SHAPE, call, cfg, cache, 0, other, k)
        # both alike, but not what the config says
        for both in (t(B - 1, H, 5, HD), t(B, H - 1, 5, HD), t(B, H, 5, 2 * HD), t(B, H, HD), t(H, B, 5, HD)):
            refused(bt, lib, bt.BT_ERR_SHAPE, call, cfg, cache, 0, both, both)
        # more rows than there are, packed or in a larger slab, whose last one would be left behind
        refused(bt, lib, bt.BT_ERR_SHAPE, call, cfg, cache, 0, k, k, **{n: 6})
        refused(bt, lib, bt.BT_ERR_SHAPE, call, cfg, cache, 0, wide, wide, **{n: 6})
        for missing in ((None, k), (k, None)):
            refused(bt, lib, bt.BT_ERR_NULL, call, cfg, cache, 0, *missing)


def test_rows_under_a_given_stride_are_there(bt, lib):
    """A stride that the caller gives: k and v reach to the last row of the last slab."""
    cfg = config(bt)
    cache, k = kv4(bt, cfg), t(B, H, N, HD)
    flat, short = t(B * H * N - 11, HD), t(B * H * N - 12, HD)          # five rows of the last slab, four
    last = view((B, H, N, HD), lambda x: x[:, :, 11:])                  # a view that starts eleven rows into the first slab
    for call, stride, n in ((bt.bt_block_kv4_append, "src_stride", "n_new"), (bt.bt_block_kv4_read, "dst_stride", "n_rows")):
        for ok in (k, flat, last):
            passed(lib, call, cfg, cache, 0, ok, k, **{stride: N, n: 5})
            passed(lib, call, cfg, cache, 0, k, ok, **{stride: N, n: 5})
        for bad, rows in ((short, 5), (last, 6), (t(B, H, 5, HD), 5), (t(1), 1), (t(0), 1)):
            refused(bt, lib, bt.BT_ERR_SHAPE, call, cfg, cache, 0, bad, k, **{stride: N, n: rows})
            refused(bt, lib, bt.BT_ERR_SHAPE, call, cfg, cache, 0, k, bad, **{stride: N, n: rows})
        refused(bt, lib, bt.BT_ERR_SHAPE, call, cfg, cache, 0, k, k, **{stride: N + 1, n: N})
        refused(bt, lib, bt.BT_ERR_SHAPE, call, cfg, cache, 0, k, k, **{stride: N - 1, n: N})
        for wrapped in (2 ** 64 + N, N - 2 ** 64):                      # no numbers of 64 bits
            refused(bt, lib, bt.BT_ERR_SHAPE, call, cfg, cache, 0, k, k, **{stride: wrapped, n: 5})


def every_call(bt, n=1):
    """(call, its tensors in order) of every call over the low-bit operators that takes packed tensors."""
    cfg, D, P = config(bt), H * HD, 2
    cache, block, local = kv4(bt, cfg), bt.BlockCache(cfg, device="cpu"), bt.LocalCache(cfg, device="cpu")
    block.device = local.device = 0
    q, x, w, bias, qo, st = t(B, H, HD), t(B, n, D), t(3 * D, D), t(3 * D), t(B, H, n, HD), t(1, dtype=torch.int32)
    x8, w8, xs, ws = t(B, n, D, dtype=torch.int8), t(3 * D, D, dtype=torch.int8), t(B, n, dtype=torch.float32), t(3 * D, dtype=torch.float32)
    c8, cs, p8, ps, pb, po = t(B, D, dtype=torch.int8), t(B, dtype=torch.float32), t(P * D, D, dtype=torch.int8), t(P * D, dtype=torch.float32), t(P * D), t(B, P, D)
    space, mask = t(bt.bt_workspace_bytes_kv4(cfg), dtype=torch.uint8), t(B, dtype=torch.uint8)
    return [
        (lambda a, o, s: bt.bt_block_decode_attn_kv4(cfg, cache, 1, a, o, space, dev_status=s), [q, q, st]),
        (lambda a, k, v, o, s: bt.bt_block_decode_step_kv4(cfg, cache, 1, a, k, v, o, space, dev_status=s), [q, q, q, q, st]),
        (lambda a, b, c, d, s: bt.bt_block_qkv_project_append_kv4(cfg, cache, 1, a, b, c, d, n_rows=n, dev_status=s), [x, w, bias, qo, st]),
        (lambda b, c: bt.bt_rows_quantize_i8(x, b, c), [x8, xs]),
        (lambda *a: bt.bt_prefix_project_i8(cfg, *a), [c8, cs, p8, ps, pb, po, st]),
        (lambda *a: bt.bt_block_qkv_project_append_i8(cfg, block, 1, *a[:-1], n_rows=n, dev_status=a[-1]), [x8, xs, w8, ws, bias, qo, st]),
        (lambda *a: bt.bt_local_qkv_project_append_i8(cfg, local, 1, *a[:-2], n_rows=n, reset_mask=a[-2], dev_status=a[-1]), [x8, xs, w8, ws, bias, qo, mask, st]),
        (lambda *a: bt.bt_block_qkv_project_append_i8_kv4(cfg, cache, 1, *a[:-1], n_rows=n, dev_status=a[-1]), [x8, xs, w8, ws, bias, qo, st]),
    ]


@pytest.mark.parametrize("n", [1, 3])
def test_every_tensor_is_as_large_as_the_call_takes(bt, lib, n):
    """One element less than the call reads or writes is refused; more than that is not (a buffer for the most rows serves fewer)."""
    for call, args in every_call(bt, n):
        passed(lib, call, *args)
        for i in range(len(args)):
            less, more = t(args[i].numel() - 1, dtype=args[i].dtype), t(args[i].numel() + 1, dtype=args[i].dtype)
            refused(bt, lib, bt.BT_ERR_SHAPE, call, *args[:i], less, *args[i + 1:])
            passed(lib, call, *args[:i], more, *args[i + 1:])


def test_every_tensor_has_its_type(bt, lib):
    for call, args in every_call(bt):
        for i, arg in enumerate(args):
            if arg.dtype is torch.int32:
                continue                                     # the status word: any four bytes
            for kind in (torch.float32, torch.float16, torch.int8, torch.uint8, torch.bfloat16, torch.int64):
                if kind is arg.dtype or (arg.dtype is torch.uint8 and kind is torch.int8):
                    continue
                refused(bt, lib, bt.BT_ERR_UNSUPPORTED, call, *args[:i], t(*arg.shape, dtype=kind), *args[i + 1:])
    x8, steps = t(4, 64, dtype=torch.int8), t(4, dtype=torch.float32)
    refused(bt, lib, bt.BT_ERR_UNSUPPORTED, bt.bt_rows_quantize_i8, t(4, 64, dtype=torch.float32), x8, steps)
    rows = t(B, H, 1, HD, dtype=torch.float32)
    cfg = config(bt)
    for call in (bt.bt_block_kv4_append, bt.bt_block_kv4_read):
        for k, v in ((rows, t(B, H, 1, HD)), (t(B, H, 1, HD), rows)):
            refused(bt, lib, bt.BT_ERR_UNSUPPORTED, call, cfg, kv4(bt, cfg), 0, k, v)


def test_caches_are_the_config_s(bt, lib):
    """A cache made for another config is refused: other sizes, or fewer layers; one that differs in what the cache does not depend on is taken."""
    cfg, D = config(bt), H * HD
    q, x, w, rows, x8, xs = t(3, 4, 2 * HD), t(3, 1, D), t(3 * D, D), t(B, H, 1, HD), t(B, 1, D, dtype=torch.int8), t(B, dtype=torch.float32)
    w8, ws, qo, space = t(3 * D, D, dtype=torch.int8), t(3 * D, dtype=torch.float32), t(B, H, 1, HD), t(1 << 20, dtype=torch.uint8)

    def calls(cache):
        return ((bt.bt_block_kv4_append, cfg, cache, 0, rows, rows), (bt.bt_block_kv4_read, cfg, cache, 0, rows, rows),
                (bt.bt_block_decode_attn_kv4, cfg, cache, 0, q, q, space), (bt.bt_block_decode_step_kv4, cfg, cache, 0, q, q, q, q, space),
                (bt.bt_block_qkv_project_append_kv4, cfg, cache, 0, x, w, None, qo),
                (bt.bt_block_qkv_project_append_i8_kv4, cfg, cache, 0, x8, xs, w8, ws, None, qo))

    for other in (dict(batch=B - 1), dict(batch=B + 1), dict(heads=H + 1), dict(head_dim=128), dict(max_blocks=N - 1), dict(max_blocks=N + 1), dict(n_layers=1)):
        for call, *args in calls(kv4(bt, config(bt, **other))):
            refused(bt, lib, bt.BT_ERR_SHAPE, call, *args)
    for other in (dict(), dict(n_layers=3), dict(block_len=7), dict(prefix_len=1), dict(decode_splits=5), dict(softmax_scale=0.5)):
        for call, *args in calls(kv4(bt, config(bt, **other))):
            passed(lib, call, *args)


def test_caches_of_16_bits_hold_what_integers_are_projected_into(bt, lib):
    cfg, D = config(bt), H * HD
    x8, xs, w8, ws, qo = t(B, 1, D, dtype=torch.int8), t(B, dtype=torch.float32), t(3 * D, D, dtype=torch.int8), t(3 * D, dtype=torch.float32), t(B, H, 1, HD)
    for other, code in ((dict(), 0), (dict(n_layers=3), 0), (dict(batch=B - 1), bt.BT_ERR_SHAPE), (dict(n_layers=1), bt.BT_ERR_SHAPE),
                        (dict(max_blocks=N - 1, block_len=3), bt.BT_ERR_SHAPE)):
        made = config(bt, **other)
        block, local = bt.BlockCache(made, device="cpu"), bt.LocalCache(made, device="cpu")
        block.device = local.device = 0
        for call, cache in ((bt.bt_block_qkv_project_append_i8, block), (bt.bt_local_qkv_project_append_i8, local)):
            if code:
                refused(bt, lib, code, call, cfg, cache, 0, x8, xs, w8, ws, None, qo)
            else:
                passed(lib, call, cfg, cache, 0, x8, xs, w8, ws, None, qo)
            # [B,D]: its last axis is not taken for a number of rows
            refused(bt, lib, bt.BT_ERR_SHAPE, call, cfg, cache, 0, t(B, D, dtype=torch.int8), xs, w8, ws, None, qo)


def test_cache_tensors_are_what_they_should_be(bt):
    cfg = config(bt)
    good = bt.BlockCacheKV4(cfg, device="cpu")
    bt.BlockCacheKV4(cfg, device="cpu", kv=good.kv, length=good.len)
    for bad in (dict(kv=good.kv.to(torch.int8)), dict(length=good.len.long()), dict(length=good.len[:1]), dict(length=good.len.reshape(-1))):
        with pytest.raises(AssertionError):
            bt.BlockCacheKV4(cfg, device="cpu", **bad)


def test_a_config_that_changes(bt, lib):
    """What is worked out from a config's fields follows them."""
    cfg, rows = config(bt), t(B, H, 1, HD)
    cache = kv4(bt, cfg)
    passed(lib, bt.bt_block_kv4_append, cfg, cache, 0, rows, rows)
    for name, value in (("batch", B + 1), ("heads", 1), ("head_dim", 128), ("max_blocks", N + 1), ("n_layers", 3)):
        was = getattr(cfg, name)
        setattr(cfg, name, value)
        refused(bt, lib, bt.BT_ERR_SHAPE, bt.bt_block_kv4_append, cfg, cache, 0, rows, rows)
        setattr(cfg, name, was)
        passed(lib, bt.bt_block_kv4_append, cfg, cache, 0, rows, rows)
    with pytest.raises(AttributeError):
        cfg.no_such_field
    cfg.note = "kept"                          # an attribute of the caller's own
    cfg.batch, other = B, copy.copy(cfg)
    other.batch = B + 1
    assert cfg.note == "kept" and cfg.sizes == (B, H, HD, N) and other.sizes == (B + 1, H, HD, N)


def test_a_cache_of_other_types_is_refused(bt, lib):
    """A bf16 cache whose tensors the kernels would take for others: made as before, refused by the calls that look."""
    cfg, D = config(bt), H * HD
    good = bt.BlockCache(cfg, device="cpu")
    x8, xs, w8, ws, qo = t(B, 1, D, dtype=torch.int8), t(B, dtype=torch.float32), t(3 * D, D, dtype=torch.int8), t(3 * D, dtype=torch.float32), t(B, H, 1, HD)
    for bad in (dict(k=good.k.half()), dict(v=good.v.float()), dict(length=good.len.long()), dict(length=good.len[:1]),
                dict(length=torch.zeros((B, 2), dtype=torch.int32).T)):
        cache = bt.BlockCache(cfg, device="cpu", **{**dict(k=good.k, v=good.v, length=good.len), **bad})
        assert cache.device == -2
        refused(bt, lib, bt.BT_ERR_UNSUPPORTED, bt.bt_block_qkv_project_append_i8, cfg, cache, 0, x8, xs, w8, ws, None, qo)
