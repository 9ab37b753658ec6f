// C-ABI layer: argument validation, layer offsets, dispatch to the kernels.
// Nothing here touches device memory on the host side or allocates any.
#include <math.h>

#include "../../include/bt.h"
#include "bt_kernels.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;

bool config_ok(const bt_config* c)
{
    return c && c->batch > 0 && c->heads > 0 && c->head_dim > 0 && c->block_len > 0 && c->prefix_len > 0 &&
           c->max_blocks > 0 && c->n_layers > 0 && c->decode_splits >= 0 && c->softmax_scale >= 0.f &&
           isfinite(c->softmax_scale);
}

bt_status check_config(const bt_config* c, int layer)
{
    if (!c) return BT_ERR_NULL;
    if (!config_ok(c)) return BT_ERR_SHAPE;
    if (layer < 0 || layer >= c->n_layers) return BT_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128) return BT_ERR_UNSUPPORTED;
    if (c->heads * (c->head_dim / 8) > 256) return BT_ERR_UNSUPPORTED;  // one CTA must cover a sequence
    if (c->decode_splits > 64) return BT_ERR_UNSUPPORTED;
    return BT_OK;
}

float scale_log2(const bt_config* c)
{
    const float s = c->softmax_scale > 0.f ? c->softmax_scale : 1.0f / sqrtf((float)c->head_dim);
    return s * kLog2e;
}

// `rows`: how many a query may have to read
int choose_splits_for(const bt_config* c, int rows)
{
    if (c->decode_splits > 0) return c->decode_splits;
    // enough work items to reach every SM several times over, each of at least 128 rows (four chunks of the
    // streaming kernel; below that the per-item costs show) - short caches may still be cut into up to 4
    // parts of at least 16 rows
    const long long bh = (long long)c->batch * c->heads;
    const long long target = 512;
    long long s = (target + bh - 1) / bh;
    long long by_rows = rows / 128;
    const long long small = rows / 16 < 4 ? rows / 16 : 4;
    if (by_rows < small) by_rows = small;
    if (by_rows < 1) by_rows = 1;
    if (s > by_rows) s = by_rows;
    if (s > 32) s = 32;
    if (s < 1) s = 1;
    return (int)s;
}
int choose_splits(const bt_config* c) { return choose_splits_for(c, c->max_blocks); }

inline size_t block_layer_elems(const bt_config* c) { return (size_t)c->batch * c->heads * c->max_blocks * c->head_dim; }
inline int local_cap(const bt_config* c) { return c->prefix_len + c->block_len; }
inline size_t local_layer_elems(const bt_config* c) { return (size_t)c->batch * c->heads * local_cap(c) * 2 * c->head_dim; }

bt::CacheView block_view(const bt_config* c, const bt_block_cache* cache, int layer)
{
    bt::CacheView v;
    v.k = (char*)cache->k + block_layer_elems(c) * layer * 2;
    v.v = (char*)cache->v + block_layer_elems(c) * layer * 2;
    v.len = cache->len + (size_t)layer * c->batch;
    v.slab_stride = (int64_t)c->max_blocks * c->head_dim;
    v.row_stride = c->head_dim;
    v.cap = c->max_blocks;
    return v;
}

bt::CacheView local_view(const bt_config* c, const bt_local_cache* cache, int layer)
{
    bt::CacheView v;
    char* base = (char*)cache->kv + local_layer_elems(c) * layer * 2;
    v.k = base;
    v.v = base + (size_t)c->head_dim * 2;
    v.len = cache->len + (size_t)layer * c->batch;
    v.slab_stride = (int64_t)local_cap(c) * 2 * c->head_dim;
    v.row_stride = 2 * c->head_dim;
    v.cap = local_cap(c);
    return v;
}

inline bt_status cuda_status(cudaError_t e) { return e == cudaSuccess ? BT_OK : BT_ERR_CUDA; }

// The kernels move data in 16-byte pieces (128-bit loads and stores, cp.async, bulk and tensor copies):
// every tensor base must sit on a 16-byte boundary, length arrays on a 4-byte one.  NULL passes (it
// is either optional or refused as BT_ERR_NULL elsewhere).
inline bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool al4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool block_cache_aligned(const bt_block_cache* c) { return al16(c->k) && al16(c->v) && al4(c->len); }
inline bool local_cache_aligned(const bt_local_cache* c) { return al16(c->kv) && al4(c->len); }

// what bt_block_decode_attn (k_new == NULL) and bt_block_decode_step check before anything is enqueued
bt_status decode_validate(const bt_config* cfg, const bt_block_cache* cache, int layer, const void* q, const void* k_new,
                                 const void* v_new, bool step, const void* out, const void* workspace, size_t workspace_bytes,
                                 const uint32_t* dev_status)
{
    bt_status st = check_config(cfg, layer);
    if (st != BT_OK) return st;
    if (!cache || !cache->k || !cache->v || !cache->len || !q || !out) return BT_ERR_NULL;
    if (step && (!k_new || !v_new)) return BT_ERR_NULL;
    const bool need_ws = choose_splits(cfg) > 1 || step;
    if (need_ws && (!workspace || workspace_bytes < bt_workspace_bytes(cfg))) return BT_ERR_WORKSPACE;
    if (!block_cache_aligned(cache) || !al16(q) || !al16(out) || !al16(k_new) || !al16(v_new) || !al4(dev_status) ||
        (need_ws && !al16(workspace)))
        return BT_ERR_UNSUPPORTED;
    return BT_OK;
}

}  // namespace

namespace bt {
bt_status validate_decode_attn_args(const bt_config* cfg, const bt_block_cache* cache, int layer, const void* q, const void* out,
                                    const uint32_t* dev_status)
{
    // a workspace that cannot be refused: only the other arguments are judged
    return decode_validate(cfg, cache, layer, q, nullptr, nullptr, false, out, reinterpret_cast<const void*>(uintptr_t(16)),
                           ~size_t(0), dev_status);
}
}  // namespace bt

extern "C" {

int bt_version(void) { return 300; }

const char* bt_status_string(bt_status s)
{
    switch (s) {
        case BT_OK: return "BT_OK";
        case BT_ERR_NULL: return "BT_ERR_NULL";
        case BT_ERR_SHAPE: return "BT_ERR_SHAPE";
        case BT_ERR_UNSUPPORTED: return "BT_ERR_UNSUPPORTED";
        case BT_ERR_CAPACITY: return "BT_ERR_CAPACITY";
        case BT_ERR_WORKSPACE: return "BT_ERR_WORKSPACE";
        case BT_ERR_CUDA: return "BT_ERR_CUDA";
    }
    return "BT_ERR_?";
}

int bt_decode_splits(const bt_config* cfg)
{
    if (check_config(cfg, 0) != BT_OK) return 0;
    return choose_splits(cfg);
}

// Workspace layout: the split partials ([B*H][splits][hd+4] floats, absent when the row range is not
// split), then the arrival counters ([B*H] + [B] int32).
static size_t partial_bytes(const bt_config* cfg)
{
    const int s = choose_splits(cfg);
    return s <= 1 ? 0 : (size_t)s * cfg->batch * cfg->heads * (cfg->head_dim + 4) * sizeof(float);
}
static size_t counter_bytes(const bt_config* cfg) { return ((size_t)cfg->batch * cfg->heads + cfg->batch) * sizeof(int32_t); }

size_t bt_workspace_bytes(const bt_config* cfg)
{
    if (check_config(cfg, 0) != BT_OK) return 0;
    return partial_bytes(cfg) + counter_bytes(cfg);
}

bt_status bt_workspace_init(const bt_config* cfg, void* workspace, size_t workspace_bytes, void* stream)
{
    bt_status st = check_config(cfg, 0);
    if (st != BT_OK) return st;
    if (!workspace) return BT_ERR_NULL;
    if (workspace_bytes < bt_workspace_bytes(cfg)) return BT_ERR_WORKSPACE;
    if (!al16(workspace)) return BT_ERR_UNSUPPORTED;
    return cuda_status(cudaMemsetAsync((char*)workspace + partial_bytes(cfg), 0, counter_bytes(cfg), (cudaStream_t)stream));
}

bt_status bt_block_kv_append(const bt_config* cfg, bt_block_cache* cache, int layer, const void* k_new,
                             const void* v_new, int n_new, uint32_t* dev_status, void* stream)
{
    bt_status st = check_config(cfg, layer);
    if (st != BT_OK) return st;
    if (!cache || !cache->k || !cache->v || !cache->len || !k_new || !v_new) return BT_ERR_NULL;
    if (n_new <= 0) return BT_ERR_SHAPE;
    if (n_new > cfg->max_blocks) return BT_ERR_CAPACITY;
    if (!block_cache_aligned(cache) || !al16(k_new) || !al16(v_new) || !al4(dev_status)) return BT_ERR_UNSUPPORTED;
    return cuda_status(bt::launch_kv_append(block_view(cfg, cache, layer), cfg->batch, cfg->heads, cfg->head_dim,
                                            k_new, v_new, n_new, dev_status, (cudaStream_t)stream));
}

// the arguments of the streaming decode kernel (k_new == NULL: nothing is appended)
static void fill_decode_args(bt::DecodeArgs& a, const bt_config* cfg, const bt_block_cache* cache, int layer, const void* q,
                             const void* k_new, const void* v_new, void* out, void* workspace, int splits, uint32_t* dev_status)
{
    const bool need_ws = splits > 1 || k_new != nullptr;
    bt::CacheView v = block_view(cfg, cache, layer);
    a.q = q;
    a.k = v.k;
    a.v = v.v;
    a.len = v.len;
    a.out = out;
    a.ws = (float*)workspace;
    a.counters = need_ws ? (int32_t*)((char*)workspace + partial_bytes(cfg)) : nullptr;
    a.k_new = k_new;
    a.v_new = v_new;
    a.dev_status = dev_status;
    a.B = cfg->batch;
    a.H = cfg->heads;
    a.hd = cfg->head_dim;
    a.n_max = cfg->max_blocks;
    a.splits = splits;
    a.scale_log2 = scale_log2(cfg);
}

// append (optional) + attention in one launch; the arguments have passed decode_validate
static bt_status decode_launch(const bt_config* cfg, bt_block_cache* cache, int layer, const void* q, const void* k_new,
                               const void* v_new, void* out, void* workspace, size_t workspace_bytes,
                               uint32_t* dev_status, void* stream)
{
    (void)workspace_bytes;
    bt::DecodeArgs a;
    fill_decode_args(a, cfg, cache, layer, q, k_new, v_new, out, workspace, choose_splits(cfg), dev_status);
    return cuda_status(bt::launch_block_decode(a, (cudaStream_t)stream));
}

bt_status bt_block_decode_attn(const bt_config* cfg, const bt_block_cache* cache, int layer, const void* q,
                               void* out, void* workspace, size_t workspace_bytes, uint32_t* dev_status,
                               void* stream)
{
    bt_status st = decode_validate(cfg, cache, layer, q, nullptr, nullptr, false, out, workspace, workspace_bytes, dev_status);
    if (st != BT_OK) return st;
    // without a row to append the kernel only reads the cache
    return decode_launch(cfg, const_cast<bt_block_cache*>(cache), layer, q, nullptr, nullptr, out, workspace,
                         workspace_bytes, dev_status, stream);
}

bt_status bt_block_decode_step(const bt_config* cfg, bt_block_cache* cache, int layer, const void* q,
                               const void* k_new, const void* v_new, void* out, void* workspace,
                               size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    bt_status st = decode_validate(cfg, cache, layer, q, k_new, v_new, true, out, workspace, workspace_bytes, dev_status);
    if (st != BT_OK) return st;
    return decode_launch(cfg, cache, layer, q, k_new, v_new, out, workspace, workspace_bytes, dev_status, stream);
}

bt_status bt_block_decode_step_multi(const bt_config* cfg, bt_block_cache* cache, int layer, const void* q,
                                     const void* k_new, const void* v_new, int n_q, void* out, void* workspace,
                                     size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    bt_status st = check_config(cfg, layer);
    if (st != BT_OK) return st;
    if (!cache || !cache->k || !cache->v || !cache->len || !q || !k_new || !v_new || !out) return BT_ERR_NULL;
    if (n_q <= 0) return BT_ERR_SHAPE;
    if (n_q > cfg->max_blocks) return BT_ERR_CAPACITY;
    if (!workspace || workspace_bytes < bt_workspace_bytes(cfg)) return BT_ERR_WORKSPACE;
    if (!block_cache_aligned(cache) || !al16(workspace) || !al4(dev_status)) return BT_ERR_UNSUPPORTED;
    bt::CacheView v = block_view(cfg, cache, layer);
    bt::MultiDecodeArgs a;
    a.q = q;
    a.k_new = k_new;
    a.v_new = v_new;
    a.k = v.k;
    a.v = v.v;
    a.len = v.len;
    a.out = out;
    a.counters = (int32_t*)((char*)workspace + partial_bytes(cfg));
    a.dev_status = dev_status;
    a.B = cfg->batch;
    a.H = cfg->heads;
    a.hd = cfg->head_dim;
    a.n_max = cfg->max_blocks;
    a.m = n_q;
    a.scale_log2 = scale_log2(cfg);
    if (!bt::multi_decode_supported(a)) return BT_ERR_UNSUPPORTED;
    return cuda_status(bt::launch_block_decode_multi(a, (cudaStream_t)stream));
}

bt_status bt_local_kv_reset(const bt_config* cfg, bt_local_cache* cache, int layer, const uint8_t* seq_mask,
                            void* stream)
{
    bt_status st = check_config(cfg, layer);
    if (st != BT_OK) return st;
    if (!cache || !cache->len) return BT_ERR_NULL;
    if (!al4(cache->len)) return BT_ERR_UNSUPPORTED;
    return cuda_status(bt::launch_len_reset(cache->len + (size_t)layer * cfg->batch, cfg->batch, seq_mask,
                                            (cudaStream_t)stream));
}

bt_status bt_local_kv_append(const bt_config* cfg, bt_local_cache* cache, int layer, const void* k_new,
                             const void* v_new, int n_new, uint32_t* dev_status, void* stream)
{
    bt_status st = check_config(cfg, layer);
    if (st != BT_OK) return st;
    if (!cache || !cache->kv || !cache->len || !k_new || !v_new) return BT_ERR_NULL;
    if (n_new <= 0) return BT_ERR_SHAPE;
    if (n_new > local_cap(cfg)) return BT_ERR_CAPACITY;
    if (!local_cache_aligned(cache) || !al16(k_new) || !al16(v_new) || !al4(dev_status)) return BT_ERR_UNSUPPORTED;
    return cuda_status(bt::launch_kv_append(local_view(cfg, cache, layer), cfg->batch, cfg->heads, cfg->head_dim,
                                            k_new, v_new, n_new, dev_status, (cudaStream_t)stream));
}

bt_status bt_token_decode_attn(const bt_config* cfg, bt_local_cache* cache, int layer, const void* q,
                               const void* k_new, const void* v_new, int n_q, int reset_first,
                               const uint8_t* reset_mask, void* out, uint32_t* dev_status, void* stream)
{
    bt_status st = check_config(cfg, layer);
    if (st != BT_OK) return st;
    if (!cache || !cache->kv || !cache->len || !q || !out) return BT_ERR_NULL;
    if ((k_new == nullptr) != (v_new == nullptr)) return BT_ERR_NULL;
    if (n_q <= 0) return BT_ERR_SHAPE;
    if (n_q > local_cap(cfg)) return BT_ERR_CAPACITY;
    if (!local_cache_aligned(cache) || !al16(q) || !al16(k_new) || !al16(v_new) || !al16(out) || !al4(dev_status))
        return BT_ERR_UNSUPPORTED;
    bt::TokenArgs a;
    a.kv = (char*)cache->kv + local_layer_elems(cfg) * layer * 2;
    a.len = cache->len + (size_t)layer * cfg->batch;
    a.q = q;
    a.k_new = k_new;
    a.v_new = v_new;
    a.out = out;
    a.reset_mask = reset_mask;
    a.dev_status = dev_status;
    a.B = cfg->batch;
    a.H = cfg->heads;
    a.hd = cfg->head_dim;
    a.cap = local_cap(cfg);
    a.n_q = n_q;
    a.reset_first = reset_first ? 1 : 0;
    a.scale_log2 = scale_log2(cfg);
    return cuda_status(bt::launch_token_decode(a, (cudaStream_t)stream));
}

// the arguments of the prefill kernels, checked
static bt_status prefill_args(bt::PrefillArgs& a, const bt_config* cfg, const void* q, const void* k, const void* v, int n_blocks,
                              int64_t kv_seq_stride, void* out, const uint32_t* dev_status)
{
    bt_status st = check_config(cfg, 0);
    if (st != BT_OK) return st;
    if (!q || !k || !v || !out) return BT_ERR_NULL;
    if (n_blocks <= 0 || kv_seq_stride < n_blocks) return BT_ERR_SHAPE;
    if (!al16(q) || !al16(k) || !al16(v) || !al16(out) || !al4(dev_status)) return BT_ERR_UNSUPPORTED;
    a.q = q;
    a.k = k;
    a.v = v;
    a.out = out;
    a.B = cfg->batch;
    a.H = cfg->heads;
    a.hd = cfg->head_dim;
    a.T = n_blocks;
    a.kv_seq_stride = kv_seq_stride;
    a.scale_log2 = scale_log2(cfg);
    return BT_OK;
}

bt_status bt_block_prefill_attn(const bt_config* cfg, const void* q, const void* k, const void* v, int n_blocks,
                                int64_t kv_seq_stride, void* out, uint32_t* dev_status, void* stream)
{
    bt::PrefillArgs a;
    const bt_status st = prefill_args(a, cfg, q, k, v, n_blocks, kv_seq_stride, out, dev_status);
    if (st != BT_OK) return st;
    // the kernel is the caller's choice, never a silent switch: the tensor-core one unless the config asks
    // for the CUDA-core one
    if (cfg->prefill_plain) return cuda_status(bt::launch_block_prefill_simple(a, (cudaStream_t)stream));
    if (!bt::prefill_tc_supported(a)) return BT_ERR_UNSUPPORTED;  // no driver entry point for tensor maps
    return cuda_status(bt::launch_block_prefill_tc(a, dev_status, (cudaStream_t)stream));
}

bt_status bt_block_decode_step_host(const bt_config* cfg, bt_block_cache* cache, int layer, const void* q_host,
                                    const void* k_new_host, const void* v_new_host, void* out_host, void* q_dev,
                                    void* k_dev, void* v_dev, void* out_dev, void* workspace,
                                    size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    // everything bt_block_decode_step would refuse is refused here, before the first copy is enqueued
    bt_status st = check_config(cfg, layer);
    if (st != BT_OK) return st;
    if (!q_host || !k_new_host || !v_new_host || !out_host || !q_dev || !k_dev || !v_dev || !out_dev) return BT_ERR_NULL;
    st = decode_validate(cfg, cache, layer, q_dev, k_dev, v_dev, true, out_dev, workspace, workspace_bytes, dev_status);
    if (st != BT_OK) return st;
    const size_t bytes = (size_t)cfg->batch * cfg->heads * cfg->head_dim * 2;
    cudaStream_t s = (cudaStream_t)stream;
    if (cudaMemcpyAsync(k_dev, k_new_host, bytes, cudaMemcpyHostToDevice, s) != cudaSuccess) return BT_ERR_CUDA;
    if (cudaMemcpyAsync(v_dev, v_new_host, bytes, cudaMemcpyHostToDevice, s) != cudaSuccess) return BT_ERR_CUDA;
    if (cudaMemcpyAsync(q_dev, q_host, bytes, cudaMemcpyHostToDevice, s) != cudaSuccess) return BT_ERR_CUDA;
    st = decode_launch(cfg, cache, layer, q_dev, k_dev, v_dev, out_dev, workspace, workspace_bytes, dev_status, stream);
    if (st != BT_OK) return st;
    if (cudaMemcpyAsync(out_host, out_dev, bytes, cudaMemcpyDeviceToHost, s) != cudaSuccess) return BT_ERR_CUDA;
    return BT_OK;
}

// ---- long and shared contexts

static bt_status decode_window(const bt_config* cfg, const bt_block_cache* cache, int layer, const void* q, const void* k_new,
                               const void* v_new, bool step, int window, int sinks, void* out, void* workspace,
                               size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    bt_status st = decode_validate(cfg, cache, layer, q, k_new, v_new, step, out, workspace, workspace_bytes, dev_status);
    if (st != BT_OK) return st;
    if (window < 1 || sinks < 0) return BT_ERR_SHAPE;
    bt::WindowDecodeArgs a;
    a.window = window < cfg->max_blocks ? window : cfg->max_blocks;
    a.sinks = sinks < cfg->max_blocks ? sinks : cfg->max_blocks;
    const long long rows = (long long)a.window + a.sinks;
    fill_decode_args(a, cfg, cache, layer, q, k_new, v_new, out, workspace,
                     choose_splits_for(cfg, rows < cfg->max_blocks ? (int)rows : cfg->max_blocks), dev_status);
    return cuda_status(bt::launch_block_decode_window(a, (cudaStream_t)stream));
}

bt_status bt_block_decode_attn_window(const bt_config* cfg, const bt_block_cache* cache, int layer, const void* q, int window,
                                      int sinks, void* out, void* workspace, size_t workspace_bytes, uint32_t* dev_status,
                                      void* stream)
{
    return decode_window(cfg, cache, layer, q, nullptr, nullptr, false, window, sinks, out, workspace, workspace_bytes, dev_status, stream);
}

bt_status bt_block_decode_step_window(const bt_config* cfg, bt_block_cache* cache, int layer, const void* q, const void* k_new,
                                      const void* v_new, int window, int sinks, void* out, void* workspace,
                                      size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    return decode_window(cfg, cache, layer, q, k_new, v_new, true, window, sinks, out, workspace, workspace_bytes, dev_status, stream);
}

bt_status bt_block_prefill_attn_window(const bt_config* cfg, const void* q, const void* k, const void* v, int n_blocks,
                                       int64_t kv_seq_stride, int window, int sinks, void* out, uint32_t* dev_status, void* stream)
{
    bt::PrefillArgs a;
    bt_status st = prefill_args(a, cfg, q, k, v, n_blocks, kv_seq_stride, out, dev_status);
    if (st != BT_OK) return st;
    if (window < 1 || sinks < 0) return BT_ERR_SHAPE;
    if (cfg->prefill_plain || !bt::prefill_tc_supported(a)) return BT_ERR_UNSUPPORTED;
    return cuda_status(bt::launch_block_prefill_window(a, window < n_blocks ? window : n_blocks, sinks < n_blocks ? sinks : n_blocks,
                                                       dev_status, (cudaStream_t)stream));
}

// Parts into which the shared prefix is cut: with the heads and the tiles of 128 sequences enough CTAs for the SMs
// (148 on a B200; the number fixes the workspace, so it does not depend on the device), each of at least 128 rows.
static int shared_parts(const bt_config* cfg, int prefix_max)
{
    const long long tiles = (long long)cfg->heads * ((cfg->batch + 127) / 128);
    long long parts = 148 / tiles;
    const long long most = (prefix_max + 127) / 128;
    if (parts > most) parts = most;
    if (parts > 32) parts = 32;
    return parts < 1 ? 1 : (int)parts;
}
static size_t align16(size_t n) { return (n + 15) & ~(size_t)15; }

// Parts into which a sequence's own rows are cut: one while 512 rows at most or enough (sequence, head) pairs, else enough for
// eight CTAs on each of 148 SMs, each of at least 128 rows.
static int shared_splits(const bt_config* cfg)
{
    if (cfg->decode_splits > 0) return cfg->decode_splits;
    const long long bh = (long long)cfg->batch * cfg->heads;
    long long s = 8 * 148 / bh;
    const long long most = cfg->max_blocks / 128;
    if (s > most) s = most;
    if (s > 32) s = 32;
    return s < 1 || cfg->max_blocks <= 512 ? 1 : (int)s;
}

size_t bt_workspace_bytes_shared(const bt_config* cfg, int prefix_max)
{
    if (check_config(cfg, 0) != BT_OK || prefix_max <= 0) return 0;
    return align16(bt_workspace_bytes(cfg)) +
           (size_t)(shared_parts(cfg, prefix_max) + shared_splits(cfg)) * cfg->batch * cfg->heads * (cfg->head_dim + 4) * sizeof(float);
}

static bt_status decode_shared(const bt_config* cfg, const bt_block_cache* prefix, int prefix_max, const bt_block_cache* cache,
                               int layer, const void* q, const void* k_new, const void* v_new, bool step, void* out,
                               void* workspace, size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    bt_status st = check_config(cfg, layer);
    if (st != BT_OK) return st;
    if (!prefix || !prefix->k || !prefix->v || !prefix->len) return BT_ERR_NULL;
    if (prefix_max <= 0) return BT_ERR_SHAPE;
    st = decode_validate(cfg, cache, layer, q, k_new, v_new, step, out, workspace, workspace_bytes, dev_status);
    if (st != BT_OK) return st;
    if (!workspace || workspace_bytes < bt_workspace_bytes_shared(cfg, prefix_max)) return BT_ERR_WORKSPACE;
    if (!block_cache_aligned(prefix) || !al16(workspace)) return BT_ERR_UNSUPPORTED;
    // a step writes rows and lengths of the cache while the prefix is still being read
    if (step && (prefix->k == cache->k || prefix->v == cache->v || prefix->len == cache->len)) return BT_ERR_UNSUPPORTED;
    const size_t prefix_layer = (size_t)cfg->heads * prefix_max * cfg->head_dim * 2;
    bt::SharedDecodeArgs a;
    fill_decode_args(a, cfg, cache, layer, q, k_new, v_new, out, workspace, shared_splits(cfg), dev_status);
    a.counters = (int32_t*)((char*)workspace + partial_bytes(cfg));
    a.pk = (const char*)prefix->k + prefix_layer * layer;
    a.pv = (const char*)prefix->v + prefix_layer * layer;
    a.prefix_len = prefix->len + layer;
    a.cap = prefix_max;
    a.parts = (float*)((char*)workspace + align16(bt_workspace_bytes(cfg)));
    a.n_pre = shared_parts(cfg, prefix_max);
    if (!bt::shared_decode_supported(a)) return BT_ERR_UNSUPPORTED;
    const cudaError_t e = bt::launch_shared_prefix(a, (cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_status(e);
    return cuda_status(bt::launch_shared_own(a, (cudaStream_t)stream));
}

bt_status bt_block_decode_attn_shared(const bt_config* cfg, const bt_block_cache* prefix, int prefix_max, const bt_block_cache* cache,
                                      int layer, const void* q, void* out, void* workspace, size_t workspace_bytes,
                                      uint32_t* dev_status, void* stream)
{
    return decode_shared(cfg, prefix, prefix_max, cache, layer, q, nullptr, nullptr, false, out, workspace, workspace_bytes, dev_status, stream);
}

bt_status bt_block_decode_step_shared(const bt_config* cfg, const bt_block_cache* prefix, int prefix_max, bt_block_cache* cache,
                                      int layer, const void* q, const void* k_new, const void* v_new, void* out, void* workspace,
                                      size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    return decode_shared(cfg, prefix, prefix_max, cache, layer, q, k_new, v_new, true, out, workspace, workspace_bytes, dev_status, stream);
}

// Ways the row range is split when weights are summed.  Where the plain calls split, this one's workspace has room for
// as many parts as fill the kernel's seven warps on each of 148 SMs (84.6 us at 4 x 16 heads of 12001 to 16384 rows, head_dim 128, in 16
// parts; in the plain calls' 8, two warps on each, it was 91.5 when this was 86.8), each of at least 128 rows.
//   Short caches of few pairs are cut like the plain calls' too, and then pay a second launch, although a single one with the
// scores in shared memory is shorter up to 128 rows of head_dim 64 or 64 rows of 128.  Replayed back to back from a graph, us, as cut here / in one piece
// (decode_splits = 1):
//     rows:                    32          64          128         256         512
//     32 pairs, head_dim 64    7.0 / 3.4   7.0 / 4.1   7.3 / 5.3   7.5 / 8.1   8.2 / 13.9
//     32 pairs, head_dim 128   7.7 / 4.0   7.8 / 5.4   7.8 / 8.1   8.1 / 14.1  9.8 / 25.8
//     256 pairs, head_dim 64   7.8 / 3.8   7.7 / 4.4   8.0 / 5.6   9.1 / 8.4   10.2 / 14.5
//     256 pairs, head_dim 128  8.4 / 4.3   8.6 / 5.6   9.1 / 8.5   11.3 / 14.7 14.3 / 26.5
static int weights_splits(const bt_config* cfg)
{
    const int base = choose_splits(cfg);
    if (cfg->decode_splits > 0 || base == 1) return base;
    const long long s = 7 * 148 / ((long long)cfg->batch * cfg->heads), most = cfg->max_blocks / 128;
    const long long wide = s < most ? s : most;
    return wide > base ? (wide < 64 ? (int)wide : 64) : base;
}

// Do the scores of an item stay in its warp's shared memory (else they go through the workspace)?
static bool weights_in_smem(const bt_config* cfg) { return weights_splits(cfg) == 1 && cfg->max_blocks <= bt::kWeightsSmemRows; }

// Workspace of the calls that sum weights: the plain one, and unless the scores stay in shared memory per (b,h) 16 bytes, the
// scores (N_max floats) and the partials of the splits.
size_t bt_workspace_bytes_weights(const bt_config* cfg)
{
    if (check_config(cfg, 0) != BT_OK) return 0;
    if (weights_in_smem(cfg)) return bt_workspace_bytes(cfg);
    const size_t bh = (size_t)cfg->batch * cfg->heads;
    return align16(bt_workspace_bytes(cfg)) + bh * 16 + align16(bh * cfg->max_blocks * sizeof(float)) +
           bh * weights_splits(cfg) * (cfg->head_dim + 4) * sizeof(float);
}

static bt_status decode_weights(const bt_config* cfg, const bt_block_cache* cache, int layer, const void* q, const void* k_new,
                                const void* v_new, bool step, void* out, const float* weights_in, float* weights_out,
                                void* workspace, size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    bt_status st = decode_validate(cfg, cache, layer, q, k_new, v_new, step, out, workspace, workspace_bytes, dev_status);
    if (st != BT_OK) return st;
    if (!weights_out) return BT_ERR_NULL;
    if (!weights_in_smem(cfg) && (!workspace || workspace_bytes < bt_workspace_bytes_weights(cfg))) return BT_ERR_WORKSPACE;
    if (!al16(weights_in) || !al16(weights_out) || (!weights_in_smem(cfg) && !al16(workspace))) return BT_ERR_UNSUPPORTED;
    const size_t bh = (size_t)cfg->batch * cfg->heads, layer_sums = bh * cfg->max_blocks * layer;
    bt::WeightsDecodeArgs a;
    fill_decode_args(a, cfg, cache, layer, q, k_new, v_new, out, workspace, weights_splits(cfg), dev_status);
    a.w_in = weights_in ? weights_in + layer_sums : nullptr;
    a.w_out = weights_out + layer_sums;
    a.smem_rows = 0;
    a.info = nullptr;
    a.scores = nullptr;
    if (weights_in_smem(cfg)) {
        a.smem_rows = (cfg->max_blocks + 3) & ~3;
    } else {
        a.info = (int4*)((char*)workspace + align16(bt_workspace_bytes(cfg)));
        a.scores = (float*)(a.info + bh);
        a.ws = (float*)((char*)a.scores + align16(bh * cfg->max_blocks * sizeof(float)));
    }
    return cuda_status(bt::launch_block_decode_weights(a, (cudaStream_t)stream));
}

bt_status bt_block_decode_attn_weights(const bt_config* cfg, const bt_block_cache* cache, int layer, const void* q, void* out,
                                       const float* weights_in, float* weights_out, void* workspace, size_t workspace_bytes,
                                       uint32_t* dev_status, void* stream)
{
    return decode_weights(cfg, cache, layer, q, nullptr, nullptr, false, out, weights_in, weights_out, workspace, workspace_bytes,
                          dev_status, stream);
}

bt_status bt_block_decode_step_weights(const bt_config* cfg, bt_block_cache* cache, int layer, const void* q, const void* k_new,
                                       const void* v_new, void* out, const float* weights_in, float* weights_out, void* workspace,
                                       size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    return decode_weights(cfg, cache, layer, q, k_new, v_new, true, out, weights_in, weights_out, workspace, workspace_bytes,
                          dev_status, stream);
}

bt_status bt_block_kv_evict(const bt_config* cfg, bt_block_cache* cache, float* weights, int layer, int n_keep, int n_trigger,
                            int n_sinks, int n_recent, bt_block_cache* dst, float* dst_weights, int dst_max, int32_t* kept,
                            void* workspace, size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    bt_status st = check_config(cfg, layer);
    if (st != BT_OK) return st;
    if (!cache || !cache->k || !cache->v || !cache->len || !weights || !kept) return BT_ERR_NULL;
    if (dst && (!dst->k || !dst->v || !dst->len || !dst_weights)) return BT_ERR_NULL;
    if (n_keep < 1 || n_sinks < 0 || n_recent < 0 || n_trigger < 0 || n_sinks > n_keep || n_recent > n_keep - n_sinks) return BT_ERR_SHAPE;
    if (n_keep > 1 << 30) return BT_ERR_SHAPE;   // loops over the rows kept count past them by a CTA's threads
    if (n_trigger <= n_keep) n_trigger = n_keep + 1;
    if (dst) {
        if (dst_max < 1) return BT_ERR_SHAPE;
        // the longest sequence that is left whole has to fit, and so do the rows kept
        const int whole = n_trigger - 1 < cfg->max_blocks ? n_trigger - 1 : cfg->max_blocks;
        const int most = n_keep < cfg->max_blocks && n_keep > whole ? n_keep : whole;
        if (dst_max < most) return BT_ERR_CAPACITY;
        // another cache throughout, or none: the kernel for another cache does not order its reads before its writes
        if (dst->k == cache->k || dst->v == cache->v || dst->len == cache->len || dst_weights == weights) return BT_ERR_UNSUPPORTED;
    } else {
        if (dst_weights) return BT_ERR_NULL;   // sums for another cache without the cache
        if (!workspace || workspace_bytes < bt_workspace_bytes(cfg)) return BT_ERR_WORKSPACE;
        if (!al16(workspace)) return BT_ERR_UNSUPPORTED;
    }
    if (!block_cache_aligned(cache) || !al16(weights) || !al4(kept) || !al4(dev_status)) return BT_ERR_UNSUPPORTED;
    if (dst && (!block_cache_aligned(dst) || !al16(dst_weights))) return BT_ERR_UNSUPPORTED;
    const bt::CacheView v = block_view(cfg, cache, layer);
    const size_t bh = (size_t)cfg->batch * cfg->heads;
    bt::EvictArgs a;
    a.k = v.k;
    a.v = v.v;
    a.w = weights + bh * cfg->max_blocks * layer;
    a.len = v.len;
    a.in_place = dst == nullptr;
    if (dst) {
        const size_t dst_layer = bh * dst_max * cfg->head_dim * 2 * layer;
        a.dst_k = (char*)dst->k + dst_layer;
        a.dst_v = (char*)dst->v + dst_layer;
        a.dst_w = dst_weights + bh * dst_max * layer;
        a.dst_len = dst->len + (size_t)layer * cfg->batch;
        a.dst_max = dst_max;
        a.counters = nullptr;
    } else {
        a.dst_k = v.k;
        a.dst_v = v.v;
        a.dst_w = weights + bh * cfg->max_blocks * layer;
        a.dst_len = v.len;
        a.dst_max = cfg->max_blocks;
        a.counters = (int32_t*)((char*)workspace + partial_bytes(cfg)) + bh;
    }
    a.kept = kept;
    a.dev_status = dev_status;
    a.B = cfg->batch;
    a.H = cfg->heads;
    a.hd = cfg->head_dim;
    a.n_max = cfg->max_blocks;
    a.n_keep = n_keep;
    a.trigger = n_trigger;
    a.n_sinks = n_sinks;
    a.n_recent = n_recent;
    return cuda_status(bt::launch_block_kv_evict(a, (cudaStream_t)stream));
}

// ---- the block cache in 4 bits

static bt_status check_kv4(const bt_config* cfg, const bt_block_cache_kv4* cache, int layer)
{
    bt_status st = check_config(cfg, layer);
    if (st != BT_OK) return st;
    if (!cache || !cache->kv || !cache->len) return BT_ERR_NULL;
    if (cfg->max_blocks > 1 << 30) return BT_ERR_UNSUPPORTED;   // rows are counted past the end by a chunk
    return BT_OK;
}
static bool kv4_aligned(const bt_block_cache_kv4* c) { return al16(c->kv) && al4(c->len); }
static size_t kv4_slab_bytes(const bt_config* c) { return (size_t)((c->max_blocks + 15) / 16) * (c->head_dim / 64) * BT_KV4_TILE_BYTES; }
static char* kv4_layer(const bt_config* c, const bt_block_cache_kv4* cache, int layer)
{
    return (char*)cache->kv + kv4_slab_bytes(c) * c->batch * c->heads * layer;
}

static void fill_kv4_args(bt::Kv4Args& a, const bt_config* cfg, const bt_block_cache_kv4* cache, int layer, const void* k, const void* v,
                          int64_t stride, int n_rows, uint32_t* dev_status)
{
    a.k = const_cast<void*>(k);
    a.v = const_cast<void*>(v);
    a.stride = stride;
    a.kv = kv4_layer(cfg, cache, layer);
    a.slab_bytes = (int64_t)kv4_slab_bytes(cfg);
    a.len = cache->len + (size_t)layer * cfg->batch;
    a.dev_status = dev_status;
    a.B = cfg->batch;
    a.H = cfg->heads;
    a.hd = cfg->head_dim;
    a.cap = cfg->max_blocks;
    a.n_rows = n_rows;
    a.first = 0;
    a.reset = 0;
}

bt_status bt_block_kv4_append(const bt_config* cfg, bt_block_cache_kv4* cache, int layer, const void* k_new, const void* v_new, int n_new,
                              int64_t src_stride, int reset_first, uint32_t* dev_status, void* stream)
{
    bt_status st = check_kv4(cfg, cache, layer);
    if (st != BT_OK) return st;
    if (!k_new || !v_new) return BT_ERR_NULL;
    if (n_new <= 0 || src_stride < n_new) return BT_ERR_SHAPE;
    if (n_new > cfg->max_blocks) return BT_ERR_CAPACITY;
    if (!kv4_aligned(cache) || !al16(k_new) || !al16(v_new) || !al4(dev_status)) return BT_ERR_UNSUPPORTED;
    bt::Kv4Args a;
    fill_kv4_args(a, cfg, cache, layer, k_new, v_new, src_stride, n_new, dev_status);
    a.reset = reset_first ? 1 : 0;
    return cuda_status(bt::launch_kv4_append(a, (cudaStream_t)stream));
}

bt_status bt_block_kv4_read(const bt_config* cfg, const bt_block_cache_kv4* cache, int layer, int first, int n_rows, void* k_out, void* v_out,
                            int64_t dst_stride, void* stream)
{
    bt_status st = check_kv4(cfg, cache, layer);
    if (st != BT_OK) return st;
    if (!k_out || !v_out) return BT_ERR_NULL;
    if (first < 0 || n_rows <= 0 || dst_stride < n_rows) return BT_ERR_SHAPE;
    if (n_rows > cfg->max_blocks - first) return BT_ERR_CAPACITY;
    if (!kv4_aligned(cache) || !al16(k_out) || !al16(v_out)) return BT_ERR_UNSUPPORTED;
    bt::Kv4Args a;
    fill_kv4_args(a, cfg, cache, layer, k_out, v_out, dst_stride, n_rows, nullptr);
    a.first = first;
    return cuda_status(bt::launch_kv4_read(a, (cudaStream_t)stream));
}

// Ways the row range of a (sequence, head) is cut: enough parts for the kernel's warps (eight on each of 148 SMs; the number
// fixes the workspace, so it does not depend on the device), each of at least 128 rows, or of 64 while there are at most 16 (head_dim 128, where a
// warp takes longer for them: 32) parts: 32 pairs of 512 rows of 64 4.5 us in eight parts, 4.8 in four; 16 pairs of 4096 5.3 us in 32, 6.2 in 64; 16 pairs
// of 2048 of 128 5.8 us in 32, 6.2 in 16.  32 parts are joined in one go; more are worth it only for 256 rows each (8 pairs of 16384 rows of 128: 9.4 us
// in 64, 11.6 in 32; of 8192: 8.6, 8.4).  Joining costs 2 us and more, as long as a warp takes for seven times 64 rows at head_dim 64 and for
// five times at 128: where cutting does not save a warp as many, nothing is cut (512 pairs of 512 rows of 64: 6.2 us, in two parts 7.7; 64 pairs of
// 200 to 256: 4.0 us, in four 4.5; 256 pairs of 1024, which gain: 9.4 us, in four 7.5).
static int kv4_splits(const bt_config* cfg)
{
    if (cfg->decode_splits > 0) return cfg->decode_splits;
    long long s = 8 * 148 / ((long long)cfg->batch * cfg->heads);
    const long long units = cfg->max_blocks / 64, short_parts = cfg->head_dim == 64 ? 16 : 32;
    const long long few = units < short_parts ? units : short_parts;
    const long long most = units / 2 > few ? units / 2 : few;
    if (s > most) s = most;
    if (s > 32 && s > units / 4) s = units / 4 > 32 ? units / 4 : 32;
    if (s > 64) s = 64;
    return s < 1 || units * (s - 1) < (cfg->head_dim == 64 ? 7 : 5) * s ? 1 : (int)s;
}

size_t bt_workspace_bytes_kv4(const bt_config* cfg)
{
    if (check_config(cfg, 0) != BT_OK) return 0;
    const int s = kv4_splits(cfg);
    return align16(bt_workspace_bytes(cfg)) + (s <= 1 ? 0 : (size_t)s * cfg->batch * cfg->heads * (cfg->head_dim + 4) * sizeof(float));
}

static bt_status decode_kv4(const bt_config* cfg, const bt_block_cache_kv4* cache, int layer, const void* q, const void* k_new, const void* v_new,
                            bool step, void* out, void* workspace, size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    bt_status st = check_kv4(cfg, cache, layer);
    if (st != BT_OK) return st;
    if (!q || !out || (step && (!k_new || !v_new))) return BT_ERR_NULL;
    if (!workspace || workspace_bytes < bt_workspace_bytes_kv4(cfg)) return BT_ERR_WORKSPACE;
    if (!kv4_aligned(cache) || !al16(q) || !al16(out) || !al16(k_new) || !al16(v_new) || !al16(workspace) || !al4(dev_status)) return BT_ERR_UNSUPPORTED;
    bt::Kv4DecodeArgs a = {};
    a.q = q;
    a.kv = kv4_layer(cfg, cache, layer);
    a.slab_bytes = (int64_t)kv4_slab_bytes(cfg);
    a.len = cache->len + (size_t)layer * cfg->batch;
    a.out = out;
    a.ws = (float*)((char*)workspace + align16(bt_workspace_bytes(cfg)));
    a.counters = (int32_t*)((char*)workspace + partial_bytes(cfg));
    a.k_new = k_new;
    a.v_new = v_new;
    a.dev_status = dev_status;
    a.B = cfg->batch;
    a.H = cfg->heads;
    a.hd = cfg->head_dim;
    a.n_max = cfg->max_blocks;
    a.splits = kv4_splits(cfg);
    a.scale_log2 = scale_log2(cfg);
    return cuda_status(bt::launch_block_decode_kv4(a, (cudaStream_t)stream));
}

bt_status bt_block_decode_attn_kv4(const bt_config* cfg, const bt_block_cache_kv4* cache, int layer, const void* q, void* out, void* workspace,
                                   size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    return decode_kv4(cfg, cache, layer, q, nullptr, nullptr, false, out, workspace, workspace_bytes, dev_status, stream);
}

bt_status bt_block_decode_step_kv4(const bt_config* cfg, bt_block_cache_kv4* cache, int layer, const void* q, const void* k_new, const void* v_new,
                                   void* out, void* workspace, size_t workspace_bytes, uint32_t* dev_status, void* stream)
{
    return decode_kv4(cfg, cache, layer, q, k_new, v_new, true, out, workspace, workspace_bytes, dev_status, stream);
}

// ---- the linear maps either side of the attention path

// What is multiplied: bf16 x and w, or 8-bit integers with their steps.
struct Operands {
    const void* x;
    const void* w;
    const void* bias;
    bool int8;
    const float* x_steps;
    const float* w_steps;
};

static bt_status project_common(const bt_config* cfg, const Operands& op, const void* out, const uint32_t* dev_status)
{
    if (!op.x || !op.w || !out || (op.int8 && (!op.x_steps || !op.w_steps))) return BT_ERR_NULL;
    if (!al16(op.x) || !al16(op.w) || !al16(op.bias) || !al16(op.x_steps) || !al16(op.w_steps) || !al16(out) || !al4(dev_status))
        return BT_ERR_UNSUPPORTED;
    if ((long long)cfg->heads * cfg->head_dim > (1 << 20)) return BT_ERR_UNSUPPORTED;
    return BT_OK;
}

static void fill_project_args(bt::ProjectArgs& a, const Operands& op, void* out, uint32_t* dev_status)
{
    a.x = op.x;
    a.w = op.w;
    a.bias = op.bias;
    a.x_steps = op.x_steps;
    a.w_steps = op.w_steps;
    a.out = out;
    a.dev_status = dev_status;
}

static bt_status prefix_project(const bt_config* cfg, const Operands& op, void* prefix_out, uint32_t* dev_status, void* stream)
{
    bt_status st = check_config(cfg, 0);
    if (st != BT_OK) return st;
    st = project_common(cfg, op, prefix_out, dev_status);
    if (st != BT_OK) return st;
    const long long D = (long long)cfg->heads * cfg->head_dim;
    if (D * cfg->prefix_len > 0x7fffffffLL) return BT_ERR_UNSUPPORTED;
    bt::ProjectArgs a = {};
    fill_project_args(a, op, prefix_out, dev_status);
    a.M = cfg->batch;
    a.K = (int)D;
    a.N = (int)(D * cfg->prefix_len);
    a.mode = bt::kProjectPlain;
    if (!bt::project_supported(a)) return BT_ERR_UNSUPPORTED;
    return cuda_status(bt::launch_project(a, (cudaStream_t)stream));
}

static bt_status qkv_project(const bt_config* cfg, int mode, const bt::CacheView& view, const Operands& op, int n_rows, int reset_first,
                             const uint8_t* reset_mask, void* q_out, uint32_t* dev_status, void* stream)
{
    const long long D = (long long)cfg->heads * cfg->head_dim;
    if ((long long)cfg->batch * n_rows > 0x7fffffffLL / 2 || 3 * D > 0x7fffffffLL) return BT_ERR_UNSUPPORTED;
    bt::ProjectArgs a = {};
    fill_project_args(a, op, q_out, dev_status);
    a.M = cfg->batch * n_rows;
    a.K = (int)D;
    a.N = (int)(3 * D);
    a.mode = mode;
    a.cache = view;
    a.n_rows = n_rows;
    a.H = cfg->heads;
    a.hd = cfg->head_dim;
    a.reset_first = reset_first ? 1 : 0;
    a.reset_mask = reset_mask;
    if (!bt::project_supported(a)) return BT_ERR_UNSUPPORTED;
    return cuda_status(bt::launch_project(a, (cudaStream_t)stream));
}

static bt_status block_qkv_project(const bt_config* cfg, const bt_block_cache* cache, int layer, const Operands& op, int n_rows, void* q_out,
                                   uint32_t* dev_status, void* stream)
{
    bt_status st = check_config(cfg, layer);
    if (st != BT_OK) return st;
    if (!cache || !cache->k || !cache->v || !cache->len) return BT_ERR_NULL;
    st = project_common(cfg, op, q_out, dev_status);
    if (st != BT_OK) return st;
    if (n_rows <= 0) return BT_ERR_SHAPE;
    if (n_rows > cfg->max_blocks) return BT_ERR_CAPACITY;
    if (!block_cache_aligned(cache)) return BT_ERR_UNSUPPORTED;
    return qkv_project(cfg, bt::kProjectQkv, block_view(cfg, cache, layer), op, n_rows, 0, nullptr, q_out, dev_status, stream);
}

static bt_status local_qkv_project(const bt_config* cfg, const bt_local_cache* cache, int layer, const Operands& op, int n_rows, int reset_first,
                                   const uint8_t* reset_mask, void* q_out, uint32_t* dev_status, void* stream)
{
    bt_status st = check_config(cfg, layer);
    if (st != BT_OK) return st;
    if (!cache || !cache->kv || !cache->len) return BT_ERR_NULL;
    st = project_common(cfg, op, q_out, dev_status);
    if (st != BT_OK) return st;
    if (n_rows <= 0) return BT_ERR_SHAPE;
    if (n_rows > local_cap(cfg)) return BT_ERR_CAPACITY;
    if (!local_cache_aligned(cache)) return BT_ERR_UNSUPPORTED;
    return qkv_project(cfg, bt::kProjectQkv, local_view(cfg, cache, layer), op, n_rows, reset_first, reset_mask, q_out, dev_status, stream);
}

static bt_status kv4_qkv_project(const bt_config* cfg, const bt_block_cache_kv4* cache, int layer, const Operands& op, int n_rows, void* q_out,
                                 uint32_t* dev_status, void* stream)
{
    bt_status st = check_kv4(cfg, cache, layer);
    if (st != BT_OK) return st;
    st = project_common(cfg, op, q_out, dev_status);
    if (st != BT_OK) return st;
    if (n_rows <= 0) return BT_ERR_SHAPE;
    if (n_rows > cfg->max_blocks) return BT_ERR_CAPACITY;
    if (!kv4_aligned(cache)) return BT_ERR_UNSUPPORTED;
    bt::CacheView v = {};
    v.k = kv4_layer(cfg, cache, layer);
    v.len = cache->len + (size_t)layer * cfg->batch;
    v.slab_stride = (int64_t)kv4_slab_bytes(cfg);
    v.cap = cfg->max_blocks;
    return qkv_project(cfg, bt::kProjectQkvKv4, v, op, n_rows, 0, nullptr, q_out, dev_status, stream);
}

bt_status bt_prefix_project(const bt_config* cfg, const void* ctx, const void* w_prefix, const void* bias, void* prefix_out,
                            uint32_t* dev_status, void* stream)
{
    return prefix_project(cfg, {ctx, w_prefix, bias, false, nullptr, nullptr}, prefix_out, dev_status, stream);
}

bt_status bt_block_qkv_project_append(const bt_config* cfg, bt_block_cache* cache, int layer, const void* x, int n_rows,
                                      const void* w_qkv, const void* bias, void* q_out, uint32_t* dev_status, void* stream)
{
    return block_qkv_project(cfg, cache, layer, {x, w_qkv, bias, false, nullptr, nullptr}, n_rows, q_out, dev_status, stream);
}

bt_status bt_local_qkv_project_append(const bt_config* cfg, bt_local_cache* cache, int layer, const void* x, int n_rows,
                                      const void* w_qkv, const void* bias, int reset_first, const uint8_t* reset_mask,
                                      void* q_out, uint32_t* dev_status, void* stream)
{
    return local_qkv_project(cfg, cache, layer, {x, w_qkv, bias, false, nullptr, nullptr}, n_rows, reset_first, reset_mask, q_out, dev_status,
                             stream);
}

bt_status bt_block_qkv_project_append_kv4(const bt_config* cfg, bt_block_cache_kv4* cache, int layer, const void* x, int n_rows,
                                          const void* w_qkv, const void* bias, void* q_out, uint32_t* dev_status, void* stream)
{
    return kv4_qkv_project(cfg, cache, layer, {x, w_qkv, bias, false, nullptr, nullptr}, n_rows, q_out, dev_status, stream);
}

bt_status bt_rows_quantize_i8(const void* x, int64_t n_rows, int n_cols, void* x8, float* steps, void* stream)
{
    if (!x || !x8 || !steps) return BT_ERR_NULL;
    if (n_rows <= 0 || n_cols <= 0) return BT_ERR_SHAPE;
    if (n_cols % 16 != 0 || n_cols > bt::kQuantizeCols || n_rows > 0x7fffffffLL || !al16(x) || !al16(x8) || !al4(steps)) return BT_ERR_UNSUPPORTED;
    return cuda_status(bt::launch_rows_quantize(x, n_rows, n_cols, x8, steps, (cudaStream_t)stream));
}

bt_status bt_prefix_project_i8(const bt_config* cfg, const void* ctx8, const float* ctx_steps, const void* w8, const float* w_steps,
                               const void* bias, void* prefix_out, uint32_t* dev_status, void* stream)
{
    return prefix_project(cfg, {ctx8, w8, bias, true, ctx_steps, w_steps}, prefix_out, dev_status, stream);
}

bt_status bt_block_qkv_project_append_i8(const bt_config* cfg, bt_block_cache* cache, int layer, const void* x8, const float* x_steps, int n_rows,
                                         const void* w8, const float* w_steps, const void* bias, void* q_out, uint32_t* dev_status, void* stream)
{
    return block_qkv_project(cfg, cache, layer, {x8, w8, bias, true, x_steps, w_steps}, n_rows, q_out, dev_status, stream);
}

bt_status bt_local_qkv_project_append_i8(const bt_config* cfg, bt_local_cache* cache, int layer, const void* x8, const float* x_steps, int n_rows,
                                         const void* w8, const float* w_steps, const void* bias, int reset_first, const uint8_t* reset_mask,
                                         void* q_out, uint32_t* dev_status, void* stream)
{
    return local_qkv_project(cfg, cache, layer, {x8, w8, bias, true, x_steps, w_steps}, n_rows, reset_first, reset_mask, q_out, dev_status, stream);
}

bt_status bt_block_qkv_project_append_i8_kv4(const bt_config* cfg, bt_block_cache_kv4* cache, int layer, const void* x8, const float* x_steps,
                                             int n_rows, const void* w8, const float* w_steps, const void* bias, void* q_out,
                                             uint32_t* dev_status, void* stream)
{
    return kv4_qkv_project(cfg, cache, layer, {x8, w8, bias, true, x_steps, w_steps}, n_rows, q_out, dev_status, stream);
}

bt_status bt_selftest_bounded_wait(uint32_t* report, uint32_t* dev_status, void* stream)
{
    if (!dev_status) return BT_ERR_NULL;
    if (!al4(report) || !al4(dev_status)) return BT_ERR_UNSUPPORTED;
    return cuda_status(bt::launch_selftest_bounded_wait(report, dev_status, (cudaStream_t)stream));
}

}  // extern "C"
