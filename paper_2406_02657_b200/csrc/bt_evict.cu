// bt_block_kv_evict: per (sequence, head), keep the first rows, the last rows and those with the largest summed
// attention weights, in their order, and move them together.
//
// Selection (select_rows, by one CTA) works on order-preserving 32-bit keys in registers and finds the smallest key that
// stays.  Ties go to the lowest index, so the result does not depend on the order of any atomic.  A histogram of the keys' first
// digit finds the bin that the smallest key lies in.  The digit is 12 bits (10 in the fused kernel, whose shared memory is smaller), which holds
// the exponent and some mantissa: real sums crowd into few exponents, and with an 8-bit digit the lanes of a warp met in the same
// bins (35 us for 16384 rows; bisection with a barrier per step took as long).  If no more keys fell into that bin than the CTA has
// threads - the usual case - they are gathered, one per thread, and the rest goes bit by bit, a counting barrier each, until the
// count is the number wanted.  Else (many equal or close sums) the next digit of the keys in the bin is taken the same way, down to
// the last bits.  Counts per thread, scanned, then place every row.
//
// Moving: rows travel in 16-byte pieces through registers.  Into another cache all pieces are independent.  In place, row
// i of the result comes from row list[i] >= i, and list grows: a chunk is read, its readers meet, and only then is it
// written.  What a chunk writes (rows <= its own sources) is below every source of a later chunk, so one barrier per
// chunk is enough.
//
// Two shapes.  Many (sequence, head) pairs with short caches: a CTA of 128 threads selects and moves a pair, one launch
// (evict_fused_kernel).  Else a launch with a CTA per pair selects, and a second one moves with several CTAs per pair - in place, a
// cluster of them that meets once per chunk.  Into another cache, with few pairs, the first launch has a second CTA per pair that
// moves the last rows meanwhile (evict_select_move_kernel).
//
// Bound by HBM: the kept rows are read and written once, the sums read once.
#include "bt_common.cuh"
#include "bt_device.h"
#include "bt_kernels.h"

namespace bt {
namespace ev {

constexpr int kMoveThreads = 256;
constexpr int kSelectThreads = 1024;
constexpr int kKeys = 16;         // rows a thread holds in a selection round
constexpr int kUnroll = 4;        // rows a thread moves per chunk (of K and of V each)
constexpr int kSelectBits = 12;
constexpr int kFusedThreads = 128, kFusedKeys = 8, kFusedBits = 10, kFusedRows = kFusedThreads * kFusedKeys;

// Larger sum <=> larger key.  -0 counts as +0; a NaN is below everything.
__device__ __forceinline__ uint32_t key_of(float x)
{
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

template <int THREADS, int BITS>
struct SelectSmem {
    uint32_t hist[1 << BITS];
    uint32_t cand[THREADS];
    uint32_t warp_sum[32];
    uint32_t key, left, in_bin, n_cand;
};

// Writes the list of rows that stay: rows outside [lo, hi) and the `want` (< hi - lo) largest of those inside.  All
// threads of the CTA call it; the list is complete for them after the caller's next barrier.  A thread owns KEYS
// neighbouring rows per round of KEYS * THREADS.
template <int THREADS, int KEYS, int BITS>
__device__ __forceinline__ void select_rows(const float* w, int n, int lo, int hi, int want, int32_t* list, SelectSmem<THREADS, BITS>& sm)
{
    constexpr int ROUND = THREADS * KEYS, BINS = 1 << BITS, PER = BINS / THREADS;
    static_assert(ROUND < 65536, "the packed counts hold 16 bits each");
    static_assert(THREADS <= 1024 && PER * THREADS == BINS && KEYS % 4 == 0 && KEYS <= 32, "");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool vec = (reinterpret_cast<uintptr_t>(w) & 15) == 0;   // the same for all threads
    uint32_t key[KEYS], in = 0;   // in: which of them compete
    auto load = [&](int base) {
        const int j0 = base + tid * KEYS;
        // bits lo - j0 .. hi - j0 - 1 of the thread's rows
        auto first = [](int x) { return x <= 0 ? 0u : x >= 32 ? ~0u : (1u << x) - 1u; };
        in = first(hi - j0) & ~first(lo - j0) & first(KEYS);
#pragma unroll
        for (int i = 0; i < KEYS; i += 4) {
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (vec && j0 + i + 3 < n) {
                x = *reinterpret_cast<const float4*>(w + j0 + i);
            } else {
                if (j0 + i < n) x.x = w[j0 + i];
                if (j0 + i + 1 < n) x.y = w[j0 + i + 1];
                if (j0 + i + 2 < n) x.z = w[j0 + i + 2];
                if (j0 + i + 3 < n) x.w = w[j0 + i + 3];
            }
            key[i] = key_of(x.x);
            key[i + 1] = key_of(x.y);
            key[i + 2] = key_of(x.z);
            key[i + 3] = key_of(x.w);
        }
    };
    // exclusive sum over the threads in order; sm.warp_sum is free again after the caller's next barrier
    auto scan = [&](uint32_t mine, uint32_t& total) {
        uint32_t incl = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += v;
        }
        if (lane == 31) sm.warp_sum[warp] = incl;
        __syncthreads();
        const uint32_t ws = lane < THREADS / 32 ? sm.warp_sum[lane] : 0u;
        total = __reduce_add_sync(0xffffffffu, ws);
        return incl - mine + __reduce_add_sync(0xffffffffu, lane < warp ? ws : 0u);
    };
    const bool one_round = n <= ROUND;
    if (one_round) load(0);
    // rows with a key above `stay` stay for sure, and the first `left` of those equal to it
    uint32_t stay = 0xffffffffu, left = (uint32_t)want, prefix = 0;
    int shift = 32;
    while (want > 0 && shift > 0) {   // one digit at a time from the top
        const int bits = shift < BITS ? shift : BITS, above = shift;
        shift -= bits;
        for (int i = tid; i < BINS; i += THREADS) sm.hist[i] = 0;
        if (tid == 0) sm.n_cand = 0;
        __syncthreads();
        for (int base = 0; base < n; base += ROUND) {
            if (!one_round) load(base);
#pragma unroll
            for (int i = 0; i < KEYS; ++i) {
                const bool counts = (in >> i & 1u) && (above == 32 || (key[i] >> above) == (prefix >> above));
                if (__any_sync(0xffffffffu, counts)) {
                    const uint32_t digit = counts ? (key[i] >> shift) & (uint32_t)(BINS - 1) : ~0u;
                    // a warp's run of equal digits (equal sums, often zeros) counts at once
                    const bool run = __all_sync(0xffffffffu, digit == __shfl_sync(0xffffffffu, digit, 0));
                    if (counts && (!run || lane == 0)) atomicAdd(&sm.hist[digit & (uint32_t)((1 << bits) - 1)], run ? 32u : 1u);
                }
            }
        }
        __syncthreads();
        // thread t has bins BINS - 1 - t * PER, downwards
        const int b0 = BINS - 1 - tid * PER;
        uint32_t sum = 0, total;
#pragma unroll
        for (int i = 0; i < PER; ++i) sum += sm.hist[b0 - i];
        uint32_t before = scan(sum, total);
        if (before < left && left <= before + sum) {    // one thread of the CTA
            for (int i = 0; i < PER; ++i) {
                const uint32_t c = sm.hist[b0 - i];
                if (left <= before + c) {
                    sm.key = prefix | ((uint32_t)(b0 - i) << shift);
                    sm.left = left - before;
                    sm.in_bin = c;
                    break;
                }
                before += c;
            }
        }
        __syncthreads();
        prefix = sm.key;
        left = sm.left;
        const uint32_t in_bin = sm.in_bin;
        if (in_bin == left && prefix != 0u) {   // the bin stays whole: everything from its first key up
            stay = prefix - 1;
            left = 0;
            break;
        }
        if (shift == 0) {
            stay = prefix;
        } else if (in_bin <= THREADS) {         // few enough for one key per thread: the rest bit by bit
            for (int base = 0; base < n; base += ROUND) {
                if (!one_round) load(base);
#pragma unroll
                for (int i = 0; i < KEYS; ++i)
                    if ((in >> i & 1u) && (key[i] >> shift) == (prefix >> shift)) sm.cand[atomicAdd(&sm.n_cand, 1u)] = key[i];
            }
            __syncthreads();
            const bool have = tid < (int)in_bin;
            const uint32_t mine = have ? sm.cand[tid] : 0u;
            uint32_t t = prefix;
            bool exact = false;
            for (uint32_t bit = 1u << (shift - 1); bit && !exact; bit >>= 1) {
                const uint32_t c = (uint32_t)__syncthreads_count(have && mine >= (t | bit));
                if (c >= left) t |= bit;
                exact = c == left;              // the keys >= t are the ones: no need to know the smallest of them
            }
            stay = exact ? t - 1 : t;
            left = exact ? 0u : left - (uint32_t)__syncthreads_count(have && mine > t);
            break;
        }
    }
    uint32_t sure_before = 0, eq_before = 0;    // rows of earlier rounds
    for (int base = 0; base < n; base += ROUND) {
        if (!one_round) load(base);
        const int j0 = base + tid * KEYS;
        uint32_t sure = 0, eq = 0;
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            sure |= (key[i] > stay ? 1u : 0u) << i;
            eq |= (key[i] == stay ? 1u : 0u) << i;
        }
        const uint32_t exists = n - j0 >= KEYS ? (KEYS == 32 ? ~0u : (1u << (KEYS & 31)) - 1u) : n - j0 <= 0 ? 0u : (1u << (n - j0)) - 1u;
        sure = exists & (~in | sure);
        eq = left > 0 ? in & eq : 0u;
        uint32_t total;
        const uint32_t at = scan((uint32_t)__popc(sure) << 16 | (uint32_t)__popc(eq), total);
        uint32_t eq_rank = eq_before + (at & 0xffffu), pos = sure_before + (at >> 16) + min(eq_rank, left);
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const bool e = eq >> i & 1u;
            if ((sure >> i & 1u) || (e && eq_rank < left)) list[pos++] = j0 + i;
            eq_rank += e ? 1u : 0u;
        }
        sure_before += total >> 16;
        eq_before += total & 0xffffu;
        if (!one_round) __syncthreads();        // the next round's scan reuses the sums
    }
}

struct Pair {
    int bh, b, n;
    bool cut;
};
// The CTA's pair.  One thread reads the length for all: in place it changes as soon as every pair of the sequence has been
// counted in (settle_length), and a thread of its own CTA must not read it after that.
__device__ __forceinline__ Pair pair_of_cta(const EvictArgs& a, int bh)
{
    __shared__ int rows;
    Pair p;
    p.bh = bh;
    p.b = bh / a.H;
    if (threadIdx.x == 0) {
        const int n = a.len[p.b];
        rows = n < 0 ? 0 : (n > a.n_max ? a.n_max : n);
    }
    __syncthreads();
    p.n = rows;
    p.cut = p.n >= a.trigger && p.n > a.n_keep;
    return p;
}
// The same where nothing changes the length.
__device__ __forceinline__ Pair pair_of(const EvictArgs& a, int bh)
{
    Pair p;
    p.bh = bh;
    p.b = bh / a.H;
    const int n = a.len[p.b];
    p.n = n < 0 ? 0 : (n > a.n_max ? a.n_max : n);
    p.cut = p.n >= a.trigger && p.n > a.n_keep;
    return p;
}

// New length of the pair's sequence.  In place it changes once all heads have read the old one: whoever arrives last
// writes it.  (One thread of one CTA per pair.)
__device__ __forceinline__ void settle_length(const EvictArgs& a, const Pair& p)
{
    if (a.in_place) {
        int one;
        asm volatile("and.b32 %0, %1, 0;\n\tadd.s32 %0, %0, 1;" : "=r"(one) : "r"(p.n));   // issued after that read has returned
        if (atomicAdd(a.counters + p.b, one) == a.H - 1) {
            a.counters[p.b] = 0;
            if (p.cut) a.dst_len[p.b] = a.n_keep;
        }
    } else if (p.bh == p.b * a.H) {
        a.dst_len[p.b] = p.cut ? a.n_keep : min(p.n, a.dst_max);
    }
}

// Moves rows d0 .. d1 - 1 of the pair's result with a group of THREADS threads (this one is `tid`): row i comes from row list[i],
// or without a list from row i + shift.  In place, group `rank` of `ctas` takes every ctas-th chunk, and `meet` is their barrier.
template <int HD, bool IN_PLACE, int THREADS, class Meet>
__device__ __forceinline__ void move_rows(const EvictArgs& a, const int32_t* list, int shift, int bh, int d0, int d1, int rank, int ctas, int tid, Meet meet)
{
    using G = RowGeo<HD>;
    constexpr int ROWS = THREADS / G::LPR;      // rows one pass of the group covers
    constexpr int CHUNK = ROWS * kUnroll;
    static_assert(CHUNK <= THREADS, "a thread carries one sum");
    const int sub = tid % G::LPR, rg = tid / G::LPR;
    const bf16* K = reinterpret_cast<const bf16*>(a.k) + (size_t)bh * a.n_max * HD + sub * 8;
    const bf16* V = reinterpret_cast<const bf16*>(a.v) + (size_t)bh * a.n_max * HD + sub * 8;
    bf16* DK = reinterpret_cast<bf16*>(a.dst_k) + (size_t)bh * a.dst_max * HD + sub * 8;
    bf16* DV = reinterpret_cast<bf16*>(a.dst_v) + (size_t)bh * a.dst_max * HD + sub * 8;
    const float* w = a.w + (size_t)bh * a.n_max;
    float* dw = a.dst_w + (size_t)bh * a.dst_max;
    for (int r0 = d0; r0 < d1; r0 += CHUNK * ctas) {
        const int c0 = r0 + rank * CHUNK;
        uint4 kr[kUnroll], vr[kUnroll];
        int src[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int i = c0 + u * ROWS + rg;
            src[u] = i < d1 ? (list != nullptr ? list[i] : i + shift) : -1;
            if (IN_PLACE && src[u] == i) src[u] = -1;   // already where it belongs
        }
        const int wi = c0 + tid;
        const bool has_w = tid < CHUNK && wi < d1;
        const int wsrc = has_w ? (list != nullptr ? list[wi] : wi + shift) : 0;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (src[u] >= 0) {
                kr[u] = *reinterpret_cast<const uint4*>(K + (size_t)src[u] * HD);
                vr[u] = *reinterpret_cast<const uint4*>(V + (size_t)src[u] * HD);
            }
        const float wr = has_w ? w[wsrc] : 0.f;
        if (IN_PLACE) meet();
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (src[u] >= 0) {
                const size_t i = (size_t)(c0 + u * ROWS + rg) * HD;
                *reinterpret_cast<uint4*>(DK + i) = kr[u];
                *reinterpret_cast<uint4*>(DV + i) = vr[u];
            }
        if (has_w) dw[wi] = wr;
    }
}

// ---- many pairs, short caches: one CTA per pair, one launch
template <int HD, bool IN_PLACE>
__global__ void __launch_bounds__(kFusedThreads, 1024 / kFusedThreads) evict_fused_kernel(EvictArgs a)
{
    __shared__ SelectSmem<kFusedThreads, kFusedBits> sm;
    __shared__ int32_t list[kFusedRows];
    pdl_launch_dependents();
    pdl_wait();
    const Pair p = pair_of_cta(a, blockIdx.x);
    if (threadIdx.x == 0) settle_length(a, p);
    int32_t* kept = a.kept + (size_t)p.bh * a.n_keep;
    if (p.cut) {
        select_rows<kFusedThreads, kFusedKeys, kFusedBits>(a.w + (size_t)p.bh * a.n_max, p.n, a.n_sinks, p.n - a.n_recent, a.n_keep - a.n_sinks - a.n_recent, list, sm);
        __syncthreads();
        for (int i = threadIdx.x; i < a.n_keep; i += kFusedThreads) kept[i] = list[i];
    } else {
        for (int i = threadIdx.x; i < a.n_keep; i += kFusedThreads) kept[i] = -1;
        if (IN_PLACE) return;
    }
    move_rows<HD, IN_PLACE, kFusedThreads>(a, p.cut ? list : nullptr, 0, p.bh, 0, p.cut ? a.n_keep : min(p.n, a.dst_max), 0, 1, threadIdx.x, [] { __syncthreads(); });
}

// ---- few pairs or long caches: select, then move
template <int THREADS>
__device__ __forceinline__ void select_pair(const EvictArgs& a, int bh)
{
    __shared__ SelectSmem<THREADS, kSelectBits> sm;
    const Pair p = pair_of_cta(a, bh);
    if (threadIdx.x == 0) settle_length(a, p);
    int32_t* list = a.kept + (size_t)p.bh * a.n_keep;
    if (p.cut)
        select_rows<THREADS, kKeys, kSelectBits>(a.w + (size_t)p.bh * a.n_max, p.n, a.n_sinks, p.n - a.n_recent, a.n_keep - a.n_sinks - a.n_recent, list, sm);
    else
        for (int i = threadIdx.x; i < a.n_keep; i += THREADS) list[i] = -1;
}

// At 47 or 48 registers a thread the moving launch's CTAs find room beside these before they have ended (in place, 64 pairs: 69 us;
// at 61 registers 83 us).
template <int THREADS>
__global__ void __launch_bounds__(THREADS) evict_select_kernel(EvictArgs a)
{
    pdl_launch_dependents();
    pdl_wait();
    select_pair<THREADS>(a, blockIdx.x);
}

// With one more CTA per pair that moves the pair's last rows meanwhile, which stay whatever the sums; into another cache only.
template <int HD, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == kSelectThreads ? 1 : 4) evict_select_move_kernel(EvictArgs a)
{
    pdl_launch_dependents();
    pdl_wait();
    const int pairs = (int)gridDim.x / 2;
    if ((int)blockIdx.x < pairs) {
        select_pair<THREADS>(a, blockIdx.x);
    } else {
        const Pair p = pair_of(a, blockIdx.x - pairs);
        if (p.cut) move_rows<HD, false, THREADS>(a, nullptr, p.n - a.n_keep, p.bh, a.n_keep - a.n_recent, a.n_keep, 0, 1, threadIdx.x, [] {});
    }
}

// parts CTAs per pair; in place they are a cluster.  The last `moved` rows of a cut sequence are there already.  The list says
// whether the sequence was cut (in place its length has changed by now).
template <int HD, bool IN_PLACE>
__global__ void __launch_bounds__(kMoveThreads, 4) evict_move_kernel(EvictArgs a, int parts, int moved)
{
    pdl_launch_dependents();
    pdl_wait();
    const int bh = blockIdx.x / parts, part = blockIdx.x - bh * parts;
    const int32_t* list = a.kept + (size_t)bh * a.n_keep;
    const bool cut = list[0] >= 0;
    if constexpr (IN_PLACE) {
        if (!cut) return;   // the whole cluster
        move_rows<HD, true, kMoveThreads>(a, list, 0, bh, 0, a.n_keep, part, parts, threadIdx.x, [] {
            asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        });
    } else {
        const int rows = cut ? a.n_keep - moved : min(pair_of(a, bh).n, a.dst_max);
        move_rows<HD, false, kMoveThreads>(a, cut ? list : nullptr, 0, bh, (int)((long long)rows * part / parts), (int)((long long)rows * (part + 1) / parts), 0, 1, threadIdx.x, [] {});
    }
}

constexpr int kMaxCluster = 8;

template <int HD>
static cudaError_t launch_t(const EvictArgs& a, cudaStream_t stream)
{
    int dev = 0, sms = 0;
    cudaError_t e = current_device(&dev, &sms);
    if (e != cudaSuccess) return e;
    const long long pairs = (long long)a.B * a.H;
    if (pairs * kMaxCluster > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    if (pairs >= 4ll * sms && a.n_max <= kFusedRows) {
        if (a.in_place) return launch_pdl(evict_fused_kernel<HD, true>, dim3((unsigned)pairs), dim3(kFusedThreads), 0, stream, a);
        return launch_pdl(evict_fused_kernel<HD, false>, dim3((unsigned)pairs), dim3(kFusedThreads), 0, stream, a);
    }
    // Selecting leaves SMs idle where the pairs are few: they move the rows that stay in any case (60.6 -> 53.8 us at 64 pairs,
    // 4096 of 16384 rows of head_dim 128 kept, 1024 of them the last ones)
    const bool movers = !a.in_place && 2 * pairs <= sms && a.n_recent >= 256;
    const bool small = a.n_max <= kMoveThreads * kKeys;   // enough threads for one round over the sums
    const dim3 grid((unsigned)(movers ? 2 * pairs : pairs)), block(small ? kMoveThreads : kSelectThreads);
    if (movers) e = launch_pdl(small ? evict_select_move_kernel<HD, kMoveThreads> : evict_select_move_kernel<HD, kSelectThreads>, grid, block, 0, stream, a);
    else e = launch_pdl(small ? evict_select_kernel<kMoveThreads> : evict_select_kernel<kSelectThreads>, grid, block, 0, stream, a);
    if (e != cudaSuccess) return e;
    // four CTAs fit an SM; a part is at least one chunk
    constexpr int CHUNK = kMoveThreads / RowGeo<HD>::LPR * kUnroll;
    long long parts = 4ll * sms / pairs;
    if (parts < 1) parts = 1;
    const long long most = (a.n_keep + CHUNK - 1) / CHUNK;
    if (parts > most) parts = most;
    if (!a.in_place) {
        if (pairs * parts > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
        return launch_pdl(evict_move_kernel<HD, false>, dim3((unsigned)(pairs * parts)), dim3(kMoveThreads), 0, stream, a, (int)parts, movers ? a.n_recent : 0);
    }
    int cluster = 1;
    while (cluster < kMaxCluster && cluster < parts) cluster *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(pairs * cluster));
    cfg.blockDim = dim3(kMoveThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, evict_move_kernel<HD, true>, a, cluster, 0);
}

}  // namespace ev

cudaError_t launch_block_kv_evict(const EvictArgs& a, cudaStream_t stream)
{
    return a.hd == 64 ? ev::launch_t<64>(a, stream) : ev::launch_t<128>(a, stream);
}

}  // namespace bt
