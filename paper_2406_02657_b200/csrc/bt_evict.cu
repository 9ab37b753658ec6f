// bt_block_kv_evict: per (sequence, head), keep the first rows, the last rows and those with the largest summed
// attention weights, in their order, and move them together.
//
// A CTA finds the threshold of its (sequence, head) by a radix select over order-preserving 32-bit keys (four passes
// of 8 bits, histograms per warp in shared memory; sums of up to kKeyCache rows stay there as keys), turns it into the
// list of kept rows by two ballot walks (each warp a contiguous piece of rows), and moves the rows in 16-byte pieces.
// Ties go to the lowest index, so the result does not depend on the order of any atomic.
//
// In place, row i of the result comes from row list[i] >= i, and list grows: a chunk of rows is read into
// registers, the CTA meets, and only then is it written.  What chunk c writes (rows <= its own sources) is above no
// source of a later chunk and was read by every earlier one, so one barrier per chunk is enough.
//
// Bound by HBM: the kept rows are read and written once, the sums read once.
#include "bt_common.cuh"
#include "bt_device.h"
#include "bt_kernels.h"

namespace bt {
namespace ev {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kKeyCache = 4096;   // rows whose keys stay in shared memory
constexpr int kUnroll = 4;        // rows a thread moves per chunk (of K and of V each)

// Larger sum <=> larger key.  -0 counts as +0; a NaN is below everything.
__device__ __forceinline__ uint32_t key_of(float x)
{
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

template <int HD, bool IN_PLACE>
__global__ void __launch_bounds__(kThreads) evict_kernel(EvictArgs a, int parts)
{
    __shared__ uint32_t keys[kKeyCache];
    __shared__ uint32_t hist[kWarps][256];
    __shared__ uint32_t sel_key, sel_left;
    __shared__ int seg_sure[kWarps], seg_eq[kWarps];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_launch_dependents();
    pdl_wait();

    const int bh = blockIdx.x / parts, part = blockIdx.x - bh * parts, b = bh / a.H;
    int n = a.len[b];
    n = n < 0 ? 0 : (n > a.n_max ? a.n_max : n);
    const bool cut = n >= a.trigger && n > a.n_keep;
    // In place the length changes once all heads of the sequence have read it: whoever arrives last writes it.
    if (IN_PLACE && tid == 0) {
        int one;
        asm volatile("and.b32 %0, %1, 0;\n\tadd.s32 %0, %0, 1;" : "=r"(one) : "r"(n));   // issued after the read above has returned
        if (atomicAdd(a.counters + b, one) == a.H * parts - 1) {
            a.counters[b] = 0;
            if (cut) a.dst_len[b] = a.n_keep;
        }
    }
    if (!IN_PLACE && tid == 0 && part == 0 && bh == b * a.H) a.dst_len[b] = cut ? a.n_keep : min(n, a.dst_max);

    const int total = cut ? a.n_keep : (IN_PLACE ? 0 : min(n, a.dst_max));   // rows of the result that are written
    const int d0 = (int)((long long)total * part / parts), d1 = (int)((long long)total * (part + 1) / parts);
    const float* w = a.w + (size_t)bh * a.n_max;
    int32_t* list = a.kept + (size_t)bh * a.n_keep;
    if (!cut) {
        for (int i = part * kThreads + tid; i < a.n_keep; i += parts * kThreads) list[i] = -1;
    } else {
        const int lo = a.n_sinks, hi = n - a.n_recent;            // rows that compete
        const int want = a.n_keep - a.n_sinks - a.n_recent;       // how many of them stay: fewer than hi - lo
        const bool cached = n <= kKeyCache;
        auto key_at = [&](int j) { return cached ? keys[j] : key_of(w[j]); };
        if (cached) {
            for (int j = tid; j < n; j += kThreads) keys[j] = key_of(w[j]);
        }
        uint32_t prefix = 0, left = (uint32_t)want;               // the want-th largest key, 8 bits at a time from the top
        if (want > 0) {
            for (int shift = 24; shift >= 0; shift -= 8) {
                for (int i = tid; i < kWarps * 256; i += kThreads) (&hist[0][0])[i] = 0;
                __syncthreads();
                for (int j = lo + tid; j < hi; j += kThreads) {
                    const uint32_t key = key_at(j);
                    if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[warp][(key >> shift) & 255u], 1u);
                }
                __syncthreads();
                if (warp == 0) {   // lane l: bins 255 - 8 l downwards
                    uint32_t c[8], sum = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        c[i] = 0;
                        for (int q = 0; q < kWarps; ++q) c[i] += hist[q][255 - (lane * 8 + i)];
                        sum += c[i];
                    }
                    uint32_t incl = sum;
#pragma unroll
                    for (int off = 1; off < 32; off <<= 1) {
                        const uint32_t t = __shfl_up_sync(0xffffffffu, incl, off);
                        if (lane >= off) incl += t;
                    }
                    uint32_t before = incl - sum;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (before < left && left <= before + c[i]) {
                            sel_key = prefix | ((uint32_t)(255 - (lane * 8 + i)) << shift);
                            sel_left = left - before;
                        }
                        before += c[i];
                    }
                }
                __syncthreads();
                prefix = sel_key;
                left = sel_left;
            }
        }
        __syncthreads();
        // rows above the threshold stay, and the first `left` of those equal to it
        const int seg = ((n + 31) / 32 + kWarps - 1) / kWarps * 32, s0 = min(n, warp * seg), s1 = min(n, s0 + seg);
        auto look = [&](int j, bool& sure, bool& eq) {
            const bool in = j < s1, competes = in && j >= lo && j < hi;
            const uint32_t key = competes ? key_at(j) : 0u;
            sure = in && (!competes || (want > 0 && key > prefix));
            eq = competes && want > 0 && key == prefix;
        };
        int n_sure = 0, n_eq = 0;
        for (int j0 = s0; j0 < s1; j0 += 32) {
            bool sure, eq;
            look(j0 + lane, sure, eq);
            n_sure += __popc(__ballot_sync(0xffffffffu, sure));
            n_eq += __popc(__ballot_sync(0xffffffffu, eq));
        }
        if (lane == 0) {
            seg_sure[warp] = n_sure;
            seg_eq[warp] = n_eq;
        }
        __syncthreads();
        int eq_at = 0, at = 0;
        for (int q = 0; q < warp; ++q) {
            at += seg_sure[q];
            eq_at += seg_eq[q];
        }
        at += min(eq_at, (int)left);
        const uint32_t below = (1u << lane) - 1u;
        for (int j0 = s0; j0 < s1; j0 += 32) {
            bool sure, eq;
            look(j0 + lane, sure, eq);
            const uint32_t eqs = __ballot_sync(0xffffffffu, eq);
            const bool take = sure || (eq && eq_at + __popc(eqs & below) < (int)left);
            const uint32_t taken = __ballot_sync(0xffffffffu, take);
            const int pos = at + __popc(taken & below);
            if (take && pos >= d0 && pos < d1) list[pos] = j0 + lane;
            eq_at += __popc(eqs);
            at += __popc(taken);
        }
        __syncthreads();
    }

    // ---- move rows d0 .. d1 - 1 of the result
    using G = RowGeo<HD>;
    constexpr int ROWS = kThreads / G::LPR;          // rows one pass of the CTA covers
    constexpr int CHUNK = ROWS * kUnroll;
    const int sub = tid % G::LPR, rg = tid / G::LPR;
    const bf16* K = reinterpret_cast<const bf16*>(a.k) + (size_t)bh * a.n_max * HD + sub * 8;
    const bf16* V = reinterpret_cast<const bf16*>(a.v) + (size_t)bh * a.n_max * HD + sub * 8;
    bf16* DK = reinterpret_cast<bf16*>(a.dst_k) + (size_t)bh * a.dst_max * HD + sub * 8;
    bf16* DV = reinterpret_cast<bf16*>(a.dst_v) + (size_t)bh * a.dst_max * HD + sub * 8;
    float* dw = a.dst_w + (size_t)bh * a.dst_max;
    for (int c0 = d0; c0 < d1; c0 += CHUNK) {
        uint4 kr[kUnroll], vr[kUnroll];
        int src[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int i = c0 + u * ROWS + rg;
            src[u] = i < d1 ? (cut ? list[i] : i) : -1;
            if (IN_PLACE && src[u] == i) src[u] = -1;   // already where it belongs
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (src[u] >= 0) {
                kr[u] = *reinterpret_cast<const uint4*>(K + (size_t)src[u] * HD);
                vr[u] = *reinterpret_cast<const uint4*>(V + (size_t)src[u] * HD);
            }
        float wr = 0.f;
        const int wi = c0 + tid;                         // CHUNK <= kThreads: a thread carries one sum
        const bool has_w = tid < CHUNK && wi < d1;
        if (has_w) wr = w[cut ? list[wi] : wi];
        if (IN_PLACE) __syncthreads();
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (src[u] >= 0) {
                const size_t i = (size_t)(c0 + u * ROWS + rg) * HD;
                *reinterpret_cast<uint4*>(DK + i) = kr[u];
                *reinterpret_cast<uint4*>(DV + i) = vr[u];
            }
        if (has_w) dw[wi] = wr;
        static_assert(CHUNK <= kThreads, "one sum per thread");
    }
}

template <int HD>
static cudaError_t launch_t(const EvictArgs& a, cudaStream_t stream)
{
    int dev = 0, sms = 0;
    cudaError_t e = current_device(&dev, &sms);
    if (e != cudaSuccess) return e;
    const long long items = (long long)a.B * a.H;
    long long parts = 1;
    if (!a.in_place) {   // into another cache the parts of a (sequence, head) do not depend on each other
        parts = (4ll * sms + items - 1) / items;
        const long long most = (a.n_keep + 127) / 128;
        if (parts > most) parts = most;
        if (parts < 1) parts = 1;
    }
    if (items * parts > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    if (a.in_place) return launch_pdl(evict_kernel<HD, true>, dim3((unsigned)items), dim3(kThreads), 0, stream, a, 1);
    return launch_pdl(evict_kernel<HD, false>, dim3((unsigned)(items * parts)), dim3(kThreads), 0, stream, a, (int)parts);
}

}  // namespace ev

cudaError_t launch_block_kv_evict(const EvictArgs& a, cudaStream_t stream)
{
    return a.hd == 64 ? ev::launch_t<64>(a, stream) : ev::launch_t<128>(a, stream);
}

}  // namespace bt
