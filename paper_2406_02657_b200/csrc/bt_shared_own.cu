// bt_block_decode_attn_shared and bt_block_decode_step_shared: each sequence's own rows, and the join with the partial results
// over the shared prefix.
//
// Own rows: one CTA of four warps per (sequence, head, part of the row range); the warps take alternate passes of
// 4 x (256 / head_dim) rows and meet once, at the end, through shared memory.  (Short caches: a warp each.)  The kernel starts while the prefix kernel
// computes (see the wait there) and streams meanwhile, so it is built to fit beside one of that kernel's CTAs: 64 registers
// a thread and 17 KB of shared memory leave room for four CTAs there and for eight on an SM of their own.  (At that limit every
// form spills a little: 12 to 16 bytes a thread, 40 in the warp-per-pair form, around the pass loop.)  What bounds it
// is bytes in flight, 4 KB a warp in single-buffered slots, and for items of a few dozen rows the instructions around
// them (issue slots 64 % busy).  The whole call, at 512 sequences of up to 256 rows behind 8000 shared ones, 16 heads of 128,
// and at 256 of up to 128 rows behind 2041, heads of 64: 127 and 26.9 us.  On the way there: two slots a warp and six CTAs an SM
// 134 against 130 and 32.3 against 30.2 us; a persistent form with requests running ahead 159 and 32.5 us (twelve warps
// beside the prefix kernel cannot keep enough in flight); the ring of the plain decode calls 145 and 29.9 us (its CTAs need an
// SM each, so the two kernels follow each other).
//
// Join: a CTA that waited for the prefix's partials would keep its place from the next one's rows, so with many
// items each CTA leaves a partial of its own and a third launch folds them all by the log-sum-exp rule (272 or 528 bytes a
// partial, from L2).  Where all CTAs fit the GPU beside the prefix kernel's, they wait and fold at once: a launch less.
#include <type_traits>

#include "bt_common.cuh"
#include "bt_device.h"
#include "bt_kernels.h"
#include "bt_mbarrier.cuh"
#include "bt_shared_parts.cuh"

namespace bt {
namespace own {

using namespace parts;

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kUnroll = 4;      // rows of a lane group per pass, of K and of V
constexpr int kStageBytes = kUnroll * 1024;   // of one pass of a warp
constexpr int kJoinThreads = 256;

// 128-bit load past L1: this grid may start before the one ahead of it in the stream has ended
__device__ __forceinline__ uint4 ld_l2(const void* p)
{
    uint4 r;
    asm volatile("ld.global.cg.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

// 16 bytes each of K and V, global -> shared past L1: a lane's pieces of row U * (rows per pass of a lane group) from k, v on
template <int HD, int U>
__device__ __forceinline__ void copy_pieces(uint32_t slots, const char* k, const char* v, uint64_t policy)
{
    constexpr int AT = U * RowGeo<HD>::RPW * HD * 2;
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0+%3], [%1+%4], 16, %2;" ::"r"(slots), "l"(k), "l"(policy), "n"(U * 1024), "n"(AT) : "memory");
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0+%3], [%1+%4], 16, %2;" ::"r"(slots), "l"(v), "l"(policy), "n"(U * 1024 + 512), "n"(AT) : "memory");
}

template <int HD, bool JOIN, int WPI>
__global__ void __launch_bounds__(kThreads, 8) shared_own_kernel(SharedDecodeArgs a)
{
    constexpr int LPR = RowGeo<HD>::LPR, RPW = RowGeo<HD>::RPW, PASS = RPW * kUnroll, ITEMS = kWarps / WPI;
    __shared__ __align__(16) uint8_t stages[kWarps * kStageBytes];
    __shared__ float sm_state[kWarps - 1][HD + 2];   // WPI > 1: of the item's warps 1 ..: acc, m, l
    const int warp_of_cta = threadIdx.x >> 5, warp = warp_of_cta % WPI;   // warp: of the item
    const int lane = threadIdx.x & 31, sub = lane % LPR, rg = lane / LPR;
    const int item = blockIdx.x * ITEMS + warp_of_cta / WPI, bh = item / a.splits, sp = item - bh * a.splits, b = bh / a.H;
    pdl_launch_dependents();
    if (WPI == kWarps || bh < a.B * a.H) {
        uint64_t policy;   // the rows are read once
        asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
        int n = __ldcg(a.len + b);
        const uint4 qr = ld_l2(reinterpret_cast<const bf16*>(a.q) + (size_t)bh * HD + sub * 8);
        n = n < 0 ? 0 : (n > a.n_max ? a.n_max : n);
        const bool step = a.k_new != nullptr, append = step && n < a.n_max;   // a full cache takes no row: flagged, attended as it is
        float qf[8];
        unpack8(qr, qf);
#pragma unroll
        for (int i = 0; i < 8; ++i) qf[i] *= a.scale_log2;
        SoftmaxState st;
        st.init();
        bf16* K = reinterpret_cast<bf16*>(a.k) + (size_t)bh * a.n_max * HD + sub * 8;
        bf16* V = reinterpret_cast<bf16*>(a.v) + (size_t)bh * a.n_max * HD + sub * 8;
        const int per = a.splits == 1 ? n : (n + a.splits - 1) / a.splits;
        const int first = min(n, sp * per), end = min(n, first + per);
        // Pass p of this warp: rows first + (warp + p * WPI) * PASS ..  A lane copies the 16-byte pieces it will read itself, so nothing
        // but its own copies has to be waited for; its slot u holds its piece of K row u * RPW + rg, then V's.  A pass is requested
        // as soon as the one before it is in registers.
        const uint32_t slots = smem_u32(stages) + warp_of_cta * kStageBytes + lane * 16;
        // A whole pass - the usual one - has no comparison and no address but the first row's.
        auto request = [&](int r0) {
            if (r0 < end) {
                const char* k = reinterpret_cast<const char*>(K + (size_t)(r0 + rg) * HD);
                const char* v = reinterpret_cast<const char*>(V + (size_t)(r0 + rg) * HD);
                const int left = end - r0 - rg;   // rows of this lane group's column that exist from row 0 on, RPW apart
                if (r0 + PASS <= end) {
                    copy_pieces<HD, 0>(slots, k, v, policy);
                    copy_pieces<HD, 1>(slots, k, v, policy);
                    copy_pieces<HD, 2>(slots, k, v, policy);
                    copy_pieces<HD, 3>(slots, k, v, policy);
                } else {
                    if (left > 0) copy_pieces<HD, 0>(slots, k, v, policy);
                    if (left > RPW) copy_pieces<HD, 1>(slots, k, v, policy);
                    if (left > 2 * RPW) copy_pieces<HD, 2>(slots, k, v, policy);
                    if (left > 3 * RPW) copy_pieces<HD, 3>(slots, k, v, policy);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        uint64_t q2[4], acc2[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            q2[i] = pack2(qf[2 * i], qf[2 * i + 1]);
            acc2[i] = pack2(0.f, 0.f);
        }
        auto one_pass = [&](int r0, auto whole) {
            uint4 kr[kUnroll], vr[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                kr[u] = lds128(slots + u * 1024);
                vr[u] = lds128(slots + u * 1024 + 512);
            }
            // The pieces have to be read before their slots are written again.  The empty statement keeps the compiler from moving a read
            // down; what orders the reads before the asynchronous writes is the warp's barrier.
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) asm volatile("" ::"r"(kr[u].x), "r"(vr[u].x) : "memory");
            __syncwarp();
            request(r0 + WPI * PASS);
            float s[kUnroll], mt = kNegInf;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                s[u] = row_sum<LPR>(dot8_x2(q2, kr[u]));
                if (!whole && r0 + u * RPW + rg >= end) {   // no such row: its slots hold anything
                    s[u] = kNegInf;
                    vr[u] = make_uint4(0, 0, 0, 0);
                }
                mt = fmaxf(mt, s[u]);
            }
            const float mn = fmaxf(st.m, mt), m_use = softmax_reference(mn);   // this row group may have no row yet
            const float cf = ex2(st.m - m_use);
            st.l *= cf;
            const uint64_t cf2 = pack2(cf, cf);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc2[i] = fmul2(acc2[i], cf2);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const float p = ex2(s[u] - m_use);
                st.l += p;
                fma8_x2(acc2, p, vr[u]);
            }
            st.m = mn;
        };
        int r0 = first + warp * PASS;
        request(r0);
        for (; r0 < end; r0 += WPI * PASS) {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            if (r0 + PASS <= end) one_pass(r0, std::true_type());
            else one_pass(r0, std::false_type());
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack2(acc2[i], st.acc[2 * i], st.acc[2 * i + 1]);
        st.merge_row_groups<LPR>();
        if constexpr (WPI > 1) {
            static_assert(WPI == kWarps, "the barrier is the CTA's");
            if (warp > 0 && rg == 0) {
                float* mine = sm_state[warp - 1];
#pragma unroll
                for (int i = 0; i < 8; ++i) mine[sub * 8 + i] = st.acc[i];
                if (sub == 0) {
                    mine[HD] = st.m;
                    mine[HD + 1] = st.l;
                }
            }
            __syncthreads();
        }
        if (warp == 0) {
            // the length goes up once all of the sequence's items - every warp of them: hence behind the barrier - have read the old one
            int arrival = -1;
            if (step && lane == 0) arrival = atomicAdd(a.counters + (size_t)a.B * a.H + b, 1);
            if (rg > 0) st.init();
            if constexpr (WPI > 1) {
                for (int w = rg; w < kWarps - 1; w += RPW) {   // row group rg joins warps rg + 1, rg + 1 + RPW, ...
                    float a2[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) a2[i] = sm_state[w][sub * 8 + i];
                    st.merge(sm_state[w][HD], sm_state[w][HD + 1], a2);
                }
            }
            if (append && sp == a.splits - 1) {   // the new row: scored by row group 0 from the caller's buffer, stored into the cache
                const uint4 kn = ld_l2(reinterpret_cast<const bf16*>(a.k_new) + (size_t)bh * HD + sub * 8);
                const uint4 vn = ld_l2(reinterpret_cast<const bf16*>(a.v_new) + (size_t)bh * HD + sub * 8);
                const float sn = row_sum<LPR>(dot8(qf, kn));
                if (rg == 0) {
                    float one_row[8];
                    unpack8(vn, one_row);
                    st.merge(sn, 1.f, one_row);
                    *reinterpret_cast<uint4*>(K + (size_t)n * HD) = kn;
                    *reinterpret_cast<uint4*>(V + (size_t)n * HD) = vn;
                }
            }
            st.merge_row_groups<LPR>();
            float o[8];
            st.normalised(o);
            const int count = a.n_pre + a.splits;
            if constexpr (JOIN) {   // splits == 1
                pdl_wait();         // the prefix's partials are complete and visible from here on
                // this item's own one is the last of them: row group rg folds partials rg, rg + RPW, ...
                const float lse = st.lse();
                st.init();
                const float* all = a.parts + (size_t)bh * count * (HD + 4);
                if (rg < a.n_pre) fold_partials<HD, 4>(st, all + (size_t)rg * (HD + 4), (a.n_pre - rg + RPW - 1) / RPW, RPW, sub);
                if (rg == RPW - 1) st.merge(lse, 1.f, o);
                st.merge_row_groups<LPR>();
                st.normalised(o);
                if (rg == 0) *reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(a.out) + (size_t)bh * HD + sub * 8) = pack8(o);
            } else if (rg == 0) {
                float* mine = a.parts + ((size_t)bh * count + a.n_pre + sp) * (HD + 4);
                *reinterpret_cast<float4*>(mine + sub * 8) = make_float4(o[0], o[1], o[2], o[3]);
                *reinterpret_cast<float4*>(mine + sub * 8 + 4) = make_float4(o[4], o[5], o[6], o[7]);
                if (sub == 0) mine[HD] = st.lse();
            }
            if (lane == 0) {
                if (bh == b * a.H && sp == 0) {
                    if (n == 0 && !append && __ldcg(a.prefix_len) <= 0) raise_status(a.dev_status, BT_DEV_EMPTY);
                    if (step && !append) raise_status(a.dev_status, BT_DEV_OVERFLOW);
                }
                if (arrival == a.H * a.splits - 1) {
                    if (append) a.len[b] = n + 1;
                    a.counters[(size_t)a.B * a.H + b] = 0;
                }
            }
        }
    }
    // this grid's end has to imply the prefix kernel's; one waiting CTA is enough for that
    if (JOIN || blockIdx.x == gridDim.x - 1) pdl_wait();
}

// LPR lanes per (sequence, head)
template <int HD>
__global__ void __launch_bounds__(kJoinThreads) shared_join_kernel(SharedDecodeArgs a)
{
    constexpr int LPR = RowGeo<HD>::LPR;
    pdl_launch_dependents();
    pdl_wait();
    const int bh = blockIdx.x * (kJoinThreads / LPR) + threadIdx.x / LPR, sub = threadIdx.x % LPR;
    if (bh < a.B * a.H) join<HD>(a, bh, sub);
}

template <int HD, bool JOIN, int WPI>
static cudaError_t launch_j(const SharedDecodeArgs& a, int dev, cudaStream_t stream)
{
    constexpr int ITEMS = kWarps / WPI;
    const long long bh = (long long)a.B * a.H, grid = (bh * a.splits + ITEMS - 1) / ITEMS;
    if (grid * ITEMS > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    // the same split between L1 and shared memory as the prefix kernel's, so that both fit an SM
    static PerDeviceOnce carveout_set;
    cudaError_t e = carveout_set.once(dev, []() { return cudaFuncSetAttribute(shared_own_kernel<HD, JOIN, WPI>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared); });
    if (e != cudaSuccess) return e;
    e = launch_pdl(shared_own_kernel<HD, JOIN, WPI>, dim3((unsigned)grid), dim3(kThreads), 0, stream, a);
    if (e != cudaSuccess || JOIN) return e;
    constexpr int PER = kJoinThreads / RowGeo<HD>::LPR;
    return launch_pdl(shared_join_kernel<HD>, dim3((unsigned)((bh + PER - 1) / PER)), dim3(kJoinThreads), 0, stream, a);
}

template <int HD>
static cudaError_t launch_t(const SharedDecodeArgs& a, cudaStream_t stream)
{
    int dev = 0, sms = 0;
    cudaError_t e = current_device(&dev, &sms);
    if (e != cudaSuccess) return e;
    // few enough that all fit beside the prefix kernel's CTAs at once (four a SM): no CTA that waits keeps another one out
    // (11.2 against 13.4 us at 32 pairs; 33.1 against 31.8 us at 4096 pairs of 1 to 128 rows)
    if (a.splits == 1 && (long long)a.B * a.H <= 4ll * sms) return launch_j<HD, true, kWarps>(a, dev, stream);
    // a warp per item while it has at most eight passes (256 x 16 pairs of up to 32 rows behind 2041 shared ones: 19.8 against
    // 24.3 us; 128 rows: 26.8 against 28.0; 256 rows: 38.8 against 35.1)
    constexpr int kShortRows = 8 * RowGeo<HD>::RPW * kUnroll;
    if (a.splits == 1 && a.n_max <= kShortRows) return launch_j<HD, false, 1>(a, dev, stream);
    return launch_j<HD, false, kWarps>(a, dev, stream);
}

}  // namespace own

cudaError_t launch_shared_own(const SharedDecodeArgs& a, cudaStream_t stream)
{
    return a.hd == 64 ? own::launch_t<64>(a, stream) : own::launch_t<128>(a, stream);
}

}  // namespace bt
