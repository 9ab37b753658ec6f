// Attention of a whole batch over a prefix that every sequence shares: the part of bt_block_decode_attn_shared that
// is a dense product.  Per head the B queries of the batch form a [B x hd] matrix against the S prefix rows, so the
// prefix is read once per 128 sequences instead of once per sequence, and scores and weighted sums run on the
// 5th-generation tensor cores.  The result is a partial softmax state per (sequence, head, part of the prefix) -
// normalised output and log2-sum-exp, fp32 - which is joined with those of the sequence's own rows (bt_shared_own.cu).
//
// One CTA per (head, part, tile of 128 sequences).  The part's 64-row key/value tiles alternate between two softmax
// warpgroups, each with two score buffers and an output accumulator of its own in tensor memory; the two states meet
// through shared memory at the end.  Roles:
//   warps 0-3 / 4-7 : softmax over the even / odd tiles; a thread owns one query row (= one TMEM lane).  The scores
//                     are read twice from tensor memory, 32 columns at a time (once for the maximum, once for the
//                     exponentials), which keeps the kernel at 80 registers a thread (and 36 or 40 bytes spilled), so that
//                     four CTAs of the own-rows kernel fit beside it and both run at the same time.
//   warps 8, 9      : tcgen05.mma issuers of the two warpgroups (S = Q K^T; O += P V with P read from tensor memory)
//   warps 10, 11    : TMA producers of Q and K, and of V (separate rings: a K stage is free once its scores are done)
// The probabilities are rounded to bf16 where they meet V, as in the prefill kernel: one MMA takes operands of one type, and V is
// bf16.  The row sum is taken in fp32 before that.  Each weight is off by 2^-8 of itself at most, the result by 2^-8 of the weighted
// |v|: against 64 bits 2.3e-3 at the sizes below (root mean square of the error over that of the result), where the fp32 weights of
// the streaming kernels leave 1.7e-3, which is the rounding of the result.
// All waits are bounded in wall time.
//
// What bounds it: with 2041 rows a chain of four tiles per warpgroup and the launch around it (12 us of the call's 27 at 256
// sequences, 16 heads of 64); with 8000 rows of head_dim 128 the tensor pipe at 39 % and the softmax chain between its products
// (52 us alone, 512 sequences; about 60 us beside the own rows' stream; that stream is what the call's 127 us are).
#include <cuda.h>

#include "bt_common.cuh"
#include "bt_device.h"
#include "bt_kernels.h"
#include "bt_mbarrier.cuh"
#include "bt_shared_parts.cuh"
#include "bt_tcgen05.cuh"
#include "bt_tensor_map.h"

namespace bt {
namespace sp {

using namespace tc;

constexpr int BM = 128, BN = 64;       // query rows and key/value rows of a tile
constexpr int kQBoxBytes = BM * 128, kKvBoxBytes = BN * 128;
constexpr int kMmaWarp = 8, kKWarp = 10, kVWarp = 11;
constexpr int kThreads = 384;
constexpr int kStages = 2;             // of K, and of V
// Shared memory that lets one CTA on an SM, not two: they would take turns at the SM's tensor memory while other SMs have
// none (calls back to back: 181 vs 145 us at 512 sequences and 8000 rows of head_dim 128, when the ring kernel streamed the own
// rows), and leaves room for the own-rows kernel's CTAs beside it.
constexpr int kSmemOnePerSm = 116 * 1024;
constexpr uint32_t kTmemCols = 512;    // four score buffers of 64 columns, two outputs of head_dim columns
constexpr uint32_t kSpinLimit = 1u << 26;
constexpr uint64_t kWaitLimitNs = 1000000000ull;
constexpr float kRescaleThreshold = 8.0f;   // log2 units: the reference moves only when the maximum grew by more

enum {
    B_QFULL = 0,
    B_KFULL = 1,                      // [kStages]
    B_KEMPTY = B_KFULL + kStages,     // [kStages]
    B_VFULL = B_KEMPTY + kStages,     // [kStages]
    B_VEMPTY = B_VFULL + kStages,     // [kStages]
    B_SFULL = B_VEMPTY + kStages,     // [2 warpgroups][2 buffers]
    B_PFULL = B_SFULL + 4,            // [2][2], 128 arrivals
    B_PVDONE = B_PFULL + 4,           // [2], one completion per product P V
    B_OFULL = B_PVDONE + 2,           // [2], the last product is done
    B_COUNT = B_OFULL + 2
};

template <int HD>
constexpr int smem_bytes()
{
    const int used = 1024 + (HD / 64) * (kQBoxBytes + 2 * kStages * kKvBoxBytes) + 256;
    return used > kSmemOnePerSm ? used : kSmemOnePerSm;
}

__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t* dev_status)
{
    if (mbar_wait_walltime(bar, parity, abort_flag, kSpinLimit, kWaitLimitNs)) return true;
    raise_status(dev_status, BT_DEV_TIMEOUT);
    return false;
}

template <int HD>
__global__ void __launch_bounds__(kThreads, 2)
shared_prefix_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK,
                     const __grid_constant__ CUtensorMap mapV, SharedDecodeArgs a, int n_qtiles)
{
    constexpr int NB = HD / 64;
    constexpr uint32_t Q_TILE_BYTES = NB * kQBoxBytes, KV_TILE_BYTES = NB * kKvBoxBytes;
    constexpr uint32_t IDESC_S = make_idesc(BM, BN, false), IDESC_O = make_idesc(BM, HD, true);
    constexpr uint32_t COL_O0 = 4 * BN;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t sQ = base, sK = sQ + Q_TILE_BYTES, sV = sK + kStages * KV_TILE_BYTES, sBar = sV + kStages * KV_TILE_BYTES;
    uint8_t* gen_tail = gen_base + (sBar - base);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen_tail + B_COUNT * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(gen_tail + B_COUNT * 8 + 8);
    auto bar = [&](int i) { return sBar + 8u * i; };
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < B_COUNT; ++i) mbar_init(bar(i), (i >= B_PFULL && i < B_PFULL + 4) ? 128u : 1u);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (threadIdx.x == kKWarp * 32) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&mapQ) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&mapK) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&mapV) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    // The next launch on the stream is the own-rows kernel, which reads what earlier launches wrote without
    // waiting for THIS one to end.  It may start once every CTA has passed this point, so the wait comes first:
    // everything before this launch is then complete and visible to both.
    pdl_wait();
    pdl_launch_dependents();

    const int qt = blockIdx.x % n_qtiles, hk = blockIdx.x / n_qtiles, part = hk % a.n_pre, h = hk / a.n_pre;
    int rows = *a.prefix_len;
    rows = rows < 0 ? 0 : (rows > a.cap ? a.cap : rows);
    const int n_tiles = (rows + BN - 1) / BN, per = (n_tiles + a.n_pre - 1) / a.n_pre;
    const int t0 = min(n_tiles, part * per), nt = min(n_tiles, t0 + per) - t0;   // this part's tiles t0 .. t0 + nt - 1

    // after a wait that ran out: none of the copies still in flight may land once the CTA is gone
    auto drain = [&](int full, int issued) {
        for (int i = issued > kStages ? issued - kStages : 0; i < issued; ++i)
            mbar_wait_polls(bar(full + i % kStages), (i / kStages) & 1, 1u << 16);
    };

    if (warp == kKWarp) {
        if (lane == 0 && nt > 0) {
            mbar_expect_tx(bar(B_QFULL), Q_TILE_BYTES);
            for (int bx = 0; bx < NB; ++bx) tma_load_3d(sQ + bx * kQBoxBytes, &mapQ, bar(B_QFULL), bx * 64, qt * BM, h);
            int i = 0;
            for (; i < nt; ++i) {
                const uint32_t st = i % kStages;
                if (!mbar_wait(bar(B_KEMPTY + st), ((i / kStages) & 1) ^ 1, abort_flag, a.dev_status)) break;
                mbar_expect_tx(bar(B_KFULL + st), KV_TILE_BYTES);
                for (int bx = 0; bx < NB; ++bx)
                    tma_load_3d(sK + st * KV_TILE_BYTES + bx * kKvBoxBytes, &mapK, bar(B_KFULL + st), bx * 64, (t0 + i) * BN, h);
            }
            if (i < nt) drain(B_KFULL, i);
        }
    } else if (warp == kVWarp) {
        if (lane == 0) {
            int i = 0;
            for (; i < nt; ++i) {
                const uint32_t st = i % kStages;
                if (!mbar_wait(bar(B_VEMPTY + st), ((i / kStages) & 1) ^ 1, abort_flag, a.dev_status)) break;
                mbar_expect_tx(bar(B_VFULL + st), KV_TILE_BYTES);
                for (int bx = 0; bx < NB; ++bx)
                    tma_load_3d(sV + st * KV_TILE_BYTES + bx * kKvBoxBytes, &mapV, bar(B_VFULL + st), bx * 64, (t0 + i) * BN, h);
            }
            if (i < nt) drain(B_VFULL, i);
        }
    } else if (warp >= kMmaWarp) {
        // issuer of warpgroup x: S(0) S(1) | PV(0) S(2) | PV(1) S(3) ...; step k is tile 2k + x
        const int x = warp - kMmaWarp, steps = (nt - x + 1) / 2;
        bool ok = true;
        auto wait_all = [&](uint32_t b, uint32_t parity) {
            return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag, a.dev_status)) != 0;
        };
        auto issue_s = [&](int k) {
            const int i = 2 * k + x;
            const uint32_t st = i % kStages;
            if (ok && k == 0) ok = wait_all(bar(B_QFULL), 0);
            ok = ok && wait_all(bar(B_KFULL + st), (i / kStages) & 1);
            if (!ok) return;
            tc_fence_after();
            const uint32_t qlo = (sQ >> 4) | (1u << 16), klo = ((sK + st * KV_TILE_BYTES) >> 4) | (1u << 16);
            const uint32_t d_s = tmem + (uint32_t)(x * 2 + (k & 1)) * BN;
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < HD / 16; ++kk) {
                    const uint32_t qoff = (uint32_t)(((kk >> 2) * kQBoxBytes + (kk & 3) * 32) >> 4);
                    const uint32_t koff = (uint32_t)(((kk >> 2) * kKvBoxBytes + (kk & 3) * 32) >> 4);
                    mma_bf16(d_s, desc_words(qlo + qoff, kDescHiSw128), desc_words(klo + koff, kDescHiSw128), IDESC_S, kk > 0 ? 1u : 0u);
                }
                mma_commit(bar(B_SFULL + x * 2 + (k & 1)));
                mma_commit(bar(B_KEMPTY + st));
            }
            __syncwarp();
        };
        auto issue_pv = [&](int k) {
            const int i = 2 * k + x;
            const uint32_t st = i % kStages;
            ok = ok && wait_all(bar(B_VFULL + st), (i / kStages) & 1) && wait_all(bar(B_PFULL + x * 2 + (k & 1)), (k >> 1) & 1);
            if (!ok) return;
            tc_fence_after();
            const uint32_t vlo = ((sV + st * KV_TILE_BYTES) >> 4) | ((uint32_t)(kKvBoxBytes >> 4) << 16);
            const uint32_t a_p = tmem + (uint32_t)(x * 2 + (k & 1)) * BN;
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < BN / 16; ++kk)
                    mma_bf16_ts(tmem + COL_O0 + x * HD, a_p + kk * 8, desc_words(vlo + (uint32_t)kk * 128u, kDescHiSw128), IDESC_O, (k > 0 || kk > 0) ? 1u : 0u);
                mma_commit(bar(B_PVDONE + x));
                mma_commit(bar(B_VEMPTY + st));
                if (k == steps - 1) mma_commit(bar(B_OFULL + x));
            }
            __syncwarp();
        };
        if (steps > 0) issue_s(0);
        if (steps > 1) issue_s(1);
        for (int k = 0; ok && k < steps; ++k) {
            issue_pv(k);
            if (k + 2 < steps) issue_s(k + 2);
        }
    } else {
        const int x = warp >> 2, wq = warp & 3, row = wq * 32 + lane, steps = (nt - x + 1) / 2;
        const uint32_t lane_base = tmem + ((uint32_t)(wq * 32) << 16);
        const uint32_t o_addr = lane_base + COL_O0 + x * HD;
        float m_ref = kNegInf, l = 0.f;
        bool ok = true;
        auto warp_wait = [&](uint32_t b, uint32_t parity) {   // one outcome for the warp: tensor-memory loads need all its lanes
            return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag, a.dev_status)) != 0;
        };
        for (int k = 0; k < steps; ++k) {
            const int i = 2 * k + x;
            const uint32_t s_addr = lane_base + (uint32_t)(x * 2 + (k & 1)) * BN;
            const int valid = rows - (t0 + i) * BN;      // columns of this tile that are prefix rows (64 or more: all)
            ok = warp_wait(bar(B_SFULL + x * 2 + (k & 1)), (k >> 1) & 1);
            if (!ok) break;
            tc_fence_after();
            float mx = kNegInf;
#pragma unroll
            for (int c = 0; c < BN; c += 32) {
                float s[32];
                tmem_ld32(s_addr + c, s);
                if (valid < BN) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) s[j] = c + j < valid ? s[j] : kNegInf;
                }
                float m4[4] = {kNegInf, kNegInf, kNegInf, kNegInf};
#pragma unroll
                for (int j = 0; j < 32; ++j) m4[j & 3] = fmaxf(m4[j & 3], s[j]);
                mx = fmaxf(mx, fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])));
            }
            mx *= a.scale_log2;
            float factor = 1.f;
            const bool grow_ref = mx > m_ref + kRescaleThreshold;
            if (grow_ref) {
                factor = m_ref == kNegInf ? 0.f : ex2(m_ref - mx);
                m_ref = mx;
            }
            if (k > 0) {
                if (__any_sync(0xffffffffu, grow_ref)) {
                    // O is complete up to step k - 1 (step k - 2 was, before S(k) was announced: the parity is not stale)
                    ok = warp_wait(bar(B_PVDONE + x), (k - 1) & 1);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < HD; c += 32) {
                        float o[32];
                        tmem_ld32(o_addr + c, o);
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] *= factor;
                        tmem_st32(o_addr + c, o);
                    }
                }
                l *= factor;
            }
            const float m_use = softmax_reference(m_ref);
#pragma unroll
            for (int c = 0; c < BN; c += 32) {
                float s[32];
                uint32_t packed[16];
                tmem_ld32(s_addr + c, s);
                if (valid < BN) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) s[j] = c + j < valid ? s[j] : kNegInf;
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) s[j] = ex2(fmaf(s[j], a.scale_log2, -m_use));
                float l0 = 0.f, l1 = 0.f;
#pragma unroll
                for (int j = 0; j < 32; j += 2) {
                    l0 += s[j];
                    l1 += s[j + 1];
                    __nv_bfloat162 pr = __floats2bfloat162_rn(s[j], s[j + 1]);
                    packed[j >> 1] = *reinterpret_cast<uint32_t*>(&pr);
                }
                l += l0 + l1;
                tmem_st16(s_addr + (c >> 1), packed);
            }
            if (valid < BN) {
                // rows past the prefix may hold anything, and 0 x NaN is NaN: clear them before the product reads them
                const uint32_t st = i % kStages;
                // ... once they are there: the stage's last use is over with P V of step k - 1, and only then is the parity
                // of its barrier this tile's
                if (k > 0) ok = warp_wait(bar(B_PVDONE + x), (k - 1) & 1);
                ok = ok && warp_wait(bar(B_VFULL + st), (i / kStages) & 1);
                if (!ok) break;
                const int pieces = (BN - valid) * 8;
                for (int bx = 0; bx < NB; ++bx)
                    for (int p = row; p < pieces; p += 128)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(sV + st * KV_TILE_BYTES + bx * kKvBoxBytes + valid * 128 + p * 16), "r"(0u) : "memory");
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(bar(B_PFULL + x * 2 + (k & 1)));
        }
        if (ok && steps > 0) ok = warp_wait(bar(B_OFULL + x), 0);
        tc_fence_after();
        // Both warpgroups are past their products (nothing reads Q, K or V any more): the states meet in the K and V
        // area.  Warpgroup x finishes output columns x * HD/2 ..; it hands the other half over.  Float4 c4 of
        // row r lies at (c4 * 128 + r) * 16: conflict-free.
        constexpr int HALF = HD / 2;
        float4* mine = reinterpret_cast<float4*>(gen_base + Q_TILE_BYTES) + x * (HALF / 4) * BM;          // written here
        const float4* theirs = reinterpret_cast<float4*>(gen_base + Q_TILE_BYTES) + (1 - x) * (HALF / 4) * BM;
        float* ml = reinterpret_cast<float*>(gen_base);    // the Q area: [x][m | l][row]
        asm volatile("bar.sync 1, 256;" ::: "memory");
        ml[x * 256 + row] = m_ref;
        ml[x * 256 + 128 + row] = l;
#pragma unroll 1
        for (int c = 0; c < HALF; c += 32) {
            float o[32];
            if (steps > 0) {
                tmem_ld32(o_addr + (1 - x) * HALF + c, o);
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j) o[j] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) mine[(c / 4 + j) * BM + row] = make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
        const float m2 = ml[(1 - x) * 256 + row], l2 = ml[(1 - x) * 256 + 128 + row];
        const float m = fmaxf(m_ref, m2);
        const float f1 = m_ref == kNegInf ? 0.f : ex2(m_ref - m), f2 = m2 == kNegInf ? 0.f : ex2(m2 - m);
        const float total = l * f1 + l2 * f2, inv = inverse_sum(total);   // a NaN score is in l: the part becomes NaN, log2-sum-exp included
        const float g1 = f1 * inv, g2 = f2 * inv;
        const int b = qt * BM + row;
        float* dst = a.parts + (((size_t)(b < a.B ? b : 0) * a.H + h) * (a.n_pre + a.splits) + part) * (HD + 4);
#pragma unroll 1
        for (int c = 0; c < HALF; c += 32) {
            float o[32];
            if (steps > 0) {
                tmem_ld32(o_addr + x * HALF + c, o);
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j) o[j] = 0.f;
            }
            if (b < a.B && ok) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float4 t = theirs[(c / 4 + j) * BM + row];
                    *reinterpret_cast<float4*>(dst + x * HALF + c + 4 * j) =
                        make_float4(o[4 * j] * g1 + t.x * g2, o[4 * j + 1] * g1 + t.y * g2, o[4 * j + 2] * g1 + t.z * g2, o[4 * j + 3] * g1 + t.w * g2);
                }
            }
        }
        if (x == 0 && b < a.B && ok) dst[HD] = total == 0.f ? kNegInf : m + log2f(total);
        tc_fence_before();
    }

    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

// queries [B][H][hd]: box = 64 elements x 128 sequences of one head, 128-byte swizzle; sequences past B read as zeros
static bool make_query_map(CUtensorMap* m, const void* q, int hd, int B, int H)
{
    TensorMapEncodeFn fn = tensor_map_encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)hd, (cuuint64_t)B, (cuuint64_t)H};
    cuuint64_t strides[2] = {(cuuint64_t)H * hd * 2, (cuuint64_t)hd * 2};
    cuuint32_t box[3] = {64, BM, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD>
static cudaError_t launch_t(const SharedDecodeArgs& a, cudaStream_t stream)
{
    static PerDeviceOnce limit_raised;
    int dev = 0, sms = 0;
    cudaError_t e = current_device(&dev, &sms);
    if (e != cudaSuccess) return e;
    e = raise_smem_limit_once(limit_raised, dev, shared_prefix_kernel<HD>, smem_bytes<HD>());
    if (e != cudaSuccess) return e;
    // an SM's split between L1 and shared memory cannot change while a CTA runs on it: take all of it, so that the
    // own-rows kernel's CTAs still fit
    static PerDeviceOnce carveout_set;
    e = carveout_set.once(dev, []() { return cudaFuncSetAttribute(shared_prefix_kernel<HD>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared); });
    if (e != cudaSuccess) return e;
    CUtensorMap mq, mk, mv;
    if (!make_query_map(&mq, a.q, HD, a.B, a.H) || !make_slab_map(&mk, a.pk, HD, a.cap, a.cap, a.H, BN) ||
        !make_slab_map(&mv, a.pv, HD, a.cap, a.cap, a.H, BN))
        return cudaErrorInvalidValue;
    const int n_qtiles = (a.B + BM - 1) / BM;
    const long long grid = (long long)n_qtiles * a.H * a.n_pre;
    if (grid > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    return launch_pdl(shared_prefix_kernel<HD>, dim3((unsigned)grid), dim3(kThreads), (size_t)smem_bytes<HD>(), stream, mq, mk, mv, a, n_qtiles);
}

}  // namespace sp

bool shared_decode_supported(const SharedDecodeArgs& a)
{
    return (a.hd == 64 || a.hd == 128) && tensor_map_encode_fn() != nullptr;
}

cudaError_t launch_shared_prefix(const SharedDecodeArgs& a, cudaStream_t stream)
{
    return a.hd == 64 ? sp::launch_t<64>(a, stream) : sp::launch_t<128>(a, stream);
}

}  // namespace bt
