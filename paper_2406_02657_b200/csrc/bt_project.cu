// The linear maps either side of the attention path, y = W x + b on the 5th-generation tensor cores:
//   - prefix projection (paper section 2.4; appendix on token-decoder variants, "Prefix"): the
//     context embedding of a block is projected into P prefix token embeddings;
//   - QKV projection whose epilogue is the cache append (sections 2.1, 2.3, 2.4: the K,V a layer
//     computes from its input are cached): the Q part goes out as [B][H][n][hd] for the attention
//     call, the K and V parts are written straight to rows len[b] .. len[b]+n-1 of the block or
//     local cache, so no separate append pass touches them.
//
// One persistent CTA per SM, warp-specialised:
//   warps 0-7       : epilogue - two warps per quarter of the tensor-memory lanes (four, warps 0-15, where the 4-bit cache is the
//                     target) taking alternate 64-column pieces.  64 columns at a time:
//                     tensor memory -> registers, + bias, -> bf16, through a per-warp swizzled
//                     shared-memory patch so that the global stores are whole 128-byte lines (8 lanes
//                     per row piece: one head of one cache row at head_dim 64), then to q / the cache /
//                     the plain [M][N] output
//   next warp (1 lane): TMA producer - x tile [128 x 64] and W tile [BN x 64] per stage, 128-byte swizzle
//   last warp (1 lane): tcgen05.mma issuer - 128 x BN x 16 instructions, fp32 accumulators in tensor
//                     memory, double-buffered so that the epilogue of a tile runs under the next
//                     tile's products
// BN (64, 128 or 256 output features per tile) is chosen per launch so that there are enough tiles
// for every SM.  Every wait is bounded in wall time and raises BT_DEV_TIMEOUT when it runs out.
//
// Large products run the same kernel on pairs of CTAs (kCtas = 2, a cluster of two SMs, tcgen05 cta_group::2):
// a pair owns a 256 x BN tile, each CTA loads its own 128 rows of x and only HALF of the W tile (its BN/2
// output features) with plain TMA loads - no multicast - that report to the leader CTA's barrier; the leader's
// one MMA thread issues 256 x BN x 16 instructions that read both halves of W from the two CTAs' shared
// memory and accumulate each CTA's 128 rows in that CTA's tensor memory; commits are multicast to both CTAs'
// barriers; each CTA drains its own accumulator and reports to the leader.  Per CTA this moves a third less
// operand data from L2 into shared memory for the same products.  Where few tiles are left for the last round, they are cut into
// two or four parts along their output features, a part a pair.
//
// 8-bit operands (kInt8: a step per row of x and per output feature) run through the same stages and tiles: 128 bytes of a row are
// 128 values of K instead of 64, an instruction takes 32 of them, and the sums are whole numbers (at most 2048 * 128 * 128 = 2^25,
// so 32 bits hold them), which the epilogue multiplies with both steps.
//
// With the 4-bit block cache as the target (kProjectQkvKv4) the epilogue thread that holds 64 values of a K or V row, rounded to bf16
// as they would be cached, quantises them (two groups of 32); the warp then stores the codes of its 32 rows, whose bytes are interleaved
// with those of neighbouring rows, through its shared-memory patch: four rows of a tile at once as 128 contiguous bytes where they are there,
// else a row at a time.
#include <cuda.h>

#include "bt_common.cuh"
#include "bt_device.h"
#include "bt_kernels.h"
#include "bt_kv4.cuh"
#include "bt_mbarrier.cuh"
#include "bt_tcgen05.cuh"
#include "bt_tensor_map.h"

namespace bt {
namespace proj {

using namespace tc;

constexpr int BM = 128;                  // rows of x per tile (= tensor-memory lanes)
constexpr int kRowBytes = 128;           // bytes of K per stage and row: one swizzle atom (64 bf16, 128 8-bit values)
constexpr uint32_t kABytes = BM * kRowBytes;
constexpr uint32_t kSpinLimit = 1u << 26;
constexpr uint64_t kWaitLimitNs = 1000000000ull;  // 1 s: far beyond any legitimate wait
constexpr uint32_t kPatchBytes = 32 * 128;         // per epilogue warp: 32 rows x 64 bf16

constexpr uint32_t kPeerBitMask = 0xFEFFFFFFu;   // clears the bit that tells the two CTAs of a pair apart in a shared::cluster address

// kKv4 (the 4-bit cache is the target): 16 epilogue warps, which have twice the arithmetic to do, for 8, and a stage less for their patches
// (197 us with 8 at 16384 rows x 2048 x 6144 in 8 bits, where the product into a bf16 cache takes 140).
template <int BN, int kCtas, bool kKv4>
struct Cfg {
    static constexpr int kEpilogueWarps = kKv4 ? 16 : 8, kProducerWarp = kEpilogueWarps, kMmaWarp = kEpilogueWarps + 1;
    static constexpr int kThreads = (kEpilogueWarps + 2) * 32;
    static constexpr uint32_t kBBytes = (BN / kCtas) * kRowBytes;   // a CTA of a pair holds half of the W tile
    static constexpr uint32_t kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = kStageBytes == 48 * 1024 ? (kKv4 ? 3 : 4) : kStageBytes == 32 * 1024 ? (kKv4 ? 5 : 6) : (kKv4 ? 6 : 8);
    static constexpr uint32_t kTmemCols = 2 * BN;   // two accumulators
    static constexpr int kBarriers = 2 * kStages + 4;
    static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kEpilogueWarps * kPatchBytes + kBarriers * 8 + 16;
    static_assert(kSmemBytes <= 227 * 1024, "a CTA's shared memory");
};

struct Params {
    ProjectArgs a;
    int tiles_m, tiles_n;
    int whole, parts, items;   // tiles worked whole; parts that each of the others is cut into along its output features; both together
};
// Item i of a launch: rows of tile tm, `width` output features from `col`.
struct Piece {
    int tm, col, width;
};
template <int BN, int kCtas>
__device__ __forceinline__ Piece piece_of(int i, const Params& p)
{
    Piece w;
    int part = 0;
    w.width = BN;
    if (kCtas == 2 && i >= p.whole) {   // parts: 2 or 4
        const int shift = p.parts >> 1, s = i - p.whole;
        part = s & (p.parts - 1);
        i = p.whole + (s >> shift);
        w.width = BN >> shift;
    }
    w.tm = i / p.tiles_n;
    w.col = (i - w.tm * p.tiles_n) * BN + part * w.width;
    return w;
}

__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t* dev_status)
{
    if (mbar_wait_walltime(bar, parity, abort_flag, kSpinLimit, kWaitLimitNs)) return true;
    raise_status(dev_status, BT_DEV_TIMEOUT);
    return false;
}

// New length of sequence b after its n rows: (reset ? 0 : len) + n when they fit, else unchanged and flagged.
__device__ __forceinline__ void advance_len(int32_t* len, int b, int n, int cap, int reset_first, const uint8_t* reset_mask,
                                            uint32_t* dev_status)
{
    const bool rst = reset_mask ? (reset_mask[b] != 0) : (reset_first != 0);
    const int l = rst ? 0 : len[b];
    if (l >= 0 && l + n <= cap)
        len[b] = l + n;
    else
        raise_status(dev_status, BT_DEV_OVERFLOW);  // the sequence keeps its rows and its length
}

// Every sequence starts with the call's rows, for which there is room: no tile looks at an old length, and the one with a sequence's first
// row sets the new one, so that no launch has to follow.
__host__ __device__ __forceinline__ bool starts_anew(const ProjectArgs& a) { return a.reset_first != 0 && a.reset_mask == nullptr; }

// ---- the forms that differ between one CTA and a pair
template <int kCtas>
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t cols)
{
    if constexpr (kCtas == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {   // issued by the same warp of both CTAs of the pair
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int kCtas>
__device__ __forceinline__ void tmem_dealloc(uint32_t tmem, uint32_t cols)
{
    if constexpr (kCtas == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
}
// TMA load of a pair's CTA: lands in this CTA's shared memory, reports its bytes to the barrier named by a
// shared::cluster address (the leader's).  No multicast.
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar_cluster, int c0, int c1, int c2)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar_cluster), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
__device__ __forceinline__ void mma_bf16_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    const uint32_t z = 0;   // no output lane disabled
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5, %5, %5, %5, %5}, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(z)
        : "memory");
}
__device__ __forceinline__ void mma_s8_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    const uint32_t z = 0;   // no output lane disabled
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, {%5, %5, %5, %5, %5, %5, %5, %5}, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(z)
        : "memory");
}
// arrives, once the MMAs issued so far are done, on the barrier at this address in both CTAs of the pair
__device__ __forceinline__ void mma_commit_pair(uint32_t bar)
{
    const uint16_t both = 3;
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(both) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar_cluster)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory");
}
__device__ __forceinline__ void cluster_sync_all()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_cta_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ uint32_t lds32(uint32_t addr)
{
    uint32_t x;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(addr) : "memory");
    return x;
}
// four 8 x 8 matrices of 16-bit values out of fragments; lanes 8 i .. 8 i + 7 give the addresses of matrix i's rows
__device__ __forceinline__ void stmatrix4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi)
{
    const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ int64_t shfl64(int64_t x, int lane)
{
    const uint32_t lo = __shfl_sync(0xffffffffu, (uint32_t)x, lane), hi = __shfl_sync(0xffffffffu, (uint32_t)(x >> 32), lane);
    return (int64_t)((uint64_t)hi << 32 | lo);
}
constexpr int kCodeRow = 48;   // a row's 32 bytes of codes in the patch, 16 apart from the next so that the rows spread over the banks

// K (part 0) or V (part 1) of a warp's rows into the 4-bit cache: 64 bf16 values of this lane's row in w; the row is row rc (-1: it
// goes nowhere) of the slab whose tile with that row lies `off` bytes into the cache; quads: lanes that, with the three behind them, hold the four rows of a quad.
__device__ __forceinline__ void store_kv4(const ProjectArgs& a, const uint32_t (&w)[32], int64_t off, int rc, uint32_t quads, int part, uint32_t patch, int lane)
{
    uint8_t* const cache = reinterpret_cast<uint8_t*>(a.cache.k);
    uint32_t steps = 0;
#pragma unroll
    for (int grp = 0; grp < 2; ++grp) {
        uint4 x[4];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t* v = w + grp * 16 + i * 4;
            x[i] = make_uint4(v[0], v[1], v[2], v[3]);
            m = kv4::magnitude_max(m, kv4::magnitude_max8(x[i]));
        }
        const kv4::Step st = kv4::step_of_group<7>(kv4::magnitude_of(m));
        steps |= st.bits << (16 * grp);
        uint32_t codes[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) codes[i] = st.finite ? kv4::codes8(x[i], st.inv) : kv4::kZeroCodes;
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                     ::"r"(patch + lane * kCodeRow + grp * 16), "r"(codes[0]), "r"(codes[1]), "r"(codes[2]), "r"(codes[3]) : "memory");
    }
    if (rc >= 0) *reinterpret_cast<uint32_t*>(cache + off + kv4::kStepsAt + part * 64 + rc % kv4::kTileRows * 4) = steps;
    __syncwarp();
    const int j = lane >> 2, byte = lane & 3;
    constexpr int64_t kOffset = ((int64_t)1 << 56) - 1;
    const int64_t where = rc < 0 ? -1 : (int64_t)(rc % kv4::kTileRows) << 56 | off;   // row of the tile and where that lies
    auto quad = [&](int i) {   // rows i .. i + 3 of the warp: a quad of a tile, a word a lane
        const uint32_t rows = patch + i * kCodeRow;
        const int64_t to = shfl64(where, i);
        const int at = (int)(to >> 56);
        uint8_t* dst = cache + (to & kOffset) + lane * 4;
        if (part == 0) {   // half a unit of one of the rows
            *reinterpret_cast<uint32_t*>(dst + kv4::k_codes_at(at, 0)) = lds32(rows + (lane >> 4 << 1 | (lane >> 1 & 1)) * kCodeRow + ((lane >> 2 & 3) * 2 + (lane & 1)) * 4);
        } else {           // one byte of each of the rows
            const uint32_t from = rows + (j ^ (at >> 2 << 1)) * 4;
            const uint32_t x[4] = {lds32(from), lds32(from + kCodeRow), lds32(from + 2 * kCodeRow), lds32(from + 3 * kCodeRow)};
            const uint32_t pick = byte | (4 + byte) << 4;
            *reinterpret_cast<uint32_t*>(dst + kv4::kPartBytes + (at >> 2) * 128) = __byte_perm(__byte_perm(x[0], x[1], pick), __byte_perm(x[2], x[3], pick), 0x5410);
        }
    };
    if (quads == 0x11111111u) {
#pragma unroll
        for (int i = 0; i < 32; i += 4) quad(i);
        return;
    }
    const uint32_t done = quads * 15u;   // (no two start within four rows of each other)
#pragma unroll 1
    for (; quads; quads &= quads - 1) quad(__ffs(quads) - 1);
#pragma unroll 1
    for (int i = 0; i < 32; i += 4) {
        if ((done >> i & 15u) == 15u) continue;
        // eight lanes a row, a word of its codes each
        const int r = i + (lane >> 3), q = lane & 7;
        const int64_t to = shfl64(where, r);
        if (to >= 0 && !(done >> r & 1u)) {
            const int at = (int)(to >> 56);
            uint8_t* dst = cache + (to & kOffset);
            const uint32_t codes = lds32(patch + r * kCodeRow + q * 4);
            if (part == 0) {
                *reinterpret_cast<uint32_t*>(dst + kv4::k_codes_at(at, q)) = codes;
            } else {
                dst += kv4::v_codes_at(at, q);
#pragma unroll
                for (int b = 0; b < 4; ++b) dst[4 * b] = (uint8_t)(codes >> (8 * b));
            }
        }
    }
}

template <int BN, int kCtas, bool kInt8, bool kKv4>
__global__ void __launch_bounds__(Cfg<BN, kCtas, kKv4>::kThreads, 1)
project_tc_kernel(const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapW, const __grid_constant__ CUtensorMap mapPart, Params p)
{
    using C = Cfg<BN, kCtas, kKv4>;
    constexpr int S = C::kStages, kEpilogueWarps = C::kEpilogueWarps, kProducerWarp = C::kProducerWarp, kMmaWarp = C::kMmaWarp;
    constexpr uint32_t IDESC = kInt8 ? make_idesc_s8(BM * kCtas, BN) : make_idesc(BM * kCtas, BN, false);
    constexpr int BK = kInt8 ? kRowBytes : kRowBytes / 2;   // elements of K per stage
    const ProjectArgs& a = p.a;
    // a pair of CTAs works on one tile of 256 rows: `rank` is this CTA's half, `unit` numbers the pairs
    const uint32_t rank = kCtas == 2 ? cluster_cta_rank() : 0u;
    const int unit = (int)blockIdx.x / kCtas, n_units = (int)gridDim.x / kCtas;
    const bool leader = rank == 0;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* gen_base = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t sPatch = base + S * C::kStageBytes;
    const uint32_t sBar = sPatch + kEpilogueWarps * kPatchBytes;
    uint8_t* gen_tail = gen_base + (sBar - base);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen_tail + C::kBarriers * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(gen_tail + C::kBarriers * 8 + 8);
    auto full = [&](int s) { return sBar + 8u * s; };
    auto empty = [&](int s) { return sBar + 8u * (S + s); };
    auto acc_full = [&](int i) { return sBar + 8u * (2 * S + i); };
    auto acc_empty = [&](int i) { return sBar + 8u * (2 * S + 2 + i); };

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(acc_full(i), 1);
            mbar_init(acc_empty(i), kEpilogueWarps * kCtas);   // the leader's collects both CTAs' epilogue warps
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tmem_alloc<kCtas>(smem_u32(tmem_slot), C::kTmemCols);  // this warp allocates the tensor-memory columns and frees them at the end
    tc_fence_before();
    __syncthreads();
    if constexpr (kCtas == 2) cluster_sync_all();   // the partner's barriers exist before anything is sent to them
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    // Programmatic dependent launch: until the kernel before this one in the stream is done, nothing here
    // reads or writes global memory (the descriptor prefetch below touches only the kernel's own parameters).
    pdl_launch_dependents();

    const int n_items = p.items;                   // tiles of BM * kCtas rows, or parts of them
    const int n_kb = (a.K + BK - 1) / BK;

    if (warp == kProducerWarp) {
        if (lane == 0) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&mapX) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&mapW) : "memory");
            pdl_wait();
            uint32_t it = 0;
            bool ok = true;
            for (int item = unit; ok && item < n_items; item += n_units) {
                const Piece w = piece_of<BN, kCtas>(item, p);
                const CUtensorMap* const from = kCtas == 1 || w.width == BN ? &mapW : &mapPart;
                for (int kb = 0; kb < n_kb; ++kb, ++it) {
                    const uint32_t s = it % S;
                    ok = wait(empty(s), ((it / S) & 1) ^ 1, abort_flag, a.dev_status);
                    if (!ok) break;
                    const uint32_t dst = base + s * C::kStageBytes;
                    if constexpr (kCtas == 1) {
                        mbar_expect_tx(full(s), C::kStageBytes);
                        tma_load_3d(dst, &mapX, full(s), kb * BK, w.tm * BM, 0);
                        tma_load_3d(dst + kABytes, from, full(s), kb * BK, w.col, 0);
                    } else {
                        // both CTAs' bytes are counted on the leader's barrier, which the leader arms
                        if (leader) mbar_expect_tx(full(s), 2 * kABytes + w.width * kRowBytes);
                        const uint32_t bar = full(s) & kPeerBitMask;
                        tma_load_3d_pair(dst, &mapX, bar, kb * BK, w.tm * (2 * BM) + (int)rank * BM, 0);
                        tma_load_3d_pair(dst + kABytes, from, bar, kb * BK, w.col + (int)rank * (w.width / 2), 0);
                    }
                }
            }
            // Before the CTA goes, nothing may still be on its way to it.  One CTA: every copy this thread issued
            // has landed (at once on the normal path, where the products that consumed them are done).  A pair:
            // the last commits multicast to this CTA's "stage free" barriers have arrived, which also means the
            // products that read this CTA's shared memory are done.  Bounded when something went wrong.
            for (uint32_t back = 1; back <= (uint32_t)S && back <= it; ++back) {
                const uint32_t u = it - back;
                if constexpr (kCtas == 1) {
                    if (!mbar_wait_walltime(full(u % S), (u / S) & 1, abort_flag, kSpinLimit, kWaitLimitNs)) break;
                } else {
                    if (!mbar_wait_walltime(empty(u % S), (u / S) & 1, abort_flag, kSpinLimit, kWaitLimitNs)) break;
                }
            }
        }
    } else if (warp == kMmaWarp) {
        // The whole warp walks the loop (control flow stays warp-uniform; the outcome of every wait is agreed on by
        // a vote) and one elected lane issues: a lone lane inside a divergent branch issues tcgen05.mma slower.
        if (leader) {   // a pair's products are issued by its leader alone
            auto wait_all = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, wait(b, parity, abort_flag, a.dev_status)) != 0; };
            uint32_t it = 0, t = 0;
            bool ok = true;
            for (int item = unit; ok && item < n_items; item += n_units, ++t) {
                const uint32_t acc = t & 1;
                const uint32_t idesc = kCtas == 1 ? IDESC : with_n(IDESC, piece_of<BN, kCtas>(item, p).width);
                ok = wait_all(acc_empty(acc), ((t >> 1) & 1) ^ 1);  // the epilogue has drained this accumulator
                if (!ok) break;
                tc_fence_after();
                for (int kb = 0; kb < n_kb; ++kb, ++it) {
                    const uint32_t s = it % S;
                    ok = wait_all(full(s), (it / S) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    // descriptor low words: address in 16-byte units plus the leading-dimension field; an instruction takes
                    // 32 bytes of K inside a swizzled 128-byte row
                    const uint32_t a0 = base + s * C::kStageBytes, b0 = a0 + kABytes;
                    const uint32_t alo = (a0 >> 4) | (1u << 16), blo = (b0 >> 4) | (1u << 16);
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < kRowBytes / 32; ++kk) {
                            const uint64_t da = desc_words(alo + kk * 2, kDescHiSw128), db = desc_words(blo + kk * 2, kDescHiSw128);
                            const uint32_t more = (kb > 0 || kk > 0) ? 1u : 0u;
                            if constexpr (kInt8 && kCtas == 1) mma_s8(tmem + acc * BN, da, db, idesc, more);
                            else if constexpr (kInt8) mma_s8_pair(tmem + acc * BN, da, db, idesc, more);
                            else if constexpr (kCtas == 1) mma_bf16(tmem + acc * BN, da, db, idesc, more);
                            else mma_bf16_pair(tmem + acc * BN, da, db, idesc, more);
                        }
                        if constexpr (kCtas == 1) mma_commit(empty(s));
                        else mma_commit_pair(empty(s));
                        if (kb == n_kb - 1) {
                            if constexpr (kCtas == 1) mma_commit(acc_full(acc));
                            else mma_commit_pair(acc_full(acc));
                        }
                    }
                    __syncwarp();
                }
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue
        // warp e drains tensor-memory lane quarter e % 4 (the quarter a warp may access is its index modulo 4) and every second 64-column
        // piece (every fourth with 16 warps), starting at piece e / 4
        const int wq = warp & 3, half = warp >> 2;
        const uint32_t lane_base = tmem + ((uint32_t)(wq * 32) << 16);
        const uint32_t patch = sPatch + warp * kPatchBytes;
        const bf16* bias = reinterpret_cast<const bf16*>(a.bias);
        const int D = a.H * a.hd;
        const bool anew = !kKv4 && starts_anew(a);
        uint32_t t = 0;
        bool ok = true;
        pdl_wait();
        for (int item = unit; item < n_items; item += n_units, ++t) {
            const Piece w = piece_of<BN, kCtas>(item, p);
            const uint32_t acc = t & 1;
            // This lane's own row: where it goes among the rows of Q (or of the plain output) and in the cache, without head and
            // dimension (elements; bytes in the 4-bit cache); -1: nowhere.
            const int m = w.tm * (BM * kCtas) + (int)rank * BM + wq * 32 + lane;
            int64_t off_q = -1, off_c = -1;
            int row_rc = -1;
            uint32_t quads = 0;
            if (m < a.M && a.mode == kProjectPlain) off_q = (int64_t)m * a.N;
            if (a.mode != kProjectPlain) {
                int row_b = -1;
                if (m < a.M) {
                    row_b = m / a.n_rows;
                    const int row_i = m - row_b * a.n_rows;
                    off_q = ((int64_t)row_b * a.H * a.n_rows + row_i) * a.hd;
                    const bool rst = a.reset_mask ? (a.reset_mask[row_b] != 0) : (a.reset_first != 0);
                    const int len_old = rst ? 0 : a.cache.len[row_b];
                    if (anew && w.col == 0 && half == 0 && row_i == 0) a.cache.len[row_b] = a.n_rows;
                    if (len_old >= 0 && len_old + a.n_rows <= a.cache.cap) {   // else: no room, K and V are dropped
                        row_rc = len_old + row_i;
                        off_c = (int64_t)row_b * a.H * a.cache.slab_stride +
                                (!kKv4 ? (int64_t)row_rc * a.cache.row_stride : (int64_t)(row_rc / kv4::kTileRows) * (a.hd / 64) * kv4::kTileBytes);
                    }
                }
                if constexpr (kKv4) {   // rows of a sequence follow one another
                    const int b3 = __shfl_down_sync(0xffffffffu, row_b, 3);
                    quads = __ballot_sync(0xffffffffu, lane <= 28 && row_rc >= 0 && row_b == b3 && (row_rc & 3) == 0);
                }
            }
            float x_step = 0.f;
            if constexpr (kInt8)
                if (m < a.M) x_step = a.x_steps[m];
            // steps and bias of a lane's columns of a piece, requested a piece ahead (below)
            uint64_t ws[8];
            uint32_t bs[8];
            const int width = kCtas == 1 ? BN : w.width;
            auto columns = [&](int c0) {
                if (kKv4 || c0 >= width || w.col + c0 >= a.N) return;
                const int at = w.col + c0 + (lane & 3) * 2;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if constexpr (kInt8) ws[i] = *reinterpret_cast<const uint64_t*>(a.w_steps + at + i * 8);
                    bs[i] = bias != nullptr ? *reinterpret_cast<const uint32_t*>(bias + at + i * 8) : 0u;
                }
            };
            columns(half * 64);
            ok = wait(acc_full(acc), (t >> 1) & 1, abort_flag, a.dev_status);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int c0 = half * 64; c0 < width; c0 += kEpilogueWarps * 16) {
                const int col0 = w.col + c0;                 // first output feature of this 64-column piece
                if (col0 >= a.N) break;                        // warp-uniform
                // Where the piece goes.  head_dim is a multiple of 64 and so is col0: the 64 columns lie inside one
                // head of one of Q, K, V, so everything but the row is the same for the whole warp.
                int part = 0;                                      // 0: Q or the plain output, 1: K, 2: V
                int64_t off = off_q, add = col0;
                if (a.mode != kProjectPlain) {
                    part = col0 / D;
                    const int cc = col0 - part * D, h = cc / a.hd, d = cc - h * a.hd;
                    add = (part == 0 ? (int64_t)h * a.n_rows * a.hd : (int64_t)h * a.cache.slab_stride) + d;
                    if (part != 0) off = off_c;
                    if (kKv4 && part != 0) add += d / 64 * kv4::kTileBytes - d;
                }
                const bool to_kv4 = kKv4 && part != 0;
                off = off < 0 ? -1 : off + add;
                // * steps, + bias, -> bf16, into the patch: 16-byte piece q8 of row r at (q8 ^ (r & 7)) - or, bound for the 4-bit cache, whose groups are
                // of a row, back into the registers of the lane that has the row
                uint32_t packed[32];   // kKv4
                if constexpr (!kKv4) {
                    // A lane takes two columns of every eight, of rows g and g + 8 of the sixteen that are read at once: 8 bytes of steps and 4 of bias
                    // for every eight columns, requested before the products are done or under the piece before.  (A row a lane has every lane read all 64 columns'
                    // steps and biases, 512 bytes of L1's bandwidth an instruction: 11.9 us instead of 10.5 at 4096 rows x 1024 x 2048 in 8 bits, and
                    // 9.8 instead of 8.5 at 4096 x 256 x 2048 in bf16; requested when they are needed, 12.0 and 9.3.)
                    const int g = lane >> 2;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t r[32];
                        tmem_ld16x64_issue(lane_base + (uint32_t)(h * 16 << 16) + acc * BN + c0, r);
                        uint64_t xa = 0, xb = 0;   // steps of both rows
                        if constexpr (kInt8) {
                            const float a0 = __shfl_sync(0xffffffffu, x_step, h * 16 + g), a8 = __shfl_sync(0xffffffffu, x_step, h * 16 + 8 + g);
                            xa = pack2(a0, a0);
                            xb = pack2(a8, a8);
                        }
                        tmem_wait_ld();
                        tmem_ld_fence32(r);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float f[4];
                            if constexpr (kInt8) {   // sum * (x_step * w_step) + bias
                                const int* sum = reinterpret_cast<const int*>(r + i * 4);
                                const uint64_t b2 = pack2(bf_lo(bs[i]), bf_hi(bs[i]));
                                unpack2(ffma2(pack2((float)sum[0], (float)sum[1]), fmul2(xa, ws[i]), b2), f[0], f[1]);
                                unpack2(ffma2(pack2((float)sum[2], (float)sum[3]), fmul2(xb, ws[i]), b2), f[2], f[3]);
                            } else {
#pragma unroll
                                for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(r[i * 4 + e]);
                                if (bias != nullptr) {
                                    f[0] += bf_lo(bs[i]);
                                    f[1] += bf_hi(bs[i]);
                                    f[2] += bf_lo(bs[i]);
                                    f[3] += bf_hi(bs[i]);
                                }
                            }
                            r[i * 4] = pack_pair(f[0], f[1]);
                            r[i * 4 + 1] = pack_pair(f[2], f[3]);
                        }
                        // a matrix of 8 x 8 for every eight lanes' addresses: rows 0 .. 7 and 8 .. 15 of two pieces
                        const int row = h * 16 + (lane & 15);
#pragma unroll
                        for (int i = 0; i < 8; i += 2)
                            stmatrix4(patch + row * 128 + (((i + (lane >> 4)) ^ (row & 7)) << 4), r[i * 4], r[i * 4 + 1], r[i * 4 + 4], r[i * 4 + 5]);
                    }
                    columns(c0 + kEpilogueWarps * 16);
                } else {
                    constexpr int kAtOnce = 32;                    // accumulators in registers (18 warps are five on one of an SM's four schedulers, which leaves 96 registers a thread)
#pragma unroll
                    for (int c1 = 0; c1 < 64; c1 += kAtOnce) {
                        uint32_t r[kAtOnce];
#pragma unroll
                        for (int i = 0; i < kAtOnce; i += 32) tmem_ld32_issue(lane_base + acc * BN + c0 + c1 + i, r + i);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < kAtOnce; i += 32) tmem_ld_fence32(r + i);
#pragma unroll
                        for (int e = 0; e < kAtOnce / 8; ++e) {
                            float f[8];
                            const int q8 = c1 / 8 + e, col = col0 + q8 * 8;
                            float bf[8] = {};
                            if (bias != nullptr) unpack8(*reinterpret_cast<const uint4*>(bias + col), bf);
                            if constexpr (kInt8) {   // sum * (x_step * w_step) + bias
                                const uint64_t xs = pack2(x_step, x_step);
#pragma unroll
                                for (int i = 0; i < 8; i += 4) {
                                    const float4 ws = *reinterpret_cast<const float4*>(a.w_steps + col + i);
                                    const int* sum = reinterpret_cast<const int*>(r + e * 8 + i);
                                    unpack2(ffma2(pack2((float)sum[0], (float)sum[1]), fmul2(xs, pack2(ws.x, ws.y)), pack2(bf[i], bf[i + 1])), f[i], f[i + 1]);
                                    unpack2(ffma2(pack2((float)sum[2], (float)sum[3]), fmul2(xs, pack2(ws.z, ws.w)), pack2(bf[i + 2], bf[i + 3])), f[i + 2], f[i + 3]);
                                }
                            } else {
#pragma unroll
                                for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(r[e * 8 + i]);
                                if (bias != nullptr) {
#pragma unroll
                                    for (int i = 0; i < 8; ++i) f[i] += bf[i];
                                }
                            }
                            const uint4 y = pack8(f);
                            if (to_kv4) {
                                packed[q8 * 4] = y.x;
                                packed[q8 * 4 + 1] = y.y;
                                packed[q8 * 4 + 2] = y.z;
                                packed[q8 * 4 + 3] = y.w;
                                continue;
                            }
                            const uint32_t dst = patch + lane * 128 + ((q8 ^ (lane & 7)) << 4);
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(y.x), "r"(y.y), "r"(y.z), "r"(y.w) : "memory");
                        }
                    }
                }
                if (to_kv4) {
                    if constexpr (kKv4) store_kv4(a, packed, off, row_rc, quads, part - 1, patch, lane);
                } else {
                    __syncwarp();
                    bf16* const base_out = reinterpret_cast<bf16*>(part == 0 ? a.out : part == 1 ? a.cache.k : a.cache.v) + (lane & 7) * 8;
                    // out of the patch: 8 lanes take one row's 128 bytes, so every store instruction writes 4 whole lines
#pragma unroll
                    for (int itr = 0; itr < 8; ++itr) {
                        const int rr = itr * 4 + (lane >> 3), q8 = lane & 7;
                        const int64_t to = shfl64(off, rr);   // of that row; none where there is no room
                        const uint4 y = lds128(patch + rr * 128 + ((q8 ^ (rr & 7)) << 4));
                        if (to >= 0) *reinterpret_cast<uint4*>(base_out + to) = y;
                    }
                }
                __syncwarp();  // the patch is free for the next piece
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (kCtas == 1) mbar_arrive(acc_empty(acc));
                else mbar_arrive_cluster(acc_empty(acc) & kPeerBitMask);   // the leader's barrier
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if constexpr (kCtas == 2) cluster_sync_all();   // both CTAs are through with each other's barriers and tensor memory
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc<kCtas>(tmem, C::kTmemCols);
    }
}

// The lengths go up once every tile has read the old ones (where it needs them): a second, tiny launch behind the product (it starts
// under programmatic dependent launch while the product drains; counting the product's CTAs in on a word in
// global memory and letting the last one advance the lengths was measured 2 us slower per step).
__global__ void project_len_advance_kernel(int32_t* len, int B, int n, int cap, int reset_first, const uint8_t* reset_mask,
                                           uint32_t* dev_status)
{
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < B) advance_len(len, b, n, cap, reset_first, reset_mask, dev_status);
}

template <int BN, int kCtas, bool kInt8, bool kKv4>
static cudaError_t launch_bn(const ProjectArgs& a, int dev, int sms, int parts, cudaStream_t stream)
{
    using C = Cfg<BN, kCtas, kKv4>;
    static PerDeviceOnce limit_raised;
    cudaError_t e = raise_smem_limit_once(limit_raised, dev, project_tc_kernel<BN, kCtas, kInt8, kKv4>, C::kSmemBytes);
    if (e != cudaSuccess) return e;
    CUtensorMap mx, mw, mp;
    auto map_rows = [&a](CUtensorMap* m, const void* ptr, long long rows, int box_rows) {
        if constexpr (kInt8) return make_byte_map(m, ptr, a.K, rows, box_rows);
        else return make_slab_map(m, ptr, a.K, rows, rows, 1, box_rows);
    };
    if (!map_rows(&mx, a.x, a.M, BM) || !map_rows(&mw, a.w, a.N, BN / kCtas)) return cudaErrorInvalidValue;
    mp = mw;
    if (parts > 1 && !map_rows(&mp, a.w, a.N, BN / kCtas / parts)) return cudaErrorInvalidValue;
    Params p;
    p.a = a;
    p.tiles_m = (a.M + BM * kCtas - 1) / (BM * kCtas);
    p.tiles_n = (a.N + BN - 1) / BN;
    const long long tiles = (long long)p.tiles_m * p.tiles_n;
    if (tiles > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    const int units = sms / kCtas;
    p.parts = parts;
    p.whole = (int)(parts > 1 ? tiles / units * units : tiles);
    p.items = p.whole + (int)(tiles - p.whole) * parts;
    const int grid = (p.items < units ? p.items : units) * kCtas;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(C::kThreads);
    cfg.dynamicSmemBytes = (size_t)C::kSmemBytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCtas;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = kCtas == 2 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, project_tc_kernel<BN, kCtas, kInt8, kKv4>, mx, mw, mp, p);
}

template <int BN, int kCtas>
static cudaError_t launch_type(const ProjectArgs& a, int dev, int sms, int parts, cudaStream_t stream)
{
    if (a.mode == kProjectQkvKv4)
        return a.x_steps ? launch_bn<BN, kCtas, true, true>(a, dev, sms, parts, stream) : launch_bn<BN, kCtas, false, true>(a, dev, sms, parts, stream);
    return a.x_steps ? launch_bn<BN, kCtas, true, false>(a, dev, sms, parts, stream) : launch_bn<BN, kCtas, false, false>(a, dev, sms, parts, stream);
}

}  // namespace proj

// rows are copied in 16-byte pieces; output features come in pieces of 64 (head_dim is a multiple of 64)
bool project_supported(const ProjectArgs& a) { return a.K % (a.x_steps ? 16 : 8) == 0 && a.N % 64 == 0 && tensor_map_encode_fn() != nullptr; }

cudaError_t launch_project(const ProjectArgs& a, cudaStream_t stream)
{
    int dev = 0, sms = 0;
    cudaError_t e = current_device(&dev, &sms);
    if (e != cudaSuccess) return e;
    // Tile shape: the one with the shortest estimated launch.  All tiles of a launch take the same time, so a launch
    // lasts (rounds of tiles) x (time of one tile); a tile's time is its area per SM over the relative rate that
    // shape sustains (measured: 128 x 256 on one SM = 1; 256 x 256 on a pair 1.11, a third less operand traffic per
    // SM; the narrower tiles less, their operands being re-read more often).
    struct Shape {
        int bn, ctas;
        double rate;
    };
    const Shape shapes[4] = {{256, 2, 1.11}, {256, 1, 1.0}, {128, 1, 0.9}, {64, 1, 0.75}};
    int best = 1, best_parts = 1;
    double best_cost = 0.0;
    for (int i = 0; i < 4; ++i) {
        const Shape& sh = shapes[i];
        if (sh.ctas == 2 && sms % 2 != 0) continue;
        const long long rows = (long long)proj::BM * sh.ctas;
        const long long tiles = ((a.M + rows - 1) / rows) * ((a.N + sh.bn - 1) / sh.bn);
        const long long units = sms / sh.ctas;
        // A last round of few tiles of pairs is worked in quarters or halves of them where each still has a pair of its own: per stage a part loads
        // all of its 16 KB of x and a quarter or half of as many of W, and takes 0.6 or 0.75 of the whole's time.  us, 8-bit / bf16, without and with:
        //   80 tiles of K = 1344 (1190 rows): 16 / 26, 13 / 18;   96 of K = 2048 (1024 rows): 20 / 36, 16 / 25;   384 (4096 rows): 39 / 72, 38 / 71
        double rounds = (double)((tiles + units - 1) / units);
        int parts = 1;
        const long long rest = tiles % units;
        if (sh.ctas == 2 && tiles > units && rest > 0) {
            parts = rest * 4 <= units ? 4 : rest * 2 <= units ? 2 : 1;
            rounds -= parts == 4 ? 0.4 : parts == 2 ? 0.25 : 0.0;
        }
        const double cost = rounds * (double)(proj::BM * sh.bn) / sh.rate;
        if (i == 0 || cost < best_cost - 1e-9) {
            best = i;
            best_parts = parts;
            best_cost = cost;
        }
    }
    switch (best) {
        case 0: e = proj::launch_type<256, 2>(a, dev, sms, best_parts, stream); break;
        case 1: e = proj::launch_type<256, 1>(a, dev, sms, 1, stream); break;
        case 2: e = proj::launch_type<128, 1>(a, dev, sms, 1, stream); break;
        default: e = proj::launch_type<64, 1>(a, dev, sms, 1, stream); break;
    }
    if (e != cudaSuccess || a.mode == kProjectPlain || proj::starts_anew(a)) return e;
    const int B = a.M / a.n_rows;
    return launch_pdl(proj::project_len_advance_kernel, dim3((B + 255) / 256), dim3(256), 0, stream, a.cache.len, B, a.n_rows,
                      a.cache.cap, a.reset_first, a.reset_mask, a.dev_status);
}

}  // namespace bt
