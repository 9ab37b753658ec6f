// Block-decoder decode attention over the 4-bit cache (paper section 2.3), with the append of a step fused in.
//
// With (s, u) the step and code of K, (t, w) those of V, g(d) the group of 32 dimensions that d lies in:
//   score_j = scale * sum_g s_jg sum_{d in g} q_d u_jd,     out_d = sum_j (p_j t_jg(d)) w_jd / sum_j p_j.
// Codes are small whole numbers, exact in bf16, and steps can be taken out of both sums, so the inner sums are products of bf16
// matrices.  What bounds the kernel is the 1.125 hd bytes a row of the cache, 3.6 times fewer than of the bf16 one, and next to
// it the instructions: a value that is unpacked to fp32 and multiplied on its own costs three issue slots or more, and the slots
// of 148 SMs then last for 6.7 TB/s at best.  Unpacked in pairs to bf16 (a shift, a masked or, a subtraction of two: 1.4 slots a
// value) and multiplied by warp-level m16n8k16 instructions it is less than half.
//
//   scores:  A = codes of 16 rows x 16 dimensions; B = the query, each of its columns with the values of one group only and zeros
//            elsewhere, so that a column of the result is the sum of one group.  Columns alternate between the two groups of
//            64 dimensions, so that all four lanes that share a row hold its sums; lane c of them goes on with tile c of a chunk.
//   output:  A = codes of V transposed, 16 dimensions x 16 rows (a word of eight codes from each of four rows a lane); B = the
//            weights p t of a group, as two bf16 columns, the rounded weight and what the rounding left (2^-17 of the weight in
//            all; one column alone would cost 2^-9, and the columns are there).
// Subtracting the offset of the unpacked codes pairwise, not from the sums, keeps the products as small as they are.
//
// As in the streaming kernel of the bf16 cache: one persistent CTA per SM, every warp on its own with a ring of chunks (64 rows,
// one bulk copy: tiles hold K and V), work items (sequence, head, part of the rows), partial results joined by the part that ends
// last, the length raised by the item that reads it last.  A new row is quantised by the warp that owns the last row, stored into
// the cache, and put into the copied chunk, where it is attended like any other: a step gives what append and attention give.
#include "bt_decode_ring.cuh"
#include "bt_kv4.cuh"

namespace bt {
namespace kv4 {

using ring::Cursor;

constexpr int kChunkTiles = 4, kChunkRows = kChunkTiles * kTileRows;
constexpr uint32_t kPollLimit = 1u << 24;   // polls of one wait before giving up (each poll suspends briefly)

template <int HD>
struct Geo {
    static constexpr int PLANES = HD / 64;
    static constexpr int TILE = PLANES * kTileBytes;
    static constexpr int STAGE = kChunkTiles * TILE;
    static constexpr int COLS = 4 * PLANES;                       // weights: (group, rounded or rest)
    static constexpr int WEIGHT_TILE = (COLS * 8 + 8) * 4;        // 8 row pairs a column; 8 words apart from a multiple of 32 banks
    static constexpr int WEIGHTS = kChunkTiles * WEIGHT_TILE;
};
template <int HD>
constexpr int smem_bytes(int warps, int stages) { return warps * (stages * (Geo<HD>::STAGE + 8) + Geo<HD>::WEIGHTS); }

__device__ __forceinline__ void lds64(uint32_t addr, uint32_t& x, uint32_t& y)
{
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(x), "=r"(y) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr)
{
    uint32_t x;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(addr) : "memory");
    return x;
}
__device__ __forceinline__ void sts32(uint32_t addr, uint32_t x) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(x) : "memory"); }

// Codes R and R + 4 of a word as a pair of bf16: 128 + (u + 8) is a bf16 with the code in its low bits, and 136 less is exact.
template <int R>
__device__ __forceinline__ uint32_t code_pair(uint32_t w)
{
    uint32_t x = ((w >> (4 * R)) & 0x000f000fu) | 0x43004300u, d;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(x), "r"(0x43084308u));
    return d;
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the largest of a warp's values that are numbers
__device__ __forceinline__ float warp_max(float x)
{
    float m;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(x));
    return m;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Rows r0 .. r1 - 1 of a work item; n counts the new row, which is row n - 1 and lies here when new_row is set.
struct Work {
    int bh, sp, b, n, r0, r1;
    bool new_row, overflow;
};
__device__ __forceinline__ Work work_at(const Cursor& c, const Kv4DecodeArgs& a)
{
    Work w;
    w.bh = c.bh;
    w.sp = c.sp;
    w.b = c.b;
    int n = a.len[w.b];
    n = n < 0 ? 0 : (n > a.n_max ? a.n_max : n);
    const bool append = a.k_new != nullptr && n < a.n_max;   // a full cache takes no row: flagged, attended as it is
    w.overflow = a.k_new != nullptr && !append;
    n += append ? 1 : 0;
    w.n = n;
    // whole chunks per part, as even as that goes (trailing parts may be empty)
    const int chunks = (n + kChunkRows - 1) / kChunkRows;
    const int per = a.splits == 1 ? chunks : (chunks + a.splits - 1) / a.splits;
    w.r0 = min(n, w.sp * per * kChunkRows);
    w.r1 = min(n, w.r0 + per * kChunkRows);
    w.new_row = append && w.r1 == n && w.r0 < n;
    return w;
}

template <int HD, int STAGES, int MAX_WARPS>
__global__ void __launch_bounds__(MAX_WARPS * 32, 1) block_decode_kv4_kernel(Kv4DecodeArgs a)
{
    using G = Geo<HD>;
    constexpr int PLANES = G::PLANES, LPR = HD / 8;
    extern __shared__ __align__(128) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, c = lane & 3;   // row and column of a fragment
    const int n_warps = blockDim.x >> 5;
    const uint32_t ring0 = smem_u32(smem) + warp * (STAGES * G::STAGE);
    const uint32_t wbuf = smem_u32(smem) + n_warps * (STAGES * G::STAGE) + warp * G::WEIGHTS;
    const uint32_t bar0 = smem_u32(smem) + n_warps * (STAGES * G::STAGE + G::WEIGHTS) + warp * (STAGES * 8);
    uint8_t* const ring_ptr = smem + warp * (STAGES * G::STAGE);

    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(bar0 + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    pdl_launch_dependents();

    const int n_items = a.B * a.H * a.splits;
    const int stride = n_warps * gridDim.x;
    const int first = warp * gridDim.x + blockIdx.x;   // neighbouring items go to different SMs
    uint8_t* const kv = reinterpret_cast<uint8_t*>(a.kv);
    pdl_wait();

    // ---- producer cursor (kept by every lane, acted on by lane 0): next chunk to request
    const ring::Step step = ring::step_of(stride, a);
    Cursor pc = ring::cursor_at(first < n_items ? first : 0, a);
    pc.item = first;
    int p_row = 0;
    Work pw = {};
    auto p_seek = [&]() {   // move to the next item that has rows
        for (; pc.item < n_items; ring::advance(pc, step, a)) {
            pw = work_at(pc, a);
            p_row = pw.r0;
            if (pw.r0 < pw.r1) return;
        }
    };
    uint32_t issued = 0, consumed = 0;
    auto issue_one = [&]() {
        if (pc.item >= n_items) return;
        const uint32_t st = issued % STAGES;
        if (lane == 0) {
            const uint32_t bytes = (uint32_t)((min(kChunkRows, pw.r1 - p_row) + kTileRows - 1) / kTileRows) * G::TILE;
            mbar_expect_tx(bar0 + 8 * st, bytes);
            ring::bulk_load(ring0 + st * G::STAGE, kv + (size_t)pw.bh * a.slab_bytes + (size_t)(p_row / kTileRows) * G::TILE, bytes,
                            bar0 + 8 * st, policy);
        }
        ++issued;
        p_row += kChunkRows;
        if (p_row >= pw.r1) {
            ring::advance(pc, step, a);
            p_seek();
        }
    };
    p_seek();
    for (int s = 0; s < STAGES; ++s) issue_one();

    // ---- consumer: whole items, chunk by chunk
    bool alive = true;
    Cursor cc = ring::cursor_at(first < n_items ? first : 0, a);
    cc.item = first;
    // The length update of an item is settled one item later: the count it depends on comes back from L2.  (lane 0 only)
    int pend_arrival = -1, pend_b = 0, pend_n = 0;
    bool pend_overflow = false;
    auto settle = [&]() {
        if (pend_arrival == a.H * a.splits - 1) {
            // that item was the last of its sequence to read the old length: raise it
            if (!pend_overflow) a.len[pend_b] = pend_n;
            a.counters[(size_t)a.B * a.H + pend_b] = 0;
        }
    };
    // the query of the next item is fetched an item ahead
    const bf16* Qall = reinterpret_cast<const bf16*>(a.q);
    uint4 q_next[PLANES][2];
    auto fetch_q = [&](int bh) {
#pragma unroll
        for (int p = 0; p < PLANES; ++p)
#pragma unroll
            for (int i = 0; i < 2; ++i) q_next[p][i] = ld_plain(Qall + (size_t)bh * HD + p * 64 + c * 16 + i * 8);
    };
    if (first < n_items) fetch_q(cc.bh);
    for (; alive && cc.item < n_items;) {
        const Work w = work_at(cc, a);
        Cursor cn = cc;
        ring::advance(cn, step, a);
        // An item counts itself in as soon as its own read of the length has returned (the increment is computed from it).
        int seq_arrival = -1;
        if (a.k_new != nullptr && lane == 0) {
            int one;
            asm volatile("and.b32 %0, %1, 0;\n\tadd.s32 %0, %0, 1;" : "=r"(one) : "r"(w.n));
            seq_arrival = atomicAdd(a.counters + (size_t)a.B * a.H + w.b, one);
        }
        // Query fragments: lane c holds dimensions 16 c .. 16 c + 15 of a plane, in the order of the codes of two words; in the
        // columns of the other group it holds zeros.
        uint32_t qf[PLANES][2][4];
        const uint32_t own_group = (g & 1) == (c >> 1) ? 0xffffffffu : 0u;
#pragma unroll
        for (int p = 0; p < PLANES; ++p)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 x = q_next[p][i];
                qf[p][i][0] = __byte_perm(x.x, x.z, 0x5410) & own_group;
                qf[p][i][1] = __byte_perm(x.x, x.z, 0x7632) & own_group;
                qf[p][i][2] = __byte_perm(x.y, x.w, 0x5410) & own_group;
                qf[p][i][3] = __byte_perm(x.y, x.w, 0x7632) & own_group;
            }
        if (cn.item < n_items) fetch_q(cn.bh);
        float m = kNegInf, l = 0.f;
        float o[PLANES][4][4];
#pragma unroll
        for (int p = 0; p < PLANES; ++p)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[p][r][i] = 0.f;

        for (int row = w.r0; row < w.r1; row += kChunkRows) {
            const uint32_t sidx = consumed % STAGES;
            // the outcome is made warp-uniform: what follows needs all 32 lanes
            if (!__all_sync(0xffffffffu, mbar_wait_polls(bar0 + 8 * sidx, (consumed / STAGES) & 1, kPollLimit))) {
                alive = false;
                break;
            }
            const uint32_t st = ring0 + sidx * G::STAGE;
            const int nvalid = min(kChunkRows, w.r1 - row), ntiles = (nvalid + kTileRows - 1) / kTileRows;
            if (w.new_row && row + kChunkRows >= w.r1) {
                // the new row, eight values a lane: lanes 0 .. LPR - 1 K, the next V (at head_dim 64 the upper half repeats them)
                const int part = (lane / LPR) & 1, piece = lane % LPR;
                const uint4 x = ld_plain(reinterpret_cast<const bf16*>(part == 0 ? a.k_new : a.v_new) + (size_t)w.bh * HD + piece * 8);
                const Step sg = step_of_lanes(x);
                const uint32_t codes = codes8(x, sg);
                if (lane < 2 * LPR) {
                    const int r = w.n - 1 - row;
                    const uint32_t tile = (uint32_t)(r / kTileRows) * G::TILE + (piece / 8) * kTileBytes;
                    const uint32_t code_at = tile + part * kPartBytes + (r % kTileRows) * 32 + (piece & 7) * 4;
                    const uint32_t step_at = tile + kStepsAt + part * 64 + (r % kTileRows) * 4 + ((piece >> 2) & 1) * 2;
                    uint8_t* copy = ring_ptr + sidx * G::STAGE;
                    uint8_t* held = kv + (size_t)w.bh * a.slab_bytes + (size_t)(row / kTileRows) * G::TILE;
                    *reinterpret_cast<uint32_t*>(copy + code_at) = codes;
                    *reinterpret_cast<uint32_t*>(held + code_at) = codes;
                    if ((piece & 3) == 0) {
                        *reinterpret_cast<uint16_t*>(copy + step_at) = (uint16_t)sg.bits;
                        *reinterpret_cast<uint16_t*>(held + step_at) = (uint16_t)sg.bits;
                    }
                }
                __syncwarp();
            }
            // ---- scores of rows 16 c + g and 16 c + g + 8 of the chunk, in this lane
            float s0 = 0.f, s1 = 0.f;
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                float acc[kChunkTiles][4];
#pragma unroll
                for (int t = 0; t < kChunkTiles; ++t) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[t][i] = 0.f;
                    if (t < ntiles) {
                        const uint32_t at = st + t * G::TILE + p * kTileBytes + g * 32 + c * 8;
                        uint32_t x[2], y[2];
                        lds64(at, x[0], x[1]);
                        lds64(at + 8 * 32, y[0], y[1]);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            mma(acc[t], code_pair<0>(x[i]), code_pair<0>(y[i]), code_pair<1>(x[i]), code_pair<1>(y[i]), qf[p][i][0], qf[p][i][1]);
                            mma(acc[t], code_pair<2>(x[i]), code_pair<2>(y[i]), code_pair<3>(x[i]), code_pair<3>(y[i]), qf[p][i][2], qf[p][i][3]);
                        }
                    }
                }
                float mine[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float lo = c & 1 ? acc[1][i] : acc[0][i], hi = c & 1 ? acc[3][i] : acc[2][i];
                    mine[i] = c & 2 ? hi : lo;
                }
                const uint32_t steps = st + c * G::TILE + p * kTileBytes + kStepsAt + g * 4;
                const uint32_t k0 = lds32(steps), k1 = lds32(steps + 8 * 4);
                s0 = fmaf(mine[1], bf_hi(k0), fmaf(mine[0], bf_lo(k0), s0));
                s1 = fmaf(mine[3], bf_hi(k1), fmaf(mine[2], bf_lo(k1), s1));
            }
            const bool in0 = 16 * c + g < nvalid, in1 = 16 * c + g + 8 < nvalid;
            s0 = in0 ? s0 * a.scale_log2 : kNegInf;
            s1 = in1 ? s1 * a.scale_log2 : kNegInf;
            const float mn = fmaxf(m, warp_max(fmaxf(s0, s1)));
            const float m_use = softmax_reference(mn);
            if (mn > m) {   // warp-uniform; where the maximum stays the factor is one
                const float cf = ex2(m - m_use);
                l *= cf;
#pragma unroll
                for (int p = 0; p < PLANES; ++p)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[p][r][i] *= cf;
                m = mn;
            }
            const float p0 = ex2(s0 - m_use), p1 = ex2(s1 - m_use);
            l += p0 + p1;
            // ---- weights of the two rows, a pair of them a word: column 2 (group) the rounded ones, column 2 (group) + 1 the rest
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                const uint32_t steps = st + c * G::TILE + p * kTileBytes + kStepsAt + 64 + g * 4;
                const uint32_t v0 = lds32(steps), v1 = lds32(steps + 8 * 4);
#pragma unroll
                for (int gl = 0; gl < 2; ++gl) {
                    const float w0 = in0 ? p0 * (gl ? bf_hi(v0) : bf_lo(v0)) : 0.f;
                    const float w1 = in1 ? p1 * (gl ? bf_hi(v1) : bf_lo(v1)) : 0.f;
                    const uint32_t near = pack_bf16(w0, w1);
                    const uint32_t rest = pack_bf16(w0 - bf_lo(near), w1 - bf_hi(near));
                    const uint32_t at = wbuf + c * G::WEIGHT_TILE + (2 * (2 * p + gl)) * 32 + ((g & 3) * 2 + (g >> 2)) * 4;
                    sts32(at, near);
                    sts32(at + 32, rest);
                }
            }
            __syncwarp();
            // ---- weighted codes of V: rows c, c + 8 | c + 4, c + 12 of a tile are this lane's pairs
#pragma unroll
            for (int t = 0; t < kChunkTiles; ++t) {
                if (t < ntiles) {
                    uint32_t b0, b1;
                    lds64(wbuf + t * G::WEIGHT_TILE + (g % G::COLS) * 32 + c * 8, b0, b1);
#pragma unroll
                    for (int p = 0; p < PLANES; ++p) {
                        const uint32_t at = st + t * G::TILE + p * kTileBytes + kPartBytes + c * 32 + g * 4;
                        const uint32_t x0 = lds32(at), x1 = lds32(at + 4 * 32), x2 = lds32(at + 8 * 32), x3 = lds32(at + 12 * 32);
                        const uint32_t l02 = __byte_perm(x0, x2, 0x5410), h02 = __byte_perm(x0, x2, 0x7632);
                        const uint32_t l13 = __byte_perm(x1, x3, 0x5410), h13 = __byte_perm(x1, x3, 0x7632);
                        mma(o[p][0], code_pair<0>(l02), code_pair<0>(h02), code_pair<0>(l13), code_pair<0>(h13), b0, b1);
                        mma(o[p][1], code_pair<1>(l02), code_pair<1>(h02), code_pair<1>(l13), code_pair<1>(h13), b0, b1);
                        mma(o[p][2], code_pair<2>(l02), code_pair<2>(h02), code_pair<2>(l13), code_pair<2>(h13), b0, b1);
                        mma(o[p][3], code_pair<3>(l02), code_pair<3>(h02), code_pair<3>(l13), code_pair<3>(h13), b0, b1);
                    }
                }
            }
            // The stage and the weights have been read by every lane before either is written again; what was put into the stage
            // by this warp is ordered before the copy engine's writes.
            if (w.new_row) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            ++consumed;
            issue_one();
        }
        if (!alive) break;
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
        // Lane (g, c) holds dimensions 8 g .. 8 g + 7 of a plane under the weights of group c: the ones that count where that is
        // their group.  Rounded weights and rests are added up here.
        auto own_piece = [&](int p) { return c == 2 * p + (g >> 2); };
        auto piece = [&](int p, float (&f)[8]) {
            const float inv = inverse_sum(l);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                f[r] = (o[p][r][0] + o[p][r][1]) * inv;
                f[r + 4] = (o[p][r][2] + o[p][r][3]) * inv;
            }
        };
        bf16* const out = reinterpret_cast<bf16*>(a.out) + (size_t)w.bh * HD;
        if (a.splits == 1) {
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                float f[8];
                piece(p, f);
                if (own_piece(p)) *reinterpret_cast<uint4*>(out + p * 64 + g * 8) = pack8(f);
            }
        } else {
            float* ws = a.ws + ((size_t)w.bh * a.splits + w.sp) * (HD + 4);
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                float f[8];
                piece(p, f);
                if (own_piece(p)) {
                    *reinterpret_cast<float4*>(ws + p * 64 + g * 8) = make_float4(f[0], f[1], f[2], f[3]);
                    *reinterpret_cast<float4*>(ws + p * 64 + g * 8 + 4) = make_float4(f[4], f[5], f[6], f[7]);
                }
            }
            if (lane == 0) ws[HD] = l == 0.f ? kNegInf : m + log2f(l);
            __threadfence();   // the partial is visible before this item counts itself in
            __syncwarp();
            int last = 0;
            if (lane == 0) last = atomicAdd(a.counters + w.bh, 1) == a.splits - 1;
            last = __shfl_sync(0xffffffffu, last, 0);
            if (last) {   // every part of (b,h) has written: fold the partials (normalised, weight 2^lse each)
                __threadfence();
                const int sub = lane % LPR;
                SoftmaxState state;
                state.init();
                for (int s2 = lane / LPR; s2 < a.splits; s2 += 32 / LPR) {
                    const float* part = a.ws + ((size_t)w.bh * a.splits + s2) * (HD + 4);
                    const float lse = __ldcg(part + HD);
                    const float4 x = __ldcg(reinterpret_cast<const float4*>(part + sub * 8));
                    const float4 y = __ldcg(reinterpret_cast<const float4*>(part + sub * 8 + 4));
                    const float a2[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                    state.merge(lse, 1.f, a2);
                }
                state.merge_row_groups<LPR>();
                if (lane < LPR) {
                    float f[8];
                    state.normalised(f);
                    *reinterpret_cast<uint4*>(out + sub * 8) = pack8(f);
                }
                if (lane == 0) a.counters[w.bh] = 0;
            }
        }
        if (w.sp == 0 && cc.h == 0 && lane == 0) {
            if (w.n == 0) raise_status(a.dev_status, BT_DEV_EMPTY);
            if (w.overflow) raise_status(a.dev_status, BT_DEV_OVERFLOW);
        }
        settle();
        pend_arrival = seq_arrival;
        pend_b = w.b;
        pend_n = w.n;
        pend_overflow = w.overflow;
        cc = cn;
    }
    settle();
    if (!alive) {
        // a copy never completed: report it, give the copies still in flight one more bounded wait so
        // that none lands in shared memory after the CTA is gone, and leave
        if (lane == 0) raise_status(a.dev_status, BT_DEV_TIMEOUT);
        for (; consumed < issued; ++consumed)
            if (!mbar_wait_polls(bar0 + 8 * (consumed % STAGES), (consumed / STAGES) & 1, kPollLimit)) break;
    }
}

#ifndef BT_KV4_WARPS_64
#define BT_KV4_WARPS_64 16
#define BT_KV4_STAGES_64 3
#define BT_KV4_WARPS_128 8
#define BT_KV4_STAGES_128 3
#endif

template <int HD, int STAGES, int MAX_WARPS>
static cudaError_t launch_t(const Kv4DecodeArgs& a, cudaStream_t stream)
{
    int dev = 0, sms = 0;
    cudaError_t e = current_device(&dev, &sms);
    if (e != cudaSuccess) return e;
    static PerDeviceOnce limit_raised;
    e = raise_smem_limit_once(limit_raised, dev, block_decode_kv4_kernel<HD, STAGES, MAX_WARPS>, smem_bytes<HD>(MAX_WARPS, STAGES));
    if (e != cudaSuccess) return e;
    const long long items = (long long)a.B * a.H * a.splits;
    if (items > 0x7fffffffLL - 4096) return cudaErrorInvalidConfiguration;
    const long long grid = items < sms ? items : sms;
    const long long each = (items + grid - 1) / grid;
    const int warps = (int)(each < MAX_WARPS ? each : MAX_WARPS);
    return launch_pdl(block_decode_kv4_kernel<HD, STAGES, MAX_WARPS>, dim3((unsigned)grid), dim3(warps * 32), (size_t)smem_bytes<HD>(warps, STAGES), stream, a);
}

}  // namespace kv4

cudaError_t launch_block_decode_kv4(const Kv4DecodeArgs& a, cudaStream_t stream)
{
    return a.hd == 64 ? kv4::launch_t<64, BT_KV4_STAGES_64, BT_KV4_WARPS_64>(a, stream) : kv4::launch_t<128, BT_KV4_STAGES_128, BT_KV4_WARPS_128>(a, stream);
}

}  // namespace bt
