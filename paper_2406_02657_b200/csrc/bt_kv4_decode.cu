// Block-decoder decode attention over the 4-bit cache (paper section 2.3), with the append of a step fused in.
//
// With (s, u) the step and code of K, (t, w) those of V, g(d) the group of 32 dimensions that d lies in:
//   score_j = scale * sum_g s_jg sum_{d in g} q_d u_jd,     out_d = sum_j (p_j t_jg(d)) w_jd / sum_j p_j.
// What bounds the kernel is the 1.125 hd bytes a row of the cache, 3.6 times fewer than of the bf16 one, and next to it the
// instructions: at 6.5 TB/s a scheduler has 800 cycles for 64 rows of 64 dimensions (8192 values), so a value may not be unpacked to
// fp32 and multiplied on its own (three slots or more).  Codes stay whole numbers here: one mask gives the codes u + 8 of four even dimensions as
// bytes, another those of four odd ones as 16 (u + 8), and warp-level m16n8k32 integer instructions multiply them (8 cycles each, half of
// what 16-bit floats would take; unpacking to those also takes seven integer instructions for eight values instead of two).
// The other operand becomes whole numbers cut into bytes, and the sums are exact:
//   scores:  A = codes of 16 rows x 32 dimensions; B = the query, times a power of two that brings a group's largest value to 2^21 .. 2^22 (odd
//            dimensions to 2^17 .. 2^18: half a step of the rounding is 2^-18 of the group's largest at most), as three signed bytes, of which each has
//            two columns: the values of one group of a plane and zeros elsewhere, and the other's.  The lanes that share a row then hold
//            the sums of one byte each; two exchanges between them, with shifts, give lane c the whole sums of tile c of a unit.
//            (Every byte in every column, one after the other into the same sums, needs no exchange but three times the products: 128 us where
//            this takes 118 over 24 x 16 items of 12001 to 16000 rows of 128, at the clock that the power limit leaves.)
//   output:  A = codes of V transposed, 16 dimensions x 32 rows; B = the weights p t of a group as whole numbers of 32 bits, times a power
//            of two that has the group's largest so far at 2^28 .. 2^32 (so that the rounding, 2^-29 of the largest, does not add up over a
//            million rows), a byte in each of four columns (2 groups x 4 bytes).  Sums are kept as 32-bit whole numbers until what they are
//            relative to changes.
// Products of the same bytes with rows of eights give what the offsets of the codes add.
//
// As in the streaming kernel of the bf16 cache: one persistent CTA per SM, every warp on its own with a ring of chunks (64 or 128
// rows, one bulk copy: tiles hold K and V), work items (sequence, head, part of the rows), partial results joined by the part that ends
// last, the length raised by the item that reads it last.  A new row is quantised by the warp that owns the last row, stored into
// the cache, and put into the copied chunk, where it is attended like any other: a step gives what append and attention give.
#include <type_traits>

#include "bt_decode_ring.cuh"
#include "bt_kv4.cuh"

namespace bt {
namespace kv4 {

constexpr int kUnitTiles = 4, kUnitRows = kUnitTiles * kTileRows;   // rows that a warp scores at once, two a lane
constexpr uint32_t kPollLimit = 1u << 24;   // polls of one wait before giving up (each poll suspends briefly)

// UNITS: units of a chunk.  Two planes of a unit or two units of a plane go through the arithmetic together: what a chunk costs beside its
// products is shared, and a warp has twice the independent instructions.
template <int HD, int UNITS>
struct Geo {
    static constexpr int PLANES = HD / 64;
    static constexpr int ROWS = UNITS * kUnitRows;
    static constexpr int TILE = PLANES * kTileBytes;
    static constexpr int STAGE = UNITS * kUnitTiles * TILE;
    static constexpr int WEIGHT_TILE = 8 * kTileRows + 16;        // 8 columns (group, byte) of 16 rows; 16 more spread the tiles over the banks
    static constexpr int WEIGHT_PLANE = kUnitTiles * WEIGHT_TILE;   // of a unit
    static constexpr int WEIGHTS = UNITS * PLANES * WEIGHT_PLANE;
};
template <int HD, int UNITS>
constexpr int smem_bytes(int warps, int stages) { return warps * (stages * (Geo<HD, UNITS>::STAGE + 8) + Geo<HD, UNITS>::WEIGHTS); }

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
__device__ __forceinline__ void sts16(uint32_t addr, uint32_t x) { asm volatile("st.shared.u16 [%0], %1;" ::"r"(addr), "h"((uint16_t)x) : "memory"); }

// four codes of a word as bytes: u + 8 of the even dimensions, 16 (u + 8) of the odd ones
__device__ __forceinline__ uint32_t even_codes(uint32_t w) { return w & 0x0f0f0f0fu; }
__device__ __forceinline__ uint32_t odd_codes(uint32_t w) { return w & 0xf0f0f0f0u; }
// D (16 x 8, 32-bit whole numbers) += A (16 x 32, unsigned bytes) B (32 x 8, signed or unsigned bytes)
__device__ __forceinline__ void mma_signed(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_signed_from(int (&d)[4], int even, int odd, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%10,%11};"
        : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "r"(even), "r"(odd));
}
__device__ __forceinline__ void mma_unsigned(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.u8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 2^(TO - e) for a largest magnitude 2^e <= x < 2^(e + 1) of what is multiplied with it, as far as that is a normal number
template <int TO>
__device__ __forceinline__ float power_to(float x)
{
    const int e = (int)(__float_as_uint(x) >> 23) & 255;                       // 127 + e
    return __uint_as_float((uint32_t)(254 + TO - max(e, 1 + TO)) << 23);        // exponent field 127 + TO - e, at most 253
}
__device__ __forceinline__ float inverse_power(float x) { return __uint_as_float(0x7f000000u - __float_as_uint(x)); }
__device__ __forceinline__ uint32_t whole(float x)
{
    uint32_t w;
    asm("cvt.rni.u32.f32 %0, %1;" : "=r"(w) : "f"(x));
    return w;
}
// x, NaN included, but no infinity above
__device__ __forceinline__ float at_most_largest(float x)
{
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(3.40282347e38f));
    return y;
}
// a byte of each of four words
__device__ __forceinline__ uint32_t gather_byte(const uint32_t (&w)[4], int byte)
{
    const uint32_t pick = byte | (4 + byte) << 4;
    return __byte_perm(__byte_perm(w[0], w[1], pick), __byte_perm(w[2], w[3], pick), 0x5410);
}
constexpr uint32_t kEightsEven = 0x08080808u, kEightsOdd = 0x80808080u;   // what even_codes and odd_codes give for codes of 0
constexpr float kWholeAt = 12582912.f;   // 1.5 * 2^23
constexpr uint32_t kWholeBits = 0x4B400000u;
constexpr int kUnitsPerSum = 512;        // 64 rows add at most 64 * 240 * 255 to a sum of bytes: 2^31 holds 548 times that
constexpr float kHeadroom = 2.f;         // how far (log2) scores may exceed what weights are relative to before that changes: a weight is 4
                                         // at most then, and its product with the largest step there is, 146 * 2^118, a number of fp32
constexpr int kJoin = 32;               // partial results requested at once, a warp's weights
constexpr int kWeightTo = 28;            // the largest weight to 2^28 .. 2^29; it may grow until ...
constexpr float kWeightEnd = 4294967296.f;
// the largest of a warp's values that are numbers
__device__ __forceinline__ float warp_max(float x)
{
    float m;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(x));
    return m;
}
struct Params : Kv4DecodeArgs {
    Divisor by_splits, by_heads;
};

// Work item (b, h, part): its rows r0 .. r1 - 1; n counts the new row, which is row n - 1 and lies here when new_row is set.
struct Work {
    int bh, sp, b, n, r0, r1;
    bool new_row, overflow;
};
__device__ __forceinline__ int sequence_of(int item, const Params& a) { return divide(divide(item, a.by_splits), a.by_heads); }
__device__ __forceinline__ Work work_of(int item, const Params& a, int n)   // n: the sequence's length
{
    Work w;
    w.bh = divide(item, a.by_splits);
    w.sp = item - w.bh * a.splits;
    w.b = divide(w.bh, a.by_heads);
    n = n < 0 ? 0 : (n > a.n_max ? a.n_max : n);
    const bool append = a.k_new != nullptr && n < a.n_max;   // a full cache takes no row: flagged, attended as it is
    w.overflow = a.k_new != nullptr && !append;
    n += append ? 1 : 0;
    w.n = n;
    // whole units per part, as even as that goes (trailing parts may be empty)
    const int per = divide((n + kUnitRows - 1) / kUnitRows + a.splits - 1, a.by_splits) * kUnitRows;
    w.r0 = min(n, w.sp * per);
    w.r1 = min(n, w.r0 + per);
    w.new_row = append && w.r1 == n && w.r0 < n;
    return w;
}

template <int HD, int UNITS, int STAGES, int MAX_WARPS>
__global__ void __launch_bounds__(MAX_WARPS * 32, 1) block_decode_kv4_kernel(const __grid_constant__ Params a)
{
    using G = Geo<HD, UNITS>;
    constexpr int PLANES = G::PLANES, LPR = HD / 8;
    extern __shared__ __align__(128) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, c = lane & 3;   // row and column of a fragment
    const int own_by_2 = c & 2 ? 65536 : 1, got_by_2 = c & 2 ? 1 : 65536, own_by_1 = c & 1 ? 256 : 1, got_by_1 = c & 1 ? 1 : 256;   // byte c of a sum
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
    // While the kernel before this one drains, have the chunks that this warp will request first brought into L2: which those are comes
    // from a look at the length that may be out of date (read past L1), so it is a hint and decides nothing.
    if (first < n_items && lane == 0) {
        const Work h = work_of(first, a, __ldcg(a.len + sequence_of(first, a)));
        const uint32_t bytes = (uint32_t)((min(STAGES * G::ROWS, h.r1 - h.r0) + kTileRows - 1) / kTileRows) * G::TILE;
        if (bytes > 0)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(kv + (size_t)h.bh * a.slab_bytes + (size_t)(h.r0 / kTileRows) * G::TILE), "r"(bytes) : "memory");
    }
    pdl_wait();

    // ---- producer (kept by every lane, acted on by lane 0): where the next chunk to request lies
    int p_item = first, p_left = 0;   // rows of that item not yet requested
    const uint8_t* p_from = kv;
    auto p_seek = [&]() {   // to an item that has rows
        for (; p_item < n_items; p_item += stride) {
            const Work w = work_of(p_item, a, a.len[sequence_of(p_item, a)]);
            p_left = w.r1 - w.r0;
            p_from = kv + (size_t)w.bh * a.slab_bytes + (size_t)(w.r0 / kTileRows) * G::TILE;
            if (p_left > 0) return;
        }
    };
    uint32_t issued = 0, consumed = 0;
    auto issue_one = [&]() {
        if (p_left <= 0) return;
        const uint32_t st = issued % STAGES;
        if (lane == 0) {
            const uint32_t bytes = (uint32_t)((min(G::ROWS, p_left) + kTileRows - 1) / kTileRows) * G::TILE;
            mbar_expect_tx(bar0 + 8 * st, bytes);
            ring::bulk_load(ring0 + st * G::STAGE, p_from, bytes, bar0 + 8 * st, policy);
        }
        ++issued;
        p_from += G::STAGE;
        p_left -= G::ROWS;
        if (p_left <= 0) {
            p_item += stride;
            p_seek();
        }
    };
    p_seek();
    for (int s = 0; s < STAGES; ++s) issue_one();

    // ---- consumer: whole items, chunk by chunk
    bool alive = true;
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
    if (first < n_items) fetch_q(divide(first, a.by_splits));
    for (int item = first; item < n_items; item += stride) {
        const Work w = work_of(item, a, a.len[sequence_of(item, a)]);
        // An item counts itself in as soon as its own read of the length has returned (the increment is computed from it).
        int seq_arrival = -1;
        if (a.k_new != nullptr && lane == 0) {
            int one;
            asm volatile("and.b32 %0, %1, 0;\n\tadd.s32 %0, %0, 1;" : "=r"(one) : "r"(w.n));
            seq_arrival = atomicAdd(a.counters + (size_t)a.B * a.H + w.b, one);
        }
        // Query fragments: lane (g, c) holds, of dimensions 16 c .. 16 c + 15 of a plane in the order of the codes of two words, byte g >> 1 for
        // the column of group g & 1: zeros where the dimensions are the other group's, and in the two columns that are left.
        uint32_t qf[PLANES][2][2];         // word, even | odd dimensions
        int q_from[PLANES][2];             // what the sums of a byte of a group (columns 2 c, 2 c + 1) start from, so that the codes' eights are taken out
        float q_unit[PLANES][2];           // what a group's whole sum has to be multiplied with
        {
            const uint32_t own = (g & 1) == (c >> 1) && g < 6 ? 0xffffffffu : 0u;
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                // (lanes c and c ^ 1 have the dimensions of one group, lanes c ^ 2 the other's)
                uint32_t top = magnitude_of(magnitude_max(magnitude_max8(q_next[p][0]), magnitude_max8(q_next[p][1])));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                const float to = power_to<21>(__uint_as_float(top << 16));
                // a query with a value that is not finite gives NaN throughout
                const float unit = top < 0x7f80u ? inverse_power(to) : __uint_as_float(0x7fffffffu), other = __shfl_xor_sync(0xffffffffu, unit, 2);
                q_unit[p][0] = c & 2 ? other : unit;
                q_unit[p][1] = c & 2 ? unit : other;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float f[8];
                    unpack8(q_next[p][i], f);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        // Adding 1.5 * 2^23 rounds to whole numbers and leaves them in the low bits: kWholeBits + n.  Bytes 0 .. 255 then stand
                        // for digits -128 .. 127.
                        uint32_t x[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[j] = __float_as_uint(fmaf(f[2 * j + h], h ? to * 0.0625f : to, kWholeAt)) + (0x00808080u - kWholeBits);
                        qf[p][i][h] = (gather_byte(x, g >> 1) ^ 0x80808080u) & own;
                    }
                }
                int off[4];
                mma_signed_from(off, 0, 0, kEightsEven, kEightsEven, kEightsOdd, kEightsOdd, qf[p][0][0], qf[p][0][1]);
                mma_signed(off, kEightsEven, kEightsEven, kEightsOdd, kEightsOdd, qf[p][1][0], qf[p][1][1]);
                q_from[p][0] = -off[0];
                q_from[p][1] = -off[1];
            }
        }
        if (item + stride < n_items) fetch_q(divide(item + stride, a.by_splits));
        float m = kNegInf, l = 0.f;                // what scores are relative to, the sum of 2^(score - m)
        // of every group: the largest weight p t that this lane has had, and the power of two for the largest of all lanes'
        float w_most[PLANES][2], w_to[PLANES][2];
        float o[PLANES][4][2], bad[PLANES][2];     // even | odd dimension; not a number once a step of V was none
        int sums[PLANES][4][4], eights[PLANES][4], pending = 0;
#pragma unroll
        for (int p = 0; p < PLANES; ++p) {
            bad[p][0] = bad[p][1] = 0.f;
            w_most[p][0] = w_most[p][1] = 0.f;
            w_to[p][0] = w_to[p][1] = power_to<kWeightTo>(0.f);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                o[p][r][0] = o[p][r][1] = 0.f;
                eights[p][r] = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) sums[p][r][i] = 0;
            }
        }
        // the whole-number sums of bytes b and b + 1 of the weights into the outputs (lanes with odd c: bytes 2 and 3, 2^16 times as much in the end)
        auto flush = [&]() {
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    o[p][r][0] += fmaf(256.f, (float)(sums[p][r][1] - eights[p][1]), (float)(sums[p][r][0] - eights[p][0]));
                    o[p][r][1] += fmaf(256.f, (float)(sums[p][r][3] - eights[p][3]), (float)(sums[p][r][2] - eights[p][2]));
#pragma unroll
                    for (int i = 0; i < 4; ++i) sums[p][r][i] = 0;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) eights[p][i] = 0;
            }
            pending = 0;
        };

        // The rows of a chunk: N units, of which nvalid rows are there.
        auto chunk = [&](auto units, uint32_t st, int nvalid) {
            constexpr int N = decltype(units)::value;
            // ---- scores of rows 16 c + 2 g and 16 c + 2 g + 1 of every unit, in this lane
            float s[N][2];
            float t[N][PLANES][2][2];   // steps of V, then weights: group, row
            bool in[N][2];
            const uint32_t own_tile = st + c * G::TILE + g * 8;
            float top = kNegInf;
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const uint32_t tile0 = st + u * (kUnitTiles * G::TILE);
                s[u][0] = s[u][1] = 0.f;
#pragma unroll
                for (int p = 0; p < PLANES; ++p) {
                    int acc[kUnitTiles][4];
                    // (Tiles that the chunk has not are multiplied all the same: what a stage holds there is whole numbers too, and their
                    // scores are set aside below.  Without branches the tiles' instructions interleave.)
#pragma unroll
                    for (int k = 0; k < kUnitTiles; ++k) {
                        const uint4 x = lds128(tile0 + k * G::TILE + p * kTileBytes + lane * 16);   // two words of the even row, two of the odd
                        const uint32_t a0 = even_codes(x.x), a1 = even_codes(x.z), a2 = odd_codes(x.x), a3 = odd_codes(x.z);
                        const uint32_t b0 = even_codes(x.y), b1 = even_codes(x.w), b2 = odd_codes(x.y), b3 = odd_codes(x.w);
                        mma_signed_from(acc[k], q_from[p][0], q_from[p][1], a0, a1, a2, a3, qf[p][0][0], qf[p][0][1]);
                        mma_signed(acc[k], b0, b1, b2, b3, qf[p][1][0], qf[p][1][1]);
                    }
                    // Lane c has byte c of all tiles' sums (lane 3: zeros) and needs all bytes of tile c's: tiles are exchanged with lane c ^ 2,
                    // two bytes away, then with lane c ^ 1.
                    int two[2][4];
                    float mine[4];
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int keep = c & 2 ? acc[2 + k][i] : acc[k][i];
                            const int got = __shfl_xor_sync(0xffffffffu, c & 2 ? acc[k][i] : acc[2 + k][i], 2);
                            two[k][i] = keep * own_by_2 + got * got_by_2;
                        }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int keep = c & 1 ? two[1][i] : two[0][i];
                        const int got = __shfl_xor_sync(0xffffffffu, c & 1 ? two[0][i] : two[1][i], 1);
                        mine[i] = (float)(keep * own_by_1 + got * got_by_1);
                    }
                    uint32_t k0, k1;
                    lds64(own_tile + u * (kUnitTiles * G::TILE) + p * kTileBytes + kStepsAt, k0, k1);
                    // (the query's power of two goes to the step, so that nothing between is larger than the products themselves)
                    s[u][0] = fmaf(mine[1], at_most_largest(bf_hi(k0) * q_unit[p][1]), fmaf(mine[0], at_most_largest(bf_lo(k0) * q_unit[p][0]), s[u][0]));
                    s[u][1] = fmaf(mine[3], at_most_largest(bf_hi(k1) * q_unit[p][1]), fmaf(mine[2], at_most_largest(bf_lo(k1) * q_unit[p][0]), s[u][1]));
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    in[u][r] = u * kUnitRows + 16 * c + 2 * g + r < nvalid;
                    s[u][r] = in[u][r] ? s[u][r] * a.scale_log2 : kNegInf;
                    top = fmaxf(top, s[u][r]);
                }
                // steps of V of the two rows; a row that is not there has no weight whatever its step is
#pragma unroll
                for (int p = 0; p < PLANES; ++p) {
                    uint32_t v[2];
                    lds64(own_tile + u * (kUnitTiles * G::TILE) + p * kTileBytes + kStepsAt + 64, v[0], v[1]);
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        v[r] = in[u][r] ? v[r] : 0u;
                        t[u][p][0][r] = bf_lo(v[r]);
                        t[u][p][1][r] = bf_hi(v[r]);
                        bad[p][0] = fmaf(0.f, t[u][p][0][r], bad[p][0]);
                        bad[p][1] = fmaf(0.f, t[u][p][1][r], bad[p][1]);
                    }
                }
            }
            // What scores are relative to changes (for all of the warp) when one would leave the headroom.
            const float mn = fmaxf(m, warp_max(top));
            const bool grown = mn > m + kHeadroom || (m == kNegInf && mn > m);
            const float cf = grown ? ex2(m - mn) : 1.f;
            m = grown ? mn : m;
            const float m_use = softmax_reference(m);
            l *= cf;
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                w_most[p][0] *= cf;
                w_most[p][1] *= cf;
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const float p0 = ex2(s[u][0] - m_use), p1 = ex2(s[u][1] - m_use);
                l += p0 + p1;
#pragma unroll
                for (int p = 0; p < PLANES; ++p)
#pragma unroll
                    for (int gl = 0; gl < 2; ++gl) {
                        t[u][p][gl][0] *= p0;
                        t[u][p][gl][1] *= p1;
                        w_most[p][gl] = fmaxf(w_most[p][gl], fmaxf(t[u][p][gl][0], t[u][p][gl][1]));
                    }
            }
            // ... and what the weights of a group are relative to, then and when one would leave 32 bits.  (A power of two for all
            // groups would take the precision of those whose steps are small beside another's; it would save 0.9 of 60.6 us over 24 x 16 items of
            // 12001 to 16000 rows of 64, 0.7 of 115.6 of 128.  One vote for all that leads here: three ways in are compiled as copies, and the code
            // then outgrows what is near an SM: 5.2 us instead of 4.5 over 32 pairs of 512 rows in eight parts.)
            float end = 0.f;
#pragma unroll
            for (int p = 0; p < PLANES; ++p) end = fmaxf(end, fmaxf(w_most[p][0] * w_to[p][0], w_most[p][1] * w_to[p][1]));
            if (__any_sync(0xffffffffu, grown || pending >= kUnitsPerSum || end >= kWeightEnd)) {
                if (pending > 0) flush();
#pragma unroll
                for (int p = 0; p < PLANES; ++p) {
                    float co = 0.f;   // of the group whose weights this lane's outputs are under
#pragma unroll
                    for (int gl = 0; gl < 2; ++gl) {
                        const float to = power_to<kWeightTo>(warp_max(w_most[p][gl]));
                        if (gl == c >> 1) co = cf * to * inverse_power(w_to[p][gl]);   // at most 2, in this order
                        w_to[p][gl] = to;
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        o[p][r][0] *= co;
                        o[p][r][1] *= co;
                    }
                }
            }
            pending += N;
            // ---- weights of the rows: column 4 (group) + byte of a plane
#pragma unroll
            for (int u = 0; u < N; ++u) {
#pragma unroll
                for (int p = 0; p < PLANES; ++p) {
#pragma unroll
                    for (int gl = 0; gl < 2; ++gl) {
                        const uint32_t at = wbuf + (u * PLANES + p) * G::WEIGHT_PLANE + c * G::WEIGHT_TILE + gl * (4 * kTileRows) + 2 * g;
                        const uint32_t x = whole(t[u][p][gl][0] * w_to[p][gl]), y = whole(t[u][p][gl][1] * w_to[p][gl]);
                        sts16(at, __byte_perm(x, y, 0x0040));
                        sts16(at + kTileRows, __byte_perm(x, y, 0x0051));
                        sts16(at + 2 * kTileRows, __byte_perm(x, y, 0x0062));
                        sts16(at + 3 * kTileRows, __byte_perm(x, y, 0x0073));
                    }
                }
            }
            __syncwarp();
            // ---- weighted codes of V: rows 4 c .. 4 c + 3 of two tiles are this lane's
#pragma unroll
            for (int u = 0; u < N; ++u) {
#pragma unroll
                for (int k = 0; k < kUnitTiles; k += 2) {   // (rows that are not there have weights of zero)
#pragma unroll
                    for (int p = 0; p < PLANES; ++p) {
                        const uint32_t wt = wbuf + (u * PLANES + p) * G::WEIGHT_PLANE + k * G::WEIGHT_TILE + lane * 4;
                        const uint32_t b0 = lds32(wt), b1 = lds32(wt + G::WEIGHT_TILE);
                        const uint32_t at = st + (u * kUnitTiles + k) * G::TILE + p * kTileBytes + kPartBytes + c * 128 + ((g ^ (2 * c)) << 4);
                        const uint4 x = lds128(at), y = lds128(at + G::TILE);
                        mma_unsigned(sums[p][0], even_codes(x.x), odd_codes(x.x), even_codes(y.x), odd_codes(y.x), b0, b1);
                        mma_unsigned(sums[p][1], even_codes(x.y), odd_codes(x.y), even_codes(y.y), odd_codes(y.y), b0, b1);
                        mma_unsigned(sums[p][2], even_codes(x.z), odd_codes(x.z), even_codes(y.z), odd_codes(y.z), b0, b1);
                        mma_unsigned(sums[p][3], even_codes(x.w), odd_codes(x.w), even_codes(y.w), odd_codes(y.w), b0, b1);
                        mma_unsigned(eights[p], kEightsEven, kEightsOdd, kEightsEven, kEightsOdd, b0, b1);
                    }
                }
            }
        };

        for (int row = w.r0; row < w.r1; row += G::ROWS) {
            const uint32_t sidx = consumed % STAGES;
            // the outcome is made warp-uniform: what follows needs all 32 lanes
            if (!__all_sync(0xffffffffu, mbar_wait_polls(bar0 + 8 * sidx, (consumed / STAGES) & 1, kPollLimit))) {
                alive = false;
                break;
            }
            const uint32_t st = ring0 + sidx * G::STAGE;
            const int nvalid = min(G::ROWS, w.r1 - row);
            if (w.new_row && row + G::ROWS >= w.r1) {
                // the new row, eight values a lane: lanes 0 .. LPR - 1 K, the next V (at head_dim 64 the upper half repeats them)
                const int part = (lane / LPR) & 1, piece = lane % LPR;
                const uint4 x = ld_plain(reinterpret_cast<const bf16*>(part == 0 ? a.k_new : a.v_new) + (size_t)w.bh * HD + piece * 8);
                const Step sg = step_of_lanes(x);
                const uint32_t codes = sg.finite ? codes8(x, sg.inv) : kZeroCodes;
                if (lane < 2 * LPR) {
                    const int r = w.n - 1 - row, in_tile = r % kTileRows, j = piece & 7;
                    const uint32_t tile = (uint32_t)(r / kTileRows) * G::TILE + (piece / 8) * kTileBytes;
                    const uint32_t step_at = tile + kStepsAt + part * 64 + in_tile * 4 + (j >> 2) * 2;
                    uint8_t* copy = ring_ptr + sidx * G::STAGE;
                    uint8_t* held = kv + (size_t)w.bh * a.slab_bytes + (size_t)(row / kTileRows) * G::TILE;
                    if (part == 0) {
                        const uint32_t at = tile + k_codes_at(in_tile, j);
                        *reinterpret_cast<uint32_t*>(copy + at) = codes;
                        *reinterpret_cast<uint32_t*>(held + at) = codes;
                    } else {
                        const uint32_t at = tile + v_codes_at(in_tile, j);
#pragma unroll
                        for (int i = 0; i < 4; ++i) copy[at + 4 * i] = held[at + 4 * i] = (uint8_t)(codes >> (8 * i));
                    }
                    if ((j & 3) == 0) {
                        *reinterpret_cast<uint16_t*>(copy + step_at) = (uint16_t)sg.bits;
                        *reinterpret_cast<uint16_t*>(held + step_at) = (uint16_t)sg.bits;
                    }
                }
                __syncwarp();
            }
            // a chunk of one unit, or of two where it has more than 64 rows
            if (UNITS == 1 || nvalid <= kUnitRows) chunk(std::integral_constant<int, 1>(), st, nvalid);
            else chunk(std::integral_constant<int, UNITS>(), st, nvalid);
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
        flush();
        // Lane (g, c) holds dimensions 8 g .. 8 g + 7 of a plane under two bytes of the weights of group c >> 1: the low ones in lanes of even c,
        // the high ones in those of odd c.  They count where that is the dimensions' group, and are added up here.
        const bool own_piece = c == 2 * (g >> 2);
        // (The sum of the weights divides first: with the weights' power of two it could leave the normal numbers.)
        const float share = (c & 1 ? 65536.f : 1.f) * inverse_sum(l);
        auto piece = [&](int p, float (&f)[8]) {
            const bool bad0 = __any_sync(0xffffffffu, bad[p][0] != 0.f), bad1 = __any_sync(0xffffffffu, bad[p][1] != 0.f);
            const float u = (g < 4 ? bad0 : bad1) ? __uint_as_float(0x7fffffffu) : inverse_power(c & 2 ? w_to[p][1] : w_to[p][0]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                f[2 * r] = o[p][r][0] * share;
                f[2 * r + 1] = o[p][r][1] * (share * 0.0625f);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (f[i] + __shfl_xor_sync(0xffffffffu, f[i], 1)) * u;
        };
        bf16* const out = reinterpret_cast<bf16*>(a.out) + (size_t)w.bh * HD;
        if (a.splits == 1) {
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                float f[8];
                piece(p, f);
                if (own_piece) *reinterpret_cast<uint4*>(out + p * 64 + g * 8) = pack8(f);
            }
        } else {
            float* ws = a.ws + ((size_t)w.bh * a.splits + w.sp) * (HD + 4);
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                float f[8];
                piece(p, f);
                if (own_piece) {
                    *reinterpret_cast<float4*>(ws + p * 64 + g * 8) = make_float4(f[0], f[1], f[2], f[3]);
                    *reinterpret_cast<float4*>(ws + p * 64 + g * 8 + 4) = make_float4(f[4], f[5], f[6], f[7]);
                }
            }
            if (lane == 0) ws[HD] = l == 0.f ? kNegInf : m + log2f(l);
            // The partial is visible before this item counts itself in, and the others' partials to the item that comes last: release and acquire
            // by the lane that counts, and for the other lanes by the warp's barriers before and after.
            __syncwarp();
            int last = 0;
            if (lane == 0) {
                int before;
                asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(a.counters + w.bh) : "memory");
                last = before == a.splits - 1;
            }
            last = __shfl_sync(0xffffffffu, last, 0);
            if (last) {   // every part of (b,h) has written: fold the partials (normalised, weight 2^lse each)
                __syncwarp();
                // HD / 32 dimensions a lane, of 32 parts at once, and the weights, two parts a lane at most (splits <= 64): all requested before any is used
                constexpr int DIMS = HD / 32;
                const float* parts = a.ws + (size_t)w.bh * a.splits * (HD + 4);
                float x[kJoin][DIMS];
                auto request = [&](int s0) {
#pragma unroll
                    for (int i = 0; i < kJoin; ++i) {
#pragma unroll
                        for (int j = 0; j < DIMS; ++j) x[i][j] = 0.f;
                        if (s0 + i < a.splits) {
                            const float* part = parts + (s0 + i) * (HD + 4) + lane * DIMS;
                            if constexpr (DIMS == 4) {
                                const float4 v = __ldcg(reinterpret_cast<const float4*>(part));
                                x[i][0] = v.x, x[i][1] = v.y, x[i][2] = v.z, x[i][3] = v.w;
                            } else {
                                const float2 v = __ldcg(reinterpret_cast<const float2*>(part));
                                x[i][0] = v.x, x[i][1] = v.y;
                            }
                        }
                    }
                };
                float lse0 = lane < a.splits ? __ldcg(parts + lane * (HD + 4) + HD) : kNegInf;
                float lse1 = lane + 32 < a.splits ? __ldcg(parts + (lane + 32) * (HD + 4) + HD) : kNegInf;
                request(0);
                const float ref = softmax_reference(warp_max(fmaxf(lse0, lse1)));
                lse0 = ex2(lse0 - ref);
                lse1 = ex2(lse1 - ref);
                float total = lse0 + lse1;
#pragma unroll
                for (int off = 16; off >= 1; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
                // (the weights' sum divides them before they meet a partial: several partials near the end of fp32 add up to one)
                const float inv = inverse_sum(total);
                lse0 *= inv;
                lse1 *= inv;
                float f[DIMS];
#pragma unroll
                for (int i = 0; i < DIMS; ++i) f[i] = 0.f;
                auto add = [&](float weights) {   // of the 32 parts in x, one a lane; 0 past the last part
#pragma unroll
                    for (int i = 0; i < kJoin; ++i) {
                        const float weight = __shfl_sync(0xffffffffu, weights, i);
#pragma unroll
                        for (int j = 0; j < DIMS; ++j) f[j] = fmaf(weight, x[i][j], f[j]);
                    }
                };
                add(lse0);
                if (a.splits > kJoin) {
                    request(kJoin);
                    add(lse1);
                }
#pragma unroll
                for (int i = 0; i < DIMS; i += 2) {
                    const __nv_bfloat162 pair = __floats2bfloat162_rn(f[i], f[i + 1]);
                    *reinterpret_cast<__nv_bfloat162*>(out + lane * DIMS + i) = pair;
                }
                if (lane == 0) a.counters[w.bh] = 0;
            }
        }
        if (w.sp == 0 && w.bh == w.b * a.H && lane == 0) {
            if (w.n == 0) raise_status(a.dev_status, BT_DEV_EMPTY);
            if (w.overflow) raise_status(a.dev_status, BT_DEV_OVERFLOW);
        }
        settle();
        pend_arrival = seq_arrival;
        pend_b = w.b;
        pend_n = w.n;
        pend_overflow = w.overflow;
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

template <int HD, int UNITS, int STAGES, int MAX_WARPS>
static cudaError_t launch_t(const Kv4DecodeArgs& a, int dev, int sms, cudaStream_t stream)
{
    static PerDeviceOnce limit_raised;
    const cudaError_t e = raise_smem_limit_once(limit_raised, dev, block_decode_kv4_kernel<HD, UNITS, STAGES, MAX_WARPS>, smem_bytes<HD, UNITS>(MAX_WARPS, STAGES));
    if (e != cudaSuccess) return e;
    const long long items = (long long)a.B * a.H * a.splits;
    if (items > 0x7fffffffLL - 4096) return cudaErrorInvalidConfiguration;
    Params p;
    static_cast<Kv4DecodeArgs&>(p) = a;
    p.by_splits = divisor_of((uint32_t)a.splits);
    p.by_heads = divisor_of((uint32_t)a.H);
    const long long grid = items < sms ? items : sms;
    // Items are dealt whole: of the warp counts down to five eighths of the most, the one that leaves the fewest warps without an item in
    // the last round (4096 items on 148 SMs: 14 warps, 1.98 rounds of two; 16 warps 1.73).
    int warps = MAX_WARPS;
    double best = 0.0;
    for (int w = MAX_WARPS; w >= MAX_WARPS * 5 / 8; --w) {
        const long long slots = grid * w, rounds = (items + slots - 1) / slots;
        const double fill = (double)items / (double)(rounds * slots);
        if (fill > best + 1e-9) {
            best = fill;
            warps = w;
        }
    }
    const long long each = (items + grid - 1) / grid;
    if (each < warps) warps = (int)each;
    return launch_pdl(block_decode_kv4_kernel<HD, UNITS, STAGES, MAX_WARPS>, dim3((unsigned)grid), dim3(warps * 32), (size_t)smem_bytes<HD, UNITS>(warps, STAGES), stream, p);
}

}  // namespace kv4

cudaError_t launch_block_decode_kv4(const Kv4DecodeArgs& a, cudaStream_t stream)
{
    int dev = 0, sms = 0;
    const cudaError_t e = current_device(&dev, &sms);
    if (e != cudaSuccess) return e;
    if (a.hd == 128) return kv4::launch_t<128, 1, 2, 8>(a, dev, sms, stream);
    // Head_dim 64: with at most eight items an SM, a warp each and chunks of two units; with more, 16 warps an SM (126 registers a thread),
    // of which each spends half as long on an item's beginning and end.  us, 16 warps / eight:
    //   items of 48 to 64 rows:     1024: 3.4 / 3.5,  1536: 3.8 / 5.2,   4096: 7.2 / 9.4
    //   items of 384 to 512 rows:   1024: 9.4 / 8.3,  1536: 11.1 / 13.9, 4096: 23.9 / 26.4
    if ((long long)a.B * a.H * a.splits > 8LL * sms) return kv4::launch_t<64, 1, 2, 16>(a, dev, sms, stream);
    return kv4::launch_t<64, 2, 2, 8>(a, dev, sms, stream);
}

}  // namespace bt
