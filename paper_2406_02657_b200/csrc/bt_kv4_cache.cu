// Writing rows into the 4-bit block cache and reading them back (the cache of the block decoder, paper section 2.3, in a quarter
// of the bytes).  Both are bound by memory: 4 hd bytes of bf16 and 1.125 hd bytes of codes and steps a row.
//
// One warp takes a tile (16 rows x 64 dimensions of K and V).  Eight lanes hold a row's 64 dimensions, 16 bytes each, and a group
// of eight lanes takes four consecutive rows, so that a lane group ends up with the steps of four rows and a lane with a unit of V codes,
// and writes either in one 16-byte store; the eight loads (K and V of four rows) are all in flight before the first is used.
#include "bt_device.h"
#include "bt_kernels.h"
#include "bt_kv4.cuh"

namespace bt {
namespace kv4 {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kFusedWarps = 16;   // at most: a warp for every tile of a sequence

struct Params : Kv4Args {
    int tiles, planes, items;   // tiles of a slab that the call may touch; all the call's
    Divisor by_tiles, by_planes, by_heads;
};
// where item (slab, tile, plane) of a call lies; items count planes fastest
struct Item {
    int slab, tile, plane;
};
__device__ __forceinline__ Item item_at(int i, const Params& a)
{
    Item it;
    const int t = divide(i, a.by_planes);
    it.plane = i - t * a.planes;
    it.slab = divide(t, a.by_tiles);
    it.tile = t - it.slab * a.tiles;
    return it;
}

// Rows start .. start + n_rows - 1 of a slab, as far as they lie in its `tile`-th tile from start's on.
__device__ __forceinline__ void write_tile(const Params& a, const Item& it, int start, int lane)
{
    const int tile = start / kTileRows + it.tile;
    const int first = tile * kTileRows, end = start + a.n_rows;
    if (first >= end) return;
    const int g = lane >> 3, sub = lane & 7;
    const size_t src0 = ((size_t)it.slab * a.stride) * a.hd + it.plane * 64 + sub * 8;
    uint4 k[4], v[4];
    bool there[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = first + g * 4 + i;
        there[i] = r >= start && r < end;
        k[i] = v[i] = make_uint4(0, 0, 0, 0);
        if (there[i]) {
            const size_t src = src0 + (size_t)(r - start) * a.hd;
            k[i] = ld_stream(reinterpret_cast<const bf16*>(a.k) + src);
            v[i] = ld_stream(reinterpret_cast<const bf16*>(a.v) + src);
        }
    }
    uint8_t* dst = reinterpret_cast<uint8_t*>(a.kv) + (size_t)it.slab * a.slab_bytes + ((size_t)tile * a.planes + it.plane) * kTileBytes;
    const bool all = there[0] && there[3];
    // Largest magnitudes, K's and V's of a row in one word, over the four lanes of a group, so that lane j of them ends up with row j's:
    // it works out both steps of that row.
    uint32_t m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t mk = magnitude_max8(k[i]), mv = magnitude_max8(v[i]);
        m[i] = magnitude_max(__byte_perm(mk, mv, 0x5410), __byte_perm(mk, mv, 0x7632));
    }
    const bool up2 = (lane & 2) != 0, up1 = (lane & 1) != 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) m[i] = magnitude_max(up2 ? m[i + 2] : m[i], __shfl_xor_sync(0xffffffffu, up2 ? m[i] : m[i + 2], 2));
    m[0] = magnitude_max(up1 ? m[1] : m[0], __shfl_xor_sync(0xffffffffu, up1 ? m[0] : m[1], 1)) & 0x7fff7fffu;
    const Step sk = step_of_group<7>(m[0] & 0xffffu), sv = step_of_group<7>(m[0] >> 16);
    {
        const int r = first + g * 4 + (lane & 3);
        if (r >= start && r < end) {
            uint16_t* at = reinterpret_cast<uint16_t*>(dst + kStepsAt) + (g * 4 + (lane & 3)) * 2 + (sub >> 2);
            at[0] = (uint16_t)sk.bits;
            at[32] = (uint16_t)sv.bits;
        }
    }
    uint32_t ck[4], cv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        ck[i] = codes8(k[i], __shfl_sync(0xffffffffu, sk.inv, (lane & 28) + i));
        cv[i] = codes8(v[i], __shfl_sync(0xffffffffu, sv.inv, (lane & 28) + i));
    }
    // groups that are not finite: the warp looks for them together, hardly ever finds one
    const uint32_t bad_k = __ballot_sync(0xffffffffu, !sk.finite), bad_v = __ballot_sync(0xffffffffu, !sv.finite);
    if (bad_k | bad_v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (bad_k >> ((lane & 28) + i) & 1u) ck[i] = kZeroCodes;
            if (bad_v >> ((lane & 28) + i) & 1u) cv[i] = kZeroCodes;
        }
    }
    // a 16-byte unit of K is two rows' codes of two neighbouring lanes: the even lane takes the first two rows, the odd one the others
    const uint32_t x = __shfl_xor_sync(0xffffffffu, up1 ? ck[0] : ck[2], 1), y = __shfl_xor_sync(0xffffffffu, up1 ? ck[1] : ck[3], 1);
    if (all) {
        const uint4 unit = up1 ? make_uint4(x, ck[2], y, ck[3]) : make_uint4(ck[0], x, ck[1], y);
        *reinterpret_cast<uint4*>(dst + k_codes_at(g * 4 + (up1 ? 2 : 0), sub & 6)) = unit;
        *reinterpret_cast<uint4*>(dst + v_unit_at(g, sub)) = transpose4x4(make_uint4(cv[0], cv[1], cv[2], cv[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (there[i]) {
                *reinterpret_cast<uint32_t*>(dst + k_codes_at(g * 4 + i, sub)) = ck[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) dst[v_codes_at(g * 4 + i, sub) + 4 * j] = (uint8_t)(cv[i] >> (8 * j));
            }
    }
}

// FUSED: CTA = sequence, which raises its own length; else any warp takes any tile, and the length is raised by a launch behind
// this one - or by this one, when the rows start anew and no warp looks at the old length.
template <bool FUSED>
__global__ void __launch_bounds__(FUSED ? kFusedWarps * 32 : kThreads) kv4_append_kernel(const __grid_constant__ Params a)
{
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    if constexpr (FUSED) {   // items: those of one sequence, one for each warp
        const int b = blockIdx.x;
        const int start = a.len[b];
        const bool ok = start >= 0 && start <= a.cap - a.n_rows;
        __syncthreads();
        if (ok) {
            Item it = item_at(warp, a);
            it.slab += b * a.H;
            write_tile(a, it, start, lane);
        }
        if (threadIdx.x == 0) {
            if (ok) a.len[b] = start + a.n_rows;
            else raise_status(a.dev_status, BT_DEV_OVERFLOW);
        }
    } else {
        const int i = (int)blockIdx.x * kWarps + warp;
        if (i >= a.items) return;
        const Item it = item_at(i, a);
        const int b = divide(it.slab, a.by_heads);
        const int start = a.reset ? 0 : a.len[b];
        if (start < 0 || start > a.cap - a.n_rows) return;   // flagged by the launch that raises the lengths
        write_tile(a, it, start, lane);
        if (a.reset && it.slab == b * a.H && it.tile == 0 && it.plane == 0 && lane == 0) a.len[b] = a.n_rows;
    }
}

__global__ void kv4_len_kernel(int32_t* len, int B, int n, int cap, uint32_t* dev_status)
{
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= B) return;
    const int l = len[b];
    if (l >= 0 && l <= cap - n) len[b] = l + n;
    else raise_status(dev_status, BT_DEV_OVERFLOW);
}

__global__ void __launch_bounds__(kThreads) kv4_read_kernel(const __grid_constant__ Params a)
{
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, i = (int)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const Item it = item_at(i, a);
    pdl_wait();
    if (i >= a.items) return;
    const int len = a.len[divide(it.slab, a.by_heads)];
    const int end = min(min(len, a.cap), a.first + a.n_rows);
    const int tile = a.first / kTileRows + it.tile, row0 = tile * kTileRows;
    if (row0 >= end) return;
    const int g = lane >> 3, sub = lane & 7;
    const uint8_t* src = reinterpret_cast<const uint8_t*>(a.kv) + (size_t)it.slab * a.slab_bytes + ((size_t)tile * a.planes + it.plane) * kTileBytes;
    uint32_t codes[2][4], steps[2][4];
    // a 16-byte unit of K is two rows' codes of two neighbouring lanes: the even lane reads the first two rows, the odd one the others
    const bool odd = (lane & 1) != 0;
    const uint4 two = *reinterpret_cast<const uint4*>(src + k_codes_at(g * 4 + (odd ? 2 : 0), sub & 6));
    const uint32_t x = __shfl_xor_sync(0xffffffffu, odd ? two.x : two.y, 1), y = __shfl_xor_sync(0xffffffffu, odd ? two.z : two.w, 1);
    codes[0][0] = odd ? x : two.x;
    codes[0][1] = odd ? y : two.z;
    codes[0][2] = odd ? two.y : x;
    codes[0][3] = odd ? two.w : y;
    const uint4 unit = transpose4x4(*reinterpret_cast<const uint4*>(src + v_unit_at(g, sub)));
    codes[1][0] = unit.x;
    codes[1][1] = unit.y;
    codes[1][2] = unit.z;
    codes[1][3] = unit.w;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        const uint4 four = *reinterpret_cast<const uint4*>(src + kStepsAt + part * 64 + g * 16);
        steps[part][0] = four.x;
        steps[part][1] = four.y;
        steps[part][2] = four.z;
        steps[part][3] = four.w;
    }
    const size_t dst0 = ((size_t)it.slab * a.stride) * a.hd + it.plane * 64 + sub * 8;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        bf16* out = reinterpret_cast<bf16*>(part == 0 ? a.k : a.v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = row0 + g * 4 + j;
            if (r < a.first || r >= end) continue;
            *reinterpret_cast<uint4*>(out + dst0 + (size_t)(r - a.first) * a.hd) =
                values8(codes[part][j], sub < 4 ? steps[part][j] & 0xffffu : steps[part][j] >> 16);
        }
    }
}

// false: more items than 31 bits count (no device holds such a cache)
static bool fill(Params& p, const Kv4Args& a, long long tiles, long long slabs)
{
    static_cast<Kv4Args&>(p) = a;
    p.planes = a.hd / 64;
    const long long items = slabs * tiles * p.planes;
    if (items > 0x7fffffffLL - kThreads) return false;
    p.tiles = (int)tiles;
    p.items = (int)items;
    p.by_tiles = divisor_of((uint32_t)tiles);
    p.by_planes = divisor_of((uint32_t)p.planes);
    p.by_heads = divisor_of((uint32_t)a.H);
    return true;
}
static dim3 grid_of(const Params& p) { return dim3((unsigned)((p.items + kWarps - 1) / kWarps)); }

}  // namespace kv4

cudaError_t launch_kv4_append(const Kv4Args& a, cudaStream_t stream)
{
    // rows that start inside a tile may reach into one more
    const long long tiles = ((long long)a.n_rows + (a.reset ? 1 : 2) * (kv4::kTileRows - 1)) / kv4::kTileRows;
    const long long each = a.H * tiles * (a.hd / 64);   // items of a sequence
    // One launch where a CTA has a warp for every item of a sequence.  us, one launch / two:
    //   one item a warp, a row of 16 heads of 64:     32 sequences: 2.8 / 3.1,   256: 4.1 / 4.9
    //   two items a warp, a row of 16 heads of 128:   32 sequences: 4.4 / 3.1,   256: 6.8 / 7.1;   16 rows of 16 heads of 64, 64 sequences: 5.1 / 3.7
    // (Eight CTAs, a cluster, a sequence: 6.5 us over 13 x 7 x 487 rows of 64, two launches 4.4.)
    const bool fused = !a.reset && each <= kv4::kFusedWarps;
    kv4::Params p;
    if (!kv4::fill(p, a, tiles, fused ? a.H : (long long)a.B * a.H)) return cudaErrorInvalidConfiguration;
    if (fused) return launch_pdl(kv4::kv4_append_kernel<true>, dim3(a.B), dim3((unsigned)each * 32), 0, stream, p);
    const cudaError_t e = launch_pdl(kv4::kv4_append_kernel<false>, kv4::grid_of(p), dim3(kv4::kThreads), 0, stream, p);
    if (e != cudaSuccess || a.reset) return e;
    return launch_pdl(kv4::kv4_len_kernel, dim3((a.B + 255) / 256), dim3(256), 0, stream, a.len, a.B, a.n_rows, a.cap, a.dev_status);
}

cudaError_t launch_kv4_read(const Kv4Args& a, cudaStream_t stream)
{
    kv4::Params p;
    if (!kv4::fill(p, a, (a.first + a.n_rows - 1) / kv4::kTileRows - a.first / kv4::kTileRows + 1, (long long)a.B * a.H)) return cudaErrorInvalidConfiguration;
    return launch_pdl(kv4::kv4_read_kernel, kv4::grid_of(p), dim3(kv4::kThreads), 0, stream, p);
}

}  // namespace bt
