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

// where item (slab, tile, plane) of a call lies; items count planes fastest
struct Item {
    int slab, tile, plane;
};
__device__ __forceinline__ Item item_at(long long i, int tiles, int planes)
{
    Item it;
    const long long t = i / planes;
    it.plane = (int)(i - t * planes);
    it.slab = (int)(t / tiles);
    it.tile = (int)(t - (long long)it.slab * tiles);
    return it;
}

// Rows start .. start + n_rows - 1 of a slab, as far as they lie in its `tile`-th tile from start's on.
__device__ __forceinline__ void write_tile(const Kv4Args& a, const Item& it, int start, int lane)
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
    uint8_t* dst = reinterpret_cast<uint8_t*>(a.kv) + (size_t)it.slab * a.slab_bytes + (size_t)(tile * (a.hd / 64) + it.plane) * kTileBytes;
    const bool all = there[0] && there[3];
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        uint32_t steps[4], codes[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4& x = part == 0 ? k[i] : v[i];
            const Step st = step_of_lanes(x);
            codes[i] = codes8(x, st);
            steps[i] = st.bits | __shfl_down_sync(0xffffffffu, st.bits, 4) << 16;   // both groups' (lanes 0 of eight)
        }
        if (part == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (there[i]) *reinterpret_cast<uint32_t*>(dst + k_codes_at(g * 4 + i, sub)) = codes[i];
        } else if (all) {
            *reinterpret_cast<uint4*>(dst + v_unit_at(g, sub)) = transpose4x4(make_uint4(codes[0], codes[1], codes[2], codes[3]));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (there[i])
#pragma unroll
                    for (int j = 0; j < 4; ++j) dst[v_codes_at(g * 4 + i, sub) + 4 * j] = (uint8_t)(codes[i] >> (8 * j));
        }
        if (sub == 0) {
            uint32_t* at = reinterpret_cast<uint32_t*>(dst + kStepsAt + part * 64) + g * 4;
            if (all) {
                *reinterpret_cast<uint4*>(at) = make_uint4(steps[0], steps[1], steps[2], steps[3]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (there[i]) at[i] = steps[i];
            }
        }
    }
}

// FUSED: CTA = sequence, which raises its own length; else any warp takes any tile, and the length is raised by a launch behind
// this one - or by this one, when the rows start anew and no warp looks at the old length.
template <bool FUSED>
__global__ void __launch_bounds__(kThreads) kv4_append_kernel(Kv4Args a, int tiles)
{
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, planes = a.hd / 64;
    pdl_wait();
    if constexpr (FUSED) {
        const int b = blockIdx.x;
        const int start = a.len[b];
        const bool ok = start >= 0 && start <= a.cap - a.n_rows;
        __syncthreads();
        const int items = a.H * tiles * planes;
        if (ok)
            for (int i = warp; i < items; i += kWarps) {
                Item it = item_at(i, tiles, planes);
                it.slab += b * a.H;
                write_tile(a, it, start, lane);
            }
        if (threadIdx.x == 0) {
            if (ok) a.len[b] = start + a.n_rows;
            else raise_status(a.dev_status, BT_DEV_OVERFLOW);
        }
    } else {
        const long long i = (long long)blockIdx.x * kWarps + warp;
        if (i >= (long long)a.B * a.H * tiles * planes) return;
        const Item it = item_at(i, tiles, planes);
        const int b = it.slab / a.H;
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

__global__ void __launch_bounds__(kThreads) kv4_read_kernel(Kv4Args a, int tiles)
{
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, planes = a.hd / 64;
    const long long i = (long long)blockIdx.x * kWarps + warp;
    pdl_wait();
    if (i >= (long long)a.B * a.H * tiles * planes) return;
    const Item it = item_at(i, tiles, planes);
    const int len = a.len[it.slab / a.H];
    const int end = min(min(len, a.cap), a.first + a.n_rows);
    const int tile = a.first / kTileRows + it.tile, row0 = tile * kTileRows;
    if (row0 >= end) return;
    const int g = lane >> 3, sub = lane & 7;
    const uint8_t* src = reinterpret_cast<const uint8_t*>(a.kv) + (size_t)it.slab * a.slab_bytes + (size_t)(tile * planes + it.plane) * kTileBytes;
    uint32_t codes[2][4], steps[2][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) codes[0][j] = *reinterpret_cast<const uint32_t*>(src + k_codes_at(g * 4 + j, sub));
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
            float f[8];
            values8(codes[part][j], sub < 4 ? bf_lo(steps[part][j]) : bf_hi(steps[part][j]), f);
            *reinterpret_cast<uint4*>(out + dst0 + (size_t)(r - a.first) * a.hd) = pack8(f);
        }
    }
}

}  // namespace kv4

cudaError_t launch_kv4_append(const Kv4Args& a, cudaStream_t stream)
{
    const int planes = a.hd / 64;
    // rows that start inside a tile may reach into one more
    const int tiles = (int)(((long long)a.n_rows + (a.reset ? 1 : 2) * (kv4::kTileRows - 1)) / kv4::kTileRows);
    const long long per_sequence = (long long)a.H * tiles * planes, items = per_sequence * a.B;
    if (!a.reset && per_sequence <= 8 * kv4::kWarps)
        return launch_pdl(kv4::kv4_append_kernel<true>, dim3(a.B), dim3(kv4::kThreads), 0, stream, a, tiles);
    const long long ctas = (items + kv4::kWarps - 1) / kv4::kWarps;
    if (ctas > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    const cudaError_t e = launch_pdl(kv4::kv4_append_kernel<false>, dim3((unsigned)ctas), dim3(kv4::kThreads), 0, stream, a, tiles);
    if (e != cudaSuccess || a.reset) return e;
    return launch_pdl(kv4::kv4_len_kernel, dim3((a.B + 255) / 256), dim3(256), 0, stream, a.len, a.B, a.n_rows, a.cap, a.dev_status);
}

cudaError_t launch_kv4_read(const Kv4Args& a, cudaStream_t stream)
{
    const int tiles = (a.first + a.n_rows - 1) / kv4::kTileRows - a.first / kv4::kTileRows + 1;
    const long long items = (long long)a.B * a.H * tiles * (a.hd / 64), ctas = (items + kv4::kWarps - 1) / kv4::kWarps;
    if (ctas > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    return launch_pdl(kv4::kv4_read_kernel, dim3((unsigned)ctas), dim3(kv4::kThreads), 0, stream, a, tiles);
}

}  // namespace bt
