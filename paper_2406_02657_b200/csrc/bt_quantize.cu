// Rows quantised to 8 bits, a step for each (the activations of a token, the weights of an output channel):
//   s = bf16(max|x| / 127) as fp32,  x8 = round(x / s), halves away from zero.
// A step of 8 significant bits costs nothing (max|x| / s stays below 127.5, the codes' range) and makes every rounding the one of
// the exact quotient (see bt_kv4.cuh).  A step below 2^-126 is 0 and its codes are zeros; a row with a value that is not finite has
// the step NaN and codes of zero, so that whatever is computed from it is NaN.
//
// Bound by memory: 3 bytes a value.  One warp takes a row and keeps it in registers between the maximum and the rounding.
#include "bt_device.h"
#include "bt_kernels.h"
#include "bt_kv4.cuh"

namespace bt {
namespace quant {

// 8 values -> 8 codes of eight bits
__device__ __forceinline__ uint2 bytes8(const uint4& r, float inv)
{
    constexpr float kWhole = 12582912.0f;   // 1.5 * 2^23: the low byte of the sum is the whole number nearest
    float f[8];
    unpack8(r, f);
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(fmaf(f[i], inv, kWhole));
    uint2 w;
    w.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    w.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
    return w;
}

// PIECES 8-value pieces a lane: rows of up to 256 * PIECES values; WARPS rows a CTA
template <int PIECES, int WARPS>
__global__ void __launch_bounds__(WARPS * 32) rows_quantize_kernel(const bf16* __restrict__ x, long long rows, int cols, int8_t* __restrict__ x8,
                                                                 float* __restrict__ steps)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
    if (row >= rows) return;
    x += row * cols;
    x8 += row * cols;
    const int pieces = cols / 8;
    uint4 r[PIECES];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int at = lane + 32 * i;
        r[i] = at < pieces ? ld_stream(x + at * 8) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) m = kv4::magnitude_max(m, kv4::magnitude_max8(r[i]));
    m = __reduce_max_sync(0xffffffffu, kv4::magnitude_of(m));
    const kv4::Step st = kv4::step_of_group<127>(m);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int at = lane + 32 * i;
        if (at < pieces) *reinterpret_cast<uint2*>(x8 + at * 8) = st.finite ? bytes8(r[i], st.inv) : make_uint2(0, 0);
    }
    if (lane == 0) steps[row] = __uint_as_float(st.bits << 16);
}

template <int PIECES, int WARPS>
static cudaError_t launch_p(const void* x, long long rows, int cols, void* x8, float* steps, cudaStream_t stream)
{
    const long long ctas = (rows + WARPS - 1) / WARPS;
    if (ctas > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    return launch_pdl(rows_quantize_kernel<PIECES, WARPS>, dim3((unsigned)ctas), dim3(WARPS * 32), 0, stream, reinterpret_cast<const bf16*>(x), rows, cols,
                      reinterpret_cast<int8_t*>(x8), steps);
}

}  // namespace quant

cudaError_t launch_rows_quantize(const void* x, long long rows, int cols, void* x8, float* steps, cudaStream_t stream)
{
    // 16 rows a CTA where rows are long (16384 x 2048: 16.8 us, with 8 19.5; floor 15.3), 8 where they are short (4096 x 1024: 2.9 us, with 16 3.2)
    if (cols <= 512) return quant::launch_p<2, 8>(x, rows, cols, x8, steps, stream);
    if (cols <= 1024) return quant::launch_p<4, 8>(x, rows, cols, x8, steps, stream);
    return quant::launch_p<8, 16>(x, rows, cols, x8, steps, stream);
}

}  // namespace bt
