// bt_block_decode_attn_weights and bt_block_decode_step_weights: the streaming decode kernel with each row's
// attention weight added to a running sum.
//
// A row's weight 2^(s - lse) needs the whole item's maximum and sum, so its score s is kept until they are known: in
// shared memory while one warp sees all of a short cache (the sums are then updated by that warp, in the same
// launch), else in the workspace, and a second launch adds the weights - 12 bytes a row beside the 4 * head_dim that
// the attention reads.
#include "bt_decode_ring.cuh"

namespace bt {
namespace ring {

constexpr int kAddThreads = 256;
constexpr int kAddRows = kAddThreads * 4;   // rows of one CTA

__global__ void __launch_bounds__(kAddThreads) weights_add_kernel(WeightsDecodeArgs a, int pieces)
{
    pdl_launch_dependents();
    pdl_wait();
    const int bh = blockIdx.x / pieces, r0 = (blockIdx.x - bh * pieces) * kAddRows;
    const int4 info = a.info[bh];   // lse, rows, appended row or -1
    const float lse = __int_as_float(info.x);
    const int n = min(info.y, a.n_max);   // an item that gave up (BT_DEV_TIMEOUT) has left whatever the workspace held
    if (r0 >= n) return;
    const size_t base = (size_t)bh * a.n_max;
    const int r = r0 + (int)threadIdx.x * 4;
    if ((a.n_max & 3) == 0 && r + 3 < n && !(info.z >= r && info.z < r + 4)) {
        const float4 s = *reinterpret_cast<const float4*>(a.scores + base + r);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (a.w_in != nullptr) x = *reinterpret_cast<const float4*>(a.w_in + base + r);
        x.x += ex2(s.x - lse);
        x.y += ex2(s.y - lse);
        x.z += ex2(s.z - lse);
        x.w += ex2(s.w - lse);
        *reinterpret_cast<float4*>(a.w_out + base + r) = x;
    } else {
        for (int i = r; i < min(r + 4, n); ++i)
            a.w_out[base + i] = (a.w_in != nullptr && i != info.z ? a.w_in[base + i] : 0.f) + ex2(a.scores[base + i] - lse);
    }
}

}  // namespace ring

cudaError_t launch_block_decode_weights(const WeightsDecodeArgs& a, cudaStream_t stream)
{
    const cudaError_t e = a.hd == 64 ? ring::launch_t<64, ring::kWeights>(a, stream) : ring::launch_t<128, ring::kWeights>(a, stream);
    if (e != cudaSuccess || a.smem_rows) return e;
    const long long pieces = (a.n_max + ring::kAddRows - 1) / ring::kAddRows, grid = pieces * a.B * a.H;
    if (grid > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    return launch_pdl(ring::weights_add_kernel, dim3((unsigned)grid), dim3(ring::kAddThreads), 0, stream, a, (int)pieces);
}

}  // namespace bt
