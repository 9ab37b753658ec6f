// bt_block_decode_attn_window and bt_block_decode_step_window: the streaming decode kernel over the first `sinks`
// and the last `window` rows of each sequence.
#include "bt_decode_ring.cuh"

namespace bt {

cudaError_t launch_block_decode_window(const WindowDecodeArgs& a, cudaStream_t stream)
{
    return a.hd == 64 ? ring::launch_t<64, ring::kWindow>(a, stream) : ring::launch_t<128, ring::kWindow>(a, stream);
}

}  // namespace bt
