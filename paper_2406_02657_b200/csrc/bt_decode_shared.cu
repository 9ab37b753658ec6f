// bt_block_decode_attn_shared and bt_block_decode_step_shared: the streaming decode kernel over each sequence's own
// rows, joined with the partial results over the shared prefix.
#include "bt_decode_ring.cuh"

namespace bt {

cudaError_t launch_block_decode_shared(const SharedDecodeArgs& a, cudaStream_t stream)
{
    return a.hd == 64 ? ring::launch_t<64, ring::kShared>(a, stream) : ring::launch_t<128, ring::kShared>(a, stream);
}

}  // namespace bt
