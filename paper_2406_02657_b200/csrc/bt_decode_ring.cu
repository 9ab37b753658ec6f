// bt_block_decode_attn and bt_block_decode_step: the streaming decode kernel over every cached row.
#include "bt_decode_ring.cuh"

namespace bt {

cudaError_t launch_block_decode(const DecodeArgs& a, cudaStream_t stream)
{
    return a.hd == 64 ? ring::launch_t<64, ring::kPlain>(a, stream) : ring::launch_t<128, ring::kPlain>(a, stream);
}

}  // namespace bt
