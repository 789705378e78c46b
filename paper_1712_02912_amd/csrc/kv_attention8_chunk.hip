// Attention of chunks over a cache of 8 bits.
#include "kv_attention_chunk_launch.h"

namespace pq {

int launch_kv_attention8_chunk(pq_ctx *ctx, const attention_args &a, bool some_few) {
    return a.cache.elem == PQ_ELEM_F16 ? chunk_dim<_Float16, e4m3>(ctx, a, some_few) : chunk_dim<__bf16, e4m3>(ctx, a, some_few);
}

}  // namespace pq
