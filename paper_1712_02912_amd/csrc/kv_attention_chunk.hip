// Launches of the attention of chunks (kv_attention_chunk.h), alone or together with that of few rows (kv_attention_few.h).
#include "kv_attention_chunk.h"

namespace pq {

// splits: parts of the keys; blocks of chunks come first, part after part, then those of few rows (the chunks' take longer)
template <class T, int D, int WAVES> __global__ __launch_bounds__(64 * WAVES, D > 128 ? 1 : 2) void kv_attention_chunk_kernel(attention_args a, chunk_split split) {
    __shared__ __attribute__((aligned(16))) unsigned char pool[CHUNK_POOL<D>];
    chunk_block<T, D, WAVES>(a, split, blockIdx.x, blockIdx.y, pool);
}
template <class T, int D> __global__ __launch_bounds__(64 * JOIN_ROWS) void kv_attention_chunk_join_kernel(attention_args a, chunk_split split) {
    chunk_join_block<T, D>(a, split, blockIdx.x);
}

// Both kinds of requests in one launch, so that neither waits for the other's last blocks: first the chunks' blocks, which take
// longer, part after part, then those of few rows.
template <class T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, D > 128 ? 1 : 2) void kv_attention_mixed_kernel(attention_args a, chunk_split split, int chunk_blocks, few_line line) {
    constexpr int POOL = CHUNK_POOL<D> > FEW_POOL<D, WAVES> ? CHUNK_POOL<D> : FEW_POOL<D, WAVES>;
    __shared__ __attribute__((aligned(16))) unsigned char pool[POOL];
    const int b = blockIdx.x;
    if (b < chunk_blocks * split.splits) chunk_block<T, D, WAVES>(a, split, b % chunk_blocks, b / chunk_blocks, pool);
    else few_block<T, D, WAVES>(a, line, b - chunk_blocks * split.splits, pool);
}
template <class T, int D>
__global__ __launch_bounds__(64 * JOIN_ROWS) void kv_attention_mixed_join_kernel(attention_args a, chunk_split split, int few_blocks, int slices, few_line line) {
    const int b = blockIdx.x;
    if (b < few_blocks) few_join_block<T, D, JOIN_ROWS>(a, line, b / slices, b % slices);
    else chunk_join_block<T, D>(a, split, b - few_blocks);
}

template <class T, int D, int WAVES> static int chunk_run(pq_ctx *ctx, const attention_args &a, bool some_few) {
    constexpr int M = 32 * WAVES;
    const int64_t indexes = a.ntokens * a.group / M + a.nreq, rows = a.ntokens * a.q_heads;
    // Fewer tiles of rows than twice the compute units: the keys of each are split, down to 512 keys a part.
    const int64_t full = (a.ntokens * a.group + M - 1) / M, tiles = (full > a.nreq ? full : a.nreq) * a.cache.heads;
    int64_t splits = 2 * ctx->num_cu / tiles, most = ((int64_t)a.width * a.cache.block_size + 511) / 512;
    if (a.window > 0 && most > (a.window + 511) / 512) most = (a.window + 511) / 512;
    if (splits > most) splits = most;
    chunk_split split = {splits < 1 ? 1 : (int)splits, some_few, nullptr, nullptr};
    const int64_t chunk_blocks = indexes * a.cache.heads;
    if (chunk_blocks * split.splits > INT_MAX - (1 << 20) || rows > INT_MAX) return fail(ctx, PQ_EUNSUPPORTED, "kv_attention: %lld rows in one call", (long long)rows);
    const size_t slots = split.splits > 1 ? (size_t)rows * split.splits : 0, ws = slots * (D + 2) * sizeof(float);
    size_t ws_at = 0;
    few_line line = {};
    if (some_few) {
        if (const int rc = few_prepare(ctx, a, WAVES, ws, &line, &ws_at)) return rc;
        if (line.row_waves > JOIN_ROWS) line.row_waves = JOIN_ROWS;
    } else if (ws > 0) {
        if (const int rc = buf_reserve(ctx, &ctx->read_ws, ws, "parts of the attention")) return rc;
    }
    if (split.splits > 1) {
        split.parts = (float *)((char *)ctx->read_ws.p + ws_at);
        split.stats = split.parts + slots * D;
    }
    const int joins = split.splits > 1 ? (int)((rows + JOIN_ROWS - 1) / JOIN_ROWS) : 0;
    if (some_few) {
        const int64_t all = chunk_blocks * split.splits + line.blocks;
        kv_attention_mixed_kernel<T, D, WAVES><<<(unsigned)all, 64 * WAVES, 0, ctx->stream>>>(a, split, (int)chunk_blocks, line);
        const int slices = few_slices(line, FEW_ROWS, JOIN_ROWS);
        const int64_t few_blocks = (int64_t)a.nreq * a.cache.heads * slices;
        if (few_blocks + joins > INT_MAX) return fail(ctx, PQ_EUNSUPPORTED, "kv_attention: %d requests in one call", a.nreq);
        kv_attention_mixed_join_kernel<T, D><<<(unsigned)(few_blocks + joins), 64 * JOIN_ROWS, 0, ctx->stream>>>(a, split, (int)few_blocks, slices, line);
    } else {
        kv_attention_chunk_kernel<T, D, WAVES><<<dim3((unsigned)chunk_blocks, split.splits), 64 * WAVES, 0, ctx->stream>>>(a, split);
        if (joins > 0) kv_attention_chunk_join_kernel<T, D><<<joins, 64 * JOIN_ROWS, 0, ctx->stream>>>(a, split);
    }
    PQ_HIP(ctx, hipGetLastError());
    return PQ_OK;
}

template <class T> static int chunk_dim(pq_ctx *ctx, const attention_args &a, bool some_few) {
    const bool many = a.ntokens * a.group >= (int64_t)a.nreq * 192;
    switch (a.cache.dim) {
    case 64: return many ? chunk_run<T, 64, 8>(ctx, a, some_few) : chunk_run<T, 64, 4>(ctx, a, some_few);
    case 96: return many ? chunk_run<T, 96, 8>(ctx, a, some_few) : chunk_run<T, 96, 4>(ctx, a, some_few);
    case 128: return many ? chunk_run<T, 128, 8>(ctx, a, some_few) : chunk_run<T, 128, 4>(ctx, a, some_few);
    default: return chunk_run<T, 256, 4>(ctx, a, some_few);
    }
}

int launch_kv_attention_chunk(pq_ctx *ctx, const attention_args &a, bool some_few) {
    return a.cache.elem == PQ_ELEM_F16 ? chunk_dim<_Float16>(ctx, a, some_few) : chunk_dim<__bf16>(ctx, a, some_few);
}

}  // namespace pq
