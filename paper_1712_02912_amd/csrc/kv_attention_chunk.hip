// Launches of the attention of chunks (kv_attention_chunk.h), alone or together with that of few rows (kv_attention_few.h).
#include "kv_attention_chunk.h"

namespace pq {

// Waves of a SIMD that registers are to be left for.  (Left alone, blocks of four waves over 64 dimensions come to 168 to 171
// registers; three waves have 168: 40 us for 23 requests of 1 to 517 tokens with windows of 1024 keys, 44 us with two waves.)
template <int D, int WAVES> constexpr int CHUNK_RESIDENT = D > 128 ? 1 : D == 64 && WAVES == 4 ? 3 : 2;

template <class T, int D, int WAVES> __global__ __launch_bounds__(64 * WAVES, (CHUNK_RESIDENT<D, WAVES>)) void kv_attention_chunk_kernel(attention_args a, chunk_split split) {
    __shared__ __attribute__((aligned(16))) unsigned char pool[CHUNK_POOL<D>];
    chunk_block<T, D, WAVES>(a, split, blockIdx.x, blockIdx.y, pool);
}
template <class T, int D> __global__ __launch_bounds__(64 * JOIN_ROWS) void kv_attention_chunk_join_kernel(attention_args a, chunk_split split) {
    chunk_join_block<T, D>(a, split, blockIdx.x);
}

// Both kinds of requests in one launch, so that neither waits for the other's last blocks: first the chunks' blocks, which take
// longer, part after part, then those of few rows.
template <class T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, (CHUNK_RESIDENT<D, WAVES>)) void kv_attention_mixed_kernel(attention_args a, chunk_split split, int chunk_blocks, few_line line) {
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
    // Tiles of rows that leave compute units without work: the keys of each are split, down to 256 keys a part, into one round of
    // the blocks that the chip holds.  Of blocks of eight waves over 96 and 128 dimensions two rounds are better, which end more
    // evenly (512 rows of 8 heads over 30 512 keys of 128 dimensions: 121 us, 131 us in one round), of 64 they cost more in parts
    // than that (700 rows of 8 heads over 9700 keys: 42 us, in one round 34 us).  Parts of 512 keys at least: 31 us for 4 requests of
    // 1 to 20 tokens over windows of 305 keys, 256 dimensions, 21 us with 256; in two rounds 45 us for 4 requests of 1 to 264 tokens
    // over windows of 1388 keys, 50 us with 256.
    const int64_t tiles = ((a.ntokens * a.group + M - 1) / M + a.nreq / 2) * a.cache.heads;
    constexpr bool two_rounds = D > 64 && D <= 128 && WAVES == 8;
    constexpr int waves = D > 128 ? 4 : two_rounds ? 16 : 8, least = two_rounds ? 512 : 256;
    const int64_t keys = (int64_t)a.width * a.cache.block_size, seen = a.window > 0 && a.window < keys ? a.window : keys;
    const int64_t most = (seen + least - 1) / least;
    int64_t splits = ctx->num_cu * waves / WAVES / (tiles > 0 ? tiles : 1);
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
    // Eight waves share each tile of keys where requests have rows for them.  12 requests of 1 to 300 tokens, 7 heads on each of 4,
    // 128 dimensions: 90 us with eight, 82 with four; 8 requests of 200 tokens, 8 heads on each of 8: 164 and 185 us; two chunks of
    // 2048, 4 heads on each of 8: 707 and 794 us.
    const bool many = a.ntokens * a.group >= (int64_t)a.nreq * 512;
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
