// Launches of the attention of few rows per head (kv_attention_few.h).
#include <algorithm>

#include "kv_attention_few.h"

namespace pq {

template <class T, class C, int D> __global__ __launch_bounds__(256, D > 128 ? 1 : 2) void kv_attention_few_kernel(attention_args a, few_line line) {
    __shared__ __attribute__((aligned(16))) unsigned char pool[FEW_POOL<D, 4>];
    few_block<T, C, D, 4>(a, line, blockIdx.x, pool);
}
template <class T, class C, int D, int WAVES> __global__ __launch_bounds__(64 * WAVES) void kv_attention_few_join_kernel(attention_args a, few_line line) {
    few_join_block<T, C, D, WAVES>(a, line, blockIdx.x, blockIdx.y);
}
__global__ __launch_bounds__(1024) void kv_attention_starts_kernel(attention_args a, int unit, int64_t *starts) { few_starts<1024>(a, unit, starts); }

int few_prepare(pq_ctx *ctx, const attention_args &a, int waves, size_t more, few_line *line, size_t *ws_used) {
    const int dim = a.cache.dim, per_cu = (dim > 128 ? 4 : 8) / waves;
    *line = {};
    line->unit = waves * FEW_TILE;
    line->blocks = ctx->num_cu * per_cu;
    // Short tables: a block for each (request, head), without a line and parts to join.  A unit takes a block about 1.3 us (2.6 us of
    // 256 dimensions), the line's sums and its second launch about 6 us.  4 requests of 41 keys, 8 heads: 5.7 us, 9.7 us by the
    // line; with 874 keys (7 units) of 12 requests, 8 heads, it is 22.9 and 17.2 us.  Where there are as many (request, head) as
    // the line has blocks, blocks wait less for each other: 96 requests of 1001 keys, 8 heads: 55 and 59 us, of 2001 keys 96 and
    // 89 us.
    const int64_t held = (int64_t)a.width * a.cache.block_size, seen = a.window > 0 ? std::min(held, (int64_t)a.window + FEW_ROWS) : held;
    const bool many = (int64_t)a.nreq * a.cache.heads >= line->blocks;
    const int64_t most = (many ? 1024 : 512) / (dim > 128 ? 4 : 1);
    if (seen <= most) {
        line->each = true;
        line->blocks = a.nreq * a.cache.heads;
        *ws_used = 0;
        return PQ_OK;
    }
    const size_t starts = align_up(((size_t)a.nreq + 1) * sizeof(int64_t), 256), slots = (size_t)line->blocks * 2 * FEW_ROWS;
    *ws_used = align_up(starts + slots * (dim + 2) * sizeof(float), 256);
    if (const int rc = buf_reserve(ctx, &ctx->read_ws, *ws_used + more, "parts of the attention")) return rc;
    line->starts_out = (int64_t *)ctx->read_ws.p;
    line->parts = (float *)((char *)ctx->read_ws.p + starts);
    line->stats = line->parts + slots * dim;
    if (a.nreq > FEW_MAX) {
        kv_attention_starts_kernel<<<1, 1024, 0, ctx->stream>>>(a, line->unit, line->starts_out);
        line->starts = line->starts_out;
    }
    // a wave for every fourth part of a row, about (2 requests of up to 30 000 keys, 2 heads of 64 dimensions: 19 us, with four waves
    // 22 us)
    const int64_t parts = line->blocks / ((int64_t)a.nreq * a.cache.heads);
    line->row_waves = parts >= 32 ? 16 : parts >= 4 ? 4 : 1;
    return PQ_OK;
}

template <class T, class C, int D> static int few_typed(pq_ctx *ctx, const attention_args &a, int most_rows) {
    const int64_t items = (int64_t)a.nreq * a.cache.heads;
    if (!grid_fits(items, 256)) return fail(ctx, PQ_EUNSUPPORTED, "kv_attention: %d requests in one call", a.nreq);
    few_line line;
    size_t ws_used;
    if (const int rc = few_prepare(ctx, a, 4, 0, &line, &ws_used)) return rc;
    kv_attention_few_kernel<T, C, D><<<line.blocks, 256, 0, ctx->stream>>>(a, line);
    if (line.each) {
        PQ_HIP(ctx, hipGetLastError());
        return PQ_OK;
    }
    if (line.row_waves > 4) kv_attention_few_join_kernel<T, C, D, 16><<<dim3((unsigned)items, few_slices(line, most_rows, 16)), 1024, 0, ctx->stream>>>(a, line);
    else kv_attention_few_join_kernel<T, C, D, 4><<<dim3((unsigned)items, few_slices(line, most_rows, 4)), 256, 0, ctx->stream>>>(a, line);
    PQ_HIP(ctx, hipGetLastError());
    return PQ_OK;
}

template <class T, class C> static int few_dim(pq_ctx *ctx, const attention_args &a, int most_rows) {
    switch (a.cache.dim) {
    case 64: return few_typed<T, C, 64>(ctx, a, most_rows);
    case 96: return few_typed<T, C, 96>(ctx, a, most_rows);
    case 128: return few_typed<T, C, 128>(ctx, a, most_rows);
    default: return few_typed<T, C, 256>(ctx, a, most_rows);
    }
}

int launch_kv_attention_few(pq_ctx *ctx, const attention_args &a, int most_rows) {
    return a.cache.elem == PQ_ELEM_F16 ? few_dim<_Float16, _Float16>(ctx, a, most_rows) : few_dim<__bf16, __bf16>(ctx, a, most_rows);
}
int launch_kv_attention8_few(pq_ctx *ctx, const attention_args &a, int most_rows) {
    return a.cache.elem == PQ_ELEM_F16 ? few_dim<_Float16, e4m3>(ctx, a, most_rows) : few_dim<__bf16, e4m3>(ctx, a, most_rows);
}

}  // namespace pq
