// Norm and position rotation of heads, as the appends to both kinds of cache share them (kv_cache_kernels.hip, kv_cache8_kernels.hip).
//
// A head is held by a group of lanes, each with one unit of 2 V elements: V firsts and V seconds of rotated pairs, or 2 V
// neighbours of the part that is not rotated.  So a rotation needs no exchange between lanes, only the norm's sum does,
// and every element is read and written once, 16 bytes at a time where the layout allows it.
#pragma once
#include "elem.h"
#include "pq_internal.h"

namespace pq {

struct append_args {
    pq_heads q, k, v;
    pq_kv_cache cache;
    const int32_t *positions;
    const int64_t *slots;
    const float *cos_table, *sin_table, *q_weight, *k_weight;
    void *q_out;
    int64_t ntokens, max_positions;
    float eps;
    int q_heads, rot, norm, rows;   // rows of a token: q_heads + 2 cache.heads
};

struct append_row {
    const void *from;
    void *to;             // null: nowhere
    const float *weight;
    bool turned;          // query or key: norm and rotation
    bool zero;            // query of a token without a position
};

template <class T> __device__ __forceinline__ append_row append_locate(const append_args &a, int64_t t, int row, bool placed, int64_t slot) {
    append_row r;
    const pq_kv_cache &c = a.cache;
    if (row < a.q_heads) {
        r.from = (const T *)a.q.p + t * a.q.token_stride + row * a.q.head_stride;
        r.to = (T *)a.q_out + (t * a.q_heads + row) * c.dim;
        r.weight = a.q_weight;
        r.turned = true;
        r.zero = !placed;
        return r;
    }
    const bool is_key = row < a.q_heads + c.heads;
    const int h = row - a.q_heads - (is_key ? 0 : c.heads);
    const int64_t place = slot % c.block_size, block = slot / c.block_size;
    const int64_t *strides = is_key ? c.key_strides : c.value_strides;
    const pq_heads &from = is_key ? a.k : a.v;
    r.from = (const T *)from.p + t * from.token_stride + h * from.head_stride;
    r.to = placed && slot >= 0 && block < c.nblocks ? (T *)(is_key ? c.keys : c.values) + block * strides[0] + place * strides[1] + h * strides[2] : nullptr;
    r.weight = a.k_weight;
    r.turned = is_key;
    r.zero = false;
    return r;
}

// The places of unit u: element i of the first half at x + i * step, of the second half at y + i * step.
template <int V, bool PAIRS> struct append_unit {
    int first, second, angle;   // angle: entry of the rotation tables, -1 in the part that is not rotated
    __device__ __forceinline__ append_unit(int u, int rot) {
        const int turned = rot / 2 / V;
        if (u < turned) {
            first = PAIRS ? 2 * V * u : V * u;
            second = PAIRS ? first + V : first + rot / 2;
            angle = V * u;
        } else {
            first = rot + 2 * V * (u - turned);
            second = first + V;
            angle = -1;
        }
    }
};

// rotates a unit in place; x, y: its halves as they lie in memory
template <int V, bool PAIRS, class F> __device__ __forceinline__ void append_turn(F (&x)[V], F (&y)[V], const F (&c)[V], const F (&s)[V]) {
    if constexpr (!PAIRS) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const F a = x[i], b = y[i];
            x[i] = a * c[i] - b * s[i];
            y[i] = a * s[i] + b * c[i];
        }
    } else {   // pair i: elements 2 i and 2 i + 1 of x followed by y
        F z[2 * V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            z[i] = x[i];
            z[V + i] = y[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const F a = z[2 * i], b = z[2 * i + 1];
            z[2 * i] = a * c[i] - b * s[i];
            z[2 * i + 1] = a * s[i] + b * c[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x[i] = z[i];
            y[i] = z[V + i];
        }
    }
}

constexpr int APPEND_THREADS = 256;

// The heads of a grid's threads, gl lanes for each (a power of two, at least the number of units).
template <class T, int V, bool PAIRS> __device__ __forceinline__ void append_rows(const append_args &a, int gl, int64_t thread) {
    const int64_t group = thread / gl;
    const int u = threadIdx.x & (gl - 1), dim = a.cache.dim;
    const int64_t t = group / a.rows;
    if (t >= a.ntokens) return;
    const bool active = u < dim / (2 * V);
    const append_unit<V, PAIRS> unit(active ? u : 0, a.rot);
    typedef elem_vec<T, V> vec;
    typedef elem_vec<float, V> fvec;

    const int32_t p = a.positions[t];
    const int64_t slot = a.slots[t];
    const bool placed = p >= 0 && (a.rot == 0 || p < a.max_positions);
    const append_row row = append_locate<T>(a, t, (int)(group - t * a.rows), placed, slot);
    if (!row.to) return;   // (all lanes of a head: what stands here is the row's, and so are the branches below)
    vec x, y;
    fvec c, s;
    if (active) {
        x = *(const vec *)((const T *)row.from + unit.first);
        y = *(const vec *)((const T *)row.from + unit.second);
        if (row.turned && placed && unit.angle >= 0) {
            c = *(const fvec *)(a.cos_table + (int64_t)p * (a.rot / 2) + unit.angle);
            s = *(const fvec *)(a.sin_table + (int64_t)p * (a.rot / 2) + unit.angle);
        }
    }
    if (row.turned) {
        float fx[V], fy[V], sum = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            fx[e] = active ? (float)x.v[e] : 0.f;
            fy[e] = active ? (float)y.v[e] : 0.f;
            sum += fx[e] * fx[e] + fy[e] * fy[e];
        }
        if (a.norm) {
            for (int d = gl / 2; d > 0; d /= 2) sum += __shfl_xor(sum, d);
            const float r = 1.f / sqrtf(sum / (float)dim + a.eps);
            if (active && row.weight) {
                const fvec wx = *(const fvec *)(row.weight + unit.first), wy = *(const fvec *)(row.weight + unit.second);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    fx[e] *= r * wx.v[e];
                    fy[e] *= r * wy.v[e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    fx[e] *= r;
                    fy[e] *= r;
                }
            }
        }
        if (active && placed && unit.angle >= 0) append_turn<V, PAIRS>(fx, fy, c.v, s.v);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            x.v[e] = (T)(row.zero ? 0.f : fx[e]);
            y.v[e] = (T)(row.zero ? 0.f : fy[e]);
        }
    }
    if (active) {
        *(vec *)((T *)row.to + unit.first) = x;
        *(vec *)((T *)row.to + unit.second) = y;
    }
}

// Any even dim and layout: one wave per head, element pairs one at a time, the row read again after the norm (16 384 tokens
// of 48 heads of 128 dimensions take 402 us, 77 us by groups of lanes; 4099 of 36 heads of 80 dimensions in f32 66 and 24 us).
template <class T, bool PAIRS> __device__ __forceinline__ void append_rows_general(const append_args &a, int64_t block) {
    const int lane = threadIdx.x & 63, dim = a.cache.dim;
    const int64_t item = (block * APPEND_THREADS + threadIdx.x) / 64;
    const int64_t t = item / a.rows;
    if (t >= a.ntokens) return;
    const int32_t p = a.positions[t];
    const bool placed = p >= 0 && (a.rot == 0 || p < a.max_positions);
    const append_row row = append_locate<T>(a, t, (int)(item - t * a.rows), placed, a.slots[t]);
    if (!row.to) return;
    const T *from = (const T *)row.from;
    T *to = (T *)row.to;
    float r = 1.f;
    if (row.turned && a.norm) {
        float sum = 0.f;
        for (int i = lane; i < dim; i += 64) sum += (float)from[i] * (float)from[i];
        for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d);
        r = 1.f / sqrtf(sum / (float)dim + a.eps);
    }
    for (int u = lane; u < dim / 2; u += 64) {
        const append_unit<1, PAIRS> unit(u, a.rot);
        if (!row.turned) {
            to[unit.first] = from[unit.first];
            to[unit.second] = from[unit.second];
            continue;
        }
        float x[1] = {(float)from[unit.first]}, y[1] = {(float)from[unit.second]};
        if (a.norm) {
            x[0] *= r * (row.weight ? row.weight[unit.first] : 1.f);
            y[0] *= r * (row.weight ? row.weight[unit.second] : 1.f);
        }
        if (placed && unit.angle >= 0) {
            const float c[1] = {a.cos_table[(int64_t)p * (a.rot / 2) + unit.angle]}, s[1] = {a.sin_table[(int64_t)p * (a.rot / 2) + unit.angle]};
            append_turn<1, PAIRS>(x, y, c, s);
        }
        to[unit.first] = (T)(row.zero ? 0.f : x[0]);
        to[unit.second] = (T)(row.zero ? 0.f : y[0]);
    }
}

}  // namespace pq
