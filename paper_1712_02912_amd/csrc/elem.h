// Element types of the reading step (pq_elem): loads to fp32, stores rounded once to the nearest, and vectors of them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pq_read.h"

namespace pq {

template <int E> struct elem_of;
template <> struct elem_of<PQ_ELEM_F32> { typedef float type; };
template <> struct elem_of<PQ_ELEM_F16> { typedef _Float16 type; };
template <> struct elem_of<PQ_ELEM_BF16> { typedef __bf16 type; };

// N elements that one load or store moves
template <class T, int N> struct __attribute__((aligned(sizeof(T) * N))) elem_vec { T v[N]; };

static inline size_t elem_bytes(int elem) { return elem == PQ_ELEM_F32 ? 4 : 2; }

}  // namespace pq
