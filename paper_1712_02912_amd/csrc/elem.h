// Elements of the reading step (pq_elem): vectors of them, and their sizes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pq_read.h"

namespace pq {

// N elements that one load or store moves
template <class T, int N> struct __attribute__((aligned(sizeof(T) * N))) elem_vec { T v[N]; };

static inline size_t elem_bytes(int elem) { return elem == PQ_ELEM_F32 ? 4 : 2; }

}  // namespace pq
