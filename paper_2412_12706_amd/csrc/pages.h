// What the kernels of the paged cache share: its description on the device, and conversions.
#pragma once
#include <hip/hip_bf16.h>

#include "kvqp_internal.h"

namespace kvqp {

// kvqp_pages and the rows of a call, as kernels take them.
struct PageArgs {
    uint8_t *k_codes, *v_codes;
    float *k_scale, *v_scale;
    uint16_t *open_k, *open_v;
    const int32_t *table, *lengths, *open_slot, *row_start;
    int batch, n_kv_heads, gq, n_pages, max_pages, n_open, n_rows;
};

// A sequence as the device arrays state it, cut to what the buffers have.
struct Sequence {
    int b, row0, rows, length;     // its number, its rows of the call, and its tokens with them
    __device__ int position(int i) const { return length - rows + i; }      // of row i; negative: no token of the sequence
};

__device__ inline int page_of(const PageArgs& a, int b, int block) {      // block < max_pages; -1: no page
    const int page = a.table[(size_t)b * a.max_pages + block];
    return (unsigned)page < (unsigned)a.n_pages ? page : -1;
}
__device__ inline int slot_of(const PageArgs& a, int b) {
    const int slot = a.open_slot ? a.open_slot[b] : b;
    return (unsigned)slot < (unsigned)a.n_open ? slot : -1;
}

// Work is numbered by sequence without a sum over those before: sequence b's pieces (at most rows / T + per of them) begin at
// row_start[b] / T + per * b, which grows by at least as much from one to the next; with one row per sequence piece b is sequence b's.  All threads of a
// workgroup look for the one that holds `piece`, one sequence each, with its length at the same time; b = -1 (for all) where there is none.  `found`: LDS.
__device__ inline int first_piece(const PageArgs& a, const Sequence& s, int T, int per) { return a.row_start ? s.row0 / T + per * s.b : s.b; }
__device__ inline Sequence owner_of_piece(const PageArgs& a, int piece, int T, int per, int P, Sequence* found) {
    const int most = a.max_pages * P;
    if (!a.row_start) return {piece, piece, 1, min(max(a.lengths[piece], 0), most)};
    if (threadIdx.x == 0) found->b = -1;
    __syncthreads();
    Sequence mine = {-2, 0, 0, 0};
    for (int b = threadIdx.x; b < a.batch; b += blockDim.x) {
        const int r0 = min(max(a.row_start[b], 0), a.n_rows), r1 = min(max(a.row_start[b + 1], 0), a.n_rows), length = a.lengths[b];
        if (r1 > r0 && piece >= r0 / T + per * b && piece < r1 / T + per * (b + 1)) mine = {b, r0, r1 - r0, min(max(length, 0), most)};
    }
    if (mine.b >= 0) atomicMax(&found->b, mine.b);      // (descending starts may give two)
    __syncthreads();
    if (found->b == mine.b) { found->row0 = mine.row0; found->rows = mine.rows; found->length = mine.length; }
    __syncthreads();
    return *found;
}
inline int pieces(const PageArgs& a, int T, int per) { return a.row_start ? a.n_rows / T + per * a.batch : a.batch; }

// ---- 16-bit rows as numbers ----
typedef float f8v __attribute__((ext_vector_type(8)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef __bf16 b8v __attribute__((ext_vector_type(8)));

template <bool BF>
__device__ inline f8v numbers(uint4 w) {
    if constexpr (BF) return __builtin_convertvector(__builtin_bit_cast(b8v, w), f8v);
    else return __builtin_convertvector(__builtin_bit_cast(h8v, w), f8v);
}
template <bool BF>
__device__ inline uint4 rounded(f8v x) {      // to nearest, ties to even
    if constexpr (BF) return __builtin_bit_cast(uint4, __builtin_convertvector(x, b8v));
    else return __builtin_bit_cast(uint4, __builtin_convertvector(x, h8v));
}
template <bool BF>
__device__ inline float largest_finite() { return BF ? 3.38953139e38f : 65504.f; }

// 2^e, -126 <= e <= 127
__host__ __device__ inline float two_to(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

}  // namespace kvqp
