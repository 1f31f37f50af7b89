// Rotary positions, and the paged cache's traffic: appending rows (rotated, quantized by blocks) and reading them back.
#include <hip/hip_runtime.h>

#include "pages.h"

namespace kvqp {

// ---- rotation ----
// Eight threads share a row: thread u has two pieces of eight channels, and with them eight whole pairs, in either layout; the eight threads' first
// pieces are next to each other, and their second ones (two neighbours a thread: 116 us instead of 110 for the case below).
struct Turn {
    const float* table;
    int n_positions, rot_dim;
    bool interleaved, inverse;
};
// Numbers (by eights) of thread u's two pieces of a row, and whether they turn.
struct Pieces {
    int lo, hi;
    bool lo_turns, hi_turns;
};
__device__ inline Pieces pieces_of(const Turn& t, int u) {
    if (!t.table) return {u, u + 8, false, false};
    const int turning = t.rot_dim >> 4;
    if (t.interleaved) return {u, u + 8, u < 2 * turning, u + 8 < 2 * turning};
    if (u < turning) return {u, u + turning, true, true};
    return {2 * turning + u - turning, 8 + u, false, false};      // (what does not turn, in two halves)
}
struct Angles {
    f8v c, s;
};
// Of pairs 8 u .. 8 u + 7, or interleaved 4 u .. 4 u + 3 and 32 places on, at a position; NaN behind the table.
__device__ inline Angles angles_at(const Turn& t, const Pieces& at, int position, int u) {
    Angles g = {};
    if (position >= t.n_positions) {
        g.c = g.s = f8v(__builtin_nanf(""));
        return g;
    }
    const float4* lo = reinterpret_cast<const float4*>(t.table + (size_t)position * t.rot_dim + (t.interleaved ? 8 : 16) * u);
    const float4* hi = lo + (t.interleaved ? 16 : 2);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float4 w = {0.f, 0.f, 0.f, 0.f};
        if (j < 2 ? at.lo_turns : at.hi_turns) w = j < 2 ? lo[j] : hi[j - 2];
        g.c[2 * j] = w.x; g.s[2 * j] = w.y; g.c[2 * j + 1] = w.z; g.s[2 * j + 1] = w.w;
    }
    if (t.inverse) g.s = -g.s;
    return g;
}
// (products and sums rounded one by one, as the definition has it: the build allows no contraction)
__device__ inline void turn(f8v& x, f8v& y, const Pieces& at, const Angles& g, bool interleaved) {
    if (!interleaved) {
        const f8v a = x * g.c - y * g.s, b = y * g.c + x * g.s;
        if (at.lo_turns) { x = a; y = b; }
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float a = x[2 * j] * g.c[j] - x[2 * j + 1] * g.s[j], b = x[2 * j + 1] * g.c[j] + x[2 * j] * g.s[j];
        const float c = y[2 * j] * g.c[4 + j] - y[2 * j + 1] * g.s[4 + j], d = y[2 * j + 1] * g.c[4 + j] + y[2 * j] * g.s[4 + j];
        if (at.lo_turns) { x[2 * j] = a; x[2 * j + 1] = b; }
        if (at.hi_turns) { y[2 * j] = c; y[2 * j + 1] = d; }
    }
}
template <bool BF>
__device__ inline void turn_words(uint4& x, uint4& y, const Pieces& at, const Angles& g, bool interleaved) {
    f8v a = numbers<BF>(x), b = numbers<BF>(y);
    turn(a, b, at, g, interleaved);
    x = rounded<BF>(a); y = rounded<BF>(b);
}

// A table entry per thread: angles in binary64, where 2^20 positions at frequency 1 still leave 2^-33 of a turn.
struct Frequencies { double f[64]; };
__global__ __launch_bounds__(256) void rope_table(Frequencies freq, int pairs, int64_t n, double magnitude, float2* table) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int64_t position = i / pairs;
    double s, c;
    sincos((double)position * freq.f[i - position * pairs], &s, &c);
    table[i] = make_float2((float)(c * magnitude), (float)(s * magnitude));
}
hipError_t launch_rope_table(const double* inv_freq, int rot_dim, int n_positions, double magnitude, float* table, hipStream_t stream) {
    Frequencies freq = {};
    for (int j = 0; j < rot_dim / 2; ++j) freq.f[j] = inv_freq[j];
    const int64_t n = (int64_t)n_positions * (rot_dim / 2);
    rope_table<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream>>>(freq, rot_dim / 2, n, magnitude, (float2*)table);
    return hipGetLastError();
}

// Bound by memory: 4 D bytes a row, and the table once for all heads.  32 rows of consecutive positions a workgroup, `per` heads of each with the same angles in
// registers.  2 x 16381 rows of 32 heads, interleaved, half of the head (541 MB): 110 us, 4.9 TB/s (a large copy 5.2); non-temporal loads and stores took 174.
// 32 rows of 32 heads: 6.8 us as a call, 3.3 in a graph.
constexpr int kAtOnce = 4;
struct RotateArgs {
    Turn t;
    const uint16_t* x; int64_t xb, xh, xr;
    uint16_t* out; int64_t ob, oh, orow;
    const int32_t* positions; int64_t positions_stride;
    int heads, rows, first, per;
};
template <bool BF>
__global__ __launch_bounds__(256) void rotate(RotateArgs a) {
    const int u = threadIdx.x & 7, row = blockIdx.x * 32 + (threadIdx.x >> 3), batch = blockIdx.z;
    if (row >= a.rows) return;
    const int position = a.positions ? a.positions[batch * a.positions_stride + row] : a.first + row;
    if (position < 0) return;
    const Pieces at = pieces_of(a.t, u);
    Angles g = {};
    if (at.lo_turns) g = angles_at(a.t, at, position, u);
    const int h0 = blockIdx.y * a.per, h1 = min(h0 + a.per, a.heads);
    const uint16_t* x = a.x + batch * a.xb + row * a.xr;
    uint16_t* out = a.out + batch * a.ob + row * a.orow;
    // (four heads' rows are requested before the first is stored)
    for (int h = h0; h < h1; h += kAtOnce) {
        uint4 lo[kAtOnce], hi[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const uint16_t* from = x + min(h + i, h1 - 1) * a.xh;
            lo[i] = *reinterpret_cast<const uint4*>(from + 8 * at.lo);
            hi[i] = *reinterpret_cast<const uint4*>(from + 8 * at.hi);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (h + i >= h1) break;
            if (at.lo_turns) turn_words<BF>(lo[i], hi[i], at, g, a.t.interleaved);
            *reinterpret_cast<uint4*>(out + (h + i) * a.oh + 8 * at.lo) = lo[i];
            *reinterpret_cast<uint4*>(out + (h + i) * a.oh + 8 * at.hi) = hi[i];
        }
    }
}
hipError_t launch_rotate(const kvqp_rope& rope, int dtype, int batch, int heads, int rows, const kvqp_rows& x, const kvqp_rows& out,
                         const int32_t* positions, bool positions_per_batch, int first, bool inverse, hipStream_t stream) {
    RotateArgs a = {{rope.table, rope.n_positions, rope.rot_dim, rope.interleaved != 0, inverse},
                    (const uint16_t*)x.data, x.batch_stride, x.head_stride, x.row_stride,
                    (uint16_t*)out.data, out.batch_stride, out.head_stride, out.row_stride,
                    positions, positions_per_batch ? rows : 0, heads, rows, first, 1};
    // (heads with the same angles as long as there are workgroups enough: sixteen a CU)
    const int64_t blocks = (int64_t)((rows + 31) / 32) * batch;
    while (a.per < 8 && a.per < heads && blocks * ((heads + a.per - 1) / a.per) > 4096) a.per *= 2;
    const dim3 grid((rows + 31) / 32, (heads + a.per - 1) / a.per, batch);
    if (dtype == KVQP_BFLOAT16) rotate<true><<<grid, dim3(256), 0, stream>>>(a);
    else rotate<false><<<grid, dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}

// ---- appending ----
struct AppendArgs {
    PageArgs p;
    Turn t;                         // table NULL: no rotation
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    const int32_t* positions;
    uint16_t* q_out;
};

// The least e >= -126 with a <= M 2^e, from a's exponent and mantissa: a = m 2^x with m in [1/2, 1), M = 7/8 2^9 or 127/128 2^7.
template <bool INT8>
__device__ inline int exponent_for(float a) {
    const uint32_t w = __builtin_bit_cast(uint32_t, a);
    const int x = (int)(w >> 23) - 126;
    const bool above = (w & 0x7FFFFF) > (INT8 ? 0x7E0000u : 0x600000u);
    return max(x - (INT8 ? 7 : 9) + (above ? 1 : 0), -126);
}
// Eight codes of numbers that a scale's inverse brought into the form's range.
template <bool INT8>
__device__ inline uint2 codes_of(f8v y) {
    if constexpr (INT8) {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = (uint32_t)(int)rintf(y[j]) & 0xFFu;
        return make_uint2(w[0] | w[1] << 8 | w[2] << 16 | w[3] << 24, w[4] | w[5] << 8 | w[6] << 16 | w[7] << 24);
    } else {
        int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
        return make_uint2((uint32_t)lo, (uint32_t)hi);
    }
}
template <bool BF>
__device__ inline f8v finite(f8v x) {
    const float most = largest_finite<BF>();
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = x[j] != x[j] ? 0.f : fminf(fmaxf(x[j], -most), most);
    return x;
}
template <bool BF>
__device__ inline uint4 finite_words(uint4 w) { return rounded<BF>(finite<BF>(numbers<BF>(w))); }
__device__ inline float largest(f8v x) {
    float m = fabsf(x[0]);
#pragma unroll
    for (int j = 1; j < 8; ++j) m = fmaxf(m, fabsf(x[j]));
    return m;
}

// A workgroup has the new tokens of one block of one sequence, for one KV head and its query heads; where the block is full now it quantizes it, with
// the tokens that the open part held before.  So one launch does all, a block's scale needs no exchange between workgroups, and a step's rows, a few KB a
// sequence, take the time of a launch and its chain (which sequence, positions, angles, rows): 96 sequences 8.5 us as a call, 7.4 in a graph.  Prompts are bound
// by memory: 4 of up to 8191 tokens, 32 query and 8 KV heads (535 MB) 118 us, 4.5 TB/s.  Codes of values are turned channel by channel in LDS.
template <bool BF, bool INT8, int P>
__global__ __launch_bounds__(256) void append(AppendArgs a) {
    constexpr int TOKENS = P < 32 ? P : 32, PASSES = P / TOKENS, GROUPS = 32 / TOKENS, AT_ONCE = kAtOnce / GROUPS;
    __shared__ Sequence found;
    __shared__ float s_max[2][4];
    __shared__ __align__(16) uint8_t s_codes[128][P + 4];
    const PageArgs& p = a.p;
    const Sequence seq = owner_of_piece(p, blockIdx.x, P, 2, P, &found);
    const int b = seq.b;
    if (b < 0) return;
    const int begin = max(seq.position(0), 0), first = begin / P;
    const int block = first + (int)blockIdx.x - first_piece(p, seq, P, 2);
    if (block < first || (int64_t)block * P >= seq.length) return;
    const int h = blockIdx.y, u = threadIdx.x & 7, token = (threadIdx.x >> 3) % TOKENS, group = (threadIdx.x >> 3) / TOKENS;
    const Pieces at = pieces_of(a.t, u);
    const int slot = slot_of(p, b), last = (seq.length - 1) / P;
    uint16_t* const open_k = p.open_k + ((int64_t)max(slot, 0) * p.n_kv_heads + h) * (2 * P * kHeadDim);
    uint16_t* const open_v = p.open_v + ((int64_t)max(slot, 0) * p.n_kv_heads + h) * (2 * P * kHeadDim);
    auto row_of = [&](int t) { return seq.row0 + t - seq.position(0); };
    auto angles = [&](int t, bool& turning) {
        Angles g = {};
        turning = at.lo_turns;
        if (turning) {
            const int position = a.positions ? a.positions[row_of(t)] : t;
            turning = position >= 0;
            if (turning) g = angles_at(a.t, at, position, u);
        }
        return g;
    };
    auto key = [&](const Angles& g, bool turning, uint4& lo, uint4& hi) {      // a row as it came into one as it is stored
        f8v y = numbers<BF>(lo), z = numbers<BF>(hi);
        if (turning) turn(y, z, at, g, a.t.interleaved);
        lo = rounded<BF>(finite<BF>(y)); hi = rounded<BF>(finite<BF>(z));
    };
    auto open_row = [&](uint16_t* open, int t) { return open + (t % (2 * P)) * kHeadDim; };
    auto keep_key = [&](int t, uint4 lo, uint4 hi) {
        *reinterpret_cast<uint4*>(open_row(open_k, t) + 8 * at.lo) = lo;
        *reinterpret_cast<uint4*>(open_row(open_k, t) + 8 * at.hi) = hi;
    };
    auto keep_value = [&](int t, uint4 lo, uint4 hi) {
        *reinterpret_cast<uint4*>(open_row(open_v, t) + 8 * u) = lo;
        *reinterpret_cast<uint4*>(open_row(open_v, t) + 8 * u + 64) = hi;
    };

    const bool full = (block + 1) * P <= seq.length;
    // The two last blocks stay in the open part.  Where the sequence's first block here began earlier, its older tokens are still to be read from
    // there: a later block that goes to the same places is stored by the first block's workgroup, behind its reads.
    const bool older = begin % P != 0;
    const bool clash = older && block > first && ((block ^ first) & 1) == 0;
    const bool keeps = slot >= 0 && block >= last - 1 && !clash;
    uint4 klo[PASSES], khi[PASSES], vlo[PASSES], vhi[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int t = block * P + i * TOKENS + token;
        klo[i] = khi[i] = vlo[i] = vhi[i] = make_uint4(0, 0, 0, 0);
        if (t >= begin && t < seq.length) {
            bool turning;
            const Angles g = angles(t, turning);
            // (the key's and the value's row, and four query heads' at a time, are requested before anything is stored)
            const uint16_t *k = a.k + row_of(t) * a.k_stride + h * kHeadDim, *v = a.v + row_of(t) * a.v_stride + h * kHeadDim + 8 * u;
            if (group == 0) { klo[i] = *reinterpret_cast<const uint4*>(k + 8 * at.lo); khi[i] = *reinterpret_cast<const uint4*>(k + 8 * at.hi); }
            if (group == GROUPS - 1) { vlo[i] = *reinterpret_cast<const uint4*>(v); vhi[i] = *reinterpret_cast<const uint4*>(v + 64); }
            if (a.q) {
                const uint16_t* x = a.q + row_of(t) * a.q_stride + h * p.gq * kHeadDim;
                uint16_t* out = a.q_out + ((int64_t)row_of(t) * p.gq * p.n_kv_heads + h * p.gq) * kHeadDim;
                for (int r = group; r < p.gq; r += GROUPS * AT_ONCE) {
                    uint4 lo[AT_ONCE], hi[AT_ONCE];
#pragma unroll
                    for (int j = 0; j < AT_ONCE; ++j) {
                        const uint16_t* from = x + min(r + j * GROUPS, p.gq - 1) * kHeadDim;
                        lo[j] = *reinterpret_cast<const uint4*>(from + 8 * at.lo);
                        hi[j] = *reinterpret_cast<const uint4*>(from + 8 * at.hi);
                    }
#pragma unroll
                    for (int j = 0; j < AT_ONCE; ++j) {
                        if (r + j * GROUPS >= p.gq) break;
                        if (turning) turn_words<BF>(lo[j], hi[j], at, g, a.t.interleaved);
                        *reinterpret_cast<uint4*>(out + (r + j * GROUPS) * kHeadDim + 8 * at.lo) = lo[j];
                        *reinterpret_cast<uint4*>(out + (r + j * GROUPS) * kHeadDim + 8 * at.hi) = hi[j];
                    }
                }
            }
            if (group == 0) {
                key(g, turning, klo[i], khi[i]);
                if (keeps) keep_key(t, klo[i], khi[i]);
            }
            if (group == GROUPS - 1) {
                vlo[i] = finite_words<BF>(vlo[i]); vhi[i] = finite_words<BF>(vhi[i]);
                if (keeps) keep_value(t, vlo[i], vhi[i]);
            }
        } else if (full && t < begin && slot >= 0) {
            if (group == 0) {
                klo[i] = *reinterpret_cast<const uint4*>(open_row(open_k, t) + 8 * at.lo);
                khi[i] = *reinterpret_cast<const uint4*>(open_row(open_k, t) + 8 * at.hi);
            }
            if (group == GROUPS - 1) {
                vlo[i] = *reinterpret_cast<const uint4*>(open_row(open_v, t) + 8 * u);
                vhi[i] = *reinterpret_cast<const uint4*>(open_row(open_v, t) + 8 * u + 64);
            }
        }
    }
    if (full) {
        float mk = 0.f, mv = 0.f;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            mk = fmaxf(mk, fmaxf(largest(numbers<BF>(klo[i])), largest(numbers<BF>(khi[i]))));
            mv = fmaxf(mv, fmaxf(largest(numbers<BF>(vlo[i])), largest(numbers<BF>(vhi[i]))));
        }
        for (int s = 1; s < 64; s *= 2) { mk = fmaxf(mk, __shfl_xor(mk, s)); mv = fmaxf(mv, __shfl_xor(mv, s)); }
        if ((threadIdx.x & 63) == 0) { s_max[0][threadIdx.x >> 6] = mk; s_max[1][threadIdx.x >> 6] = mv; }
        __syncthreads();
        mk = fmaxf(fmaxf(s_max[0][0], s_max[0][1]), fmaxf(s_max[0][2], s_max[0][3]));
        mv = fmaxf(fmaxf(s_max[1][0], s_max[1][1]), fmaxf(s_max[1][2], s_max[1][3]));
        const int ek = exponent_for<INT8>(mk), ev = exponent_for<INT8>(mv), page = page_of(p, b, block);
        const int64_t block_at = (int64_t)max(page, 0) * p.n_kv_heads + h;
        if (page >= 0 && threadIdx.x == 0) { p.k_scale[block_at] = two_to(ek); p.v_scale[block_at] = two_to(ev); }
        const float fk = two_to(-ek), fv = two_to(-ev);
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int t = i * TOKENS + token;
            if (group == 0 && page >= 0) {
                uint8_t* to = p.k_codes + (block_at * P + t) * kHeadDim;
                *reinterpret_cast<uint2*>(to + 8 * at.lo) = codes_of<INT8>(numbers<BF>(klo[i]) * fk);
                *reinterpret_cast<uint2*>(to + 8 * at.hi) = codes_of<INT8>(numbers<BF>(khi[i]) * fk);
            }
            if (group == GROUPS - 1) {
                const uint2 lo = codes_of<INT8>(numbers<BF>(vlo[i]) * fv), hi = codes_of<INT8>(numbers<BF>(vhi[i]) * fv);
                const uint32_t w[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
                for (int j = 0; j < 16; ++j) s_codes[8 * u + j + (j < 8 ? 0 : 56)][t] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
            }
        }
        __syncthreads();
        if (page >= 0) {
            uint8_t* to = p.v_codes + block_at * (P * kHeadDim);
            for (int i = threadIdx.x; i < 128 * P / 16; i += 256) {
                const uint32_t* w = reinterpret_cast<const uint32_t*>(&s_codes[i * 16 / P][i * 16 % P]);
                *reinterpret_cast<uint4*>(to + 16 * i) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
    if (block != first || !older || slot < 0) return;
    const int late = last - ((last ^ first) & 1);        // the last or the one before it: the one that goes where the first is
    if (late <= first) return;
    __syncthreads();                                     // (every thread's reads of the first block's older tokens have arrived: they are in codes)
    for (int t = late * P + token; t < min((late + 1) * P, seq.length); t += TOKENS) {
        bool turning;
        const Angles g = angles(t, turning);
        const uint16_t *k = a.k + row_of(t) * a.k_stride + h * kHeadDim, *v = a.v + row_of(t) * a.v_stride + h * kHeadDim + 8 * u;
        if (group == 0) {
            uint4 lo = *reinterpret_cast<const uint4*>(k + 8 * at.lo), hi = *reinterpret_cast<const uint4*>(k + 8 * at.hi);
            key(g, turning, lo, hi);
            keep_key(t, lo, hi);
        }
        if (group == GROUPS - 1) keep_value(t, finite_words<BF>(*reinterpret_cast<const uint4*>(v)), finite_words<BF>(*reinterpret_cast<const uint4*>(v + 64)));
    }
}

// ---- reading back ----
struct ReadArgs {
    PageArgs p;
    int first, count;
    uint16_t *k_out, *v_out;
};
// Four codes as numbers.
template <bool INT8>
__device__ inline float4 numbers_of_codes(uint32_t w) {
    if constexpr (INT8) {
        return make_float4((float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24));
    } else {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        return make_float4(lo[0], lo[1], hi[0], hi[1]);
    }
}
template <bool BF, bool INT8>
__device__ inline uint4 rows_of_codes(uint2 w, float scale) {
    const float4 lo = numbers_of_codes<INT8>(w.x), hi = numbers_of_codes<INT8>(w.y);
    f8v x = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    const float most = largest_finite<BF>();
    x *= scale;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = fminf(fmaxf(x[j], -most), most);
    return rounded<BF>(x);
}

// A workgroup has 64 tokens, counted from the sequence's beginning, of one head; values are turned back in LDS.  Bound by memory: 2 x 32768 tokens of 8 heads
// (403 MB) 83 us, 4.8 TB/s; 999 tokens 6.3 us as a call, 4.8 in a graph.
template <bool BF, bool INT8, int P>
__global__ __launch_bounds__(256) void read(ReadArgs a) {
    constexpr int PAGES = 64 / P;
    __shared__ int s_page[PAGES];
    __shared__ float s_scale[2][PAGES];
    __shared__ __align__(16) uint16_t s_v[64][kHeadDim + 8];
    const PageArgs& p = a.p;
    const int b = blockIdx.z, h = blockIdx.y, t0 = (a.first / 64 + blockIdx.x) * 64;
    const int length = min(max(p.lengths[b], 0), p.max_pages * P), begin = length / P * P;
    if (threadIdx.x < PAGES) {
        const int block = t0 / P + threadIdx.x, page = block * P < begin ? page_of(p, b, block) : -1;
        s_page[threadIdx.x] = page;
        s_scale[0][threadIdx.x] = page >= 0 ? p.k_scale[(int64_t)page * p.n_kv_heads + h] : 0.f;
        s_scale[1][threadIdx.x] = page >= 0 ? p.v_scale[(int64_t)page * p.n_kv_heads + h] : 0.f;
    }
    __syncthreads();
    // values: 16 tokens of a channel at a time, turned in LDS
    for (int i = threadIdx.x; i < 64 * kHeadDim / 16; i += 256) {
        const int part = i * 16 / (P * kHeadDim), in = i - part * (P * kHeadDim / 16), page = s_page[part];
        if (page < 0) continue;
        const uint4 w = *reinterpret_cast<const uint4*>(p.v_codes + ((int64_t)page * p.n_kv_heads + h) * (P * kHeadDim) + 16 * in);
        const int d = in * 16 / P, t = part * P + in * 16 % P;
        const uint4 lo = rows_of_codes<BF, INT8>(make_uint2(w.x, w.y), s_scale[1][part]), hi = rows_of_codes<BF, INT8>(make_uint2(w.z, w.w), s_scale[1][part]);
        const uint32_t x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int j = 0; j < 16; ++j) s_v[t + j][d] = (uint16_t)(x[j / 2] >> (16 * (j & 1)));
    }
    __syncthreads();
    const int slot = slot_of(p, b);
    const int64_t open_at = ((int64_t)max(slot, 0) * p.n_kv_heads + h) * (2 * P * kHeadDim);
    for (int i = threadIdx.x; i < 64 * 16; i += 256) {
        const int t = t0 + i / 16, c = i % 16;
        if (t < a.first || t >= a.first + a.count) continue;
        uint4 k = make_uint4(0, 0, 0, 0), v = k;
        if (t < begin) {
            const int part = (t - t0) / P, page = s_page[part];
            if (page >= 0) {
                const uint2 w = *reinterpret_cast<const uint2*>(p.k_codes + (((int64_t)page * p.n_kv_heads + h) * P + t % P) * kHeadDim + 8 * c);
                k = rows_of_codes<BF, INT8>(w, s_scale[0][part]);
                v = *reinterpret_cast<const uint4*>(&s_v[t - t0][8 * c]);
            }
        } else if (t < length && slot >= 0) {
            k = *reinterpret_cast<const uint4*>(p.open_k + open_at + (t % (2 * P)) * kHeadDim + 8 * c);
            v = *reinterpret_cast<const uint4*>(p.open_v + open_at + (t % (2 * P)) * kHeadDim + 8 * c);
        }
        const int64_t to = (((int64_t)b * p.n_kv_heads + h) * a.count + (t - a.first)) * kHeadDim + 8 * c;
        *reinterpret_cast<uint4*>(a.k_out + to) = k;
        *reinterpret_cast<uint4*>(a.v_out + to) = v;
    }
}

PageArgs page_args(const kvqp_cfg& cfg, const kvqp_pages& g, const int32_t* row_start, int n_rows) {
    return {(uint8_t*)g.k_codes, (uint8_t*)g.v_codes, g.k_scale, g.v_scale, (uint16_t*)g.open_k, (uint16_t*)g.open_v, g.table, g.lengths, g.open_slot,
            row_start, cfg.batch, cfg.n_kv_heads, cfg.n_q_heads / cfg.n_kv_heads, g.n_pages, g.max_pages, g.n_open, n_rows};
}

template <bool BF, bool INT8>
static hipError_t append_pages(const AppendArgs& a, int P, hipStream_t stream) {
    const dim3 grid(pieces(a.p, P, 2), a.p.n_kv_heads);
    if (P == 16) append<BF, INT8, 16><<<grid, dim3(256), 0, stream>>>(a);
    else if (P == 32) append<BF, INT8, 32><<<grid, dim3(256), 0, stream>>>(a);
    else append<BF, INT8, 64><<<grid, dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}
hipError_t launch_paged_append(const kvqp_cfg& cfg, const kvqp_pages& g, const kvqp_rope* rope, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                               const void* v, int64_t v_stride, int n_rows, const int32_t* row_start, const int32_t* positions, void* q_out,
                               hipStream_t stream) {
    AppendArgs a = {page_args(cfg, g, row_start, n_rows), {nullptr, 0, 0, false, false}, (const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v,
                    q_stride, k_stride, v_stride, positions, (uint16_t*)q_out};
    if (rope) a.t = {rope->table, rope->n_positions, rope->rot_dim, rope->interleaved != 0, false};
    if (g.dtype == KVQP_BFLOAT16) return g.form == KVQP_INT8 ? append_pages<true, true>(a, g.page_tokens, stream) : append_pages<true, false>(a, g.page_tokens, stream);
    return g.form == KVQP_INT8 ? append_pages<false, true>(a, g.page_tokens, stream) : append_pages<false, false>(a, g.page_tokens, stream);
}

template <bool BF, bool INT8>
static hipError_t read_pages(const ReadArgs& a, int P, hipStream_t stream) {
    const dim3 grid((a.first + a.count - 1) / 64 - a.first / 64 + 1, a.p.n_kv_heads, a.p.batch);
    if (P == 16) read<BF, INT8, 16><<<grid, dim3(256), 0, stream>>>(a);
    else if (P == 32) read<BF, INT8, 32><<<grid, dim3(256), 0, stream>>>(a);
    else read<BF, INT8, 64><<<grid, dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}
hipError_t launch_paged_read(const kvqp_cfg& cfg, const kvqp_pages& g, int first, int count, void* k_out, void* v_out, hipStream_t stream) {
    const ReadArgs a = {page_args(cfg, g, nullptr, 0), first, count, (uint16_t*)k_out, (uint16_t*)v_out};
    if (g.dtype == KVQP_BFLOAT16) return g.form == KVQP_INT8 ? read_pages<true, true>(a, g.page_tokens, stream) : read_pages<true, false>(a, g.page_tokens, stream);
    return g.form == KVQP_INT8 ? read_pages<false, true>(a, g.page_tokens, stream) : read_pages<false, false>(a, g.page_tokens, stream);
}

}  // namespace kvqp
