// Attention over the paged cache of 8-bit codes (kvqp_paged_attn).
//
// One object per row type and form: KVQP_PAGED_BITS 1 + 2 * bfloat16 + int8 compiles the kernels, none the launches.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pages.h"

namespace kvqp {

struct AttnArgs {
    PageArgs p;
    const uint16_t* q;
    int64_t q_stride;
    uint16_t* out;
    float* lse;
    unsigned int* arrivals;
    char* part;
    float logit_scale;      // sm_scale / ln 2
    int window, page_log2;
    int per_piece;          // rows of the call that a workgroup has at most
    int n_splits;
};

template <bool BF, bool INT8> hipError_t paged_rows_form(const AttnArgs& a, int row_tiles, dim3 grid, hipStream_t stream);

#ifdef KVQP_PAGED_BITS

typedef float f4v __attribute__((ext_vector_type(4)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
typedef _Float16 h2v __attribute__((ext_vector_type(2)));

constexpr float kNegBig = -1.0e30f;
constexpr float kLn2 = 0.69314718055994531f;
// Weights are 2^(kLift + logit - reference) with a reference that may lag behind the row's largest logit by up to kLag: between the two a weight
// stays below 2^15 and what binary16 holds reaches 2^-29 of the row's largest weight at least (normal numbers to 2^-18).
constexpr float kLift = 4.f, kLag = 10.f;
constexpr int kDeviceScope = 16;      // sc1 in a buffer access' cache policy

// ---- codes as binary16 numbers, times a power of two (times 1 for the keys) ----
// Eight codes of two words.
template <bool INT8>
__device__ __forceinline__ h8v halves_of_codes(uint32_t lo, uint32_t hi, float scale) {
    union { h8v v; h2v h[4]; uint32_t w[4]; } r;
    if constexpr (INT8) {
        // A biased byte under the exponent of 1024 is the number 1024 + 128 + code; both products below are exact, so the sum is the code
        // times the scale, rounded once where it is below the normal numbers.
        const _Float16 s = (_Float16)scale, z = (_Float16)(-1152.f) * s;
        lo ^= 0x80808080u; hi ^= 0x80808080u;
        r.w[0] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u);
        r.w[1] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u);
        r.w[2] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u);
        r.w[3] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u);
#pragma unroll
        for (int j = 0; j < 4; ++j) r.h[j] = __builtin_elementwise_fma(r.h[j], h2v{s, s}, h2v{z, z});
    } else {
        auto half2 = [&](uint32_t w, auto high) { return __builtin_bit_cast(h2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, decltype(high)::value)); };
        r.h[0] = half2(lo, std::false_type{}); r.h[1] = half2(lo, std::true_type{});
        r.h[2] = half2(hi, std::false_type{}); r.h[3] = half2(hi, std::true_type{});
    }
    return r.v;
}

template <bool BF>
__device__ __forceinline__ f4v product_of_rows(uint4 a, uint4 b, f4v c) {      // in the rows' own type
    if constexpr (BF) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8v, a), __builtin_bit_cast(b8v, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8v, a), __builtin_bit_cast(h8v, b), c, 0, 0, 0);
}

__device__ __forceinline__ float inverse_sum(float sum) { return sum > 0.f ? 1.f / sum : sum; }      // (a row that sees nothing: zeros; NaN stays)
__device__ __forceinline__ float log_sum(float ref, float sum) { return sum == 0.f ? -INFINITY : (ref - kLift + __builtin_amdgcn_logf(sum)) * kLn2; }

// Partial results of the splits of one piece and head: outputs in the order of the accumulators, and (reference, sum) of the rows.
struct Partials {
    __amdgpu_buffer_rsrc_t at;
    int states, rt;
    __device__ __forceinline__ Partials(const AttnArgs& a, int group, int rt_) : states(a.n_splits * rt_ * 8192), rt(rt_) {
        const int bytes = states + a.n_splits * rt_ * 128;
        at = __builtin_amdgcn_make_buffer_rsrc(a.part + (size_t)group * bytes, 0, bytes, 0x00020000);
    }
    __device__ __forceinline__ void put_output(int split, int item, f4v o) const {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4v, o), at, (split * rt * 512 + item) * 16, 0, kDeviceScope);
    }
    __device__ __forceinline__ void put_state(int split, int row, float ref, float sum) const {
        const u2v v = {__float_as_uint(ref), __float_as_uint(sum)};
        __builtin_amdgcn_raw_buffer_store_b64(v, at, states + (split * rt * 16 + row) * 8, 0, kDeviceScope);
    }
    __device__ __forceinline__ f4v output(int split, int item) const {
        return __builtin_bit_cast(f4v, __builtin_amdgcn_raw_buffer_load_b128(at, (split * rt * 512 + item) * 16, 0, kDeviceScope));
    }
    __device__ __forceinline__ float2 state(int split, int row) const {
        const u2v v = __builtin_amdgcn_raw_buffer_load_b64(at, states + (split * rt * 16 + row) * 8, 0, kDeviceScope);
        return make_float2(__uint_as_float(v[0]), __uint_as_float(v[1]));
    }
};

// ---- few rows: the tokens are split over waves and workgroups ----
//
// A wave takes 64 tokens at a time.  S^T = K Q^T by products of 16 tokens and 16 rows: a lane's column is a row (query head and new token) and its
// group kb of 16 lanes holds tokens 16 kb .. 16 kb + 15, in an order that makes its logits, turned into weights, the second operand of
// O^T = V^T P^T without leaving the lane; the first operand is 16 consecutive bytes of a channel, as pages store values.
constexpr int kSegment = 512;      // pages whose numbers and scales are in LDS at a time
template <int RT> constexpr int rows_waves() { return RT == 4 ? 4 : 8; }

template <int RT, int NW>
union RowsShared {
    struct { int page[kSegment]; float k_scale[kSegment], v_scale[kSegment]; } seg;
    uint16_t open_v[64][kHeadDim + 8];
    struct { f4v o[NW][8][64]; float ref[NW][16 * RT], sum[NW][16 * RT]; } join;
};

template <bool BF, bool INT8, int RT>
__global__ __launch_bounds__(64 * rows_waves<RT>()) void paged_rows(const AttnArgs a) {
    constexpr int NW = rows_waves<RT>();
    __shared__ RowsShared<RT, NW> sh;
    __shared__ int s_found, s_last;
    __shared__ unsigned int s_top;
    const PageArgs& p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, kb = lane >> 4;
    const int piece = blockIdx.x, h = blockIdx.y, split = blockIdx.z, P = 1 << a.page_log2;
    const int b = __builtin_amdgcn_readfirstlane(owner_of_piece(p, piece, a.per_piece, 1, &s_found));
    if (b < 0) return;
    const Sequence seq = sequence_of(p, b, P);
    const int i0 = (piece - first_piece(p, b, seq.row0, a.per_piece, 1)) * a.per_piece, n = min(a.per_piece, seq.rows - i0);
    if (n <= 0) return;

    // What the rows see: whole blocks in 64 tokens at a time (groups), and open tokens.
    const int last = seq.position(i0 + n - 1), first = seq.position(i0);
    const int begin = seq.length >> a.page_log2 << a.page_log2;
    const int lo = a.window > 0 ? max(first - a.window + 1, 0) : 0, hi = last + 1;
    const int closed = min(hi, begin);
    const int g_lo = lo / 64, groups = closed > lo ? (closed + 63) / 64 - g_lo : 0;
    const int per_split = max((groups + a.n_splits - 1) / a.n_splits, NW);
    const int active = max((groups + per_split - 1) / per_split, 1);
    if (split >= active) return;
    const int ga = g_lo + split * per_split, gb = min(ga + per_split, g_lo + groups);
    const int seen_by_all = min(first + 1, closed), hidden_to_some = a.window > 0 ? last - a.window + 1 : 0;

    // The rows: queries as the second operand, 8 channels of 64 (s >> 1) + 16 kb + 8 (s & 1) a step.
    h8v q[RT][4];
    float scale[RT];           // of logits in the exponent's base, with the factor that a bfloat16 row was divided by
    int position[RT];          // of the lane's row; -1 where there is none
    int64_t q_at[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = 16 * rt + c, i = r / p.gq;
        const bool there = i < n;
        position[rt] = there ? seq.position(i0 + i) : -1;
        q_at[rt] = (int64_t)(seq.row0 + i0 + (there ? i : 0)) * a.q_stride + (h * p.gq + r % p.gq) * kHeadDim + 16 * kb;
        scale[rt] = a.logit_scale;
        uint4 w[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) w[s] = there ? *reinterpret_cast<const uint4*>(a.q + q_at[rt] + 64 * (s >> 1) + 8 * (s & 1)) : make_uint4(0, 0, 0, 0);
        if constexpr (BF) {
            // A row over a power of two is a row of binary16 numbers, but for what is below 2^-24 of its largest: codes meet it without a conversion to bfloat16.
            float m = 0.f;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const f8v x = numbers<true>(w[s]);
#pragma unroll
                for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(x[j]));
            }
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            const int e = min(max((int)(__float_as_uint(m) >> 23) - 127, -120), 120);
#pragma unroll
            for (int s = 0; s < 4; ++s) q[rt][s] = __builtin_convertvector(numbers<true>(w[s]) * two_to(-e), h8v);
            scale[rt] *= two_to(e);
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s) q[rt][s] = __builtin_bit_cast(h8v, w[s]);
        }
    }

    f4v o[RT][8];
    float ref[RT], sum[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        ref[rt] = kNegBig; sum[rt] = 0.f;
#pragma unroll
        for (int t = 0; t < 8; ++t) o[rt][t] = f4v{0.f, 0.f, 0.f, 0.f};
    }
    // Logits of one row tile (four to each of four token tiles) into weights; O and the sum follow the reference.
    auto weigh = [&](int rt, f4v (&x)[4], f8v (&w)[2]) {
        float m = x[0][0];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) m = fmaxf(m, x[t][i]);
        if (__any(m > ref[rt] + kLag)) {
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            m = fmaxf(m, ref[rt]);
            const float f = __builtin_amdgcn_exp2f(ref[rt] - m);
            ref[rt] = m;
            sum[rt] *= f;
#pragma unroll
            for (int t = 0; t < 8; ++t) o[rt][t] *= f;
        }
        const float by = kLift - ref[rt];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(x[t][i] + by);
                sum[rt] += e;
                w[t >> 1][4 * (t & 1) + i] = e;
            }
    };

    float v_top = two_to(-126);        // values are accumulated over the largest scale so far: codes times 2^0 and less fit binary16
    const int seg_groups = kSegment >> (6 - a.page_log2);
    for (int s0 = ga; s0 < gb; s0 += seg_groups) {
        const int s1 = min(s0 + seg_groups, gb), first_block = s0 << (6 - a.page_log2), blocks = (s1 - s0) << (6 - a.page_log2);
        __syncthreads();
        if (threadIdx.x == 0) s_top = __float_as_uint(v_top);
        __syncthreads();
        int holes = 0;
        float top = 0.f;
        for (int i = threadIdx.x; i < blocks; i += 64 * NW) {
            const int block = first_block + i;
            int page = -1;
            if ((int64_t)block * P < closed) page = page_of(p, b, block);
            float ks = 0.f, vs = 0.f;
            if (page >= 0) { ks = p.k_scale[(int64_t)page * p.n_kv_heads + h]; vs = p.v_scale[(int64_t)page * p.n_kv_heads + h]; }
            if (page < 0 && (int64_t)block * P < closed && block * P + P > lo) holes = 1;
            sh.seg.page[i] = page; sh.seg.k_scale[i] = ks; sh.seg.v_scale[i] = vs;
            top = fmaxf(top, vs);
        }
        atomicMax(&s_top, __float_as_uint(top));
        holes = __syncthreads_or(holes);
        top = __uint_as_float(s_top);
        if (top > v_top) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int t = 0; t < 8; ++t) o[rt][t] *= v_top / top;
            v_top = top;
        }
        const float v_over = 1.f / v_top;

        u4v kw[8], vw[8];
        auto load_keys = [&](int g) {
            const int token = 16 * (c >> 2) + (c & 3), at = (g - s0) * 64 + token;
            const int page = max(sh.seg.page[at >> a.page_log2], 0);
            const uint8_t* k = p.k_codes + (((int64_t)page * p.n_kv_heads + h) * P + (at & (P - 1))) * kHeadDim + 16 * kb;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int half = 0; half < 2; ++half) kw[2 * t + half] = *reinterpret_cast<const u4v*>(k + 4 * t * kHeadDim + 64 * half);
        };
        auto load_values = [&](int g) {
            const int at = (g - s0) * 64 + 16 * kb;
            const int page = max(sh.seg.page[at >> a.page_log2], 0);
            const uint8_t* v = p.v_codes + ((int64_t)page * p.n_kv_heads + h) * (P * kHeadDim) + c * P + (at & (P - 1));
#pragma unroll
            for (int t = 0; t < 8; ++t) vw[t] = *reinterpret_cast<const u4v*>(v + 16 * t * P);
        };
        int g = s0 + wave;
        if (g < s1) { load_keys(g); load_values(g); }
        for (; g < s1; g += NW) {
            const int mine = ((g - s0) * 64 + 16 * kb) >> a.page_log2;       // the page of the lane's 16 tokens
            const float ks = sh.seg.k_scale[mine], vs = sh.seg.v_scale[mine] * v_over;
            const bool there = sh.seg.page[mine] >= 0;
            const int next = g + NW;
            f4v x[RT][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) x[rt][t] = f4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const u4v w = kw[2 * t + half];
                    const h8v k0 = halves_of_codes<INT8>(w[0], w[1], 1.f), k1 = halves_of_codes<INT8>(w[2], w[3], 1.f);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        x[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[rt][2 * half], x[rt][t], 0, 0, 0);
                        x[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[rt][2 * half + 1], x[rt][t], 0, 0, 0);
                    }
                }
            }
            if (next < s1) load_keys(next);
            const bool edge = holes || 64 * g < hidden_to_some || 64 * g + 64 > seen_by_all;
            h8v w[RT][2];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float f = ks * scale[rt];
#pragma unroll
                for (int t = 0; t < 4; ++t) x[rt][t] *= f;
                if (edge) {
                    const int low = a.window > 0 ? position[rt] - a.window : -1;
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int token = 64 * g + 16 * kb + 4 * t + i;
                            if (!(there && token <= position[rt] && token > low)) x[rt][t][i] = -INFINITY;
                        }
                }
                f8v e[2];
                weigh(rt, x[rt], e);
                w[rt][0] = __builtin_convertvector(e[0], h8v);
                w[rt][1] = __builtin_convertvector(e[1], h8v);
            }
            if (edge && !there) {      // (nothing was stored there: it may hold NaN)
#pragma unroll
                for (int t = 0; t < 8; ++t) vw[t] = u4v{0, 0, 0, 0};
            }
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const h8v v0 = halves_of_codes<INT8>(vw[t][0], vw[t][1], vs), v1 = halves_of_codes<INT8>(vw[t][2], vw[t][3], vs);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, w[rt][0], o[rt][t], 0, 0, 0);
                    o[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, w[rt][1], o[rt][t], 0, 0, 0);
                }
            }
            if (next < s1) load_values(next);
        }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int t = 0; t < 8; ++t) o[rt][t] *= v_top;
    __syncthreads();

    // The open tokens, by one wave of the last split, in the rows' own type; bfloat16 weights are two numbers each, so that they are as exact as the others.
    const int slot = slot_of(p, b), open = max(hi - begin, 0);
    if (open > 0 && slot >= 0 && split == active - 1 && wave == (gb - ga) % NW) {
        const int64_t at = ((int64_t)slot * p.n_kv_heads + h) * (2 * P * kHeadDim);
        const int from = begin & (2 * P - 1);            // (a block's rows are next to each other)
        for (int i = lane; i < 64 * 16; i += 64) {
            const int t = i >> 4;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (t < open) v = *reinterpret_cast<const uint4*>(p.open_v + at + (from + t) * kHeadDim + 8 * (i & 15));
            *reinterpret_cast<uint4*>(&sh.open_v[t][8 * (i & 15)]) = v;
        }
        uint4 kr[4][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int off = 16 * (c >> 2) + 4 * t + (c & 3);
#pragma unroll
            for (int s = 0; s < 4; ++s)
                kr[t][s] = off < open ? *reinterpret_cast<const uint4*>(p.open_k + at + (from + off) * kHeadDim + 64 * (s >> 1) + 16 * kb + 8 * (s & 1)) : make_uint4(0, 0, 0, 0);
        }
        uint4 w[RT][2], w_rest[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            uint4 qr[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if constexpr (BF) qr[s] = position[rt] >= 0 ? *reinterpret_cast<const uint4*>(a.q + q_at[rt] + 64 * (s >> 1) + 8 * (s & 1)) : make_uint4(0, 0, 0, 0);
                else qr[s] = __builtin_bit_cast(uint4, q[rt][s]);
            }
            const int low = a.window > 0 ? position[rt] - a.window : -1;
            f4v x[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                x[t] = f4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < 4; ++s) x[t] = product_of_rows<BF>(kr[t][s], qr[s], x[t]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int off = 16 * kb + 4 * t + i, token = begin + off;
                    x[t][i] = off < open && token <= position[rt] && token > low ? x[t][i] * a.logit_scale : -INFINITY;
                }
            }
            f8v e[2];
            weigh(rt, x, e);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                w[rt][s] = rounded<BF>(e[s]);
                if constexpr (BF) w_rest[rt][s] = rounded<BF>(e[s] - numbers<BF>(w[rt][s]));
            }
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                uint32_t v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    v[j] = (uint32_t)sh.open_v[16 * kb + 8 * s + 2 * j][16 * t + c] | (uint32_t)sh.open_v[16 * kb + 8 * s + 2 * j + 1][16 * t + c] << 16;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    o[rt][t] = product_of_rows<BF>(make_uint4(v[0], v[1], v[2], v[3]), w[rt][s], o[rt][t]);
                    if constexpr (BF) o[rt][t] = product_of_rows<BF>(make_uint4(v[0], v[1], v[2], v[3]), w_rest[rt][s], o[rt][t]);
                }
            }
    }
    __syncthreads();

    // ---- the waves' results together ----
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        sum[rt] += __shfl_xor(sum[rt], 16);
        sum[rt] += __shfl_xor(sum[rt], 32);
        if (kb == 0) { sh.join.ref[wave][16 * rt + c] = ref[rt]; sh.join.sum[wave][16 * rt + c] = sum[rt]; }
    }
    __syncthreads();
    const int group = piece * p.n_kv_heads + h, per_row = p.gq;
    const Partials parts(a, group, RT);
    auto out_at = [&](int r) { return ((int64_t)(seq.row0 + i0 + r / per_row) * p.gq * p.n_kv_heads + h * p.gq + r % per_row); };
    const int rows = n * p.gq;
    auto store_out = [&](int r, int t, f4v x, float by) {
        x *= by;
        uint2 w;
        if constexpr (BF) {
            typedef __bf16 b4v __attribute__((ext_vector_type(4)));
            w = __builtin_bit_cast(uint2, __builtin_convertvector(x, b4v));
        } else {
            typedef _Float16 h4v __attribute__((ext_vector_type(4)));
            w = __builtin_bit_cast(uint2, __builtin_convertvector(x, h4v));
        }
        *reinterpret_cast<uint2*>(a.out + out_at(r) * kHeadDim + 16 * t + 4 * kb) = w;
    };
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float top = kNegBig, total = 0.f;
        for (int w = 0; w < NW; ++w) top = fmaxf(top, sh.join.ref[w][16 * rt + c]);
        for (int w = 0; w < NW; ++w) total = __builtin_fmaf(sh.join.sum[w][16 * rt + c], __builtin_amdgcn_exp2f(sh.join.ref[w][16 * rt + c] - top), total);
        const float f = __builtin_amdgcn_exp2f(ref[rt] - top);
        if (rt) __syncthreads();
#pragma unroll
        for (int t = 0; t < 8; ++t) sh.join.o[wave][t][lane] = o[rt][t] * f;
        __syncthreads();
        const int r = 16 * rt + c;
        if (wave == 0 && kb == 0) {
            if (active > 1) parts.put_state(split, r, top, total);
            else if (a.lse && r < rows) a.lse[out_at(r)] = log_sum(top, total);
        }
        for (int t = wave; t < 8; t += NW) {
            f4v x = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < NW; ++w) x += sh.join.o[w][t][lane];
            if (active > 1) parts.put_output(split, (8 * rt + t) * 64 + lane, x);
            else if (r < rows) store_out(r, t, x, inverse_sum(total));
        }
    }
    if (active == 1) return;

    // ---- the last workgroup to arrive joins the splits, in their order ----
    // The partials were stored past this die's L2, and the wait returns when the stores have been acknowledged from there; so whoever sees the
    // counter sees them, with loads that do not look into its own L2.
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        unsigned int* count = &a.arrivals[group];
        const unsigned before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = before == (unsigned)(active - 1);
        if (s_last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) return;
    for (int item = threadIdx.x; item < RT * 512; item += 64 * NW) {
        const int r = 16 * (item >> 9) + c;
        float top = kNegBig, total = 0.f;
        f4v x = {0.f, 0.f, 0.f, 0.f};
        for (int s0 = 0; s0 < active; s0 += 4) {
            f4v v[4];
            float2 m[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int s = min(s0 + u, active - 1);
                v[u] = parts.output(s, item);
                m[u] = parts.state(s, r);
            }
            float higher = top;
#pragma unroll
            for (int u = 0; u < 4; ++u) higher = fmaxf(higher, m[u].x);
            const float f = __builtin_amdgcn_exp2f(top - higher);
            x *= f; total *= f;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float w = s0 + u < active ? __builtin_amdgcn_exp2f(m[u].x - higher) : 0.f;
                x += v[u] * w;
                total = __builtin_fmaf(m[u].y, w, total);
            }
            top = higher;
        }
        if (r < rows) {
            store_out(r, (item >> 6) & 7, x, inverse_sum(total));
            if (a.lse && (item & 0x1C0) == 0 && kb == 0) a.lse[out_at(r)] = log_sum(top, total);
        }
    }
}

template <bool BF, bool INT8>
hipError_t paged_rows_form(const AttnArgs& a, int row_tiles, dim3 grid, hipStream_t stream) {
    if (row_tiles == 1) paged_rows<BF, INT8, 1><<<grid, dim3(64 * rows_waves<1>()), 0, stream>>>(a);
    else if (row_tiles == 2) paged_rows<BF, INT8, 2><<<grid, dim3(64 * rows_waves<2>()), 0, stream>>>(a);
    else paged_rows<BF, INT8, 4><<<grid, dim3(64 * rows_waves<4>()), 0, stream>>>(a);
    return hipGetLastError();
}
template hipError_t paged_rows_form<(KVQP_PAGED_BITS - 1) / 2 != 0, (KVQP_PAGED_BITS - 1) % 2 != 0>(const AttnArgs&, int, dim3, hipStream_t);

#else

// ---- launches ----
constexpr int kMostParts = 2048;                    // partial results of 16 rows each that a workspace has room for
constexpr size_t kPartBytes = 8192 + 128;
struct PagedPlan {
    int row_tiles, per_piece, pieces, n_splits;
    size_t ws_bytes;
};
static PagedPlan plan_paged(const kvqp_cfg& cfg, int n_rows, bool has_starts, int64_t most_tokens) {
    const int gq = cfg.n_q_heads / cfg.n_kv_heads, columns = (n_rows + cfg.batch - 1) / cfg.batch >= 64 ? 64 : (n_rows + cfg.batch - 1) / cfg.batch * gq;
    PagedPlan r;
    r.row_tiles = columns <= 16 ? 1 : columns <= 32 ? 2 : 4;
    r.per_piece = 16 * r.row_tiles / gq;
    r.pieces = has_starts ? n_rows / r.per_piece + cfg.batch : cfg.batch;
    const int64_t units = (int64_t)std::max(cfg.batch, n_rows / r.per_piece) * cfg.n_kv_heads, groups = (int64_t)r.pieces * cfg.n_kv_heads;
    int64_t splits = (1024 + units - 1) / units;
    splits = std::min({splits, (int64_t)64, kMostParts / (r.row_tiles * groups), most_tokens / 512 + 1});
    if (groups > KVQP_PAGED_COUNTERS / 4 || splits < 1) splits = 1;
    r.n_splits = (int)splits;
    r.ws_bytes = splits > 1 ? KVQP_PAGED_COUNTERS + groups * splits * r.row_tiles * kPartBytes : 0;
    return r;
}
size_t paged_workspace_bound(const kvqp_cfg& cfg, int n_rows) {
    (void)cfg; (void)n_rows;
    return KVQP_PAGED_COUNTERS + kMostParts * kPartBytes;
}
size_t paged_workspace_need(const kvqp_cfg& cfg, const kvqp_pages& g, int n_rows, bool has_starts) {
    return plan_paged(cfg, n_rows, has_starts, (int64_t)g.max_pages * g.page_tokens).ws_bytes;
}

PageArgs page_args(const kvqp_cfg& cfg, const kvqp_pages& g, const int32_t* row_start, int n_rows);

hipError_t launch_paged_attn(const kvqp_cfg& cfg, const kvqp_pages& g, const void* q, int64_t q_stride, int n_rows, const int32_t* row_start, int window,
                             void* out, float* lse, void* ws, hipStream_t stream) {
    const PagedPlan plan = plan_paged(cfg, n_rows, row_start != nullptr, (int64_t)g.max_pages * g.page_tokens);
    const AttnArgs a = {page_args(cfg, g, row_start, n_rows), (const uint16_t*)q, q_stride, (uint16_t*)out, lse, (unsigned int*)ws,
                        (char*)ws + KVQP_PAGED_COUNTERS, cfg.sm_scale * 1.4426950408889634f, window, g.page_tokens == 16 ? 4 : g.page_tokens == 32 ? 5 : 6,
                        plan.per_piece, plan.n_splits};
    const dim3 grid(plan.pieces, cfg.n_kv_heads, plan.n_splits);
    if (g.dtype == KVQP_BFLOAT16)
        return g.form == KVQP_INT8 ? paged_rows_form<true, true>(a, plan.row_tiles, grid, stream) : paged_rows_form<true, false>(a, plan.row_tiles, grid, stream);
    return g.form == KVQP_INT8 ? paged_rows_form<false, true>(a, plan.row_tiles, grid, stream) : paged_rows_form<false, false>(a, plan.row_tiles, grid, stream);
}

__global__ __launch_bounds__(256) void clear_paged_counters(uint32_t* at) {
    for (int i = threadIdx.x; i < KVQP_PAGED_COUNTERS / 4; i += 256) at[i] = 0u;
}
hipError_t launch_paged_init(void* ws, hipStream_t stream) {
    clear_paged_counters<<<dim3(1), dim3(256), 0, stream>>>((uint32_t*)ws);
    return hipGetLastError();
}

#endif

}  // namespace kvqp
