// Attention of several query rows over the packed cache: the drafted tokens of a speculative step
// (kvqp_tree_attn), and the attention weight that every cached token receives from such rows
// (kvqp_accumulate_weights, which is what an eviction goes by).
//
// Per KV head there are R = Gq * N query rows (N tokens, Gq query heads).  With l[r, t] =
// sm_scale q[r] . K[t] over all tokens that row r sees,
//   lse[r] = log sum_t exp(l[r, t])      out[r] = sum_t exp(l[r, t] - lse[r]) V[t]
//   weight[t] = sum_r exp(l[r, t] - lse[r])
// K and V are code * scale + zero of the packed part, and plain rows of the tail and of the drafted
// tokens.  The cache is read once per 64 rows; a row costs 512 multiply-adds per token, and every
// operand twice (see below).  32 layers of 8192 tokens at 4 bits (345 MB), on cards that differ by a tenth: 16 rows take 79 to 86 us (4.0 to
// 4.4 TB/s), 32 rows 103 to 118 and 64 rows 192, bound by instruction issue and power.
//
// Layout on gfx950.  A wave takes blocks of 32 tokens, for all rows of its workgroup (16, 32 or 64).
// Both products run transposed, S^T[token, row] = K Q^T and O^T[channel, row] = V^T P^T, with
// v_mfma_f32_16x16x32_f16: lane (n = lane % 16, kb = lane / 16) then holds, of row n, the logits of
// tokens 16 H + 4 kb + i, and these are exactly the tokens whose value codes the cache's
// tile-transposed layout gives the same lane as the other operand.  Probabilities stay in the lane
// that computed them, a row's reference, sum and output are that lane's (times four), and nothing
// crosses lanes inside the loop except the rare change of a reference.
//
// Exactness.  Logits are exact to about 2^-22 although the operands are binary16:
//   keys per channel: the codes times q * s split into binary16 hi + lo parts (v_pk_mul, and v_pk_fma for
//     what the product lost), or above 32 rows code * s split so times q; q . z comes from a product of
//     sixteen groups' zeros at a time.  (Codes are whole numbers: as subnormals code * 2^-24, which cost one
//     AND, the matrix unit lines products up by their nominal exponents and loses what lies below, 2e-5 of a weight);
//   keys per token: code * s split the same way times q, and z (its rows are constant over a group of
//     channels) times the sums of q over 32 channels, again hi + lo.
// Query rows are scaled by a power of two to a largest element of 64 .. 128, so that the lo parts do
// not run into binary16's subnormals.  Products that a large scale would take out of binary16's range are formed apart (wide_bits).
// Weights enter the second product as hi + lo too, and values as code * s, hi + lo, while the zeros take a product of their own: its rows are
// the groups of channels.  (A value rounded to binary16, code * s + z, adds as
// much error as the output's own rounding: 2.8e-4 where the formula rounded once has 2.1e-4.  The parts cost ten matrix instructions a block and
// tile of rows: 32 layers of 8192 tokens, 32 rows: 101 -> 110 us; one layer of 16384 tokens, 256 rows: 49 -> 56.)
#include <algorithm>
#include <initializer_list>

#include "kvqp_internal.h"

namespace kvqp {
namespace {

typedef _Float16 h2v __attribute__((ext_vector_type(2)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef float f4v __attribute__((ext_vector_type(4)));

union Frag {  // one MFMA 16x16x32 f16 input operand of a lane: 8 halves
    h8v v;
    uint32_t u[4];
    h2v h[4];
    uint4 q;
};

// The most waves of a workgroup, by its rows in tiles of 16: as many as the registers of a CU leave room for (168 and 256 per lane).
// A launch may use fewer.  (Sixteen for one tile, with 128 registers each: 73.4 us where twelve
// take 68.5, 32 layers of 8192 tokens, 16 rows.)
constexpr int most_waves(int rt) { return rt <= 2 ? 12 : 8; }
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNegBig = -1.0e30f;     // reference of a row that has seen nothing
// A row's reference moves when a logit (log2) passes it by kSlack, and then to kBoost below that logit: a wave's largest weight of a row is 2^kBoost
// to 2^kSlack, and the hi + lo parts (binary16, cut toward zero) are off by 2^-21 of a weight down to 2^-3, 2^-11 of the largest and less.  Smaller
// ones' lo parts end at binary16's lowest step: 2^-24, 2^-32 of the largest.
constexpr float kSlack = 12.0f, kBoost = 8.0f;

__device__ __forceinline__ h2v as_h2(uint32_t u) { union { uint32_t u; h2v h; } c; c.u = u; return c.h; }
__device__ __forceinline__ uint32_t as_u32(h2v h) { union { uint32_t u; h2v h; } c; c.h = h; return c.u; }
__device__ __forceinline__ float half_to_float(uint16_t u) { return __half2float(__ushort_as_half(u)); }
__device__ __forceinline__ h2v splat(float x) { return h2v{(_Float16)x, (_Float16)x}; }
// two binary32 values cut (toward zero) to binary16, (lo, hi) half-words
__device__ __forceinline__ uint32_t pack_rtz(float lo, float hi) {
    typedef __fp16 fp16x2 __attribute__((ext_vector_type(2)));
    union { fp16x2 h; uint32_t u; } c; c.h = __builtin_amdgcn_cvt_pkrtz(lo, hi); return c.u;
}
// Data that passes between lanes of one wave through its own LDS: the hardware keeps a wave's LDS accesses in order, this keeps
// the compiler from moving accesses of different types across each other.
__device__ __forceinline__ void lds_order() { asm volatile("" ::: "memory"); }
__device__ __forceinline__ f4v mfma(const Frag& a, const Frag& b, f4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, b.v, c, 0, 0, 0); }

// sum / max over the four lanes that share lane % 16
__device__ __forceinline__ float rows4_max(float v) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float rows4_add(float v) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The higher of two numbers out of the matrix unit, as the middle one of three: fmaxf would quiet both first, an instruction each, and an
// instruction written in assembly would not wait for the matrix unit.
__device__ __forceinline__ float higher(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, 3.4028235e38f); }
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, 0xF, 0xF, true));
}
constexpr int kQuadXor1 = 0xB1, kQuadXor2 = 0x4E, kRowHalfMirror = 0x141, kRowMirror = 0x140;
// sum / max over the 16 lanes of a row of lanes, in every lane
__device__ __forceinline__ float row16_add(float v) {
    v += dpp<kQuadXor1>(v); v += dpp<kQuadXor2>(v); v += dpp<kRowHalfMirror>(v); v += dpp<kRowMirror>(v);
    return v;
}
__device__ __forceinline__ float row16_max(float v) {
    v = fmaxf(v, dpp<kQuadXor1>(v)); v = fmaxf(v, dpp<kQuadXor2>(v)); v = fmaxf(v, dpp<kRowHalfMirror>(v)); v = fmaxf(v, dpp<kRowMirror>(v));
    return v;
}

// ---- codes ----
// Pairs of fields as whole numbers in binary16.  With the exponent of 1024 put over a field that begins at bit SH of its half-word (and
// ends below bit 10) it reads 1024 + 2^SH code; fields keep their places where they can.  The masks come from vector registers:
// v_and_or_b32 takes one constant, and masking and setting the exponent are one instruction then.
template <int BITS> struct Fields {
    uint32_t mask[BITS == 2 ? 4 : BITS == 4 ? 2 : 1];
    __device__ __forceinline__ Fields() {
        if constexpr (BITS == 8) mask[0] = 0x00FF00FFu;
        else if constexpr (BITS == 4) { mask[0] = 0x000F000Fu; mask[1] = 0x00F000F0u; }
        else if constexpr (BITS == 2) { mask[0] = 0x00030003u; mask[1] = 0x000C000Cu; mask[2] = 0x00300030u; mask[3] = 0x00C000C0u; }
        if constexpr (BITS != 16)
#pragma unroll
            for (uint32_t& m : mask) asm("" : "+v"(m));
    }
    template <int SH> __device__ __forceinline__ static h2v whole(uint32_t w, uint32_t m) {
        const h2v x = as_h2((w & m) | 0x64006400u);
        if constexpr (SH == 0) return x - splat(1024.0f);
        else return __builtin_elementwise_fma(x, splat(1.0f / (1 << SH)), splat(-1024.0f / (1 << SH)));
    }
    // eight codes of one (4 bits, 2 bits: half of one) or two words
    __device__ __forceinline__ void eight(uint32_t a, uint32_t b, h2v* c) const {
        if constexpr (BITS == 8) {
            c[0] = whole<0>(a, mask[0]); c[1] = whole<0>(a >> 8, mask[0]);
            c[2] = whole<0>(b, mask[0]); c[3] = whole<0>(b >> 8, mask[0]);
        } else if constexpr (BITS == 4) {
            c[0] = whole<0>(a, mask[0]); c[1] = whole<4>(a, mask[1]);
            c[2] = whole<0>(a >> 8, mask[0]); c[3] = whole<4>(a >> 8, mask[1]);
        } else if constexpr (BITS == 2) {
            c[0] = whole<0>(a, mask[0]); c[1] = whole<2>(a, mask[1]); c[2] = whole<4>(a, mask[2]); c[3] = whole<6>(a, mask[3]);
        }
    }
};
// Eight consecutive channels of a key row (step s of a lane's 32 channels): c[r] is the pair 8 s + 2 r, + 1.
template <int BITS>
__device__ __forceinline__ void key_whole(const Fields<BITS>& f, const uint32_t (&w)[BITS], int s, h2v* c) {
    if constexpr (BITS == 8) f.eight(w[2 * s], w[2 * s + 1], c);
    else if constexpr (BITS == 4) f.eight(w[s], 0u, c);
    else if constexpr (BITS == 2) f.eight((s & 1) ? w[s >> 1] >> 8 : w[s >> 1], 0u, c);
}
// Value codes of a 32-token block, channel tile `tile`: pair i holds tokens 4 kb + i and 16 + 4 kb + i of channel 16 tile + n.
template <int BITS> struct VGeom {
    static constexpr int kWpt = v_words_per_tile(BITS);
    static constexpr int kWords = 8 * kWpt;            // a lane's words of a superblock
};
template <int BITS>
__device__ __forceinline__ void value_whole(const Fields<BITS>& f, const uint32_t (&w)[VGeom<BITS>::kWords], int tile, int odd, h2v* c) {
    if constexpr (BITS == 8) f.eight(w[2 * tile], w[2 * tile + 1], c);
    else if constexpr (BITS == 4) f.eight(w[tile], 0u, c);
    else if constexpr (BITS == 2) f.eight(w[tile] >> (8 * odd), 0u, c);
}

}  // namespace

struct TreeArgs {
    const uint16_t* q;        // [B*Hkv, R, D]
    const uint32_t* k_codes;
    const uint32_t* v_codes;
    const uint16_t* k_scale;
    const uint16_t* k_zero;
    const uint16_t* v_scale;
    const uint16_t* v_zero;
    const uint16_t* tail_k;
    const uint16_t* tail_v;
    const uint16_t* k_new;    // [B*Hkv, N, D]
    const uint16_t* v_new;
    const uint32_t* mask;     // [B or 1, N, mask_words], or NULL: row i sees new tokens 0 .. i
    unsigned int* arrivals;   // [heads * row_blocks] at the head of the workspace, zero between launches
    float* part;              // per (head, row block): [splits][8 RT][64] float4 of outputs, then [splits][16 RT] (reference, sum)
    uint16_t* out;            // [B*Hkv, R, D]
    float* lse;               // [B*Hkv, R] (read by the weights kernel), or NULL
    float* weights;           // [B*Hkv, w_cap]
    const int32_t* head_n_kept;
    size_t mask_stride;       // words from one batch item's mask to the next
    long long w_cap;
    int n_kept, n_cap, tail_len, tail_cap;
    int heads, n_kv_heads;
    int rows, n_new;          // R, N
    int row_blocks, n_splits, n_waves;
    bool once;                // loads go round the memory-side cache (rows_once)
    int units_per_wg;         // weights: blocks of 32 tokens of a workgroup
    int group_log2;           // G = 32, 64 or 128
    float sm_scale, decay;
};

namespace {

// Tokens of one head, cut to the launch's bound so that no value found in memory leads a load past the buffers.
__device__ __forceinline__ int head_tokens(const TreeArgs& a, int bh) {
    if (!a.head_n_kept) return a.n_kept;
    const int n = a.head_n_kept[bh];
    return n < 0 ? 0 : (n > a.n_kept ? a.n_kept : n);
}

// ---- query rows in LDS ----
// Row tile rt, step s: lane (n, kb) finds channels 32 kb + 8 s .. + 7 of row 16 rt + n at [(4 rt + s) * 64 + lane].
template <int RT> struct QueryTiles {
    uint4 frag[RT * 4 * 64];
    uint32_t sums[RT * 64];       // per (row, kb): the sum of the row's 32 channels as binary16 hi, lo
    float factor[RT * 16];        // 2^-k of a row that was scaled by 2^k
};
// A thread's share of the rows row0 .. row0 + 16 RT - 1 of one head, eight channels each (zeros past the head's last row): requested first ...
template <int RT> struct QueryPieces { uint4 w[RT]; };        // (at least 256 threads)
template <int RT>
__device__ __forceinline__ QueryPieces<RT> request_queries(const TreeArgs& a, int bh, int row0) {
    QueryPieces<RT> p;
    const int per = blockDim.x >> 4;
#pragma unroll
    for (int j = 0; j < RT; ++j) {
        const int r = (threadIdx.x >> 4) + j * per;
        p.w[j] = make_uint4(0u, 0u, 0u, 0u);
        if (r < 16 * RT && row0 + r < a.rows) p.w[j] = *reinterpret_cast<const uint4*>(a.q + ((size_t)bh * a.rows + row0 + r) * kHeadDim + 8 * (threadIdx.x & 15));
    }
    return p;
}
// ... and, behind whatever else the caller has requested meanwhile, put into LDS.
template <int RT>
__device__ __forceinline__ void stage_queries(const QueryPieces<RT>& p, QueryTiles<RT>& sq) {
    const int seg = threadIdx.x & 15, per = blockDim.x >> 4;
#pragma unroll
    for (int j0 = 0; j0 < RT; ++j0) {
        const int r = (threadIdx.x >> 4) + j0 * per;
        if (r >= 16 * RT) break;
        const uint32_t u[4] = {p.w[j0].x, p.w[j0].y, p.w[j0].z, p.w[j0].w};
        float x[8], top = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = half_to_float((uint16_t)(u[j] & 0xffffu)); x[2 * j + 1] = half_to_float((uint16_t)(u[j] >> 16));
            top = fmaxf(top, fmaxf(fabsf(x[2 * j]), fabsf(x[2 * j + 1])));
        }
        top = row16_max(top);
        // (a power of two, so nothing is rounded that matters: the largest element becomes 64 .. 128)
        const int k = top > 0.0f ? 133 - (int)((__float_as_uint(top) >> 23) & 0xffu) : 0;
        const float up = __uint_as_float((uint32_t)(127 + k) << 23);
        Frag f;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] *= up; x[2 * j + 1] *= up;
            f.h[j] = h2v{(_Float16)x[2 * j], (_Float16)x[2 * j + 1]};
            sum += (float)f.h[j][0] + (float)f.h[j][1];
        }
        sum += dpp<kQuadXor1>(sum); sum += dpp<kQuadXor2>(sum);
        const int rt = r >> 4, n = r & 15, kb = seg >> 2;
        sq.frag[(4 * rt + (seg & 3)) * 64 + kb * 16 + n] = f.q;
        if ((seg & 3) == 0) {
            const _Float16 hi = (_Float16)sum, lo = (_Float16)(sum - (float)hi);
            sq.sums[rt * 64 + kb * 16 + n] = as_u32(h2v{hi, lo});
        }
        if (seg == 0) sq.factor[r] = __uint_as_float((uint32_t)(127 - k) << 23);
    }
}

// ---- keys of a block: what a wave holds of 32 tokens, two tiles of 16 ----
// One wave's private LDS: the block's scale rows, one request per row and wave, read back where they are needed.
struct __align__(16) ScaleStrip {
    uint32_t k_scale[64];                    // per channel: one group's row
    uint32_t v_scale[64], v_zero[64];        // [group of channels][kb][i][H]
};

template <int BITS, int AXIS> struct KeyWords {
    uint32_t w[2][BITS];
    uint32_t scale[2], zero[2];      // keys per channel: a dword of the group's scales; per token: the lane's own group of its two tokens
};
// Where a head's packed arrays begin.  A block's address is the same for the whole wave (scalar registers); a lane adds 32 bits that never change.
struct HeadBase { const char *k, *v, *ks, *kz, *vs, *vz; };
__device__ __forceinline__ size_t uniform(size_t x) {
    return (size_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x) | (size_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(x >> 32)) << 32;
}
template <int BITS, int AXIS>
__device__ __forceinline__ HeadBase head_base(const TreeArgs& a, int bh) {
    constexpr int SB = v_superblock(BITS), SBW = v_superblock_words(BITS);
    HeadBase h;
    h.k = reinterpret_cast<const char*>(a.k_codes) + uniform((size_t)bh * a.n_cap * (kHeadDim * BITS / 8));
    h.v = reinterpret_cast<const char*>(a.v_codes) + uniform((size_t)bh * (size_t)((a.n_cap + SB - 1) / SB) * (SBW * 4));
    const size_t per_token = uniform((size_t)bh * a.n_cap << (8 - a.group_log2));      // bytes: D / G numbers a token
    const size_t per_group = uniform((size_t)bh * (size_t)((a.n_cap + (1 << a.group_log2) - 1) >> a.group_log2) * (kHeadDim * 2));
    const size_t key = AXIS == KVQP_KEY_PER_CHANNEL ? per_group : per_token;
    h.ks = reinterpret_cast<const char*>(a.k_scale) + key;
    h.kz = reinterpret_cast<const char*>(a.k_zero) + key;
    h.vs = reinterpret_cast<const char*>(a.v_scale) + per_token;
    h.vz = reinterpret_cast<const char*>(a.v_zero) + per_token;
    return h;
}
// ONCE: data that goes round the memory-side cache (32 layers of 8192 tokens, 16 rows: 74.9 -> 68.7 us at 4 bits, 116 -> 105 at 8; caches that
// are still there from the last call, 68 MB: 19 -> 23).  Keys of 16 bits never do: a lane's piece of a row takes four loads, a quarter of a line each.
template <typename T, bool ONCE = false> __device__ __forceinline__ T load_at(const char* uniform, uint32_t lane_bytes) {
    if constexpr (ONCE) {
        typedef uint32_t V __attribute__((ext_vector_type(sizeof(T) / 4)));
        union { V v; T t; } c;
        c.v = __builtin_nontemporal_load(reinterpret_cast<const V*>(uniform + lane_bytes));
        return c.t;
    } else {
        return *reinterpret_cast<const T*>(uniform + lane_bytes);
    }
}
// (unseen, or the compiler adds it to the head's address before the loop, 64 bits per lane and array, and a block's to that)
__device__ __forceinline__ uint32_t unseen(uint32_t lane_bytes) { asm volatile("" : "+v"(lane_bytes)); return lane_bytes; }

template <int BITS, int AXIS, bool ONCE>
__device__ __forceinline__ void load_keys(const HeadBase& h, int group_log2, int blk, int lane, KeyWords<BITS, AXIS>& k) {
    const int n = lane & 15, kb = lane >> 4;
    const char* p = h.k + (size_t)blk * (32 * kHeadDim * BITS / 8);
    const uint32_t off = unseen((uint32_t)(n * (kHeadDim * BITS / 8) + kb * (4 * BITS)));
#pragma unroll
    for (int H = 0; H < 2; ++H) {
        const char* pH = p + H * (16 * kHeadDim * BITS / 8);
        if constexpr (BITS == 2) {
            const uint2 u = load_at<uint2, ONCE>(pH, off);
            k.w[H][0] = u.x; k.w[H][1] = u.y;
        } else {
#pragma unroll
            for (int j = 0; j < BITS / 4; ++j) {
                const uint4 u = load_at<uint4, ONCE && BITS != 16>(pH + 16 * j, off);
                k.w[H][4 * j] = u.x; k.w[H][4 * j + 1] = u.y; k.w[H][4 * j + 2] = u.z; k.w[H][4 * j + 3] = u.w;
            }
        }
    }
    if constexpr (BITS != 16) {
        if constexpr (AXIS == KVQP_KEY_PER_CHANNEL) {
            const size_t row = (size_t)((32 * blk) >> group_log2) * (kHeadDim * 2);
            const uint32_t at = unseen(4u * lane);
            k.scale[0] = load_at<uint32_t>(h.ks + row, at);
        } else {
            const size_t row = (size_t)blk << (13 - group_log2);         // 32 tokens of 256 / G bytes
            const uint32_t at = unseen((uint32_t)((n << (7 - group_log2)) + ((32 * kb) >> group_log2)) * 2u);
#pragma unroll
            for (int H = 0; H < 2; ++H) {
                const size_t half = (size_t)H << (12 - group_log2);
                k.scale[H] = load_at<uint16_t>(h.ks + row + half, at);
                k.zero[H] = load_at<uint16_t>(h.kz + row + half, at);
            }
        }
    }
}

// With two or four row tiles the compiler forms operands far ahead and spills them; nothing moves across the end of a step then.  (A spilled
// register's reload waits for every load in flight: 32 layers of 8192 tokens, 64 rows: 306 -> 165 us.  Spreading vector instructions evenly
// between the matrix instructions, by hand or by s_setprio, changed nothing.)
template <int RT> __device__ __forceinline__ void end_step() { if constexpr (RT >= 2) __builtin_amdgcn_sched_barrier(0); }

// Keys per channel: q . z of the key groups of the wave's next sixteen blocks (blk, blk + step, ... , none beyond last), by one product of sixteen
// rows of zeros instead of one row sixteen times: bias[j][row] for the j-th of them.  (A product per block: 4 of 36 matrix instructions a row tile;
// 32 layers of 8192 tokens, 32 rows: 100.6 us with them, 97.5 without.)
constexpr int kBiasBlocks = 16;
template <int RT>
__device__ __forceinline__ void refresh_bias(const HeadBase& h, int group_log2, int blk, int step, int last, int lane, const uint4* frag, float* bias) {
    const int n = lane & 15, kb = lane >> 4;
    const char* row = h.kz + (size_t)((32 * min(blk + n * step, last)) >> group_log2) * (kHeadDim * 2) + 64 * kb;
    Frag z[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) z[s].q = *reinterpret_cast<const uint4*>(row + 16 * s);
    lds_order();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        f4v az = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            Frag q;
            q.q = frag[(4 * rt + s) * 64 + lane];
            az = mfma(z[s], q, az);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) bias[(4 * kb + i) * (16 * RT) + 16 * rt + n] = az[i];
    }
    lds_order();
}

// Scales that would take a product out of binary16's range: 0x8000 in each half of two scales that is LIMIT (its bits) or more.  (They are not
// negative: the sum's sign bit says it.)
template <uint32_t LIMIT> __device__ __forceinline__ uint32_t wide_bits(uint32_t scales) { return (scales + (0x8000u - LIMIT) * 0x10001u) & 0x80008000u; }
__device__ __forceinline__ bool any(bool mine) { return __builtin_amdgcn_ballot_w64(mine) != 0ull; }
__device__ __forceinline__ uint32_t scaled(uint32_t two, float by) { return as_u32(as_h2(two) * splat(by)); }
// Keys: 256 and more (255 codes, and 128 q's, times less stay below 65504).  They are left out of a block's product and get another one, kWide
// taken from the scale and given to the other operand, so that the small ones beside them lose nothing.  (Almost no block has any; looking for
// them, here and among the values, takes six instructions of some five hundred.)
constexpr uint32_t kWideKey = 0x5C00u;
constexpr float kWide = 256.0f;
// Values: where the highest code times the scale would pass 65504; the block's scales and zeros are quartered then, and with them, for the time
// being, the outputs so far.
template <int BITS> constexpr uint32_t kWideValue = BITS == 2 ? 0x7400u : BITS == 4 ? 0x6C00u : 0x5C00u;       // 16384, 4096, 256

// Makes a block's key scales ready for the product: the wide ones are taken out and returned, times 1 / kWide (the others' places: 0); keys
// per channel: the rest goes to the strip, whence every lane reads its 32 channels.
template <int BITS, int AXIS>
__device__ __forceinline__ uint32_t ready_keys(KeyWords<BITS, AXIS>& k, ScaleStrip& strip, int lane, bool& wide) {
    wide = false;
    uint32_t out = 0u;
    if constexpr (BITS != 16) {
        constexpr bool kChannel = AXIS == KVQP_KEY_PER_CHANNEL;
        uint32_t two = kChannel ? k.scale[0] : k.scale[0] | k.scale[1] << 16;
        const uint32_t bits = wide_bits<kWideKey>(two);
        wide = any(bits != 0u);
        if (wide) {
            const uint32_t mask = (bits >> 15) * 0xFFFFu;
            out = scaled(two & mask, 1.0f / kWide);
            two &= ~mask;
            if constexpr (kChannel) k.scale[0] = two;
            else { k.scale[0] = two & 0xFFFFu; k.scale[1] = two >> 16; }
        }
        if constexpr (kChannel) {
            lds_order();
            strip.k_scale[lane] = k.scale[0];
            lds_order();
        }
    }
    return out;
}
// Logits of a block for RT row tiles, before the rows' factors (and, keys per channel, without q . z): acc[rt][H][i] is token 16 H + 4 kb + i of row 16 rt + n.  The four
// steps of eight channels run outermost, so that only one step's operands are held beside the sums.  WIDE: those of scales taken by 1 / kWide, added to acc.
template <int BITS, int AXIS, int RT, bool WIDE>
__device__ __forceinline__ void key_products(const Fields<BITS>& fields, const KeyWords<BITS, AXIS>& k, const uint4* frag, const uint32_t* sums, ScaleStrip& strip, int lane, f4v (&acc)[RT][2]) {
    constexpr bool kChannel = BITS != 16 && AXIS == KVQP_KEY_PER_CHANNEL, kToken = BITS != 16 && AXIS == KVQP_KEY_PER_TOKEN;
    constexpr bool kCodes = kChannel && RT <= 2;       // codes by themselves are an operand
    const int kb = lane >> 4;
    auto query = [&](int rt, int s) {
        Frag q;
        q.q = frag[(4 * rt + s) * 64 + lane];
        if constexpr (WIDE && !kCodes)
#pragma unroll
            for (int r = 0; r < 4; ++r) q.h[r] *= splat(kWide);
        return q;
    };
    if constexpr (!WIDE)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[rt][0] = acc[rt][1] = f4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        end_step<RT>();
        Frag a[2];
        if constexpr (BITS == 16) {
#pragma unroll
            for (int H = 0; H < 2; ++H)
#pragma unroll
                for (int r = 0; r < 4; ++r) a[H].u[r] = k.w[H][4 * s + r];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const Frag q = query(rt, s);
                acc[rt][0] = mfma(a[0], q, acc[rt][0]); acc[rt][1] = mfma(a[1], q, acc[rt][1]);
            }
        } else if constexpr (kChannel) {
            Frag sc;
            sc.q = *reinterpret_cast<const uint4*>(&strip.k_scale[16 * kb + 4 * s]);
#pragma unroll
            for (int H = 0; H < 2; ++H) {
                key_whole<BITS>(fields, k.w[H], s, a[H].h);
                if constexpr (WIDE && kCodes)
#pragma unroll
                    for (int r = 0; r < 4; ++r) a[H].h[r] *= splat(kWide);
            }
            if constexpr (kCodes) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const Frag q = query(rt, s);
                    Frag hi, lo;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        hi.h[r] = q.h[r] * sc.h[r];
                        lo.h[r] = __builtin_elementwise_fma(q.h[r], sc.h[r], -hi.h[r]);
                    }
                    acc[rt][0] = mfma(a[0], hi, acc[rt][0]); acc[rt][1] = mfma(a[1], hi, acc[rt][1]);
                    acc[rt][0] = mfma(a[0], lo, acc[rt][0]); acc[rt][1] = mfma(a[1], lo, acc[rt][1]);
                }
            } else {
                // (Four tiles of rows: the codes take the scales, which are two tiles.  32 layers of 8192 tokens, 64 rows: 162.5 -> 158.5 us, their
                // weights 95.3 -> 88.8.)
                Frag b[2];
#pragma unroll
                for (int H = 0; H < 2; ++H)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const h2v c = a[H].h[r];
                        a[H].h[r] = c * sc.h[r];
                        b[H].h[r] = __builtin_elementwise_fma(c, sc.h[r], -a[H].h[r]);
                    }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const Frag q = query(rt, s);
                    acc[rt][0] = mfma(a[0], q, acc[rt][0]); acc[rt][1] = mfma(a[1], q, acc[rt][1]);
                    acc[rt][0] = mfma(b[0], q, acc[rt][0]); acc[rt][1] = mfma(b[1], q, acc[rt][1]);
                }
            }
        } else if constexpr (kToken) {
            Frag b[2];
#pragma unroll
            for (int H = 0; H < 2; ++H) {
                const h2v sc = as_h2(k.scale[H] * 0x10001u);
                h2v c[4];
                key_whole<BITS>(fields, k.w[H], s, c);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    a[H].h[r] = c[r] * sc;
                    b[H].h[r] = __builtin_elementwise_fma(c[r], sc, -a[H].h[r]);
                }
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const Frag q = query(rt, s);
                acc[rt][0] = mfma(a[0], q, acc[rt][0]); acc[rt][1] = mfma(a[1], q, acc[rt][1]);
                acc[rt][0] = mfma(b[0], q, acc[rt][0]); acc[rt][1] = mfma(b[1], q, acc[rt][1]);
            }
        }
    }
    if constexpr (kToken && !WIDE) {
        Frag z[2];
#pragma unroll
        for (int H = 0; H < 2; ++H) { z[H].u[0] = k.zero[H] * 0x10001u; z[H].u[1] = z[H].u[2] = z[H].u[3] = 0u; }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            Frag qs;
            qs.u[0] = sums[rt * 64 + lane]; qs.u[1] = qs.u[2] = qs.u[3] = 0u;
            acc[rt][0] = mfma(z[0], qs, acc[rt][0]); acc[rt][1] = mfma(z[1], qs, acc[rt][1]);
        }
    }
}

// The same from a block's keys as they were loaded.
template <int BITS, int AXIS, int RT>
__device__ __forceinline__ void key_product(const Fields<BITS>& fields, KeyWords<BITS, AXIS>& k, const uint4* frag, const uint32_t* sums, ScaleStrip& strip, int lane, f4v (&acc)[RT][2]) {
    bool wide;
    const uint32_t wide_scales = ready_keys<BITS, AXIS>(k, strip, lane, wide);
    key_products<BITS, AXIS, RT, false>(fields, k, frag, sums, strip, lane, acc);
    if constexpr (BITS != 16)
        if (wide) {
            // (unseen, or the unpacked codes stay in registers from the first product on, and others spill)
#pragma unroll
            for (int H = 0; H < 2; ++H)
#pragma unroll
                for (uint32_t& w : k.w[H]) asm volatile("" : "+v"(w));
            if constexpr (AXIS == KVQP_KEY_PER_CHANNEL) {
                lds_order();
                strip.k_scale[lane] = wide_scales;
                lds_order();
            } else {
                k.scale[0] = wide_scales & 0xFFFFu; k.scale[1] = wide_scales >> 16;
            }
            key_products<BITS, AXIS, RT, true>(fields, k, frag, sums, strip, lane, acc);
        }
}

// ---- state of a wave's rows ----
template <int RT> struct RowState {
    f4v o[RT][8];          // O^T: channel 16 tile + 4 kb + i of row 16 rt + n
    // Below 16 bits, the packed tokens' zeros' share: channels 32 i .. + 31 of row 16 rt + n, the same in its four lanes.  With four tiles of rows
    // lane kb has tile kb's alone, or others spill (16384 tokens, 256 rows: 61.4 us with one for each, 56.0 so; two tiles, 32 layers of 8192 tokens:
    // 110.6 with one for each, 112.5 so).
    f4v z[RT <= 2 ? RT : 1];
    float ref[RT], sum[RT];
};
template <int RT>
__device__ __forceinline__ void clear(RowState<RT>& st) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        st.ref[rt] = kNegBig; st.sum[rt] = 0.f;
#pragma unroll
        for (int t = 0; t < 8; ++t) st.o[rt][t] = f4v{0.f, 0.f, 0.f, 0.f};
    }
    for (f4v& z : st.z) z = f4v{0.f, 0.f, 0.f, 0.f};
}
// (outputs alone)
template <int RT>
__device__ __forceinline__ void rescale(RowState<RT>& st, float by) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int c = 0; c < 8; ++c) st.o[rt][c] *= by;
    for (f4v& z : st.z) z *= by;
}
// Moves references where logits have passed them, turns acc + bias (a block's logits before the rows' factors, -inf where unseen) into weights x
// and adds them up.
template <int RT>
__device__ __forceinline__ void softmax_step(RowState<RT>& st, const f4v (&acc)[RT][2], const float (&factor)[RT], const float (&bias)[RT], float (&x)[RT][8]) {
    bool past = false;
    float top[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const f4v &p = acc[rt][0], &q = acc[rt][1];
        top[rt] = (higher(higher(higher(p[0], p[1]), higher(p[2], p[3])), higher(higher(q[0], q[1]), higher(q[2], q[3]))) + bias[rt]) * factor[rt];
        past |= top[rt] > st.ref[rt] + kSlack;
    }
    if (__builtin_amdgcn_ballot_w64(past) != 0ull) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float t = rows4_max(top[rt]);          // (all four lanes of a row decide alike)
            const float ref = t > st.ref[rt] + kSlack ? t - kBoost : st.ref[rt];
            const float f = __builtin_amdgcn_exp2f(st.ref[rt] - ref);
            st.ref[rt] = ref;
            st.sum[rt] *= f;
#pragma unroll
            for (int c = 0; c < 8; ++c) st.o[rt][c] *= f;
            if constexpr (RT <= 2) st.z[rt] *= f;
            else if (rt == (int)(threadIdx.x >> 4 & 3)) st.z[0] *= f;
        }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float add = __builtin_fmaf(bias[rt], factor[rt], -st.ref[rt]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[rt][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[rt][j >> 2][j & 3], factor[rt], add));
            st.sum[rt] += x[rt][j];
        }
        asm("" : "+v"(st.sum[rt]));       // (or the compiler adds up behind the products, and keeps 8 RT weights in registers until then)
    }
}
// Weights as operands: pair i holds tokens 4 kb + i and 16 + 4 kb + i; hi + lo parts, cut toward zero.
struct WeightOperand { Frag hi, lo; };
// (minus is -1 that the compiler does not know: the widening and the exact subtraction are one v_fma_mix_f32)
__device__ __forceinline__ void weight_operand(const float (&p)[8], float minus, WeightOperand& o) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o.hi.u[i] = pack_rtz(p[i], p[4 + i]);
        o.lo.u[i] = pack_rtz(__builtin_fmaf((float)o.hi.h[i][0], minus, p[i]), __builtin_fmaf((float)o.hi.h[i][1], minus, p[4 + i]));
    }
}
template <int RT>
__device__ __forceinline__ void value_product(RowState<RT>& st, const Frag& v, int tile, const WeightOperand (&p)[RT]) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) st.o[rt][tile] = mfma(v, p[rt].hi, st.o[rt][tile]);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) st.o[rt][tile] = mfma(v, p[rt].lo, st.o[rt][tile]);
}

// ---- values of a packed block ----
template <int BITS> struct ValueWords {
    uint32_t w[VGeom<BITS>::kWords];
    uint32_t scale, zero;
};
template <int BITS, bool ONCE>
__device__ __forceinline__ void load_values(const HeadBase& h, int group_log2, int blk, int lane, ValueWords<BITS>& v) {
    constexpr int SB = v_superblock(BITS), SBW = v_superblock_words(BITS);
    const char* p = h.v + (size_t)(32 * blk / SB) * (SBW * 4);
    const uint32_t at_lane = unseen(16u * lane);
#pragma unroll
    for (int j = 0; j < VGeom<BITS>::kWords / 4; ++j) {
        const uint4 u = load_at<uint4, ONCE>(p + 1024 * j, at_lane);
        v.w[4 * j] = u.x; v.w[4 * j + 1] = u.y; v.w[4 * j + 2] = u.z; v.w[4 * j + 3] = u.w;
    }
    if constexpr (BITS != 16) {
        // 32 tokens' scales are 32 D / G numbers in a row; lanes past the last repeat it
        const size_t row = (size_t)blk << (13 - group_log2);
        const uint32_t at = unseen(4u * min(lane, (16 << (7 - group_log2)) - 1));
        v.scale = load_at<uint32_t>(h.vs + row, at);
        v.zero = load_at<uint32_t>(h.vz + row, at);
    }
}
// Scales and zeros to the strip, in the order in which the lanes of a token's block want them.
template <int BITS>
__device__ __forceinline__ void strip_values(const TreeArgs& a, const ValueWords<BITS>& v, ScaleStrip& strip, int lane) {
    const int cg_log2 = 7 - a.group_log2;
    uint16_t* s = reinterpret_cast<uint16_t*>(strip.v_scale);
    uint16_t* z = reinterpret_cast<uint16_t*>(strip.v_zero);
    lds_order();
    if (lane < 16 << cg_log2) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int t = (2 * lane + e) >> cg_log2, g = (2 * lane + e) & ((1 << cg_log2) - 1);
            const int at = g * 32 + (t & 15) * 2 + (t >> 4);
            s[at] = (uint16_t)(v.scale >> (16 * e));
            z[at] = (uint16_t)(v.zero >> (16 * e));
        }
    }
    lds_order();
}

// ---- plain rows (tail, drafted tokens) ----
constexpr int kPlainStride = kHeadDim + 8;      // halves between two rows of a value tile in LDS
struct __align__(16) PlainTile { uint16_t v[32 * kPlainStride]; };

// A workgroup's LDS: while blocks are worked on, and while the waves' states become one (outputs of JOIN row tiles at a time).
template <int RT> union WaveScratch { struct { ScaleStrip strip; float bias[kBiasBlocks * 16 * RT]; } packed; PlainTile tile; };
constexpr int kMostSplits = 64;
constexpr int join_tiles(int rt) { return rt == 4 ? 2 : 1; }
template <int RT> union __align__(16) TreeShared {
    struct { QueryTiles<RT> sq; WaveScratch<RT> wave[most_waves(RT)]; } run;
    struct { f4v o[most_waves(RT)][join_tiles(RT) * 8][64]; float ref[most_waves(RT)][16 * RT], sum[most_waves(RT)][16 * RT]; } join;
    struct { float weight[kMostSplits][16 * RT], sum[kMostSplits][16 * RT], inverse[16 * RT]; } last;       // of a row block's splits
};
// One row block's partial results in the workspace, written and read with accesses at device scope (sc1): workgroups of one row block
// run on different dies, whose L2 caches do not see each other within a launch.
constexpr int kDeviceScope = 16;      // sc1 in a buffer access' cache policy
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
template <int I> struct IntC { static constexpr int value = I; };
struct Partials {
    __amdgpu_buffer_rsrc_t at;
    int states, rt;                   // where references and sums begin
    __device__ __forceinline__ Partials(const TreeArgs& a, int group, int rt_) : states(a.n_splits * rt_ * 8192), rt(rt_) {
        const int bytes = states + a.n_splits * rt_ * 128;
        at = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>(a.part) + (size_t)group * bytes, 0, bytes, 0x00020000);
    }
    __device__ __forceinline__ void put_output(int split, int item, f4v o) const {
        u4v v = {__float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]), __float_as_uint(o[3])};
        __builtin_amdgcn_raw_buffer_store_b128(v, at, (split * rt * 512 + item) * 16, 0, kDeviceScope);
    }
    __device__ __forceinline__ void put_state(int split, int row, float ref, float sum) const {
        u2v v = {__float_as_uint(ref), __float_as_uint(sum)};
        __builtin_amdgcn_raw_buffer_store_b64(v, at, states + (split * rt * 16 + row) * 8, 0, kDeviceScope);
    }
    __device__ __forceinline__ f4v output(int split, int item) const {
        const u4v v = __builtin_amdgcn_raw_buffer_load_b128(at, (split * rt * 512 + item) * 16, 0, kDeviceScope);
        return f4v{__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3])};
    }
    __device__ __forceinline__ float2 state(int split, int row) const {
        const u2v v = __builtin_amdgcn_raw_buffer_load_b64(at, states + (split * rt * 16 + row) * 8, 0, kDeviceScope);
        return make_float2(__uint_as_float(v[0]), __uint_as_float(v[1]));
    }
};
__device__ __forceinline__ uint2 halves_of(const f4v& o, float by) {
    Frag h;
    h.h[0] = h2v{(_Float16)(o[0] * by), (_Float16)(o[1] * by)};
    h.h[1] = h2v{(_Float16)(o[2] * by), (_Float16)(o[3] * by)};
    return make_uint2(h.u[0], h.u[1]);
}
// (a row that sees nothing: zeros, and minus infinity)
__device__ __forceinline__ float inverse_sum(float sum) { return sum > 0.0f ? 1.0f / sum : sum; }
__device__ __forceinline__ float log_sum(float ref, float sum) { return sum == 0.0f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * kLn2; }

template <int BITS, int AXIS, int RT, bool ONCE>
__global__ __launch_bounds__(64 * most_waves(RT), most_waves(RT) / 4) void tree_attn(const TreeArgs a) {
    __shared__ TreeShared<RT> sh;
    __shared__ int s_last;
    QueryTiles<RT>& sq = sh.run.sq;

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, kb = lane >> 4, waves = blockDim.x >> 6;
    // Workgroups go to the eight dies in turn: the row blocks of one stretch of a cache get numbers eight apart, so that
    // they run on one die at about the same time and share what its L2 holds.
    const int pair = __builtin_amdgcn_readfirstlane(blockIdx.x / (8 * a.row_blocks) * 8 + blockIdx.x % 8), rb = __builtin_amdgcn_readfirstlane(blockIdx.x / 8 % a.row_blocks);
    if (pair >= a.heads * a.n_splits) return;
    const int bh = __builtin_amdgcn_readfirstlane(pair / a.n_splits), split = pair - bh * a.n_splits;
    const int row0 = rb * RT * 16;
    // (loads return in order: the queries first, then the wave's first block, which is on its way while they are put into LDS)
    const QueryPieces<RT> pieces = request_queries<RT>(a, bh, row0);

    const int n_tok = __builtin_amdgcn_readfirstlane(head_tokens(a, bh));
    const int packed = (n_tok + 31) / 32, tail = (a.tail_len + 31) / 32, fresh = (a.n_new + 31) / 32;
    const int units = packed + tail + fresh;
    const int share = __builtin_amdgcn_readfirstlane((int)((unsigned)units / (unsigned)a.n_splits)), rest = units - share * a.n_splits;
    const int u0 = share * split + min(split, rest), u1 = u0 + share + (split < rest ? 1 : 0);
    const int end = min(u1, packed);
    int blk = u0 + wave;
    const HeadBase base = head_base<BITS, AXIS>(a, bh);
    KeyWords<BITS, AXIS> kw;
    ValueWords<BITS> vw;
    if (blk < end) {
        load_keys<BITS, AXIS, ONCE>(base, a.group_log2, blk, lane, kw);
        load_values<BITS, ONCE>(base, a.group_log2, blk, lane, vw);
    }
    stage_queries<RT>(pieces, sq);
    ScaleStrip& strip = sh.run.wave[wave].packed.strip;
    float* biases = sh.run.wave[wave].packed.bias;

    RowState<RT> st;
    clear(st);
    float minus = -1.0f;
    asm("" : "+s"(minus));
    __syncthreads();
    const float c_q = a.sm_scale * kLog2e;
    float factor[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) factor[rt] = fmaxf(sq.factor[16 * rt + n] * c_q, 1.2e-38f);      // (above 0, for the -inf of unseen tokens)

    // ---- packed blocks ----
    {
        const Fields<BITS> fields;
        int turn = 0;
        if (blk < end) {
#pragma unroll 1
            for (; blk < end; blk += waves) {
                const int next = min(blk + waves, end - 1);
                f4v acc[RT][2];
                float bias[RT] = {};
                if constexpr (BITS != 16 && AXIS == KVQP_KEY_PER_CHANNEL) {
                    if (turn == 0) refresh_bias<RT>(base, a.group_log2, blk, waves, end - 1, lane, sq.frag, biases);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) bias[rt] = biases[turn * (16 * RT) + 16 * rt + n];
                    turn = (turn + 1) % kBiasBlocks;
                }
                key_product<BITS, AXIS, RT>(fields, kw, sq.frag, sq.sums, strip, lane, acc);
                load_keys<BITS, AXIS, ONCE>(base, a.group_log2, next, lane, kw);
                if (32 * blk + 32 > n_tok) {     // (uniform) the head's last block: tokens past its count are unseen
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (32 * blk + 16 * (j >> 2) + 4 * kb + (j & 3) >= n_tok) acc[rt][j >> 2][j & 3] = -INFINITY;
                }
                float x[RT][8];
                softmax_step<RT>(st, acc, factor, bias, x);
                bool wide = false;
                if constexpr (BITS != 16) {
                    wide = any(wide_bits<kWideValue<BITS>>(vw.scale) != 0u);
                    if (wide) {
                        vw.scale = scaled(vw.scale, 0.25f); vw.zero = scaled(vw.zero, 0.25f);
                        rescale<RT>(st, 0.25f);
                    }
                }
                WeightOperand p[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) weight_operand(x[rt], minus, p[rt]);
                if constexpr (BITS != 16) strip_values<BITS>(a, vw, strip, lane);
                if constexpr (BITS != 16) {
                    // (lane n has the zeros of the group that channel 32 (n % 4) is in)
                    Frag z;
                    z.q = *reinterpret_cast<const uint4*>(&strip.v_zero[16 * ((32 * (n & 3)) >> a.group_log2) + 4 * kb]);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        const f4v sums = mfma(z, p[rt].lo, mfma(z, p[rt].hi, RT <= 2 ? st.z[RT <= 2 ? rt : 0] : f4v{0.f, 0.f, 0.f, 0.f}));
                        if constexpr (RT <= 2) st.z[rt] = sums;
                        else if (rt == kb) st.z[0] += sums;
                    }
                }
                Frag s;
#pragma unroll
                for (int tile = 0; tile < 8; ++tile) {
                    Frag v;
                    if constexpr (BITS == 16) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) v.u[i] = vw.w[4 * tile + i];
                    } else {
                        Frag lo;
                        h2v c[4];
                        value_whole<BITS>(fields, vw.w, tile, blk & 1, c);
                        if ((tile & 1) == 0) {       // (a group has at least two tiles)
                            const int g = (16 * tile) >> a.group_log2;
                            s.q = *reinterpret_cast<const uint4*>(&strip.v_scale[16 * g + 4 * kb]);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            v.h[i] = c[i] * s.h[i];
                            lo.h[i] = __builtin_elementwise_fma(c[i], s.h[i], -v.h[i]);
                        }
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) st.o[rt][tile] = mfma(lo, p[rt].hi, st.o[rt][tile]);
                    }
                    value_product<RT>(st, v, tile, p);
                    if (tile & 1) end_step<RT>();
                }
                if (wide) rescale<RT>(st, 4.0f);
                load_values<BITS, ONCE>(base, a.group_log2, next, lane, vw);
            }
            if constexpr (BITS != 16)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float z = RT <= 2 ? st.z[RT <= 2 ? rt : 0][i] : __shfl(st.z[0][i], 16 * rt + n);
                        st.o[rt][2 * i] += z; st.o[rt][2 * i + 1] += z;
                    }
        }
    }

    // ---- tail rows and drafted tokens ----
    {
        PlainTile& tile_v = sh.run.wave[wave].tile;
        const int first = max(u0, packed);
#pragma unroll 1
        for (int u = first + wave; u < u1; u += waves) {
            const bool drafted = u >= packed + tail;
            const int t0 = 32 * (drafted ? u - packed - tail : u - packed), len = drafted ? a.n_new : a.tail_len;
            const size_t row = drafted ? (size_t)bh * a.n_new : (size_t)bh * a.tail_cap;
            const uint16_t* kp = (drafted ? a.k_new : a.tail_k) + row * kHeadDim;
            const uint16_t* vp = (drafted ? a.v_new : a.tail_v) + row * kHeadDim;
            KeyWords<16, KVQP_KEY_PER_CHANNEL> pk;
#pragma unroll
            for (int H = 0; H < 2; ++H) {
                const uint16_t* p = kp + (size_t)min(t0 + 16 * H + n, len - 1) * kHeadDim + 32 * kb;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint4 w = *reinterpret_cast<const uint4*>(p + 8 * j);
                    pk.w[H][4 * j] = w.x; pk.w[H][4 * j + 1] = w.y; pk.w[H][4 * j + 2] = w.z; pk.w[H][4 * j + 3] = w.w;
                }
            }
            uint4 rows[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                rows[j] = make_uint4(0u, 0u, 0u, 0u);
                if (t0 + 4 * j + kb < len) rows[j] = *reinterpret_cast<const uint4*>(vp + (size_t)(t0 + 4 * j + kb) * kHeadDim + 8 * n);
            }
            lds_order();
            bool odd_value = false;       // a value that is not finite
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t u4[4] = {rows[j].x, rows[j].y, rows[j].z, rows[j].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) odd_value |= (u4[e] & 0x7C00u) == 0x7C00u || (u4[e] & 0x7C000000u) == 0x7C000000u;
                *reinterpret_cast<uint4*>(&tile_v.v[(4 * j + kb) * kPlainStride + 8 * n]) = rows[j];
            }
            lds_order();
            f4v acc[RT][2];
            {
                key_product<16, KVQP_KEY_PER_CHANNEL, RT>(Fields<16>(), pk, sq.frag, sq.sums, strip, lane, acc);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    // which of the block's 32 tokens the row sees
                    uint32_t seen = t0 + 32 <= len ? 0xFFFFFFFFu : (1u << (len - t0)) - 1u;
                    if (drafted) {
                        const int r = row0 + 16 * rt + n;
                        const int i = r < a.rows ? r % a.n_new : 0;
                        if (a.mask) seen &= a.mask[(size_t)(bh / a.n_kv_heads) * a.mask_stride + (size_t)i * ((a.n_new + 31) / 32) + t0 / 32];
                        else seen &= i >= t0 + 31 ? 0xFFFFFFFFu : i < t0 ? 0u : (2u << (i - t0)) - 1u;
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (!((seen >> (16 * (j >> 2) + 4 * kb + (j & 3))) & 1u)) acc[rt][j >> 2][j & 3] = -INFINITY;
                }
            }
            float x[RT][8];
            const float none[RT] = {};
            softmax_step<RT>(st, acc, factor, none, x);
            WeightOperand p[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) weight_operand(x[rt], minus, p[rt]);
            if (drafted && __builtin_amdgcn_ballot_w64(odd_value) != 0ull) {
                // Values that are not finite reach only the rows that see them (a weight of 0 would make them NaN in the matrix product):
                // they are added here, one token at a time, and taken out of the tile.
#pragma unroll 1
                for (int t = 0; t < 32; ++t) {
                    const int j = 4 * (t >> 4) + (t & 3);
                    float w[RT];
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        float mine = x[rt][0];
#pragma unroll
                        for (int e = 1; e < 8; ++e) mine = j == e ? x[rt][e] : mine;
                        w[rt] = __shfl(mine, 16 * ((t >> 2) & 3) + n);
                    }
                    const uint16_t* row = &tile_v.v[t * kPlainStride + 4 * kb];
#pragma unroll
                    for (int c = 0; c < 8; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t u = row[16 * c + i];
                            const float v = (u & 0x7C00u) == 0x7C00u ? half_to_float((uint16_t)u) : 0.0f;
#pragma unroll
                            for (int rt = 0; rt < RT; ++rt) st.o[rt][c][i] += w[rt] != 0.0f ? w[rt] * v : 0.0f;
                        }
                }
                lds_order();
#pragma unroll 1
                for (int t = 0; t < 32; ++t) {
                    uint32_t* two = reinterpret_cast<uint32_t*>(&tile_v.v[t * kPlainStride + 2 * lane]);
                    const uint32_t u = *two;
                    *two = ((u & 0x7C00u) == 0x7C00u ? 0u : u & 0xFFFFu) | ((u & 0x7C000000u) == 0x7C000000u ? 0u : u & 0xFFFF0000u);
                }
                lds_order();
            }
#pragma unroll
            for (int tile = 0; tile < 8; ++tile) {
                Frag v;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t lo = tile_v.v[(4 * kb + i) * kPlainStride + 16 * tile + n], hi = tile_v.v[(16 + 4 * kb + i) * kPlainStride + 16 * tile + n];
                    v.u[i] = lo | (hi << 16);
                }
                value_product<RT>(st, v, tile, p);
            }
        }
    }

    // ---- the waves' states become one ----
    // Every wave brings its outputs to the rows' highest reference; then the threads share the sums over the waves among them, JOIN row
    // tiles at a time.  (Pairs of waves, halving their number, took 3.9 us for twelve waves of 32 rows, this 3.)
    constexpr int JOIN = join_tiles(RT);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) st.sum[rt] = rows4_add(st.sum[rt]);
    __syncthreads();
    if (kb == 0)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) { sh.join.ref[wave][16 * rt + n] = st.ref[rt]; sh.join.sum[wave][16 * rt + n] = st.sum[rt]; }
    __syncthreads();
    float ref[RT], sum[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        // (all of them requested at once; a wave that is not there repeats the first, at weight 0)
        float r[most_waves(RT)], s[most_waves(RT)];
#pragma unroll
        for (int w = 0; w < most_waves(RT); ++w) { r[w] = sh.join.ref[w < waves ? w : 0][16 * rt + n]; s[w] = sh.join.sum[w < waves ? w : 0][16 * rt + n]; }
        ref[rt] = r[0];
#pragma unroll
        for (int w = 1; w < most_waves(RT); ++w) ref[rt] = fmaxf(ref[rt], r[w]);
        sum[rt] = 0.f;
#pragma unroll
        for (int w = 0; w < most_waves(RT); ++w) sum[rt] = __builtin_fmaf(w < waves ? s[w] : 0.f, __builtin_amdgcn_exp2f(r[w] - ref[rt]), sum[rt]);
        const float f = __builtin_amdgcn_exp2f(st.ref[rt] - ref[rt]);
#pragma unroll
        for (int t = 0; t < 8; ++t) st.o[rt][t] *= f;
    }
    const Partials parts(a, bh * a.row_blocks + rb, RT);
    if (wave == 0 && kb == 0) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int r = row0 + 16 * rt + n;
            if (a.n_splits > 1) parts.put_state(split, 16 * rt + n, ref[rt], sum[rt]);
            else if (a.lse && r < a.rows) a.lse[(size_t)bh * a.rows + r] = log_sum(ref[rt], sum[rt]);
        }
    }
#pragma unroll
    for (int j0 = 0; j0 < RT; j0 += JOIN) {
        if (j0) __syncthreads();
#pragma unroll
        for (int rt = 0; rt < JOIN; ++rt)
#pragma unroll
            for (int t = 0; t < 8; ++t) sh.join.o[wave][8 * rt + t][lane] = st.o[j0 + rt][t];
        __syncthreads();
        for (int slot = wave; slot < 8 * JOIN; slot += waves) {
            f4v o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int w = 0; w < waves; w += 4) {          // (workgroups have whole fours of waves)
                f4v four[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) four[u] = sh.join.o[w + u][slot][lane];
                o += (four[0] + four[1]) + (four[2] + four[3]);
            }
            const int t = slot & 7;
            if (a.n_splits > 1) {
                parts.put_output(split, (j0 * 8 + slot) * 64 + lane, o);
            } else {
                float total = sum[j0];
#pragma unroll
                for (int rt = 1; rt < JOIN; ++rt) total = (slot >> 3) == rt ? sum[j0 + rt] : total;
                const int r = row0 + 16 * (j0 + (slot >> 3)) + n;
                if (r < a.rows) *reinterpret_cast<uint2*>(a.out + ((size_t)bh * a.rows + r) * kHeadDim + 16 * t + 4 * kb) = halves_of(o, inverse_sum(total));
            }
        }
    }
    if (a.n_splits == 1) return;

    // ---- the last workgroup of a row block to arrive joins its splits ----
    // The partials were stored past this die's L2, and the wait returns when the stores have been acknowledged from there; so whoever sees the
    // counter sees them, with loads that do not look into its own L2.
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        unsigned int* count = &a.arrivals[bh * a.row_blocks + rb];
        const unsigned before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = before == (unsigned)(a.n_splits - 1);
        if (s_last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) return;
    if constexpr (RT <= 2) {
        // A thread has its item's splits to itself, states and outputs together, four or eight at a time: what is requested
        // beyond the last split costs time too (sixteen at a time: 16.6 us where three splits take 14.4).
        auto join = [&](auto batch) {
            constexpr int BATCH = decltype(batch)::value;
#pragma unroll 1
            for (int item = threadIdx.x; item < RT * 512; item += blockDim.x) {
                const int row = 16 * (item >> 9) + n, r = row0 + row;         // (64 items of one wave: one tile of one row tile)
                float top = kNegBig, total = 0.f;
                f4v o = {0.f, 0.f, 0.f, 0.f};
                for (int s0 = 0; s0 < a.n_splits; s0 += BATCH) {
                    f4v v[BATCH];
                    float2 m[BATCH];
#pragma unroll
                    for (int u = 0; u < BATCH; ++u) {
                        const int s = min(s0 + u, a.n_splits - 1);
                        v[u] = parts.output(s, item);
                        m[u] = parts.state(s, row);
                    }
                    float higher = top;
#pragma unroll
                    for (int u = 0; u < BATCH; ++u) higher = fmaxf(higher, m[u].x);
                    const float f = __builtin_amdgcn_exp2f(top - higher);
                    o *= f; total *= f;
#pragma unroll
                    for (int u = 0; u < BATCH; ++u) {
                        const float g = s0 + u < a.n_splits ? __builtin_amdgcn_exp2f(m[u].x - higher) : 0.f;
                        o += v[u] * g;
                        total = __builtin_fmaf(m[u].y, g, total);
                    }
                    top = higher;
                }
                if (r < a.rows) {
                    *reinterpret_cast<uint2*>(a.out + ((size_t)bh * a.rows + r) * kHeadDim + 16 * ((item >> 6) & 7) + 4 * kb) = halves_of(o, inverse_sum(total));
                    if (a.lse && (item & 0x1C0) == 0 && kb == 0) a.lse[(size_t)bh * a.rows + r] = log_sum(top, total);
                }
            }
        };
        if (a.n_splits <= 4) join(IntC<4>{});
        else join(IntC<8>{});
    } else {
        // (two items a thread and eight splits of each in flight; the first of them while 16 RT threads turn the splits' states into weights)
        constexpr int ITEMS = 2;
        const int stride = blockDim.x;
#pragma unroll 1
        for (int item0 = 0; item0 < RT * 512; item0 += ITEMS * stride) {
            f4v o[ITEMS];
#pragma unroll
            for (int e = 0; e < ITEMS; ++e) o[e] = f4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int s0 = 0; s0 < a.n_splits; s0 += 8) {
                f4v v[ITEMS][8];
#pragma unroll
                for (int e = 0; e < ITEMS; ++e)
#pragma unroll
                    for (int u = 0; u < 8; ++u) v[e][u] = parts.output(min(s0 + u, a.n_splits - 1), min(item0 + e * stride + (int)threadIdx.x, RT * 512 - 1));
                if (item0 == 0 && s0 == 0) {
                    if ((int)threadIdx.x < 16 * RT) {
                        float top = kNegBig, total = 0.f;
                        for (int s1 = 0; s1 < a.n_splits; s1 += 16) {
                            float2 m[16];
#pragma unroll
                            for (int u = 0; u < 16; ++u) m[u] = parts.state(min(s1 + u, a.n_splits - 1), threadIdx.x);
#pragma unroll
                            for (int u = 0; u < 16; ++u) {
                                top = fmaxf(top, m[u].x);
                                sh.last.weight[s1 + u][threadIdx.x] = m[u].x;
                                sh.last.sum[s1 + u][threadIdx.x] = m[u].y;
                            }
                        }
                        for (int s1 = 0; s1 < a.n_splits; s1 += 16) {
                            float g[16], l[16];
#pragma unroll
                            for (int u = 0; u < 16; ++u) { g[u] = sh.last.weight[s1 + u][threadIdx.x]; l[u] = sh.last.sum[s1 + u][threadIdx.x]; }
#pragma unroll
                            for (int u = 0; u < 16; ++u) {
                                g[u] = s1 + u < a.n_splits ? __builtin_amdgcn_exp2f(g[u] - top) : 0.f;
                                total = __builtin_fmaf(s1 + u < a.n_splits ? l[u] : 0.f, g[u], total);
                                sh.last.weight[s1 + u][threadIdx.x] = g[u];
                            }
                        }
                        sh.last.inverse[threadIdx.x] = inverse_sum(total);
                        const int r = row0 + threadIdx.x;
                        if (a.lse && r < a.rows) a.lse[(size_t)bh * a.rows + r] = log_sum(top, total);
                    }
                    __syncthreads();
                }
#pragma unroll
                for (int e = 0; e < ITEMS; ++e) {
                    const int row = 16 * (min(item0 + e * stride + (int)threadIdx.x, RT * 512 - 1) >> 9) + n;
#pragma unroll
                    for (int u = 0; u < 8; ++u) o[e] += v[e][u] * sh.last.weight[s0 + u][row];      // (0 past the last split)
                }
            }
#pragma unroll
            for (int e = 0; e < ITEMS; ++e) {
                const int item = item0 + e * stride + threadIdx.x, row = 16 * (item >> 9) + n, r = row0 + row;       // (64 items of a wave: one tile of a row tile)
                if (item < RT * 512 && r < a.rows)
                    *reinterpret_cast<uint2*>(a.out + ((size_t)bh * a.rows + r) * kHeadDim + 16 * ((item >> 6) & 7) + 4 * kb) = halves_of(o[e], sh.last.inverse[row]);
            }
        }
    }
}

// ---- weights that tokens receive ----
// A wave has its blocks of 32 tokens for good and goes over all rows, up to 64 of them in LDS at a time; the sum of a token's
// column is that wave's alone, so it is added to the running one without atomics, in one fixed order.
constexpr int kWeightWaves = 8, kWeightThreads = 64 * kWeightWaves;

// Sums of eight values over the 16 lanes of a row of lanes; lane n gets that of value n % 8.  (Two values become one at every exchange:
// 22 instructions where a sum for each takes 32 and a choice.)
__device__ __forceinline__ float column_sums(const float (&v)[8], int n) {
    float a[4], b[2];
    auto join = [](bool odd, float x, float y, auto other) { const float keep = odd ? y : x, give = odd ? x : y; return keep + other(give); };
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = join(n & 1, v[2 * j], v[2 * j + 1], [](float x) { return dpp<kQuadXor1>(x); });
#pragma unroll
    for (int j = 0; j < 2; ++j) b[j] = join(n & 2, a[2 * j], a[2 * j + 1], [](float x) { return dpp<kQuadXor2>(x); });
    const float c = join(n & 4, b[0], b[1], [](float x) { return dpp<kRowHalfMirror>(dpp<0x1B /* quad_perm [3,2,1,0] */>(x)); });      // (lane ^ 4)
    return c + dpp<0x128 /* row_ror:8 */>(c);
}

template <int BITS, int AXIS, int RT, bool ONCE>
__global__ __launch_bounds__(kWeightThreads, 4) void add_weights(const TreeArgs a) {
    __shared__ QueryTiles<RT> sq;
    __shared__ ScaleStrip s_strip[kWeightWaves];
    __shared__ float s_lse[RT * 16];
    constexpr bool kBias = BITS != 16 && AXIS == KVQP_KEY_PER_CHANNEL;
    __shared__ float s_bias[kBias ? kWeightWaves * kBiasBlocks * 16 * RT : 1];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, kb = lane >> 4;
    const int bh = blockIdx.y;
    const int n_tok = __builtin_amdgcn_readfirstlane(head_tokens(a, bh));
    const int packed = (n_tok + 31) / 32, units = packed + (a.tail_len + 31) / 32;
    // (A head with a count of its own is divided among all the workgroups that the longest one has: 32 rows
    // over heads of 4,000 to 32,000 tokens took 28.2 us so, 31.3 where each took the longest head's share.)
    const int per_wg = a.head_n_kept ? (int)((unsigned)(units + gridDim.x - 1) / gridDim.x) : a.units_per_wg;
    const int u0 = blockIdx.x * per_wg, u1 = min(u0 + per_wg, units);
    if (u0 >= units) return;
    float* weights = a.weights + (size_t)bh * a.w_cap;
    ScaleStrip& strip = s_strip[wave];

#pragma unroll 1
    for (int row0 = 0; row0 < a.rows; row0 += RT * 16) {
        if (row0) __syncthreads();
        const QueryPieces<RT> pieces = request_queries<RT>(a, bh, row0);
        stage_queries<RT>(pieces, sq);
        if (threadIdx.x < RT * 16) {
            const int r = row0 + threadIdx.x;
            const float l = r < a.rows ? a.lse[(size_t)bh * a.rows + r] : -INFINITY;
            s_lse[threadIdx.x] = l == -INFINITY ? -INFINITY : -l;
        }
        __syncthreads();
        const float decay = row0 ? 1.0f : a.decay;
        // (in natural units up to the exponential: sm_scale and the rows' powers of two are exact)
        float factor[RT], minus_lse[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) { factor[rt] = sq.factor[16 * rt + n] * a.sm_scale; minus_lse[rt] = s_lse[16 * rt + n]; }
        // A row that saw nothing, and one past the last, gives nothing whatever it and the keys hold: its lane does not take part.  (A row of zeros
        // times an infinite key is NaN, and no addend makes that 0.)
        auto gives = [&](int rt) { return minus_lse[rt] != -INFINITY; };
        auto weight = [&](float logit, int rt, float add) { return __builtin_amdgcn_exp2f(__builtin_fmaf(logit, factor[rt], add) * kLog2e); };
        // lane n < 8 of a row of lanes stores token 16 (n / 4) + 4 kb + n % 4
        auto store = [&](const float (&cs)[8], float* w, int t0, int len) {
            const float mine = column_sums(cs, n);
            const int t = t0 + 16 * (n >> 2) + 4 * kb + (n & 3);
            if (n < 8 && t < len) w[t] = decay != 0.0f ? __builtin_fmaf(decay, w[t], mine) : mine;
        };
        const int end = min(u1, packed);
        int blk = u0 + wave;
        if (blk < end) {
            const Fields<BITS> fields;
            const HeadBase base = head_base<BITS, AXIS>(a, bh);
            KeyWords<BITS, AXIS> kw;
            load_keys<BITS, AXIS, ONCE>(base, a.group_log2, blk, lane, kw);
            float* biases = s_bias + (kBias ? wave * kBiasBlocks * 16 * RT : 0);
            int turn = 0;
#pragma unroll 1
            for (; blk < end; blk += kWeightWaves) {
                f4v acc[RT][2];
                float add[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) add[rt] = minus_lse[rt];
                if constexpr (kBias) {
                    if (turn == 0) refresh_bias<RT>(base, a.group_log2, blk, kWeightWaves, end - 1, lane, sq.frag, biases);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) add[rt] = __builtin_fmaf(biases[turn * (16 * RT) + 16 * rt + n], factor[rt], minus_lse[rt]);
                    turn = (turn + 1) % kBiasBlocks;
                }
                key_product<BITS, AXIS, RT>(fields, kw, sq.frag, sq.sums, strip, lane, acc);
                load_keys<BITS, AXIS, ONCE>(base, a.group_log2, min(blk + kWeightWaves, end - 1), lane, kw);
                float cs[8] = {};
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    if (gives(rt))
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float w = weight(acc[rt][j >> 2][j & 3], rt, add[rt]);
                            cs[j] = rt ? cs[j] + w : w;
                        }
                store(cs, weights, 32 * blk, n_tok);
            }
        }
#pragma unroll 1
        for (int u = max(u0, packed) + wave; u < u1; u += kWeightWaves) {
            const int t0 = 32 * (u - packed);
            KeyWords<16, KVQP_KEY_PER_CHANNEL> kw;
#pragma unroll
            for (int H = 0; H < 2; ++H) {
                const uint16_t* p = a.tail_k + ((size_t)bh * a.tail_cap + min(t0 + 16 * H + n, a.tail_len - 1)) * kHeadDim + 32 * kb;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint4 w = *reinterpret_cast<const uint4*>(p + 8 * j);
                    kw.w[H][4 * j] = w.x; kw.w[H][4 * j + 1] = w.y; kw.w[H][4 * j + 2] = w.z; kw.w[H][4 * j + 3] = w.w;
                }
            }
            f4v acc[RT][2];
            key_product<16, KVQP_KEY_PER_CHANNEL, RT>(Fields<16>(), kw, sq.frag, sq.sums, strip, lane, acc);
            float cs[8] = {};
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                // the last row of the tail that the query row sees
                const int last = gives(rt) ? a.tail_len - a.n_new + (row0 + 16 * rt + n) % a.n_new - t0 - 4 * kb : -1;
#pragma unroll
                for (int j = 0; j < 8; ++j) cs[j] += 16 * (j >> 2) + (j & 3) <= last ? weight(acc[rt][j >> 2][j & 3], rt, minus_lse[rt]) : 0.0f;
            }
            store(cs, weights + n_tok, t0, a.tail_len);
        }
    }
}

template <int BITS, int AXIS, int RT>
hipError_t run_tree(const TreeArgs& a, hipStream_t stream) {
    const int pairs = (a.heads * a.n_splits + 7) / 8 * 8;
    const dim3 grid(pairs * a.row_blocks), block(64 * a.n_waves);
    constexpr bool kOnce = RT <= 2 || BITS == 16;
    if (kOnce && a.once) tree_attn<BITS, AXIS, RT, kOnce><<<grid, block, 0, stream>>>(a);
    else tree_attn<BITS, AXIS, RT, false><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
}
template <int BITS, int AXIS>
hipError_t run_tree_rt(const TreeArgs& a, int rt, hipStream_t stream) {
    if (rt == 1) return run_tree<BITS, AXIS, 1>(a, stream);
    if (rt == 2) return run_tree<BITS, AXIS, 2>(a, stream);
    return run_tree<BITS, AXIS, 4>(a, stream);
}
template <int BITS, int AXIS>
hipError_t run_weights(const TreeArgs& a0, hipStream_t stream) {
    TreeArgs a = a0;
    // Two workgroups per CU are there at a time: as many blocks to each as make that one round, and at least one per wave.
    const int units = (a.n_kept + 31) / 32 + (a.tail_len + 31) / 32, per_head = std::max(1, 512 / a.heads);
    a.units_per_wg = ((units + per_head - 1) / per_head + kWeightWaves - 1) / kWeightWaves * kWeightWaves;
    const dim3 grid((units + a.units_per_wg - 1) / a.units_per_wg, a.heads), block(kWeightThreads);
    if (BITS != 16 && a.rows <= 16 && a.once) add_weights<BITS, AXIS, 1, BITS != 16><<<grid, block, 0, stream>>>(a);
    else if (a.rows <= 16) add_weights<BITS, AXIS, 1, false><<<grid, block, 0, stream>>>(a);
    else if (a.rows <= 32) add_weights<BITS, AXIS, 2, false><<<grid, block, 0, stream>>>(a);
    else add_weights<BITS, AXIS, 4, false><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

// (one object per bit width, side by side)
template <int BITS> hipError_t tree_bits(const TreeArgs& a, int rt, int axis, hipStream_t stream);
template <int BITS> hipError_t weights_bits(const TreeArgs& a, int axis, hipStream_t stream);
#ifdef KVQP_TREE_BITS
template <> hipError_t tree_bits<KVQP_TREE_BITS>(const TreeArgs& a, int rt, int axis, hipStream_t stream) {
    if constexpr (KVQP_TREE_BITS != 16) {
        if (axis == KVQP_KEY_PER_TOKEN) return run_tree_rt<KVQP_TREE_BITS, KVQP_KEY_PER_TOKEN>(a, rt, stream);
    }
    return run_tree_rt<KVQP_TREE_BITS, KVQP_KEY_PER_CHANNEL>(a, rt, stream);
}
template <> hipError_t weights_bits<KVQP_TREE_BITS>(const TreeArgs& a, int axis, hipStream_t stream) {
    if constexpr (KVQP_TREE_BITS != 16) {
        if (axis == KVQP_KEY_PER_TOKEN) return run_weights<KVQP_TREE_BITS, KVQP_KEY_PER_TOKEN>(a, stream);
    }
    return run_weights<KVQP_TREE_BITS, KVQP_KEY_PER_CHANNEL>(a, stream);
}
#else
template <> hipError_t tree_bits<2>(const TreeArgs&, int, int, hipStream_t);
template <> hipError_t tree_bits<4>(const TreeArgs&, int, int, hipStream_t);
template <> hipError_t tree_bits<8>(const TreeArgs&, int, int, hipStream_t);
template <> hipError_t tree_bits<16>(const TreeArgs&, int, int, hipStream_t);
template <> hipError_t weights_bits<2>(const TreeArgs&, int, hipStream_t);
template <> hipError_t weights_bits<4>(const TreeArgs&, int, hipStream_t);
template <> hipError_t weights_bits<8>(const TreeArgs&, int, hipStream_t);
template <> hipError_t weights_bits<16>(const TreeArgs&, int, hipStream_t);

TreePlan plan_tree(const kvqp_cfg& cfg, int n_rows, int n_kept, int tail_len) {
    TreePlan p;
    const int rows = cfg.n_q_heads / cfg.n_kv_heads * n_rows;
    p.row_tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    p.row_blocks = (rows + 16 * p.row_tiles - 1) / (16 * p.row_tiles);
    const long long base = (long long)cfg.batch * cfg.n_kv_heads * p.row_blocks;
    const int units = (n_kept + 31) / 32 + (tail_len + 31) / 32 + (n_rows + 31) / 32;
    // By 105 shapes of 1 to 48 sequences, 32 to 16384 tokens and 4 to 80 rows, each with 4 to 12 waves and 1 to 32 splits, the rule is within 3 %
    // of the best in 95, 10 % off at most (profiles/tree_plan_sweep.txt): eight waves (four where there are no more blocks, twelve where every CU
    // has a long head to itself); splits from 20 blocks of 32 tokens on (34 blocks, 4 rows: 9.8 us in four, 12.4 in one), one to eight blocks, or
    // about a block to a wave, as far as there are CUs, but sixteen splits are enough until each has 32 blocks (joining more takes longer than
    // they save).
    p.most_splits = (int)std::max(1LL, std::min(256 / base, (long long)kMostSplits));
    p.n_splits = units <= 20 ? 1 : std::max(1, std::min({p.most_splits, (units + 4) / 8, std::max(16, units / 32)}));
    p.n_waves = units <= 4 ? 4 : std::min(base >= 128 && p.n_splits == 1 ? 12 : 8, most_waves(p.row_tiles));
    const size_t one = (size_t)base * (16 * p.row_tiles) * (kHeadDim + 2) * sizeof(float);
    p.ws_bytes = p.n_splits > 1 ? kTreeCounterBytes + one * p.n_splits : 0;
    p.ws_bound = p.most_splits > 1 ? kTreeCounterBytes + one * p.most_splits : 0;
    return p;
}

// Whether the call's loads of codes go round the 256 MB memory-side cache: as cfg's hint says, and without one where the call alone has more
// than 96 MB.  (Calls that arithmetic bounds always load normally.)
static bool rows_once(const kvqp_cfg& cfg, const kvqp_cache& c, int tensors) {
    if (cfg.decode_cache_hint != KVQP_CACHE_AUTO) return cfg.decode_cache_hint == KVQP_CACHE_STREAM;
    return (double)cfg.batch * cfg.n_kv_heads * c.n_kept * (kHeadDim * cfg.bits / 8) * tensors > 96.0 * (1 << 20);
}

static TreeArgs common_args(const kvqp_cfg& cfg, const kvqp_cache& c, int n_rows) {
    TreeArgs a = {};
    a.k_codes = (const uint32_t*)c.k_codes; a.v_codes = (const uint32_t*)c.v_codes;
    a.k_scale = (const uint16_t*)c.k_scale; a.k_zero = (const uint16_t*)c.k_zero;
    a.v_scale = (const uint16_t*)c.v_scale; a.v_zero = (const uint16_t*)c.v_zero;
    a.tail_k = (const uint16_t*)c.tail_k; a.tail_v = (const uint16_t*)c.tail_v;
    a.head_n_kept = c.head_n_kept;
    a.n_kept = c.n_kept; a.n_cap = layout_tokens(c, c.n_kept); a.tail_len = c.tail_len; a.tail_cap = c.tail_cap;
    a.heads = cfg.batch * cfg.n_kv_heads; a.n_kv_heads = cfg.n_kv_heads;
    a.n_new = n_rows; a.rows = cfg.n_q_heads / cfg.n_kv_heads * n_rows;
    a.group_log2 = cfg.bits == 16 || cfg.group_size == 128 ? 7 : cfg.group_size == 64 ? 6 : 5;
    a.sm_scale = cfg.sm_scale;
    a.row_blocks = a.n_splits = 1;
    return a;
}

hipError_t launch_tree(const kvqp_cfg& cfg, const void* q, const void* k_new, const void* v_new, const uint32_t* mask, bool mask_per_batch,
                       int n_rows, const kvqp_cache& cache, void* out, float* lse, void* ws, const TreePlan& plan, hipStream_t stream) {
    TreeArgs a = common_args(cfg, cache, n_rows);
    a.q = (const uint16_t*)q; a.k_new = (const uint16_t*)k_new; a.v_new = (const uint16_t*)v_new;
    a.mask = mask; a.mask_stride = mask_per_batch ? (size_t)n_rows * ((n_rows + 31) / 32) : 0;
    a.once = rows_once(cfg, cache, 2);
    a.out = (uint16_t*)out; a.lse = lse; a.arrivals = (unsigned int*)ws; a.part = (float*)((char*)ws + kTreeCounterBytes);
    a.row_blocks = plan.row_blocks; a.n_splits = plan.n_splits; a.n_waves = plan.n_waves;
    switch (cfg.bits) {
        case 2: return tree_bits<2>(a, plan.row_tiles, cfg.key_axis, stream);
        case 4: return tree_bits<4>(a, plan.row_tiles, cfg.key_axis, stream);
        case 8: return tree_bits<8>(a, plan.row_tiles, cfg.key_axis, stream);
        default: return tree_bits<16>(a, plan.row_tiles, cfg.key_axis, stream);
    }
}

__global__ __launch_bounds__(256) void clear_counters(uint32_t* at) {
    for (int i = threadIdx.x; i < (int)(kTreeCounterBytes / 4); i += 256) at[i] = 0u;
}
hipError_t launch_tree_init(void* ws, hipStream_t stream) {
    clear_counters<<<dim3(1), dim3(256), 0, stream>>>((uint32_t*)ws);
    return hipGetLastError();
}

hipError_t launch_weights(const kvqp_cfg& cfg, const void* q, const float* lse, int n_rows, const kvqp_cache& cache, float* weights, int w_cap,
                          float decay, hipStream_t stream) {
    TreeArgs a = common_args(cfg, cache, n_rows);
    a.q = (const uint16_t*)q; a.lse = const_cast<float*>(lse); a.weights = weights; a.w_cap = w_cap; a.decay = decay;
    a.once = rows_once(cfg, cache, 1);
    switch (cfg.bits) {
        case 2: return weights_bits<2>(a, cfg.key_axis, stream);
        case 4: return weights_bits<4>(a, cfg.key_axis, stream);
        case 8: return weights_bits<8>(a, cfg.key_axis, stream);
        default: return weights_bits<16>(a, cfg.key_axis, stream);
    }
}
#endif

}  // namespace kvqp
