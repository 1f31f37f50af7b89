// Attention over the paged cache of 8-bit codes (kvqp_paged_attn).
//
//   out = sum_t w_t v_t / sum_t w_t,   w_t = 2^(kLift + l_t - r),   l_t = (sm_scale / ln 2) q k_t,   lse = ln 2 (r - kLift + log2 sum_t w_t),
// in one pass over the tokens: r is a reference near the largest l_t so far, and O and the sum are brought to a new one when it moves.  Two kernels: paged_rows
// for up to 64 rows of a KV head (query heads times new tokens), bound by reading the codes, and paged_tiles for more, bound by issue and the matrix cores.
// Numbers below were measured on an MI355X.
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
    int slots;              // workgroups of a KV head
    int most_shares;        // how many shares the work of a KV head is cut into at most; 0: sequences are not split
    int at_once;            // workgroups of a KV head that a single sequence is cut into at most
    bool once;              // loads of codes go past the memory-side cache (one tile of rows)
};

// Groups of 64 tokens that a workgroup has at least, and the most sequences among which work is shared out.
constexpr int kLeastGroups = 4;      // (one a wave)
[[maybe_unused]] constexpr int kMostSplitBatch = 512;

template <bool BF, bool INT8> hipError_t paged_form(const AttnArgs& a, int row_tiles, hipStream_t stream);

#ifdef KVQP_PAGED_BITS

typedef float f4v __attribute__((ext_vector_type(4)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
typedef _Float16 h2v __attribute__((ext_vector_type(2)));

constexpr float kLowest = -3.402823466e38f;      // reference of a row that has seen nothing: binary32 has no logit below it
constexpr float kLn2 = 0.69314718055994531f;
// Weights are 2^(kLift + logit - reference) with a reference that may lag behind the row's largest logit by up to kLag: between the two a weight
// stays below 2^15 and what binary16 holds reaches 2^-29 of the row's largest weight at least (normal numbers to 2^-18).
constexpr float kLift = 4.f, kLag = 10.f;
constexpr int kDeviceScope = 16;      // sc1 in a buffer access' cache policy

constexpr f4v kZero = {0.f, 0.f, 0.f, 0.f};

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

// Partial results of one workgroup of a split piece: outputs in the order of the accumulators, and (reference, sum) of the rows.
struct Partials {
    __amdgpu_buffer_rsrc_t at;
    int bytes, states, joined;      // of a workgroup's results, where the rows' states begin, and those of several workgroups' joined results
    mutable int states_read;
    // part: the first of `splits` workgroups' results, which follow each other
    __device__ __forceinline__ Partials(const AttnArgs& a, int64_t part, int splits, int row_tiles)
        : bytes(row_tiles * 8448), states(row_tiles * 8192), joined(row_tiles * 8320), states_read(row_tiles * 8192) {
        at = __builtin_amdgcn_make_buffer_rsrc(a.part + part * bytes, 0, splits * bytes, 0x00020000);
    }
    __device__ __forceinline__ void put_output(int split, int item, f4v o) const {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4v, o), at, split * bytes + item * 16, 0, kDeviceScope);
    }
    __device__ __forceinline__ void put_state(int split, int row, float ref, float sum) const {
        const u2v v = {__float_as_uint(ref), __float_as_uint(sum)};
        __builtin_amdgcn_raw_buffer_store_b64(v, at, split * bytes + states + row * 8, 0, kDeviceScope);
    }
    __device__ __forceinline__ void put_joined(int split, int row, float ref, float sum) const {
        const u2v v = {__float_as_uint(ref), __float_as_uint(sum)};
        __builtin_amdgcn_raw_buffer_store_b64(v, at, split * bytes + joined + row * 8, 0, kDeviceScope);
    }
    __device__ __forceinline__ void use_joined(bool yes) const { states_read = yes ? joined : states; }
    __device__ __forceinline__ f4v output(int split, int item) const {
        return __builtin_bit_cast(f4v, __builtin_amdgcn_raw_buffer_load_b128(at, split * bytes + item * 16, 0, kDeviceScope));
    }
    __device__ __forceinline__ float2 state(int split, int row) const {
        const u2v v = __builtin_amdgcn_raw_buffer_load_b64(at, split * bytes + states_read + row * 8, 0, kDeviceScope);
        return make_float2(__uint_as_float(v[0]), __uint_as_float(v[1]));
    }
};

// ---- what both kernels do with a piece of a sequence's rows ----

// Which sequence, piece of its rows and split of its tokens a workgroup has.  Only the device knows the lengths, so every wave looks at all of them:
// the work of a KV head, groups of 64 tokens times pieces of rows, is cut into shares of one size, and each piece of a sequence of g groups is split
// into ceil(g / share).  (Only more than a share is split, so the split pieces' workgroups are less than twice as many as the shares.)
struct Slot {
    Sequence seq;
    int piece, split, splits;
    int part;               // number of the piece's first workgroup among those of split pieces
};
__device__ __forceinline__ Slot find_slot(const AttnArgs& a, int slot, Sequence* s_found) {
    const PageArgs& p = a.p;
    auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    if (a.most_shares == 0) {
        const Sequence s = owner_of_piece(p, slot, a.per_piece, 1, 1 << a.page_log2, s_found);
        const Sequence u = {uniform(s.b), uniform(s.row0), uniform(s.rows), uniform(s.length)};
        const int piece = u.b < 0 ? 0 : slot - first_piece(p, u, a.per_piece, 1);
        return {{piece * a.per_piece < u.rows ? u.b : -1, u.row0, u.rows, u.length}, piece, 0, 1, 0};
    }
    const int lane = threadIdx.x & 63, most = p.max_pages << a.page_log2;
    struct Share { Sequence seq; int pieces, groups; };
    bool falling = false;      // starts that descend
    // (loads without a branch, so that all are on their way at once; what is behind the last sequence counts for nothing)
    auto look = [&](int b) {
        const int at = min(b, p.batch - 1);
        int r0 = at, r1 = at + 1;
        if (p.row_start) { r0 = p.row_start[at]; r1 = p.row_start[at + 1]; }
        falling |= r1 < r0;
        Share s;
        s.seq.b = b;
        s.seq.row0 = min(max(r0, 0), p.n_rows);
        s.seq.rows = b < p.batch ? max(min(r1, p.n_rows) - s.seq.row0, 0) : 0;
        s.seq.length = min(max(p.lengths[at], 0), most);
        s.pieces = (s.seq.rows + a.per_piece - 1) / a.per_piece;
        const int seen = a.window > 0 ? min(s.seq.length, a.window + min(s.seq.rows, a.per_piece)) : s.seq.length;
        s.groups = (seen + 63) / 64;
        return s;
    };
    if (p.batch == 1) {
        const Share one = look(0);
        // (equal pieces: as many splits as are on the chip together.  512 rows of 32 heads over 16000 tokens: 158 us, with 384 shares 200)
        const int splits = max(min(a.at_once / max(one.pieces, 1), (one.groups + kLeastGroups - 1) / kLeastGroups), 1);
        const int piece = slot / splits;
        return {{piece < one.pieces ? 0 : -1, uniform(one.seq.row0), uniform(one.seq.rows), uniform(one.seq.length)}, uniform(piece), uniform(slot % splits), uniform(splits),
                uniform(piece * splits)};
    }
    // (lane l has sequences 4 l .. 4 l + 3 of 256)
    Share mine[4];
    float work = 0.f;
    for (int b0 = p.batch > 256 ? 256 : 0; b0 >= 0; b0 -= 256) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            mine[j] = look(b0 + 4 * lane + j);
            work += (float)mine[j].pieces * (float)mine[j].groups;
        }
    }
    // (sequences that have the same rows may be more work than the launch has workgroups for, and a split piece would wait for its last ones: none begins)
    if (__any(falling)) return {{-1, 0, 0, 0}, 0, 0, 1, 0};
#pragma unroll
    for (int d = 1; d < 64; d *= 2) work += __shfl_xor(work, d);
    const float share = fmaxf(work / (float)a.most_shares, (float)kLeastGroups);
    int workgroups = 0, parts = 0;      // of the 256 sequences before
    Slot s = {{-1, 0, 0, 0}, 0, 0, 1, 0};
    for (int b0 = 0; b0 < p.batch; b0 += 256) {
        int n[4], m[4], splits[4], upto = 0, parts_upto = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (b0) mine[j] = look(b0 + 4 * lane + j);
            splits[j] = max((int)ceilf((float)mine[j].groups / share), 1);
            n[j] = mine[j].pieces * splits[j];
            m[j] = splits[j] > 1 ? n[j] : 0;
            upto += n[j]; parts_upto += m[j];
        }
        const int own = upto, own_parts = parts_upto;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(upto, d), y = __shfl_up(parts_upto, d);
            if (lane >= d) { upto += x; parts_upto += y; }
        }
        int at = slot - (workgroups + upto - own), part = parts + parts_upto - own_parts;
        bool hit = false;
        Slot t = s;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (!hit && at >= 0 && at < n[j]) {
                hit = true;
                t = {mine[j].seq, at / splits[j], at % splits[j], splits[j], part + at / splits[j] * splits[j]};
            }
            at -= n[j];
            part += m[j];
        }
        const uint64_t who = __ballot(hit);
        if (who) {
            const int from = __ffsll((unsigned long long)who) - 1;
            auto of = [&](int x) { return __builtin_amdgcn_readlane(x, from); };
            return {{of(t.seq.b), of(t.seq.row0), of(t.seq.rows), of(t.seq.length)}, of(t.piece), of(t.split), of(t.splits), of(t.part)};
        }
        workgroups += __builtin_amdgcn_readlane(upto, 63);
        parts += __builtin_amdgcn_readlane(parts_upto, 63);
    }
    return s;
}

// The tokens that a workgroup's rows see, in groups of 64 from token 0: whole blocks, and open tokens behind them.
struct Range {
    Sequence seq;
    int i0, n;                  // rows of the sequence: i0 .. i0 + n - 1
    int first, last;            // their positions
    int begin, closed, open;    // where the open block begins; whole blocks' tokens that are seen end there; open tokens that are seen
    int lo;                     // first token that any row sees
    int ga, gb;                 // groups of this workgroup
    int split, active, part;    // its number among those that have some, and where their results go
    __device__ __forceinline__ bool find(const AttnArgs& a, int slot, Sequence* s_found) {
        const Slot s = find_slot(a, slot, s_found);
        seq = s.seq;
        if (seq.b < 0 || (s.splits > 1 && s.part + s.splits > 2 * a.most_shares)) return false;      // (the second: lengths that change meanwhile)
        i0 = s.piece * a.per_piece;
        n = min(a.per_piece, seq.rows - i0);
        first = seq.position(i0);
        last = first + n - 1;
        begin = seq.length >> a.page_log2 << a.page_log2;
        lo = a.window > 0 ? max(first - a.window + 1, 0) : 0;
        closed = min(last + 1, begin);
        open = max(last + 1 - begin, 0);
        const int g_lo = lo / 64, groups = closed > lo ? (closed + 63) / 64 - g_lo : 0;
        const int each = max((groups + s.splits - 1) / s.splits, kLeastGroups);
        split = s.split; part = s.part;
        active = max((groups + each - 1) / each, 1);
        ga = g_lo + split * each;
        gb = min(ga + each, g_lo + groups);
        return split < active;
    }
    // (a head's parts are next to each other)
    __device__ __forceinline__ int64_t part_of_head(const AttnArgs& a, int h) const { return (int64_t)h * (2 * a.most_shares) + part; }
};

// Of one row tile a lane has one row (column c) and eight tokens at a time; O^T of the tile is eight accumulators of 16 channels.
// A weight is 2^(logit + lift), lift = kLift - reference.  (The sums are of the weights before they are rounded for the value product: a product with ones
// would save the additions, and leave the sum 2^-12 off.)
template <int RT>
struct Sums {
    f4v o[RT][8];
    float sums[RT], lift[RT];      // (a lane's sum: of its own tokens)
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            lift[rt] = -kLowest;
            sums[rt] = 0.f;
#pragma unroll
            for (int t = 0; t < 8; ++t) o[rt][t] = f4v{0.f, 0.f, 0.f, 0.f};
        }
    }
    __device__ __forceinline__ void times(float f) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int t = 0; t < 8; ++t) o[rt][t] *= f;
    }
    // Products of queries and keys, times f > 0 the logits, into weights; O and the sum follow the reference, which moves when a row has gone far beyond it.
    // (The highest is sought among the exponents: a sum that comes out of a product would cost a further instruction each.)
    __device__ __forceinline__ f8v weigh(int rt, const f4v (&x)[2], float f) {
        f8v w;
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = __builtin_fmaf(x[j >> 2][j & 3], f, lift[rt]);
        const float most = fmaxf(fmaxf(fmaxf(fmaxf(w[0], w[1]), w[2]), fmaxf(w[3], w[4])), fmaxf(fmaxf(w[5], w[6]), w[7]));
        if (__any(most > kLift + kLag)) {
            float m = fmaxf(fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), x[0][2]), fmaxf(x[0][3], x[1][0])), fmaxf(fmaxf(x[1][1], x[1][2]), x[1][3])) * f;
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            // Far from 0 a reference is rounded by whole powers of two, up to 1.5 * 2^-23 m with m's own rounding and this one: from 2^22 on it is that much too low, so that
            // the row's largest weight is none too small, and what is too large for binary16 then is cut to what the lag allows.  (Logits so near each other are one.)
            float lower = kLift - m;
            const float more = __builtin_fmaf(fabsf(m), 0x1p-22f, -1.f);
            if (more > 0.f && more < INFINITY) lower += more;
            lower = fminf(lift[rt], lower);
            const float by = __builtin_amdgcn_exp2f(lower - lift[rt]);
            lift[rt] = lower;
            sums[rt] *= by;
#pragma unroll
            for (int t = 0; t < 8; ++t) o[rt][t] *= by;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                w[j] = __builtin_fmaf(x[j >> 2][j & 3], f, lower);
                w[j] = w[j] > kLift + kLag ? kLift + kLag : w[j];      // (NaN stays)
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = __builtin_amdgcn_exp2f(w[j]);
        sums[rt] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
        return w;
    }
    __device__ __forceinline__ float reference(int rt) const { return kLift - lift[rt]; }
    __device__ __forceinline__ float sum(int rt) const {
        float x = sums[rt];
        x += __shfl_xor(x, 16);
        return x + __shfl_xor(x, 32);
    }
};
// Eight weights as the second operand of the value product.  For binary16 rows they are two numbers each (TWO), w and what its rounding left: one alone, off by up to 2^-12 of itself,
// adds nearly as much error as the output's own rounding does (1.1 to 1.5 times the error of the formula rounded once; with two 1.000).  The products with the rest cost a prompt of
// 8192 tokens 135 us of 725; where reading the codes is the bound, nothing (32 x 8192 tokens 97.4 and 97.8).  Of bfloat16 outputs, whose rounding is eight times as
// large, one number makes the error 1.0075 times as large at most, and suffices.
template <bool TWO>
struct Weights {
    h8v w, rest;
    __device__ __forceinline__ void put(f8v y) {
        w = __builtin_convertvector(y, h8v);
        if constexpr (TWO) {
            float minus = -1.f;
            asm("" : "+s"(minus));      // (a multiply-add takes binary16 as it is; a subtraction, which a known factor would make of it, converts first)
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = __builtin_fmaf((float)w[j], minus, y[j]);
            rest = __builtin_convertvector(y, h8v);
        }
    }
    __device__ __forceinline__ f4v product(h8v v, f4v o) const {
        o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w, o, 0, 0, 0);
        if constexpr (TWO) o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, rest, o, 0, 0, 0);
        return o;
    }
};
// (a masked product is minus infinity: the factor must not be 0, also where a block of zeros has the smallest scale)
__device__ __forceinline__ float logit_factor(float key_scale, float row_scale) { return fmaxf(key_scale * row_scale, 1e-36f); }

// Row r of a workgroup: new token r / gq of its piece, query head r % gq of the KV head's.
__device__ __forceinline__ const uint16_t* query_at(const AttnArgs& a, const Range& w, int h, int r) {
    const int i = r / a.p.gq;
    return a.q + (int64_t)(w.seq.row0 + w.i0 + (i < w.n ? i : 0)) * a.q_stride + (h * a.p.gq + r % a.p.gq) * kHeadDim;
}
__device__ __forceinline__ int64_t result_at(const AttnArgs& a, const Range& w, int h, int r) {
    return (int64_t)(w.seq.row0 + w.i0 + r / a.p.gq) * (a.p.gq * a.p.n_kv_heads) + h * a.p.gq + r % a.p.gq;
}
template <bool BF>
__device__ __forceinline__ void store_out(const AttnArgs& a, const Range& w, int h, int r, int t, int kb, f4v x, float by) {
    x *= by;
    uint2 y;
    if constexpr (BF) {
        typedef __bf16 b4v __attribute__((ext_vector_type(4)));
        y = __builtin_bit_cast(uint2, __builtin_convertvector(x, b4v));
    } else {
        typedef _Float16 h4v __attribute__((ext_vector_type(4)));
        y = __builtin_bit_cast(uint2, __builtin_convertvector(x, h4v));
    }
    *reinterpret_cast<uint2*>(a.out + result_at(a, w, h, r) * kHeadDim + 16 * t + 4 * kb) = y;
}

// A row's query as binary16 fragments: 8 channels from 32 s + 8 kb (or, WIDE, 64 (s >> 1) + 16 kb + 8 (s & 1): 16 bytes of a key at a time) for the lane's
// column.  A bfloat16 row times a power of two, such that its largest element is 2^15 to 2^16, is a row of binary16 numbers, but for what is below 2^-29 of that: so codes
// meet it without a conversion to bfloat16, and the logits' factor takes the power back.
template <bool BF, bool WIDE>
__device__ __forceinline__ float query_fragments(const uint16_t* q, bool there, int kb, float logit_scale, h8v (&out)[4]) {
    uint4 w[4];
#pragma unroll
    for (int s = 0; s < 4; ++s)
        w[s] = *reinterpret_cast<const uint4*>(q + (WIDE ? 64 * (s >> 1) + 16 * kb + 8 * (s & 1) : 32 * s + 8 * kb));
    if (!there) {
#pragma unroll
        for (int s = 0; s < 4; ++s) w[s] = make_uint4(0, 0, 0, 0);
    }
    if constexpr (BF) {
        float m = 0.f;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const f8v x = numbers<true>(w[s]);
#pragma unroll
            for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(x[j]));
        }
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const int e = min(max((int)(__float_as_uint(m) >> 23) - 142, -120), 113);
#pragma unroll
        for (int s = 0; s < 4; ++s) out[s] = __builtin_convertvector(numbers<true>(w[s]) * two_to(-e), h8v);
        return logit_scale * two_to(e);
    } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) out[s] = __builtin_bit_cast(h8v, w[s]);
        return logit_scale;
    }
}

// Open tokens, for one wave's rows r0 ..: in the rows' own type, weights as two numbers of it each.
// Values come from LDS ([64][kHeadDim + 8], zeros behind the last).
typedef uint16_t OpenValues[64][kHeadDim + 8];
__device__ __forceinline__ void stage_open_values(const AttnArgs& a, const Range& w, int h, int slot, OpenValues& s_v, int thread, int threads) {
    const int P = 1 << a.page_log2, from = w.begin & (2 * P - 1);            // (a block's rows are next to each other)
    const uint16_t* v = a.p.open_v + ((int64_t)slot * a.p.n_kv_heads + h) * (2 * P * kHeadDim) + from * kHeadDim;
    for (int i = thread; i < (w.open + 31) / 32 * 32 * 16; i += threads) {
        const int t = i >> 4;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (t < w.open) x = *reinterpret_cast<const uint4*>(v + t * kHeadDim + 8 * (i & 15));
        *reinterpret_cast<uint4*>(&s_v[t][8 * (i & 15)]) = x;
    }
}
template <bool BF, int RT>
__device__ __forceinline__ void attend_open(const AttnArgs& a, const Range& w, int h, int slot, const OpenValues& s_v, int r0, Sums<RT>& st) {
    const int lane = threadIdx.x & 63, c = lane & 15, kb = lane >> 4, P = 1 << a.page_log2, from = w.begin & (2 * P - 1);
    const uint16_t* keys = a.p.open_k + ((int64_t)slot * a.p.n_kv_heads + h) * (2 * P * kHeadDim) + from * kHeadDim;
    // 32 tokens at a time, in their order: of tile t of them a lane has tokens 16 t + 4 kb .. + 3.
#pragma unroll 1
    for (int t0 = 0; t0 < w.open; t0 += 32) {
        f4v x[RT][2];
        uint4 k[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int off = min(t0 + 16 * t + c, w.open - 1);      // (what is behind the last is masked)
#pragma unroll
            for (int s = 0; s < 4; ++s) k[t][s] = *reinterpret_cast<const uint4*>(keys + off * kHeadDim + 32 * s + 8 * kb);
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int r = r0 + 16 * rt + c, i = r / a.p.gq;
            const uint16_t* rows = query_at(a, w, h, r);
            const int position = i < w.n ? w.first + i : -1, low = a.window > 0 ? position - a.window : -1;
            uint4 q[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) q[s] = *reinterpret_cast<const uint4*>(rows + 32 * s + 8 * kb);      // (a row that is not there sees nothing)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                x[rt][t] = f4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < 4; ++s) x[rt][t] = product_of_rows<BF>(k[t][s], q[s], x[rt][t]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int off = t0 + 16 * t + 4 * kb + j, token = w.begin + off;
                    const bool hidden = (off >= w.open) | (token > position) | (token <= low);
                    x[rt][t][j] = hidden ? -INFINITY : x[rt][t][j];
                }
            }
        }
        uint4 e[RT], e_rest[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const f8v y = st.weigh(rt, x[rt], a.logit_scale);
            e[rt] = rounded<BF>(y);
            e_rest[rt] = rounded<BF>(y - numbers<BF>(e[rt]));
        }
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            uint32_t v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = t0 + 16 * (j >> 1) + 4 * kb + 2 * (j & 1);
                v[j] = (uint32_t)s_v[r][16 * t + c] | (uint32_t)s_v[r + 1][16 * t + c] << 16;
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                st.o[rt][t] = product_of_rows<BF>(make_uint4(v[0], v[1], v[2], v[3]), e[rt], st.o[rt][t]);
                st.o[rt][t] = product_of_rows<BF>(make_uint4(v[0], v[1], v[2], v[3]), e_rest[rt], st.o[rt][t]);
            }
        }
    }
}

// Numbers and scales of a stretch of pages, in LDS.
constexpr int kSegment = 512;
struct Segment {
    int page[kSegment];
    float k_scale[kSegment], v_scale[kSegment];
};
// In steps, so that other loads can be on their way at the same time.
template <int THREADS>
struct PageNumbers {
    int mine[kSegment / THREADS];
    int holes;                // a block that is seen has no page
    __device__ __forceinline__ void request(const AttnArgs& a, const Range& w, int first_block, int blocks) {
        holes = 0;
#pragma unroll
        for (int u = 0; u < kSegment / THREADS; ++u) {
            const int i = threadIdx.x + THREADS * u, block = first_block + i;
            const int page = a.p.table[(int64_t)w.seq.b * a.p.max_pages + min(block, a.p.max_pages - 1)];
            // (what is before every row's window may be anything, the scales of a page that another sequence has by now as well: not there)
            const bool read = i < blocks && (int64_t)block << a.page_log2 < w.closed && (int64_t)(block + 1) << a.page_log2 > w.lo;
            const bool there = read && (unsigned)page < (unsigned)a.p.n_pages;
            mine[u] = there ? page : -1;
            holes |= read && !there;
        }
    }
    __device__ __forceinline__ bool put(Segment& seg) const {
#pragma unroll
        for (int u = 0; u < kSegment / THREADS; ++u) seg.page[threadIdx.x + THREADS * u] = mine[u];
        return __syncthreads_or(holes) != 0;
    }
};
// A value's code of the largest scale is multiplied by as much as binary16 has room for, so that codes of smaller scales are normal numbers for longer (e4m3:
// 448 2^7; integers: what they are converted by is 1152 2^5).
template <bool INT8> constexpr float kValueLift = INT8 ? 32.f : 128.f;
// top: the largest scale of values so far, over kValueLift, of all threads in *s_top
template <int THREADS, bool INT8>
__device__ __forceinline__ float look_up_scales(const AttnArgs& a, int h, float top, Segment& seg, const PageNumbers<THREADS>& pages, unsigned int* s_top) {
    float most = top;
#pragma unroll
    for (int u = 0; u < kSegment / THREADS; ++u) {
        const int64_t at = (int64_t)max(pages.mine[u], 0) * a.p.n_kv_heads + h;
        float ks = a.p.k_scale[at], vs = a.p.v_scale[at];
        if (pages.mine[u] < 0) { ks = 1.f; vs = 0.f; }
        const int i = threadIdx.x + THREADS * u;
        seg.k_scale[i] = ks; seg.v_scale[i] = vs;
        most = fmaxf(most, vs * (1.f / kValueLift<INT8>));
    }
    if (most > top) atomicMax(s_top, __float_as_uint(most));
    __syncthreads();
    return __uint_as_float(__builtin_amdgcn_readfirstlane(*s_top));
}

// Results of a piece's splits are joined by the last workgroup to arrive, in the order of the splits (no atomics on results: the same bits every time); where
// there are more than 16, by 16 at a time, the last of each 16 first, and then the last of those their results (96 splits of 16 rows read by one workgroup
// alone took 9 us).
// Partials are stored past this die's L2, and the wait returns when the stores have been acknowledged from there; so whoever sees the
// counter sees them, with loads that do not look into its own L2.
__device__ __forceinline__ bool arrived_last(unsigned int* count, int of, int* s_last) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        const unsigned before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *s_last = before == (unsigned)(of - 1);
        if (*s_last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return *s_last != 0;
}
constexpr int kJoin = 16;
template <bool BF, int RT>
__device__ __forceinline__ void join_splits(const AttnArgs& a, const Range& w, int h, const Partials& parts, int* s_last) {
    static_assert(RT == 1 || RT % 2 == 0, "a thread takes items of two row tiles at a time: an odd number of tiles would end behind the outputs, in the rows' states");
    constexpr int row_tiles = RT;
    unsigned int* const counts = a.arrivals + w.part_of_head(a, h);
    const int c = threadIdx.x & 15, kb = (threadIdx.x & 63) >> 4, rows = w.n * a.p.gq;
    // results from, from + step, ... below upto: MOST of an item (four channels of a row) are requested at once, for ITEMS items of a thread, two of a
    // row tile and then the next.  (What is requested beyond the last costs time too: 16 where four splits would do makes a call of 1024 tokens 3 us longer.)
    auto join_by = [&](auto most, auto items, int from, int step, int upto, auto take) {
        constexpr int MOST = decltype(most)::value, ITEMS = decltype(items)::value, TILES = (ITEMS + 1) / 2;
        for (int item0 = threadIdx.x; item0 < row_tiles * 512; item0 += 256 * ITEMS) {
            const int r0 = 16 * (item0 >> 9) + c;
            float top[TILES], total[TILES];
            f4v x[ITEMS];
#pragma unroll
            for (int t = 0; t < TILES; ++t) { top[t] = kLowest; total[t] = 0.f; }
#pragma unroll
            for (int e = 0; e < ITEMS; ++e) x[e] = f4v{0.f, 0.f, 0.f, 0.f};
            for (int s0 = from; s0 < upto; s0 += MOST * step) {
                f4v v[ITEMS][MOST];
                float2 m[TILES][MOST];
#pragma unroll
                for (int u = 0; u < MOST; ++u) {
                    const int s = s0 + u * step < upto ? s0 + u * step : s0;
#pragma unroll
                    for (int t = 0; t < TILES; ++t) m[t][u] = parts.state(s, r0 + 16 * t);
#pragma unroll
                    for (int e = 0; e < ITEMS; ++e) v[e][u] = parts.output(s, item0 + 256 * e);
                }
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    float higher = top[t];
#pragma unroll
                    for (int u = 0; u < MOST; ++u) higher = fmaxf(higher, m[t][u].x);
                    const float f = __builtin_amdgcn_exp2f(top[t] - higher);
                    total[t] *= f;
#pragma unroll
                    for (int e = 2 * t; e < ITEMS && e < 2 * t + 2; ++e) x[e] *= f;
#pragma unroll
                    for (int u = 0; u < MOST; ++u) {
                        const float by = s0 + u * step < upto ? __builtin_amdgcn_exp2f(m[t][u].x - higher) : 0.f;
                        total[t] = __builtin_fmaf(m[t][u].y, by, total[t]);
#pragma unroll
                        for (int e = 2 * t; e < ITEMS && e < 2 * t + 2; ++e) x[e] += v[e][u] * by;
                    }
                    top[t] = higher;
                }
            }
#pragma unroll
            for (int e = 0; e < ITEMS; ++e) take(item0 + 256 * e, r0 + 16 * (e / 2), x[e], top[e / 2], total[e / 2]);
        }
    };
    auto join = [&](int from, int step, int upto, auto take) {
        const int n = (upto - from + step - 1) / step;
        constexpr std::integral_constant<int, RT >= 2 ? 4 : 2> items;
        if (n <= 2) join_by(std::integral_constant<int, 2>{}, items, from, step, upto, take);
        else if (n <= 4) join_by(std::integral_constant<int, 4>{}, items, from, step, upto, take);
        else if (n <= 8) join_by(std::integral_constant<int, 8>{}, items, from, step, upto, take);
        else join_by(std::integral_constant<int, kJoin>{}, std::integral_constant<int, 1>{}, from, step, upto, take);
    };
    int step = 1;
    if (w.active > kJoin) {
        const int from = w.split / kJoin * kJoin, upto = min(from + kJoin, w.active);
        if (!arrived_last(counts + from, upto - from, s_last)) return;
        // (an item's result takes its place in the first of the 16, which its own thread has read; a row's state, which others read too, a place of its own)
        if (upto - from > 1) {
            join(from, 1, upto, [&](int item, int r, f4v x, float top, float total) {
                parts.put_output(from, item, x);
                if ((item & 0x1C0) == 0 && kb == 0) parts.put_joined(from, r, top, total);
            });
        } else {
            for (int r = threadIdx.x; r < 16 * row_tiles; r += 256) {
                const float2 m = parts.state(from, r);
                parts.put_joined(from, r, m.x, m.y);
            }
        }
        step = kJoin;
        if (!arrived_last(counts + 1, (w.active + kJoin - 1) / kJoin, s_last)) return;
    } else if (!arrived_last(counts, w.active, s_last)) {
        return;
    }
    parts.use_joined(step > 1);
    join(0, step, w.active, [&](int item, int r, f4v x, float top, float total) {
        if (r < rows) {
            store_out<BF>(a, w, h, r, (item >> 6) & 7, kb, x, inverse_sum(total));
            if (a.lse && (item & 0x1C0) == 0 && kb == 0) a.lse[result_at(a, w, h, r)] = log_sum(top, total);
        }
    });
}

// ---- few rows: the tokens are split over waves and workgroups ----
//
// A wave takes 64 tokens at a time.  S^T = K Q^T by products of 16 tokens and 16 rows: a lane's column is a row (query head and new token) and its
// group kb of 16 lanes holds tokens 16 kb .. 16 kb + 15, in an order that makes its logits, turned into weights, the second operand of
// O^T = V^T P^T without leaving the lane; the first operand is 16 consecutive bytes of a channel, as pages store values.
//
// Codes go from memory to registers, each wave's own: nobody else in the workgroup needs them, so LDS would add a round trip.  A wave requests the next 64
// tokens' keys while it works on values, and their values after that.  32 sequences of 8192 tokens, 8 KV heads of 4 query heads (538 MB): 98 us,
// 5.5 TB/s, more than a large copy reaches.  One sequence of 1024 tokens: 9.6 us, the chain of launch, lengths, table, codes and join.
// 17 .. 32 rows take two tiles of 16 (two waves a SIMD by registers), more than 32 several workgroups of 32 each, so that keys and values are read
// from memory 1.1 times and else from the caches (40 rows of a KV head for each of 48 sequences of up to 16001 tokens, bfloat16 and int8: 212 us for 791 MB, twice through matrix and vector
// instructions; tiles of 3 and 4 would need 512 registers a lane, and are not used; the kernel of many rows takes 208 .. 303).
constexpr int kRowsWaves = 4;

template <int RT, int NW>
union RowsShared {
    struct { h8v q[RT][4][64]; Segment seg; } run;
    OpenValues open_v;
    struct { f4v o[NW][8][64]; float ref[NW][16 * RT], sum[NW][16 * RT]; } join;
};

template <bool BF, bool INT8, int RT, bool ONCE>
__global__ __launch_bounds__(64 * kRowsWaves, RT == 1 ? 3 : 2) void paged_rows(const AttnArgs a) {
    constexpr int NW = kRowsWaves, THREADS = 64 * NW;
    __shared__ RowsShared<RT, NW> sh;
    __shared__ Sequence s_slot;
    __shared__ int s_last;
    __shared__ unsigned int s_top;
    const PageArgs& p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, kb = lane >> 4;
    const int h = blockIdx.x % p.n_kv_heads, P = 1 << a.page_log2;
    Range w;
    if (!w.find(a, blockIdx.x / p.n_kv_heads, &s_slot)) return;
    const int ga = w.ga, gb = w.gb, active = w.active, split = w.split;
    const int seen_by_all = min(w.first + 1, w.closed), hidden_to_some = a.window > 0 ? w.last - a.window + 1 : 0;

    const int seg_groups = kSegment >> (6 - a.page_log2);
    PageNumbers<THREADS> pages;
    pages.request(a, w, ga << (6 - a.page_log2), min(gb - ga, seg_groups) << (6 - a.page_log2));
    float scale[RT];           // of logits in the exponent's base
    int position[RT];          // of the lane's row; -1 where there is none
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = 16 * rt + c, i = r / p.gq;
        position[rt] = i < w.n ? w.first + i : -1;
        h8v q[4];
        scale[rt] = query_fragments<BF, true>(query_at(a, w, h, r), i < w.n, kb, a.logit_scale, q);
        if (wave == 0) {       // (in LDS: a wave reads a fragment once for all tokens of a group)
#pragma unroll
            for (int s = 0; s < 4; ++s) sh.run.q[rt][s][lane] = q[s];
        }
    }
    Sums<RT> st;
    st.clear();

    float v_top = two_to(-126);        // values are accumulated over the largest scale so far, divided by kValueLift
    Segment& seg = sh.run.seg;
    for (int s0 = ga; s0 < gb; s0 += seg_groups) {
        const int s1 = min(s0 + seg_groups, gb);
        __syncthreads();
        if (threadIdx.x == 0) s_top = __float_as_uint(v_top);
        if (s0 > ga) pages.request(a, w, s0 << (6 - a.page_log2), (s1 - s0) << (6 - a.page_log2));
        const bool holes = pages.put(seg);

        u4v kw[8], vw[8];
        auto load_keys = [&](int g) {
            const int token = 16 * (c >> 2) + (c & 3), at = (g - s0) * 64 + token;
            const int page = max(seg.page[at >> a.page_log2], 0);
            const uint8_t* k = p.k_codes + (((int64_t)page * p.n_kv_heads + h) * P + (at & (P - 1))) * kHeadDim + 16 * kb;
            if constexpr (ONCE) {
#pragma unroll
                for (int t = 0; t < 8; ++t) kw[t] = __builtin_nontemporal_load(reinterpret_cast<const u4v*>(k + 4 * (t >> 1) * kHeadDim + 64 * (t & 1)));
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t) kw[t] = *reinterpret_cast<const u4v*>(k + 4 * (t >> 1) * kHeadDim + 64 * (t & 1));
            }
        };
        auto load_values = [&](int g) {
            const int at = (g - s0) * 64 + 16 * kb;
            const int page = max(seg.page[at >> a.page_log2], 0);
            const uint8_t* v = p.v_codes + ((int64_t)page * p.n_kv_heads + h) * (P * kHeadDim) + c * P + (at & (P - 1));
            if constexpr (ONCE) {
#pragma unroll
                for (int t = 0; t < 8; ++t) vw[t] = __builtin_nontemporal_load(reinterpret_cast<const u4v*>(v + 16 * t * P));
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t) vw[t] = *reinterpret_cast<const u4v*>(v + 16 * t * P);
            }
        };
        int g = s0 + wave;
        if (g < s1) { load_keys(g); load_values(g); }
        const float top = look_up_scales<THREADS, INT8>(a, h, v_top, seg, pages, &s_top);
        if (top > v_top) {
            st.times(v_top / top);
            v_top = top;
        }
        const float v_over = 1.f / v_top;
        // (more: whether the wave has another group.  The last step is a copy of its own: behind a branch the compiler would not know how many loads are
        // on their way, and wait for the values that were requested last before it takes the keys)
        auto step = [&](auto more) {
            const int at = ((g - s0) * 64 + 16 * kb) >> a.page_log2;       // the page of the lane's 16 tokens
            const float ks = seg.k_scale[at], vs = seg.v_scale[at] * v_over;
            const bool there = seg.page[at] >= 0;
            const bool edge = holes || 64 * g < hidden_to_some || 64 * g + 64 > seen_by_all;
            if (edge && !there) {      // (nothing was stored there: it may hold NaN)
#pragma unroll
                for (int t = 0; t < 8; ++t) vw[t] = u4v{0, 0, 0, 0};
            }
            // Half of the tokens at a time, tokens 16 kb + 8 half .. + 7 of a lane: fewer registers.
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f4v x[RT][2];
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    h8v q[RT];
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) q[rt] = sh.run.q[rt][s][lane];
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const u4v y = kw[2 * (2 * half + t) + (s >> 1)];
                        const h8v k = halves_of_codes<INT8>(y[2 * (s & 1)], y[2 * (s & 1) + 1], 1.f);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) x[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[rt], s ? x[rt][t] : kZero, 0, 0, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);      // (what is converted ahead of its product costs registers)
                }
                if (half == 1 && decltype(more)::value) load_keys(g + NW);
                Weights<!BF> e[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    if (edge) {
                        const int low = a.window > 0 ? position[rt] - a.window : -1;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int token = 64 * g + 16 * kb + 8 * half + j;
                            const bool hidden = !there | (token > position[rt]) | (token <= low);
                            x[rt][j >> 2][j & 3] = hidden ? -INFINITY : x[rt][j >> 2][j & 3];
                        }
                    }
                    e[rt].put(st.weigh(rt, x[rt], logit_factor(ks, scale[rt])));
                }
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const h8v v = halves_of_codes<INT8>(vw[t][2 * half], vw[t][2 * half + 1], vs);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) st.o[rt][t] = e[rt].product(v, st.o[rt][t]);
                    if (t & 1) __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (decltype(more)::value) load_values(g + NW);
        };
        for (; g + NW < s1; g += NW) step(std::true_type{});
        if (g < s1) step(std::false_type{});
    }
    st.times(v_top);
    __syncthreads();
    const int slot = w.open > 0 && split == active - 1 ? slot_of(p, w.seq.b) : -1;
    if (slot >= 0 && wave == (gb - ga) % NW) {       // (a wave that has the fewest groups)
        stage_open_values(a, w, h, slot, sh.open_v, lane, 64);
        __builtin_amdgcn_wave_barrier();
        attend_open<BF>(a, w, h, slot, sh.open_v, 0, st);
    }
    __syncthreads();

    // ---- the waves' results together ----
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float sum = st.sum(rt);
        if (kb == 0) { sh.join.ref[wave][16 * rt + c] = st.reference(rt); sh.join.sum[wave][16 * rt + c] = sum; }
    }
    __syncthreads();
    const int rows = w.n * p.gq;
    const Partials parts(a, w.part_of_head(a, h), active, RT);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float top = kLowest, total = 0.f;
        for (int v = 0; v < NW; ++v) top = fmaxf(top, sh.join.ref[v][16 * rt + c]);
        for (int v = 0; v < NW; ++v) total = __builtin_fmaf(sh.join.sum[v][16 * rt + c], __builtin_amdgcn_exp2f(sh.join.ref[v][16 * rt + c] - top), total);
        const float f = __builtin_amdgcn_exp2f(st.reference(rt) - top);
        if (rt) __syncthreads();
#pragma unroll
        for (int t = 0; t < 8; ++t) sh.join.o[wave][t][lane] = st.o[rt][t] * f;
        __syncthreads();
        const int r = 16 * rt + c;
        if (wave == 0 && kb == 0) {
            if (active > 1) parts.put_state(split, r, top, total);
            else if (a.lse && r < rows) a.lse[result_at(a, w, h, r)] = log_sum(top, total);
        }
        for (int t = wave; t < 8; t += NW) {
            f4v x = {0.f, 0.f, 0.f, 0.f};
            for (int v = 0; v < NW; ++v) x += sh.join.o[v][t][lane];
            if (active > 1) parts.put_output(split, (8 * rt + t) * 64 + lane, x);
            else if (r < rows) store_out<BF>(a, w, h, r, t, kb, x, inverse_sum(total));
        }
    }
    if (active > 1) join_splits<BF, RT>(a, w, h, parts, &s_last);
}

// ---- many rows: the rows are split over waves, which share the tokens ----
//
// Each of four waves has 32 rows to itself and goes over all tokens of its workgroup, 64 at a time.  Codes become binary16 numbers once, on their way
// into LDS, where the next tile is built beside the one in use, and the codes of the one after it are on their way; products and layouts are those of the kernel above.
//
// A prompt of 8192 tokens, 32 heads: 590 us (bfloat16), 0.93 PFLOP/s (a large matrix product reaches 1.19); binary16, whose weights are two numbers, 707 to 750 on four
// cards.  A wave takes 2600 to 3000 cycles for 64 tokens of its 32 rows (binary16: 3200 and more): 1024 (1536) of matrix instructions, 512 of exponentials, 900 (1030) of other vector
// instructions, and the two waves of a SIMD overlap these little.  With weights of one number, which took 580 to 590, no difference made, or longer: operands read from LDS a phase
// ahead (580), the second half's key product before the first half's exponentials in one block (713: it spills), three waves a SIMD with one tile in LDS (1183: it
// spills), wave priorities for either phase (606, 620).  32 rows a wave, because each fragment read from LDS then meets two row tiles: LDS is busy for 34 to 42 % of the time.
constexpr int kTileWaves = 4, kTileRows = 2;
struct TilesShared {
    union {
        struct { h8v k[2][64 * 16], v[2][64 * 16]; } tile;
        OpenValues open_v;
    };
    Segment seg;
};
// Where 8 channels (chunk) of a key, and 8 tokens (chunk) of a channel, lie in a tile: any eight lanes that read (consecutive rows) or write (the two chunks
// of a thread's 16 bytes one after the other, whatever the page size) at the same time meet all eight places of 128 bytes.
__device__ __forceinline__ int key_place(int row, int chunk) { return row * 16 + ((chunk >> 1 | (chunk & 1) << 3) ^ (row & 7)); }
__device__ __forceinline__ int value_place(int channel, int chunk) {
    const int line = channel >> 1;
    return line * 16 + ((chunk >> 1 | (channel & 1) << 2 | (chunk & 1) << 3) ^ ((line & 1) << 1 | (line >> 1 & 1)));
}

template <bool BF, bool INT8>
__global__ __launch_bounds__(64 * kTileWaves, 2) void paged_tiles(const AttnArgs a) {
    constexpr int NW = kTileWaves, RT = kTileRows, THREADS = 64 * NW;
    __shared__ TilesShared sh;
    __shared__ Sequence s_slot;
    __shared__ int s_last;
    __shared__ unsigned int s_top;
    const PageArgs& p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, kb = lane >> 4, P = 1 << a.page_log2;
    // Heads take turns (with eight of them each die has one head's pages in its L2); later pieces, which see more, begin first.
    const int h = blockIdx.x % p.n_kv_heads;
    Range w;
    if (!w.find(a, a.slots - 1 - blockIdx.x / p.n_kv_heads, &s_slot)) return;
    const int ga = w.ga, gb = w.gb, active = w.active, split = w.split;

    const int r0 = 16 * RT * wave, rows = w.n * p.gq;
    // (of this wave's rows; a wave without any sees nothing)
    const int my_first = w.first + r0 / p.gq, my_last = r0 < rows ? w.first + (min(r0 + 16 * RT, rows) - 1) / p.gq : -1;
    const int seen_by_all = min(my_first + 1, w.closed), hidden_to_some = a.window > 0 ? my_last - a.window + 1 : 0, my_lo = a.window > 0 ? my_first - a.window + 1 : 0;
    const int seg_groups = kSegment >> (6 - a.page_log2);
    PageNumbers<THREADS> pages;
    pages.request(a, w, ga << (6 - a.page_log2), min(gb - ga, seg_groups) << (6 - a.page_log2));
    h8v q[RT][4];
    float scale[RT];
    int position[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = r0 + 16 * rt + c, i = r / p.gq;
        position[rt] = i < w.n ? w.first + i : -1;
        scale[rt] = query_fragments<BF, false>(query_at(a, w, h, r), i < w.n, kb, a.logit_scale, q[rt]);
    }
    Sums<RT> st;
    st.clear();

    float v_top = two_to(-126);
    Segment& seg = sh.seg;
    for (int s0 = ga; s0 < gb; s0 += seg_groups) {
        const int s1 = min(s0 + seg_groups, gb);
        __syncthreads();
        if (threadIdx.x == 0) s_top = __float_as_uint(v_top);
        if (s0 > ga) pages.request(a, w, s0 << (6 - a.page_log2), (s1 - s0) << (6 - a.page_log2));
        const bool holes = pages.put(seg);

        // A thread's share of a tile: 16 bytes of two keys, and 16 tokens of two channels.
        u4v kw[2], vw[2];
        // (a wave's 64 pieces are of one page whatever the page size, so a page's place is worked out by scalar instructions)
        auto key_token = [&](int u) { return (threadIdx.x + THREADS * u) >> 3; };
        auto value_bytes = [&](int u) { return (threadIdx.x + THREADS * u) * 16; };      // into the tile's pages, [channel][P] each
        auto page_place = [&](int g, int u) { return ((g - s0) * 64 + 8 * wave + 32 * u) >> a.page_log2; };      // in the segment, of keys and values alike
        auto request = [&](int g) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int64_t block = ((int64_t)max(__builtin_amdgcn_readfirstlane(seg.page[page_place(g, u)]), 0) * p.n_kv_heads + h) * (P * kHeadDim);
                const uint8_t *k = p.k_codes + block, *v = p.v_codes + block;
                kw[u] = *reinterpret_cast<const u4v*>(k + (uint32_t)((key_token(u) & (P - 1)) * kHeadDim + 16 * (threadIdx.x & 7)));
                vw[u] = *reinterpret_cast<const u4v*>(v + (uint32_t)(value_bytes(u) & (P * kHeadDim - 1)));
            }
        };
        float v_over;
        auto build = [&](int g) {
            h8v* k = sh.tile.k[(g - s0) & 1];
            h8v* v = sh.tile.v[(g - s0) & 1];
            const bool gaps = holes || 64 * (g + 1) > w.closed || 64 * g < w.lo;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                // (the order of a tile's rows: the kernel above)
                const int token = key_token(u), row = 16 * ((token >> 2) & 3) + 4 * (token >> 4) + (token & 3), m = threadIdx.x & 7;
                k[key_place(row, 2 * m)] = halves_of_codes<INT8>(kw[u][0], kw[u][1], 1.f);
                k[key_place(row, 2 * m + 1)] = halves_of_codes<INT8>(kw[u][2], kw[u][3], 1.f);
                const int part = value_bytes(u) >> (a.page_log2 + 7), in = value_bytes(u) & (P * kHeadDim - 1), page_at = page_place(g, u);
                const float vs = seg.v_scale[page_at] * v_over;
                u4v y = vw[u];
                if (gaps && seg.page[page_at] < 0) y = u4v{0, 0, 0, 0};      // (nothing was stored there: it may hold NaN)
                const int channel = in >> a.page_log2, chunk = ((part << a.page_log2) + (in & (P - 1))) >> 3;
                v[value_place(channel, chunk)] = halves_of_codes<INT8>(y[0], y[1], vs);
                v[value_place(channel, chunk + 1)] = halves_of_codes<INT8>(y[2], y[3], vs);
            }
        };
        // (requests behind the last tile repeat it: without a branch the compiler knows how many loads are on their way)
        request(s0);
        const float top = look_up_scales<THREADS, INT8>(a, h, v_top, seg, pages, &s_top);
        if (top > v_top) {
            st.times(v_top / top);
            v_top = top;
        }
        v_over = 1.f / v_top;
        build(s0);
        request(min(s0 + 1, s1 - 1));
        __syncthreads();
        for (int g = s0; g < s1; ++g) {
            if (64 * g <= my_last && 64 * g + 63 >= my_lo) {
                const h8v* k_tile = sh.tile.k[(g - s0) & 1];
                const h8v* v_tile = sh.tile.v[(g - s0) & 1];
                const int at = ((g - s0) * 64 + 16 * kb) >> a.page_log2;
                const float ks = seg.k_scale[at];
                const bool there = seg.page[at] >= 0;
                float factor[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) factor[rt] = logit_factor(ks, scale[rt]);
                const bool edge = holes || 64 * g < hidden_to_some || 64 * g + 64 > seen_by_all;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    f4v x[RT][2];
#pragma unroll
                    for (int s = 0; s < 4; ++s)
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            const h8v k = k_tile[key_place(16 * (2 * half + t) + c, 4 * s + kb)];
#pragma unroll
                            for (int rt = 0; rt < RT; ++rt) x[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[rt][s], s ? x[rt][t] : kZero, 0, 0, 0);
                        }
                    Weights<!BF> e[RT];
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        if (edge) {
                            const int low = a.window > 0 ? position[rt] - a.window : -1;
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const int token = 64 * g + 16 * kb + 8 * half + j;
                                const bool hidden = !there | (token > position[rt]) | (token <= low);
                                x[rt][j >> 2][j & 3] = hidden ? -INFINITY : x[rt][j >> 2][j & 3];
                            }
                        }
                        e[rt].put(st.weigh(rt, x[rt], factor[rt]));
                    }
#pragma unroll
                    for (int t = 0; t < 8; ++t) {
                        const h8v v = v_tile[value_place(16 * t + c, 2 * kb + half)];
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) st.o[rt][t] = e[rt].product(v, st.o[rt][t]);
                    }
                }
            }
            if (g + 1 < s1) build(g + 1);
            request(min(g + 2, s1 - 1));
            __syncthreads();
        }
    }
    st.times(v_top);
    const int slot = w.open > 0 && split == active - 1 ? slot_of(p, w.seq.b) : -1;
    if (slot >= 0) {
        __syncthreads();
        stage_open_values(a, w, h, slot, sh.open_v, threadIdx.x, THREADS);
        __syncthreads();
        if (my_last >= w.begin) attend_open<BF>(a, w, h, slot, sh.open_v, r0, st);
    }
    const Partials parts(a, w.part_of_head(a, h), active, RT * NW);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float total = st.sum(rt);
        const int r = r0 + 16 * rt + c;
        if (kb == 0) {
            if (active > 1) parts.put_state(split, r, st.reference(rt), total);
            else if (a.lse && r < rows) a.lse[result_at(a, w, h, r)] = log_sum(st.reference(rt), total);
        }
        const float by = inverse_sum(total);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            if (active > 1) parts.put_output(split, (8 * (RT * wave + rt) + t) * 64 + lane, st.o[rt][t]);
            else if (r < rows) store_out<BF>(a, w, h, r, t, kb, st.o[rt][t], by);
        }
    }
    if (active > 1) join_splits<BF, RT * NW>(a, w, h, parts, &s_last);
}

template <bool BF, bool INT8>
hipError_t paged_form(const AttnArgs& a, int row_tiles, hipStream_t stream) {
    const dim3 grid((unsigned)a.slots * a.p.n_kv_heads), threads(256);
    if (row_tiles == 1 && a.once) paged_rows<BF, INT8, 1, true><<<grid, threads, 0, stream>>>(a);
    else if (row_tiles == 1) paged_rows<BF, INT8, 1, false><<<grid, threads, 0, stream>>>(a);
    else if (row_tiles == 2) paged_rows<BF, INT8, 2, false><<<grid, threads, 0, stream>>>(a);
    else paged_tiles<BF, INT8><<<grid, threads, 0, stream>>>(a);
    return hipGetLastError();
}
template hipError_t paged_form<(KVQP_PAGED_BITS - 1) / 2 != 0, (KVQP_PAGED_BITS - 1) % 2 != 0>(const AttnArgs&, int, hipStream_t);

#else

// ---- launches ----
constexpr size_t kPartBytes = 8192 + 2 * 128;       // a workgroup's results of 16 rows
struct PagedPlan {
    int row_tiles, per_piece, slots, most_shares, at_once;
    size_t ws_bytes;
};
// Shares in all, where three, two and two workgroups fit a CU: more of them even out lengths and make more to join.  256, 384, 512 of one tile: 48 sequences of 1 .. 8192
// tokens 94, 107, 88 us, 8 of 4096 20.9, 21.0, 20.1, one of 1024 9.6, 9.7, 9.9.  384, 512, 768 of two: 64 rows of 48 sequences 232, 213, 200, of 4 sequences
// 34, 30, 47.  256, 384, 512 of tiles: a piece in a window 73, 63, 80, 4 x 256 rows 115, 88, 106.  (With more than 384 heads many rows are not split.)
static int shares_of(const kvqp_cfg& cfg, int row_tiles) { return (row_tiles == 8 ? 384 : 512) / cfg.n_kv_heads; }
static size_t workspace_of(const kvqp_cfg& cfg, int row_tiles, int shares) {
    return shares ? KVQP_PAGED_COUNTERS + (size_t)cfg.n_kv_heads * 2 * shares * row_tiles * kPartBytes : 0;
}
static PagedPlan plan_paged(const kvqp_cfg& cfg, int n_rows, bool has_starts, int64_t most_tokens) {
    // (rows of a call over its sequences, as if they were equal.  Columns: a KV head's rows of a sequence.  One tile of 16 rows where they fit, for a third wave a
    // SIMD; 64 columns as two workgroups of 32 take 212 us where the kernel of many rows, half of its rows empty, takes 208 to 303)
    const int gq = cfg.n_q_heads / cfg.n_kv_heads, each = (n_rows + cfg.batch - 1) / cfg.batch, columns = each >= 128 ? 128 : each * gq;
    PagedPlan r;
    r.row_tiles = columns > 64 ? 8 : columns > 16 ? 2 : 1;
    r.per_piece = 16 * r.row_tiles / gq;
    const int pieces = has_starts ? n_rows / r.per_piece + cfg.batch : cfg.batch;      // (at most: each sequence's last may be short)
    r.most_shares = shares_of(cfg, r.row_tiles);
    if (most_tokens <= 64 * kLeastGroups || cfg.batch > kMostSplitBatch) r.most_shares = 0;
    r.at_once = r.most_shares ? 512 / cfg.n_kv_heads : 0;
    r.slots = pieces + std::max(r.most_shares, r.at_once);
    r.ws_bytes = workspace_of(cfg, r.row_tiles, r.most_shares);
    return r;
}
// (of this plan and those of fewer rows, which may have fewer tiles and, with more than 384 heads, need more)
size_t paged_workspace_bound(const kvqp_cfg& cfg, int n_rows) {
    const PagedPlan most = plan_paged(cfg, n_rows, true, INT64_MAX);
    size_t bytes = KVQP_PAGED_COUNTERS;
    if (cfg.batch <= kMostSplitBatch)
        for (int tiles : {1, 2, 8})
            if (tiles <= most.row_tiles) bytes = std::max(bytes, workspace_of(cfg, tiles, shares_of(cfg, tiles)));
    return bytes;
}
int64_t paged_attn_workgroups(const kvqp_cfg& cfg, const kvqp_pages& g, int n_rows, bool has_starts) {
    return (int64_t)plan_paged(cfg, n_rows, has_starts, (int64_t)g.max_pages * g.page_tokens).slots * cfg.n_kv_heads;
}
size_t paged_workspace_need(const kvqp_cfg& cfg, const kvqp_pages& g, int n_rows, bool has_starts) {
    return plan_paged(cfg, n_rows, has_starts, (int64_t)g.max_pages * g.page_tokens).ws_bytes;
}

PageArgs page_args(const kvqp_cfg& cfg, const kvqp_pages& g, const int32_t* row_start, int n_rows);

// Whether a step's codes are more than what may stay in the memory-side cache, as far as the host knows: the pages that the sequences can have.  Loads past it
// save what allocating there costs where nothing is read again before it is gone (past it and not, three caches of one size in turn: 32 x 8192 tokens of 8 heads, 512 MB,
// 97 and 103 us; 256 MB 55 and 57; 128 MB 33 and 34; 94 MB 27 and 26; 64 MB 21 and 20).  Where 17 .. 64 rows are, pieces read each other's codes from there, and none go past it.
static bool rows_once(const kvqp_cfg& cfg, const kvqp_pages& g) {
    if (cfg.decode_cache_hint != KVQP_CACHE_AUTO) return cfg.decode_cache_hint == KVQP_CACHE_STREAM;
    return std::min((double)g.n_pages, (double)cfg.batch * g.max_pages) * g.page_tokens * cfg.n_kv_heads * 2 * kHeadDim > 96.0 * (1 << 20);
}

hipError_t launch_paged_attn(const kvqp_cfg& cfg, const kvqp_pages& g, const void* q, int64_t q_stride, int n_rows, const int32_t* row_start, int window,
                             void* out, float* lse, void* ws, hipStream_t stream) {
    const PagedPlan plan = plan_paged(cfg, n_rows, row_start != nullptr, (int64_t)g.max_pages * g.page_tokens);
    const AttnArgs a = {page_args(cfg, g, row_start, n_rows), (const uint16_t*)q, q_stride, (uint16_t*)out, lse, (unsigned int*)ws,
                        (char*)ws + KVQP_PAGED_COUNTERS, cfg.sm_scale * 1.4426950408889634f, (int64_t)window < (int64_t)g.max_pages * g.page_tokens ? window : 0, g.page_tokens == 16 ? 4 : g.page_tokens == 32 ? 5 : 6,
                        plan.per_piece, plan.slots, plan.most_shares, plan.at_once, rows_once(cfg, g)};
    if (g.dtype == KVQP_BFLOAT16)
        return g.form == KVQP_INT8 ? paged_form<true, true>(a, plan.row_tiles, stream) : paged_form<true, false>(a, plan.row_tiles, stream);
    return g.form == KVQP_INT8 ? paged_form<false, true>(a, plan.row_tiles, stream) : paged_form<false, false>(a, plan.row_tiles, stream);
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
