// Eviction from a packed cache by accumulated attention weight: the heaviest tokens of every head (or
// the heaviest units of neighbouring tokens) move, in their order, into another cache.
//
//   score[u] = float(sum over the unit's tokens of weight[t]), summed in binary64
//   kept     = the m highest scores, equal ones going to the lower unit, in ascending order
//
// Two launches.  pick_heaviest finds the cut of one head per workgroup: a radix selection on 32-bit order keys (11 + 11 +
// 10 bits, a histogram in LDS each) and one ordered pass that writes the survivors; up to 256 units are ranked by counting
// instead, and for small caches the second launch does that, too.  move_tokens gathers: nothing is rounded anew -- codes,
// scales and zeros of values, of keys per token and of whole key groups are copied bit by bit, value codes from and into
// the tile-transposed words -- except where tokens of different key groups form a new one (keys per channel, units smaller
// than a group): those keys are read back as binary16 numbers and quantized again, by the cache's quantizer.  (A new group
// whose tokens were one group before is copied too: what lies before the first token that leaves is never touched.)
// Many heads are bound by memory: the survivors' bytes are read and written once (a value word holds 4 to 16 tokens, so
// what lies between survivors comes along).  256 heads of 8192 tokens to 6144, 4 bits: 110.8 us for 533 MB, 4.8 TB/s of the
// 5.2 that a large copy reaches, behind 12.4 us of selection.  Few heads are bound by latency, keys that are quantized again
// by vector instructions (16 heads of 12003 tokens to 8001, 2 bits: 12 + 18.6 us, vector ALUs 90 % busy, where 27 MB would take 5; a key code takes
// 24 of them, nine for its group's minimum and maximum and eight to be quantized again, a value field eight).
#include <type_traits>

#include "kvqp_internal.h"

namespace kvqp {
namespace {

constexpr int kBins = 2048;
constexpr int kMoveThreads = 256;

struct EvictArgs {
    kvqp_cache src, dst;
    const float* weights;
    float* weights_out;
    int32_t* idx;             // [heads, bound]
    int32_t* list;            // the same for the caller, or NULL
    long long w_cap, w_cap_out;
    int n_kept, src_cap, dst_cap;
    int n_keep, unit, bound;
    int group_log2, token_blocks;
};

__device__ __forceinline__ int source_tokens(const EvictArgs& a, int bh) {
    if (!a.src.head_n_kept) return a.n_kept;
    const int n = a.src.head_n_kept[bh];
    return n < 0 ? 0 : (n > a.n_kept ? a.n_kept : n);
}
// Tokens of the incomplete last unit, which always stays, and whole units that stay beside it.
struct Cut { int short_unit, units, keep_units, kept; };
__host__ __device__ inline Cut cut_of(int n, int n_keep, int unit) {
    Cut c;
    c.short_unit = n % unit;
    c.units = n / unit;
    c.keep_units = n <= n_keep ? c.units : (n_keep - c.short_unit) / unit;
    c.kept = c.keep_units * unit + c.short_unit;
    return c;
}

// Order key: higher for larger numbers, -0 as +0, NaN below everything.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    return x != x ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
// (a unit's weights are requested 32 at a time)
__device__ __forceinline__ uint32_t unit_key(const float* w, int u, int unit) {
    if (unit == 1) return order_key(w[u]);
    double sum = 0.0;
#pragma unroll 1
    for (int b = 0; b < unit; b += 32) {
        float x[32];
#pragma unroll
        for (int t = 0; t < 32; ++t) x[t] = w[u * unit + b + t];
#pragma unroll
        for (int t = 0; t < 32; ++t) sum += (double)x[t];
    }
    return order_key((float)sum);
}

// Sum of the first `wave` of at most 16 numbers in LDS.
__device__ __forceinline__ uint32_t waves_before(const uint32_t* s, int wave, int lane) {
    uint32_t v = (lane & 15) < wave ? s[lane & 15] : 0u;
    v += __builtin_amdgcn_update_dpp(0u, v, 0xB1 /* quad_perm [1,0,3,2] */, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0u, v, 0x4E /* quad_perm [2,3,0,1] */, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0u, v, 0x141 /* row_half_mirror */, 0xF, 0xF, true);
    return v + __builtin_amdgcn_update_dpp(0u, v, 0x140 /* row_mirror */, 0xF, 0xF, true);
}

// Sum over the lanes up to this one: within rows of 16 lanes, then the rows' totals.
__device__ __forceinline__ uint32_t lanes_up_to(uint32_t v) {
    v += __builtin_amdgcn_update_dpp(0u, v, 0x111 /* row_shr:1 */, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0u, v, 0x112 /* row_shr:2 */, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0u, v, 0x114 /* row_shr:4 */, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0u, v, 0x118 /* row_shr:8 */, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0u, v, 0x142 /* row_bcast:15 */, 0xA, 0xF, false);
    return v + __builtin_amdgcn_update_dpp(0u, v, 0x143 /* row_bcast:31 */, 0xC, 0xF, false);
}
// Lanes below this one whose bit is set, and `more`.
__device__ __forceinline__ uint32_t lanes_below(unsigned long long bits, uint32_t more) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)bits, more));
}
constexpr uint32_t kOddTurn = 16u;       // the odd lanes' histogram has its bins this far apart from the others', in other banks

// The same for up to 256 units a head: a thread counts the units that come before its own, by score and then by position.
// (Whole evictions of 8 heads, and by the selection below: 33 units of 32 tokens 7.7 us and 10.3, 256 of 32 tokens 13.6 and 15.4, 256 single
// tokens 9.1 and 8.7.)
constexpr int kFewUnits = 256;
struct FewUnits {
    uint4 key[kFewUnits / 4];
    int unit[kFewUnits];            // those that stay, in order
    uint32_t wave[4];
};
__device__ __forceinline__ void rank_few(const EvictArgs& a, int bh, const Cut& cut, FewUnits& s) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t key = tid < cut.units ? unit_key(a.weights + (size_t)bh * a.w_cap, tid, a.unit) : 0u;
    reinterpret_cast<uint32_t*>(s.key)[tid] = key;
    __syncthreads();
    uint32_t before = 0u;
#pragma unroll 1
    for (int b = 0; 64 * b < cut.units; ++b) {           // (keys past the last unit are 0, and come after every unit)
        const uint4* keys = s.key + 16 * b;
        if (b != wave) {          // (equal keys of lower units come before this one, those of higher ones after it)
            const uint32_t least = key + (b > wave);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const uint4 k = keys[j];
                before += (k.x >= least) + (k.y >= least) + (k.z >= least) + (k.w >= least);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const uint4 k = keys[j];
                before += (k.x >= key + (4 * j >= lane)) + (k.y >= key + (4 * j + 1 >= lane)) + (k.z >= key + (4 * j + 2 >= lane)) + (k.w >= key + (4 * j + 3 >= lane));
            }
        }
    }
    const bool stays = tid < cut.units && before < (uint32_t)cut.keep_units;
    const unsigned long long all = __builtin_amdgcn_ballot_w64(stays);
    if (lane == 0) s.wave[wave] = (uint32_t)__builtin_popcountll(all);
    __syncthreads();
    uint32_t at = lanes_below(all, 0u);
    for (int w = 0; w < wave; ++w) at += s.wave[w];
    if (stays) s.unit[at] = tid;
    __syncthreads();
}
// The token of place i
__device__ __forceinline__ int token_at(const EvictArgs& a, const Cut& cut, const FewUnits& s, int i) {
    const int whole = cut.keep_units * a.unit;
    return i < whole ? s.unit[i >> __builtin_ctz(a.unit)] * a.unit + (i & (a.unit - 1)) : cut.units * a.unit + i - whole;
}
__global__ __launch_bounds__(kFewUnits) void pick_of_few(const EvictArgs a) {
    __shared__ FewUnits s;
    const int bh = blockIdx.x;
    const Cut cut = cut_of(source_tokens(a, bh), a.n_keep, a.unit);
    rank_few(a, bh, cut, s);
    for (int i = threadIdx.x; i < cut.kept; i += kFewUnits) {
        const int t = token_at(a, cut, s, i);
        a.idx[(size_t)bh * a.bound + i] = t;
        if (a.list) a.list[(size_t)bh * a.bound + i] = t;
    }
    if (a.dst.head_n_kept && threadIdx.x == 0) a.dst.head_n_kept[bh] = cut.kept;
}

// One head per workgroup.  Every wave has a stretch of consecutive units, 64 at a time.  The keys of up to
// KEYS such steps stay in LDS (KEYS == 0: any number, read again in every pass).
template <int KEYS, int THREADS>
__global__ __launch_bounds__(THREADS) void pick_heaviest(const EvictArgs a) {
    constexpr int WAVES = THREADS / 64, PER = kBins / THREADS;
    __shared__ uint32_t s_hist[2][kBins];
    __shared__ uint32_t s_key[KEYS > 0 ? KEYS * THREADS : 1];
    __shared__ uint32_t s_wave[3][WAVES];
    __shared__ uint32_t s_found[3];
    const int bh = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = source_tokens(a, bh);
    const Cut cut = cut_of(n, a.n_keep, a.unit);
    const float* w = a.weights + (size_t)bh * a.w_cap;
    int32_t* idx = a.idx + (size_t)bh * a.bound;
    int32_t* list = a.list ? a.list + (size_t)bh * a.bound : nullptr;
    if (a.dst.head_n_kept && tid == 0) a.dst.head_n_kept[bh] = cut.kept;
    auto put = [&](int at, int token) {
        idx[at] = token;
        if (list) list[at] = token;
    };
    if (cut.keep_units == cut.units) {       // nothing leaves
        for (int t = tid; t < n; t += THREADS) put(t, t);
        return;
    }
    for (int t = tid; t < cut.short_unit; t += THREADS) put(cut.keep_units * a.unit + t, cut.units * a.unit + t);
    if (cut.keep_units == 0) return;

    const int steps = (cut.units + THREADS - 1) / THREADS, u0 = wave * steps * 64;
    uint32_t* own = s_key + wave * KEYS * 64 + lane;         // the lane's keys, 64 words apart
    if constexpr (KEYS > 0) {
        if (a.unit == 1) {       // (requested eight at a time: a branch per step would wait for each)
#pragma unroll 1
            for (int j0 = 0; j0 < steps; j0 += 8) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = w[min(u0 + 64 * (j0 + j) + lane, cut.units - 1)];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j0 + j < KEYS) own[64 * (j0 + j)] = order_key(x[j]);
            }
        } else {
#pragma unroll 1
            for (int j = 0; j < steps; ++j) own[64 * j] = u0 + 64 * j + lane < cut.units ? unit_key(w, u0 + 64 * j + lane, a.unit) : 0u;
        }
    }
    // body(unit, its key, whether there is such a unit) for the wave's units, in order.  (Four steps' keys are read together and the rest is
    // rolled up: every launch fetches its code anew, and keys in registers, with the loops unrolled, took 20 us instead of 15 for 16 heads of 12003.)
    const int u1 = min(u0 + 64 * steps, cut.units);
    auto each = [&](auto body) {
        constexpr int BATCH = KEYS > 4 ? 4 : 1;
#pragma unroll 1
        for (int j0 = 0; j0 < steps; j0 += BATCH) {
            uint32_t k[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int u = u0 + 64 * (j0 + j) + lane;
                k[j] = KEYS > 0 ? own[64 * (j0 + j)] : u < u1 ? unit_key(w, u, a.unit) : 0u;
            }
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int u = u0 + 64 * (j0 + j) + lane;
                body(u, k[j], u < u1);
            }
        }
    };

    // The leading bits of the last unit's key that stays, and how many of the units with those very bits do.  Mostly two passes tell them
    // apart: as soon as all units of a bin stay, the rest of their keys does not matter.
    uint32_t prefix = 0u, mask = 0u, want = (uint32_t)cut.keep_units;
#pragma unroll
    for (int b = 0; b < PER; ++b) s_hist[0][tid + b * THREADS] = s_hist[1][tid + b * THREADS] = 0u;
    __syncthreads();
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        uint32_t* hist = s_hist[pass & 1];
        // (the first pass finds few bins full: even and odd lanes have a histogram each, so that fewer of them wait for one counter)
        uint32_t* mine = pass == 0 && (lane & 1) ? s_hist[1] : hist;
        const uint32_t turn = pass == 0 && (lane & 1) ? kOddTurn : 0u;
        each([&](int, uint32_t k, bool valid) {
            if (valid && (k & mask) == prefix) atomicAdd(&mine[((k >> shift) & ((1u << bits) - 1u)) ^ turn], 1u);
        });
        __syncthreads();
        // bins from the highest down: thread t has PER of them
        uint32_t c[PER], all = 0u;
#pragma unroll
        for (int b = 0; b < PER; ++b) {
            const int bin = kBins - 1 - PER * tid - b;
            c[b] = hist[bin];
            hist[bin] = 0u;           // (for the pass after the next)
            if (pass == 0) {
                c[b] += s_hist[1][bin ^ kOddTurn];
                s_hist[1][bin ^ kOddTurn] = 0u;
            }
            all += c[b];
        }
        uint32_t before = lanes_up_to(all);
        if (lane == 63) s_wave[0][wave] = before;
        __syncthreads();
        before += waves_before(s_wave[0], wave, lane) - all;
#pragma unroll
        for (int b = 0; b < PER; ++b) {
            if (before < want && want <= before + c[b]) {
                s_found[0] = (uint32_t)(kBins - 1 - PER * tid - b); s_found[1] = want - before; s_found[2] = c[b];
            }
            before += c[b];
        }
        __syncthreads();
        prefix |= s_found[0] << shift;
        mask |= ((1u << bits) - 1u) << shift;
        want = s_found[1];
        if (want == s_found[2]) break;        // (uniform)
    }

    // How many stay in the stretches before this wave's, then its own in order.
    uint32_t above = 0u, equal = 0u;
    each([&](int, uint32_t k, bool valid) {
        above += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(valid && (k & mask) > prefix));
        equal += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(valid && (k & mask) == prefix));
    });
    if (lane == 0) { s_wave[1][wave] = above; s_wave[2][wave] = equal; }
    __syncthreads();
    above = waves_before(s_wave[1], wave, lane);
    equal = waves_before(s_wave[2], wave, lane);
    each([&](int u, uint32_t k, bool valid) {
        k &= mask;
        const unsigned long long ba = __builtin_amdgcn_ballot_w64(valid && k > prefix), be = __builtin_amdgcn_ballot_w64(valid && k == prefix);
        const uint32_t e = lanes_below(be, equal);
        const uint32_t at = lanes_below(ba, above) + min(e, want);
        if (valid && (k > prefix || (k == prefix && e < want))) {
            if (a.unit == 1) put((int)at, u);
            else
                for (int t = 0; t < a.unit; ++t) put((int)at * a.unit + t, u * a.unit + t);
        }
        above += (uint32_t)__builtin_popcountll(ba);
        equal += (uint32_t)__builtin_popcountll(be);
    });
}

__device__ __forceinline__ float half_to_float(uint32_t u) { return __half2float(__ushort_as_half((unsigned short)u)); }

// Where a token keeps its values (layout statement in kvqp.h): channel 16 tile + n is in word `word` + place(tile, n) of the head, BITS bits from bit `shift`.
struct ValuePlace { uint32_t word, shift; };
template <int BITS> __device__ __forceinline__ ValuePlace value_place(int t) {
    constexpr int kFields = 16 / BITS, kSb = v_superblock(BITS);
    const int low = t % kSb, run = 4 * (low / 32) + low % 4;
    return {(uint32_t)(t / kSb) * v_superblock_words(BITS) + (uint32_t)(low / 4 % 4 * 64 + run / kFields),
            (uint32_t)(16 * (low / 16 % 2) + BITS * (run % kFields))};
}

__device__ __forceinline__ uint32_t xor_rows(uint32_t v, bool far) {     // the lane 16 (far: 32) further
    const auto r = far ? __builtin_amdgcn_permlane32_swap(v, v, false, false) : __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return (threadIdx.x & (far ? 32 : 16)) ? r[0] : r[1];
}
typedef _Float16 h2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ h2v as_h2(uint32_t u) { union { uint32_t u; h2v h; } c; c.u = u; return c.h; }
__device__ __forceinline__ uint32_t as_u32(h2v h) { union { uint32_t u; h2v h; } c; c.h = h; return c.u; }

// One key group's parameters, by channel.
struct GroupParams { float zero, inv; };

// REGROUP: 0, or log2 of the group size where key groups are formed anew (a workgroup has whole ones).
// RANKS: every workgroup finds its head's survivors itself; idx is not there.
template <int BITS, int REGROUP, bool RANKS>
__global__ __launch_bounds__(kMoveThreads) void move_tokens(const EvictArgs a, int key_axis) {
    constexpr bool QUANT = BITS != 16;
    constexpr int TB = REGROUP == 7 ? 128 : 64, GROUPS = REGROUP ? TB >> REGROUP : 1;
    __shared__ int s_idx[TB];
    __shared__ ValuePlace s_place[TB];
    __shared__ uint32_t s_min[REGROUP ? 4 * GROUPS * 64 : 1], s_max[REGROUP ? 4 * GROUPS * 64 : 1];    // [wave][group][channel pair]
    __shared__ GroupParams s_par[REGROUP ? GROUPS * kHeadDim : 1];
    __shared__ std::conditional_t<RANKS, FewUnits, char> s_few;
    const int bh = blockIdx.y, tid = threadIdx.x;
    const int n_src = source_tokens(a, bh);
    const Cut cut = cut_of(n_src, a.n_keep, a.unit);
    const int kept = cut.kept;
    if ((int)blockIdx.x >= a.token_blocks) {
        // the tail, its weights, and zeros for tokens to come
        if (RANKS && a.dst.head_n_kept && tid == 0) a.dst.head_n_kept[bh] = kept;
        const size_t from = (size_t)bh * a.src.tail_cap * kHeadDim, to = (size_t)bh * a.dst.tail_cap * kHeadDim;
        for (int i = tid; i < a.src.tail_len * 16; i += kMoveThreads) {
            reinterpret_cast<uint4*>((uint16_t*)a.dst.tail_k + to)[i] = reinterpret_cast<const uint4*>((const uint16_t*)a.src.tail_k + from)[i];
            reinterpret_cast<uint4*>((uint16_t*)a.dst.tail_v + to)[i] = reinterpret_cast<const uint4*>((const uint16_t*)a.src.tail_v + from)[i];
        }
        if (a.weights_out) {
            const float* w = a.weights + (size_t)bh * a.w_cap + n_src;
            float* o = a.weights_out + (size_t)bh * a.w_cap_out;
            for (long long i = kept + tid; i < a.w_cap_out; i += kMoveThreads) o[i] = i - kept < a.src.tail_len ? w[i - kept] : 0.0f;
        }
        return;
    }
    const int t0 = blockIdx.x * TB;
    if (t0 >= kept) return;
    const int ntok = min(TB, kept - t0), rows = rows32(ntok);
    if constexpr (RANKS) rank_few(a, bh, cut, s_few);
    if (tid < TB) {
        const int i = t0 + min(tid, ntok - 1);
        int t;
        if constexpr (RANKS) {
            t = token_at(a, cut, s_few, i);
            if (a.list) a.list[(size_t)bh * a.bound + i] = t;
        } else {
            t = a.idx[(size_t)bh * a.bound + i];
        }
        s_idx[tid] = t;
        s_place[tid] = value_place<BITS>(t);
    }
    __syncthreads();

    // Everything is requested before anything is stored: one trip to memory for a workgroup, not one per kind of data
    // (256 heads of 8192 tokens to 6144, 4 bits: 211 us with a trip for each, 113 this way).
    float weight = 0.0f;
    if (a.weights_out && tid < ntok) weight = a.weights[(size_t)bh * a.w_cap + s_idx[tid]];
    // scales and zeros that belong to tokens: 4, 2 or 1 numbers a token and array; a thread has one token of one or two of four arrays
    constexpr int META = QUANT ? (4 * TB) / kMoveThreads : 0;
    const int cg_log2 = 7 - a.group_log2;
    uint2 meta[META > 0 ? META : 1];
    const uint16_t* const meta_src[4] = {(const uint16_t*)a.src.v_scale, (const uint16_t*)a.src.v_zero, (const uint16_t*)a.src.k_scale, (const uint16_t*)a.src.k_zero};
    uint16_t* const meta_dst[4] = {(uint16_t*)a.dst.v_scale, (uint16_t*)a.dst.v_zero, (uint16_t*)a.dst.k_scale, (uint16_t*)a.dst.k_zero};
    const int arrays = key_axis == KVQP_KEY_PER_TOKEN ? 4 : 2;
#pragma unroll
    for (int m = 0; m < META; ++m) {
        const int item = m * kMoveThreads + tid, which = item / TB, t = item % TB;
        meta[m] = make_uint2(0u, 0u);
        if (which < arrays && t < ntok) {
            const uint16_t* p = (which == 0 ? meta_src[0] : which == 1 ? meta_src[1] : which == 2 ? meta_src[2] : meta_src[3]) +
                                (((size_t)bh * a.src_cap + s_idx[t]) << cg_log2);
            if (cg_log2 == 2) meta[m] = *reinterpret_cast<const uint2*>(p);
            else if (cg_log2 == 1) meta[m].x = *reinterpret_cast<const uint32_t*>(p);
            else meta[m].x = *p;
        }
    }
    // key code rows: BITS pieces of 16 bytes
    constexpr int PIECES = REGROUP ? 0 : TB * BITS / kMoveThreads;
    uint4 piece[PIECES > 0 ? PIECES : 1];
    if constexpr (!REGROUP) {
        const uint4* f = (const uint4*)a.src.k_codes + (size_t)bh * a.src_cap * BITS;
#pragma unroll
        for (int i = 0; i < (PIECES > 0 ? PIECES : 1); ++i) {
            const int item = i * kMoveThreads + tid, t = item / BITS;
            piece[i] = make_uint4(0u, 0u, 0u, 0u);
            if (t < ntok) piece[i] = f[(size_t)s_idx[t] * BITS + item % BITS];
        }
    }
    // value codes: a thread makes WORDS words of E fields each
    constexpr int SB = v_superblock(BITS), SBW = v_superblock_words(BITS), WPT = v_words_per_tile(BITS), E = 32 / BITS, HALF = E / 2;
    constexpr int WORDS = TB / SB * SBW / kMoveThreads;
    const uint32_t* vs = (const uint32_t*)a.src.v_codes + (size_t)bh * (size_t)((a.src_cap + SB - 1) / SB) * SBW;
    uint32_t* vd = (uint32_t*)a.dst.v_codes + ((size_t)bh * (size_t)((a.dst_cap + SB - 1) / SB) + t0 / SB) * SBW;
    uint32_t got[WORDS][E];
    auto token_of = [&](int w, int e) {       // which of the workgroup's tokens field e of the thread's word w holds
        const int i = w * kMoveThreads + tid, y = i % SBW / 256 * 4 + i % 4, kb = i / 64 % 4, run = y % WPT * HALF + e % HALF;
        return i / SBW * SB + 32 * (run / 4) + 16 * (e / HALF) + 4 * kb + run % 4;
    };
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
        const int i = w * kMoveThreads + tid, y = i % SBW / 256 * 4 + i % 4;
        const uint32_t place = (uint32_t)(y / WPT * WPT / 4 * 256 + i / 4 % 16 * 4 + y / WPT * WPT % 4);
#pragma unroll
        for (int e = 0; e < E; ++e) got[w][e] = vs[s_place[token_of(w, e)].word + place];
    }

    if (a.weights_out && tid < ntok) a.weights_out[(size_t)bh * a.w_cap_out + t0 + tid] = weight;
#pragma unroll
    for (int m = 0; m < META; ++m) {
        const int item = m * kMoveThreads + tid, which = item / TB, t = item % TB;
        if (which < arrays && t < rows) {
            uint16_t* p = (which == 0 ? meta_dst[0] : which == 1 ? meta_dst[1] : which == 2 ? meta_dst[2] : meta_dst[3]) +
                          (((size_t)bh * a.dst_cap + t0 + t) << cg_log2);
            if (cg_log2 == 2) *reinterpret_cast<uint2*>(p) = meta[m];
            else if (cg_log2 == 1) *reinterpret_cast<uint32_t*>(p) = meta[m].x;
            else *p = (uint16_t)meta[m].x;
        }
    }
    if constexpr (!REGROUP) {
        uint4* o = (uint4*)a.dst.k_codes + ((size_t)bh * a.dst_cap + t0) * BITS;
#pragma unroll
        for (int i = 0; i < (PIECES > 0 ? PIECES : 1); ++i) {
            const int item = i * kMoveThreads + tid;
            if (item / BITS < rows) o[item] = piece[i];
        }
    }
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
        uint32_t word = 0u;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t shift = s_place[token_of(w, e)].shift;
            const uint32_t field = BITS == 16 ? (got[w][e] >> shift) & 0xFFFFu : __builtin_amdgcn_ubfe(got[w][e], shift, BITS);
            word |= field << (16 * (e / HALF) + BITS * (e % HALF));
        }
        if (ntok < TB) {       // (uniform) the head's last tokens: zeros behind them
            uint32_t there = 0u;
#pragma unroll
            for (int e = 0; e < E; ++e) there |= (token_of(w, e) < ntok ? (1u << BITS) - 1u : 0u) << (16 * (e / HALF) + BITS * (e % HALF));
            word &= there;
        }
        const int i = w * kMoveThreads + tid;
        if (i / SBW * SB < ntok) vd[i] = word;
    }

    if constexpr (QUANT) {
        if (REGROUP || key_axis == KVQP_KEY_PER_CHANNEL) {
            // keys per channel: the groups' rows of scales and zeros, and (REGROUP) the codes of groups that are formed anew
            const int group_log2 = REGROUP ? REGROUP : a.group_log2, group = 1 << group_log2;
            const size_t sg = (size_t)((a.src_cap + group - 1) >> group_log2), dg = (size_t)((a.dst_cap + group - 1) >> group_log2);
            const int groups = (ntok + group - 1) >> group_log2;
            if constexpr (!REGROUP) {
                for (int i = tid; i < groups * (kHeadDim / 2); i += kMoveThreads) {
                    const int g = i / (kHeadDim / 2), d = i % (kHeadDim / 2);
                    if (t0 & (group - 1)) continue;      // (a group that began in an earlier workgroup's tokens)
                    const size_t from = ((size_t)bh * sg + (s_idx[g << group_log2] >> group_log2)) * (kHeadDim / 2) + d;
                    const size_t to = ((size_t)bh * dg + (t0 >> group_log2) + g) * (kHeadDim / 2) + d;
                    ((uint32_t*)a.dst.k_scale)[to] = ((const uint32_t*)a.src.k_scale)[from];
                    ((uint32_t*)a.dst.k_zero)[to] = ((const uint32_t*)a.src.k_zero)[from];
                }
            } else {
                constexpr int R = TB / 16;          // a thread's rows: r, r + 16, ..., channels 8 c8 .. 8 c8 + 7
                const int c8 = tid & 15, r = tid >> 4, wave = tid >> 6;
                constexpr int rpg_log2 = REGROUP - 4;         // 2, 4 or 8 of a thread's rows make a group
                const uint32_t* kc = (const uint32_t*)a.src.k_codes + (size_t)bh * a.src_cap * (4 * BITS);
                const uint16_t* ks = (const uint16_t*)a.src.k_scale + (size_t)bh * sg * kHeadDim + 8 * c8;
                const uint16_t* kz = (const uint16_t*)a.src.k_zero + (size_t)bh * sg * kHeadDim + 8 * c8;
                uint32_t code[R][BITS == 8 ? 2 : 1];
                h2v x[R][4];
                uint4 s4[R], z4[R];
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    const int t = s_idx[min(r + 16 * j, ntok - 1)];
                    if constexpr (BITS == 8) { const uint2 u = *reinterpret_cast<const uint2*>(kc + (size_t)t * 32 + 2 * c8); code[j][0] = u.x; code[j][1] = u.y; }
                    else if constexpr (BITS == 4) code[j][0] = kc[(size_t)t * 16 + c8];
                    else code[j][0] = kc[(size_t)t * 8 + c8 / 2] >> (8 * (c8 & 1));
                    s4[j] = *reinterpret_cast<const uint4*>(ks + (size_t)(t >> group_log2) * kHeadDim);
                    z4[j] = *reinterpret_cast<const uint4*>(kz + (size_t)(t >> group_log2) * kHeadDim);
                }
                // bit of element e's field in its word
                auto bit_of = [](int e) { return BITS == 8 ? 8 * (e % 4 / 2) + 16 * (e % 2) : BITS * (e / 2) + 16 * (e % 2); };
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    const uint32_t s[4] = {s4[j].x, s4[j].y, s4[j].z, s4[j].w}, z[4] = {z4[j].x, z4[j].y, z4[j].z, z4[j].w};
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float c = (float)__builtin_amdgcn_ubfe(code[j][BITS == 8 ? e / 4 : 0], bit_of(e), BITS);
                        const float v = __builtin_fmaf(c, half_to_float((s[e / 2] >> (16 * (e % 2))) & 0xffffu), half_to_float((z[e / 2] >> (16 * (e % 2))) & 0xffffu));
                        // (a group that reaches the largest binary16 number may read back above it: its scale was rounded up)
                        x[j][e / 2][e % 2] = (_Float16)fminf(fmaxf(v, -65504.0f), 65504.0f);
                    }
                }
                // minima and maxima of the groups' channels: a thread's rows, the wave's four row lanes, the four waves.  (Rows past
                // the count repeat the last token, which is of the last group.)
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    if (g >= groups) break;       // (uniform)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        h2v lo = {(_Float16)65504.0f, (_Float16)65504.0f}, hi = -lo;
#pragma unroll
                        for (int j = 0; j < R; ++j)
                            if (j >> rpg_log2 == g) { lo = __builtin_elementwise_min(lo, x[j][q]); hi = __builtin_elementwise_max(hi, x[j][q]); }
                        lo = __builtin_elementwise_min(lo, as_h2(xor_rows(as_u32(lo), false))); hi = __builtin_elementwise_max(hi, as_h2(xor_rows(as_u32(hi), false)));
                        lo = __builtin_elementwise_min(lo, as_h2(xor_rows(as_u32(lo), true))); hi = __builtin_elementwise_max(hi, as_h2(xor_rows(as_u32(hi), true)));
                        if ((tid & 48) == 0) { s_min[(wave * GROUPS + g) * 64 + 4 * c8 + q] = as_u32(lo); s_max[(wave * GROUPS + g) * 64 + 4 * c8 + q] = as_u32(hi); }
                    }
                }
                __syncthreads();
                // A group whose tokens were one group before: it begins where one began, has no gap, and is as long as that one.
                auto same_group = [&](int g, int& first) {
                    const int members = min(group, ntok - (g << group_log2));
                    first = s_idx[g << group_log2];
                    return (first & (group - 1)) == 0 && s_idx[(g << group_log2) + members - 1] - first == members - 1 && members == min(group, n_src - first);
                };
                for (int i = tid; i < groups * kHeadDim; i += kMoveThreads) {
                    const int g = i / kHeadDim, d = i % kHeadDim;
                    float lo = 65504.0f, hi = -65504.0f;
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        lo = fminf(lo, (float)as_h2(s_min[(v * GROUPS + g) * 64 + d / 2])[d % 2]);
                        hi = fmaxf(hi, (float)as_h2(s_max[(v * GROUPS + g) * 64 + d / 2])[d % 2]);
                    }
                    const __half sh = __float2half_rn(__fdiv_rn(__fsub_rn(hi, lo), (float)((1 << BITS) - 1)));
                    const float sf = __half2float(sh);
                    s_par[i] = {lo, sf == 0.0f ? 0.0f : __fdiv_rn(1.0f, sf)};
                    int first;
                    const bool same = same_group(g, first);
                    const size_t from = ((size_t)bh * sg + (first >> group_log2)) * kHeadDim + d, to = ((size_t)bh * dg + (t0 >> group_log2) + g) * kHeadDim + d;
                    ((uint16_t*)a.dst.k_scale)[to] = same ? ((const uint16_t*)a.src.k_scale)[from] : __half_as_ushort(sh);
                    ((uint16_t*)a.dst.k_zero)[to] = same ? ((const uint16_t*)a.src.k_zero)[from] : __half_as_ushort(__float2half_rn(lo));
                }
                __syncthreads();
                uint32_t* out = (uint32_t*)a.dst.k_codes + ((size_t)bh * a.dst_cap + t0) * (4 * BITS);
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    if (g >= groups) break;
                    GroupParams par[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) par[e] = s_par[g * kHeadDim + 8 * c8 + e];
                    int first;
                    const bool same = same_group(g, first);
#pragma unroll
                    for (int j = 0; j < R; ++j) {
                        const int t = r + 16 * j;
                        if (j >> rpg_log2 != g || t >= rows) continue;      // (the same for the 16 lanes of a row)
                        uint32_t w[2] = {0u, 0u};
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            // (added to 3 2^22, a number is rounded to a whole one, half to even, in the lowest bits:
                            // five instructions a code instead of seven)
                            const float c = __fadd_rn(__fmul_rn(__fsub_rn((float)x[j][e / 2][e % 2], par[e].zero), par[e].inv), 12582912.0f);
                            w[BITS == 8 ? e / 4 : 0] += __float_as_uint(__builtin_amdgcn_fmed3f(c, 12582912.0f, 12582912.0f + (float)((1 << BITS) - 1))) << bit_of(e);
                        }
                        // (what the number that was added leaves above the codes)
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[BITS == 8 ? e / 4 : 0] -= __float_as_uint(12582912.0f) << bit_of(e);
                        if (same) { w[0] = BITS == 2 ? code[j][0] & 0x00FF00FFu : code[j][0]; if constexpr (BITS == 8) w[1] = code[j][1]; }
                        if (t >= ntok) w[0] = w[1] = 0u;
                        if constexpr (BITS == 8) *reinterpret_cast<uint2*>(out + (size_t)t * 32 + 2 * c8) = make_uint2(w[0], w[1]);
                        else if constexpr (BITS == 4) out[(size_t)t * 16 + c8] = w[0];
                        else {
                            // the word spans this lane's channels and its neighbour's
                            uint32_t both = w[0] << (8 * (c8 & 1));
                            both |= __builtin_amdgcn_update_dpp(0u, both, 0xB1 /* quad_perm [1,0,3,2] */, 0xF, 0xF, true);
                            if (!(c8 & 1)) out[(size_t)t * 8 + c8 / 2] = both;
                        }
                    }
                }
            }
        }
    }
}

template <int BITS, bool RANKS>
hipError_t move_bits(const EvictArgs& a0, int heads, int key_axis, bool regroup, hipStream_t stream) {
    EvictArgs a = a0;
    const int tb = regroup && a.group_log2 == 7 ? 128 : 64;          // (as move_tokens has it)
    a.token_blocks = (a.bound + tb - 1) / tb;
    const dim3 grid(a.token_blocks + 1, heads), block(kMoveThreads);
    if constexpr (BITS != 16) {
        if (regroup) {
            if (a.group_log2 == 5) move_tokens<BITS, 5, RANKS><<<grid, block, 0, stream>>>(a, key_axis);
            else if (a.group_log2 == 6) move_tokens<BITS, 6, RANKS><<<grid, block, 0, stream>>>(a, key_axis);
            else move_tokens<BITS, 7, RANKS><<<grid, block, 0, stream>>>(a, key_axis);
            return hipGetLastError();
        }
    }
    move_tokens<BITS, 0, RANKS><<<grid, block, 0, stream>>>(a, key_axis);
    return hipGetLastError();
}
template <bool RANKS>
hipError_t move(const EvictArgs& a, const kvqp_cfg& cfg, int heads, bool regroup, hipStream_t stream) {
    switch (cfg.bits) {
        case 2: return move_bits<2, RANKS>(a, heads, cfg.key_axis, regroup, stream);
        case 4: return move_bits<4, RANKS>(a, heads, cfg.key_axis, regroup, stream);
        case 8: return move_bits<8, RANKS>(a, heads, cfg.key_axis, regroup, stream);
        default: return move_bits<16, RANKS>(a, heads, cfg.key_axis, regroup, stream);
    }
}

}  // namespace

int evict_kept(int n, int n_keep, int unit) { return cut_of(n, n_keep, unit).kept; }

hipError_t launch_evict(const kvqp_cfg& cfg, const kvqp_cache& src, const float* weights, int w_cap, int n_keep, int unit, int bound,
                        const kvqp_cache& dst, float* weights_out, int w_cap_out, int32_t* list, int32_t* idx, hipStream_t stream) {
    EvictArgs a = {};
    a.src = src; a.dst = dst;
    a.weights = weights; a.weights_out = weights_out; a.idx = idx; a.list = list;
    a.w_cap = w_cap; a.w_cap_out = w_cap_out;
    a.n_kept = src.n_kept; a.src_cap = layout_tokens(src, src.n_kept); a.dst_cap = layout_tokens(dst, bound);
    a.n_keep = n_keep; a.unit = unit; a.bound = bound;
    a.group_log2 = cfg.bits == 16 || cfg.group_size == 128 ? 7 : cfg.group_size == 64 ? 6 : 5;
    const int heads = cfg.batch * cfg.n_kv_heads;
    const int units = src.n_kept / unit;
    const bool regroup = cfg.bits != 16 && cfg.key_axis == KVQP_KEY_PER_CHANNEL && unit % cfg.group_size != 0;
    // Where moving takes two workgroups per CU at most, each ranks its head's few units for itself and one launch does all (4 bits; 8 heads of
    // 33 units of 32 tokens, 136 workgroups: 5.9 us, 7.8 in two launches; 32 heads of 32 units, 480: 7.2 and 9.0; 64 heads, 960: 13.0 and 11.4).
    if (units <= kFewUnits && (long long)heads * (bound / 64 + 2) <= 512) return move<true>(a, cfg, heads, regroup, stream);
    if (units <= kFewUnits) pick_of_few<<<dim3(heads), dim3(kFewUnits), 0, stream>>>(a);
    else if (units <= 1024) pick_heaviest<4, 256><<<dim3(heads), dim3(256), 0, stream>>>(a);
    else if (units <= 8192) pick_heaviest<8, 1024><<<dim3(heads), dim3(1024), 0, stream>>>(a);
    else if (units <= 32768) pick_heaviest<32, 1024><<<dim3(heads), dim3(1024), 0, stream>>>(a);
    else pick_heaviest<0, 1024><<<dim3(heads), dim3(1024), 0, stream>>>(a);
    const hipError_t rc = hipGetLastError();
    if (rc != hipSuccess) return rc;
    return move<false>(a, cfg, heads, regroup, stream);
}

}  // namespace kvqp
