// Eviction from a packed cache by accumulated attention weight: the heaviest tokens of every head (or
// the heaviest units of neighbouring tokens) move, in their order, into another cache.
//
//   score[u] = float(sum over the unit's tokens of weight[t]), summed in binary64
//   kept     = the m highest scores, equal ones going to the lower unit, in ascending order
//
// Two launches.  pick_heaviest finds the cut of one head per workgroup: a radix selection on 32-bit order keys (11 + 11 + 10
// bits, a histogram in LDS each) and one ordered pass that writes the survivors.  move_tokens gathers: nothing is rounded
// anew -- codes, scales and zeros of values, of keys per token and of whole key groups are copied bit by bit, value codes
// from and into the tile-transposed words -- except where tokens of different key groups form a new one (keys per channel,
// units smaller than a group): those keys are read back as binary16 numbers and quantized again, by the cache's quantizer.
// (A new group whose tokens were one group before is copied too: what lies before the first token that leaves is never touched.)
// Both are bound by memory: the survivors' bytes are read and written once (a value word holds 4 to 16 tokens, so
// what lies between survivors comes along).
#include "kvqp_internal.h"

namespace kvqp {
namespace {

constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64, kBins = 2048;
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
    int group, token_blocks;
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
__device__ __forceinline__ uint32_t unit_key(const float* w, int u, int unit) {
    if (unit == 1) return order_key(w[u]);
    double sum = 0.0;
    for (int t = 0; t < unit; ++t) sum += (double)w[u * unit + t];
    return order_key((float)sum);
}

__global__ __launch_bounds__(kPickThreads) void pick_heaviest(const EvictArgs a) {
    __shared__ uint32_t s_hist[kBins];
    __shared__ uint32_t s_wave[kPickWaves], s_wave2[kPickWaves];
    __shared__ uint32_t s_found[2];
    const int bh = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
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
        for (int t = tid; t < n; t += kPickThreads) put(t, t);
        return;
    }
    for (int t = tid; t < cut.short_unit; t += kPickThreads) put(cut.keep_units * a.unit + t, cut.units * a.unit + t);
    if (cut.keep_units == 0) return;

    // The key of the last unit that stays, and how many of those with that very key do.
    uint32_t prefix = 0u, mask = 0u, want = (uint32_t)cut.keep_units;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int b = tid; b < kBins; b += kPickThreads) s_hist[b] = 0u;
        __syncthreads();
        for (int u = tid; u < cut.units; u += kPickThreads) {
            const uint32_t k = unit_key(w, u, a.unit);
            if ((k & mask) == prefix) atomicAdd(&s_hist[(k >> shift) & ((1u << bits) - 1u)], 1u);
        }
        __syncthreads();
        // bins from the highest down: thread t has bins kBins - 1 - 2 t and the one below
        const int hi = kBins - 1 - 2 * tid;
        const uint32_t c0 = s_hist[hi], c1 = s_hist[hi - 1];
        uint32_t before = c0 + c1;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(before, d);
            if (lane >= d) before += o;
        }
        if (lane == 63) s_wave[wave] = before;
        __syncthreads();
        before -= c0 + c1;
        for (int v = 0; v < wave; ++v) before += s_wave[v];
        if (before < want && want <= before + c0) { s_found[0] = (uint32_t)hi; s_found[1] = want - before; }
        else if (before + c0 < want && want <= before + c0 + c1) { s_found[0] = (uint32_t)hi - 1u; s_found[1] = want - before - c0; }
        __syncthreads();
        prefix |= s_found[0] << shift;
        mask |= ((1u << bits) - 1u) << shift;
        want = s_found[1];
    }

    // Every wave has a stretch of its own: how many stay in the stretches before it, then its own in order.
    const int seg = ((cut.units + kPickWaves - 1) / kPickWaves + 63) / 64 * 64;
    const int u0 = wave * seg, u1 = min(u0 + seg, cut.units);
    uint32_t above = 0u, equal = 0u;
    for (int u = u0; u < u1; u += 64) {
        const uint32_t k = u + lane < u1 ? unit_key(w, u + lane, a.unit) : 0u;
        above += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(u + lane < u1 && k > prefix));
        equal += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(u + lane < u1 && k == prefix));
    }
    if (lane == 0) { s_wave[wave] = above; s_wave2[wave] = equal; }
    __syncthreads();
    above = equal = 0u;
    for (int v = 0; v < wave; ++v) { above += s_wave[v]; equal += s_wave2[v]; }
    const unsigned long long below = (1ull << lane) - 1ull;
    for (int u = u0; u < u1; u += 64) {
        const uint32_t k = u + lane < u1 ? unit_key(w, u + lane, a.unit) : 0u;
        const unsigned long long ba = __builtin_amdgcn_ballot_w64(u + lane < u1 && k > prefix);
        const unsigned long long be = __builtin_amdgcn_ballot_w64(u + lane < u1 && k == prefix);
        const uint32_t e = equal + (uint32_t)__builtin_popcountll(be & below);
        const uint32_t at = above + (uint32_t)__builtin_popcountll(ba & below) + min(e, want);
        const bool stays = u + lane < u1 && (k > prefix || (k == prefix && e < want));
        if (stays)
            for (int t = 0; t < a.unit; ++t) put((int)at * a.unit + t, (u + lane) * a.unit + t);
        above += (uint32_t)__builtin_popcountll(ba);
        equal += (uint32_t)__builtin_popcountll(be);
    }
}

__device__ __forceinline__ float half_to_float(uint32_t u) { return __half2float(__ushort_as_half((unsigned short)u)); }

// One field of a value word: where token t keeps channel 16 tile + n (layout statement in kvqp.h).
template <int BITS> struct ValuePlace {
    static constexpr int kWpt = v_words_per_tile(BITS), kFields = 16 / BITS, kSb = v_superblock(BITS);
    uint32_t word;      // of the head, for tile 0 and n = 0
    int wl, shift;
    __device__ __forceinline__ explicit ValuePlace(int t) {
        const int low = t % kSb, blk = low / 32, H = low / 16 % 2, kb = low / 4 % 4, i = low % 4;
        const int run = 4 * blk + i;
        wl = run / kFields;
        shift = 16 * H + BITS * (run % kFields);
        word = (uint32_t)(t / kSb) * v_superblock_words(BITS) + kb * 64;
    }
    __device__ __forceinline__ uint32_t at(int tile, int n) const {
        const int y = tile * kWpt + wl;
        return word + (uint32_t)((y / 4) * 256 + n * 4 + y % 4);
    }
};

// Quantizes keys of new groups (keys per channel): the WG's TB survivors, whole groups of them.
template <int BITS, int TB>
__device__ __forceinline__ void regroup_keys(const EvictArgs& a, int bh, int n_src, int t0, int ntok, const int (&s_idx)[TB], float (&s_min)[4][2][kHeadDim], float (&s_max)[4][2][kHeadDim]) {
    constexpr int R = TB / 16;
    const int c8 = threadIdx.x & 15, r = threadIdx.x >> 4, wave = threadIdx.x >> 6;
    const int rows_per_group = a.group / 16, n_groups = (ntok + a.group - 1) / a.group;      // 2, 4 or 8 of a thread's rows
    const uint32_t* kc = (const uint32_t*)a.src.k_codes + (size_t)bh * a.src_cap * (kHeadDim * BITS / 32);
    const size_t src_groups = (size_t)(a.src_cap + a.group - 1) / a.group;
    const uint16_t* ks = (const uint16_t*)a.src.k_scale + (size_t)bh * src_groups * kHeadDim;
    const uint16_t* kz = (const uint16_t*)a.src.k_zero + (size_t)bh * src_groups * kHeadDim;
    _Float16 x[R][8];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int t = s_idx[min(r + 16 * j, ntok - 1)];
        uint32_t w[2];
        if constexpr (BITS == 8) { const uint2 u = *reinterpret_cast<const uint2*>(kc + (size_t)t * 32 + 2 * c8); w[0] = u.x; w[1] = u.y; }
        else if constexpr (BITS == 4) w[0] = w[1] = kc[(size_t)t * 16 + c8];
        else w[0] = w[1] = kc[(size_t)t * 8 + c8 / 2] >> (8 * (c8 & 1));
        const size_t row = (size_t)(t / a.group) * kHeadDim + 8 * c8;
        const uint4 s4 = *reinterpret_cast<const uint4*>(ks + row), z4 = *reinterpret_cast<const uint4*>(kz + row);
        const uint32_t s[4] = {s4.x, s4.y, s4.z, s4.w}, z[4] = {z4.x, z4.y, z4.z, z4.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int shift = BITS == 8 ? 8 * ((e % 4) / 2) + 16 * (e % 2) : BITS * (e / 2) + 16 * (e % 2);
            const float code = (float)((w[BITS == 8 ? e / 4 : 0] >> shift) & ((1u << BITS) - 1u));
            const uint32_t sh = (s[e / 2] >> (16 * (e % 2))) & 0xffffu, zh = (z[e / 2] >> (16 * (e % 2))) & 0xffffu;
            // (a group that reaches the largest binary16 number may read back above it: its scale was rounded up)
            x[j][e] = (_Float16)fminf(fmaxf(__builtin_fmaf(code, half_to_float(sh), half_to_float(zh)), -65504.0f), 65504.0f);
        }
    }
    // minima and maxima of the groups' channels: a thread's rows, the wave's four row lanes, the four waves
    for (int g = 0; g < n_groups; ++g) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float lo = 65504.0f, hi = -65504.0f;
#pragma unroll
            for (int j = 0; j < R; ++j)        // (rows past the count repeat the last token, which is of the last group)
                if (j / rows_per_group == g || (r + 16 * j >= ntok && g == n_groups - 1)) { lo = fminf(lo, (float)x[j][e]); hi = fmaxf(hi, (float)x[j][e]); }
            lo = fminf(lo, __shfl_xor(lo, 16)); hi = fmaxf(hi, __shfl_xor(hi, 16));
            lo = fminf(lo, __shfl_xor(lo, 32)); hi = fmaxf(hi, __shfl_xor(hi, 32));
            if ((threadIdx.x & 48) == 0) { s_min[wave][g][8 * c8 + e] = lo; s_max[wave][g][8 * c8 + e] = hi; }
        }
    }
    __syncthreads();
    uint32_t* out = (uint32_t*)a.dst.k_codes + ((size_t)bh * a.dst_cap + t0) * (kHeadDim * BITS / 32);
    const size_t dst_groups = (size_t)(a.dst_cap + a.group - 1) / a.group;
    const size_t row0 = ((size_t)bh * dst_groups + t0 / a.group) * kHeadDim + 8 * c8;
    for (int g = 0; g < n_groups; ++g) {
        // (uniform) one group as it was: it begins where one began, has no gap, and is as long as that one
        const int members = min(a.group, ntok - g * a.group), first = s_idx[g * a.group], last = s_idx[g * a.group + members - 1];
        const bool same = first % a.group == 0 && last - first == members - 1 && members == min(a.group, n_src - first);
        float zf[8], inv[8];
        uint32_t sw[4] = {0u, 0u, 0u, 0u}, zw[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int d = 8 * c8 + e;
            const float lo = fminf(fminf(s_min[0][g][d], s_min[1][g][d]), fminf(s_min[2][g][d], s_min[3][g][d]));
            const float hi = fmaxf(fmaxf(s_max[0][g][d], s_max[1][g][d]), fmaxf(s_max[2][g][d], s_max[3][g][d]));
            const __half sh = __float2half_rn(__fdiv_rn(__fsub_rn(hi, lo), (float)((1 << BITS) - 1)));
            const float sf = __half2float(sh);
            zf[e] = lo;
            inv[e] = sf == 0.0f ? 0.0f : __fdiv_rn(1.0f, sf);
            sw[e / 2] |= (uint32_t)__half_as_ushort(sh) << (16 * (e % 2));
            zw[e / 2] |= (uint32_t)__half_as_ushort(__float2half_rn(lo)) << (16 * (e % 2));
        }
        if (same) {
            const size_t row = (size_t)(first / a.group) * kHeadDim + 8 * c8;
            const uint4 s4 = *reinterpret_cast<const uint4*>(ks + row), z4 = *reinterpret_cast<const uint4*>(kz + row);
            sw[0] = s4.x; sw[1] = s4.y; sw[2] = s4.z; sw[3] = s4.w;
            zw[0] = z4.x; zw[1] = z4.y; zw[2] = z4.z; zw[3] = z4.w;
        }
        if (r == 0) {
            *reinterpret_cast<uint4*>((uint16_t*)a.dst.k_scale + row0 + (size_t)g * kHeadDim) = make_uint4(sw[0], sw[1], sw[2], sw[3]);
            *reinterpret_cast<uint4*>((uint16_t*)a.dst.k_zero + row0 + (size_t)g * kHeadDim) = make_uint4(zw[0], zw[1], zw[2], zw[3]);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int t = r + 16 * j;
            // (a group of 32 or more takes all of a thread's rows j .. at once: no lane of a row of lanes is left out)
            if (j / rows_per_group != g || t >= rows32(ntok)) continue;
            uint32_t w[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float c = rintf(__fmul_rn(__fsub_rn((float)x[j][e], zf[e]), inv[e]));
                const uint32_t code = (uint32_t)fminf(fmaxf(c, 0.0f), (float)((1 << BITS) - 1));
                const int shift = BITS == 8 ? 8 * ((e % 4) / 2) + 16 * (e % 2) : BITS * (e / 2) + 16 * (e % 2);
                w[BITS == 8 ? e / 4 : 0] |= code << shift;
            }
            if (same && t < ntok) {
                const size_t row = (size_t)s_idx[t];
                if constexpr (BITS == 8) { const uint2 u = *reinterpret_cast<const uint2*>(kc + row * 32 + 2 * c8); w[0] = u.x; w[1] = u.y; }
                else if constexpr (BITS == 4) w[0] = kc[row * 16 + c8];
                else w[0] = (kc[row * 8 + c8 / 2] >> (8 * (c8 & 1))) & 0x00FF00FFu;
            }
            if (t >= ntok) w[0] = w[1] = 0u;
            if constexpr (BITS == 8) *reinterpret_cast<uint2*>(out + (size_t)t * 32 + 2 * c8) = make_uint2(w[0], w[1]);
            else if constexpr (BITS == 4) out[(size_t)t * 16 + c8] = w[0];
            else {
                // the word spans this lane's channels and its neighbour's
                uint32_t whole = w[0] << (8 * (c8 & 1));
                whole |= __shfl_xor(whole, 1);
                if (!(c8 & 1)) out[(size_t)t * 8 + c8 / 2] = whole;
            }
        }
    }
}

template <int BITS, int TB, bool REGROUP>
__global__ __launch_bounds__(kMoveThreads) void move_tokens(const EvictArgs a, int key_axis) {
    __shared__ int s_idx[TB];
    __shared__ float s_min[REGROUP ? 4 : 1][2][REGROUP ? kHeadDim : 1], s_max[REGROUP ? 4 : 1][2][REGROUP ? kHeadDim : 1];
    const int bh = blockIdx.y, tid = threadIdx.x;
    const int n_src = source_tokens(a, bh);
    const int kept = cut_of(n_src, a.n_keep, a.unit).kept;
    if ((int)blockIdx.x >= a.token_blocks) {
        // the tail, its weights, and zeros for tokens to come
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
    for (int t = tid; t < TB; t += kMoveThreads) s_idx[t] = a.idx[(size_t)bh * a.bound + t0 + min(t, ntok - 1)];
    __syncthreads();
    if (a.weights_out)
        for (int t = tid; t < ntok; t += kMoveThreads) a.weights_out[(size_t)bh * a.w_cap_out + t0 + t] = a.weights[(size_t)bh * a.w_cap + s_idx[t]];

    // value codes, a word at a time: all its fields' source words are requested before they are put together
    {
        using P = ValuePlace<BITS>;
        constexpr int SBW = v_superblock_words(BITS), E = 32 / BITS;
        const size_t src_sb = (size_t)(a.src_cap + P::kSb - 1) / P::kSb, dst_sb = (size_t)(a.dst_cap + P::kSb - 1) / P::kSb;
        const uint32_t* vs = (const uint32_t*)a.src.v_codes + (size_t)bh * src_sb * SBW;
        uint32_t* vd = (uint32_t*)a.dst.v_codes + ((size_t)bh * dst_sb + t0 / P::kSb) * SBW;
        const int words = (ntok + P::kSb - 1) / P::kSb * SBW;
        for (int i = tid; i < words; i += kMoveThreads) {
            const int sb = i / SBW, in = i % SBW;
            const int y = in / 256 * 4 + in % 4, n = in / 4 % 16, kb = in / 64 % 4;
            const int tile = y / P::kWpt, wl = y % P::kWpt;
            uint32_t got[E];
            int shift[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int H = e / P::kFields, run = wl * P::kFields + e % P::kFields;
                const int t = sb * P::kSb + 32 * (run / 4) + 16 * H + 4 * kb + run % 4;
                const P p(s_idx[min(t, ntok - 1)]);
                got[e] = vs[p.at(tile, n)];
                shift[e] = p.shift;
            }
            uint32_t w = 0u;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int H = e / P::kFields, run = wl * P::kFields + e % P::kFields;
                const int t = sb * P::kSb + 32 * (run / 4) + 16 * H + 4 * kb + run % 4;
                const uint32_t field = (got[e] >> shift[e]) & (uint32_t)((1ull << BITS) - 1ull);
                w |= t < ntok ? field << (16 * H + BITS * (e % P::kFields)) : 0u;
            }
            vd[i] = w;
        }
    }
    if constexpr (BITS != 16) {
        // scales and zeros that belong to tokens: 4, 2 or 1 numbers each
        const int cg = kHeadDim / a.group;
        auto copy = [&](const void* from, void* to) {
            const uint16_t* f = (const uint16_t*)from + (size_t)bh * a.src_cap * cg;
            uint16_t* o = (uint16_t*)to + ((size_t)bh * a.dst_cap + t0) * cg;
            for (int i = tid; i < rows * cg; i += kMoveThreads) {
                const int t = i / cg;
                o[i] = t < ntok ? f[(size_t)s_idx[t] * cg + i % cg] : (uint16_t)0;
            }
        };
        copy(a.src.v_scale, a.dst.v_scale);
        copy(a.src.v_zero, a.dst.v_zero);
        if (key_axis == KVQP_KEY_PER_TOKEN) {
            copy(a.src.k_scale, a.dst.k_scale);
            copy(a.src.k_zero, a.dst.k_zero);
        } else if constexpr (!REGROUP) {
            // whole groups: their rows of scales and zeros
            const size_t sg = (size_t)(a.src_cap + a.group - 1) / a.group, dg = (size_t)(a.dst_cap + a.group - 1) / a.group;
            for (int i = tid; i < (ntok + a.group - 1) / a.group * (kHeadDim / 2); i += kMoveThreads) {
                const int g = i / (kHeadDim / 2), d = i % (kHeadDim / 2);
                if ((t0 + g * a.group) % a.group) continue;      // (a group that began in an earlier workgroup's tokens)
                const size_t from = ((size_t)bh * sg + s_idx[g * a.group] / a.group) * (kHeadDim / 2) + d;
                const size_t to = ((size_t)bh * dg + t0 / a.group + g) * (kHeadDim / 2) + d;
                ((uint32_t*)a.dst.k_scale)[to] = ((const uint32_t*)a.src.k_scale)[from];
                ((uint32_t*)a.dst.k_zero)[to] = ((const uint32_t*)a.src.k_zero)[from];
            }
        }
    }
    if constexpr (REGROUP) {
        regroup_keys<BITS, TB>(a, bh, n_src, t0, ntok, s_idx, s_min, s_max);
    } else {
        // key code rows: BITS pieces of 16 bytes
        const uint4* f = (const uint4*)a.src.k_codes + (size_t)bh * a.src_cap * BITS;
        uint4* o = (uint4*)a.dst.k_codes + ((size_t)bh * a.dst_cap + t0) * BITS;
        for (int i = tid; i < rows * BITS; i += kMoveThreads) {
            const int t = i / BITS;
            o[i] = t < ntok ? f[(size_t)s_idx[t] * BITS + i % BITS] : make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

template <int BITS>
hipError_t move_bits(const EvictArgs& a0, int heads, int key_axis, bool regroup, hipStream_t stream) {
    EvictArgs a = a0;
    const int tb = regroup && a.group == 128 ? 128 : 64;
    a.token_blocks = (a.bound + tb - 1) / tb;
    const dim3 grid(a.token_blocks + 1, heads), block(kMoveThreads);
    if constexpr (BITS != 16) {
        if (regroup && tb == 128) { move_tokens<BITS, 128, true><<<grid, block, 0, stream>>>(a, key_axis); return hipGetLastError(); }
        if (regroup) { move_tokens<BITS, 64, true><<<grid, block, 0, stream>>>(a, key_axis); return hipGetLastError(); }
    }
    move_tokens<BITS, 64, false><<<grid, block, 0, stream>>>(a, key_axis);
    return hipGetLastError();
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
    a.group = cfg.bits == 16 ? kHeadDim : cfg.group_size;
    const int heads = cfg.batch * cfg.n_kv_heads;
    pick_heaviest<<<dim3(heads), dim3(kPickThreads), 0, stream>>>(a);
    const hipError_t rc = hipGetLastError();
    if (rc != hipSuccess) return rc;
    const bool regroup = cfg.bits != 16 && cfg.key_axis == KVQP_KEY_PER_CHANNEL && unit % cfg.group_size != 0;
    switch (cfg.bits) {
        case 2: return move_bits<2>(a, heads, cfg.key_axis, regroup, stream);
        case 4: return move_bits<4>(a, heads, cfg.key_axis, regroup, stream);
        case 8: return move_bits<8>(a, heads, cfg.key_axis, regroup, stream);
        default: return move_bits<16>(a, heads, cfg.key_axis, regroup, stream);
    }
}

}  // namespace kvqp
