// k_sample.hip.h -- draw one entry of each row of logits from given uniform
// numbers, after temperature, top-k, top-p and min-p.
//
// With m the row's largest logit (NaN counts as -inf), c = log2(e) / T and
// z_i = (l_i - m) c, entry i weighs w_i = 2^40 2^z_i.  Weights are whole numbers
// (entry_weight), so every sum is exact and no split of a row over lanes, waves or
// strips changes a draw.  Entries are ranked by logit, equal ones by index; every
// filter keeps a first part of that order:
//   top-k   the first k entries
//   top-p   of those, each whose predecessors weigh less than
//           floor(p 2^24) W / 2^24 (rounded down), W their sum; and the first
//   min-p   each that weighs at least floor(min_p 2^40)
// The draw is the lowest index whose running sum of kept weights exceeds
// floor(u 2^24) W' / 2^24 (rounded down), W' the kept sum.  The
// log-probability is (l - m) / T - ln(W' / 2^40).
//
// k_sample_few, k_sample_tiny: rows of up to 8 entries, one thread to a row, and of up to
// 64, 16 to 64 lanes to a row; ranks by comparing every pair of entries.  1,048,576 rows of
// two fp32 entries 7.4 us, 21 MB: by then the call's host path is as long.
// k_sample: longer rows, one workgroup to a row, which is read twice: for its largest
// entry, then for the weights.  It is read again rather than held in registers, so that
// two workgroups of 1,024 threads fit a CU and one weighs while the other reads; the
// second read comes from the last-level cache.  Without cuts an entry costs 21 vector
// instructions in the second pass and a row of 2 bytes an entry is bound by both passes
// alike: 512 rows of 151,001 bf16 in 66-70 us, 2.2-2.3 TB/s (the first pass alone 5.4 TB/s).
// The end of the kept part is found without sorting.  top-p: the second pass bins the
// weights by z in LDS (64-bit atomics), a third lists the entries of the bin in which the
// cut lies, and an ever finer part of the rank's code (logit, then index) is binned until few
// enough entries are left to compare each with each: 1,024 rows of 131,072 bf16 in 210 us,
// 51 vector instructions an entry.  top-k: the entries near the largest are listed, as deep
// as counts by z say that the cut lies, and cut in the same way.
// k_sample_top, _chunk, _draw: few long rows, each shared among workgroups; one row of
// 131,072 bf16 with top-k and top-p in 20 us, three launches of 3, 6 and 12 us.
#pragma once

#include "head_common.hip.h"

namespace rlsim_dev {

struct SampleArgs {
    const void* logits;
    uint64_t stride;              // elements from row to row
    uint32_t rows, V;
    float T, top_p, min_p;        // one value for the call ...
    uint32_t top_k;               // (0: all)
    const float* T_rows;          // ... or one for each row, where not null
    const int32_t* top_k_rows;
    const float* top_p_rows;
    const float* min_p_rows;
    const float* u;
    int32_t* token;
    float* logp;                  // or null
};

// A call of few rows shares each among several workgroups, a chunk of `chunk` entries (a
// multiple of 64 vectors) to each; what they hand on, by workgroup (row * chunks + chunk) or row.
constexpr uint32_t kSplitGroups = 1024u;  // most workgroups of such a call
constexpr uint32_t kSplitChunks = 32u;    // most chunks of a row
constexpr uint32_t kSplitList = 3072u;    // entries listed for a row
constexpr uint32_t kSplitBins = 657u;
struct SampleSplit {
    uint32_t chunk, chunks;
    float* top;                   // [groups] largest entry of the chunk
    uint32_t* top_at;             // [groups] the first one's index
    uint64_t* sum;                // [groups] weight
    uint64_t* part_w;             // [groups][kSplitBins] weights by bins of z
    uint64_t* list;               // [rows][chunks][room] codes
    uint32_t room;                // kSplitList / chunks
    uint32_t* count;              // [groups] entries listed
    float* list_z;                // [groups] all with z above this are listed
};

// A row's settings.  T <= 0 or NaN: the first of the largest entries.
struct SampleRow {
    float T, c;
    uint32_t k;                   // V: all
    uint32_t p24;                 // floor(p 2^24), 2^24: all
    uint64_t least;               // smallest weight kept
    uint32_t u24;
    bool greedy;
};

constexpr uint32_t kAllP = 1u << 24;

__device__ __forceinline__ SampleRow sample_row(const SampleArgs& a, uint32_t row)
{
    SampleRow s;
    s.T = a.T_rows ? a.T_rows[row] : a.T;
    const int32_t k = a.top_k_rows ? a.top_k_rows[row] : (int32_t)(a.top_k < a.V ? a.top_k : 0u);
    const float p = a.top_p_rows ? a.top_p_rows[row] : a.top_p;
    const float min_p = a.min_p_rows ? a.min_p_rows[row] : a.min_p;
    s.k = k > 0 && (uint32_t)k < a.V ? (uint32_t)k : a.V;
    s.p24 = p < 1.0f ? (uint32_t)(__builtin_fmaxf(p, 0.0f) * 0x1p24f) : kAllP;     // NaN: all
    s.least = min_p > 0.0f ? (uint64_t)(__builtin_fminf(min_p, 1.0f) * 0x1p40f) : 0u;
    s.u24 = (uint32_t)(__builtin_fminf(__builtin_fmaxf(a.u[row], 0.0f), 1.0f - 0x1p-24f) * 0x1p24f);
    s.greedy = !(s.T > 0.0f) || s.k == 1u;
    s.c = 0x1.715476p+0f / s.T;
    return s;
}

// floor(whole share / 2^24) for share <= 2^24 and whole < 2^62
__device__ __forceinline__ uint64_t share24(uint64_t whole, uint32_t share)
{
    return (whole >> 24) * share + (((whole & 0xFFFFFFu) * share) >> 24);
}

// z = (l - m) c, 0 for the largest entries (also where m or c is infinite); weights
// are 0 where z < kLastZ or NaN.
constexpr float kLastZ = -41.0f;
__device__ __forceinline__ float entry_z(float l, float m, float c) { return l == m ? 0.0f : (l - m) * c; }

// 2^40 2^z as a whole number: 2^f on [-1/2, 1/2] in fp32, Horner form with one
// rounding per operation (relative error 1.9e-7), truncated to 24 bits and shifted by the
// whole part of z.  Coefficients scaled by 2^40, so that P 2^n is the weight before its
// fraction is cut off; it needs at most 24 bits, so fp32 holds it too.  (entry_weight32
// leaves the fraction on: every use of it cuts it off.)
// z + 1.5 2^23 rounds z to the whole number n that its low bits then show.  At -41, to
// which the maximum raises all below it and NaN, P 2^n is less than 1.
__device__ __forceinline__ float entry_weight32(float z)
{
    z = __builtin_fmaxf(z, kLastZ);
    const float y = z + 0x1.8p23f;
    const float f = z - (y - 0x1.8p23f);
    float P = f * 0x1.5bb994p+30f + 0x1.3cea84p+33f;
    P = P * f + 0x1.c6b754p+35f;
    P = P * f + 0x1.ebf9bcp+37f;
    P = P * f + 0x1.62e42ap+39f;
    P = P * f + 0x1p40f;
    return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, P) + (__builtin_bit_cast(uint32_t, y) << 23));
}
__device__ __forceinline__ uint64_t whole_weight(float w)        // w < 2^41, without its fraction
{
    const float high = __builtin_truncf(w * 0x1p-32f);
    return (uint64_t)(uint32_t)high << 32 | (uint32_t)__builtin_fmaf(high, -0x1p32f, w);
}
__device__ __forceinline__ uint64_t entry_weight(float z) { return whole_weight(entry_weight32(z)); }

// A whole number ascending in rank: larger logits first, then lower indices, -0 and +0
// equal.  `ibits` bits hold an index; above them stand the logit's bits, without those
// that are 0 in the row's type.
template <int D>
__device__ __forceinline__ uint64_t rank_code(float l, uint32_t i, uint32_t ibits)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, l + 0.0f);
    const uint32_t down = b >> 31 ? b : 0x7FFFFFFFu - b;
    return (uint64_t)(down >> Elem<D>::kZeroBits) << ibits | i;
}
template <int D>
__device__ __forceinline__ float rank_logit(uint64_t code, uint32_t ibits)
{
    constexpr uint32_t Z = Elem<D>::kZeroBits;
    const uint32_t down = (uint32_t)(code >> ibits) << Z;
    return __builtin_bit_cast(float, down >> 31 ? down : 0x7FFFFFFFu - (down | ((1u << Z) - 1u)));
}

__device__ __forceinline__ float sample_logp(float l, float m, float T, uint64_t whole)
{
    const float above = l == m ? 0.0f : (l - m) / T;
    return above - __builtin_logf((float)whole * 0x1p-40f);
}

// ---------------------------------------------------------------------------
template <int D, int N>
__global__ __launch_bounds__(256) void k_sample_few(SampleArgs a)
{
    using El = Elem<D>;
    const float none = -__builtin_inff();
    for (uint32_t row = blockIdx.x * 256u + threadIdx.x; row < a.rows; row += gridDim.x * 256u) {
        const typename El::Word* const p = static_cast<const typename El::Word*>(a.logits) + (uint64_t)row * a.stride;
        float l[N], m = none;
        uint64_t w[N], whole = 0u;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) {
            l[e] = e < a.V ? El::one(p[e]) : none;
            l[e] = l[e] == l[e] ? l[e] : none;
            m = __builtin_fmaxf(m, l[e]);
        }
        const SampleRow s = sample_row(a, row);
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) w[e] = l[e] > none ? entry_weight(entry_z(l[e], m, s.c)) : 0u;
        if (s.k < a.V || s.p24 < kAllP || s.greedy) {
            uint32_t rank[N];
            uint64_t before[N], all = 0u;         // the entries ahead of each: how many, and their weight
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) {
                rank[e] = 0u;
                before[e] = 0u;
#pragma unroll
                for (uint32_t j = 0; j < N; ++j) {
                    const bool ahead = l[j] > l[e] || (l[j] == l[e] && j < e);
                    rank[e] += ahead ? 1u : 0u;
                    before[e] += ahead ? w[j] : 0u;
                }
                all += rank[e] < s.k ? w[e] : 0u;
            }
            const uint64_t target = share24(all, s.p24);
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) {
                const bool keep = rank[e] == 0u || (!s.greedy && rank[e] < s.k && (s.p24 == kAllP || before[e] < target));
                w[e] = keep ? w[e] : 0u;
            }
        }
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) {
            w[e] = w[e] >= s.least ? w[e] : 0u;
            whole += w[e];
        }
        const uint64_t target = share24(whole, s.u24);
        uint64_t running = 0u;
        int32_t token = -1;
        float found = m;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) {
            running += w[e];
            if (token < 0 && running > target) {
                token = (int32_t)e;
                found = l[e];
            }
        }
        a.token[row] = token;
        if (a.logp) a.logp[row] = s.greedy || token < 0 ? 0.0f : sample_logp(found, m, s.T, whole);
    }
}

// ---------------------------------------------------------------------------
template <int D, int G>
__global__ __launch_bounds__(256) void k_sample_tiny(SampleArgs a)
{
    using El = Elem<D>;
    const uint32_t e = threadIdx.x % G;
    const uint32_t per_group = 256u / G;
    // every lane of a wave runs the same number of rounds
    for (uint32_t first = blockIdx.x * per_group; first < a.rows; first += gridDim.x * per_group) {
        const uint32_t row = first + threadIdx.x / G;
        const bool live_row = row < a.rows;
        const uint32_t r = live_row ? row : a.rows - 1u;
        const SampleRow s = sample_row(a, r);
        float l = -__builtin_inff();
        if (e < a.V) {
            const float x = El::one(static_cast<const typename El::Word*>(a.logits)[(uint64_t)r * a.stride + e]);
            l = x == x ? x : l;
        }
        float m = l;
#pragma unroll
        for (int off = G / 2; off >= 1; off /= 2) m = __builtin_fmaxf(m, __shfl_xor(m, off, G));
        uint64_t w = l > -__builtin_inff() ? entry_weight(entry_z(l, m, s.c)) : 0u;
        uint32_t rank = 0u;               // entries before this one, and what they weigh
        uint64_t before = 0u;
        if (s.k < a.V || s.p24 < kAllP || s.greedy) {
            for (uint32_t j = 0; j < a.V; ++j) {
                const float lj = __shfl(l, (int)j, G);
                const uint64_t wj = __shfl(w, (int)j, G);
                const bool ahead = lj > l || (lj == l && j < e);
                rank += ahead ? 1u : 0u;
                before += ahead ? wj : 0u;
            }
            uint64_t whole = rank < s.k ? w : 0u;
#pragma unroll
            for (int off = G / 2; off >= 1; off /= 2) whole += __shfl_xor(whole, off, G);
            const bool keep = rank == 0u || (!s.greedy && rank < s.k && (s.p24 == kAllP || before < share24(whole, s.p24)));
            w = keep ? w : 0u;
        }
        w = w >= s.least ? w : 0u;
        uint64_t running = w;
#pragma unroll
        for (int off = 1; off < G; off *= 2) {
            const uint64_t x = __shfl_up(running, (unsigned)off, G);
            running += e >= (uint32_t)off ? x : 0u;
        }
        const uint64_t whole = __shfl(running, G - 1, G);
        const uint64_t target = share24(whole, s.u24);
        // one lane of a row holds the step in which the running sum passes the target
        if (live_row && running > target && running - w <= target) {
            a.token[row] = (int32_t)e;
            if (a.logp) a.logp[row] = s.greedy ? 0.0f : sample_logp(l, m, s.T, whole);
        }
        if (live_row && e == 0u && m == -__builtin_inff()) {
            a.token[row] = -1;
            if (a.logp) a.logp[row] = 0.0f;
        }
    }
}

// ---------------------------------------------------------------------------
constexpr uint32_t kSubBins = 256u;       // bins of eight bits of a code
constexpr uint32_t kFew = 128u;           // entries compared each with each

template <int NT>
struct SampleShared {
    static constexpr uint32_t NW = NT / 64;
    static constexpr uint32_t kList = NT == 64 ? 256u : NT == 256 ? 1024u : 3072u;
    // bins of z: -kPerZ z, 0 .. 41 kPerZ, padded to a multiple of 64; in longer rows finer
    // ones, so that the bin of a cut fits the list
    static constexpr uint32_t kPerZ = NT == 1024 ? 16u : NT == 256 ? 8u : 4u;
    static constexpr uint32_t kUsedBins = 41u * kPerZ + 1u, kBins = (kUsedBins + 63u) / 64u * 64u;
    static constexpr uint32_t kParts = NT == 1024 ? 8u : NW;      // of a row, with bins of their own
    float f[NW];
    uint64_t sum[kSplitChunks + 1u], group[NW];
    uint64_t part_w[kParts][kUsedBins];
    uint64_t w[kBins];
    uint32_t n[kBins];
    union {
        struct {
            uint64_t sub_w[kSubBins];
            uint32_t sub_n[kSubBins];
        };
        struct { uint64_t few_code[kFew], few_w[kFew]; };
    };
    uint64_t list_code[kList];
    uint32_t found;                       // bin of the cut
    uint64_t before_n, before_w;          // entries, and weight, of the bins before it
    uint64_t cut, cut_w;                  // code of the entry looked for, weight up to it
    uint32_t count, few, near, far, best;  // near, far: the list's logit parts' range (near: inverted)
};

// First bin at which the running sum of counts (by_weight: of weights) reaches
// `target`; B bins, B / 64 to a lane.  Run by the first wave.
template <uint32_t B, class Sh>
__device__ __forceinline__ void find_bin(Sh& sh, const uint32_t* n, const uint64_t* w, bool by_weight, uint64_t target)
{
    constexpr uint32_t P = B / 64u;
    const uint32_t lane = threadIdx.x;
    uint64_t sn = 0u, sw = 0u;
#pragma unroll
    for (uint32_t j = 0; j < P; ++j) {
        sn += n[lane * P + j];
        sw += w[lane * P + j];
    }
    const uint64_t tn = wave_scan(sn), tw = wave_scan(sw);
    uint64_t bn = tn - sn, bw = tw - sw;
    const uint64_t before = by_weight ? bw : bn, upto = by_weight ? tw : tn;
    if (before < target && target <= upto) {
#pragma unroll
        for (uint32_t j = 0; j < P; ++j) {
            const uint64_t n_j = n[lane * P + j], w_j = w[lane * P + j];
            const uint64_t b = by_weight ? bw : bn, m = by_weight ? w_j : n_j;
            if (b < target && target <= b + m) {
                sh.found = lane * P + j;
                sh.before_n = bn;
                sh.before_w = bw;
            }
            bn += n_j;
            bw += w_j;
        }
    }
}

// Entries among which one is looked for: those whose code - first, shifted by
// `shift`, is `prefix` (64: all); n of them, behind others of the given count and
// weight.
struct Among {
    uint64_t first, prefix;
    uint32_t shift, n;
    uint64_t before_n, before_w;
    __device__ __forceinline__ bool holds(uint64_t code) const { return shift == 64u || (code - first) >> shift == prefix; }
};

// Narrow `in` by eight bits of the codes: to the bin in which the running count
// (by_weight: weight) in the codes' order reaches `target`.  visit(f) calls f(code,
// weight) for this thread's entries.
template <uint32_t NT, class Sh, class Visit>
__device__ __forceinline__ void narrow(Sh& sh, Among& in, Visit visit, bool by_weight, uint64_t target)
{
    const uint32_t down = in.shift < 8u ? 0u : in.shift - 8u;
    for (uint32_t j = threadIdx.x; j < kSubBins; j += NT) {
        sh.sub_n[j] = 0u;
        sh.sub_w[j] = 0u;
    }
    __syncthreads();
    visit([&](uint64_t code, uint64_t w) {
        if (in.holds(code)) {
            const uint32_t b = (uint32_t)((code - in.first) >> down) & 255u;
            atomicAdd(&sh.sub_n[b], 1u);
            atomicAdd((unsigned long long*)&sh.sub_w[b], (unsigned long long)w);
        }
    });
    __syncthreads();
    if (threadIdx.x < 64u)
        find_bin<kSubBins>(sh, sh.sub_n, sh.sub_w, by_weight, target - (by_weight ? in.before_w : in.before_n));
    __syncthreads();
    in.prefix = (in.shift == 64u ? 0u : in.prefix << (in.shift - down)) | sh.found;
    in.shift = down;
    in.n = sh.sub_n[sh.found];
    in.before_n += sh.before_n;
    in.before_w += sh.before_w;
    __syncthreads();
}

// The listed entry at which the running count (by_weight: weight) in the order of the
// codes reaches `target`: its code goes to sh.cut, the weight up to and with it to
// sh.cut_w.  code_of and weight_of give a listed entry's.
template <uint32_t NT, class Sh, class Code, class Weight>
__device__ __forceinline__ void find_listed(Sh& sh, Among in, uint32_t listed, Code code_of, Weight weight_of, bool by_weight,
                                            uint64_t target)
{
    auto visit = [&](auto f) {
        for (uint32_t j = threadIdx.x; j < listed; j += NT) f(code_of(j), weight_of(j));
    };
    // (with a shift of 0 one entry is left: the loop ends and the list holds what it gets even
    // if another kernel changes the logits meanwhile)
    while (in.n > kFew && in.shift) narrow<NT>(sh, in, visit, by_weight, target);
    in.n = min(in.n, kFew);
    if (threadIdx.x == 0u) sh.few = 0u;
    __syncthreads();
    visit([&](uint64_t code, uint64_t w) {
        if (in.holds(code)) {
            const uint32_t at = atomicAdd(&sh.few, 1u);
            if (at < kFew) {
                sh.few_code[at] = code;
                sh.few_w[at] = w;
            }
        }
    });
    __syncthreads();
    // L lanes to an entry share the comparisons
    constexpr uint32_t L = NT > kFew ? NT / kFew : 1u;
    for (uint32_t i = threadIdx.x / L; i < kFew; i += NT / L) {
        const bool real = i < in.n;
        const uint64_t code = real ? sh.few_code[i] : 0u, own = real ? sh.few_w[i] : 0u;
        uint32_t ahead_n = 0u;
        uint64_t ahead_w = 0u;
        for (uint32_t j = threadIdx.x % L; j < in.n; j += L) {
            const bool ahead = sh.few_code[j] < code;
            ahead_n += ahead ? 1u : 0u;
            ahead_w += ahead ? sh.few_w[j] : 0u;
        }
#pragma unroll
        for (int off = (int)L / 2; off >= 1; off /= 2) {
            ahead_n += (uint32_t)__shfl_xor((int)ahead_n, off, 64);
            ahead_w += __shfl_xor(ahead_w, off, 64);
        }
        const uint64_t bw = in.before_w + ahead_w, b = by_weight ? bw : in.before_n + ahead_n, mine = by_weight ? own : 1u;
        if (real && b < target && target <= b + mine) {
            sh.cut = code;
            sh.cut_w = bw + own;
        }
    }
    __syncthreads();
}

// z from which a row's entries are listed at first, where a top-k cut is expected: at a
// thousandth of the largest weight.
constexpr float kNearZ = -10.0f;

template <int D, int NT>
struct SampleGroup {
    using R = Row<D, NT, 0>;
    using Sh = SampleShared<NT>;
    using El = Elem<D>;
    static constexpr uint32_t E = R::E, NW = R::NW;

    const SampleArgs& a;
    Sh& sh;
    R& x;
    const SampleRow& s;
    const uint32_t row;
    const float m;
    const uint32_t ibits;         // of an index
    const uint32_t from;          // index of x's first entry

    __device__ __forceinline__ float z(float l) const { return entry_z(l, m, s.c); }
    static __device__ __forceinline__ uint32_t bin_of(float z) { return (uint32_t)(z * -(float)Sh::kPerZ); }
    __device__ __forceinline__ void answer(uint32_t i, float logp) const
    {
        a.token[row] = (int32_t)i;
        if (a.logp) a.logp[row] = logp;
    }

    // The draw from the whole row, with the weights weigh(entry, index): the wave's
    // part, then the thread's, then the entry in which the running sum passes the
    // target.  `mine` is this thread's sum over its vectors.
    template <class F>
    __device__ __forceinline__ void draw(uint64_t mine, F weigh)
    {
        const uint64_t end = x.lane < x.tail ? weigh(x.last, x.vectors * E + x.lane) : 0u;
        mine = wave_total(mine);
        if (x.lane == 0u) sh.sum[x.wave] = mine;
        if (x.wave == 0u) {
            const uint64_t t = wave_total(end);
            if (x.lane == 0u) sh.sum[NW] = t;
        }
        __syncthreads();
        pick(NW, x.seg * 64u, weigh);
    }
    // The same from the sums in sh.sum: of `parts` parts, `vectors` vectors each, and the tail.
    template <class F>
    __device__ __forceinline__ void pick(uint32_t parts, uint32_t vectors, F weigh)
    {
        const uint64_t end = x.lane < x.tail ? weigh(x.last, x.vectors * E + x.lane) : 0u;
        const uint64_t mine = x.lane <= parts ? sh.sum[x.lane] : 0u, running = wave_scan(mine);
        const uint64_t whole = lane_u64(running, 63);
        const uint64_t target = share24(whole, s.u24);
        const uint64_t past = __ballot(running > target);     // the last one's passes it
        const int part_lane = past ? (int)__builtin_ctzll(past) : (int)parts;
        const uint32_t part = (uint32_t)part_lane;
        uint64_t before = lane_u64(running, part_lane) - lane_u64(mine, part_lane);
        if (part == parts) {              // the tail's lanes
            if (x.wave == 0u) {
                const uint64_t upto = before + wave_scan(end);
                if (upto > target && upto - end <= target) answer(x.vectors * E + x.lane, sample_logp(x.last, m, s.T, whole));
            }
            return;
        }
        // the part's vectors, a run of consecutive ones to each thread
        const uint32_t run = (vectors + NT - 1u) / NT;
        const uint32_t v0 = part * vectors + threadIdx.x * run;
        const uint32_t limit = min((part + 1u) * vectors, x.vectors), v1 = min(v0 + run, limit);
        uint64_t own = 0u;
        for (uint32_t v = v0; v < v1; ++v) {
            const Vec16 y = x.vector(v);
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) own += weigh(El::get(y, e), v * E + e);
        }
        uint64_t upto = wave_scan(own);
        if (NW > 1u) {
            if (x.lane == 63u) sh.group[x.wave] = upto;
            __syncthreads();
            const uint64_t upto_wave = wave_scan(x.lane < NW ? sh.group[x.lane] : 0u);
            if (x.wave) before += lane_u64(upto_wave, (int)x.wave - 1);
        }
        upto += before;
        if (upto > target && upto - own <= target) {
            uint64_t t = upto - own;
            uint32_t at = 0u;
            float found = 0.0f;
            bool done = false;
            for (uint32_t v = v0; v < v1 && !done; ++v) {
                const Vec16 y = x.vector(v);
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) {
                    const float l = El::get(y, e);
                    t += weigh(l, v * E + e);
                    if (!done && t > target) {
                        at = v * E + e;
                        found = l;
                        done = true;
                    }
                }
            }
            answer(at, sample_logp(found, m, s.T, whole));
        }
    }

    // Append to the list, for the whole wave: the entries e whose bit is set in `hits`, with
    // the codes code_of(e).  sh.count counts; only the first kList are listed.
    template <uint32_t N, class F>
    __device__ __forceinline__ void append(uint32_t hits, F code_of)
    {
        if (__ballot(hits != 0u) == 0u) return;
        const uint32_t n = (uint32_t)__builtin_popcount(hits), upto = wave_scan(n);
        uint32_t at = 0u;
        if (x.lane == 63u) at = atomicAdd(&sh.count, upto);
        at = (uint32_t)__builtin_amdgcn_readlane((int)at, 63) + upto - n;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) {
            if (hits >> e & 1u) {
                if (at < Sh::kList) sh.list_code[at] = code_of(e);
                ++at;
            }
        }
    }
    __device__ __forceinline__ uint64_t listed_weight(uint32_t j) const { return entry_weight(z(rank_logit<D>(sh.list_code[j], ibits))); }
    __device__ __forceinline__ uint64_t code(float l, uint32_t i) const { return rank_code<D>(l, i, ibits); }
    // Append the row's entries for which want(entry) holds.
    template <class F>
    __device__ __forceinline__ void append_vector(const Vec16& y, uint32_t v, F want)
    {
        bool any = false;
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) any = any | want(El::get(y, e));
        if (__ballot(any) == 0u) return;
        uint32_t hits = 0u;
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) hits |= want(El::get(y, e)) ? 1u << e : 0u;
        append<E>(hits, [&](uint32_t e) { return code(El::get(y, e), from + v * E + e); });
    }
    template <class F>
    __device__ __forceinline__ void append_tail(F want)
    {
        if (x.wave == 0u)
            append<1>(want(x.last) ? 1u : 0u, [&](uint32_t) { return code(x.last, from + x.vectors * E + x.lane); });
    }
    __device__ __forceinline__ void clear_list()
    {
        __syncthreads();
        if (threadIdx.x == 0u) {
            sh.count = 0u;
            sh.near = 0u;
            sh.far = 0u;
        }
        __syncthreads();
    }
    // The range of the `n` listed codes; returns them as the entries among which to look,
    // behind others of the given count and weight.
    __device__ __forceinline__ Among close_list(uint32_t n, uint64_t before_n, uint64_t before_w)
    {
        uint32_t far = 0u, near = 0u;
        for (uint32_t j = threadIdx.x; j < n; j += NT) {
            const uint64_t c = sh.list_code[j];
            far = max(far, (uint32_t)(c >> ibits));
            near = max(near, ~(uint32_t)(c >> ibits));
        }
        return range(far, near, n, before_n, before_w);
    }
    __device__ __forceinline__ Among range(uint32_t far, uint32_t near, uint32_t n, uint64_t before_n, uint64_t before_w)
    {
        far = wave_max(far);
        near = wave_max(near);
        if (x.lane == 0u && far) {
            atomicMax(&sh.far, far);
            atomicMax(&sh.near, near);
        }
        __syncthreads();
        const uint32_t first = ~sh.near, span = sh.far - first;
        const uint32_t bits = span ? ibits + 32u - (uint32_t)__builtin_clz(span) : ibits;
        return Among{(uint64_t)first << ibits, 0u, max(bits, 8u), n, before_n, before_w};
    }

    // Cut, by top-k at first, and draw from the list.  False: the list does not
    // reach the cut.
    __device__ __forceinline__ bool draw_listed()
    {
        const uint32_t listed = sh.count;
        if (listed > Sh::kList || listed < s.k) return false;
        const Among rank = close_list(listed, 0u, 0u);
        uint64_t whole = 0u, weight = 0u;
        auto code = [&](uint32_t j) { return sh.list_code[j]; };
        auto plain = [&](uint32_t j) { return listed_weight(j); };
        uint64_t cut = ~0ull;
        // top-k, then top-p: one piece of code for both
        for (uint32_t by_weight = 0u; by_weight < 2u; ++by_weight) {
            uint64_t target = s.k;
            if (by_weight) {
                if (s.p24 == kAllP) continue;
                target = share24(whole, s.p24);
                target = target ? target : 1u;
            }
            find_listed<NT>(sh, rank, listed, code, plain, by_weight != 0u, target);
            cut = sh.cut;
            if (by_weight == 0u) whole = sh.cut_w;
        }
        // what is left, by index
        auto index = [&](uint32_t j) { return sh.list_code[j] & ((1ull << ibits) - 1u); };
        auto kept = [&](uint32_t j) {
            const uint64_t w = listed_weight(j);
            return sh.list_code[j] <= cut && w >= s.least ? w : 0u;
        };
        weight = 0u;
        for (uint32_t j = threadIdx.x; j < listed; j += NT) weight += kept(j);
        weight = wave_total(weight);
        __syncthreads();
        if (x.lane == 0u) sh.sum[x.wave] = weight;
        __syncthreads();
        weight = 0u;
        for (uint32_t j = 0; j < NW; ++j) weight += sh.sum[j];
        const Among order{0u, 0u, max(ibits, 8u), listed, 0u, 0u};
        find_listed<NT>(sh, order, listed, index, kept, true, share24(weight, s.u24) + 1u);
        if (threadIdx.x == 0u) {
            const uint32_t i = (uint32_t)sh.cut;
            answer(i, sample_logp(x.entry(i), m, s.T, weight));
        }
        return true;
    }

    // Draw where top-p is the first cut.  One pass bins the weights by z, each part of the
    // row in bins of its own: they give the row's weight and the bin in which the cut lies,
    // and later the parts' kept weights without another pass.  The entries of that bin are
    // listed and the cut found among them.
    __device__ __forceinline__ void bin_weights()
    {
        for (uint32_t j = threadIdx.x; j < Sh::kParts * Sh::kUsedBins; j += NT) (&sh.part_w[0][0])[j] = 0u;
        __syncthreads();
        uint64_t* const mine = sh.part_w[x.wave / (NW / Sh::kParts)];
        auto bin = [&](float l) {
            const float zi = (l - m) * s.c;
            if (zi > kLastZ) atomicAdd((unsigned long long*)&mine[bin_of(zi)], (unsigned long long)entry_weight(zi));
        };
        x.each([&](float l, uint32_t) { bin(l); });
        if (x.wave == 0u) bin(x.last);
        __syncthreads();
    }
    // part_w: [parts][kUsedBins], parts of part_vectors vectors; the row's tail counts to
    // part `tail_part`.
    __device__ __forceinline__ void draw_top_p(const uint64_t* part_w, uint32_t parts, uint32_t part_vectors, uint32_t tail_part)
    {
        for (uint32_t j = threadIdx.x; j < Sh::kBins; j += NT) {
            uint64_t w = 0u;
            if (j < Sh::kUsedBins) {
#pragma unroll 8
                for (uint32_t q = 0; q < parts; ++q) w += part_w[q * Sh::kUsedBins + j];
            }
            sh.w[j] = w;
        }
        __syncthreads();
        uint64_t whole = 0u;
        for (uint32_t j = x.lane; j < Sh::kBins; j += 64u) whole += sh.w[j];
        whole = wave_total(whole);
        uint64_t target = share24(whole, s.p24);
        target = target ? target : 1u;
        if (threadIdx.x < 64u) find_bin<Sh::kBins>(sh, sh.n, sh.w, true, target);     // (counts are not looked at)
        __syncthreads();
        const uint32_t b = sh.found;
        uint64_t before_w = sh.before_w;
        // Where min-p's end lies, a margin of 0.01 in z to both sides, far more than the weights'
        // error: bins [b0, b1] have to be looked into, those before are kept.  If they end
        // before the cut's bin, top-p cuts nothing off.
        uint32_t b0 = b, b1 = b;
        if (s.least) {
            const float least_z = __builtin_log2f((float)s.least) - 40.0f;
            b0 = min(b, bin_of(__builtin_fminf(least_z + 0.01f, 0.0f)));
            b1 = min(b, bin_of(__builtin_fmaxf(least_z - 0.01f, kLastZ)));
        }
        const bool by_top_p = b1 == b;
        if (by_top_p)
            for (uint32_t j = b0; j < b; ++j) before_w -= sh.w[j];
        // the bins' ends are exact in fp32
        const float upper = -(float)b0 / (float)Sh::kPerZ, lower = -(float)(b1 + 1u) / (float)Sh::kPerZ;
        auto in_bins = [&](float l) {
            const float zi = (l - m) * s.c;
            return zi <= upper && zi > lower;
        };
        x.each_vector([&](const Vec16& y, uint32_t v) { append_vector(y, v, in_bins); });
        append_tail(in_bins);
        __syncthreads();
        const uint32_t n = sh.count;
        const bool listed = n <= Sh::kList;
        uint64_t cut = ~0ull;
        if (by_top_p) {
            const Among in = listed ? close_list(n, 0u, before_w) : narrow_to_list(b0, b1, n, 0u, before_w, true, target);
            find_listed<NT>(sh, in, in.n, [&](uint32_t j) { return sh.list_code[j]; }, [&](uint32_t j) { return listed_weight(j); },
                            true, target);
            cut = sh.cut;
        }
        auto weigh = [&](float l, uint32_t i) { return weigh_kept(l, i, cut); };
        if (!listed) {
            uint64_t mine = 0u;
            x.each_again_vectors([&](float l, uint32_t i) { mine += weigh(l, i); });
            draw(mine, weigh);
            return;
        }
        // a part's kept weight: the bins before, and what of the listed ones is kept
        for (uint32_t q = x.wave; q < parts; q += NW) {
            uint64_t w = 0u;
#pragma unroll 8
            for (uint32_t j = x.lane; j < b0; j += 64u) w += part_w[q * Sh::kUsedBins + j];
            w = wave_total(w);
            if (x.lane == 0u) sh.sum[q] = w;
        }
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < n; j += NT) {
            const uint64_t w = listed_weight(j);
            if (sh.list_code[j] <= cut && w >= s.least) {
                const uint32_t v = (uint32_t)(sh.list_code[j] & ((1ull << ibits) - 1u)) / E;
                atomicAdd((unsigned long long*)&sh.sum[v < x.vectors ? v / part_vectors : tail_part], (unsigned long long)w);
            }
        }
        __syncthreads();
        pick_parts(parts, part_vectors, tail_part, weigh);
    }
    // pick() where sh.sum counts the tail to part tail_part
    template <class F>
    __device__ __forceinline__ void pick_parts(uint32_t parts, uint32_t part_vectors, uint32_t tail_part, F weigh)
    {
        if (x.wave == 0u) {
            const uint64_t end = wave_total(x.lane < x.tail ? weigh(x.last, x.vectors * E + x.lane) : 0u);
            if (x.lane == 0u) {
                sh.sum[tail_part] -= end;
                sh.sum[parts] = end;
            }
        }
        __syncthreads();
        pick(parts, part_vectors, weigh);
    }
    __device__ __forceinline__ uint64_t weigh_kept(float l, uint32_t i, uint64_t cut) const
    {
        const float zi = z(l);
        const uint64_t w = zi >= kLastZ && code(l, i) <= cut ? entry_weight(zi) : 0u;
        return w >= s.least ? w : 0u;
    }

    // f(entry, index, z) for the row's live entries, from another read
    template <class F>
    __device__ __forceinline__ void each_live(F f)
    {
        x.each_again([&](float l, uint32_t i) {
            const float zi = z(l);
            if (zi >= kLastZ) f(l, i, zi);
        });
    }
    // Where bins b0 to b1 of z hold more entries than the list: narrow them by their codes until
    // the list takes what is left, and list it.
    __device__ __forceinline__ Among narrow_to_list(uint32_t b0, uint32_t b1, uint32_t n, uint64_t before_n, uint64_t before_w, bool by_weight,
                                                    uint64_t target)
    {
        Among in{0u, 0u, 64u, n, before_n, before_w};
        auto visit = [&](auto f) {
            each_live([&](float l, uint32_t i, float zi) {
                if (bin_of(zi) >= b0 && bin_of(zi) <= b1) f(code(l, i), entry_weight(zi));
            });
        };
        if (n > Sh::kList) {              // the range of the bin's codes
            clear_list();
            uint32_t far = 0u, near = 0u;
            visit([&](uint64_t c, uint64_t) {
                far = max(far, (uint32_t)(c >> ibits));
                near = max(near, ~(uint32_t)(c >> ibits));
            });
            in = range(far, near, n, before_n, before_w);
        }
        while (in.n > Sh::kList && in.shift) narrow<NT>(sh, in, visit, by_weight, target);
        in.n = min(in.n, Sh::kList);
        clear_list();
        visit([&](uint64_t c, uint64_t) {
            if (in.holds(c)) {
                const uint32_t at = atomicAdd(&sh.count, 1u);
                if (at < Sh::kList) sh.list_code[at] = c;
            }
        });
        __syncthreads();
        return close_list(in.n, in.before_n, in.before_w);
    }

    // Without a top-k or top-p cut: an entry's weight, if min-p keeps it, and this thread's sum of
    // them, whole numbers less than 2^53.  With min-p few entries come near it: the others
    // are told by their z, with a margin of 0.01, far more than the weights' error.
    __device__ __forceinline__ uint64_t weigh_uncut(float l) const
    {
        const uint64_t w = entry_weight((l - m) * s.c);
        return w >= s.least ? w : 0u;
    }
    __device__ __forceinline__ double sum_uncut(bool tail) const
    {
        double sum = 0.0;
        if (s.least == 0u) {
            auto add = [&](float l, uint32_t) { sum += (double)__builtin_truncf(entry_weight32((l - m) * s.c)); };
            if (tail) x.each_and_tail(add);
            else x.each(add);
        } else {
            const float least = (float)s.least, near = __builtin_log2f(least) - 40.01f;
            auto add = [&](float l, uint32_t) {
                const float zi = (l - m) * s.c;
                if (zi >= near) {
                    const float w = __builtin_truncf(entry_weight32(zi));
                    sum += w >= least ? (double)w : 0.0;
                }
            };
            if (tail) x.each_and_tail(add);
            else x.each(add);
        }
        return sum;
    }
    // The draw without cuts from a row whose largest entry or scale is infinite.
    __device__ __forceinline__ void draw_odd()
    {
        auto weigh = [&](float l, uint32_t) {
            const uint64_t w = entry_weight(z(l));
            return w >= s.least ? w : 0u;
        };
        uint64_t mine = 0u;
        x.each_again_vectors([&](float l, uint32_t i) { mine += weigh(l, i); });
        draw(mine, weigh);
    }
    __device__ __forceinline__ void list_from(float z0)
    {
        auto want = [&](float l) { return (l - m) * s.c >= z0; };
        x.each_vector([&](const Vec16& y, uint32_t v) { append_vector(y, v, want); });
        append_tail(want);
        __syncthreads();
    }
    // The z, a multiple of -1/2, from which to list a row's (a chunk's) entries: down to where
    // the largest k are among them (then `enough` is set), if `room` takes that many, else
    // as far as it takes them.  Counts go to sh.n.
    static constexpr uint32_t kDepths = 128u;         // down to kLastZ and beyond
    __device__ __forceinline__ float list_depth(uint32_t room, bool& enough)
    {
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < kDepths; j += NT) sh.n[j] = 0u;
        __syncthreads();
        auto count = [&](float l) {
            const float zi = (l - m) * s.c;
            if (zi > kLastZ) atomicAdd(&sh.n[(uint32_t)(zi * -2.0f)], 1u);
        };
        x.each([&](float l, uint32_t) { count(l); });
        if (x.wave == 0u) count(x.last);
        __syncthreads();
        // entries in the depths up to this lane's two
        const uint32_t here = sh.n[2u * x.lane], next = sh.n[2u * x.lane + 1u];
        const uint32_t upto1 = wave_scan(here + next), upto0 = upto1 - next;
        const uint64_t room0 = __ballot(upto0 <= room), room1 = __ballot(upto1 <= room);
        const uint64_t k0 = __ballot(upto0 >= s.k), k1 = __ballot(upto1 >= s.k);
        // depths (of 2 lanes) that fit, a first part of all; the first that reaches k
        const uint32_t fit = (uint32_t)(__builtin_popcountll(room0) + __builtin_popcountll(room1));
        const uint32_t f0 = k0 ? 2u * (uint32_t)__builtin_ctzll(k0) : kDepths, f1 = k1 ? 2u * (uint32_t)__builtin_ctzll(k1) + 1u : kDepths;
        const uint32_t need = min(f0, f1) + 1u;       // depths that hold the first k
        enough = need <= fit || fit == kDepths;
        return __builtin_fmaxf(-0.5f * (float)min(need, fit), kLastZ);        // entries with z > this (none: 0)
    }
    __device__ __forceinline__ void list_above(float z0)
    {
        auto want = [&](float l) { return (l - m) * s.c > z0; };
        x.each_vector([&](const Vec16& y, uint32_t v) { append_vector(y, v, want); });
        append_tail(want);
        __syncthreads();
    }
    // Cut and draw, the entries from kNearZ on being listed.
    __device__ __forceinline__ void draw_near()
    {
        bool done = draw_listed();
        if (!done) {
            bool enough;
            const float z0 = list_depth(Sh::kList, enough);
            if (enough) {
                clear_list();
                list_above(z0);
                done = draw_listed();
            }
        }
        if (!done) draw_dense();
    }

    // Cut and draw where too many entries are close to the largest: bins of z for the
    // whole row, the cut's bin listed, then a pass over the row.
    __device__ __forceinline__ void draw_dense()
    {
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < Sh::kBins; j += NT) {
            sh.n[j] = 0u;
            sh.w[j] = 0u;
        }
        __syncthreads();
        each_live([&](float, uint32_t, float zi) {
            const uint32_t b = bin_of(zi);
            atomicAdd(&sh.n[b], 1u);
            atomicAdd((unsigned long long*)&sh.w[b], (unsigned long long)entry_weight(zi));
        });
        __syncthreads();
        uint64_t n = 0u, whole = 0u;      // the row's, in every thread
        for (uint32_t j = x.lane; j < Sh::kBins; j += 64u) {
            n += sh.n[j];
            whole += sh.w[j];
        }
        n = wave_total(n);
        whole = wave_total(whole);
        uint64_t cut = ~0ull;
        for (uint32_t by_weight = 0u; by_weight < 2u; ++by_weight) {
            uint64_t target = s.k;
            if (by_weight == 0u) {
                if (n <= s.k) continue;
            } else {
                if (s.p24 == kAllP) continue;
                target = share24(whole, s.p24);
                target = target ? target : 1u;
            }
            __syncthreads();
            if (threadIdx.x < 64u) find_bin<Sh::kBins>(sh, sh.n, sh.w, by_weight != 0u, target);
            __syncthreads();
            const uint32_t bin = sh.found;
            const Among in = narrow_to_list(bin, bin, sh.n[bin], sh.before_n, sh.before_w, by_weight != 0u, target);
            find_listed<NT>(sh, in, in.n, [&](uint32_t j) { return sh.list_code[j]; },
                            [&](uint32_t j) { return listed_weight(j); }, by_weight != 0u, target);
            cut = sh.cut;
            if (by_weight == 0u) whole = sh.cut_w;
        }
        auto weigh = [&](float l, uint32_t i) { return weigh_kept(l, i, cut); };
        uint64_t mine = 0u;
        x.each_again_vectors([&](float l, uint32_t i) { mine += weigh(l, i); });
        draw(mine, weigh);
    }
};

// What a row's settings and largest entry ask for.
enum class SampleKind { kEmpty, kGreedy, kOdd, kUncut, kTopP, kTopK };
__device__ __forceinline__ SampleKind sample_kind(const SampleArgs& a, const SampleRow& s, float m)
{
    if (m == -__builtin_inff()) return SampleKind::kEmpty;
    if (s.greedy) return SampleKind::kGreedy;
    if (!(m < __builtin_inff() && s.c < __builtin_inff())) return SampleKind::kOdd;
    if (s.k < a.V) return SampleKind::kTopK;
    return s.p24 < kAllP ? SampleKind::kTopP : SampleKind::kUncut;
}

// CUTS: a row of the call may have a top-k or top-p cut.  Without them the kernel is small
// (512 rows of 151,001 bf16 in 66 instead of 78 us); with all of it 64 registers do not hold
// the state of two workgroups of 1,024 threads to a CU, and 41 (bf16; fp32 43, fp16 57) go to
// scratch memory.
template <int D, int NT, bool CUTS>
__global__ __launch_bounds__(NT, NT == 1024 ? 8 : 4) void k_sample(SampleArgs a)
{
    using R = Row<D, NT, 0>;
    using Sh = SampleShared<NT>;
    __shared__ Sh sh;
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        R x;
        x.open(a.logits, row, a.stride, a.V);
        const SampleRow s = sample_row(a, row);
        if (threadIdx.x == 0u) {
            sh.best = 0xFFFFFFFFu;
            sh.count = 0u;
            sh.near = 0u;
            sh.far = 0u;
        }
        const float m = uniform(group_max<R::NW>(x.max(), sh.f));
        if (R::NW == 1u) __syncthreads();
        SampleGroup<D, NT> g{a, sh, x, s, row, m, 32u - (uint32_t)__builtin_clz(a.V), 0u};
        const SampleKind kind = sample_kind(a, s, m);
        if (kind == SampleKind::kEmpty) {
            if (threadIdx.x == 0u) g.answer(0xFFFFFFFFu, 0.0f);
        } else if (kind == SampleKind::kGreedy) {
            uint32_t at = 0xFFFFFFFFu;
            x.each_and_tail([&](float l, uint32_t i) { at = l == m && i < at ? i : at; });
            if (at != 0xFFFFFFFFu) atomicMin(&sh.best, at);
            __syncthreads();
            if (threadIdx.x == 0u) g.answer(sh.best, 0.0f);
        } else if (kind == SampleKind::kOdd) {
            if constexpr (CUTS) g.draw_dense();
            else g.draw_odd();
        } else if (!CUTS || kind == SampleKind::kUncut) {
            g.draw((uint64_t)g.sum_uncut(false), [&](float l, uint32_t) { return g.weigh_uncut(l); });
        } else if constexpr (CUTS) {
            if (kind == SampleKind::kTopP) {
                g.bin_weights();
                g.draw_top_p(&sh.part_w[0][0], Sh::kParts, x.seg * 64u * (R::NW / Sh::kParts), 0u);
            } else {
                g.list_from(kNearZ);
                g.draw_near();
            }
        }
        __syncthreads();                  // the row's shared memory is used again
    }
}

// ---------------------------------------------------------------------------
// Few rows: each is shared among workgroups, so that a single row's latency is that of a
// chunk.  The first kernel finds the chunks' largest entries, the second weighs, bins or
// lists them, the third makes the draws.  Three launches, because what one workgroup
// tells another within a kernel has to pass the XCDs' separate L2 caches: with a counter by
// which the last workgroup of a row went on to its draw, the write-backs of 448
// workgroups took 64 rows of 50,001 from 69 to 119 us.
constexpr uint32_t kSplitThreads = 1024u;

template <int D>
__global__ __launch_bounds__(kSplitThreads) void k_sample_top(SampleArgs a, SampleSplit p)
{
    using R = Row<D, (int)kSplitThreads, 0>;
    __shared__ float sh[R::NW];
    __shared__ uint32_t best;
    const uint32_t row = blockIdx.y, from = blockIdx.x * p.chunk, group = row * p.chunks + blockIdx.x;
    R x;
    x.open(a.logits, row, a.stride, min(p.chunk, a.V - from), from);
    if (threadIdx.x == 0u) best = 0xFFFFFFFFu;
    const float m = uniform(group_max<R::NW>(x.max(), sh));
    uint32_t at = 0xFFFFFFFFu;
    x.each_and_tail([&](float l, uint32_t i) { at = l == m && i < at ? i : at; });
    if (at != 0xFFFFFFFFu) atomicMin(&best, at);
    __syncthreads();
    if (threadIdx.x == 0u) {
        p.top[group] = m;
        p.top_at[group] = from + best;
    }
}

// The row's largest entry, from its chunks': the first chunk that has it goes to `first`.
__device__ __forceinline__ float split_top(const SampleSplit& p, uint32_t row, uint32_t& first)
{
    const uint32_t lane = threadIdx.x % 64u;
    const float top = lane < p.chunks ? p.top[row * p.chunks + lane] : -__builtin_inff();
    const float m = uniform(wave_max(top));
    first = (uint32_t)__builtin_ctzll(__ballot(top == m));
    return m;
}

template <int D>
__global__ __launch_bounds__(kSplitThreads, 8) void k_sample_chunk(SampleArgs a, SampleSplit p)
{
    constexpr int NT = (int)kSplitThreads;
    using R = Row<D, NT, 0>;
    using Sh = SampleShared<NT>;
    __shared__ Sh sh;
    static_assert(Sh::kList == kSplitList && Sh::kUsedBins == kSplitBins);
    const uint32_t row = blockIdx.y, from = blockIdx.x * p.chunk, group = row * p.chunks + blockIdx.x;
    const SampleRow s = sample_row(a, row);
    uint32_t first;
    const float m = split_top(p, row, first);
    const SampleKind kind = sample_kind(a, s, m);
    if (kind == SampleKind::kEmpty || kind == SampleKind::kGreedy || kind == SampleKind::kOdd) return;
    if (threadIdx.x == 0u) sh.count = 0u;
    R x;
    x.open(a.logits, row, a.stride, min(p.chunk, a.V - from), from);
    SampleGroup<D, NT> part{a, sh, x, s, row, m, 32u - (uint32_t)__builtin_clz(a.V), from};
    __syncthreads();
    if (kind == SampleKind::kUncut) {
        const uint64_t w = wave_total((uint64_t)part.sum_uncut(true));
        if (x.lane == 0u) sh.group[x.wave] = w;
        __syncthreads();
        if (threadIdx.x < 64u) {
            const uint64_t all = wave_total(x.lane < R::NW ? sh.group[x.lane] : 0u);
            if (x.lane == 0u) p.sum[group] = all;
        }
    } else if (kind == SampleKind::kTopP) {
        part.bin_weights();
        for (uint32_t j = threadIdx.x; j < Sh::kUsedBins; j += NT) {
            uint64_t w = 0u;
            for (uint32_t q = 0; q < Sh::kParts; ++q) w += sh.part_w[q][j];
            p.part_w[(uint64_t)group * kSplitBins + j] = w;
        }
    } else {
        bool enough;
        const float z0 = part.list_depth(p.room, enough);
        part.list_above(z0);
        const uint32_t n = min(sh.count, p.room);             // (list_depth keeps within it)
        for (uint32_t j = threadIdx.x; j < n; j += NT) p.list[(uint64_t)group * p.room + j] = sh.list_code[j];
        if (threadIdx.x == 0u) {
            p.count[group] = n;
            p.list_z[group] = enough ? -__builtin_inff() : z0;
        }
    }
}

template <int D>
__global__ __launch_bounds__(kSplitThreads) void k_sample_draw(SampleArgs a, SampleSplit p)
{
    constexpr int NT = (int)kSplitThreads;
    using R = Row<D, NT, 0>;
    __shared__ SampleShared<NT> sh;
    const uint32_t row = blockIdx.x, group0 = row * p.chunks;
    const SampleRow s = sample_row(a, row);
    uint32_t first;
    const float m = split_top(p, row, first);
    const SampleKind kind = sample_kind(a, s, m);
    R x;
    x.open(a.logits, row, a.stride, a.V);
    SampleGroup<D, NT> g{a, sh, x, s, row, m, 32u - (uint32_t)__builtin_clz(a.V), 0u};
    const uint32_t chunk_vectors = p.chunk / R::E, last = p.chunks - 1u;
    if (kind == SampleKind::kUncut)
        for (uint32_t j = threadIdx.x; j < p.chunks; j += NT) sh.sum[j] = p.sum[group0 + j];
    if (threadIdx.x == 0u) {
        sh.count = 0u;
        sh.near = 0u;
        sh.far = 0u;
    }
    __syncthreads();
    if (kind == SampleKind::kTopK) {
        // the chunks' lists down to where all of them reach
        const uint32_t lane = threadIdx.x % 64u;
        const float z0 = uniform(wave_max(lane < p.chunks ? p.list_z[group0 + lane] : -__builtin_inff()));
        for (uint32_t j = threadIdx.x; j < p.chunks * p.room; j += NT) {
            const uint32_t q = j / p.room;
            if (j - q * p.room >= p.count[group0 + q]) continue;
            const uint64_t code = p.list[(uint64_t)group0 * p.room + j];
            if (g.z(rank_logit<D>(code, g.ibits)) > z0) sh.list_code[atomicAdd(&sh.count, 1u)] = code;
        }
        __syncthreads();
    }
    if (kind == SampleKind::kEmpty) {
        if (threadIdx.x == 0u) g.answer(0xFFFFFFFFu, 0.0f);
    } else if (kind == SampleKind::kGreedy) {
        if (threadIdx.x == 0u) g.answer(p.top_at[group0 + first], 0.0f);
    } else if (kind == SampleKind::kOdd) {
        g.draw_dense();
    } else if (kind == SampleKind::kUncut) {
        g.pick_parts(p.chunks, chunk_vectors, last, [&](float l, uint32_t) { return g.weigh_uncut(l); });
    } else if (kind == SampleKind::kTopP) {
        g.draw_top_p(p.part_w + (uint64_t)group0 * kSplitBins, p.chunks, chunk_vectors, last);
    } else {
        g.draw_near();
    }
}

}  // namespace rlsim_dev
