// k_distill.hip.h -- distillation of a student's rows of logits from the top
// logits of a teacher: the loss of each row and its gradient.
//
// The teacher gives k slots of (entry, logit) and, optionally, r, the log of the sum
// of exp(t / tau) over the entries it does not list.  p is the softmax of t / tau (and
// r), q the student's softmax of s / tau, and
//   loss      = tau^2 [ sum_j p_j (ln p_j - ln q_j) + p_r (ln p_r - ln q_r) ]
//   dloss/ds  = tau (q - p) at a listed entry, tau q (1 - p_r / q_r) elsewhere,
// q_r being the unlisted entries' part of q.  q_r is summed over these entries alone, against
// the largest of them (a bit for each entry of the row says which are listed): as
// 1 - sum q_j it would vanish in rounding where the teacher lists nearly all of the mass.
// Exponentials and a thread's sum of them are fp32; what meets in a row's loss is 64 bits, and in
// rows of more than 64 entries so are its gradient's factors.  A gradient is rounded once, to
// the logits' type.
//
// A slot is left out if its entry lies outside the row (-1 marks an empty one) or
// stands in an earlier slot.  A row without any teacher mass has loss 0 and gradient 0
// whatever its logits; so has the gradient of a row of weight 0.
//
// k_distill_few, k_distill_tiny: rows of up to 8 entries, one thread to a row, and of up to
// 64, 16 to 64 lanes to a row.  1,048,576 rows of two fp32 entries 13 us, 42 MB.
// k_distill: longer rows, one workgroup to a row, which is read once for the sum of its
// exponentials against a running maximum and used again for the gradient: from registers
// up to 16,384 2-byte entries, read again beyond (2,048 x 131,072 bf16: as fast in
// registers, one workgroup to a CU, as read again by two).  Bound by the bytes of both
// passes: that case 285-292 us, 3.7 TB/s of logits read and gradient written; 4,097 x 5,003 fp32
// 50-55 us, 3.0-3.3 TB/s; the losses alone of 1,024 x 50,001 fp16 26-29 us, 3.5-3.9 TB/s.
// k_distill_chunk, _join: few long rows, each shared among workgroups; 8 x 262,144 fp32 in
// 14 us, two launches of 5 and 9 us.
// The gradient may overwrite the logits: a thread writes only what it has read, and the
// listed entries' logits are taken before the first write.
#pragma once

#include "head_common.hip.h"

namespace rlsim_dev {

struct DistillArgs {
    const void* logits;
    uint64_t stride;              // elements from row to row
    uint32_t rows, V;
    const void* teacher;          // [rows][k] logits
    uint64_t teacher_stride;
    int teacher_dtype;
    const void* index;            // [rows][k] entries, int32 or int64
    uint64_t index_stride;
    uint32_t index64, k;
    float tau, scale;             // scale: log2(e) / tau
    double inv_tau;
    const float* rest;            // [rows] or null
    const float* weight;          // [rows] or null (1)
    float* loss;                  // [rows] or null
    void* grad;                   // or null
    uint64_t grad_stride;
    uint32_t past_cache;          // the gradient is larger than the last-level cache
};

constexpr uint32_t kNoEntry = 0xFFFFFFFFu;
constexpr float kLowest = -3.40282347e38f;

// A call of few rows shares each among up to 64 workgroups, a chunk of `chunk` entries (a
// multiple of 64 vectors) to each; what the first kernel hands on, by workgroup
// (row * chunks + chunk) or by slot (row * k + slot).
constexpr uint32_t kDistillSplitGroups = 1024u;   // most workgroups of such a call
struct DistillSplit {
    uint32_t chunk, chunks;
    float* mu;                    // [groups] largest entry of the chunk's sum
    double* sum;                  // [groups]
    uint32_t* entry;              // [rows][k]
    float* logit;                 // [rows][k]
};

// A teacher slot: its entry (kNoEntry: left out) and its logit.
struct Slot { uint32_t entry; float t; };
__device__ __forceinline__ Slot load_slot(const DistillArgs& a, uint64_t row, uint32_t j)
{
    Slot s{kNoEntry, -__builtin_inff()};
    const uint64_t at = row * a.index_stride + j;
    const int64_t i = a.index64 ? static_cast<const int64_t*>(a.index)[at] : (int64_t)static_cast<const int32_t*>(a.index)[at];
    if (i >= 0 && i < (int64_t)a.V) {
        s.entry = (uint32_t)i;
        const float t = load_any(a.teacher, row * a.teacher_stride + j, a.teacher_dtype);
        s.t = t == t ? t : __builtin_inff();      // a NaN must not look like an empty row
    }
    return s;
}
__device__ __forceinline__ float rest_value(const DistillArgs& a, uint64_t row)
{
    const float r = a.rest[row];
    return r == r ? r : __builtin_inff();
}

// e^((s - m) / tau) on the exp2 unit, for the row's entries
__device__ __forceinline__ float exp_entry(const DistillArgs& a, float s, float m)
{
    return __builtin_amdgcn_exp2f((s - m) * a.scale);
}
// e^x for the few values whose error would show in the loss: the exponent's whole part
// apart, the rest of it within [-1/2, 1/2] on the unit
__device__ __forceinline__ float exp_slot(double x)
{
    const double z = x * 1.4426950408889634;
    const double n = __builtin_rint(__builtin_fmax(z, -1000.0));
    return __builtin_ldexpf(__builtin_amdgcn_exp2f((float)(z - n)), (int)n);
}

// e^x, x <= 0, for what stands for many entries: the power series of e^(f ln 2 / 64), |f| <= 1/2,
// up to the third power, to the 64th: 2.3e-9, with few constants, each of which takes two
// registers.  0 where fp32 has 0, so that a mass too small for it counts as none.
__device__ __forceinline__ double exp_part(double x)
{
    const double z = x * 1.4426950408889634;
    if (z < -150.0) return 0.0;
    const double n = __builtin_rint(z), y = (z - n) * (0.6931471805599453 / 64.0);
    double e = __builtin_fma(y, 1.0 / 6.0, 0.5);
    e = __builtin_fma(e, y, 1.0);
    e = __builtin_fma(e, y, 1.0);
#pragma unroll
    for (int square = 0; square < 6; ++square) e *= e;
    return __builtin_ldexp(e, (int)n);
}

// A row's logarithms: in short rows of x rounded to fp32, with what was rounded off to first
// order, in longer ones of 64 bits.
struct Log32 {
    __device__ static double of(double x)
    {
        const float f = (float)x;
        return (double)__builtin_logf(f) + (x - (double)f) * (double)(1.0f / f);
    }
};
struct Log64 {
    __device__ static double of(double x) { return ::log(x); }
};

// The loss is ln(sum of student exponentials / sum of teacher ones) plus the mean over p of
// (t - mt) / tau - (s - m) / tau, the logits against their largest.  It is small where
// the student follows its teacher, so what is left of it after the cancellation needs
// more than fp32: differences, sums and logarithms, and in longer rows the exponentials that
// stand for many entries (the teacher's rest, the student's unlisted part; rounded to fp32 each
// showed as 2^-25 tau^2 in the loss), are in 64 bits, which for a few values a row costs nothing
// beside the row.  (Fp32 sums and logarithms of short rows: 1,048,576 rows of two fp32 entries
// 13.3 instead of 13.6 us, losses 4.5e-7 off instead of 1.4e-7.)
// e (x - y) with 0 for e = 0
__device__ __forceinline__ double excess(double e, double x, double y)
{
    return e == 0.0 ? 0.0 : e * (x - y);
}

// A student's row: the largest logit m, and mu and sum, the largest of the pass's entries
// (the unlisted ones where there is a rest, else all) and the sum of their exponentials
// against it, which so cannot vanish beside the listed ones'.  listed: the others' sum
// against m.  0 stands for a largest logit of -inf.
struct Student {
    float m, mu;
    double sum, whole;
    double share;                                 // e^((mu - m) / tau)
};
// ln of an entry's part of `whole`, and (log_rest) of the unlisted entries'
__device__ __forceinline__ double log_part(const DistillArgs& a, float logit, float m)
{
    return ((double)logit - (double)m) * a.inv_tau;
}
__device__ __forceinline__ Student student_row(float m, float mu, double sum, double share, double listed)
{
    Student s{m, mu, sum, 0.0, 0.0};
    s.share = sum == 0.0 ? 0.0 : share;
    s.whole = listed + sum * s.share;
    return s;
}
template <class Log>
__device__ __forceinline__ double log_rest(const DistillArgs& a, const Student& s)
{
    return s.sum == 0.0 ? -__builtin_inf() : log_part(a, s.mu, s.m) + Log::of(s.sum);
}
// `excesses`: their sum over the teacher's values, whose exponentials sum to sum_t
template <class Log>
__device__ __forceinline__ float row_loss(const DistillArgs& a, const Student& s, double excesses, double sum_t)
{
    const double mean = excesses / sum_t;         // +inf where q = 0 < p
    return a.tau * a.tau * (float)(s.whole == 0.0 ? mean : mean + Log::of(s.whole / sum_t));
}

// What a row's gradient is made of: listed entries e^((s - m) / tau) listed - p weighted,
// others e^((s - mu) / tau) other.  Both are differences that nearly cancel where the student
// follows its teacher, so longer rows, whose sums have 64 bits, take them with Real = double:
// four roundings of the factors to fp32 were 2e-6 of the gradient of a row whose first entry
// holds 0.83 of the student and 0.88 of the teacher.
template <class Real> struct GradScale { Real weighted, listed, other; };
template <class Real>
__device__ __forceinline__ GradScale<Real> grad_scale(const DistillArgs& a, const Student& s, float weight, Real p_rest)
{
    GradScale<Real> g;
    g.weighted = (Real)a.tau * (Real)weight;
    const Real inv = s.whole == 0.0 ? (Real)0 : (Real)1 / (Real)s.whole;     // a row of -inf: q = 0
    g.listed = g.weighted * inv;
    g.other = g.weighted * ((Real)s.share * inv - (p_rest == (Real)0 || s.sum == 0.0 ? (Real)0 : p_rest / (Real)s.sum));
    return g;
}

// ---------------------------------------------------------------------------
template <int D, int N>
__global__ __launch_bounds__(256) void k_distill_few(DistillArgs a)
{
    using El = Elem<D>;
    const float none = -__builtin_inff();
    for (uint32_t row = blockIdx.x * 256u + threadIdx.x; row < a.rows; row += gridDim.x * 256u) {
        const typename El::Word* const logits = static_cast<const typename El::Word*>(a.logits) + (uint64_t)row * a.stride;
        float s[N], t[N], e_t[N], e_s[N];
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) {
            s[e] = e < a.V ? El::one(logits[e]) : none;
            t[e] = none;
        }
        const float weight = a.weight ? a.weight[row] : 1.0f;
        const float rest = a.rest ? rest_value(a, row) : none;
        uint32_t listed = 0u;             // a bit for each entry; the first slot that names it counts
        for (uint32_t j = 0; j < a.k; ++j) {
            const Slot slot = load_slot(a, row, j);
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) t[e] = slot.entry == e && !(listed >> e & 1u) ? slot.t : t[e];
            listed |= slot.entry != kNoEntry ? 1u << slot.entry : 0u;
        }
        float top_t = none, m = none, mu = none;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) {
            top_t = __builtin_fmaxf(top_t, t[e]);
            m = __builtin_fmaxf(m, s[e]);
            mu = __builtin_fmaxf(mu, a.rest && (listed >> e & 1u) ? none : s[e]);
        }
        m = m == none ? 0.0f : m;
        mu = mu == none ? 0.0f : mu;
        const double mt = __builtin_fmax((double)top_t * a.inv_tau, (double)rest), x_rest = (double)rest - mt;
        const bool empty = mt == -__builtin_inf();
        const double e_rest = a.rest ? (double)exp_slot(x_rest) : 0.0;
        double sum = 0.0, apart = 0.0, sum_t = e_rest;
        double d = 0.0;
        if (a.rest) {
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) {
                const bool in = listed >> e & 1u;
                const double x = (double)t[e] * a.inv_tau - mt;
                e_t[e] = in ? exp_slot(x) : 0.0f;
                if (in) d += excess(e_t[e], x, log_part(a, s[e], m));
                e_s[e] = e >= a.V ? 0.0f : exp_slot(log_part(a, s[e], in ? m : mu));
                (in ? apart : sum) += (double)e_s[e];
                sum_t += (double)e_t[e];
            }
        } else {
            // The logits' differences alone, in fp32: at most 12 roundings, so off by no more than
            // 2^-20 (|x| + |y|) of an entry's part, x and y its distances from the largest.
            float excesses = 0.0f;
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) {
                const bool in = listed >> e & 1u;
                e_t[e] = in ? exp_entry(a, t[e], top_t) : 0.0f;
                e_s[e] = e >= a.V ? 0.0f : exp_entry(a, s[e], m);
                if (e_t[e] != 0.0f) excesses += e_t[e] * (((t[e] - top_t) - (s[e] - m)) * (float)a.inv_tau);
                sum += (double)e_s[e];
                sum_t += (double)e_t[e];
            }
            d = (double)excesses;
        }
        const Student st = student_row(m, mu, sum, a.rest ? (double)exp_slot(log_part(a, mu, m)) : 1.0, apart);
        if (a.rest) d += excess(e_rest, x_rest, log_rest<Log32>(a, st));
        if (a.loss) a.loss[row] = empty ? 0.0f : row_loss<Log32>(a, st, d, sum_t);
        if (a.grad) {
            const float inv_t = 1.0f / (float)sum_t;
            const GradScale<float> g = grad_scale(a, st, weight, a.rest ? (float)e_rest * inv_t : 0.0f);
            typename El::Word* const grad = static_cast<typename El::Word*>(a.grad) + (uint64_t)row * a.grad_stride;
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) {
                const bool in = listed >> e & 1u;
                float ds = e_s[e] * (a.rest && in ? g.listed : g.other) - (in ? e_t[e] * inv_t * g.weighted : 0.0f);
                if (empty || weight == 0.0f) ds = 0.0f;
                if (e < a.V) grad[e] = El::word(ds);
            }
        }
    }
}

// ---------------------------------------------------------------------------
template <int D, int G>
__global__ __launch_bounds__(256) void k_distill_tiny(DistillArgs a)
{
    using El = Elem<D>;
    const uint32_t e = threadIdx.x % G;
    const uint32_t per_group = 256u / G;
    const float none = -__builtin_inff();
    auto row_max = [](float x) {
#pragma unroll
        for (int off = G / 2; off >= 1; off /= 2) x = __builtin_fmaxf(x, __shfl_xor(x, off, G));
        return x;
    };
    auto row_total = [](double x) {       // rotations within 16 lanes, then across them
        auto turned = [&](uint64_t y) { return __builtin_bit_cast(double, y); };
        x += turned(dpp_u64<0x128, 0xf>(__builtin_bit_cast(uint64_t, x)));
        x += turned(dpp_u64<0x124, 0xf>(__builtin_bit_cast(uint64_t, x)));
        x += turned(dpp_u64<0x122, 0xf>(__builtin_bit_cast(uint64_t, x)));
        x += turned(dpp_u64<0x121, 0xf>(__builtin_bit_cast(uint64_t, x)));
#pragma unroll
        for (int off = 16; off < G; off *= 2) x += __shfl_xor(x, off, G);
        return x;
    };
    for (uint32_t first = blockIdx.x * per_group; first < a.rows; first += gridDim.x * per_group) {
        const uint32_t row = first + threadIdx.x / G;
        const bool live_row = row < a.rows;
        const uint32_t r = live_row ? row : a.rows - 1u;
        const float s = e < a.V ? El::one(static_cast<const typename El::Word*>(a.logits)[(uint64_t)r * a.stride + e]) : none;
        const float weight = a.weight ? a.weight[r] : 1.0f;
        const float rest = a.rest ? rest_value(a, r) : none;
        // this entry's slot: the first that names it
        bool listed = false;
        float t = none;
        for (uint32_t j0 = 0; j0 < a.k; j0 += G) {
            const Slot slot = j0 + e < a.k ? load_slot(a, r, j0 + e) : Slot{kNoEntry, none};
            const uint32_t n = min((uint32_t)G, a.k - j0);
            for (uint32_t j = 0; j < n; ++j) {
                const uint32_t entry = (uint32_t)__shfl((int)slot.entry, (int)j, G);
                const float tj = __shfl(slot.t, (int)j, G);
                t = entry == e && !listed ? tj : t;
                listed = listed || entry == e;
            }
        }
        const double mt = __builtin_fmax((double)row_max(t) * a.inv_tau, (double)rest);
        const bool apart = a.rest && listed;          // not among the entries of the rest
        const float m0 = row_max(s), mu0 = row_max(apart ? none : s);
        const float m = m0 == none ? 0.0f : m0, mu = mu0 == none ? 0.0f : mu0;
        const bool empty = mt == -__builtin_inf();
        const double x = (double)t * a.inv_tau - mt, x_rest = (double)rest - mt;
        const float et = listed ? exp_slot(x) : 0.0f;
        const double e_rest = a.rest ? (double)exp_slot(x_rest) : 0.0, sum_t = row_total((double)et) + e_rest;
        const float inv_t = 1.0f / (float)sum_t, p = et * inv_t, p_rest = a.rest ? (float)e_rest * inv_t : 0.0f;
        const float es = e >= a.V ? 0.0f : apart ? exp_slot(log_part(a, s, m)) : exp_entry(a, s, mu);
        const double sum = row_total(apart ? 0.0 : (double)es);
        const Student st = student_row(m, mu, sum, a.rest ? (double)exp_slot(log_part(a, mu, m)) : 1.0, row_total(apart ? (double)es : 0.0));
        double d = row_total(listed ? excess(et, x, log_part(a, s, m)) : 0.0);
        if (a.rest) d += excess(e_rest, x_rest, log_rest<Log32>(a, st));
        if (!live_row) continue;
        if (a.loss && e == 0u) a.loss[row] = empty ? 0.0f : row_loss<Log32>(a, st, d, sum_t);
        if (a.grad && e < a.V) {
            const GradScale<float> g = grad_scale(a, st, weight, p_rest);
            float ds = es * (apart ? g.listed : g.other) - (listed ? p * g.weighted : 0.0f);
            if (empty || weight == 0.0f) ds = 0.0f;
            static_cast<typename El::Word*>(a.grad)[(uint64_t)row * a.grad_stride + e] = El::word(ds);
        }
    }
}

// ---------------------------------------------------------------------------
// Shared memory beside the reductions': a bit for each entry of the row that is listed,
// then k entries, k teacher logits (then probabilities) and k student logits.
inline __host__ __device__ uint32_t distill_shared_bytes(uint32_t k, uint32_t V) { return (V + 31u) / 32u * 4u + 12u * k; }

template <int NW>
struct DistillShared {
    float max[3][NW];
    double sum[4][NW];
    uint32_t again, mass;                 // whether a slot repeats an earlier one's entry; any has mass
};

// A row, or a chunk of one `from` entries behind its start, as a workgroup's kernel works on
// it; entry, prob and logit hold the row's slots in shared memory.
template <int D, int NT, int NV>
struct DistillGroup {
    using R = Row<D, NT, NV>;
    using El = Elem<D>;
    static constexpr uint32_t E = R::E;
    static constexpr int NW = NT / 64;

    const DistillArgs& a;
    DistillShared<NW>& sh;
    R& x;
    const uint32_t row, from, length;
    uint32_t* const bits;                 // of the chunk's entries: listed
    uint32_t* const entry;                // kNoEntry: left out
    float* const prob;                    // teacher's logit, then exponential
    float* const logit;                   // the student's
    float weight, rest;

    __device__ __forceinline__ void read_scalars()
    {
        weight = uniform(a.weight ? a.weight[row] : 1.0f);
        rest = uniform(a.rest ? rest_value(a, row) : -__builtin_inff());
    }
    __device__ __forceinline__ char* grad() const
    {
        return static_cast<char*>(a.grad) + ((uint64_t)row * a.grad_stride + from) * El::kBytes;
    }
    // Gradients larger than the last-level cache go past it: 2,048 x 131,072 bf16 in 292
    // instead of 312 us.
    __device__ __forceinline__ void store(uint32_t i, const Vec16& v) const
    {
        if (i >= x.vectors) return;
        const typename El::Packed w = {v.w[0], v.w[1], v.w[2], v.w[3]};
        typename El::Packed* const to = reinterpret_cast<typename El::Packed*>(grad()) + i;
        if (a.past_cache) __builtin_nontemporal_store(w, to);
        else *to = w;
    }
    __device__ __forceinline__ void store_one(uint32_t i, float v) const
    {
        reinterpret_cast<typename El::Word*>(grad())[i] = El::word(v);
    }
    __device__ __forceinline__ void store_zeros() const
    {
        for (uint32_t v = 0; v < x.seg; ++v)
            if (x.any(v)) store(x.index(v), Vec16{{0u, 0u, 0u, 0u}});
        if (threadIdx.x < x.tail) store_one(x.vectors * E + threadIdx.x, 0.0f);
    }

    // Mark the chunk's listed entries; a slot that repeats an earlier one's is left out.
    // Returns whether a slot has mass.  Slots outside the chunk are kNoEntry here.
    __device__ __forceinline__ bool mark_listed()
    {
        const uint32_t tid = threadIdx.x;
        const float none = -__builtin_inff();
        for (uint32_t j = tid; j < (length + 31u) / 32u; j += NT) bits[j] = 0u;
        if (tid == 0u) {
            sh.again = 0u;
            sh.mass = 0u;
        }
        __syncthreads();
        for (uint32_t j = tid; j < a.k; j += NT) {
            if (entry[j] == kNoEntry) continue;
            const uint32_t i = entry[j] - from;
            if (atomicOr(&bits[i / 32u], 1u << (i % 32u)) >> (i % 32u) & 1u) sh.again = 1u;
            if (prob[j] != none) sh.mass = 1u;
        }
        __syncthreads();
        if (sh.again == 0u) return sh.mass != 0u;
        uint32_t gone = 0u, left = 0u;    // a bit for each of this thread's slots
        for (uint32_t j = tid, b = 1u; j < a.k; j += NT, b <<= 1) {
            bool repeats = false;
            for (uint32_t i = 0; i < j; ++i) repeats = repeats || entry[i] == entry[j];
            gone |= repeats ? b : 0u;
            left |= !repeats && entry[j] != kNoEntry && prob[j] != none ? 1u : 0u;
        }
        __syncthreads();
        for (uint32_t j = tid, b = 1u; j < a.k; j += NT, b <<= 1)
            if (gone & b) entry[j] = kNoEntry;
        return __syncthreads_or((int)left) != 0;
    }

    // One pass: this thread's largest entry and the exponentials' sum against it, which
    // shrinks as a larger one comes; with a rest, without the listed entries.  It starts
    // from the lowest value, so that a row of -inf has a sum of 0.  A vector is added by
    // pairs: short chains of roundings.
    __device__ __forceinline__ void add_row(float& largest, float& sum)
    {
        const uint32_t at = x.vectors * E + x.lane;
        if (a.rest && x.lane < x.tail && (bits[at / 32u] >> (at % 32u) & 1u)) x.last = -__builtin_inff();
        float mine = kLowest, total = 0.0f;
        x.each_vector([&](const Vec16& y, uint32_t i) {
            Vec16 v = y;
            const uint32_t first = i * E;
            const uint32_t b = a.rest && i < x.vectors ? bits[first / 32u] >> (first % 32u) & ((1u << E) - 1u) : 0u;
            if (b) {
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) v = b >> e & 1u ? El::with_neg_inf(v, e) : v;
            }
            float s[E], top = mine;
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) {
                s[e] = El::get(v, e);
                top = __builtin_fmaxf(top, s[e]);
            }
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) s[e] = exp_entry(a, s[e], top);
#pragma unroll
            for (uint32_t n = E / 2u; n >= 1u; n /= 2u)
#pragma unroll
                for (uint32_t e = 0; e < n; ++e) s[e] += s[e + n];
            total = __builtin_fmaf(total, exp_entry(a, mine, top), s[0]);
            mine = top;
        });
        if (x.wave == 0u) {
            const float top = __builtin_fmaxf(mine, x.last);
            total = __builtin_fmaf(total, exp_entry(a, mine, top), exp_entry(a, x.last, top));
            mine = top;
        }
        largest = mine;
        sum = total;
    }

    // Loss (where `owner`) and gradient, from each thread's largest entry and sum.
    __device__ __forceinline__ void finish(float mine, double sum, bool owner)
    {
        const uint32_t tid = threadIdx.x;
        // the largest values of the row, the listed entries and the teacher's
        float top_l = kLowest, top_t = -__builtin_inff();
        for (uint32_t j = tid; j < a.k; j += NT) {
            if (entry[j] == kNoEntry) continue;
            top_l = __builtin_fmaxf(top_l, logit[j]);
            top_t = __builtin_fmaxf(top_t, prob[j]);
        }
        float mu = wave_max(mine);
        top_l = wave_max(top_l);
        top_t = wave_max(top_t);
        if (NW > 1) {
            if (x.lane == 0u) {
                sh.max[0][x.wave] = mu;
                sh.max[1][x.wave] = top_l;
                sh.max[2][x.wave] = top_t;
            }
            __syncthreads();
            const uint32_t q = min(x.lane, (uint32_t)NW - 1u);
            mu = wave_max(sh.max[0][q]);
            top_l = wave_max(sh.max[1][q]);
            top_t = wave_max(sh.max[2][q]);
        }
        const float m = a.rest ? __builtin_fmaxf(mu, top_l) : mu;
        const double mt = uniform(__builtin_fmax((double)top_t * a.inv_tau, (double)rest));
        const double x_rest = (double)rest - mt, e_rest = uniform(a.rest ? exp_part(x_rest) : 0.0);
        const double share = uniform(exp_part(log_part(a, mu, m)));
        // the sums, and the excesses of the loss
        double part = sum * (double)exp_entry(a, mine, mu), listed = 0.0, sum_t = 0.0, d = 0.0;
        for (uint32_t j = tid; j < a.k; j += NT) {
            if (entry[j] == kNoEntry) continue;
            const double t = (double)prob[j] * a.inv_tau - mt, y = log_part(a, logit[j], m);
            const float e = exp_slot(t);
            prob[j] = e;
            sum_t += (double)e;
            d += excess(e, t, y);
            if (a.rest) listed += (double)exp_slot(y);
        }
        part = wave_total(part);
        listed = wave_total(listed);
        sum_t = wave_total(sum_t);
        d = wave_total(d);
        if (NW > 1) {
            if (x.lane == 0u) {
                sh.sum[0][x.wave] = part;
                sh.sum[1][x.wave] = listed;
                sh.sum[2][x.wave] = sum_t;
                sh.sum[3][x.wave] = d;
            }
            __syncthreads();
            const bool in = x.lane < (uint32_t)NW;
            part = wave_total(in ? sh.sum[0][x.lane] : 0.0);
            listed = wave_total(in ? sh.sum[1][x.lane] : 0.0);
            sum_t = wave_total(in ? sh.sum[2][x.lane] : 0.0);
            d = wave_total(in ? sh.sum[3][x.lane] : 0.0);
        }
        sum_t += e_rest;
        const Student st = student_row(m, mu, part, share, listed);
        if (a.grad) {
            const double inv_t = 1.0 / sum_t;
            const GradScale<double> g = grad_scale(a, st, weight, a.rest ? e_rest * inv_t : 0.0);
            const bool zero = weight == 0.0f;
            const float scale = uniform((float)g.other);
            // in scalar registers, of which one wave's forms have fewer to spare: as many waves
            // to a SIMD as with fp32 factors
            const double to_listed = NW > 1 ? uniform(g.listed) : g.listed;
            const double to_prob = NW > 1 ? uniform(inv_t * g.weighted) : inv_t * g.weighted;
            auto other = [&](float s) { return zero ? 0.0f : exp_entry(a, s, mu) * scale; };
            x.each_vector([&](const Vec16& y, uint32_t i) {
                float f[E];
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) f[e] = other(El::get(y, e));
                store(i, El::pack(f));
            });
            if (tid < x.tail) store_one(x.vectors * E + tid, other(x.last));
            __syncthreads();              // the listed entries over what the pass wrote
            for (uint32_t j = tid; j < a.k; j += NT) {
                const uint32_t i = entry[j] - from;       // (kNoEntry and others' entries: past the chunk)
                if (entry[j] != kNoEntry && i < length)
                    store_one(i, zero ? 0.0f : (float)((double)exp_slot(log_part(a, logit[j], m)) * to_listed
                                                       - (double)prob[j] * to_prob));
            }
        }
        if (a.loss && owner && tid == 0u) {       // last: the logarithms take many registers
            if (a.rest) d += excess(e_rest, x_rest, log_rest<Log64>(a, st));
            a.loss[row] = row_loss<Log64>(a, st, d, sum_t);
        }
    }
};

template <int D, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void k_distill(DistillArgs a)
{
    using G = DistillGroup<D, NT, NV>;
    __shared__ DistillShared<G::NW> sh;
    extern __shared__ uint32_t bits[];
    uint32_t* const entry = bits + (a.V + 31u) / 32u;
    float* const prob = reinterpret_cast<float*>(entry + a.k);
    float* const logit = prob + a.k;
    const uint32_t tid = threadIdx.x;
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        typename G::R x;
        x.open(a.logits, row, a.stride, a.V);
        G g{a, sh, x, row, 0u, a.V, bits, entry, prob, logit, 0.0f, 0.0f};
        g.read_scalars();
        for (uint32_t j = tid; j < a.k; j += NT) {
            const Slot s = load_slot(a, row, j);
            entry[j] = s.entry;
            prob[j] = s.t;
            if (s.entry != kNoEntry) logit[j] = x.entry(s.entry);
        }
        const bool empty = !g.mark_listed() && g.rest == -__builtin_inff();
        if (empty || (g.weight == 0.0f && !a.loss)) {
            if (a.loss && tid == 0u) a.loss[row] = 0.0f;
            if (a.grad) g.store_zeros();
        } else {
            float mine, sum;
            g.add_row(mine, sum);
            g.finish(mine, (double)sum, true);
        }
        __syncthreads();                  // the row's shared memory is used again
    }
}

// ---------------------------------------------------------------------------
// Few rows: each is shared among workgroups, a chunk of its entries to each.  The first
// kernel sums the chunks and takes the student's logits at the listed entries, which a
// gradient in place overwrites in the second; that one joins the chunks' sums, each
// workgroup for itself, and writes its chunk's gradient.
constexpr int kDistillSplitThreads = 256;

template <int D>
__global__ __launch_bounds__(kDistillSplitThreads) void k_distill_chunk(DistillArgs a, DistillSplit p)
{
    constexpr int NT = kDistillSplitThreads;
    using G = DistillGroup<D, NT, 0>;
    __shared__ DistillShared<G::NW> sh;
    extern __shared__ uint32_t bits[];
    uint32_t* const entry = bits + p.chunk / 32u;
    float* const prob = reinterpret_cast<float*>(entry + a.k);
    const uint32_t row = blockIdx.y, from = blockIdx.x * p.chunk, length = min(p.chunk, a.V - from), tid = threadIdx.x;
    typename G::R x;
    x.open(a.logits, row, a.stride, length, from);
    G g{a, sh, x, row, from, length, bits, entry, prob, prob, 0.0f, 0.0f};
    uint32_t* const entries = p.entry + (uint64_t)row * a.k;
    for (uint32_t j = tid; j < a.k; j += NT) {
        const uint32_t i = load_slot(a, row, j).entry;
        entry[j] = i != kNoEntry && i - from < length ? i : kNoEntry;
        prob[j] = 0.0f;
        if (i == kNoEntry && blockIdx.x == 0u) entries[j] = kNoEntry;
    }
    __syncthreads();
    // which slots are this chunk's, as some of them are left out
    uint32_t own = 0u;
    for (uint32_t j = tid, b = 1u; j < a.k; j += NT, b <<= 1) own |= entry[j] != kNoEntry ? b : 0u;
    (void)g.mark_listed();
    for (uint32_t j = tid, b = 1u; j < a.k; j += NT, b <<= 1) {
        if (!(own & b)) continue;
        entries[j] = entry[j];
        if (entry[j] != kNoEntry) p.logit[(uint64_t)row * a.k + j] = x.entry(entry[j] - from);
    }
    float mine, sum;
    g.add_row(mine, sum);
    const float mu = group_max<G::NW>(mine, sh.max[0]);
    double part = wave_total((double)sum * (double)exp_entry(a, mine, mu));
    if (x.lane == 0u) sh.sum[0][x.wave] = part;
    __syncthreads();
    part = wave_total(x.lane < (uint32_t)G::NW ? sh.sum[0][x.lane] : 0.0);
    if (tid == 0u) {
        p.mu[row * p.chunks + blockIdx.x] = mu;
        p.sum[row * p.chunks + blockIdx.x] = part;
    }
}

template <int D>
__global__ __launch_bounds__(kDistillSplitThreads) void k_distill_join(DistillArgs a, DistillSplit p)
{
    constexpr int NT = kDistillSplitThreads;
    using G = DistillGroup<D, NT, 0>;
    __shared__ DistillShared<G::NW> sh;
    extern __shared__ uint32_t entry[];
    float* const prob = reinterpret_cast<float*>(entry + a.k);
    float* const logit = prob + a.k;
    const uint32_t row = blockIdx.y, from = blockIdx.x * p.chunk, length = min(p.chunk, a.V - from), tid = threadIdx.x;
    typename G::R x;
    x.open(a.logits, row, a.stride, length, from);
    G g{a, sh, x, row, from, length, nullptr, entry, prob, logit, 0.0f, 0.0f};
    g.read_scalars();
    int mass = 0;
    for (uint32_t j = tid; j < a.k; j += NT) {
        const uint32_t i = p.entry[(uint64_t)row * a.k + j];
        entry[j] = i;
        if (i == kNoEntry) continue;
        prob[j] = load_slot(a, row, j).t;
        logit[j] = p.logit[(uint64_t)row * a.k + j];
        mass |= prob[j] != -__builtin_inff() ? 1 : 0;
    }
    const bool empty = __syncthreads_or(mass) == 0 && g.rest == -__builtin_inff();
    const bool owner = blockIdx.x == 0u;
    if (empty || (g.weight == 0.0f && !a.loss)) {
        if (a.loss && owner && tid == 0u) a.loss[row] = 0.0f;
        if (a.grad) g.store_zeros();
        return;
    }
    const bool in = x.lane < p.chunks;
    const float mu_c = in ? p.mu[row * p.chunks + x.lane] : kLowest, mu = wave_max(mu_c);
    const double sum = wave_total(in ? p.sum[row * p.chunks + x.lane] * (double)exp_slot(log_part(a, mu_c, mu)) : 0.0);
    g.finish(mu, tid == 0u ? sum : 0.0, owner);
}

}  // namespace rlsim_dev
