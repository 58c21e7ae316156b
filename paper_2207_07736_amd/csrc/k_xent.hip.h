// k_xent.hip.h -- the output layer's cross entropy: products of rows on the matrix cores
// with what the loss does to each tile of logits while it is in registers.
//
// All products are of one form, C[m][n] = sum_k A[m][k] B[n][k].  An operand lies in
// memory with k in consecutive elements ("along") or with m or n so ("across"); those are
// turned on their way from LDS to the matrix cores, by its transposing reads:
//   logits     A = matrix (vocabulary x dim) along,   B = hidden (rows x dim) along
//   dhidden    A = matrix (piece x dim) across,       B = dz     (rows x piece) along
//   dmatrix    A = hidden (rows x dim) across,        B = dz     (rows x piece) across
// A wave's tile of C has four consecutive m in a lane's registers, and n over its lanes:
// a row's softmax sums run within a lane, and outputs leave as runs along the row.
#pragma once

#include <type_traits>

#include "head_common.hip.h"
#include "learn_dispatch.h"

namespace rlsim_dev {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

// What a row of the call needs in the gradient's tiles.
struct XentRow {
    float largest, inv_sum, weight;
    int32_t target;                               // -1: the row counts for nothing
};

// The rows' targets as given: -1 for one outside the vocabulary.
struct XentTarget {
    const void* p;
    int bytes;
    uint32_t vocab;
    __device__ __forceinline__ int32_t operator()(uint32_t r) const
    {
        const int64_t t = bytes == 1   ? (int64_t) static_cast<const uint8_t*>(p)[r]
                          : bytes == 4 ? (int64_t) static_cast<const int32_t*>(p)[r]
                                       : static_cast<const int64_t*>(p)[r];
        return t >= 0 && t < (int64_t)vocab ? (int32_t)t : -1;
    }
};

struct XentGemm {
    const char* A;
    const char* B;
    uint64_t lda, ldb;                            // bytes between rows
    uint64_t part_a, part_b;                      // bytes between the parts of fp32 factors
    uint32_t M, N;
    uint32_t K;                                   // the summed dimension; along operands may go on behind it (of
    uint32_t steps, products;                     // fp32 they are 0 there), across ones end; products of parts
    uint32_t tiles_m, tiles_n, share;             // share: workgroups to a tile
    uint32_t m0;                                  // logits: first entry of the piece
    uint32_t vocab;
    XentTarget target;                            // logits
    float2* part;                                 // logits, losses: [wave columns][rows_k]
    float* zt;
    uint32_t part0, rows_k;
    const XentRow* row;                           // logits, gradient
    const float* wmax;
    char* dz;                                     // [parts][rows_k][piece], with the rows' weights
    char* dz_plain;                               // fp16: without them, or null
    uint64_t dz_ld, dz_part;                      // bytes
    float* sum;                                   // gradients' products: [share][N][sum_ld]
    uint64_t sum_ld, sum_share;                   // elements
    uint32_t add;                                 // to what is there
    char* out;                                    // gradients' products, rounded: [N][M]
    uint64_t out_ld;                              // bytes
    const XentRow* out_row;                       // dhidden: a row's weight
};

// What becomes of a tile: softmax sums, the logits' gradient, fp32 sums, a gradient.
enum : int { kXentLoss = 0, kXentDz = 1, kXentSum = 2, kXentOut = 3 };

template <int D> struct Matrix;
template <> struct Matrix<kHeadBF16> {
    __device__ __forceinline__ static f32x16 mma(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Matrix<kHeadF16> {
    __device__ __forceinline__ static f32x16 mma(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

// fp32 as a sum of three bf16 parts of 8 bits each (what is not finite stays in the first).
__device__ __forceinline__ void cut3(float x, uint16_t (&p)[3])
{
    p[0] = Elem<kHeadBF16>::word(x);
    const float r1 = x - Elem<kHeadBF16>::one(p[0]);
    const bool fine = __builtin_fabsf(r1) < __builtin_inff();      // false for NaN too
    p[1] = fine ? Elem<kHeadBF16>::word(r1) : (uint16_t)0;
    const float r2 = r1 - Elem<kHeadBF16>::one(p[1]);
    p[2] = fine ? Elem<kHeadBF16>::word(r2) : (uint16_t)0;
}

// dz of fp16 factors is kept times 2^14, as probabilities below 2^-14 would lose bits.
constexpr float kDzUp = 16384.0f, kDzDown = 1.0f / 16384.0f;
// The power of two that brings the largest weight to [1/2, 1), for fp16.
// (No weights: 1.)
__device__ __forceinline__ float weight_scale(const float* wmax)
{
    if (!wmax) return 1.0f;
    const int e = (int)(__builtin_bit_cast(uint32_t, *wmax) >> 23 & 0xFFu);
    if (e == 0 || e == 255) return 1.0f;          // none, denormal or not finite
    return __builtin_bit_cast(float, (uint32_t)(min(max(253 - e, 1), 254)) << 23);
}

// Lane l has entries 0 .. 3 of two blocks of 8, lane l + 32 entries 4 .. 7 of both: lane l
// gets the first block whole, lane l + 32 the second.
__device__ __forceinline__ u32x4 eight_of(const uint16_t (&w)[8])
{
    const uint32_t a0 = w[0] | (uint32_t)w[1] << 16, a1 = w[2] | (uint32_t)w[3] << 16;
    const uint32_t b0 = w[4] | (uint32_t)w[5] << 16, b1 = w[6] | (uint32_t)w[7] << 16;
    const auto s0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false);
    const auto s1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
    return u32x4{s0[0], s1[0], s0[1], s1[1]};
}

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// A gradient's last factor: 0 for dhidden's rows that do not count, whatever the product
// is; of fp16 what dz was scaled by, and the row's weight where dz is without it.
template <int F>
struct OutScale {
    float by = 1.0f;
    bool counts = true;
    __device__ __forceinline__ OutScale(const XentRow* row, const float* wmax, uint32_t n)
    {
        if (row) counts = row[n].target >= 0;
        if (F == kHeadF16) by = row ? row[n].weight * kDzDown : kDzDown / weight_scale(wmax);
    }
    __device__ __forceinline__ float operator()(float x) const { return counts ? x * by : 0.0f; }
};

// Entries m .. m + 3 of a row of M, rounded.
template <int F>
__device__ __forceinline__ void put_four(char* row, uint32_t m, uint32_t M, float x0, float x1, float x2, float x3)
{
    using El = Elem<F>;
    using Word = typename El::Word;
    struct __attribute__((packed, aligned(El::kBytes))) Four { Word w[4]; } four{{El::word(x0), El::word(x1), El::word(x2), El::word(x3)}};
    if (m + 4u <= M) {
        *reinterpret_cast<Four*>(row + (uint64_t)m * El::kBytes) = four;
    } else {
#pragma unroll
        for (uint32_t e = 0; e < 3u; ++e)
            if (m + e < M) reinterpret_cast<Word*>(row)[m + e] = four.w[e];
    }
}

// Entries m .. m + 7 of a row of M, of 16 bits.
__device__ __forceinline__ void put_eight(char* row, uint32_t m, uint32_t M, u32x4 w)
{
    typedef uint32_t Packed __attribute__((ext_vector_type(4), aligned(2)));
    if (m + 8u <= M) {
        *reinterpret_cast<Packed*>(row + 2ull * m) = w;
    } else {
#pragma unroll
        for (uint32_t e = 0; e < 7u; ++e)
            if (m + e < M) reinterpret_cast<uint16_t*>(row)[m + e] = (uint16_t)(w[e / 2u] >> 16u * (e % 2u));
    }
}

// One operand of a tile: R rows of C (m or n), 32 k of them at a time in LDS, which has 64
// banks of 4 bytes.
//
// Along: a row is 64 bytes, 4 chunks of 16; chunk c of row r lies at place c ^ (r / 4) % 4
// of it, so that 16 lanes that read one chunk of 16 rows meet all banks (by (r / 2) % 4, which
// suits 32 banks, half of the reads' cycles were conflicts).
// Across: row k is 2 R bytes; its blocks of 32 bytes lie at place b ^ turn(k), so that the 32
// bytes of 4 rows k that 16 lanes turn, and those of the next 16 lanes, meet all banks.
template <bool ACROSS, uint32_t R, uint32_t NW>
struct Operand {
    static constexpr uint32_t kBytes = R * 64u;                  // of LDS, for a step of 32 k
    static constexpr uint32_t kParts = R / 16u;                  // that one wave loads at once; where there are fewer
    static constexpr uint32_t kLoads = (kParts + NW - 1u) / NW;  // than waves, two load the same
    static_assert(kParts % NW == 0u || NW % kParts == 0u);
    static constexpr uint32_t kRowChunks = R / 8u;               // across: chunks of 16 bytes of a row k
    uint32_t at[kLoads];                                         // bytes from the tile's first

    __device__ __forceinline__ static uint32_t turn(uint32_t k) { return ((k & 3u) ^ (k & 1u) << 2) & (R / 16u - 1u); }
    __device__ __forceinline__ static uint32_t place(uint32_t i, uint32_t wave, uint32_t lane)    // of 16 bytes in LDS
    {
        return (i * NW + wave) % kParts * 64u + lane;
    }

    // base: the tile's first row of C; rows: how many there are in all.  What lies behind
    // the last one is taken from the last ones again.
    __device__ __forceinline__ void open(uint32_t base, uint32_t rows, uint32_t ld, uint32_t wave, uint32_t lane)
    {
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) {
            const uint32_t p = place(i, wave, lane);
            if (ACROSS) {
                const uint32_t k = p / kRowChunks, c = p % kRowChunks ^ 2u * turn(k);
                const uint32_t last = (rows + 7u) / 8u - 1u;                     // chunk of a whole row
                at[i] = min(base / 8u + c, last) * 16u + k * ld;
            } else {
                const uint32_t r = p / 4u, c = p % 4u ^ r / 4u % 4u;
                at[i] = (min(base + r, rows - 1u) - min(base, rows - 1u)) * ld + c * 16u;
            }
        }
    }
    __device__ __forceinline__ static uint64_t first(uint32_t base, uint32_t rows, uint64_t ld)
    {
        return ACROSS ? 0u : min(base, rows - 1u) * ld;
    }
    // 32 k from p on into LDS.  CUT: of the first `left` of them, a multiple of 8 along; what lies
    // behind is the row's last chunk, or the last row k, again.
    template <bool CUT>
    __device__ __forceinline__ void fetch(const char* p, char* to, uint32_t ld, uint32_t left, uint32_t wave, uint32_t lane) const
    {
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) {
            uint32_t off = at[i];
            if (ACROSS && CUT) {
                const uint32_t k = place(i, wave, lane) / kRowChunks;
                off -= (k - min(k, left - 1u)) * ld;
            }
            if (!ACROSS && CUT) {
                const uint32_t q = place(i, wave, lane), c = q % 4u ^ q / 4u / 4u % 4u;
                off -= (c - min(c, (left + 7u) / 8u - 1u)) * 16u;
            }
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p + off),
                                             (__attribute__((address_space(3))) void*)(to + (i * NW + wave) % kParts * 1024u), 16, 0, 0);
        }
    }
};
// The fragments of F blocks of 32 rows of C, for the 16 k of half `h` of a step.
template <bool ACROSS, uint32_t R, uint32_t F>
struct Fragments {
    uint32_t at[F];
    u32x4 v[2][F];
    __device__ __forceinline__ void open(uint32_t base, uint32_t lane)
    {
#pragma unroll
        for (uint32_t i = 0; i < F; ++i) {
            if (ACROSS) {
                const uint32_t p = lane % 16u, k = 8u * (lane / 32u) + p / 4u;
                const uint32_t block = (base + i * 32u) / 16u + lane / 16u % 2u;
                at[i] = k * (R * 2u) + (block ^ Operand<true, R, 1u>::turn(k)) * 32u + p % 4u * 8u;
            } else {
                at[i] = (base + i * 32u + lane % 32u) * 64u + (lane / 32u ^ lane / 4u % 4u) * 16u;
            }
        }
    }
    // Along: 0 instead of what has k at or behind `left`, which lies in other rows.
    template <uint32_t H>
    __device__ __forceinline__ void cut(uint32_t left, uint32_t lane)
    {
        if (ACROSS || left >= 16u * H + 16u) return;
#pragma unroll
        for (uint32_t i = 0; i < F; ++i)
            if (16u * H + lane / 32u * 8u >= left) v[H][i] = u32x4{0u, 0u, 0u, 0u};
    }
    template <uint32_t H>
    __device__ __forceinline__ void read(const char* from)
    {
#pragma unroll
        for (uint32_t i = 0; i < F; ++i) {
            if (ACROSS) {
                typedef __attribute__((address_space(3))) i16x4* At;
                const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(from + at[i] + H * (R * 32u)));
                const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(from + at[i] + H * (R * 32u) + R * 8u));
                const uint2 l = __builtin_bit_cast(uint2, lo), u = __builtin_bit_cast(uint2, hi);
                v[H][i] = u32x4{l.x, l.y, u.x, u.y};
            } else {
                v[H][i] = *reinterpret_cast<const u32x4*>(from + (at[i] ^ H * 32u));
            }
        }
    }
};

// At most N of this wave's loads are still under way; none of its reads of LDS is.  (The
// builtin, not the instruction as text: the compiler counts them too.)
template <int N>
__device__ __forceinline__ void loads_left()
{
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
}
__device__ __forceinline__ void reads_done() { __builtin_amdgcn_s_waitcnt(0xC07F); }
// The order of a half step's instructions: reads of LDS and loads between the matrix
// instructions, whose 32 cycles hide their issue.
template <int MMA, int READS, int LOADS>
__device__ __forceinline__ void mix()
{
    constexpr int kPer = MMA > 2 ? (READS + MMA - 3) / (MMA - 2) : READS;
#pragma unroll
    for (int i = 0; i < MMA; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (i * kPer < READS) __builtin_amdgcn_sched_group_barrier(0x100, kPer, 0);
        if (i < LOADS) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
    }
}
// The workgroup's waves meet.  No access to memory moves over it; what is under way stays so.
__device__ __forceinline__ void meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// D: the type of the factors' (parts'), F: of the call (fp32: three parts); AA, BA: whether
// A and B lie across.
template <int D, int F, int BM, int BN, int WM, int WN, bool AA, bool BA, int EPI>
__global__ __launch_bounds__(64 * WM * WN) void k_xent_gemm(XentGemm a)
{
    constexpr uint32_t NW = WM * WN;
    constexpr uint32_t FM = BM / WM / 32, FN = BN / WN / 32;
    using OpA = Operand<AA, BM, NW>;
    using OpB = Operand<BA, BN, NW>;
    // Four steps' operands.  Arrays of their own, and a loop that names them: the compiler has
    // to see that a read of one does not touch what loads under way write to another.
    constexpr uint32_t kStage = OpA::kBytes + OpB::kBytes;
    __shared__ __attribute__((aligned(1024))) char sh0[kStage], sh1[kStage], sh2[kStage], sh3[kStage];

    const uint32_t lane = threadIdx.x % 64u, wave = uniform(threadIdx.x / 64u);
    const uint32_t wm = wave / WN, wn = wave % WN;

    // Workgroups go round the 8 XCDs: each takes a run of tiles of its own, so that its L2
    // sees the same operands again.  Within a run m goes fastest past 8 columns of n.
    const uint32_t tiles = a.tiles_m * a.tiles_n;
    uint32_t id = blockIdx.x;
    {
        const uint32_t q = tiles / 8u, r = tiles % 8u, x = id % 8u, i = id / 8u;
        id = x * q + min(x, r) + i;
    }
    constexpr uint32_t G = 8u;
    const uint32_t band = id / (G * a.tiles_m), in = id % (G * a.tiles_m);
    const uint32_t width = min(G, a.tiles_n - band * G);
    const uint32_t tn = band * G + in % width, tm = in / width;
    const uint32_t m_base = tm * BM, n_base = tn * BN;

    OpA op_a;
    OpB op_b;
    const uint32_t lda = (uint32_t)a.lda, ldb = (uint32_t)a.ldb;
    op_a.open(m_base, a.M, lda, wave, lane);
    op_b.open(n_base, a.N, ldb, wave, lane);
    const char* const A0 = a.A + OpA::first(m_base, a.M, a.lda);
    const char* const B0 = a.B + OpB::first(n_base, a.N, a.ldb);
    const uint64_t step_a = AA ? 32u * a.lda : 64u, step_b = BA ? 32u * a.ldb : 64u;

    // the parts of product p, small products first: (2,0) (1,1) (0,2) (1,0) (0,1) (0,0)
    const uint32_t all = a.steps * a.products;
    const uint32_t first = (uint32_t)((uint64_t)all * blockIdx.y / a.share);
    const uint32_t last = (uint32_t)((uint64_t)all * (blockIdx.y + 1u) / a.share);
    uint32_t product = first / a.steps, step = first % a.steps;
    const char *pa, *pb;
    auto locate = [&]() {
        const uint32_t i = a.products == 1u ? 0u : 0x001012u >> (4u * product) & 15u;
        const uint32_t j = a.products == 1u ? 0u : 0x010210u >> (4u * product) & 15u;
        pa = A0 + i * a.part_a + step * step_a;
        pb = B0 + j * a.part_b + step * step_b;
    };
    locate();
    // CUT: K may end within the step.
    auto fetch = [&](auto cut, char* to) {
        constexpr bool CUT = decltype(cut)::value;
        const uint32_t left = CUT ? a.K - step * 32u : 32u;
        op_a.template fetch<CUT>(pa, to, lda, left, wave, lane);
        op_b.template fetch<CUT && !BA>(pb, to + OpA::kBytes, ldb, left, wave, lane);
        pa += step_a;
        pb += step_b;
        ++step;
        if (F == kHeadF32 && step == a.steps) {
            step = 0u;
            ++product;
            if (product < a.products) locate();
        }
    };
    constexpr int kEach = OpA::kLoads + OpB::kLoads, kReads = FM * (AA ? 2u : 1u) + FN * (BA ? 2u : 1u);

    f32x16 c[FM][FN];
#pragma unroll
    for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
        for (uint32_t j = 0; j < FN; ++j) c[i][j] = f32x16{};

    Fragments<AA, BM, FM> x;
    Fragments<BA, BN, FN> y;
    x.open(wm * (BM / WM), lane);
    y.open(wn * (BN / WN), lane);

    // Up to four steps of 32 k are in LDS or under way.  While a half step of 16 k is
    // multiplied, the next one's fragments are read; the workgroup meets once, in the middle
    // of a step, after which the next one may be read.
    auto cut = [&](auto half, uint32_t t) {       // (parts of fp32 are copies that end with whole steps)
        constexpr uint32_t H = decltype(half)::value;
        if (F == kHeadF32 || a.K >= t * 32u + 32u) return;
        x.template cut<H>(a.K - t * 32u, lane);
        y.template cut<H>(a.K - t * 32u, lane);
    };
    auto one_step = [&](auto steady, uint32_t t, char* now, char* next, char* ahead) {
        constexpr bool kSteady = decltype(steady)::value;        // three more steps are to come
        reads_done();                             // of the first half
        x.template read<1>(now);
        y.template read<1>(now + OpA::kBytes);
        if (!kSteady) cut(std::integral_constant<uint32_t, 1u>{}, t);
#pragma unroll
        for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
            for (uint32_t j = 0; j < FN; ++j) c[i][j] = Matrix<D>::mma(x.v[0][i], y.v[0][j], c[i][j]);
        mix<FM * FN, kReads, 0>();
        __builtin_amdgcn_sched_barrier(0);
        if (kSteady || t + 2u < last) loads_left<kEach>();       // the next step has arrived
        else loads_left<0>();
        reads_done();
        meet();
        if (kSteady) fetch(std::false_type{}, ahead);
        else if (t + 3u < last) fetch(std::true_type{}, ahead);
        if (kSteady || t + 1u < last) {
            x.template read<0>(next);
            y.template read<0>(next + OpA::kBytes);
            if (!kSteady) cut(std::integral_constant<uint32_t, 0u>{}, t + 1u);
        }
#pragma unroll
        for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
            for (uint32_t j = 0; j < FN; ++j) c[i][j] = Matrix<D>::mma(x.v[1][i], y.v[1][j], c[i][j]);
        mix<FM * FN, kReads, kSteady ? kEach : 0>();
        __builtin_amdgcn_sched_barrier(0);
    };
    if (first < last) {
        fetch(std::true_type{}, sh0);
        if (first + 2u < last) {
            fetch(std::true_type{}, sh1);
            fetch(std::true_type{}, sh2);
            loads_left<2 * kEach>();
        } else {
            if (first + 1u < last) fetch(std::true_type{}, sh1);
            loads_left<0>();
        }
        meet();
        x.template read<0>(sh0);
        y.template read<0>(sh0 + OpA::kBytes);
        cut(std::integral_constant<uint32_t, 0u>{}, first);
        uint32_t t = first;
        constexpr std::true_type steady{};
        constexpr std::false_type ending{};
#pragma unroll 1
        for (; t + 6u < last; t += 4u) {
            one_step(steady, t, sh0, sh1, sh3);
            one_step(steady, t + 1u, sh1, sh2, sh0);
            one_step(steady, t + 2u, sh2, sh3, sh1);
            one_step(steady, t + 3u, sh3, sh0, sh2);
        }
#pragma unroll 1
        for (; t < last; t += 4u) {
            one_step(ending, t, sh0, sh1, sh3);
            if (t + 1u < last) one_step(ending, t + 1u, sh1, sh2, sh0);
            if (t + 2u < last) one_step(ending, t + 2u, sh2, sh3, sh1);
            if (t + 3u < last) one_step(ending, t + 3u, sh3, sh0, sh2);
        }
    }

    const uint32_t m_wave = m_base + wm * (BM / WM) + 4u * (lane / 32u);
#pragma unroll
    for (uint32_t j = 0; j < FN; ++j) {
        const uint32_t n = n_base + wn * (BN / WN) + j * 32u + lane % 32u;
        if (EPI == kXentLoss) {
            // largest logit and sum of this wave's entries of row n, and the target's logit
            float top = -__builtin_inff();
            const int32_t target = n < a.N ? a.target(n) : -1;
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                for (uint32_t e = 0; e < 16u; ++e) {
                    const uint32_t v = a.m0 + m_wave + i * 32u + e / 4u * 8u + e % 4u;
                    if (v >= a.vocab) c[i][j][e] = -__builtin_inff();
                    top = __builtin_fmaxf(top, c[i][j][e]);
                    if ((int32_t)v == target) a.zt[n] = c[i][j][e];
                }
            top = __builtin_fmaxf(top, __shfl_xor(top, 32));
            const float from = top == -__builtin_inff() ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                for (uint32_t e = 0; e < 16u; ++e) sum += exp_of(c[i][j][e] - from);
            sum += __shfl_xor(sum, 32);
            if (lane < 32u && n < a.N) a.part[(uint64_t)(a.part0 + tm * WM + wm) * a.rows_k + n] = float2{top, sum};
        }
        if (EPI == kXentDz) {
            XentRow r{0.0f, 0.0f, 0.0f, -1};
            if (n < a.N) r = a.row[n];
            const float up = F == kHeadF16 ? kDzUp : 1.0f;
            const float weight = F == kHeadF16 ? r.weight * weight_scale(a.wmax) * kDzUp : r.weight;
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                for (uint32_t q = 0; q < 4u; ++q) {
#pragma unroll
                    for (uint32_t e = 0; e < 4u; ++e) {
                        const uint32_t v = a.m0 + m_wave + i * 32u + q * 8u + e;
                        float p = exp_of(c[i][j][4u * q + e] - r.largest) * r.inv_sum;
                        if ((int32_t)v == r.target) p -= 1.0f;
                        c[i][j][4u * q + e] = v >= a.vocab || r.target < 0 ? 0.0f : p;
                    }
                }
            if (n < a.rows_k) {
                char* const to = a.dz + n * a.dz_ld;
#pragma unroll
                for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                    for (uint32_t q = 0; q < 4u; q += 2u) {
                        uint16_t w[3][8], plain[8];
#pragma unroll
                        for (uint32_t e = 0; e < 8u; ++e) {
                            const float p = c[i][j][4u * q + e];
                            const float pw = p == 0.0f ? 0.0f : p * weight;
                            uint16_t cut[3];
                            if (F == kHeadF32) cut3(pw, cut);
                            else cut[0] = Elem<D>::word(pw);
#pragma unroll
                            for (uint32_t s = 0; s < (F == kHeadF32 ? 3u : 1u); ++s) w[s][e] = cut[s];
                            plain[e] = F == kHeadF16 ? Elem<D>::word(p * up) : (uint16_t)0;
                        }
                        const uint64_t m = m_base + wm * (BM / WM) + i * 32u + (q + lane / 32u) * 8u;
#pragma unroll
                        for (uint32_t s = 0; s < (F == kHeadF32 ? 3u : 1u); ++s)
                            *reinterpret_cast<u32x4*>(to + s * a.dz_part + 2u * m) = eight_of(w[s]);
                        if (F == kHeadF16 && a.dz_plain)
                            *reinterpret_cast<u32x4*>(a.dz_plain + n * a.dz_ld + 2u * m) = eight_of(plain);
                    }
            }
        }
        if (EPI == kXentSum) {
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                for (uint32_t q = 0; q < 4u; ++q) {
                    const uint32_t m = m_wave + i * 32u + q * 8u;
                    if (n < a.N && m < a.sum_ld) {        // sum_ld: M up to a multiple of 4
                        float4* to = reinterpret_cast<float4*>(a.sum + blockIdx.y * a.sum_share + n * a.sum_ld + m);
                        float4 s{c[i][j][4u * q], c[i][j][4u * q + 1u], c[i][j][4u * q + 2u], c[i][j][4u * q + 3u]};
                        if (a.add) {
                            const float4 old = *to;
                            s.x += old.x, s.y += old.y, s.z += old.z, s.w += old.w;
                        }
                        *to = s;
                    }
                }
        }
        if (EPI == kXentOut && n < a.N) {
            const OutScale<F> scale(a.out_row, a.wmax, n);
            char* const to = a.out + n * a.out_ld;
            if (F == kHeadF32) {
#pragma unroll
                for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                    for (uint32_t q = 0; q < 4u; ++q)
                        put_four<F>(to, m_wave + i * 32u + q * 8u, a.M, scale(c[i][j][4u * q]), scale(c[i][j][4u * q + 1u]),
                                    scale(c[i][j][4u * q + 2u]), scale(c[i][j][4u * q + 3u]));
            } else {
#pragma unroll
                for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                    for (uint32_t q = 0; q < 4u; q += 2u) {
                        uint16_t w[8];
#pragma unroll
                        for (uint32_t e = 0; e < 8u; ++e) w[e] = (uint16_t)Elem<F>::word(scale(c[i][j][4u * q + e]));
                        put_eight(to, m_base + wm * (BM / WM) + i * 32u + (q + lane / 32u) * 8u, a.M, eight_of(w));
                    }
            }
        }
    }
}

// Rows' largest logits and sums from their parts (or as given), the losses, and what the
// gradient's tiles need of a row.
struct XentJoin {
    const float2* part;                           // null: stats is an input
    uint32_t parts, rows, rows_k;
    const float* zt;
    XentTarget target;
    const float* weight;
    float* stats;
    float* loss;
    XentRow* row;                                 // null: losses alone
};
// Of two runs of a row, each its largest logit and its sum of exp(z - largest).
__device__ __forceinline__ float2 joined(float2 p, float2 q)
{
    const float top = __builtin_fmaxf(p.x, q.x), from = top == -__builtin_inff() ? 0.0f : top;
    return float2{top, p.y * exp_of(p.x - from) + q.y * exp_of(q.x - from)};
}
constexpr uint32_t kJoinRows = 4u, kJoinRuns = 256u / kJoinRows;    // of a workgroup; threads to a row
__device__ __forceinline__ void xent_join(const XentJoin& a, uint32_t block)
{
    __shared__ float2 sh[kJoinRuns][kJoinRows];
    const uint32_t x = threadIdx.x % kJoinRows, y = threadIdx.x / kJoinRows, r = block * kJoinRows + x;
    float2 s{-__builtin_inff(), 0.0f};
    if (a.part) {
        if (r < a.rows) {
#pragma unroll 8
            for (uint32_t i = y; i < a.parts; i += kJoinRuns) s = joined(s, a.part[(uint64_t)i * a.rows_k + r]);
        }
        sh[y][x] = s;
        __syncthreads();
        for (uint32_t half = kJoinRuns / 2u; half != 0u; half /= 2u) {
            if (y < half) sh[y][x] = joined(sh[y][x], sh[y + half][x]);
            __syncthreads();
        }
        if (y != 0u) return;
        s = sh[0][x];
    } else if (y != 0u) {
        return;
    }
    if (r >= a.rows) return;
    if (!a.part) s = reinterpret_cast<const float2*>(a.stats)[r];
    else if (a.stats) reinterpret_cast<float2*>(a.stats)[r] = s;
    const int32_t target = a.target(r);
    if (a.loss) a.loss[r] = target < 0 ? 0.0f : logf(s.y) + (s.x - a.zt[r]);
    if (a.row) {
        const float w = a.weight ? a.weight[r] : 1.0f;
        const bool counts = target >= 0 && w != 0.0f;
        a.row[r] = XentRow{s.x, 1.0f / s.y, counts ? w : 0.0f, counts ? target : -1};
    }
}

// The largest finite |weight| of the rows that count.
__global__ __launch_bounds__(1024) void k_xent_wmax(XentTarget target, const float* weight, uint32_t rows, float* wmax)
{
    __shared__ float sh[16];
    float top = 0.0f;
    for (uint32_t r = threadIdx.x; r < rows; r += 1024u) {
        const float w = __builtin_fabsf(weight[r]);
        if (w < __builtin_inff() && target(r) >= 0) top = __builtin_fmaxf(top, w);
    }
    top = group_max<16>(top, sh);
    if (threadIdx.x == 0u) *wmax = top;
}

// Rows as the products read them: whole steps wide, fp32 in three parts; rows that do not
// count are 0 where they are told.
struct XentLay {
    const char* from;                             // [R][C]
    uint64_t ld;                                  // bytes
    uint32_t R, C, wide, tall;                    // wide: elements of a row of the copy, a multiple of 8;
    char* to;                                     // [parts][tall][wide], 0 behind R and C
    uint64_t part;                                // bytes
    XentTarget target;                            // p null: all rows count
    const float* weight;
    uint32_t blocks;
};
template <int F>
__device__ __forceinline__ void xent_lay(const XentLay& a, uint32_t block)
{
    using El = Elem<F>;
    constexpr uint32_t P = F == kHeadF32 ? 3u : 1u;
    const uint32_t per = a.wide / 8u;
    const uint64_t all = (uint64_t)a.tall * per;
    for (uint64_t i = (uint64_t)block * 256u + threadIdx.x; i < all; i += (uint64_t)a.blocks * 256u) {
        const uint32_t r = (uint32_t)(i / per), c = (uint32_t)(i % per) * 8u;
        uint16_t w[P][8] = {};
        if (r < a.R && (!a.target.p || (a.target(r) >= 0 && !(a.weight && a.weight[r] == 0.0f)))) {
            struct __attribute__((packed, aligned(El::kBytes))) Eight { typename El::Word w[8]; } x{};
            const auto* from = reinterpret_cast<const typename El::Word*>(a.from + r * a.ld) + c;
            if (c + 8u <= a.C) {
                x = *reinterpret_cast<const Eight*>(from);
            } else {
#pragma unroll
                for (uint32_t e = 0; e < 7u; ++e)
                    if (c + e < a.C) x.w[e] = from[e];
            }
#pragma unroll
            for (uint32_t e = 0; e < 8u; ++e) {
                uint16_t cut[3] = {(uint16_t)x.w[e], 0, 0};
                if (F == kHeadF32) cut3(El::one(x.w[e]), cut);
#pragma unroll
                for (uint32_t p = 0; p < P; ++p) w[p][e] = cut[p];
            }
        }
#pragma unroll
        for (uint32_t p = 0; p < P; ++p)
            *reinterpret_cast<u32x4*>(a.to + p * a.part + i * 16u) =
                u32x4{w[p][0] | (uint32_t)w[p][1] << 16, w[p][2] | (uint32_t)w[p][3] << 16,
                      w[p][4] | (uint32_t)w[p][5] << 16, w[p][6] | (uint32_t)w[p][7] << 16};
    }
}

// Two copies in one launch, or the rows' sums and a copy.
template <int F>
__global__ __launch_bounds__(256) void k_xent_lays(XentLay a, XentLay b)
{
    if (blockIdx.x < a.blocks) xent_lay<F>(a, blockIdx.x);
    else xent_lay<F>(b, blockIdx.x - a.blocks);
}
template <int F>
__global__ __launch_bounds__(256) void k_xent_join(XentJoin a, XentLay b)
{
    const uint32_t blocks = (a.rows + kJoinRows - 1u) / kJoinRows;
    if (blockIdx.x < blocks) xent_join(a, blockIdx.x);
    else xent_lay<F>(b, blockIdx.x - blocks);
}

// A gradient from its shares: summed in order, scaled, rounded once.
struct XentRound {
    const float* sum;
    uint64_t ld, share_ld;
    uint32_t share, rows, dim;
    const XentRow* row;                           // dhidden: rows that do not count are 0; fp16: a row's weight
    const float* wmax;                            // dmatrix of fp16: the weights' scale
    char* out;
    uint64_t out_ld;                              // bytes
    uint32_t blocks;
};
template <int F>
__device__ __forceinline__ void xent_round(const XentRound& a, uint32_t block)
{
    const uint32_t per = (a.dim + 3u) / 4u;       // of four entries
    const uint64_t i = (uint64_t)block * 256u + threadIdx.x;
    if (i >= (uint64_t)a.rows * per) return;
    const uint32_t n = (uint32_t)(i / per), d = (uint32_t)(i % per) * 4u;
    float4 s{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
    for (uint32_t k = 0; k < a.share; ++k) {
        const float4 x = *reinterpret_cast<const float4*>(a.sum + k * a.share_ld + n * a.ld + d);
        s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
    }
    const OutScale<F> scale(a.row, a.wmax, n);
    put_four<F>(a.out + n * a.out_ld, d, a.dim, scale(s.x), scale(s.y), scale(s.z), scale(s.w));
}
template <int F>
__global__ __launch_bounds__(256) void k_xent_round(XentRound a, XentRound b)
{
    if (blockIdx.x < a.blocks) xent_round<F>(a, blockIdx.x);
    else xent_round<F>(b, blockIdx.x - a.blocks);
}

}  // namespace rlsim_dev
