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
//
// The logits are computed twice (for the sums; for dz, piece by piece): 8 rows dim vocab
// operations for a loss with its gradients, where an array of all logits would allow 6.
// 4,096 rows of 4,096 on 131,072 in bf16, ms: sums 3.53 (1,246 TFLOP/s), dz 4.03 (1,091),
// dhidden 3.72 (1,182), dmatrix 3.59 (1,226); the library's plain product reaches 1,475 to 1,495.
// The matrix units are busy for 71 % of the sums' cycles and 53, 63 and 67 % of the others', at
// 1.55 to 1.84 GHz.  The dz launches write 134 MB each; 224 MB reach memory.  Tried, TFLOP/s of
// the sums beside 1,209 to 1,234 in the same run: four waves of 128 x 128 with 512 registers
// 1,167, tiles of 128 x 128 875, a raised wave priority 1,241 (no difference).
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
    float miss;                                   // 1 - softmax of the target, not as a difference
    float unused[3];
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

constexpr int kDzUp = 14;                         // see XentRefs
__device__ __forceinline__ int ref_of(uint32_t stored) { return stored ? (int)stored - 1024 : 0; }

// A gradient's last factor: 0 for dhidden's rows that do not count, whatever the product
// is, and their weight where dz is without it; the power of two that dz was scaled by.
struct OutScale {
    const XentRow* row;                           // dhidden, or null
    const uint32_t* ref;                          // dz carries 2^(kDzUp - ref), or null
    int32_t up;                                   // else the result is due 2^up
    uint32_t weigh;
    // for row n, found once
    struct Row {
        float by;
        int up;
        bool counts;
        __device__ __forceinline__ float operator()(float x) const { return counts ? ldexpf(x * by, up) : 0.0f; }
    };
    __device__ __forceinline__ Row at(uint32_t n) const
    {
        Row r{1.0f, ref ? ref_of(*ref) - kDzUp : up, true};
        if (row) {
            r.counts = row[n].target >= 0;
            if (weigh) r.by = row[n].weight;
        }
        return r;
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
    const int32_t* up_n;                          // exponents of what rows of hidden (bf16: for dmatrix) and
    const int32_t* up_m;                          // of matrix (fp32) were divided by
    const uint32_t* refs;                         // XentRefs' results
    char* dz_w;                                   // [dz_w_parts][rows_k][piece] for dmatrix: fp16, with the rows' weights, or null
    char* dz;                                     // for dhidden: of the factors' type, without them, or null
    uint32_t dz_w_parts;
    uint32_t dz_stack;                            // bf16, fp16: rows from dz's first part to its second, or 0: one part
    uint64_t dz_ld, dz_part;                      // bytes
    float* sum;                                   // gradients' products: [share][N][sum_ld]
    uint64_t sum_ld, sum_share;                   // elements
    uint32_t add;                                 // to what is there
    const uint32_t* sum_ref;                      // fp32, dhidden: refs' entry of the piece, or null
    char* out;                                    // gradients' products, rounded: [N][M]
    uint64_t out_ld;                              // bytes
    OutScale scale;
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

// fp32 (scaled to below 2^15) as a sum of two fp16 parts: to 22 bits at worst, and to 2^-25
// where it is small.  What is not finite stays in the first.
__device__ __forceinline__ void cut2(float x, uint16_t& hi, uint16_t& lo)
{
    hi = Elem<kHeadF16>::word(x);
    const float rest = x - Elem<kHeadF16>::one(hi);
    lo = __builtin_fabsf(rest) < __builtin_inff() ? Elem<kHeadF16>::word(rest) : (uint16_t)0;
}

// The exponent e of a finite x: |x| < 2^(e + 1) (of 0 and of denormals -127).
__device__ __forceinline__ int exponent_of(float x) { return (int)(__builtin_bit_cast(uint32_t, x) >> 23 & 0xFFu) - 127; }

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

// D: the type of the factors (parts), F: of the call (fp32: two parts); AA, BA: whether
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

    // the parts of product p, small products first: (1,0) (0,1) (0,0), or (0,1) (0,0) where only B
    // has two
    constexpr bool kProducts = F == kHeadF32 || (F == kHeadF16 && BA);
    const uint32_t all = a.steps * a.products;
    const uint32_t first = (uint32_t)((uint64_t)all * blockIdx.y / a.share);
    const uint32_t last = (uint32_t)((uint64_t)all * (blockIdx.y + 1u) / a.share);
    uint32_t product = first / a.steps, step = first % a.steps;
    const char *pa, *pb;
    auto locate = [&]() {
        const uint32_t i = a.products == 1u ? 0u : F == kHeadF32 && product == 0u;
        const uint32_t j = a.products == 1u ? 0u : product + 2u == a.products;
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
        if (kProducts && step == a.steps) {
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
        constexpr bool kSteady = decltype(steady)::value;        // four more steps are to come
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
        for (; t + 7u < last; t += 4u) {          // the last step is not among those loaded here: K may end in it
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
    if (F == kHeadF32 && (EPI == kXentLoss || EPI == kXentDz)) {
        // the logits: what the factors were divided by comes back
        int up_n[FN];
#pragma unroll
        for (uint32_t j = 0; j < FN; ++j) up_n[j] = a.up_n[min(n_base + wn * (BN / WN) + j * 32u + lane % 32u, a.N - 1u)];
#pragma unroll
        for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
            for (uint32_t q = 0; q < 4u; ++q) {
                const int4 up = *reinterpret_cast<const int4*>(a.up_m + m_wave + i * 32u + q * 8u);
                const int up_m[4] = {up.x, up.y, up.z, up.w};
#pragma unroll
                for (uint32_t j = 0; j < FN; ++j)
#pragma unroll
                    for (uint32_t e = 0; e < 4u; ++e) c[i][j][4u * q + e] = ldexpf(c[i][j][4u * q + e], up_n[j] + up_m[e]);
                __builtin_amdgcn_sched_barrier(0);        // few of these loads at a time: registers
            }
    }
#pragma unroll
    for (uint32_t j = 0; j < FN; ++j) {
        const uint32_t n = n_base + wn * (BN / WN) + j * 32u + lane % 32u;
        if (EPI == kXentLoss) {
            // largest logit of this wave's entries of row n, their sum without the target's, and
            // the target's logit
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
                for (uint32_t e = 0; e < 16u; ++e) {
                    const uint32_t v = a.m0 + m_wave + i * 32u + e / 4u * 8u + e % 4u;
                    sum += (int32_t)v == target ? 0.0f : exp_of(c[i][j][e] - from);
                }
            sum += __shfl_xor(sum, 32);
            if (lane < 32u && n < a.N) a.part[(uint64_t)(a.part0 + tm * WM + wm) * a.rows_k + n] = float2{top, sum};
        }
        if (EPI == kXentDz) {
            XentRow r{0.0f, 0.0f, 0.0f, -1};
            if (n < a.N) r = a.row[n];
            // by powers of two to below 2^kDzUp: over the rows, with weights and what the rows of
            // hidden were divided by, or (fp32) over the piece
            int up = kDzUp - ref_of(a.refs[0]);
            if (F != kHeadF16) up += a.up_n[min(n, a.N - 1u)];
            const float weight = r.weight;
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                for (uint32_t q = 0; q < 4u; ++q) {
#pragma unroll
                    for (uint32_t e = 0; e < 4u; ++e) {
                        const uint32_t v = a.m0 + m_wave + i * 32u + q * 8u + e;
                        float p = exp_of(c[i][j][4u * q + e] - r.largest) * r.inv_sum;
                        if ((int32_t)v == r.target) p = -r.miss;
                        c[i][j][4u * q + e] = v >= a.vocab || r.target < 0 ? 0.0f : p;
                    }
                }
            if (n < a.rows_k) {
#pragma unroll
                for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                    for (uint32_t q = 0; q < 4u; q += 2u) {
                        constexpr uint32_t P = F == kHeadF32 ? 2u : 1u;
                        const uint64_t at = n * a.dz_ld + 2u * (m_base + wm * (BM / WM) + i * 32u + (q + lane / 32u) * 8u);
                        // dmatrix's factor: fp16 has 3 bits more than bf16, at the price of one scale
                        // for the call.  Below 2^-28 of the call's largest |weight| x 2^up_n an entry
                        // loses digits, below 2^-39 it is 0.  fp32 has two parts, and fp16 where few
                        // rows decide (kXentFewRows).
                        if (a.dz_w) {
                            uint16_t w[2][8];
#pragma unroll
                            for (uint32_t e = 0; e < 8u; ++e) {
                                const float pw = ldexpf(c[i][j][4u * q + e] * weight, up);      // of rows that do not count 0 by 0
                                if (F != kHeadBF16) cut2(pw, w[0][e], w[1][e]);
                                else w[0][e] = Elem<kHeadF16>::word(pw);
                            }
                            *reinterpret_cast<u32x4*>(a.dz_w + at) = eight_of(w[0]);
                            if (F == kHeadF32 || (F == kHeadF16 && a.dz_w_parts == 2u))
                                *reinterpret_cast<u32x4*>(a.dz_w + at + a.dz_part) = eight_of(w[1]);
                        }
                        // dhidden's factor, in the type that the matrix is multiplied in: bf16, whose
                        // rounding averages out over the vocabulary; fp16 times 2^kDzUp, so that
                        // probabilities from 2^-28 on keep their digits; a second part as rows where
                        // there is room (kXentStackRows); two parts for fp32.
                        if (a.dz && !(a.dz_stack && n >= a.dz_stack)) {
                            uint16_t w[2][8];
#pragma unroll
                            for (uint32_t e = 0; e < 8u; ++e) {
                                const float p = c[i][j][4u * q + e];
                                if (F == kHeadBF16) {
                                    w[0][e] = Elem<kHeadBF16>::word(p);
                                    w[1][e] = Elem<kHeadBF16>::word(p - Elem<kHeadBF16>::one(w[0][e]));
                                }
                                if (F == kHeadF16) cut2(ldexpf(p, kDzUp), w[0][e], w[1][e]);
                                if (F == kHeadF32) {
                                    const int up_m = a.up_m[m_wave + i * 32u + (q + e / 4u) * 8u + e % 4u];
                                    cut2(ldexpf(p, up_m + kDzUp - ref_of(a.refs[1])), w[0][e], w[1][e]);
                                }
                            }
#pragma unroll
                            for (uint32_t s = 0; s < P; ++s) *reinterpret_cast<u32x4*>(a.dz + at + s * a.dz_part) = eight_of(w[s]);
                            if (P == 1u && a.dz_stack) *reinterpret_cast<u32x4*>(a.dz + at + a.dz_stack * a.dz_ld) = eight_of(w[1]);
                        }
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
                        if (F == kHeadF32 && a.sum_ref) {        // pieces are scaled each by its own power of two
                            const int up = ref_of(*a.sum_ref) - kDzUp;
                            s = float4{ldexpf(s.x, up), ldexpf(s.y, up), ldexpf(s.z, up), ldexpf(s.w, up)};
                        }
                        if (a.add) {
                            const float4 old = *to;
                            s.x += old.x, s.y += old.y, s.z += old.z, s.w += old.w;
                        }
                        *to = s;
                    }
                }
        }
        if (EPI == kXentOut && n < a.N) {
            const OutScale::Row scale = a.scale.at(n);
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
// gradient's tiles need of a row.  The target's own term is kept out of the sums: of a row
// whose softmax is nearly all its target's, the loss and the target's gradient are the rest,
// which 1 minus the softmax would round away.
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
    const int32_t target = a.target(r);
    float own = 0.0f;                             // the target's term
    if (a.part) {
        if (target >= 0) own = exp_of(a.zt[r] - (s.x == -__builtin_inff() ? 0.0f : s.x));
        if (a.stats) {
            a.stats[3u * (uint64_t)r] = s.x;
            a.stats[3u * (uint64_t)r + 1u] = s.y;
            a.stats[3u * (uint64_t)r + 2u] = own;
        }
    } else {
        s = float2{a.stats[3u * (uint64_t)r], a.stats[3u * (uint64_t)r + 1u]};
        own = a.stats[3u * (uint64_t)r + 2u];
    }
    if (a.loss) a.loss[r] = target < 0 ? 0.0f : own == 1.0f ? log1pf(s.y) : logf(s.y + own) + (s.x - a.zt[r]);
    if (a.row) {
        const float w = a.weight ? a.weight[r] : 1.0f;
        const bool counts = target >= 0 && w != 0.0f;
        const float inv_sum = 1.0f / (s.y + own);
        a.row[r] = XentRow{s.x, inv_sum, counts ? w : 0.0f, counts ? target : -1, s.y * inv_sum, {}};
    }
}

// The powers of two that dz is scaled by where it is held in fp16, so that the largest that
// it can be is just below 2^kDzUp (a probability below 2^-14 would lose bits of fp16):
//   out[0]  for dmatrix, a bound of |weight| 2^up_n over the rows that count
//   out[1]  for dhidden (fp32), of 2^up_m over the piece
struct XentRefs {
    XentTarget target;
    const float* weight;
    const int32_t* up_n;                          // or null
    const int32_t* up_m;                          // or null
    uint32_t rows, count;
    uint32_t* out;                                // exponents and 1024, 0 for none; null: not wanted
    uint32_t blocks;                              // more than one: out is 0 before
};
constexpr uint32_t kRefRows = 4096u;              // of a workgroup
__device__ __forceinline__ void xent_refs(const XentRefs& a, uint32_t block)
{
    __shared__ uint32_t sh[2][4];
    uint32_t top_n = 0u, top_m = 0u;
#pragma unroll 4
    for (uint32_t r = block * 256u + threadIdx.x; r < a.rows; r += a.blocks * 256u) {
        const float w = a.weight ? a.weight[r] : 1.0f;
        const bool counts = __builtin_fabsf(w) < __builtin_inff() && w != 0.0f && a.target(r) >= 0;
        if (counts) top_n = max(top_n, (uint32_t)(1024 + exponent_of(w) + 1 + (a.up_n ? a.up_n[r] : 0)));
    }
    if (a.up_m) {
#pragma unroll 4
        for (uint32_t v = 4u * (block * 256u + threadIdx.x); v < a.count; v += a.blocks * 1024u) {
            const int4 up = *reinterpret_cast<const int4*>(a.up_m + v);          // whole fours: copies end with steps
            top_m = max(top_m, (uint32_t)(1024 + max(max(up.x, up.y), max(up.z, up.w))));
        }
    }
    top_n = wave_max(top_n);
    top_m = wave_max(top_m);
    if (threadIdx.x % 64u == 0u) {
        sh[0][threadIdx.x / 64u] = top_n;
        sh[1][threadIdx.x / 64u] = top_m;
    }
    __syncthreads();
    if (threadIdx.x < 2u) {
        const uint32_t* const x = sh[threadIdx.x];
        const uint32_t top = max(max(x[0], x[1]), max(x[2], x[3]));
        if (a.blocks == 1u) a.out[threadIdx.x] = top;
        else atomicMax(a.out + threadIdx.x, top);         // the order does not matter
    }
}
__global__ __launch_bounds__(256) void k_xent_refs(XentRefs a) { xent_refs(a, blockIdx.x); }
__global__ void k_xent_refs_none(uint32_t* out)
{
    if (threadIdx.x < 2u) out[threadIdx.x] = 0u;
}

// Rows as the products read them: whole steps wide; rows that do not count are 0 where they
// are told.  Cut rows are divided by a power of two, so that the largest entry is between
// 2^14 and 2^15, and held in fp16: fp32 in two parts, bf16 in one (exactly, but for what is
// below 2^-28 of the largest).
struct XentLay {
    const char* from;                             // [R][C]
    uint64_t ld;                                  // bytes
    uint32_t R, C, wide, tall;                    // wide: elements of a row of the copy, a multiple of 8;
    char* to;                                     // [parts][tall][wide], 0 behind R and C
    uint64_t part;                                // bytes
    XentTarget target;                            // p null: all rows count
    const float* weight;
    int32_t* up;                                  // cut: [tall] exponents of what rows were divided by, or null
    uint32_t cut;
    uint32_t blocks;
    __device__ __forceinline__ bool counts(uint32_t r) const
    {
        return r < R && (!target.p || (target(r) >= 0 && !(weight && weight[r] == 0.0f)));
    }
};
// Cut: a wave to a row.
template <int F>
__device__ __forceinline__ void xent_cut(const XentLay& a, uint32_t block)
{
    using El = Elem<F>;
    using Word = typename El::Word;
    struct __attribute__((packed, aligned(El::kBytes))) Four { Word x[4]; };
    const uint32_t lane = threadIdx.x % 64u;
    for (uint32_t r = uniform(block * 4u + threadIdx.x / 64u); r < a.tall; r += a.blocks * 4u) {
        const Word* const from = reinterpret_cast<const Word*>(a.from + r * a.ld);
        const bool counts = a.counts(r);
        auto load = [&](uint32_t c) {
            Four f{};
            if (counts && c + 4u <= a.C) {
                f = *reinterpret_cast<const Four*>(from + c);
            } else if (counts) {
#pragma unroll
                for (uint32_t e = 0; e < 3u; ++e)
                    if (c + e < a.C) f.x[e] = from[c + e];
            }
            return f;
        };
        uint32_t top = 0u;                        // of the finite ones, as bits
        for (uint32_t c = 4u * lane; c < a.C; c += 256u) {
            const Four f = load(c);
#pragma unroll
            for (uint32_t e = 0; e < 4u; ++e) {
                const uint32_t bits = __builtin_bit_cast(uint32_t, El::one(f.x[e])) & 0x7FFFFFFFu;
                top = max(top, bits < 0x7F800000u ? bits : 0u);
            }
        }
        top = wave_max(top);
        const int up = top ? exponent_of(__builtin_bit_cast(float, top)) - 14 : -500;     // a row of 0 sets no scale
        if (lane == 0u && a.up) a.up[r] = up;
        for (uint32_t c = 4u * lane; c < a.wide; c += 256u) {
            const Four f = load(c);
            uint16_t hi[4], lo[4];
#pragma unroll
            for (uint32_t e = 0; e < 4u; ++e) cut2(ldexpf(El::one(f.x[e]), -up), hi[e], lo[e]);
            char* const to = a.to + ((uint64_t)r * a.wide + c) * 2u;
            *reinterpret_cast<uint2*>(to) = uint2{hi[0] | (uint32_t)hi[1] << 16, hi[2] | (uint32_t)hi[3] << 16};
            if (F == kHeadF32)
                *reinterpret_cast<uint2*>(to + a.part) = uint2{lo[0] | (uint32_t)lo[1] << 16, lo[2] | (uint32_t)lo[3] << 16};
        }
    }
}
template <int F>
__device__ __forceinline__ void xent_lay(const XentLay& a, uint32_t block)
{
    if (F != kHeadF16 && a.cut) {
        xent_cut<F>(a, block);
        return;
    }
    const uint32_t per = a.wide / 8u;
    const uint64_t all = (uint64_t)a.tall * per;
    for (uint64_t i = (uint64_t)block * 256u + threadIdx.x; i < all; i += (uint64_t)a.blocks * 256u) {
        const uint32_t r = (uint32_t)(i / per), c = (uint32_t)(i % per) * 8u;
        struct __attribute__((packed, aligned(2))) Eight { uint16_t w[8]; } x{};
        if (a.counts(r)) {
            const auto* from = reinterpret_cast<const uint16_t*>(a.from + r * a.ld) + c;
            if (c + 8u <= a.C) {
                x = *reinterpret_cast<const Eight*>(from);
            } else {
#pragma unroll
                for (uint32_t e = 0; e < 7u; ++e)
                    if (c + e < a.C) x.w[e] = from[e];
            }
        }
        *reinterpret_cast<u32x4*>(a.to + i * 16u) = __builtin_bit_cast(u32x4, x);
    }
}

// Three copies in one launch; the rows' sums and the powers of two in one.
template <int F>
__global__ __launch_bounds__(256) void k_xent_lays(XentLay a, XentLay b, XentLay c)
{
    if (blockIdx.x < a.blocks) xent_lay<F>(a, blockIdx.x);
    else if (blockIdx.x < a.blocks + b.blocks) xent_lay<F>(b, blockIdx.x - a.blocks);
    else xent_lay<F>(c, blockIdx.x - a.blocks - b.blocks);
}
__global__ __launch_bounds__(256) void k_xent_join(XentJoin a, XentRefs c)
{
    const uint32_t blocks = (a.rows + kJoinRows - 1u) / kJoinRows;
    if (blockIdx.x < blocks) xent_join(a, blockIdx.x);
    else xent_refs(c, blockIdx.x - blocks);
}

// A gradient from its shares: summed in order, scaled, rounded once.
struct XentRound {
    const float* sum;
    uint64_t ld, share_ld;
    uint32_t share, rows, dim;
    uint32_t stack;                               // rows to the second part's sums, or 0
    OutScale scale;
    char* out;
    uint64_t out_ld;                              // bytes
    uint32_t blocks;
};
template <int F>
__device__ __forceinline__ void xent_round(const XentRound& a, uint32_t block)
{
    const uint32_t per = (a.dim + 3u) / 4u;       // of four entries
    for (uint64_t i = (uint64_t)block * 256u + threadIdx.x; i < (uint64_t)a.rows * per; i += (uint64_t)a.blocks * 256u) {
        const uint32_t n = (uint32_t)(i / per), d = (uint32_t)(i % per) * 4u;
        float4 s{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
        for (uint32_t k = 0; k < a.share; ++k) {
            const float4 x = *reinterpret_cast<const float4*>(a.sum + k * a.share_ld + n * a.ld + d);
            s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
        }
        if (a.stack) {
            float4 t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
            for (uint32_t k = 0; k < a.share; ++k) {
                const float4 x = *reinterpret_cast<const float4*>(a.sum + k * a.share_ld + (n + a.stack) * a.ld + d);
                t.x += x.x, t.y += x.y, t.z += x.z, t.w += x.w;
            }
            s.x += t.x, s.y += t.y, s.z += t.z, s.w += t.w;
        }
        const OutScale::Row scale = a.scale.at(n);
        put_four<F>(a.out + n * a.out_ld, d, a.dim, scale(s.x), scale(s.y), scale(s.z), scale(s.w));
    }
}
template <int F>
__global__ __launch_bounds__(256) void k_xent_round(XentRound a, XentRound b)
{
    if (blockIdx.x < a.blocks) xent_round<F>(a, blockIdx.x);
    else xent_round<F>(b, blockIdx.x - a.blocks);
}

}  // namespace rlsim_dev
