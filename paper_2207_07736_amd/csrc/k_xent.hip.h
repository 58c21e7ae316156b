// k_xent.hip.h -- the output layer's cross entropy: products of rows on the matrix cores
// with what the loss does to each tile of logits while it is in registers.
//
// All four products are of one form, C[m][n] = sum_k A[m][k] B[n][k], both operands with k
// in consecutive elements:
//   logits     A = matrix   (vocabulary x dim),   B = hidden (rows x dim)
//   dhidden    A = matrix^T (dim x piece),        B = dz     (rows x piece)
//   dmatrix    A = hidden^T (dim x rows),         B = dz^T   (piece x rows)
// A wave's tile of C has four consecutive m in a lane's registers, and n over its lanes:
// a row's softmax sums run within a lane, and outputs leave as runs along the row.
#pragma once

#include "head_common.hip.h"
#include "learn_dispatch.h"

namespace rlsim_dev {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// What a row of the call needs in the gradient's tiles.
struct XentRow {
    float largest, inv_sum, weight;
    int32_t target;                               // -1: the row counts for nothing
};

struct XentGemm {
    const char* A;
    const char* B;
    uint64_t lda, ldb;                            // bytes between rows
    uint64_t part_a, part_b;                      // bytes between the parts of fp32 factors
    uint32_t M, N;
    uint32_t steps, products;                     // steps of one product of parts, how many products
    uint32_t tiles_m, tiles_n, share;             // share: workgroups to a tile
    uint32_t m0;                                  // logits: first entry of the piece
    uint32_t vocab;
    const int32_t* target;                        // logits
    float2* part;                                 // logits, losses: [wave columns][rows_k]
    float* zt;
    uint32_t part0, rows_k;
    const XentRow* row;                           // logits, gradient
    const float* wmax;
    char* dz;                                     // [parts][rows][piece]
    char* dzt;                                    // [parts][piece][rows_k]
    uint64_t dz_ld, dzt_ld, dz_part, dzt_part;    // bytes
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
__device__ __forceinline__ float weight_scale(float wmax)
{
    const int e = (int)(__builtin_bit_cast(uint32_t, wmax) >> 23 & 0xFFu);
    if (e == 0 || e == 255) return 1.0f;          // none, denormal or not finite
    return __builtin_bit_cast(float, (uint32_t)(min(max(253 - e, 1), 254)) << 23);
}

// This wave's loads have arrived (those into LDS are counted as loads, which a barrier
// alone does not wait for), then the workgroup's.
__device__ __forceinline__ void loads_and_group()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// A gradient's last factor: of dhidden the row's weight (and 0 for rows that do not
// count, whatever the product is), of fp16 what dz was scaled by.
template <int F>
struct OutScale {
    float by = 1.0f;
    bool counts = true;
    __device__ __forceinline__ OutScale(const XentRow* row, const float* wmax, uint32_t n)
    {
        const float down = F == kHeadF16 ? kDzDown : 1.0f;
        if (row) {
            counts = row[n].target >= 0;
            by = row[n].weight * down;
        } else if (F == kHeadF16) {
            by = down / weight_scale(*wmax);
        }
    }
    __device__ __forceinline__ float operator()(float x) const { return counts ? x * by : 0.0f; }
};

// D: the type of the factors' (parts'), F: of the call (fp32: three parts).
template <int D, int F, int BM, int BN, int WM, int WN, int EPI>
__global__ __launch_bounds__(64 * WM * WN) void k_xent_gemm(XentGemm a)
{
    constexpr uint32_t NW = WM * WN;
    constexpr uint32_t FM = BM / WM / 32, FN = BN / WN / 32;
    constexpr uint32_t LA = BM * 8 / (64 * NW), LB = BN * 8 / (64 * NW);   // loads of 16 bytes a thread
    static_assert(LA * 64 * NW == BM * 8 && LB * 64 * NW == BN * 8);
    __shared__ __attribute__((aligned(1024))) char sh[2][(BM + BN) * 128];

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

    // A row of 64 elements is 8 chunks of 16 bytes; chunk c of row r lies at place c ^ r % 8
    // of the row in LDS, so that the lanes that read one chunk of 8 rows meet all banks.
    // Rows behind the last one are the last one again (a tile may lie behind it whole).
    const uint32_t m_from = min(m_base, a.M - 1u), n_from = min(n_base, a.N - 1u);
    uint32_t at_a[LA], at_b[LB];
    const uint32_t chunk = (lane % 8u ^ lane / 8u) * 16u;
#pragma unroll
    for (uint32_t i = 0; i < LA; ++i)
        at_a[i] = (min(m_base + (i * NW + wave) * 8u + lane / 8u, a.M - 1u) - m_from) * (uint32_t)a.lda + chunk;
#pragma unroll
    for (uint32_t i = 0; i < LB; ++i)
        at_b[i] = (min(n_base + (i * NW + wave) * 8u + lane / 8u, a.N - 1u) - n_from) * (uint32_t)a.ldb + chunk;
    const char* const A0 = a.A + (uint64_t)m_from * a.lda;
    const char* const B0 = a.B + (uint64_t)n_from * a.ldb;

    // the parts of product p, small products first: (2,0) (1,1) (0,2) (1,0) (0,1) (0,0)
    const uint32_t all = a.steps * a.products;
    const uint32_t first = (uint32_t)((uint64_t)all * blockIdx.y / a.share);
    const uint32_t last = (uint32_t)((uint64_t)all * (blockIdx.y + 1u) / a.share);
    uint32_t product = first / a.steps, step = first % a.steps;
    const char *pa, *pb;
    auto locate = [&]() {
        const uint32_t i = a.products == 1u ? 0u : 0x001012u >> (4u * product) & 15u;
        const uint32_t j = a.products == 1u ? 0u : 0x010210u >> (4u * product) & 15u;
        pa = A0 + i * a.part_a + step * 128u;
        pb = B0 + j * a.part_b + step * 128u;
    };
    locate();
    auto fetch = [&](char* to) {
#pragma unroll
        for (uint32_t i = 0; i < LA; ++i)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(pa + at_a[i]),
                                             (__attribute__((address_space(3))) void*)(to + (i * NW + wave) * 1024u), 16, 0, 0);
#pragma unroll
        for (uint32_t i = 0; i < LB; ++i)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(pb + at_b[i]),
                                             (__attribute__((address_space(3))) void*)(to + BM * 128u + (i * NW + wave) * 1024u), 16, 0, 0);
        pa += 128;
        pb += 128;
        if (++step == a.steps) {
            step = 0u;
            ++product;
            if (product < a.products) locate();
        }
    };

    f32x16 c[FM][FN];
#pragma unroll
    for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
        for (uint32_t j = 0; j < FN; ++j) c[i][j] = f32x16{};

    const uint32_t row_a = (wm * (BM / WM) + lane % 32u) * 128u, row_b = BM * 128u + (wn * (BN / WN) + lane % 32u) * 128u;
    auto multiply = [&](const char* from) {
#pragma unroll
        for (uint32_t k = 0; k < 4u; ++k) {
            const uint32_t place = ((2u * k + lane / 32u) ^ lane % 8u) * 16u;
            u32x4 x[FM], y[FN];
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i) x[i] = *reinterpret_cast<const u32x4*>(from + row_a + i * 4096u + place);
#pragma unroll
            for (uint32_t j = 0; j < FN; ++j) y[j] = *reinterpret_cast<const u32x4*>(from + row_b + j * 4096u + place);
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                for (uint32_t j = 0; j < FN; ++j) c[i][j] = Matrix<D>::mma(x[i], y[j], c[i][j]);
        }
    };

    // One step is in registers' work while the next one's loads are under way.
    if (first < last) {
        fetch(sh[0]);
#pragma unroll 1
        for (uint32_t t = first; t < last; t += 2u) {
            loads_and_group();
            if (t + 1u < last) fetch(sh[1]);
            multiply(sh[0]);
            loads_and_group();
            if (t + 1u < last) {
                if (t + 2u < last) fetch(sh[0]);
                multiply(sh[1]);
            }
        }
    }

    const uint32_t m_wave = m_base + wm * (BM / WM) + 4u * (lane / 32u);
#pragma unroll
    for (uint32_t j = 0; j < FN; ++j) {
        const uint32_t n = n_base + wn * (BN / WN) + j * 32u + lane % 32u;
        if (EPI == kXentLoss) {
            // largest logit and sum of this wave's entries of row n, and the target's logit
            float top = -__builtin_inff();
            const int32_t target = n < a.N ? a.target[n] : -1;
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
            const float weight = F == kHeadF16 ? r.weight * weight_scale(*a.wmax) * kDzUp : r.weight;
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                for (uint32_t q = 0; q < 4u; ++q) {
                    const uint32_t m = m_wave + i * 32u + q * 8u;
                    uint16_t w[3][4];
#pragma unroll
                    for (uint32_t e = 0; e < 4u; ++e) {
                        const uint32_t v = a.m0 + m + e;
                        float p = exp_of(c[i][j][4u * q + e] - r.largest) * r.inv_sum;
                        if ((int32_t)v == r.target) p -= 1.0f;
                        if (v >= a.vocab || r.target < 0) p = 0.0f;
                        if (F == kHeadF32) {
                            uint16_t x[3], y[3];
                            cut3(p, x);
                            cut3(p == 0.0f ? 0.0f : p * weight, y);
#pragma unroll
                            for (uint32_t s = 0; s < 3u; ++s) {
                                w[s][e] = x[s];
                                if (n < a.rows_k)
                                    *reinterpret_cast<uint16_t*>(a.dzt + s * a.dzt_part + (m + e) * a.dzt_ld + 2u * n) = y[s];
                            }
                        } else {
                            w[0][e] = Elem<D>::word(p * up);
                            if (n < a.rows_k)
                                *reinterpret_cast<uint16_t*>(a.dzt + (m + e) * a.dzt_ld + 2u * n) = Elem<D>::word(p == 0.0f ? 0.0f : p * weight);
                        }
                    }
                    if (n < a.N) {
#pragma unroll
                        for (uint32_t s = 0; s < (F == kHeadF32 ? 3u : 1u); ++s) {
                            struct alignas(8) Four { uint16_t w[4]; } four{{w[s][0], w[s][1], w[s][2], w[s][3]}};
                            *reinterpret_cast<Four*>(a.dz + s * a.dz_part + n * a.dz_ld + 2u * m) = four;
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
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                for (uint32_t q = 0; q < 4u; ++q) {
                    const uint32_t m = m_wave + i * 32u + q * 8u;
                    using Word = typename Elem<F>::Word;
                    struct __attribute__((packed, aligned(Elem<F>::kBytes))) Four { Word w[4]; } four;
#pragma unroll
                    for (uint32_t e = 0; e < 4u; ++e) four.w[e] = Elem<F>::word(scale(c[i][j][4u * q + e]));
                    if (m + 4u <= a.M) {
                        *reinterpret_cast<Four*>(to + (uint64_t)m * sizeof(Word)) = four;
                    } else {
#pragma unroll
                        for (uint32_t e = 0; e < 3u; ++e)
                            if (m + e < a.M) reinterpret_cast<Word*>(to)[m + e] = four.w[e];
                    }
                }
        }
    }
}

// Targets as int32, -1 for those outside the vocabulary, and the largest |weight|.
struct XentPrepare {
    const void* target;
    int bytes;
    uint32_t rows, rows_k, vocab;
    int32_t* out;
};
__global__ __launch_bounds__(256) void k_xent_targets(XentPrepare a, float* wmax)
{
    const uint32_t r = blockIdx.x * 256u + threadIdx.x;
    if (r == 0u) *wmax = 0.0f;
    if (r >= a.rows_k) return;
    int64_t t = -1;
    if (r < a.rows)
        t = a.bytes == 1   ? (int64_t) static_cast<const uint8_t*>(a.target)[r]
            : a.bytes == 4 ? (int64_t) static_cast<const int32_t*>(a.target)[r]
                           : static_cast<const int64_t*>(a.target)[r];
    a.out[r] = t >= 0 && t < (int64_t)a.vocab ? (int32_t)t : -1;
}

// Rows' largest logits and sums from their parts (or as given), the losses, and what the
// gradient's tiles need of a row.
struct XentJoin {
    const float2* part;                           // null: stats is an input
    uint32_t parts, rows, rows_k;
    const float* zt;
    const int32_t* target;
    const float* weight;
    float* stats;
    float* loss;
    XentRow* row;                                 // null: losses alone
    float* wmax;
};
__global__ __launch_bounds__(256) void k_xent_join(XentJoin a)
{
    __shared__ float2 sh[16][16];
    const uint32_t x = threadIdx.x % 16u, y = threadIdx.x / 16u, r = blockIdx.x * 16u + x;
    float2 s{-__builtin_inff(), 0.0f};
    if (a.part) {
        if (r < a.rows) {
#pragma unroll 4
            for (uint32_t i = y; i < a.parts; i += 16u) s.x = __builtin_fmaxf(s.x, a.part[(uint64_t)i * a.rows_k + r].x);
            const float from = s.x == -__builtin_inff() ? 0.0f : s.x;
#pragma unroll 4
            for (uint32_t i = y; i < a.parts; i += 16u) {
                const float2 p = a.part[(uint64_t)i * a.rows_k + r];
                s.y += p.y * exp_of(p.x - from);
            }
        }
        sh[y][x] = s;
        __syncthreads();
        if (y != 0u) return;
        for (uint32_t i = 1; i < 16u; ++i) s.x = __builtin_fmaxf(s.x, sh[i][x].x);
        const float from = s.x == -__builtin_inff() ? 0.0f : s.x;
        s.y = 0.0f;
        for (uint32_t i = 0; i < 16u; ++i) s.y += sh[i][x].y * exp_of(sh[i][x].x - from);
    } else if (y != 0u) {
        return;
    }
    if (r >= a.rows) return;
    if (!a.part) s = reinterpret_cast<const float2*>(a.stats)[r];
    else if (a.stats) reinterpret_cast<float2*>(a.stats)[r] = s;
    const int32_t target = a.target[r];
    if (a.loss) a.loss[r] = target < 0 ? 0.0f : logf(s.y) + (s.x - a.zt[r]);
    if (a.row) {
        const float w = a.weight ? a.weight[r] : 1.0f;
        const bool counts = target >= 0 && w != 0.0f;
        a.row[r] = XentRow{s.x, 1.0f / s.y, counts ? w : 0.0f, counts ? target : -1};
        // for finite weights the order of these does not matter
        if (counts && __builtin_fabsf(w) < __builtin_inff())
            atomicMax(reinterpret_cast<uint32_t*>(a.wmax), __builtin_bit_cast(uint32_t, __builtin_fabsf(w)));
    }
}

// Rows as the products read them: whole steps wide, fp32 in three parts, and transposed.
struct XentLay {
    const char* from;                             // [R][C]
    uint64_t ld;                                  // bytes
    uint32_t R, C;
    char* straight;                               // [parts][R][straight_ld], or null
    uint64_t straight_ld, straight_part;          // bytes
    uint32_t wide;                                // elements of a straight row
    char* across;                                 // [parts][C][across_ld], or null
    uint64_t across_ld, across_part;
    uint32_t tall;                                // elements of a transposed row
    const XentRow* row;                           // rows that do not count are 0 across
};
template <int F>
__global__ __launch_bounds__(256) void k_xent_lay(XentLay a)
{
    using El = Elem<F>;
    constexpr uint32_t P = F == kHeadF32 ? 3u : 1u;
    __shared__ uint16_t tile[P][64][66];
    const uint32_t c0 = blockIdx.x * 64u, r0 = blockIdx.y * 64u;
    const uint32_t x = threadIdx.x % 64u;
    for (uint32_t y = threadIdx.x / 64u; y < 64u; y += 4u) {
        const uint32_t r = r0 + y, c = c0 + x;
        uint16_t w[3] = {0, 0, 0};
        if (r < a.R && c < a.C) {
            const auto word = reinterpret_cast<const typename El::Word*>(a.from + r * a.ld)[c];
            if (F == kHeadF32) cut3(El::one(word), w);
            else w[0] = (uint16_t)word;
        }
        if (a.straight && r < a.R && c < a.wide)
            for (uint32_t p = 0; p < P; ++p)
                *reinterpret_cast<uint16_t*>(a.straight + p * a.straight_part + r * a.straight_ld + 2ull * c) = w[p];
        const bool counts = !a.row || (r < a.R && a.row[r].target >= 0);
        for (uint32_t p = 0; p < P; ++p) tile[p][y][x] = counts ? w[p] : (uint16_t)0;
    }
    if (!a.across) return;
    __syncthreads();
    for (uint32_t y = threadIdx.x / 64u; y < 64u; y += 4u) {
        const uint32_t c = c0 + y, r = r0 + x;
        if (c < a.C && r < a.tall)
            for (uint32_t p = 0; p < P; ++p)
                *reinterpret_cast<uint16_t*>(a.across + p * a.across_part + c * a.across_ld + 2ull * r) = tile[p][x][y];
    }
}

// A gradient from its shares: summed in order, scaled, rounded once.
struct XentRound {
    const float* sum;
    uint64_t ld, share_ld;
    uint32_t share, rows, dim;
    const XentRow* row;                           // dhidden: a row's weight; rows that do not count are 0
    const float* wmax;                            // dmatrix of fp16: the weights' scale
    char* out;
    uint64_t out_ld;                              // bytes
};
template <int F>
__global__ __launch_bounds__(256) void k_xent_round(XentRound a)
{
    using El = Elem<F>;
    const uint32_t per = (a.dim + 255u) / 256u;
    const uint32_t n = blockIdx.x / per, d = blockIdx.x % per * 256u + threadIdx.x;
    if (d >= a.dim) return;
    float s = 0.0f;
    for (uint32_t i = 0; i < a.share; ++i) s += a.sum[i * a.share_ld + n * a.ld + d];
    const OutScale<F> scale(a.row, a.wmax, n);
    reinterpret_cast<typename El::Word*>(a.out + n * a.out_ld)[d] = El::word(scale(s));
}

}  // namespace rlsim_dev
