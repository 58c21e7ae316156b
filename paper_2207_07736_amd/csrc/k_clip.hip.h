// k_clip.hip.h -- the global norm of many tensors, and their scaling by it.
//
// norm = sqrt(sum x^2).  One pass sums squares in 64 bits, a block of elements to a
// workgroup; the next adds the workgroups' sums in their order, every workgroup for
// itself, and scales.  The sums are at most 6,144 and one to a tensor.  Up to some thousands
// of them from the cache are cheaper than a launch between the two; of very many tensors they
// are most of the call, whose time grows with the square of the tensors' number (of 64 elements
// each: 5,000 0.5 ms, 20,000 3.1, 100,000 51).  The tensors come as kernel arguments, so that a
// captured call keeps no table anywhere else.
//
// Memory bounds both: 48 tensors of 400 M bf16 elements, 800 MB, take 132 us = 6.1 TB/s to
// read and, into tensors of their own, 298 us = 5.4 TB/s; in place the call takes 452.  A call
// within its limit writes nothing: 150 MB in 25 + 6 us.
#pragma once

#include <type_traits>

#include "head_common.hip.h"
#include "learn_dispatch.h"

namespace rlsim_dev {

struct ClipTensor {
    const char* data;
    char* out;
    uint64_t elements;
};
struct ClipArgs {
    ClipTensor t[kClipTensors];
    uint32_t first[kClipTensors + 1];     // the first block of each tensor, of the launch's
    uint8_t dtype[kClipTensors], out_dtype[kClipTensors];
    uint32_t count, base;                 // tensors; blocks of the launches before
    uint32_t blocks;                      // of the whole call
    uint32_t past_cache;                  // more bytes than the last-level cache holds
    uint64_t chunk;                       // elements of a block
    double max_norm;
    double* sums;                         // [blocks]
    float* norm;
};

template <int NT>
__device__ __forceinline__ double group_sum(double x, double* sh)
{
    x = wave_total(x);
    if (threadIdx.x % 64u == 0u) sh[threadIdx.x / 64u] = x;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < NT / 64; ++w) s += sh[w];
    __syncthreads();
    return s;
}

// f(vector of 16 bytes, index) for the whole ones of [from, to), g(float, index) for the rest;
// NT consecutive threads share them.
template <int D, uint32_t NT, class F, class G>
__device__ __forceinline__ void each_vector(const char* p, uint64_t from, uint64_t to, F f, G g)
{
    using El = Elem<D>;
    constexpr uint32_t U = NT == 64u ? 2u : 8u;
    const uint32_t thread = threadIdx.x % NT;
    const uint64_t vectors = (to - from) / El::kPerVec;
    const auto* v = reinterpret_cast<const typename El::Run*>(p + from * El::kBytes);
    for (uint64_t i0 = thread; i0 < vectors; i0 += NT * U) {
        typename El::Run y[U];
#pragma unroll
        for (uint32_t j = 0; j < U; ++j)
            if (i0 + j * NT < vectors) y[j] = v[i0 + j * NT];
#pragma unroll
        for (uint32_t j = 0; j < U; ++j)
            if (i0 + j * NT < vectors) {
                const Vec16 w{{y[j].w[0], y[j].w[1], y[j].w[2], y[j].w[3]}};
                f(w, from + (i0 + j * NT) * El::kPerVec);
            }
    }
    for (uint64_t i = from + vectors * El::kPerVec + thread; i < to; i += NT)
        g(El::one(reinterpret_cast<const typename El::Word*>(p)[i]), i);
}

template <int D, uint32_t NT>
__device__ __forceinline__ double clip_squares(const char* p, uint64_t from, uint64_t to)
{
    double s = 0.0;
    each_vector<D, NT>(p, from, to,
                 [&](const Vec16& v, uint64_t) {
#pragma unroll
                     for (uint32_t e = 0; e < Elem<D>::kPerVec; ++e) {
                         const double x = (double)Elem<D>::get(v, e);
                         s = __builtin_fma(x, x, s);
                     }
                 },
                 [&](float x, uint64_t) { s = __builtin_fma((double)x, (double)x, s); });
    return s;
}

// max_norm / norm as by 2^up: up is 0 but for factors below fp32's normal numbers, which would
// lose digits that the products have.
struct ClipFactor {
    float by;
    int up;
    __device__ __forceinline__ float operator()(float x) const { return ldexpf(x * by, up); }
};
__device__ __forceinline__ ClipFactor clip_factor(double norm, double max_norm)
{
    if (!(norm > max_norm && norm < (double)__builtin_inff())) return ClipFactor{1.0f, 0};
    const double f = max_norm / norm;
    if (f >= 0x1p-126) return ClipFactor{(float)f, 0};
    int up;
    const float by = (float)frexp(f, &up);
    return ClipFactor{by, up};
}

// STREAM: outputs that the last-level cache would not keep go past it, and leave it to what
// the norm's pass has read last, which is scaled first.
template <int D, int O, uint32_t NT, bool STREAM>
__device__ __forceinline__ void clip_scale(const char* p, char* out, uint64_t from, uint64_t to, ClipFactor scale)
{
    using To = Elem<O>;
    each_vector<D, NT>(p, from, to,
                 [&](const Vec16& v, uint64_t i) {
                     constexpr uint32_t E = Elem<D>::kPerVec;
                     struct __attribute__((packed, aligned(To::kBytes))) Run { typename To::Word w[E]; } r;
#pragma unroll
                     for (uint32_t e = 0; e < E; ++e) r.w[e] = To::word(scale(Elem<D>::get(v, e)));
                     if (STREAM) {
                         typedef uint32_t Words __attribute__((ext_vector_type(E * To::kBytes / 4u), aligned(2)));
                         __builtin_nontemporal_store(__builtin_bit_cast(Words, r), reinterpret_cast<Words*>(out + i * To::kBytes));
                     } else {
                         *reinterpret_cast<Run*>(out + i * To::kBytes) = r;
                     }
                 },
                 [&](float x, uint64_t i) { reinterpret_cast<typename To::Word*>(out)[i] = To::word(scale(x)); });
}

// The tensor of a block of the launch.
__device__ __forceinline__ uint32_t clip_tensor(const ClipArgs& a, uint32_t block)
{
    uint32_t lo = 0u, hi = a.count;
    while (hi - lo > 1u) {
        const uint32_t mid = (lo + hi) / 2u;
        if (a.first[mid] <= block) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <uint32_t NT>
__device__ __forceinline__ double squares_of(const ClipArgs& a, uint32_t block)
{
    const uint32_t k = clip_tensor(a, block);
    const uint64_t from = (uint64_t)(block - a.first[k]) * a.chunk, to = min(from + a.chunk, a.t[k].elements);
    return a.dtype[k] == kHeadF32    ? clip_squares<kHeadF32, NT>(a.t[k].data, from, to)
           : a.dtype[k] == kHeadBF16 ? clip_squares<kHeadBF16, NT>(a.t[k].data, from, to)
                                     : clip_squares<kHeadF16, NT>(a.t[k].data, from, to);
}

template <uint32_t NT, bool STREAM>
__device__ __forceinline__ void scale_block(const ClipArgs& a, uint32_t block, ClipFactor scale)
{
    const uint32_t k = clip_tensor(a, block);
    const ClipTensor& t = a.t[k];
    if (scale.by == 1.0f && scale.up == 0 && t.data == t.out) return;
    const uint64_t from = (uint64_t)(block - a.first[k]) * a.chunk, to = min(from + a.chunk, t.elements);
    auto to_type = [&](auto in) {
        constexpr int D = decltype(in)::value;
        if (a.out_dtype[k] == kHeadF32) clip_scale<D, kHeadF32, NT, STREAM>(t.data, t.out, from, to, scale);
        else if (a.out_dtype[k] == kHeadBF16) clip_scale<D, kHeadBF16, NT, STREAM>(t.data, t.out, from, to, scale);
        else clip_scale<D, kHeadF16, NT, STREAM>(t.data, t.out, from, to, scale);
    };
    if (a.dtype[k] == kHeadF32) to_type(std::integral_constant<int, kHeadF32>{});
    else if (a.dtype[k] == kHeadBF16) to_type(std::integral_constant<int, kHeadBF16>{});
    else to_type(std::integral_constant<int, kHeadF16>{});
}

__global__ __launch_bounds__(256) void k_clip_squares(ClipArgs a)
{
    __shared__ double sh[4];
    const double s = group_sum<256>(squares_of<256u>(a, blockIdx.x), sh);
    if (threadIdx.x == 0u) a.sums[a.base + blockIdx.x] = s;
}

__global__ __launch_bounds__(256) void k_clip_scale(ClipArgs a)
{
    __shared__ double sh[4];
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < a.blocks; i += 256u) s += a.sums[i];
    const double norm = sqrt(group_sum<256>(s, sh));
    if (a.base + blockIdx.x == 0u && threadIdx.x == 0u) *a.norm = (float)norm;
    if (!a.count) return;
    const uint32_t block = a.first[a.count] - 1u - blockIdx.x;     // from the end: what was read last
    const ClipFactor scale = clip_factor(norm, a.max_norm);
    if (a.past_cache) scale_block<256u, true>(a, block, scale);
    else scale_block<256u, false>(a, block, scale);
}

// Few elements: one workgroup, one launch.  Its waves take blocks in turn.
__global__ __launch_bounds__(1024) void k_clip_small(ClipArgs a)
{
    __shared__ double sh[16];
    double s = 0.0;
    const uint32_t blocks = a.first[a.count], wave = uniform(threadIdx.x / 64u);
    for (uint32_t b = wave; b < blocks; b += 16u) s += squares_of<64u>(a, b);
    const double norm = sqrt(group_sum<1024>(s, sh));
    if (threadIdx.x == 0u) *a.norm = (float)norm;
    const ClipFactor scale = clip_factor(norm, a.max_norm);
    for (uint32_t b = wave; b < blocks; b += 16u) scale_block<64u, false>(a, b, scale);
}

}  // namespace rlsim_dev
