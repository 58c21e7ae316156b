// head_common.hip.h -- rows of logits: loads, wave and workgroup reductions, and
// how a workgroup holds a row, shared by the output head's kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rlsim_dev {

constexpr uint32_t kHeadMaxVocab = 1u << 20;      // entries of a row
constexpr uint32_t kHeadMaxTeacher = 1024u;       // teacher slots of a row

// Element types of a row, numbered as the ABI numbers them.
enum : int { kHeadF32 = 0, kHeadBF16 = 1, kHeadF16 = 2 };

struct Vec16 { uint32_t w[4]; };                  // 16 bytes of a row

template <int D> struct Elem;
template <> struct Elem<kHeadF32> {
    static constexpr uint32_t kBytes = 4u, kPerVec = 4u;
    static constexpr uint32_t kNegInf = 0xFF800000u;             // a word of -inf entries
    static constexpr uint32_t kZeroBits = 0u;                    // of an entry as a float
    struct __attribute__((packed, aligned(4))) Run { uint32_t w[4]; };
    typedef uint32_t Packed __attribute__((ext_vector_type(4), aligned(4)));
    using Word = uint32_t;
    __device__ static float get(const Vec16& v, uint32_t e) { return __builtin_bit_cast(float, v.w[e]); }
    __device__ static Vec16 with_neg_inf(Vec16 v, uint32_t e) { v.w[e] = kNegInf; return v; }
    __device__ static float one(Word x) { return __builtin_bit_cast(float, x); }
    __device__ static Word word(float x) { return __builtin_bit_cast(uint32_t, x); }
    __device__ static Vec16 pack(const float (&f)[kPerVec])
    {
        return Vec16{{word(f[0]), word(f[1]), word(f[2]), word(f[3])}};
    }
};
template <> struct Elem<kHeadBF16> {
    static constexpr uint32_t kBytes = 2u, kPerVec = 8u;
    static constexpr uint32_t kNegInf = 0xFF80FF80u;
    static constexpr uint32_t kZeroBits = 16u;
    struct __attribute__((packed, aligned(2))) Run { uint32_t w[4]; };
    typedef uint32_t Packed __attribute__((ext_vector_type(4), aligned(2)));
    using Word = uint16_t;
    __device__ static float get(const Vec16& v, uint32_t e)
    {
        const uint32_t w = v.w[e / 2u];
        return __builtin_bit_cast(float, e % 2u ? w & 0xFFFF0000u : w << 16);
    }
    __device__ static Vec16 with_neg_inf(Vec16 v, uint32_t e)
    {
        const uint32_t mask = e % 2u ? 0xFFFF0000u : 0xFFFFu;
        v.w[e / 2u] = (v.w[e / 2u] & ~mask) | (kNegInf & mask);
        return v;
    }
    __device__ static float one(Word x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
    __device__ static Word word(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }   // to nearest, ties to even
    __device__ static Vec16 pack(const float (&f)[kPerVec])
    {
        Vec16 v;
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) v.w[i] = (uint32_t)word(f[2u * i]) | (uint32_t)word(f[2u * i + 1u]) << 16;
        return v;
    }
};
template <> struct Elem<kHeadF16> {
    static constexpr uint32_t kBytes = 2u, kPerVec = 8u;
    static constexpr uint32_t kNegInf = 0xFC00FC00u;
    static constexpr uint32_t kZeroBits = 13u;
    struct __attribute__((packed, aligned(2))) Run { uint32_t w[4]; };
    typedef uint32_t Packed __attribute__((ext_vector_type(4), aligned(2)));
    using Word = uint16_t;
    __device__ static float get(const Vec16& v, uint32_t e)
    {
        return one((uint16_t)(v.w[e / 2u] >> (16u * (e % 2u))));
    }
    __device__ static Vec16 with_neg_inf(Vec16 v, uint32_t e)
    {
        const uint32_t mask = e % 2u ? 0xFFFF0000u : 0xFFFFu;
        v.w[e / 2u] = (v.w[e / 2u] & ~mask) | (kNegInf & mask);
        return v;
    }
    __device__ static float one(Word x) { return (float)__builtin_bit_cast(_Float16, x); }
    __device__ static Word word(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }  // to nearest, ties to even
    __device__ static Vec16 pack(const float (&f)[kPerVec])
    {
        Vec16 v;
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) v.w[i] = (uint32_t)word(f[2u * i]) | (uint32_t)word(f[2u * i + 1u]) << 16;
        return v;
    }
};

// One entry of an array of any of the three types.
__device__ __forceinline__ float load_any(const void* p, uint64_t i, int dtype)
{
    if (dtype == kHeadF32) return static_cast<const float*>(p)[i];
    const uint16_t x = static_cast<const uint16_t*>(p)[i];
    return dtype == kHeadBF16 ? Elem<kHeadBF16>::one(x) : Elem<kHeadF16>::one(x);
}

// ---------------------------------------------------------------------------
// Waves.  Lane 63 ends up with the whole wave's value after the shifts by 1, 2, 4
// and 8 within rows of 16 lanes and the two broadcasts of a row's last lane into
// the next rows.  Every lane of the wave has to be active.
// ---------------------------------------------------------------------------
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t old, uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_f32(float old, float x)
{
    return __builtin_bit_cast(float, dpp_u32<CTRL, ROWS>(__builtin_bit_cast(uint32_t, old), __builtin_bit_cast(uint32_t, x)));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp_u64(uint64_t x)       // 0 where no lane feeds
{
    return (uint64_t)dpp_u32<CTRL, ROWS>(0u, (uint32_t)(x >> 32)) << 32 | dpp_u32<CTRL, ROWS>(0u, (uint32_t)x);
}
__device__ __forceinline__ float last_lane(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ uint64_t lane_u64(uint64_t x, int lane)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32
           | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
}

__device__ __forceinline__ float wave_max(float x)
{
    const float lo = -__builtin_inff();
    x = __builtin_fmaxf(x, dpp_f32<0x111, 0xf>(lo, x));
    x = __builtin_fmaxf(x, dpp_f32<0x112, 0xf>(lo, x));
    x = __builtin_fmaxf(x, dpp_f32<0x114, 0xf>(lo, x));
    x = __builtin_fmaxf(x, dpp_f32<0x118, 0xf>(lo, x));
    x = __builtin_fmaxf(x, dpp_f32<0x142, 0xa>(lo, x));
    x = __builtin_fmaxf(x, dpp_f32<0x143, 0xc>(lo, x));
    return last_lane(x);
}
__device__ __forceinline__ double wave_total(double x)
{
    auto add = [&](uint64_t y) { x += __builtin_bit_cast(double, y); };
    add(dpp_u64<0x111, 0xf>(__builtin_bit_cast(uint64_t, x)));
    add(dpp_u64<0x112, 0xf>(__builtin_bit_cast(uint64_t, x)));
    add(dpp_u64<0x114, 0xf>(__builtin_bit_cast(uint64_t, x)));
    add(dpp_u64<0x118, 0xf>(__builtin_bit_cast(uint64_t, x)));
    add(dpp_u64<0x142, 0xa>(__builtin_bit_cast(uint64_t, x)));
    add(dpp_u64<0x143, 0xc>(__builtin_bit_cast(uint64_t, x)));
    return __builtin_bit_cast(double, lane_u64(__builtin_bit_cast(uint64_t, x), 63));
}
// Running sum over the lanes, this lane's own included.
__device__ __forceinline__ uint64_t wave_scan(uint64_t x)
{
    x += dpp_u64<0x111, 0xf>(x);
    x += dpp_u64<0x112, 0xf>(x);
    x += dpp_u64<0x114, 0xf>(x);
    x += dpp_u64<0x118, 0xf>(x);
    x += dpp_u64<0x142, 0xa>(x);
    x += dpp_u64<0x143, 0xc>(x);
    return x;
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x)
{
    x += dpp_u32<0x111, 0xf>(0u, x);
    x += dpp_u32<0x112, 0xf>(0u, x);
    x += dpp_u32<0x114, 0xf>(0u, x);
    x += dpp_u32<0x118, 0xf>(0u, x);
    x += dpp_u32<0x142, 0xa>(0u, x);
    x += dpp_u32<0x143, 0xc>(0u, x);
    return x;
}
__device__ __forceinline__ uint64_t wave_total(uint64_t x) { return lane_u64(wave_scan(x), 63); }

__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
    x = max(x, dpp_u32<0x111, 0xf>(0u, x));
    x = max(x, dpp_u32<0x112, 0xf>(0u, x));
    x = max(x, dpp_u32<0x114, 0xf>(0u, x));
    x = max(x, dpp_u32<0x118, 0xf>(0u, x));
    x = max(x, dpp_u32<0x142, 0xa>(0u, x));
    x = max(x, dpp_u32<0x143, 0xc>(0u, x));
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// A wave-uniform value in a scalar register.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
__device__ __forceinline__ float uniform(float x)
{
    return __builtin_bit_cast(float, uniform(__builtin_bit_cast(uint32_t, x)));
}
__device__ __forceinline__ uint64_t uniform(uint64_t x);
__device__ __forceinline__ double uniform(double x)
{
    return __builtin_bit_cast(double, uniform(__builtin_bit_cast(uint64_t, x)));
}
__device__ __forceinline__ uint64_t uniform(uint64_t x)
{
    return (uint64_t)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x);
}

// The largest value over a workgroup of NW waves, in every thread and wave-uniform; `sh`
// holds NW values that no thread still reads from an earlier use.
template <int NW>
__device__ __forceinline__ float group_max(float x, float* sh)
{
    x = wave_max(x);
    if (NW == 1) return x;
    const uint32_t lane = threadIdx.x % 64u;
    if (lane == 0u) sh[threadIdx.x / 64u] = x;
    __syncthreads();
    return wave_max(lane < (uint32_t)NW ? sh[lane] : -__builtin_inff());
}
// ---------------------------------------------------------------------------
// A row (V entries of it, `from` entries behind its start) as a workgroup of NT threads sees it: whole 16-byte vectors, then up to
// kPerVec - 1 entries of tail, one to a lane of the first wave.  A wave owns `seg`
// consecutive strips of 64 vectors, so that index order is (wave, strip, lane,
// entry).  NV > 0: up to NV strips a wave, held in registers from one read of the
// row; NV = 0: every pass reads the row again.  Rows need only their element's
// alignment (global memory takes 16-byte accesses at any address).
// Vectors and tail lanes past the row's end hold -inf.
// ---------------------------------------------------------------------------
template <int D, int NT, int NV>
struct Row {
    using El = Elem<D>;
    static constexpr uint32_t E = El::kPerVec;
    static constexpr uint32_t NW = NT / 64;
    const char* p;
    uint32_t vectors, tail, seg, wave, lane;
    Vec16 reg[NV ? NV : 1];
    float last;                                   // this lane's entry of the tail (first wave)

    __device__ __forceinline__ void open(const void* logits, uint64_t row, uint64_t stride, uint32_t V, uint32_t from = 0u)
    {
        p = static_cast<const char*>(logits) + (row * stride + from) * El::kBytes;
        vectors = V / E;
        tail = V % E;
        seg = (vectors + 64u * NW - 1u) / (64u * NW);
        wave = uniform(threadIdx.x / 64u);
        lane = threadIdx.x % 64u;
        if (NV) {
#pragma unroll
            for (uint32_t v = 0; v < (uint32_t)NV; ++v) reg[v] = load(v);
        }
        last = -__builtin_inff();
        if (lane < tail) last = entry(vectors * E + lane);
    }
    __device__ __forceinline__ float entry(uint32_t i) const
    {
        return El::one(reinterpret_cast<const typename El::Word*>(p)[i]);
    }
    __device__ __forceinline__ Vec16 vector(uint32_t i) const          // i < vectors
    {
        const typename El::Run r = reinterpret_cast<const typename El::Run*>(p)[i];
        return Vec16{{r.w[0], r.w[1], r.w[2], r.w[3]}};
    }
    // whether strip v of this wave holds any vector (wave-uniform), and this lane's
    // vector of it
    __device__ __forceinline__ bool any(uint32_t v) const { return v < seg && (wave * seg + v) * 64u < vectors; }
    __device__ __forceinline__ uint32_t index(uint32_t v) const { return (wave * seg + v) * 64u + lane; }
    __device__ __forceinline__ Vec16 load(uint32_t v) const
    {
        Vec16 x{{El::kNegInf, El::kNegInf, El::kNegInf, El::kNegInf}};
        if (any(v) && index(v) < vectors) x = vector(index(v));
        return x;
    }
    // f(vector, number of the vector) for each vector of this lane; U strips are loaded
    // before the first of them is used
    template <int U, class F>
    __device__ __forceinline__ void stream(F f) const
    {
#pragma unroll 1
        for (uint32_t v = 0; v < seg && any(v); v += (uint32_t)U) {
            Vec16 y[U];
#pragma unroll
            for (uint32_t j = 0; j < (uint32_t)U; ++j) y[j] = load(v + j);
#pragma unroll
            for (uint32_t j = 0; j < (uint32_t)U; ++j)
                if (any(v + j)) f(y[j], index(v + j));
        }
    }
    template <class F>
    __device__ __forceinline__ void each_vector(F f) const
    {
        if (NV) {
#pragma unroll
            for (uint32_t v = 0; v < (uint32_t)NV; ++v)
                if (any(v)) f(reg[v], index(v));
        } else {
            stream<4>(f);
        }
    }
    // f(entry, its index) for each entry of this lane's vectors
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
        each_vector([&](const Vec16& x, uint32_t i) {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) f(El::get(x, e), i * E + e);
        });
    }
    // the same, and for the tail
    template <class F>
    __device__ __forceinline__ void each_and_tail(F f) const
    {
        each(f);
        if (wave == 0u) f(last, vectors * E + lane);
    }
    // both again, from one more read of the row: small code for passes that few rows need
    template <class F>
    __device__ __forceinline__ void each_again_vectors(F f) const
    {
        stream<1>([&](const Vec16& y, uint32_t i) {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) f(El::get(y, e), i * E + e);
        });
    }
    template <class F>
    __device__ __forceinline__ void each_again(F f) const
    {
        each_again_vectors(f);
        if (wave == 0u) f(last, vectors * E + lane);
    }
    __device__ __forceinline__ float max() const
    {
        float m = -__builtin_inff();
        each([&](float l, uint32_t) { m = __builtin_fmaxf(m, l); });
        return __builtin_fmaxf(m, last);
    }
};

}  // namespace rlsim_dev
