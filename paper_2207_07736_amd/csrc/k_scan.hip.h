// k_scan.hip.h -- the gated recurrence over rows in time and its backward pass.
//
//   a_t = sigmoid(gate_t), h_t = a_t h'_{t-1} + (1 - a_t) x_t, h'_t = done_t ? 0 : h_t
//
// A step is an affine map of the state, so a stretch of steps is one too (two numbers a
// channel), but for the end of an episode, which takes 0 in place of the state whatever the
// state is: a product of 0 would hand on a NaN or an infinity as a NaN.  A map that holds an
// end says so, and its sum is taken as it is.  Where there are channels enough, a thread goes through all steps of its two
// channels; where there are not, time is cut into segments: one launch finds each
// segment's map, the next joins them to the state each segment starts from, and the third
// goes through the rows.  Backward is the same from the end.  No result depends on how the
// workgroups are placed or timed.
//
// What bounds it, where there is enough of it, is memory: two channels a thread, 16 steps'
// loads under way before the first is used.  200 x 4,096 x 64 fp32: forward 133 us = 4.8 TB/s,
// backward 211 us = 5.0 TB/s (a large copy: 4.9).  65,536 x 2,048 bf16, cut: maps 133 and 136 us
// = 4.0 TB/s, rows 166 us = 5.1 and 313 us = 4.3; reading the rows twice is the price of the
// cut.  Small calls are bound by a run's chain and, where cut, by three launches.  With a few
// waves to a CU the loads of a run wait for the run before it: 1,000 x 2,048 x 64 in bf16
// 278 us forward and 408 backward for floors of 161 and 268.  Backward in fp16 is slower yet
// (1,083 us there) and keeps some registers in scratch memory; without that it takes 847.
#pragma once

#include <type_traits>

#include "head_common.hip.h"
#include "learn_dispatch.h"

namespace rlsim_dev {

struct ScanArgs {
    const char* x;
    const char* gate;
    const char* dy;              // backward, or null
    char* y;                     // forward: y; backward: dx
    char* dgate;
    uint64_t x_step, x_seq, gate_step, gate_seq, dy_step, dy_seq, y_step, y_seq, dgate_step, dgate_seq;   // bytes
    const float* state;          // forward: state; backward: dlast; or null
    const uint8_t* done;
    float* marks;
    float* last;                 // forward: last; backward: dstate; or null
    float* map_a;                // [segments][n channels]: a segment's map, product (or kScanReset)
    float* map_b;                // and sum; once joined, the state that the segment starts from
    uint32_t T, n, channels, groups, segments, seg_len;
    uint32_t backward;
};

// sigmoid(g) and 1 - sigmoid(g): the smaller of the two is never a difference.  Each is within
// (2 |g| + 8) 2^-24 of itself: exp2's argument is |g| log2(e) in 24 bits, so the smaller one
// loses digits as it gets small.  The reciprocal is the hardware's with one Newton step.
struct Gate { float a, take; };
__device__ __forceinline__ Gate gate_of(float g)
{
    const float E = __builtin_amdgcn_exp2f(-__builtin_fabsf(g) * 1.4426950408889634f);
    const float d = 1.0f + E;
    float r = __builtin_amdgcn_rcpf(d);
    r = __builtin_fmaf(r, __builtin_fmaf(-d, r, 1.0f), r);
    const float s = E * r;
    return g >= 0.0f ? Gate{r, s} : Gate{s, r};
}

// A map's product: of gates, kScanTiny at least while none of them is 0; kScanReset where an
// episode ends within the map.
constexpr float kScanReset = -1.0f, kScanTiny = 0x1p-149f;
__device__ __forceinline__ float scan_product(float p, float q)
{
    return __builtin_fmaxf(p * q, __builtin_fminf(__builtin_fminf(p, q), kScanTiny));
}
// What a map makes of the state h, and of a map before it.  An infinite state stays one however
// far it is carried; of a finite one the tiny product leaves nothing.
__device__ __forceinline__ float scan_through(float p, float q, float h)
{
    const float carried = __builtin_fmaf(p == kScanTiny ? 0.0f : p, h, q);
    const float kept = __builtin_fabsf(h) == __builtin_inff() && p > 0.0f ? h + q : carried;
    return p < 0.0f ? q : kept;
}
__device__ __forceinline__ float scan_joined(float p, float after)
{
    const float least = __builtin_fminf(p, after);
    return least < 0.0f ? least : scan_product(p, after);
}

// V consecutive elements as loaded, turned to floats when used.
template <int D, int V>
struct Channels {
    using El = Elem<D>;
    using Word = typename El::Word;
    static constexpr uint32_t kWords = (El::kBytes * V + 3u) / 4u;
    struct __attribute__((packed, aligned(El::kBytes))) Run { Word w[V]; };
    Run r;
    __device__ __forceinline__ void load(const char* p) { r = *reinterpret_cast<const Run*>(p); }
    __device__ __forceinline__ float get(int i) const { return El::one(r.w[i]); }
    __device__ __forceinline__ static void store(char* p, const float (&f)[V], uint32_t from)
    {
        Run o;
#pragma unroll
        for (int i = 0; i < V; ++i) o.w[i] = El::word(f[i]);
        if (from == 0u) {
            *reinterpret_cast<Run*>(p) = o;
        } else {
#pragma unroll
            for (int i = 1; i < V; ++i)
                if ((uint32_t)i >= from) reinterpret_cast<Word*>(p)[i] = o.w[i];
        }
    }
};

// Which channels of which sequence a thread has.  The last group of a row of channels that
// V does not divide reaches back over the group before it (loads stay vectors inside the
// row) and stores only what is its own, from `from` on.
template <int V>
struct Lane {
    uint32_t seq, c, from;
    uint64_t flat;               // of [n][channels]
    __device__ __forceinline__ Lane(const ScanArgs& a, uint64_t q)
    {
        uint32_t group;
        if (q < 0x100000000ull) {
            seq = (uint32_t)q / a.groups;
            group = (uint32_t)q % a.groups;
        } else {
            seq = (uint32_t)(q / a.groups);
            group = (uint32_t)(q % a.groups);
        }
        c = group * V;
        from = 0u;
        if (c + V > a.channels) {
            from = c + V - a.channels;
            c -= from;
        }
        flat = (uint64_t)seq * a.channels + c;
    }
    __device__ __forceinline__ void put(float* p, const float (&f)[V]) const
    {
        Channels<kHeadF32, V>::store(reinterpret_cast<char*>(p + flat), f, from);
    }
    __device__ __forceinline__ void get(const float* p, float (&f)[V]) const
    {
        Channels<kHeadF32, V> r;
        r.load(reinterpret_cast<const char*>(p + flat));
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = r.get(i);
    }
};

// The lane's offset in an array's row of one step: 32 bits, so that a step's address is one
// uniform number and this, unless sequences lie further apart (WIDE).
template <bool WIDE, int D, int V>
__device__ __forceinline__ auto lane_offset(const Lane<V>& l, uint64_t seq_bytes)
{
    using Off = std::conditional_t<WIDE, uint64_t, uint32_t>;
    return (Off)(l.seq * (Off)seq_bytes + (Off)l.c * Elem<D>::kBytes);
}

// The bits of U steps' done flags, from step t on (t1: the end).
template <uint32_t U>
__device__ __forceinline__ uint32_t ends_of(const ScanArgs& a, uint32_t t, uint32_t t1, uint32_t seq)
{
    uint32_t ends = 0u;
    if (a.done) {
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint8_t* row = a.done + (uint64_t)min(t + u, t1 - 1u) * a.n;
            ends |= (row[seq] ? 1u : 0u) << u;
        }
    }
    return ends;
}

// Steps [t0, t1) forward for one thread, U at a time: the loads of a run are made before
// its first step.  ROWS: y and the marks are written; else only the map is kept, and whether an
// episode ends in it returned.
template <int D, int V, uint32_t U, bool WIDE, bool ROWS>
__device__ __forceinline__ bool scan_forward(const ScanArgs& a, const Lane<V>& l, uint32_t t0, uint32_t t1, float (&h)[V],
                                             float (&prod)[V])
{
    uint32_t reset = 0u;
    const auto ox = lane_offset<WIDE, D, V>(l, a.x_seq), og = lane_offset<WIDE, D, V>(l, a.gate_seq),
               oy = lane_offset<WIDE, D, V>(l, a.y_seq);
    for (uint32_t t = t0; t < t1; t += U) {
        Channels<D, V> x[U], g[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint64_t at = min(t + u, t1 - 1u);
            x[u].load(a.x + at * a.x_step + ox);
            g[u].load(a.gate + at * a.gate_step + og);
        }
        const uint32_t ends = ends_of<U>(a, t, t1, l.seq);
        if (!ROWS) reset |= ends;
        if (ROWS && a.marks && (U == kScanMark || t % kScanMark == 0u)) l.put(a.marks + (uint64_t)(t / kScanMark) * a.n * a.channels, h);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            if (t + u < t1) {
                float out[V];
                const bool end = ends >> u & 1u;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const Gate k = gate_of(g[u].get(i));
                    h[i] = __builtin_fmaf(k.a, h[i], k.take * x[u].get(i));
                    out[i] = h[i];
                    if (end) h[i] = 0.0f;
                    if (!ROWS) prod[i] = scan_product(prod[i], k.a);
                }
                if (ROWS) Channels<D, V>::store(a.y + (uint64_t)(t + u) * a.y_step + oy, out, l.from);
            }
        }
    }
    return reset != 0u;
}

template <int D, int V, bool WIDE>
__global__ __launch_bounds__(256) void k_scan_maps(ScanArgs a)
{
    const uint64_t all = (uint64_t)a.n * a.groups, stride = (uint64_t)gridDim.x * 256u;
    const uint32_t s = blockIdx.y, t0 = s * a.seg_len, t1 = min(t0 + a.seg_len, a.T);
    for (uint64_t q = (uint64_t)blockIdx.x * 256u + threadIdx.x; q < all; q += stride) {
        const Lane<V> l(a, q);
        float h[V], prod[V];
#pragma unroll
        for (int i = 0; i < V; ++i) { h[i] = 0.0f; prod[i] = 1.0f; }
        if (scan_forward<D, V, kScanMark, WIDE, false>(a, l, t0, t1, h, prod)) {
#pragma unroll
            for (int i = 0; i < V; ++i) prod[i] = kScanReset;
        }
        const uint64_t at = (uint64_t)s * a.n * a.channels;
        l.put(a.map_a + at, prod);
        l.put(a.map_b + at, h);
    }
}

// Segments' maps to the states they start from.  A workgroup has 16 channels; each of its 16
// rows of threads joins a run of segments, the runs meet in LDS, and each row goes through
// its run again from there.  Backward, segment 0 is the last.
__global__ __launch_bounds__(256) void k_scan_join(ScanArgs a)
{
    __shared__ float sa[16][16], sb[16][16];
    const uint64_t C = (uint64_t)a.n * a.channels;
    const uint32_t x = threadIdx.x % 16u, y = threadIdx.x / 16u;
    const uint64_t c = (uint64_t)blockIdx.x * 16u + x;
    const uint32_t run = (a.segments + 15u) / 16u, j0 = min(y * run, a.segments), j1 = min(j0 + run, a.segments);
    auto at = [&](uint32_t j) { return (uint64_t)(a.backward ? a.segments - 1u - j : j) * C + c; };
    // a few maps' loads at a time, before the first is used
    constexpr uint32_t U = 4u;
    auto each = [&](auto f) {
        for (uint32_t j = j0; j < j1; j += U) {
            float p[U], q[U];
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                const uint64_t k = at(min(j + u, j1 - 1u));
                p[u] = a.map_a[k];
                q[u] = a.map_b[k];
            }
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                const bool in = j + u < j1;       // else the map that changes nothing
                f(j + u, in ? p[u] : 1.0f, in ? q[u] : 0.0f);
            }
        }
    };
    float A = 1.0f, B = 0.0f;
    if (c < C) {
        each([&](uint32_t, float p, float q) {
            B = scan_through(p, q, B);
            A = scan_joined(A, p);
        });
    }
    sa[y][x] = A;
    sb[y][x] = B;
    __syncthreads();
    if (c >= C) return;
    float h = a.state ? a.state[c] : 0.0f;
    for (uint32_t k = 0; k < y; ++k) h = scan_through(sa[k][x], sb[k][x], h);
    each([&](uint32_t j, float p, float q) {
        if (j < j1) a.map_b[at(j)] = h;
        h = scan_through(p, q, h);
    });
}

// What a thread's segment starts from.
template <int V>
__device__ __forceinline__ void scan_start(const ScanArgs& a, const Lane<V>& l, uint32_t s, float (&h)[V])
{
    if (a.segments > 1u) {
        l.get(a.map_b + (uint64_t)s * a.n * a.channels, h);
    } else if (a.state) {
        l.get(a.state, h);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = 0.0f;
    }
}

template <int D, int V, uint32_t U, bool WIDE>
__global__ __launch_bounds__(256) void k_scan_rows(ScanArgs a)
{
    const uint64_t all = (uint64_t)a.n * a.groups, stride = (uint64_t)gridDim.x * 256u;
    const uint32_t s = blockIdx.y, t0 = s * a.seg_len, t1 = min(t0 + a.seg_len, a.T);
    for (uint64_t q = (uint64_t)blockIdx.x * 256u + threadIdx.x; q < all; q += stride) {
        const Lane<V> l(a, q);
        float h[V], unused[V];
        scan_start(a, l, s, h);
        scan_forward<D, V, U, WIDE, true>(a, l, t0, t1, h, unused);
        if (a.last && t1 == a.T) l.put(a.last, h);
    }
}

// Backward.  `R` is a_{t+1} e_{t+1} when step t is reached from the end.
template <int D, int V, bool WIDE>
__global__ __launch_bounds__(256) void k_scan_back_maps(ScanArgs a)
{
    constexpr uint32_t U = kScanMark;
    const uint64_t all = (uint64_t)a.n * a.groups, stride = (uint64_t)gridDim.x * 256u;
    const uint32_t s = blockIdx.y, t0 = s * a.seg_len, t1 = min(t0 + a.seg_len, a.T);
    const uint64_t C = (uint64_t)a.n * a.channels;
    for (uint64_t q = (uint64_t)blockIdx.x * 256u + threadIdx.x; q < all; q += stride) {
        const Lane<V> l(a, q);
        const auto og = lane_offset<WIDE, D, V>(l, a.gate_seq), od = lane_offset<WIDE, D, V>(l, a.dy_seq);
        float P[V], Q[V];
        uint32_t reset = 0u;
#pragma unroll
        for (int i = 0; i < V; ++i) { P[i] = 1.0f; Q[i] = 0.0f; }
        for (uint32_t left = t1 - t0; left != 0u;) {
            const uint32_t run = left % U ? left % U : U, t = t0 + left - run;
            Channels<D, V> g[U], d[U];
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                const uint64_t at = t + min(u, run - 1u);
                g[u].load(a.gate + at * a.gate_step + og);
                if (a.dy) d[u].load(a.dy + at * a.dy_step + od);
            }
            const uint32_t ends = ends_of<U>(a, t, t + run, l.seq);
            reset |= ends;
#pragma unroll
            for (uint32_t k = 0; k < U; ++k) {
                const uint32_t u = U - 1u - k;
                if (u < run) {
                    const bool end = ends >> u & 1u;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const Gate w = gate_of(g[u].get(i));
                        const float e = (a.dy ? d[u].get(i) : 0.0f) + (end ? 0.0f : Q[i]);
                        P[i] = scan_product(P[i], w.a);
                        Q[i] = w.a * e;
                    }
                }
            }
            left -= run;
        }
        if (reset) {
#pragma unroll
            for (int i = 0; i < V; ++i) P[i] = kScanReset;
        }
        l.put(a.map_a + s * C, P);
        l.put(a.map_b + s * C, Q);
    }
}

// A run of steps behind a mark goes forward first: the states between, of which only
// h'_{t-1} - x_t is kept, with both gates, so that these are found once.
template <int D, int V, bool WIDE>
__global__ __launch_bounds__(256, D == kHeadF32 ? 2 : 3) void k_scan_back_rows(ScanArgs a)
{
    constexpr uint32_t U = kScanMark;
    const uint64_t all = (uint64_t)a.n * a.groups, stride = (uint64_t)gridDim.x * 256u;
    const uint32_t s = blockIdx.y, t0 = s * a.seg_len, t1 = min(t0 + a.seg_len, a.T);
    const uint64_t C = (uint64_t)a.n * a.channels;
    for (uint64_t q = (uint64_t)blockIdx.x * 256u + threadIdx.x; q < all; q += stride) {
        const Lane<V> l(a, q);
        const auto ox = lane_offset<WIDE, D, V>(l, a.x_seq), og = lane_offset<WIDE, D, V>(l, a.gate_seq),
                   od = lane_offset<WIDE, D, V>(l, a.dy_seq), odx = lane_offset<WIDE, D, V>(l, a.y_seq),
                   odg = lane_offset<WIDE, D, V>(l, a.dgate_seq);
        float R[V];
        scan_start(a, l, s, R);
        // segments start at marks, so a run is what lies behind one mark
        for (uint32_t left = t1 - t0; left != 0u;) {
            const uint32_t run = left % U ? left % U : U, t = t0 + left - run;
            Channels<D, V> x[U], g[U], d[U];
            float m[V], diff[U][V];
            Gate w[U][V];
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                const uint64_t at = t + min(u, run - 1u);
                x[u].load(a.x + at * a.x_step + ox);
                g[u].load(a.gate + at * a.gate_step + og);
                if (a.dy) d[u].load(a.dy + at * a.dy_step + od);
            }
            const uint32_t ends = ends_of<U>(a, t, t + run, l.seq);
            l.get(a.marks + (uint64_t)(t / U) * C, m);
#pragma unroll
            for (uint32_t u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float in = x[u].get(i);
                    w[u][i] = gate_of(g[u].get(i));
                    diff[u][i] = m[i] - in;
                    m[i] = ends >> u & 1u ? 0.0f : __builtin_fmaf(w[u][i].a, m[i], w[u][i].take * in);
                }
#pragma unroll
            for (uint32_t k = 0; k < U; ++k) {
                const uint32_t u = U - 1u - k;
                if (u < run) {
                    float dx[V], dg[V];
                    const bool end = ends >> u & 1u;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float e = (a.dy ? d[u].get(i) : 0.0f) + (end ? 0.0f : R[i]);
                        dx[i] = w[u][i].take * e;
                        dg[i] = w[u][i].a * dx[i] * diff[u][i];
                        R[i] = w[u][i].a * e;
                    }
                    Channels<D, V>::store(a.y + (uint64_t)(t + u) * a.y_step + odx, dx, l.from);
                    Channels<D, V>::store(a.dgate + (uint64_t)(t + u) * a.dgate_step + odg, dg, l.from);
                }
            }
            left -= run;
        }
        if (a.last && s == 0u) l.put(a.last, R);
    }
}

}  // namespace rlsim_dev
