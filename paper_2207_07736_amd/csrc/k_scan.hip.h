// k_scan.hip.h -- the gated recurrence over rows in time and its backward pass.
//
//   a_t = sigmoid(gate_t), h_t = a_t h'_{t-1} + (1 - a_t) x_t, h'_t = done_t ? 0 : h_t
//
// A step is an affine map of the state, so a stretch of steps is one too (two numbers a
// channel).  Where there are channels enough, a thread goes through all steps of its few
// channels; where there are not, time is cut into segments: one launch finds each
// segment's map, the next joins the maps in front of a segment to its first state and goes
// through its rows.  Backward is the same from the end.  No result depends on how the
// workgroups are placed or timed.
#pragma once

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
    float* map_a;                // [segments][n channels]: a segment's map, product and
    float* map_b;                // sum
    uint32_t T, n, channels, groups, segments, seg_len;
};

// sigmoid(g) and 1 - sigmoid(g), each to a few units of the last place: the smaller of the
// two is never a difference.  The reciprocal is the hardware's with one Newton step.
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
#pragma unroll
        for (int i = 0; i < V; ++i)
            if ((uint32_t)i >= from) p[flat + i] = f[i];
    }
};

// Steps [t0, t1) forward for one thread, kScanMark at a time: the loads of a run are made
// before its first step.  ROWS: y and the marks are written; else only the map is kept.
template <int D, int V, bool ROWS>
__device__ __forceinline__ void scan_forward(const ScanArgs& a, const Lane<V>& l, uint32_t t0, uint32_t t1, float (&h)[V],
                                             float (&prod)[V])
{
    constexpr uint32_t U = kScanMark;
    const char* px = a.x + l.seq * a.x_seq + (uint64_t)l.c * Elem<D>::kBytes;
    const char* pg = a.gate + l.seq * a.gate_seq + (uint64_t)l.c * Elem<D>::kBytes;
    char* py = a.y + l.seq * a.y_seq + (uint64_t)l.c * Elem<D>::kBytes;
    for (uint32_t t = t0; t < t1; t += U) {
        Channels<D, V> x[U], g[U];
        uint32_t ends = 0u;
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint64_t at = min(t + u, t1 - 1u);
            x[u].load(px + at * a.x_step);
            g[u].load(pg + at * a.gate_step);
        }
        if (a.done) {
#pragma unroll
            for (uint32_t u = 0; u < U; ++u)
                ends |= (a.done[(uint64_t)min(t + u, t1 - 1u) * a.n + l.seq] ? 1u : 0u) << u;
        }
        if (ROWS && a.marks) l.put(a.marks + (uint64_t)(t / U) * a.n * a.channels, h);
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
                    if (!ROWS) prod[i] = end ? 0.0f : prod[i] * k.a;
                }
                if (ROWS) Channels<D, V>::store(py + (uint64_t)(t + u) * a.y_step, out, l.from);
            }
        }
    }
}

template <int D, int V>
__global__ __launch_bounds__(256) void k_scan_maps(ScanArgs a)
{
    const uint64_t all = (uint64_t)a.n * a.groups, stride = (uint64_t)gridDim.x * 256u;
    const uint32_t s = blockIdx.y, t0 = s * a.seg_len, t1 = min(t0 + a.seg_len, a.T);
    for (uint64_t q = (uint64_t)blockIdx.x * 256u + threadIdx.x; q < all; q += stride) {
        const Lane<V> l(a, q);
        float h[V], prod[V];
#pragma unroll
        for (int i = 0; i < V; ++i) { h[i] = 0.0f; prod[i] = 1.0f; }
        scan_forward<D, V, false>(a, l, t0, t1, h, prod);
        const uint64_t at = (uint64_t)s * a.n * a.channels;
        l.put(a.map_a + at, prod);
        l.put(a.map_b + at, h);
    }
}

template <int D, int V>
__global__ __launch_bounds__(256) void k_scan_rows(ScanArgs a)
{
    const uint64_t all = (uint64_t)a.n * a.groups, stride = (uint64_t)gridDim.x * 256u;
    const uint32_t s = blockIdx.y, t0 = s * a.seg_len, t1 = min(t0 + a.seg_len, a.T);
    const uint64_t C = (uint64_t)a.n * a.channels;
    for (uint64_t q = (uint64_t)blockIdx.x * 256u + threadIdx.x; q < all; q += stride) {
        const Lane<V> l(a, q);
        float h[V], unused[V];
#pragma unroll
        for (int i = 0; i < V; ++i) { h[i] = a.state ? a.state[l.flat + i] : 0.0f; unused[i] = 0.0f; }
#pragma unroll 8
        for (uint32_t j = 0; j < s; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) h[i] = __builtin_fmaf(a.map_a[j * C + l.flat + i], h[i], a.map_b[j * C + l.flat + i]);
        scan_forward<D, V, true>(a, l, t0, t1, h, unused);
        if (a.last && t1 == a.T) l.put(a.last, h);
    }
}

// Backward.  `R` is a_{t+1} e_{t+1} when step t is reached from the end.
template <int D, int V>
__global__ __launch_bounds__(256) void k_scan_back_maps(ScanArgs a)
{
    constexpr uint32_t U = kScanMark;
    const uint64_t all = (uint64_t)a.n * a.groups, stride = (uint64_t)gridDim.x * 256u;
    const uint32_t s = blockIdx.y, t0 = s * a.seg_len, t1 = min(t0 + a.seg_len, a.T);
    const uint64_t C = (uint64_t)a.n * a.channels;
    for (uint64_t q = (uint64_t)blockIdx.x * 256u + threadIdx.x; q < all; q += stride) {
        const Lane<V> l(a, q);
        const char* pg = a.gate + l.seq * a.gate_seq + (uint64_t)l.c * Elem<D>::kBytes;
        const char* pd = a.dy + l.seq * a.dy_seq + (uint64_t)l.c * Elem<D>::kBytes;
        float P[V], Q[V];
#pragma unroll
        for (int i = 0; i < V; ++i) { P[i] = 1.0f; Q[i] = 0.0f; }
        for (uint32_t left = t1 - t0; left != 0u;) {
            const uint32_t run = left % U ? left % U : U, t = t0 + left - run;
            Channels<D, V> g[U], d[U];
            uint32_t ends = 0u;
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                const uint64_t at = t + min(u, run - 1u);
                g[u].load(pg + at * a.gate_step);
                if (a.dy) d[u].load(pd + at * a.dy_step);
                if (a.done) ends |= (a.done[at * a.n + l.seq] ? 1u : 0u) << u;
            }
#pragma unroll
            for (uint32_t k = 0; k < U; ++k) {
                const uint32_t u = U - 1u - k;
                if (u < run) {
                    const bool end = ends >> u & 1u;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const Gate w = gate_of(g[u].get(i));
                        const float e = (a.dy ? d[u].get(i) : 0.0f) + (end ? 0.0f : Q[i]);
                        P[i] = end ? 0.0f : P[i] * w.a;
                        Q[i] = w.a * e;
                    }
                }
            }
            left -= run;
        }
        l.put(a.map_a + s * C, P);
        l.put(a.map_b + s * C, Q);
    }
}

template <int D, int V>
__global__ __launch_bounds__(256) void k_scan_back_rows(ScanArgs a)
{
    constexpr uint32_t U = kScanMark;
    const uint64_t all = (uint64_t)a.n * a.groups, stride = (uint64_t)gridDim.x * 256u;
    const uint32_t s = blockIdx.y, t0 = s * a.seg_len, t1 = min(t0 + a.seg_len, a.T);
    const uint64_t C = (uint64_t)a.n * a.channels;
    for (uint64_t q = (uint64_t)blockIdx.x * 256u + threadIdx.x; q < all; q += stride) {
        const Lane<V> l(a, q);
        const char* px = a.x + l.seq * a.x_seq + (uint64_t)l.c * Elem<D>::kBytes;
        const char* pg = a.gate + l.seq * a.gate_seq + (uint64_t)l.c * Elem<D>::kBytes;
        const char* pd = a.dy + l.seq * a.dy_seq + (uint64_t)l.c * Elem<D>::kBytes;
        char* qx = a.y + l.seq * a.y_seq + (uint64_t)l.c * Elem<D>::kBytes;
        char* qg = a.dgate + l.seq * a.dgate_seq + (uint64_t)l.c * Elem<D>::kBytes;
        float R[V];
#pragma unroll
        for (int i = 0; i < V; ++i) R[i] = a.state ? a.state[l.flat + i] : 0.0f;
#pragma unroll 8
        for (uint32_t j = a.segments - 1u; j > s; --j)
#pragma unroll
            for (int i = 0; i < V; ++i) R[i] = __builtin_fmaf(a.map_a[j * C + l.flat + i], R[i], a.map_b[j * C + l.flat + i]);
        // segments start at marks, so a run is what lies behind one mark
        for (uint32_t left = t1 - t0; left != 0u;) {
            const uint32_t run = left % U ? left % U : U, t = t0 + left - run;
            Channels<D, V> x[U], g[U], d[U];
            uint32_t ends = 0u;
            float h[U][V], m[V];
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) {
                const uint64_t at = t + min(u, run - 1u);
                x[u].load(px + at * a.x_step);
                g[u].load(pg + at * a.gate_step);
                if (a.dy) d[u].load(pd + at * a.dy_step);
                if (a.done) ends |= (a.done[at * a.n + l.seq] ? 1u : 0u) << u;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) m[i] = a.marks[(uint64_t)(t / U) * C + l.flat + i];
            // the states that the run's steps start from, as the forward pass had them
#pragma unroll
            for (uint32_t u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    h[u][i] = m[i];
                    const Gate w = gate_of(g[u].get(i));
                    m[i] = ends >> u & 1u ? 0.0f : __builtin_fmaf(w.a, m[i], w.take * x[u].get(i));
                }
#pragma unroll
            for (uint32_t k = 0; k < U; ++k) {
                const uint32_t u = U - 1u - k;
                if (u < run) {
                    float dx[V], dg[V];
                    const bool end = ends >> u & 1u;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const Gate w = gate_of(g[u].get(i));
                        const float e = (a.dy ? d[u].get(i) : 0.0f) + (end ? 0.0f : R[i]);
                        dx[i] = w.take * e;
                        dg[i] = w.a * dx[i] * (h[u][i] - x[u].get(i));
                        R[i] = w.a * e;
                    }
                    Channels<D, V>::store(qx + (uint64_t)(t + u) * a.y_step, dx, l.from);
                    Channels<D, V>::store(qg + (uint64_t)(t + u) * a.dgate_step, dg, l.from);
                }
            }
            left -= run;
        }
        if (a.last && s == 0u) l.put(a.last, R);
    }
}

}  // namespace rlsim_dev
