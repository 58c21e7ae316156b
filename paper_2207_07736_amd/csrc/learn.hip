// learn.hip -- host runtime of the learner's operators (rlsim_learner_* of
// include/rlsim.h): argument checks, choice of the kernels' forms, launches.
#include "rlsim.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>
#include <type_traits>
#include <vector>

#include "k_clip.hip.h"
#include "k_scan.hip.h"
#include "k_xent.hip.h"
#include "learn_dispatch.h"

using namespace rlsim_dev;

struct rlsim_learner {
    uint32_t max_rows = 0, max_dim = 0, max_vocab = 0;
    int device = 0;
    uint32_t cus = 1;
    hipStream_t stream = nullptr;
    char* work = nullptr;
    uint64_t clip_at = 0, xent_at = 0, bytes = 0;   // of the workspace: maps of segments, sums, cross entropy
    uint32_t clip_blocks = 0;
    char err[256] = "";
};

namespace {

thread_local char g_learn_err[256] = "";

int learn_fail(rlsim_learner* h, int code, const char* fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    (void)vsnprintf(h ? h->err : g_learn_err, sizeof h->err, fmt, ap);
    va_end(ap);
    return code;
}

// Makes the handle's device current for the scope, restoring the caller's.
struct LearnDevice {
    int prev = -1;
    bool ok = true;
    explicit LearnDevice(int dev)
    {
        if (hipGetDevice(&prev) != hipSuccess) { ok = false; return; }
        if (prev != dev && hipSetDevice(dev) != hipSuccess) ok = false;
    }
    ~LearnDevice()
    {
        int cur = -1;
        if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
    }
};

constexpr uint64_t kScanMaxStride = 1ull << 40, kXentMaxStride = 1ull << 32, kMaxElements = 1ull << 40;
constexpr uint64_t kLearnCacheBytes = 256ull << 20;
constexpr uint32_t kMaxTensors = 1u << 20, kScanMost = 1u << 30;

bool known_type(int d) { return d == RLSIM_F32 || d == RLSIM_BF16 || d == RLSIM_F16; }
uint32_t type_bytes(int d) { return d == RLSIM_F32 ? 4u : 2u; }
bool on_boundary(const void* p, uint64_t bytes) { return (uintptr_t)p % bytes == 0u; }

// ---- spans of memory -------------------------------------------------------------
// [first, last) in bytes, and which call argument it is; written ones overlap nothing but
// a span that they may be the same as.
struct Bytes {
    const char* name;
    uintptr_t first, last;
    bool written;
    int same;                                     // index of the span it may equal, or -1
};
bool overlap(const Bytes& a, const Bytes& b) { return a.first < b.last && b.first < a.last; }

struct Spans {
    Bytes b[16];
    int count = 0;
    int add(const char* name, const void* p, uint64_t bytes, bool written, int same = -1)
    {
        if (!p) return -1;
        b[count] = {name, (uintptr_t)p, (uintptr_t)p + bytes, written, same};
        return count++;
    }
    // The first clash, as two names.
    bool clash(const char** one, const char** two) const
    {
        for (int i = 0; i < count; ++i)
            for (int j = 0; j < i; ++j) {
                if (!b[i].written && !b[j].written) continue;
                if (!overlap(b[i], b[j])) continue;
                if (b[i].same == j && b[i].first == b[j].first && b[i].last == b[j].last) continue;
                *one = b[i].name;
                *two = b[j].name;
                return true;
            }
        return false;
    }
};

// ---- the gated recurrence ----------------------------------------------------------
struct Plane { const char* name; const void* p; uint64_t step, seq; bool written; };

// One array of rows of channels: alignment, strides, and that rows written are apart.
const char* check_plane(const Plane& p, const rlsim_scan& s)
{
    const uint64_t c = s.channels;
    if (!on_boundary(p.p, type_bytes(s.dtype))) return "is not aligned to its element size";
    const uint64_t step = s.T > 1u ? p.step : 0u, seq = s.n > 1u ? p.seq : 0u;
    if (step > kScanMaxStride || seq > kScanMaxStride) return "has a stride above 2^40";
    if (!p.written) return nullptr;
    // the smaller stride holds a row, the larger one all rows of the smaller
    if (s.T > 1u && step < c) return "has rows that overlap";
    if (s.n > 1u && seq < c) return "has rows that overlap";
    if (s.T > 1u && s.n > 1u) {
        const bool time_outer = step >= seq;
        const uint64_t outer = time_outer ? step : seq, inner = time_outer ? seq : step, count = time_outer ? s.n : s.T;
        if (outer < (count - 1u) * inner + c) return "has rows that overlap";
    }
    return nullptr;
}
uint64_t plane_bytes(const Plane& p, const rlsim_scan& s)
{
    const uint64_t step = s.T > 1u ? p.step : 0u, seq = s.n > 1u ? p.seq : 0u;
    return ((s.T - 1u) * step + (s.n - 1u) * seq + s.channels) * type_bytes(s.dtype);
}

int check_scan(rlsim_learner* h, const char* who, const rlsim_scan* s, const Plane* planes, int count)
{
    if (!known_type(s->dtype)) return learn_fail(h, RLSIM_EINVAL, "%s: unknown dtype", who);
    if (s->T == 0u || s->n == 0u || s->channels == 0u || s->T > kScanMost || s->n > kScanMost || s->channels > kScanMost)
        return learn_fail(h, RLSIM_EINVAL, "%s: T, n and channels must be in [1, 2^30]", who);
    if ((uint64_t)s->T * s->n > kMaxElements / s->channels)
        return learn_fail(h, RLSIM_EINVAL, "%s: more than 2^40 elements", who);
    for (int i = 0; i < count; ++i) {
        if (!planes[i].p) continue;
        if (const char* what = check_plane(planes[i], *s)) return learn_fail(h, RLSIM_EINVAL, "%s: %s %s", who, planes[i].name, what);
    }
    return RLSIM_OK;
}

template <int D, int V, bool WIDE>
void launch_scan(const rlsim_learner* h, ScanArgs a)
{
    a.groups = (a.channels + V - 1u) / V;
    const uint64_t threads = (uint64_t)a.n * a.groups, C = (uint64_t)a.n * a.channels;
    // as their registers allow: k_scan_back_rows has 256 for fp32, 168 otherwise
    const ScanCut cut = scan_cut(threads, C, a.T, h->cus, !a.backward ? 4u : D == kHeadF32 ? 2u : 3u);
    a.segments = cut.segments;
    a.seg_len = cut.seg_len;
    a.map_a = reinterpret_cast<float*>(h->work);
    a.map_b = a.map_a + kScanMapEntries;
    const dim3 grid((uint32_t)std::min<uint64_t>((threads + 255u) / 256u, 1u << 22), cut.segments), block(256);
    if (cut.segments > 1u) {
        if (a.backward) hipLaunchKernelGGL((k_scan_back_maps<D, V, WIDE>), grid, block, 0, h->stream, a);
        else hipLaunchKernelGGL((k_scan_maps<D, V, WIDE>), grid, block, 0, h->stream, a);
        hipLaunchKernelGGL(k_scan_join, dim3((uint32_t)((C + 15u) / 16u)), block, 0, h->stream, a);
    }
    if (a.backward) hipLaunchKernelGGL((k_scan_back_rows<D, V, WIDE>), grid, block, 0, h->stream, a);
    else if (a.T == 1u) hipLaunchKernelGGL((k_scan_rows<D, V, 1u, WIDE>), grid, block, 0, h->stream, a);
    else hipLaunchKernelGGL((k_scan_rows<D, V, kScanMark, WIDE>), grid, block, 0, h->stream, a);
}

template <int D>
void scan_form(const rlsim_learner* h, const ScanArgs& a, bool wide)
{
    if (a.channels < 2u) wide ? launch_scan<D, 1, true>(h, a) : launch_scan<D, 1, false>(h, a);
    else wide ? launch_scan<D, 2, true>(h, a) : launch_scan<D, 2, false>(h, a);
}

void run_scan(const rlsim_learner* h, int dtype, const ScanArgs& a)
{
    const uint64_t far = std::max({a.x_seq, a.gate_seq, a.dy_seq, a.y_seq, a.dgate_seq});
    const bool wide = far * (a.n - 1u) + 4ull * a.channels >= 1ull << 32;
    if (dtype == RLSIM_F32) scan_form<kHeadF32>(h, a, wide);
    else if (dtype == RLSIM_BF16) scan_form<kHeadBF16>(h, a, wide);
    else scan_form<kHeadF16>(h, a, wide);
}

ScanArgs scan_args(const rlsim_scan& s)
{
    ScanArgs a{};
    const uint64_t e = type_bytes(s.dtype);
    a.x = static_cast<const char*>(s.x);
    a.gate = static_cast<const char*>(s.gate);
    a.x_step = s.T > 1u ? s.x_step * e : 0u;
    a.x_seq = s.n > 1u ? s.x_seq * e : 0u;
    a.gate_step = s.T > 1u ? s.gate_step * e : 0u;
    a.gate_seq = s.n > 1u ? s.gate_seq * e : 0u;
    a.done = s.done;
    a.marks = s.marks;
    a.T = s.T;
    a.n = s.n;
    a.channels = s.channels;
    return a;
}

// ---- the output layer's cross entropy ------------------------------------------------
template <int D, int F, bool AA, bool BA, int EPI>
void launch_gemm(const rlsim_learner* h, XentGemm a, const XentTile& t)
{
    a.tiles_m = (a.M + t.m - 1u) / t.m;
    a.tiles_n = ((EPI == kXentDz ? a.rows_k : a.N) + t.n - 1u) / t.n;
    a.share = t.share;
    a.steps = (a.K + kXentK - 1u) / kXentK;
    const dim3 grid(a.tiles_m * a.tiles_n, t.share);
    if (t.n == 32u) hipLaunchKernelGGL((k_xent_gemm<D, F, 128, 32, 4, 1, AA, BA, EPI>), grid, dim3(256), 0, h->stream, a);
    else if (t.m == 128u) hipLaunchKernelGGL((k_xent_gemm<D, F, 128, 128, 2, 2, AA, BA, EPI>), grid, dim3(256), 0, h->stream, a);
    else hipLaunchKernelGGL((k_xent_gemm<D, F, 256, 256, 2, 4, AA, BA, EPI>), grid, dim3(512), 0, h->stream, a);
}

// A copy's workgroups; none for one that is not made.
uint32_t lay_blocks(const XentLay& a)
{
    const uint64_t blocks = a.cut ? (a.tall + 3ull) / 4u : ((uint64_t)a.tall * (a.wide / 8u) + 255u) / 256u;
    return (uint32_t)std::min<uint64_t>(blocks, 1u << 21);
}

template <int F>
void launch_lays(const rlsim_learner* h, XentLay a, XentLay b, XentLay c)
{
    a.blocks = lay_blocks(a);
    b.blocks = lay_blocks(b);
    c.blocks = lay_blocks(c);
    const uint32_t all = a.blocks + b.blocks + c.blocks;
    if (all) hipLaunchKernelGGL(k_xent_lays<F>, dim3(all), dim3(256), 0, h->stream, a, b, c);
}

template <int F>
void launch_round(const rlsim_learner* h, XentRound a, XentRound b)
{
    // a launch holds fewer than 2^32 threads
    a.blocks = (uint32_t)std::min<uint64_t>(((uint64_t)a.rows * ((a.dim + 3u) / 4u) + 255u) / 256u, 1u << 21);
    b.blocks = (uint32_t)std::min<uint64_t>(((uint64_t)b.rows * ((b.dim + 3u) / 4u) + 255u) / 256u, 1u << 21);
    if (a.blocks + b.blocks) hipLaunchKernelGGL(k_xent_round<F>, dim3(a.blocks + b.blocks), dim3(256), 0, h->stream, a, b);
}

// Rows that the products can read where they are.
bool as_they_are(const void* p, uint64_t stride, uint32_t dim)
{
    return dim % 8u == 0u && on_boundary(p, 16u) && stride % 8u == 0u && stride <= 1u << 22;
}

template <int D, int F>
void run_xent(const rlsim_learner* h, const rlsim_xent& x)
{
    constexpr uint32_t P = F == kHeadF32 ? 2u : 1u;
    constexpr uint64_t e = F == kHeadF32 ? 4u : 2u;
    const XentShape s = xent_shape(x.rows, x.dim, x.vocab, P);
    const XentWork o = xent_work(s);
    char* const w = h->work + h->xent_at;
    auto* part = reinterpret_cast<float2*>(w + o.part);
    auto* zt = reinterpret_cast<float*>(w + o.zt);
    auto* row = reinterpret_cast<XentRow*>(w + o.info);
    float* stats = x.stats ? x.stats : reinterpret_cast<float*>(w + o.stats);
    const bool grad = x.dhidden || x.dmatrix;
    const XentTarget target{x.target, x.target_bytes, x.vocab};
    const char* const matrix = static_cast<const char*>(x.matrix);
    auto* up_n = reinterpret_cast<int32_t*>(w + o.up_n);
    auto* up_m = reinterpret_cast<int32_t*>(w + o.up_m);
    auto* refs = reinterpret_cast<uint32_t*>(w + o.refs);

    const bool hidden_direct = P == 1u && as_they_are(x.hidden, x.hidden_stride, x.dim);
    const bool direct = P == 1u && as_they_are(x.matrix, x.matrix_stride, x.dim);
    XentGemm z{};                                 // the logits' product
    z.products = P == 1u ? 1u : 3u;
    z.K = P == 1u ? x.dim : s.dim_k;
    z.vocab = x.vocab;
    z.N = x.rows;
    z.rows_k = s.rows_k;
    z.target = target;
    z.part = part;
    z.zt = zt;
    z.row = row;
    z.up_n = up_n;
    z.up_m = up_m;
    z.refs = refs;
    z.B = hidden_direct ? static_cast<const char*>(x.hidden) : w + o.x;
    z.ldb = hidden_direct ? x.hidden_stride * e : 2ull * s.dim_k;
    z.part_b = 2ull * s.dim_k * x.rows;
    z.lda = direct ? x.matrix_stride * e : 2ull * s.dim_k;
    constexpr uint32_t cut = F == kHeadF32 ? 1u : 0u;
    XentLay hidden_lay{}, masked_lay{};           // made with the first piece of the matrix
    if (!hidden_direct)
        hidden_lay = XentLay{static_cast<const char*>(x.hidden), x.hidden_stride * e, x.rows, x.dim, s.dim_k, x.rows, w + o.x,
                             z.part_b, {}, nullptr, cut ? up_n : nullptr, cut, 0u};
    if (x.dmatrix)                                // rows that do not count may hold anything
        masked_lay = XentLay{static_cast<const char*>(x.hidden), x.hidden_stride * e, x.rows, x.dim, s.dim_k, s.rows_k, w + o.xm,
                             2ull * s.dim_k * s.rows_k, target, x.weight, F == kHeadBF16 ? up_n : nullptr, F != kHeadF16 ? 1u : 0u, 0u};

    // The piece of the vocabulary from v0, as the products read it.
    uint32_t laid = ~0u;                          // the piece that is copied now
    auto piece = [&](uint32_t v0, uint32_t count) {
        z.m0 = v0;
        z.M = count;
        const char* const from = matrix + (uint64_t)v0 * x.matrix_stride * e;
        z.A = direct ? from : w + o.w;
        z.part_a = 2ull * s.dim_k * s.piece;
        XentLay l{};
        if (!direct && laid != v0)
            l = XentLay{from, x.matrix_stride * e, count, x.dim, s.dim_k, (uint32_t)up_to(count, kXentK), w + o.w, z.part_a,
                        {}, nullptr, cut ? up_m : nullptr, cut, 0u};
        launch_lays<F>(h, hidden_lay, masked_lay, l);
        hidden_lay = masked_lay = XentLay{};
        laid = v0;
    };

    XentJoin j{};
    j.rows = x.rows;
    j.rows_k = s.rows_k;
    j.zt = zt;
    j.target = target;
    j.weight = x.weight;
    j.stats = stats;
    j.loss = x.loss;
    j.row = grad ? row : nullptr;
    if (x.loss) {
        const uint32_t width = direct ? (uint32_t)std::min<uint64_t>(x.vocab, xent_width(s.rows_k)) : s.piece;
        for (uint32_t v0 = 0u; v0 < x.vocab; v0 += width) {
            const uint32_t count = std::min(width, x.vocab - v0);
            piece(v0, count);
            const XentTile t = xent_tile(count, x.rows, (uint64_t)s.dim_k / kXentK * z.products, false, h->cus);
            z.part0 = j.parts;
            launch_gemm<D, F, false, false, kXentLoss>(h, z, t);
            j.parts += (count + t.m - 1u) / t.m * (t.m / t.span);
        }
        j.part = part;
    }
    // before a call for gradients alone, the first copies
    if (!x.loss) piece(0u, std::min(s.piece, x.vocab));
    // dz's powers of two (fp32: of the piece that the loss left in the copy)
    XentRefs refs_of{target, x.weight, F != kHeadF16 && x.dmatrix ? up_n : nullptr, F == kHeadF32 ? up_m : nullptr, x.rows,
                     z.M, grad ? refs : nullptr, 0u};
    if (refs_of.out) refs_of.blocks = (x.rows + kRefRows - 1u) / kRefRows;
    if (refs_of.blocks > 1u) hipLaunchKernelGGL(k_xent_refs_none, dim3(1), dim3(64), 0, h->stream, refs);
    hipLaunchKernelGGL(k_xent_join, dim3((x.rows + kJoinRows - 1u) / kJoinRows + refs_of.blocks), dim3(256), 0, h->stream, j, refs_of);
    if (!grad) return;

    const uint64_t dim4 = up_to(x.dim, 4u);
    z.dz_w = x.dmatrix ? w + o.dz_w : nullptr;
    z.dz_w_parts = F == kHeadF32 || (F == kHeadF16 && x.rows <= kXentFewRows) ? 2u : 1u;
    const uint32_t stack = F != kHeadF32 && x.rows <= kXentStackRows ? kXentStackRows : 0u;
    z.dz_stack = stack;
    z.dz = x.dhidden ? w + o.dz : nullptr;
    z.dz_ld = 2ull * s.piece;
    z.dz_part = z.dz_ld * s.rows_k;
    XentGemm gx{}, gw{};                          // dhidden's and dmatrix's products
    gx.products = z.products;
    gw.products = F == kHeadF32 ? 3u : z.dz_w_parts;
    gx.M = gw.M = x.dim;
    gx.sum_ld = gw.sum_ld = dim4;
    // what the products are short of (fp32's dhidden: its sums are not)
    const OutScale scale_x{row, nullptr, F == kHeadF16 ? -kDzUp : 0, 1u}, scale_w{nullptr, refs, 0, 0u};
    gx.sum_ref = F == kHeadF32 ? refs + 1 : nullptr;
    gw.scale = scale_w;
    gx.lda = z.lda;
    gx.B = z.dz;
    gx.ldb = gw.ldb = z.dz_ld;
    gx.part_b = gw.part_b = z.dz_part;
    gx.N = stack ? 2u * stack : x.rows;
    gx.sum = reinterpret_cast<float*>(w + o.dx);
    gx.sum_share = gx.N * dim4;
    gw.A = w + o.xm;
    gw.lda = 2ull * s.dim_k;
    gw.part_a = gw.lda * s.rows_k;
    gw.B = z.dz_w;
    gw.K = s.rows_k;
    gw.sum = reinterpret_cast<float*>(w + o.dw);
    const XentTile tx = xent_tile(x.dim, gx.N, (uint64_t)s.piece / kXentK * z.products, true, h->cus);
    for (uint32_t v0 = 0u; v0 < x.vocab; v0 += s.piece) {
        const uint32_t count = std::min(s.piece, x.vocab - v0);
        XentRound rx{}, rw{};
        const bool anew = laid != v0;
        piece(v0, count);
        if (F == kHeadF32 && anew) {
            refs_of.count = count;
            if (refs_of.blocks > 1u) hipLaunchKernelGGL(k_xent_refs_none, dim3(1), dim3(64), 0, h->stream, refs);
            hipLaunchKernelGGL(k_xent_refs, dim3(refs_of.blocks), dim3(256), 0, h->stream, refs_of);
        }
        launch_gemm<D, F, false, false, kXentDz>(h, z, xent_tile(count, x.rows, (uint64_t)s.dim_k / kXentK * z.products, false, h->cus));
        if (x.dhidden) {
            gx.A = z.A;
            gx.part_a = z.part_a;
            gx.K = direct ? count : (uint32_t)up_to(count, kXentK);
            gx.add = v0 ? 1u : 0u;
            launch_gemm<D, F, true, false, kXentSum>(h, gx, tx);
        }
        if (x.dmatrix) {
            const XentTile t = xent_tile(x.dim, count, s.rows_k / kXentK * gw.products, true, h->cus);
            gw.N = count;
            char* const out = static_cast<char*>(x.dmatrix) + (uint64_t)v0 * x.dmatrix_stride * e;
            if (t.share == 1u) {
                gw.out = out;
                gw.out_ld = x.dmatrix_stride * e;
                launch_gemm<kHeadF16, F, true, true, kXentOut>(h, gw, t);
            } else {
                gw.sum_share = count * dim4;
                launch_gemm<kHeadF16, F, true, true, kXentSum>(h, gw, t);
                rw = XentRound{gw.sum, dim4, gw.sum_share, t.share, count, x.dim, 0u, scale_w, out, x.dmatrix_stride * e, 0u};
            }
        }
        const bool done = count == x.vocab - v0;
        if (done && x.dhidden)
            rx = XentRound{gx.sum, dim4, gx.sum_share, tx.share, x.rows, x.dim, stack, scale_x, static_cast<char*>(x.dhidden),
                           x.dhidden_stride * e, 0u};
        launch_round<F>(h, rx, rw);
    }
}

// ---- clipping --------------------------------------------------------------------
// Whether what is written overlaps anything but its own input.
struct ClipSpan {
    uintptr_t first, last;
    uint32_t owner;                               // tensor; an in-place tensor has one span
    bool written;
};
const char* clip_clash(const rlsim_tensor* t, uint32_t count, const float* norm, bool scaling)
{
    std::vector<ClipSpan> spans;
    spans.reserve(2u * (size_t)count + 1u);
    spans.push_back({(uintptr_t)norm, (uintptr_t)norm + 4u, count, true});
    bool sorted = true;
    for (uint32_t i = 0; i < count; ++i) {
        if (!t[i].elements) continue;
        const bool in_place = !t[i].out || t[i].out == t[i].data;
        const uintptr_t d = (uintptr_t)t[i].data;
        spans.push_back({d, d + t[i].elements * type_bytes(t[i].dtype), i, in_place && scaling});
        if (!in_place) {
            const uintptr_t o = (uintptr_t)t[i].out;
            spans.push_back({o, o + t[i].elements * type_bytes(t[i].out_dtype), i, true});
        }
    }
    for (size_t i = 1; i < spans.size() && sorted; ++i) sorted = spans[i - 1].first <= spans[i].first;
    if (!sorted) std::sort(spans.begin(), spans.end(), [](const ClipSpan& a, const ClipSpan& b) { return a.first < b.first; });
    // the farthest ends so far, of what is written and of all
    uintptr_t written = 0u, any = 0u;
    for (const ClipSpan& s : spans) {
        if (s.first < written || (s.written && s.first < any)) return "an output overlaps another tensor or output";
        any = std::max(any, s.last);
        if (s.written) written = std::max(written, s.last);
    }
    return nullptr;
}

void run_clip(const rlsim_learner* h, const rlsim_tensor* t, uint32_t count, double max_norm, float* norm)
{
    uint64_t total = 0u, bytes = 0u;
    for (uint32_t i = 0; i < count; ++i) {
        total += t[i].elements;
        bytes += t[i].elements * type_bytes(t[i].dtype);
    }
    ClipArgs a{};
    // us, 400 M bf16 into tensors of their own: 458, past the cache 427
    a.past_cache = bytes > kLearnCacheBytes ? 1u : 0u;
    a.chunk = clip_chunk(total);
    a.max_norm = max_norm;
    a.sums = reinterpret_cast<double*>(h->work + h->clip_at);
    a.norm = norm;
    for (uint32_t i = 0; i < count; ++i) a.blocks += (uint32_t)((t[i].elements + a.chunk - 1u) / a.chunk);
    // twice over the tensors, as many at a time as a launch's arguments hold
    for (int pass = 0; pass < 2; ++pass) {
        uint32_t i = 0u;
        a.base = 0u;
        bool any = false;
        do {
            a.count = 0u;
            a.first[0] = 0u;
            for (; i < count && a.count < kClipTensors; ++i) {
                if (!t[i].elements) continue;
                const uint32_t k = a.count++;
                a.t[k] = {static_cast<const char*>(t[i].data), static_cast<char*>(t[i].out ? t[i].out : const_cast<void*>(t[i].data)), t[i].elements};
                a.dtype[k] = (uint8_t)t[i].dtype;
                a.out_dtype[k] = (uint8_t)(a.t[k].out == a.t[k].data ? t[i].dtype : t[i].out_dtype);
                a.first[k + 1] = a.first[k] + (uint32_t)((t[i].elements + a.chunk - 1u) / a.chunk);
            }
            if (i == count && !any && total <= kClipSmall) {
                hipLaunchKernelGGL(k_clip_small, dim3(1), dim3(1024), 0, h->stream, a);
                return;
            }
            const uint32_t blocks = a.first[a.count];
            if (pass == 0 && blocks) hipLaunchKernelGGL(k_clip_squares, dim3(blocks), dim3(256), 0, h->stream, a);
            if (pass == 1 && (blocks || !any)) hipLaunchKernelGGL(k_clip_scale, dim3(std::max(blocks, 1u)), dim3(256), 0, h->stream, a);
            a.base += blocks;
            any = true;
        } while (i < count);
    }
}

}  // namespace

extern "C" {

int rlsim_learner_create(uint32_t max_rows, uint32_t max_dim, uint32_t max_vocab, void* stream, rlsim_learner_t** out)
{
    if (!out) return learn_fail(nullptr, RLSIM_EINVAL, "rlsim_learner_create: out is NULL");
    *out = nullptr;
    const bool none = !max_rows && !max_dim && !max_vocab;
    if (!none && (!max_rows || !max_dim || !max_vocab))
        return learn_fail(nullptr, RLSIM_EINVAL, "rlsim_learner_create: max_rows, max_dim and max_vocab are all 0 or none is");
    if (max_rows > 1u << 22 || max_dim > 1u << 16 || max_vocab > 1u << 20)
        return learn_fail(nullptr, RLSIM_EINVAL, "rlsim_learner_create: max_rows must be at most 2^22, max_dim 2^16, max_vocab 2^20");
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    int cus = 0;
    if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device);
    if (e != hipSuccess) return learn_fail(nullptr, RLSIM_EDEVICE, "rlsim_learner_create: %s", hipGetErrorString(e));
    rlsim_learner* h = new (std::nothrow) rlsim_learner;
    if (!h) return learn_fail(nullptr, RLSIM_ENOMEM, "rlsim_learner_create: host allocation failed");
    h->max_rows = max_rows;
    h->max_dim = max_dim;
    h->max_vocab = max_vocab;
    h->device = device;
    h->cus = (uint32_t)std::max(cus, 1);
    h->stream = static_cast<hipStream_t>(stream);
    h->clip_blocks = 2u * kClipBlocks + kMaxTensors;
    h->clip_at = up_to(8ull * kScanMapEntries, 256u);
    h->xent_at = h->clip_at + up_to(8ull * h->clip_blocks, 256u);
    h->bytes = h->xent_at + (none ? 0u : std::max(xent_bound(max_rows, max_dim, max_vocab, 1u), xent_bound(max_rows, max_dim, max_vocab, 2u)));
    e = hipMalloc(reinterpret_cast<void**>(&h->work), h->bytes);
    if (e != hipSuccess) {
        const int code = e == hipErrorOutOfMemory ? RLSIM_ENOMEM : RLSIM_EDEVICE;
        delete h;
        (void)hipGetLastError();
        return learn_fail(nullptr, code, "rlsim_learner_create: %s", hipGetErrorString(e));
    }
    *out = h;
    return RLSIM_OK;
}

int rlsim_learner_scan(rlsim_learner_t* h, const rlsim_scan* s)
{
    static const char who[] = "rlsim_learner_scan";
    if (!h) return learn_fail(nullptr, RLSIM_EINVAL, "%s: handle is NULL", who);
    if (!s) return learn_fail(h, RLSIM_EINVAL, "%s: arguments are NULL", who);
    if (!s->x || !s->gate || !s->y) return learn_fail(h, RLSIM_EINVAL, "%s: x, gate or y is NULL", who);
    const Plane planes[] = {{"x", s->x, s->x_step, s->x_seq, false}, {"gate", s->gate, s->gate_step, s->gate_seq, false},
                            {"y", s->y, s->y_step, s->y_seq, true}};
    if (const int rc = check_scan(h, who, s, planes, 3)) return rc;
    if (!on_boundary(s->state, 4u) || !on_boundary(s->marks, 4u) || !on_boundary(s->last, 4u))
        return learn_fail(h, RLSIM_EINVAL, "%s: state, marks or last is not 4-byte aligned", who);
    const uint64_t wide = (uint64_t)s->n * s->channels * 4u, marks = (s->T + kScanMark - 1ull) / kScanMark;
    Spans b;
    for (int i = 0; i < 3; ++i) b.add(planes[i].name, planes[i].p, plane_bytes(planes[i], *s), planes[i].written);
    b.add("done", s->done, (uint64_t)s->T * s->n, false);
    const int state = b.add("state", s->state, wide, false);
    b.add("marks", s->marks, marks * wide, true);
    b.add("last", s->last, wide, true, state);
    const char *one, *two;
    if (b.clash(&one, &two)) return learn_fail(h, RLSIM_EINVAL, "%s: %s overlaps %s", who, one, two);
    LearnDevice g(h->device);
    if (!g.ok) return learn_fail(h, RLSIM_EDEVICE, "%s: cannot select the handle's device", who);
    ScanArgs a = scan_args(*s);
    const uint64_t e = type_bytes(s->dtype);
    a.y = static_cast<char*>(s->y);
    a.y_step = s->T > 1u ? s->y_step * e : 0u;
    a.y_seq = s->n > 1u ? s->y_seq * e : 0u;
    a.state = s->state;
    a.last = s->last;
    run_scan(h, s->dtype, a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return learn_fail(h, RLSIM_EDEVICE, "%s: launch: %s", who, hipGetErrorString(err));
    return RLSIM_OK;
}

int rlsim_learner_scan_grad(rlsim_learner_t* h, const rlsim_scan* s, const rlsim_scan_grad* d)
{
    static const char who[] = "rlsim_learner_scan_grad";
    if (!h) return learn_fail(nullptr, RLSIM_EINVAL, "%s: handle is NULL", who);
    if (!s || !d) return learn_fail(h, RLSIM_EINVAL, "%s: arguments are NULL", who);
    if (!s->x || !s->gate || !s->marks) return learn_fail(h, RLSIM_EINVAL, "%s: x, gate or marks is NULL", who);
    if (!d->dx || !d->dgate) return learn_fail(h, RLSIM_EINVAL, "%s: dx or dgate is NULL", who);
    const Plane planes[] = {{"x", s->x, s->x_step, s->x_seq, false}, {"gate", s->gate, s->gate_step, s->gate_seq, false},
                            {"dy", d->dy, d->dy_step, d->dy_seq, false}, {"dx", d->dx, d->dx_step, d->dx_seq, true},
                            {"dgate", d->dgate, d->dgate_step, d->dgate_seq, true}};
    if (const int rc = check_scan(h, who, s, planes, 5)) return rc;
    if (!on_boundary(s->marks, 4u) || !on_boundary(d->dlast, 4u) || !on_boundary(d->dstate, 4u))
        return learn_fail(h, RLSIM_EINVAL, "%s: marks, dlast or dstate is not 4-byte aligned", who);
    const uint64_t wide = (uint64_t)s->n * s->channels * 4u, marks = (s->T + kScanMark - 1ull) / kScanMark;
    Spans b;
    for (int i = 0; i < 5; ++i) b.add(planes[i].name, planes[i].p, planes[i].p ? plane_bytes(planes[i], *s) : 0u, planes[i].written);
    b.add("done", s->done, (uint64_t)s->T * s->n, false);
    b.add("marks", s->marks, marks * wide, false);
    const int dlast = b.add("dlast", d->dlast, wide, false);
    b.add("dstate", d->dstate, wide, true, dlast);
    const char *one, *two;
    if (b.clash(&one, &two)) return learn_fail(h, RLSIM_EINVAL, "%s: %s overlaps %s", who, one, two);
    LearnDevice g(h->device);
    if (!g.ok) return learn_fail(h, RLSIM_EDEVICE, "%s: cannot select the handle's device", who);
    ScanArgs a = scan_args(*s);
    const uint64_t e = type_bytes(s->dtype);
    const bool many = s->T > 1u, more = s->n > 1u;
    a.dy = static_cast<const char*>(d->dy);
    a.dy_step = many ? d->dy_step * e : 0u;
    a.dy_seq = more ? d->dy_seq * e : 0u;
    a.y = static_cast<char*>(d->dx);
    a.y_step = many ? d->dx_step * e : 0u;
    a.y_seq = more ? d->dx_seq * e : 0u;
    a.dgate = static_cast<char*>(d->dgate);
    a.dgate_step = many ? d->dgate_step * e : 0u;
    a.dgate_seq = more ? d->dgate_seq * e : 0u;
    a.state = d->dlast;
    a.last = d->dstate;
    a.backward = 1u;
    run_scan(h, s->dtype, a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return learn_fail(h, RLSIM_EDEVICE, "%s: launch: %s", who, hipGetErrorString(err));
    return RLSIM_OK;
}

int rlsim_learner_xent(rlsim_learner_t* h, const rlsim_xent* x)
{
    static const char who[] = "rlsim_learner_xent";
    if (!h) return learn_fail(nullptr, RLSIM_EINVAL, "%s: handle is NULL", who);
    if (!x) return learn_fail(h, RLSIM_EINVAL, "%s: arguments are NULL", who);
    if (!known_type(x->dtype)) return learn_fail(h, RLSIM_EINVAL, "%s: unknown dtype", who);
    if (!h->max_rows) return learn_fail(h, RLSIM_EINVAL, "%s: the handle was made without an output layer's sizes", who);
    if (x->rows == 0u || x->rows > h->max_rows) return learn_fail(h, RLSIM_EINVAL, "%s: rows must be in [1, max_rows]", who);
    if (x->dim == 0u || x->dim > h->max_dim) return learn_fail(h, RLSIM_EINVAL, "%s: dim must be in [1, max_dim]", who);
    if (x->vocab == 0u || x->vocab > h->max_vocab) return learn_fail(h, RLSIM_EINVAL, "%s: vocab must be in [1, max_vocab]", who);
    if (!x->hidden || !x->matrix || !x->target) return learn_fail(h, RLSIM_EINVAL, "%s: hidden, matrix or target is NULL", who);
    if (x->target_bytes != 1 && x->target_bytes != 4 && x->target_bytes != 8)
        return learn_fail(h, RLSIM_EINVAL, "%s: target_bytes must be 1, 4 or 8", who);
    if (!x->loss && !x->dhidden && !x->dmatrix) return learn_fail(h, RLSIM_EINVAL, "%s: nothing is wanted", who);
    if (!x->loss && !x->stats) return learn_fail(h, RLSIM_EINVAL, "%s: gradients alone need stats", who);
    const uint32_t e = type_bytes(x->dtype);
    struct Matrix2 { const char* name; const void* p; uint64_t stride; uint32_t rows; bool written; };
    const Matrix2 all[] = {{"hidden", x->hidden, x->hidden_stride, x->rows, false}, {"matrix", x->matrix, x->matrix_stride, x->vocab, false},
                           {"dhidden", x->dhidden, x->dhidden_stride, x->rows, true},
                           {"dmatrix", x->dmatrix, x->dmatrix_stride, x->vocab, true}};
    Spans b;
    for (const Matrix2& m : all) {
        if (!m.p) continue;
        if (m.stride < x->dim || m.stride > kXentMaxStride)
            return learn_fail(h, RLSIM_EINVAL, "%s: %s: the row stride must be in [dim, 2^32]", who, m.name);
        if (!on_boundary(m.p, e)) return learn_fail(h, RLSIM_EINVAL, "%s: %s is not aligned to its element size", who, m.name);
        b.add(m.name, m.p, ((m.rows - 1u) * m.stride + x->dim) * e, m.written);
    }
    if (!on_boundary(x->target, (uint64_t)x->target_bytes)) return learn_fail(h, RLSIM_EINVAL, "%s: target is not aligned to its element size", who);
    if (!on_boundary(x->weight, 4u) || !on_boundary(x->loss, 4u) || !on_boundary(x->stats, 4u))
        return learn_fail(h, RLSIM_EINVAL, "%s: weight, loss or stats is not 4-byte aligned", who);
    b.add("target", x->target, (uint64_t)x->rows * (uint64_t)x->target_bytes, false);
    b.add("weight", x->weight, 4ull * x->rows, false);
    b.add("loss", x->loss, 4ull * x->rows, true);
    b.add("stats", x->stats, 12ull * x->rows, x->loss != nullptr);
    const char *one, *two;
    if (b.clash(&one, &two)) return learn_fail(h, RLSIM_EINVAL, "%s: %s overlaps %s", who, one, two);
    const uint32_t parts = x->dtype == RLSIM_F32 ? 2u : 1u;
    if (xent_work(xent_shape(x->rows, x->dim, x->vocab, parts)).end > h->bytes - h->xent_at)
        return learn_fail(h, RLSIM_EINVAL, "%s: the workspace does not hold this call", who);
    LearnDevice g(h->device);
    if (!g.ok) return learn_fail(h, RLSIM_EDEVICE, "%s: cannot select the handle's device", who);
    if (x->dtype == RLSIM_F32) run_xent<kHeadF16, kHeadF32>(h, *x);
    else if (x->dtype == RLSIM_BF16) run_xent<kHeadBF16, kHeadBF16>(h, *x);
    else run_xent<kHeadF16, kHeadF16>(h, *x);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return learn_fail(h, RLSIM_EDEVICE, "%s: launch: %s", who, hipGetErrorString(err));
    return RLSIM_OK;
}

int rlsim_learner_clip(rlsim_learner_t* h, const rlsim_tensor* t, uint32_t count, double max_norm, float* norm)
{
    static const char who[] = "rlsim_learner_clip";
    if (!h) return learn_fail(nullptr, RLSIM_EINVAL, "%s: handle is NULL", who);
    if (!norm || (count && !t)) return learn_fail(h, RLSIM_EINVAL, "%s: norm or tensors is NULL", who);
    if (count > kMaxTensors) return learn_fail(h, RLSIM_EINVAL, "%s: count must be at most 2^20", who);
    if (!(max_norm > 0.0)) return learn_fail(h, RLSIM_EINVAL, "%s: max_norm must be > 0", who);
    if (!on_boundary(norm, 4u)) return learn_fail(h, RLSIM_EINVAL, "%s: norm is not 4-byte aligned", who);
    uint64_t total = 0u;
    for (uint32_t i = 0; i < count; ++i) {
        if (!known_type(t[i].dtype)) return learn_fail(h, RLSIM_EINVAL, "%s: tensor %u: unknown dtype", who, i);
        const bool in_place = !t[i].out || (t[i].out == t[i].data && t[i].out_dtype == t[i].dtype);
        if (!in_place && !known_type(t[i].out_dtype)) return learn_fail(h, RLSIM_EINVAL, "%s: tensor %u: unknown out_dtype", who, i);
        if (!t[i].elements) continue;
        if (t[i].elements > kMaxElements || (total += t[i].elements) > kMaxElements)
            return learn_fail(h, RLSIM_EINVAL, "%s: tensor %u: more than 2^40 elements", who, i);
        if (!t[i].data) return learn_fail(h, RLSIM_EINVAL, "%s: tensor %u: data is NULL", who, i);
        if (!in_place && t[i].out == t[i].data) return learn_fail(h, RLSIM_EINVAL, "%s: tensor %u: in place in another type", who, i);
        if (!on_boundary(t[i].data, type_bytes(t[i].dtype)) || (!in_place && !on_boundary(t[i].out, type_bytes(t[i].out_dtype))))
            return learn_fail(h, RLSIM_EINVAL, "%s: tensor %u is not aligned to its element size", who, i);
    }
    try {
        if (const char* what = clip_clash(t, count, norm, max_norm < INFINITY)) return learn_fail(h, RLSIM_EINVAL, "%s: %s", who, what);
    } catch (const std::exception&) {
        return learn_fail(h, RLSIM_ENOMEM, "%s: host allocation failed", who);
    }
    LearnDevice g(h->device);
    if (!g.ok) return learn_fail(h, RLSIM_EDEVICE, "%s: cannot select the handle's device", who);
    run_clip(h, t, count, max_norm, norm);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return learn_fail(h, RLSIM_EDEVICE, "%s: launch: %s", who, hipGetErrorString(err));
    return RLSIM_OK;
}

int rlsim_learner_destroy(rlsim_learner_t* h)
{
    if (!h) return RLSIM_OK;
    int rc = RLSIM_OK;
    {
        LearnDevice g(h->device);
        if (hipStreamSynchronize(h->stream) != hipSuccess) rc = RLSIM_EDEVICE;
        if (h->work) (void)hipFree(h->work);
    }
    delete h;
    return rc;
}

const char* rlsim_learner_last_error(const rlsim_learner_t* h) { return h ? h->err : g_learn_err; }

}  // extern "C"
