// head.hip -- host runtime of the output head's operators (rlsim_head_* of
// include/rlsim.h): argument checks, choice of the kernel's form, launch.
#include "rlsim.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>

#include "head_dispatch.h"
#include "k_distill.hip.h"
#include "k_sample.hip.h"

using namespace rlsim_dev;

struct rlsim_head {
    uint32_t max_rows = 0, max_vocab = 0;
    int device = 0;
    uint32_t cus = 1;
    hipStream_t stream = nullptr;
    char* work = nullptr;       // what the workgroups that share a row hand on (SampleSplit)
    uint32_t split_rows = 0;    // most rows of such a call
    char err[256] = "";
};

namespace {

thread_local char g_head_err[256] = "";

int head_fail(rlsim_head* h, int code, const char* fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    (void)vsnprintf(h ? h->err : g_head_err, sizeof h->err, fmt, ap);
    va_end(ap);
    return code;
}

// Makes the handle's device current for the scope, restoring the caller's.
struct HeadDevice {
    int prev = -1;
    bool ok = true;
    explicit HeadDevice(int dev)
    {
        if (hipGetDevice(&prev) != hipSuccess) { ok = false; return; }
        if (prev != dev && hipSetDevice(dev) != hipSuccess) ok = false;
    }
    ~HeadDevice()
    {
        int cur = -1;
        if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
    }
};

constexpr uint64_t kLastLevelBytes = 256ull << 20;
constexpr uint64_t kMaxStride = 1ull << 32;       // elements: 2^30 rows end below 2^64 bytes

bool known_dtype(int d) { return d == RLSIM_F32 || d == RLSIM_BF16 || d == RLSIM_F16; }
uint32_t dtype_bytes(int d) { return d == RLSIM_F32 ? 4u : 2u; }
bool aligned(const void* p, uint32_t bytes) { return (uintptr_t)p % bytes == 0u; }

// The rows of logits of either operator; null if they are sound.
const char* check_rows(const rlsim_head* h, int dtype, const void* logits, uint32_t rows, uint32_t vocab, uint64_t stride)
{
    if (!known_dtype(dtype)) return "unknown dtype";
    if (!logits) return "logits is NULL";
    if (rows == 0u || rows > h->max_rows) return "rows must be in [1, max_rows]";
    if (vocab == 0u || vocab > h->max_vocab) return "vocab must be in [1, max_vocab]";
    if (stride < vocab || stride > kMaxStride) return "the row stride must be in [vocab, 2^32]";
    if (!aligned(logits, dtype_bytes(dtype))) return "logits must be aligned to its element size";
    return nullptr;
}

// Workgroups of a kernel for `items` rows (or groups of rows): one each, as far as a launch
// holds fewer than 2^32 threads.  (Fewer that go through several rows each, as many as fit
// the GPU: 20,000 x 8,000 bf16 distilled in 226 us instead of 199.)
uint32_t head_grid(uint32_t items) { return std::min(items, 1u << 21); }

// Rows of up to kHeadTinyVocab entries: FEW has a thread to a row, TINY some lanes.
#define HEAD_TINY(FEW, TINY, D, h, a)                                                                                        \
    do {                                                                                                                     \
        const uint32_t lanes = (a).V <= 8u ? 1u : (a).V <= 16u ? 16u : (a).V <= 32u ? 32u : 64u;                             \
        const dim3 grid(head_grid(((a).rows + 256u / lanes - 1u) / (256u / lanes))), block(256);                            \
        if ((a).V <= 2u) hipLaunchKernelGGL((FEW<D, 2>), grid, block, 0, (h)->stream, a);                                    \
        else if ((a).V <= 4u) hipLaunchKernelGGL((FEW<D, 4>), grid, block, 0, (h)->stream, a);                               \
        else if ((a).V <= 8u) hipLaunchKernelGGL((FEW<D, 8>), grid, block, 0, (h)->stream, a);                               \
        else if ((a).V <= 16u) hipLaunchKernelGGL((TINY<D, 16>), grid, block, 0, (h)->stream, a);                            \
        else if ((a).V <= 32u) hipLaunchKernelGGL((TINY<D, 32>), grid, block, 0, (h)->stream, a);                            \
        else hipLaunchKernelGGL((TINY<D, 64>), grid, block, 0, (h)->stream, a);                                              \
    } while (0)

// The workspace of the calls that share rows, and its parts.
constexpr uint64_t kSplitGroupBytes = 8u + 8u * kSplitBins + 4u * 4u, kSplitRowBytes = 8u * kSplitList;
uint64_t split_bytes(uint32_t rows) { return kSplitGroups * kSplitGroupBytes + rows * kSplitRowBytes; }
DistillSplit distill_split(const rlsim_head* h)
{
    static_assert(kSplitRowBytes >= 8u * kHeadMaxTeacher);
    static_assert(kSplitGroups * kSplitGroupBytes >= kDistillSplitGroups * 12u);
    DistillSplit p{};
    char* at = h->work;
    p.sum = reinterpret_cast<double*>(at);
    at += 8u * kDistillSplitGroups;
    p.mu = reinterpret_cast<float*>(at);
    at += 4u * kDistillSplitGroups;
    p.entry = reinterpret_cast<uint32_t*>(at);
    at += 4ull * kHeadMaxTeacher * h->split_rows;
    p.logit = reinterpret_cast<float*>(at);
    return p;
}
SampleSplit sample_split(const rlsim_head* h)
{
    SampleSplit p{};
    char* at = h->work;
    p.sum = reinterpret_cast<uint64_t*>(at);
    at += 8u * kSplitGroups;
    p.part_w = reinterpret_cast<uint64_t*>(at);
    at += 8ull * kSplitGroups * kSplitBins;
    p.list = reinterpret_cast<uint64_t*>(at);
    at += 8ull * kSplitList * h->split_rows;
    p.top = reinterpret_cast<float*>(at);
    at += 4u * kSplitGroups;
    p.top_at = reinterpret_cast<uint32_t*>(at);
    at += 4u * kSplitGroups;
    p.count = reinterpret_cast<uint32_t*>(at);
    at += 4u * kSplitGroups;
    p.list_z = reinterpret_cast<float*>(at);
    return p;
}

template <int D>
void launch_sample(const rlsim_head* h, const SampleArgs& a)
{
    if (a.V <= kHeadTinyVocab) {
        HEAD_TINY(k_sample_few, k_sample_tiny, D, h, a);
        return;
    }
    const uint32_t shared_by = a.rows <= h->split_rows ? sample_chunks(a.rows, a.V, Elem<D>::kBytes, h->cus) : 1u;
    if (shared_by > 1u && a.rows * shared_by <= kSplitGroups) {
        SampleSplit p = sample_split(h);
        const uint32_t strip = 64u * Elem<D>::kPerVec, strips = (a.V + strip - 1u) / strip;
        p.chunk = (strips + shared_by - 1u) / shared_by * strip;
        p.chunks = (a.V + p.chunk - 1u) / p.chunk;
        p.room = kSplitList / p.chunks;
        const dim3 grid(p.chunks, a.rows), block(kSplitThreads);
        hipLaunchKernelGGL(k_sample_top<D>, grid, block, 0, h->stream, a, p);
        hipLaunchKernelGGL(k_sample_chunk<D>, grid, block, 0, h->stream, a, p);
        hipLaunchKernelGGL(k_sample_draw<D>, dim3(a.rows), block, 0, h->stream, a, p);
        return;
    }
    const uint32_t threads = sample_threads(a.V, Elem<D>::kBytes);
    const dim3 grid(head_grid(a.rows)), block(threads);
    const bool cuts = a.top_k_rows || a.top_p_rows || (a.top_k && a.top_k < a.V) || a.top_p < 1.0f;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, h->stream, a); };
    if (threads == 64u) cuts ? launch(k_sample<D, 64, true>) : launch(k_sample<D, 64, false>);
    else if (threads == 256u) cuts ? launch(k_sample<D, 256, true>) : launch(k_sample<D, 256, false>);
    else cuts ? launch(k_sample<D, 1024, true>) : launch(k_sample<D, 1024, false>);
}

template <int D>
void launch_distill(const rlsim_head* h, const DistillArgs& a)
{
    if (a.V <= kHeadTinyVocab) {
        HEAD_TINY(k_distill_few, k_distill_tiny, D, h, a);
        return;
    }
    const uint32_t shared_by = a.rows <= h->split_rows ? distill_chunks(a.rows, a.V, Elem<D>::kBytes, h->cus) : 1u;
    if (shared_by > 1u && a.rows * shared_by <= kDistillSplitGroups) {
        DistillSplit p = distill_split(h);
        const uint32_t strip = 64u * Elem<D>::kPerVec, strips = (a.V + strip - 1u) / strip;
        p.chunk = (strips + shared_by - 1u) / shared_by * strip;
        p.chunks = (a.V + p.chunk - 1u) / p.chunk;
        const dim3 grid(p.chunks, a.rows), block(kDistillSplitThreads);
        hipLaunchKernelGGL(k_distill_chunk<D>, grid, block, p.chunk / 8u + 8u * a.k, h->stream, a, p);
        hipLaunchKernelGGL(k_distill_join<D>, a.grad ? grid : dim3(1, a.rows), block, 12u * a.k, h->stream, a, p);
        return;
    }
    const HeadForm form = distill_form(a.rows, a.V, Elem<D>::kBytes, a.grad != nullptr, h->cus);
    const uint32_t grid = head_grid(a.rows);
    const uint32_t shared = distill_shared_bytes(a.k, a.V);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(form.threads), shared, h->stream, a); };
    if (form.threads == 64u && form.strips == 2u) launch(k_distill<D, 64, 2>);
    else if (form.threads == 64u) launch(k_distill<D, 64, 4>);
    else if (form.strips == 4u) launch(k_distill<D, 256, 4>);
    else if (form.strips == 8u) launch(k_distill<D, 256, 8>);
    else if (form.threads == 256u) launch(k_distill<D, 256, 0>);
    else launch(k_distill<D, 512, 0>);
}

// A kernel may use more than 64 KB of dynamic shared memory only once it is told so.
template <int D>
hipError_t allow_shared()
{
    const int bytes = (int)distill_shared_bytes(kHeadMaxTeacher, kHeadMaxVocab);
    const void* const kernels[] = {reinterpret_cast<const void*>(k_distill<D, 512, 0>),
                                   reinterpret_cast<const void*>(k_distill<D, 256, 0>),
                                   reinterpret_cast<const void*>(k_distill_chunk<D>)};
    hipError_t e = hipSuccess;
    for (const void* k : kernels)
        if (e == hipSuccess) e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    return e;
}

// The bytes that `rows` rows of `row` bytes take, `stride` bytes apart.
struct Span { uintptr_t first, last; };
Span span(const void* p, uint32_t rows, uint64_t stride, uint64_t row)
{
    return {(uintptr_t)p, (uintptr_t)p + (uint64_t)(rows - 1u) * stride + row};
}
bool overlap(Span a, Span b) { return a.first < b.last && b.first < a.last; }

}  // namespace

extern "C" {

int rlsim_head_create(uint32_t max_rows, uint32_t max_vocab, void* stream, rlsim_head_t** out)
{
    if (!out) return head_fail(nullptr, RLSIM_EINVAL, "rlsim_head_create: out is NULL");
    *out = nullptr;
    if (max_rows == 0u || max_rows > 1u << 30)
        return head_fail(nullptr, RLSIM_EINVAL, "rlsim_head_create: max_rows must be in [1, 2^30]");
    if (max_vocab == 0u || max_vocab > kHeadMaxVocab)
        return head_fail(nullptr, RLSIM_EINVAL, "rlsim_head_create: max_vocab must be in [1, 2^20]");
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    int cus = 0;
    if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device);
    if (e == hipSuccess) e = allow_shared<kHeadF32>();
    if (e == hipSuccess) e = allow_shared<kHeadBF16>();
    if (e == hipSuccess) e = allow_shared<kHeadF16>();
    if (e != hipSuccess) return head_fail(nullptr, RLSIM_EDEVICE, "rlsim_head_create: %s", hipGetErrorString(e));
    rlsim_head* h = new (std::nothrow) rlsim_head;
    if (!h) return head_fail(nullptr, RLSIM_ENOMEM, "rlsim_head_create: host allocation failed");
    // rows too short to be shared need no workspace (fp32 distillation shares the shortest)
    h->split_rows = distill_chunks(1u, max_vocab, 4u, 256u) > 1u ? std::min(max_rows, kSplitGroups / 2u) : 0u;
    if (h->split_rows) e = hipMalloc(reinterpret_cast<void**>(&h->work), split_bytes(h->split_rows));
    if (e != hipSuccess) {
        const int code = e == hipErrorOutOfMemory ? RLSIM_ENOMEM : RLSIM_EDEVICE;
        if (h->work) (void)hipFree(h->work);
        delete h;
        (void)hipGetLastError();
        return head_fail(nullptr, code, "rlsim_head_create: %s", hipGetErrorString(e));
    }
    h->max_rows = max_rows;
    h->max_vocab = max_vocab;
    h->device = device;
    h->cus = (uint32_t)std::max(cus, 1);
    h->stream = static_cast<hipStream_t>(stream);
    *out = h;
    return RLSIM_OK;
}

int rlsim_head_sample(rlsim_head_t* h, const rlsim_sample* s)
{
    if (!h) return head_fail(nullptr, RLSIM_EINVAL, "rlsim_head_sample: handle is NULL");
    if (!s) return head_fail(h, RLSIM_EINVAL, "rlsim_head_sample: arguments are NULL");
    if (const char* what = check_rows(h, s->dtype, s->logits, s->rows, s->vocab, s->row_stride))
        return head_fail(h, RLSIM_EINVAL, "rlsim_head_sample: %s", what);
    if (!s->u || !s->token) return head_fail(h, RLSIM_EINVAL, "rlsim_head_sample: u or token is NULL");
    const void* words[] = {s->u, s->token, s->logp, s->temperature_rows, s->top_k_rows, s->top_p_rows, s->min_p_rows};
    for (const void* p : words)
        if (!aligned(p, 4u)) return head_fail(h, RLSIM_EINVAL, "rlsim_head_sample: a 32-bit array is not 4-byte aligned");
    if (!s->temperature_rows && !(std::isfinite(s->temperature) && s->temperature >= 0.0f))
        return head_fail(h, RLSIM_EINVAL, "rlsim_head_sample: temperature must be finite and >= 0");
    if (!s->top_p_rows && !(s->top_p >= 0.0f)) return head_fail(h, RLSIM_EINVAL, "rlsim_head_sample: top_p must be >= 0");
    if (!s->min_p_rows && !(s->min_p >= 0.0f)) return head_fail(h, RLSIM_EINVAL, "rlsim_head_sample: min_p must be >= 0");
    HeadDevice g(h->device);
    if (!g.ok) return head_fail(h, RLSIM_EDEVICE, "rlsim_head_sample: cannot select the handle's device");
    SampleArgs a{};
    a.logits = s->logits;
    a.stride = s->row_stride;
    a.rows = s->rows;
    a.V = s->vocab;
    a.T = s->temperature;
    a.top_p = s->top_p;
    a.min_p = s->min_p;
    a.top_k = s->top_k;
    a.T_rows = s->temperature_rows;
    a.top_k_rows = s->top_k_rows;
    a.top_p_rows = s->top_p_rows;
    a.min_p_rows = s->min_p_rows;
    a.u = s->u;
    a.token = s->token;
    a.logp = s->logp;
    if (s->dtype == RLSIM_F32) launch_sample<kHeadF32>(h, a);
    else if (s->dtype == RLSIM_BF16) launch_sample<kHeadBF16>(h, a);
    else launch_sample<kHeadF16>(h, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return head_fail(h, RLSIM_EDEVICE, "rlsim_head_sample: launch: %s", hipGetErrorString(e));
    return RLSIM_OK;
}

int rlsim_head_distill(rlsim_head_t* h, const rlsim_distill* d)
{
    if (!h) return head_fail(nullptr, RLSIM_EINVAL, "rlsim_head_distill: handle is NULL");
    if (!d) return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: arguments are NULL");
    if (const char* what = check_rows(h, d->dtype, d->logits, d->rows, d->vocab, d->row_stride))
        return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: %s", what);
    if (d->k == 0u || d->k > kHeadMaxTeacher)
        return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: k must be in [1, %u]", kHeadMaxTeacher);
    if (!known_dtype(d->teacher_dtype)) return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: unknown teacher_dtype");
    if (d->index_bytes != 4 && d->index_bytes != 8)
        return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: index_bytes must be 4 or 8");
    if (!d->teacher || !d->index) return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: teacher or index is NULL");
    if (!aligned(d->teacher, dtype_bytes(d->teacher_dtype)) || !aligned(d->index, (uint32_t)d->index_bytes))
        return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: teacher or index is not aligned to its element size");
    if (d->teacher_stride < d->k || d->index_stride < d->k || d->teacher_stride > kMaxStride || d->index_stride > kMaxStride)
        return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: teacher and index strides must be in [k, 2^32]");
    // 1 / temperature and its product with log2(e) have to be finite and not 0
    if (!(d->temperature >= 0x1.0p-60f && d->temperature <= 0x1.0p60f))
        return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: temperature must be in [2^-60, 2^60]");
    const void* words[] = {d->rest, d->weight, d->loss};
    for (const void* p : words)
        if (!aligned(p, 4u)) return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: a float array is not 4-byte aligned");
    if (!d->loss && !d->grad) return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: neither loss nor grad is wanted");
    if (d->grad) {
        const uint32_t bytes = dtype_bytes(d->dtype);
        if (!aligned(d->grad, bytes)) return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: grad is not aligned to its element size");
        if (d->grad_stride < d->vocab || d->grad_stride > kMaxStride)
            return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: grad_stride must be in [vocab, 2^32]");
        const bool in_place = d->grad == d->logits && d->grad_stride == d->row_stride;
        const Span g = span(d->grad, d->rows, d->grad_stride * bytes, (uint64_t)d->vocab * bytes);
        const Span l = span(d->logits, d->rows, d->row_stride * bytes, (uint64_t)d->vocab * bytes);
        if (!in_place && overlap(g, l))
            return head_fail(h, RLSIM_EINVAL, "rlsim_head_distill: grad overlaps logits without being the same rows");
    }
    HeadDevice g(h->device);
    if (!g.ok) return head_fail(h, RLSIM_EDEVICE, "rlsim_head_distill: cannot select the handle's device");
    DistillArgs a{};
    a.logits = d->logits;
    a.stride = d->row_stride;
    a.rows = d->rows;
    a.V = d->vocab;
    a.teacher = d->teacher;
    a.teacher_stride = d->teacher_stride;
    a.teacher_dtype = d->teacher_dtype;
    a.index = d->index;
    a.index_stride = d->index_stride;
    a.index64 = d->index_bytes == 8 ? 1u : 0u;
    a.k = d->k;
    a.tau = d->temperature;
    a.inv_tau = 1.0 / (double)d->temperature;
    a.scale = (float)(1.4426950408889634 / (double)d->temperature);
    a.rest = d->rest;
    a.weight = d->weight;
    a.loss = d->loss;
    a.grad = d->grad;
    a.grad_stride = d->grad_stride;
    a.past_cache = d->grad && (uint64_t)d->rows * d->vocab * dtype_bytes(d->dtype) > kLastLevelBytes ? 1u : 0u;
    if (d->dtype == RLSIM_F32) launch_distill<kHeadF32>(h, a);
    else if (d->dtype == RLSIM_BF16) launch_distill<kHeadBF16>(h, a);
    else launch_distill<kHeadF16>(h, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return head_fail(h, RLSIM_EDEVICE, "rlsim_head_distill: launch: %s", hipGetErrorString(e));
    return RLSIM_OK;
}

int rlsim_head_destroy(rlsim_head_t* h)
{
    if (!h) return RLSIM_OK;
    int rc = RLSIM_OK;
    {
        HeadDevice g(h->device);
        if (hipStreamSynchronize(h->stream) != hipSuccess) rc = RLSIM_EDEVICE;
        if (h->work) (void)hipFree(h->work);
    }
    delete h;
    return rc;
}

const char* rlsim_head_last_error(const rlsim_head_t* h) { return h ? h->err : g_head_err; }

}  // extern "C"
