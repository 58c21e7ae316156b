// learn_host_checks.hip -- the learner's argument checks on the CPU: its host code is
// compiled in, so that calls that have to be refused can be made on a handle that no device
// made (tests/test_learn_sanitized.py builds this with AddressSanitizer and
// UndefinedBehaviorSanitizer on the host).  Every call here fails before any device work.
#include "../../paper_2207_07736_amd/csrc/learn.hip"

static int failures = 0;

#define EXPECT(cond)                                                          \
    do {                                                                      \
        if (!(cond)) {                                                        \
            fprintf(stderr, "line %d: %s\n", __LINE__, #cond);                \
            ++failures;                                                       \
        }                                                                     \
    } while (0)

// rc is EINVAL, and the handle's message names `part`.
static void refused(const rlsim_learner* h, int rc, const char* part, int line)
{
    const char* m = rlsim_learner_last_error(h);
    if (rc != RLSIM_EINVAL || !strstr(m, part)) {
        fprintf(stderr, "line %d: status %d, \"%s\" does not say \"%s\"\n", line, rc, m, part);
        ++failures;
    }
}
#define REFUSED(call, part) refused(&h, call, part, __LINE__)

static float f[1 << 16];                          // memory that nothing reads: only its addresses count
static uint8_t bytes[1 << 12];

int main()
{
    rlsim_learner_t* none = (rlsim_learner_t*)0x1;
    EXPECT(rlsim_learner_create(1, 1, 1, nullptr, nullptr) == RLSIM_EINVAL);
    const uint32_t sizes[][3] = {{0, 1, 1}, {1, 0, 1}, {1, 1, 0}, {0, 0, 1}, {(1u << 22) + 1u, 1, 1}, {1, (1u << 16) + 1u, 1},
                                 {1, 1, (1u << 20) + 1u}, {~0u, ~0u, ~0u}};
    for (const auto& s : sizes) {
        none = (rlsim_learner_t*)0x1;
        EXPECT(rlsim_learner_create(s[0], s[1], s[2], nullptr, &none) == RLSIM_EINVAL && none == nullptr);
        EXPECT(strlen(rlsim_learner_last_error(nullptr)) > 0);
    }
    EXPECT(rlsim_learner_destroy(nullptr) == RLSIM_OK);

    rlsim_learner h;
    h.max_rows = 64;
    h.max_dim = 32;
    h.max_vocab = 128;
    h.xent_at = 0;
    h.bytes = xent_bound(64, 32, 128, 2u);

    // ---- the recurrence
    EXPECT(rlsim_learner_scan(nullptr, nullptr) == RLSIM_EINVAL);
    REFUSED(rlsim_learner_scan(&h, nullptr), "NULL");
    rlsim_scan s{};
    s.dtype = RLSIM_F32;
    s.T = 20;
    s.n = 3;
    s.channels = 5;
    s.x = f;
    s.gate = f + 1000;
    s.y = f + 2000;
    s.x_step = s.gate_step = s.y_step = 15;
    s.x_seq = s.gate_seq = s.y_seq = 5;
    s.last = f + 3000;
    s.state = f + 4000;
    s.marks = f + 5000;
    s.done = bytes;
    auto scan = [&](auto change, const char* part, int line) {
        rlsim_scan c = s;
        change(c);
        refused(&h, rlsim_learner_scan(&h, &c), part, line);
    };
#define SCAN(body, part) scan([&](rlsim_scan& c) { body; }, part, __LINE__)
    SCAN(c.x = nullptr, "NULL");
    SCAN(c.gate = nullptr, "NULL");
    SCAN(c.y = nullptr, "NULL");
    SCAN(c.dtype = 7, "dtype");
    SCAN(c.T = 0, "[1, 2^30]");
    SCAN(c.n = 0, "[1, 2^30]");
    SCAN(c.channels = 0, "[1, 2^30]");
    SCAN(c.T = ~0u, "[1, 2^30]");
    SCAN(c.n = (1u << 30) + 1u, "[1, 2^30]");
    SCAN(c.channels = ~0u, "[1, 2^30]");
    SCAN((c.T = 1u << 30, c.n = 1u << 30, c.channels = 1), "2^40");
    SCAN((c.T = 1u << 30, c.n = 1u << 30, c.channels = 1u << 30), "2^40");
    SCAN(c.x = (const char*)f + 2, "aligned");
    SCAN((c.dtype = RLSIM_BF16, c.gate = (const char*)f + 1), "aligned");
    SCAN(c.state = (const float*)((const char*)f + 2), "aligned");
    SCAN(c.marks = (float*)((char*)f + 1), "aligned");
    SCAN(c.x_step = (1ull << 40) + 1u, "stride");
    SCAN(c.gate_seq = ~0ull, "stride");
    SCAN(c.y_step = 14, "overlap");
    SCAN(c.y_seq = 4, "overlap");
    SCAN((c.y_step = 5, c.y_seq = 99), "overlap");
    SCAN((c.y_step = 5, c.y_seq = 5), "overlap");
    SCAN((c.y_step = 0, c.y_seq = 100), "overlap");
    SCAN(c.y = f, "overlaps");
    SCAN(c.y = f + 299, "overlaps");
    SCAN(c.y = f + 1000 - 299, "overlaps");
    SCAN(c.last = f + 2000, "overlaps");
    SCAN(c.last = f + 4001, "overlaps");
    SCAN(c.marks = f + 3014, "overlaps");
    SCAN(c.state = f + 2010, "overlaps");
    SCAN(c.done = (const uint8_t*)(f + 2299) + 3, "overlaps");
    SCAN((c.dtype = RLSIM_F16, c.y = (char*)f + 2), "overlaps");

    // ---- its gradient
    rlsim_scan_grad g{};
    g.dy = f + 6000;
    g.dx = f + 7000;
    g.dgate = f + 8000;
    g.dy_step = g.dx_step = g.dgate_step = 15;
    g.dy_seq = g.dx_seq = g.dgate_seq = 5;
    g.dlast = f + 9000;
    g.dstate = f + 10000;
    EXPECT(rlsim_learner_scan_grad(nullptr, &s, &g) == RLSIM_EINVAL);
    REFUSED(rlsim_learner_scan_grad(&h, nullptr, &g), "NULL");
    REFUSED(rlsim_learner_scan_grad(&h, &s, nullptr), "NULL");
    auto back = [&](auto change, const char* part, int line) {
        rlsim_scan a = s;
        rlsim_scan_grad c = g;
        change(a, c);
        refused(&h, rlsim_learner_scan_grad(&h, &a, &c), part, line);
    };
#define BACK(body, part) back([&](rlsim_scan& a, rlsim_scan_grad& c) { (void)a; (void)c; body; }, part, __LINE__)
    BACK(a.marks = nullptr, "NULL");
    BACK(c.dx = nullptr, "NULL");
    BACK(c.dgate = nullptr, "NULL");
    BACK(c.dy = (const char*)f + 2, "aligned");
    BACK(c.dstate = (float*)((char*)f + 2), "aligned");
    BACK(c.dx_step = 3, "overlap");
    BACK(c.dx = c.dgate, "overlaps");
    BACK(c.dx = const_cast<void*>(a.x), "overlaps");
    BACK(c.dgate = const_cast<void*>(c.dy), "overlaps");
    BACK(c.dstate = a.marks + 3, "overlaps");
    BACK(c.dstate = const_cast<float*>(c.dlast) + 1, "overlaps");
    BACK(c.dy_step = (1ull << 40) + 1u, "stride");

    // ---- the cross entropy
    rlsim_xent x{};
    x.dtype = RLSIM_F32;
    x.rows = 8;
    x.dim = 16;
    x.vocab = 100;
    x.hidden = f;
    x.matrix = f + 1000;
    x.hidden_stride = x.matrix_stride = x.dhidden_stride = x.dmatrix_stride = 16;
    x.target_bytes = 4;
    x.target = f + 5000;
    x.weight = f + 5100;
    x.loss = f + 5200;
    x.stats = f + 5300;
    x.dhidden = f + 6000;
    x.dmatrix = f + 8000;
    EXPECT(rlsim_learner_xent(nullptr, &x) == RLSIM_EINVAL);
    REFUSED(rlsim_learner_xent(&h, nullptr), "NULL");
    auto xent = [&](auto change, const char* part, int line) {
        rlsim_xent c = x;
        change(c);
        refused(&h, rlsim_learner_xent(&h, &c), part, line);
    };
#define XENT(body, part) xent([&](rlsim_xent& c) { body; }, part, __LINE__)
    XENT(c.dtype = -1, "dtype");
    XENT(c.rows = 0, "rows");
    XENT(c.rows = 65, "rows");
    XENT(c.dim = 0, "dim");
    XENT(c.dim = 33, "dim");
    XENT(c.vocab = 0, "vocab");
    XENT(c.vocab = 129, "vocab");
    XENT(c.hidden = nullptr, "NULL");
    XENT(c.matrix = nullptr, "NULL");
    XENT(c.target = nullptr, "NULL");
    XENT(c.target_bytes = 2, "target_bytes");
    XENT((c.loss = nullptr, c.dhidden = nullptr, c.dmatrix = nullptr), "nothing");
    XENT((c.loss = nullptr, c.stats = nullptr), "stats");
    XENT(c.hidden_stride = 15, "stride");
    XENT(c.matrix_stride = (1ull << 32) + 1u, "stride");
    XENT(c.dhidden_stride = 0, "stride");
    XENT(c.dmatrix_stride = ~0ull, "stride");
    XENT(c.hidden = (const char*)f + 1, "aligned");
    XENT((c.target_bytes = 8, c.target = f + 5001), "aligned");
    XENT(c.weight = (const float*)((const char*)f + 1), "aligned");
    XENT(c.stats = (float*)((char*)f + 5300 * 4 + 1), "aligned");
    XENT(c.dhidden = f, "overlaps");
    XENT(c.dmatrix = f + 1000, "overlaps");
    XENT(c.dmatrix = f + 6100, "overlaps");
    XENT(c.loss = f + 5107, "overlaps");
    XENT(c.stats = f + 5204, "overlaps");
    XENT((c.loss = nullptr, c.dhidden = f + 5300), "overlaps");
    {
        rlsim_learner bare;
        rlsim_xent c = x;
        refused(&bare, rlsim_learner_xent(&bare, &c), "without an output layer", __LINE__);
    }

    // ---- clipping
    rlsim_tensor t[4] = {};
    for (int i = 0; i < 4; ++i) t[i] = {f + 1000 * i, nullptr, 500, RLSIM_F32, RLSIM_F32};
    float* const norm = f + 60000;
    EXPECT(rlsim_learner_clip(nullptr, t, 4, 1.0, norm) == RLSIM_EINVAL);
    REFUSED(rlsim_learner_clip(&h, t, 4, 1.0, nullptr), "NULL");
    REFUSED(rlsim_learner_clip(&h, nullptr, 4, 1.0, norm), "NULL");
    REFUSED(rlsim_learner_clip(&h, t, (1u << 20) + 1u, 1.0, norm), "count");
    for (double bad : {0.0, -1.0, (double)NAN, (double)-INFINITY}) REFUSED(rlsim_learner_clip(&h, t, 4, bad, norm), "max_norm");
    REFUSED(rlsim_learner_clip(&h, t, 4, 1.0, (float*)((char*)norm + 1)), "aligned");
    auto clip = [&](auto change, const char* part, int line) {
        rlsim_tensor c[4];
        memcpy(c, t, sizeof c);
        change(c);
        refused(&h, rlsim_learner_clip(&h, c, 4, 1.0, norm), part, line);
    };
#define CLIP(body, part) clip([&](rlsim_tensor* c) { body; }, part, __LINE__)
    CLIP(c[1].dtype = 3, "dtype");
    CLIP((c[1].out = f + 20000, c[1].out_dtype = -2), "out_dtype");
    CLIP(c[2].data = nullptr, "NULL");
    CLIP(c[2].elements = (1ull << 40) + 1u, "2^40");
    CLIP((c[2].elements = 1ull << 40, c[3].elements = 1ull << 40), "2^40");
    CLIP(c[0].data = (const char*)f + 2, "aligned");
    CLIP((c[0].out = (char*)f + 80002, c[0].out_dtype = RLSIM_F32), "aligned");
    CLIP((c[0].out = f, c[0].out_dtype = RLSIM_BF16), "another type");
    CLIP(c[3].data = c[0].data, "overlaps");
    CLIP(c[3].data = f + 499, "overlaps");
    CLIP(c[0].out = f + 1, "overlaps");
    CLIP(c[0].out = f + 2400, "overlaps");
    CLIP((c[0].out = f + 20000, c[1].out = f + 20499), "overlaps");
    CLIP(c[0].data = norm, "overlaps");
    // an output inside a long tensor that lies between
    CLIP((c[0].elements = 50000, c[1].data = f + 51000, c[2].data = f + 52000, c[3].data = f + 53000, c[3].out = f + 40000), "overlaps");
    CLIP((c[0].elements = 0, c[0].data = nullptr, c[1].data = f + 2000), "overlaps");

    if (failures) {
        fprintf(stderr, "%d failures\n", failures);
        return 1;
    }
    printf("learn host checks: OK\n");
    return 0;
}
