"""The learner's sources on the CPU: how calls are cut and the workspace's bounds, as a host
program compiled from learn_dispatch.h says them."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2207_07736_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "learn_dispatch.h"
using namespace rlsim_dev;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
static uint64_t state = 1;
static uint32_t below(uint32_t n) { state = state * 6364136223846793005ull + 1442695040888963407ull; return (uint32_t)((state >> 33) % n); }
static uint32_t size_below(uint32_t n)          // spread over the logarithm
{
    uint32_t bits = 0;
    while ((n >> bits) > 1u) ++bits;
    const uint32_t v = below((2u << below(bits + 1u)));
    return v < 1u ? 1u : v > n ? n : v;
}
int main()
{
    for (int i = 0; i < 200000; ++i) {
        const uint32_t cus = i % 2 ? 256u : 64u;
        // segments cover the steps, start at marks, none is empty, and their maps fit
        const uint32_t T = size_below(1u << 20), channels = size_below(1u << 22);
        const ScanCut c = scan_cut((channels + 1u) / 2u, channels, T, cus, 2u + i % 3u);
        CHECK(c.segments >= 1u && c.segments <= kScanSegments && (uint64_t)c.segments * c.seg_len >= T);
        CHECK((uint64_t)(c.segments - 1u) * c.seg_len < T);
        CHECK(c.segments == 1u || (c.seg_len % kScanMark == 0u && (uint64_t)c.segments * channels <= kScanMapEntries));
        // blocks of tensors
        const uint64_t total = (uint64_t)size_below(1u << 30) * size_below(1u << 10);
        CHECK(total / clip_chunk(total) <= kClipBlocks);
        // a call within a handle's bounds fits its workspace
        const uint32_t rows = size_below(1u << 22), dim = size_below(1u << 16), vocab = size_below(1u << 20);
        for (uint32_t parts : {1u, 2u}) {
            const uint64_t bound = xent_bound(rows, dim, vocab, parts);
            const uint32_t r = 1u + below(rows), d = 1u + below(dim), v = 1u + below(vocab);
            for (const XentShape& s : {xent_shape(rows, dim, vocab, parts), xent_shape(r, d, v, parts), xent_shape(1, dim, vocab, parts),
                                       xent_shape(rows, 1, vocab, parts), xent_shape(rows, dim, 1, parts), xent_shape(1, 1, vocab, parts)}) {
                CHECK(s.piece % 256u == 0u && s.piece >= 256u && s.dim_k % kXentK == 0u && s.rows_k % kXentK == 0u);
                CHECK(xent_work(s).end <= bound);
            }
            const XentShape s = xent_shape(r, d, v, parts);
            const XentWork o = xent_work(s);
            // shares of both products fit
            const uint32_t rx = parts == 1u && r <= kXentStackRows ? 2u * kXentStackRows : r;      // rows of dhidden's sums
            const XentTile x = xent_tile(d, rx, (uint64_t)s.piece / kXentK * (parts == 1u ? 1u : 3u), true, cus);
            CHECK(x.share >= 1u && up_to(d, 4u) * 4u * rx * x.share <= o.dw - o.dx);
            const uint32_t count = s.piece < v ? s.piece : v;
            const XentTile w = xent_tile(d, count, (uint64_t)s.rows_k / kXentK * (parts == 1u ? 1u : 3u), true, cus);
            CHECK(w.share == 1u || up_to(d, 4u) * 4u * count * w.share <= o.end - o.dw);
            // parts of the softmax sums fit
            uint64_t all = 0;
            for (uint32_t v0 = 0; v0 < v; v0 += s.piece) {
                const uint32_t n = s.piece < v - v0 ? s.piece : v - v0;
                const XentTile t = xent_tile(n, r, s.dim_k / kXentK * (parts == 1u ? 1u : 3u), false, cus);
                CHECK(t.share == 1u && t.m % t.span == 0u);
                all += (n + t.m - 1u) / t.m * (t.m / t.span);
            }
            CHECK(8ull * all * s.rows_k <= o.up_n - o.part);
            all = 0;
            const uint32_t width = (uint32_t)(v < xent_width(s.rows_k) ? v : xent_width(s.rows_k));
            for (uint32_t v0 = 0; v0 < v; v0 += width) {
                const uint32_t n = width < v - v0 ? width : v - v0;
                const XentTile t = xent_tile(n, r, s.dim_k / kXentK * (parts == 1u ? 1u : 3u), false, cus);
                all += (n + t.m - 1u) / t.m * (t.m / t.span);
                // a launch holds fewer than 2^32 threads
                CHECK((uint64_t)((n + t.m - 1u) / t.m) * ((r + t.n - 1u) / t.n) * 512u < 1ull << 32);
            }
            CHECK(8ull * all * s.rows_k <= o.up_n - o.part);
        }
    }
    printf("learn dispatch: OK\n");
    return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_cuts_and_bounds(tmp_path):
    src = tmp_path / "check.cpp"
    src.write_text(PROGRAM)
    exe = tmp_path / "check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0 and "OK" in res.stdout, res.stdout
