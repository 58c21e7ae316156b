"""The sizes of tests/test_gpu_learn_forms.py choose the forms that they are meant for, on the 256
CUs of this part, as a host program compiled from learn_dispatch.h says."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2207_07736_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "learn_dispatch.h"
using namespace rlsim_dev;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
constexpr uint32_t kCus = 256u;
static uint32_t segments(uint32_t T, uint32_t n, uint32_t channels, uint32_t per)
{
    const uint32_t groups = channels < 2u ? channels : (channels + 1u) / 2u;
    return scan_cut((uint64_t)n * groups, (uint64_t)n * channels, T, kCus, per).segments;
}
int main()
{
    // sequences 2^32 bytes apart: one piece and cut
    for (uint32_t channels : {1u, 33u, 64u})
        for (uint32_t per : {2u, 3u, 4u})
            CHECK(segments(1u, 2u, channels, per) == 1u && segments(40u, 2u, channels, per) == 1u && segments(130u, 2u, channels, per) == 3u);
    // 16-bit factors: 256 x 256 for every product, two pieces, long sums
    {
        const uint32_t rows = 4096u, dim = 4096u, vocab = 8492u;
        const XentShape s = xent_shape(rows, dim, vocab, 1u);
        CHECK(s.piece == 8192u);
        CHECK(xent_tile(vocab, rows, s.dim_k / kXentK, false, kCus).m == 256u);
        CHECK(xent_tile(s.piece, rows, s.dim_k / kXentK, false, kCus).m == 256u);
        const XentTile x = xent_tile(dim, rows, s.piece / kXentK, true, kCus), w = xent_tile(dim, s.piece, s.rows_k / kXentK, true, kCus);
        CHECK(x.m == 256u && x.share == 1u && w.m == 256u && w.share == 1u);
        CHECK(s.piece / kXentK >= 16u && s.rows_k / kXentK >= 16u);
        const XentTile rest = xent_tile(dim, vocab - s.piece, s.rows_k / kXentK, true, kCus);     // the last piece: shares
        CHECK(rest.m == 128u && rest.share > 1u);
    }
    // fp32: the same, three products each; and dmatrix alone in 256 x 256
    for (uint32_t rows : {4096u, 1024u}) {
        const uint32_t dim = 4096u, vocab = 4600u;
        const XentShape s = xent_shape(rows, dim, vocab, 2u);
        CHECK(s.piece == 4096u);
        const XentTile x = xent_tile(dim, rows, (uint64_t)s.piece / kXentK * 3u, true, kCus);
        const XentTile w = xent_tile(dim, s.piece, (uint64_t)s.rows_k / kXentK * 3u, true, kCus);
        CHECK(w.m == 256u && w.share == 1u && s.rows_k / kXentK >= 16u);
        CHECK((x.m == 256u) == (rows == 4096u));
    }
    // as many rows as a handle takes: 64 shares of dmatrix's sum
    {
        const XentShape s = xent_shape(1u << 22, 8u, 2u, 1u);
        CHECK(xent_tile(8u, 2u, s.rows_k / kXentK, true, kCus).share == 64u);
    }
    // clipping: more bytes than the last-level cache holds, and more blocks than one to a CU
    CHECK((150000001ull + clip_chunk(150000001ull) - 1u) / clip_chunk(150000001ull) > kCus);
    printf("learn forms: OK\n");
    return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_sizes_choose_their_forms(tmp_path):
    src = tmp_path / "check.cpp"
    src.write_text("#include <initializer_list>\n" + PROGRAM)
    exe = tmp_path / "check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0 and "OK" in res.stdout, res.stdout
