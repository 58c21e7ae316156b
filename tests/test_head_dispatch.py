"""The output head's sources on the CPU: rules of the forms and the workspace's bounds, as a
host program compiled from head_dispatch.h says them."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2207_07736_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "head_dispatch.h"
using namespace rlsim_dev;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main()
{
    for (uint32_t bytes : {2u, 4u})
        for (uint32_t cus : {64u, 256u})
            for (uint32_t rows : {1u, 2u, 7u, 64u, 200u, 256u, 257u, 511u, 512u, 513u, 4096u, 1u << 20})
                for (uint32_t vocab = 65u; vocab <= 1u << 20; vocab += vocab / 7u + 1u) {
                    const uint32_t strip = 64u * 16u / bytes, vectors = vocab / (16u / bytes);
                    uint32_t c = sample_chunks(rows, vocab, bytes, cus);
                    CHECK(c >= 1u && c <= 32u && (c == 1u || rows * c <= 1024u));
                    c = distill_chunks(rows, vocab, bytes, cus);
                    CHECK(c >= 1u && c <= 64u && (c == 1u || rows * c <= 1024u));
                    // a chunk is whole strips, none is empty, and no more than asked for
                    const uint32_t strips = (vocab + strip - 1u) / strip, chunk = (strips + c - 1u) / c * strip;
                    CHECK((vocab + chunk - 1u) / chunk <= c);
                    const uint32_t threads = sample_threads(vocab, bytes);
                    CHECK(threads == 64u || threads == 256u || threads == 1024u);
                    for (bool grad : {false, true}) {
                        const HeadForm f = distill_form(rows, vocab, bytes, grad, cus);
                        CHECK(f.strips == 0u || f.threads * f.strips >= vectors);
                        CHECK(f.threads != 512u || grad);
                    }
                }
    // few long rows are shared, many are not
    CHECK(sample_chunks(1, 131072, 2, 256) == 16u && sample_chunks(512, 131072, 2, 256) == 1u);
    CHECK(distill_chunks(8, 262144, 4, 256) == 64u && distill_chunks(512, 262144, 4, 256) == 1u);
    CHECK(sample_chunks(1, 1000, 2, 256) == 1u && distill_chunks(1, 1000, 4, 256) == 1u);
    // 512 threads only where the rows at work pass the last-level cache
    CHECK(distill_form(2048, 131072, 2, true, 256).threads == 512u && distill_form(2048, 131072, 2, false, 256).threads == 256u);
    CHECK(distill_form(600, 100000, 2, true, 256).threads == 256u && distill_form(4000, 50001, 2, true, 256).threads == 256u);
    printf("head dispatch: OK\n");
    return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_forms_and_chunks(tmp_path):
    src = tmp_path / "check.cpp"
    src.write_text(PROGRAM)
    exe = tmp_path / "check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0 and "OK" in res.stdout, res.stdout
