// head_dispatch.h -- which form of an output-head kernel a call runs, as functions
// of its sizes alone (plain C++).  All forms of the sampling kernel give the same draws.
#pragma once

#include <stdint.h>

namespace rlsim_dev {

// Rows of up to 64 entries: one thread to a row for up to 8, else one lane to an entry.
constexpr uint32_t kHeadTinyVocab = 64u;

// Threads to a row of the distillation kernel, and strips of 64 16-byte vectors that a wave
// of them holds in registers (0: the row is read again for the gradient), for rows
// of more entries.  Long rows take 256 threads, several workgroups to a CU, as long
// as the rows at work, some six to a CU, stay in the 256 MB last-level cache between their
// two reads; 512 threads, two to a CU, beyond.  256 / 512 / 1,024 threads, us, of one
// batch again and again (batches in turn, which the cache does not hold, take 70 instead of 55
// us at 1,024 rows and 84 instead of 71 at 600 x 100,000):
//   600 x 20,011 bf16        24 /   - /  35      4,000 x 50,001 bf16      260 /   - / 305
//   1,024 x 50,001 bf16      55 /   - /  73      2,000 x 50,001 f32       264 / 231 / 230
//   600 x 100,000 bf16       71 /   - /  75      2,048 x 131,072 bf16     345 / 287 / 305
//   losses alone: 600 x 50,001 f16 23 / - / 34, 2,048 x 131,072 bf16 113 / - / 137
// (1,024 threads, two to a CU, leave 64 registers a thread, which are too few.)
struct HeadForm { uint32_t threads, strips; };
inline HeadForm distill_form(uint32_t rows, uint32_t vocab, uint32_t elem_bytes, bool grad, uint32_t cus)
{
    const uint32_t vectors = vocab / (16u / elem_bytes);
    if (vectors <= 64u * 2u) return {64u, 2u};
    if (vectors <= 64u * 4u) return {64u, 4u};
    if (vectors <= 256u * 4u) return {256u, 4u};
    if (vectors <= 256u * 8u) return {256u, 8u};
    const uint64_t at_work = rows < 6u * cus ? rows : 6u * cus;
    return {!grad || at_work * vocab * elem_bytes <= 160000000ull ? 256u : 512u, 0u};
}

// Threads to a row of the sampling kernel, for rows of more entries than the tiny form's:
// one wave while a lane has at most four vectors, four up to eight a lane, then sixteen
// (256 / 1,024 threads, us: 512 x 151,001 bf16 100 / 85, with top-p 1,024 x 131,072
// 600 / 215: shorter lists and coarser bins send more rows through further passes).
inline uint32_t sample_threads(uint32_t vocab, uint32_t elem_bytes)
{
    const uint32_t vectors = vocab / (16u / elem_bytes);
    return vectors <= 64u * 4u ? 64u : vectors <= 256u * 8u ? 256u : 1024u;
}

// Workgroups that share a row of the sampling kernel (1: it has one of its own), for rows
// longer than the tiny form's: two to a CU over the call, and at least a vector to each of
// their 1,024 threads.  One to a row / shared, us: 1 x 131,072 bf16 with top-k and top-p
// 58 / 20, 64 x 50,001 of mixed settings 70 / 44, 256 x 32,000 fp32 with min-p 28 / 24.
inline uint32_t sample_chunks(uint32_t rows, uint32_t vocab, uint32_t elem_bytes, uint32_t cus)
{
    const uint32_t vectors = vocab / (16u / elem_bytes);
    const uint32_t by_rows = 2u * cus / rows, by_size = vectors / 1024u;
    const uint32_t chunks = by_rows < by_size ? by_rows : by_size;
    return chunks < 2u ? 1u : chunks < 32u ? chunks : 32u;
}

// The same for the distillation kernel, two vectors to each of 256 threads: 8 x 262,144 fp32
// 55 / 14 us.
inline uint32_t distill_chunks(uint32_t rows, uint32_t vocab, uint32_t elem_bytes, uint32_t cus)
{
    const uint32_t vectors = vocab / (16u / elem_bytes);
    const uint32_t by_rows = 2u * cus / rows, by_size = vectors / 512u;
    const uint32_t chunks = by_rows < by_size ? by_rows : by_size;
    return chunks < 2u ? 1u : chunks < 64u ? chunks : 64u;
}

}  // namespace rlsim_dev
