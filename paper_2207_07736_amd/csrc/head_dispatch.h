// head_dispatch.h -- which form of an output-head kernel a call runs, as functions
// of its sizes alone (plain C++).  All forms give the same draws.
#pragma once

#include <stdint.h>

namespace rlsim_dev {

// Rows of up to 64 entries: one thread to a row for up to 8, else one lane to an entry.
constexpr uint32_t kHeadTinyVocab = 64u;

// Threads to a row and strips of 64 16-byte vectors a wave of them holds in
// registers (0: the row is read again in each pass), for rows of more entries.
struct HeadForm { uint32_t threads, strips; };
inline HeadForm head_form(uint32_t vocab, uint32_t elem_bytes)
{
    const uint32_t vectors = vocab / (16u / elem_bytes);
    if (vectors <= 64u * 2u) return {64u, 2u};
    if (vectors <= 64u * 4u) return {64u, 4u};
    if (vectors <= 256u * 4u) return {256u, 4u};
    if (vectors <= 256u * 8u) return {256u, 8u};
    return {1024u, 0u};
}

// Threads to a row of the sampling kernel, for rows of more entries than the tiny form's.
inline uint32_t head_threads(uint32_t vocab, uint32_t elem_bytes)
{
    const uint32_t vectors = vocab / (16u / elem_bytes);
    return vectors <= 64u * 4u ? 64u : vectors <= 256u * 8u ? 256u : 1024u;
}

// Workgroups that share a row of the sampling kernel (1: it has one of its own), for rows
// longer than the tiny form's.
inline uint32_t sample_chunks(uint32_t rows, uint32_t vocab, uint32_t elem_bytes, uint32_t cus)
{
    const uint32_t vectors = vocab / (16u / elem_bytes);
    const uint32_t by_rows = 2u * cus / rows, by_size = vectors / 1024u;
    const uint32_t chunks = by_rows < by_size ? by_rows : by_size;
    return chunks < 2u ? 1u : chunks < 32u ? chunks : 32u;
}

// The same for the distillation kernel.
inline uint32_t distill_chunks(uint32_t rows, uint32_t vocab, uint32_t elem_bytes, uint32_t cus)
{
    const uint32_t vectors = vocab / (16u / elem_bytes);
    const uint32_t by_rows = 2u * cus / rows, by_size = vectors / 512u;
    const uint32_t chunks = by_rows < by_size ? by_rows : by_size;
    return chunks < 2u ? 1u : chunks < 64u ? chunks : 64u;
}

}  // namespace rlsim_dev
