// What the kernels of a step over packed prompts and new tokens take: the plan
// of its pages, the turning of its queries and keys, the prompts' attention.
#pragma once

#include "soniq_internal.h"

namespace soniq {

struct KvPlanArgs {
    int32_t* table;
    int64_t table_stride;
    int32_t max_pages;
    int32_t page_shift;
    int32_t n_pages;
    int32_t* free_pages;
    int32_t* count;            // [2]: pages in the pool, and a word that is zero between calls
    int32_t* count_out;
    const int32_t* lengths;
    const int32_t* targets;
    int32_t B;
    int32_t max_tokens;
    int32_t* starts;
    int32_t* positions;
    int64_t* slots;
    int32_t* lengths_out;
    unsigned* err;
};
constexpr int kPlanMaxSequences = 8192;
cudaError_t launch_kv_plan(const KvPlanArgs& a, cudaStream_t st);

struct RotateSide {
    const uint16_t* in;
    int64_t in_token, in_head;     // strides in elements
    uint16_t* out;
    int64_t out_token, out_head;
    const float* gain;             // [D] or null: no norm
    int32_t heads;
};
struct RotateArgs {
    RotateSide side[2];            // queries, keys
    const int32_t* positions;
    const uint64_t* turns;         // [channels / 2]
    int64_t n;
    int32_t D, channels, interleaved;
    float magnitude, eps, inverse_D;
};
cudaError_t launch_rotate_heads(const RotateArgs& a, bool bf16, cudaStream_t st);

struct PromptSide {
    const uint16_t* p;
    int64_t token, head;           // strides in elements
};
struct PromptArgs {
    PromptSide q, k, v;
    const int32_t* starts;
    int32_t B, n;
    int32_t k_heads, group;        // group: query heads per key head
    int32_t D, Dv;
    int32_t causal;
    float scale;
    uint16_t* out;
    unsigned* err;
};
// A warp to a row, of any kind; and tensor-core tiles, of rows on 16 bytes.  counters: two
// words that are zero between launches.
cudaError_t launch_prompt_rows(const PromptArgs& a, bool bf16, cudaStream_t st);
bool prompt_tile_supported(const PromptArgs& a);
cudaError_t launch_prompt_tile(const PromptArgs& a, bool bf16, unsigned* counters, cudaStream_t st);
constexpr int64_t kPromptScratchBytes = 256;

}  // namespace soniq
