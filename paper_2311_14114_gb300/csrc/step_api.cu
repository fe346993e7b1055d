// C-ABI entry points of a step over packed prompts and new tokens: argument
// validation on the host, and the kernels' launches.
#include <cmath>

#include "step_internal.h"

using namespace soniq;

namespace {

bool aligned_to(const void* p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

soniq_status launched(cudaError_t e) {
    return e == cudaSuccess ? SONIQ_OK : (e == cudaErrorNotSupported ? SONIQ_ERR_UNSUPPORTED : SONIQ_ERR_CUDA);
}

constexpr int64_t kMaxTokens = (int64_t)1 << 31;
constexpr int32_t kMaxHeads = 4096, kMaxChannels = 256;

soniq_status check_heads(const soniq_heads* h, RotateSide* s) {
    *s = RotateSide{};
    if (h == nullptr || h->heads == 0) return SONIQ_OK;
    if (h->heads < 0 || h->in == nullptr || h->out == nullptr) return SONIQ_ERR_INVALID_ARG;
    if (h->heads > kMaxHeads) return SONIQ_ERR_UNSUPPORTED;
    if (!aligned_to(h->in, 2) || !aligned_to(h->out, 2) || !aligned_to(h->gain, 4)) return SONIQ_ERR_ALIGNMENT;
    // A lone head's stride is any number, but lanes without a row form addresses with it, and a copy of no bytes needs an
    // aligned one too: 0.
    const bool one = h->heads == 1;
    *s = RotateSide{static_cast<const uint16_t*>(h->in), h->in_token_stride, one ? 0 : h->in_head_stride,
                    static_cast<uint16_t*>(h->out), h->out_token_stride, one ? 0 : h->out_head_stride, h->gain, h->heads};
    return SONIQ_OK;
}

}  // namespace

extern "C" {

soniq_status soniq_kv_plan(int32_t page_size, int64_t n_pages, int32_t* table, int64_t table_stride, int32_t max_pages,
                           int32_t* free_pages, int32_t* count, int32_t* count_out, const int32_t* lengths,
                           const int32_t* targets, int32_t B, int32_t max_tokens, int32_t* starts, int32_t* positions,
                           int64_t* slots, int32_t* lengths_out, soniq_stream_t stream) {
    if (page_size < 1 || (page_size & (page_size - 1)) != 0 || n_pages < 1 || max_pages < 0 || B < 0 || max_tokens < 0)
        return SONIQ_ERR_INVALID_ARG;
    if (page_size < 16 || page_size > 256 || n_pages > 2147483647 || B > kPlanMaxSequences ||
        (int64_t)B * max_pages > 2147483647)
        return SONIQ_ERR_UNSUPPORTED;
    if (count == nullptr || count_out == nullptr || free_pages == nullptr || starts == nullptr)
        return SONIQ_ERR_INVALID_ARG;
    if ((B > 0 && (lengths == nullptr || targets == nullptr || lengths_out == nullptr || (max_pages > 0 && table == nullptr))) ||
        (max_tokens > 0 && (positions == nullptr || slots == nullptr)))
        return SONIQ_ERR_INVALID_ARG;
    for (const void* p : {(const void*)table, (const void*)free_pages, (const void*)count, (const void*)count_out,
                          (const void*)lengths, (const void*)targets, (const void*)starts, (const void*)positions,
                          (const void*)lengths_out})
        if (!aligned_to(p, 4)) return SONIQ_ERR_ALIGNMENT;
    if (!aligned_to(slots, 8)) return SONIQ_ERR_ALIGNMENT;
    unsigned* err = device_error_word();
    if (err == nullptr) return SONIQ_ERR_CUDA;
    int shift = 0;
    while ((1 << shift) < page_size) ++shift;
    const KvPlanArgs a{table, table_stride, max_pages, shift, (int32_t)n_pages, free_pages, count, count_out, lengths,
                       targets, B, max_tokens, starts, positions, slots, lengths_out, err};
    return launched(launch_kv_plan(a, reinterpret_cast<cudaStream_t>(stream)));
}

soniq_status soniq_rotate_heads(const soniq_rotary* rotary, const int32_t* positions, int64_t n, int32_t D,
                                int32_t dtype, const soniq_heads* q, const soniq_heads* k, float eps,
                                soniq_stream_t stream) {
    if (n < 0 || D < 1 || (dtype != SONIQ_OUT_F16 && dtype != SONIQ_OUT_BF16) || !std::isfinite(eps) || eps < 0.0f)
        return SONIQ_ERR_INVALID_ARG;
    const int32_t channels = rotary != nullptr ? rotary->channels : 0;
    if (channels < 0 || channels % 2 != 0 || channels > D) return SONIQ_ERR_INVALID_ARG;
    if (channels > 0 && !std::isfinite(rotary->magnitude)) return SONIQ_ERR_INVALID_ARG;
    if (D > kMaxChannels || n > kMaxTokens) return SONIQ_ERR_UNSUPPORTED;
    RotateArgs a{};
    soniq_status st = check_heads(q, &a.side[0]);
    if (st == SONIQ_OK) st = check_heads(k, &a.side[1]);
    if (st != SONIQ_OK) return st;
    if (n == 0 || a.side[0].heads + a.side[1].heads == 0) return SONIQ_OK;
    if (channels > 0) {
        if (rotary->turns == nullptr || positions == nullptr) return SONIQ_ERR_INVALID_ARG;
        if (!aligned_to(rotary->turns, 8) || !aligned_to(positions, 4)) return SONIQ_ERR_ALIGNMENT;
        a.positions = positions;
        a.turns = rotary->turns;
        a.channels = channels;
        a.interleaved = rotary->interleaved != 0;
        a.magnitude = rotary->magnitude;
    }
    a.n = n;
    a.D = D;
    a.eps = eps;
    a.inverse_D = 1.0f / (float)D;
    return launched(launch_rotate_heads(a, dtype == SONIQ_OUT_BF16, reinterpret_cast<cudaStream_t>(stream)));
}

soniq_status soniq_prompt_attend(const void* Q, int64_t q_token_stride, int64_t q_head_stride, const void* K,
                                 int64_t k_token_stride, int64_t k_head_stride, const void* V, int64_t v_token_stride,
                                 int64_t v_head_stride, const int32_t* starts, int32_t B, int64_t n, int32_t q_heads,
                                 int32_t k_heads, int32_t D, int32_t Dv, int32_t dtype, int32_t causal, float scale,
                                 void* out, void* scratch, size_t scratch_bytes, soniq_stream_t stream) {
    if (B < 0 || n < 0 || q_heads < 1 || k_heads < 1 || q_heads % k_heads != 0 || D < 1 || Dv < 1 ||
        (dtype != SONIQ_OUT_F16 && dtype != SONIQ_OUT_BF16) || !std::isfinite(scale) || scale < 0.0f)
        return SONIQ_ERR_INVALID_ARG;
    if (D > kMaxChannels || Dv > kMaxChannels || q_heads > kMaxHeads || n > kMaxTokens / 2) return SONIQ_ERR_UNSUPPORTED;
    if (B == 0 || n == 0) return SONIQ_OK;
    if (Q == nullptr || K == nullptr || V == nullptr || starts == nullptr || out == nullptr) return SONIQ_ERR_INVALID_ARG;
    if (!aligned_to(Q, 2) || !aligned_to(K, 2) || !aligned_to(V, 2) || !aligned_to(out, 2) || !aligned_to(starts, 4))
        return SONIQ_ERR_ALIGNMENT;
    if (scratch == nullptr || (int64_t)scratch_bytes < kPromptScratchBytes) return SONIQ_ERR_INVALID_ARG;
    if (!aligned_to(scratch, 16)) return SONIQ_ERR_ALIGNMENT;
    unsigned* err = device_error_word();
    if (err == nullptr) return SONIQ_ERR_CUDA;
    const PromptArgs a{{static_cast<const uint16_t*>(Q), q_token_stride, q_head_stride},
                       {static_cast<const uint16_t*>(K), k_token_stride, k_head_stride},
                       {static_cast<const uint16_t*>(V), v_token_stride, v_head_stride},
                       starts, B, (int32_t)n, k_heads, q_heads / k_heads, D, Dv, causal != 0, scale,
                       static_cast<uint16_t*>(out), err};
    const bool bf16 = dtype == SONIQ_OUT_BF16;
    const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (!prompt_tile_supported(a)) return launched(launch_prompt_rows(a, bf16, st));
    return launched(launch_prompt_tile(a, bf16, static_cast<unsigned*>(scratch), st));
}

int64_t soniq_prompt_attend_scratch_bytes(void) { return kPromptScratchBytes; }

}  // extern "C"
