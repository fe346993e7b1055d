// Attention of packed prompts, a warp to a row: for rows that are no 16-byte
// pieces.  Bound by the instructions of its products, eight channels to a lane: 2048 tokens x
// 8 heads of 50 channels take 1.2 ms, where prompt_tile_kernel would take 0.03.
#include "prompt_rows.cuh"

namespace soniq {

namespace {

constexpr int kThreads = 256;

template <bool BF16>
__global__ void __launch_bounds__(kThreads) prompt_rows_kernel(const PromptArgs a) {
    const int warps = gridDim.x * (kThreads / 32), heads = a.k_heads * a.group;
    // sequences one after the other, in every warp
    int64_t done = 0;      // rows of those before
    int64_t mine = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    int taken = 0;
    for (int b = 0; b < a.B; ++b) {
        const int s = a.starts[b], e = a.starts[b + 1];
        const bool good = prompt_good(a, s, e, taken);
        if (prompt_good(a, s, e, 0)) taken = max(taken, e);
        if (!good) {
            if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.err, kErrKvIndex);
            continue;
        }
        const int64_t rows = (int64_t)(e - s) * heads;
        for (; mine < done + rows; mine += warps) {
            const int t = s + (int)((mine - done) / heads), head = (int)((mine - done) % heads);
            prompt_row<BF16, false>(a, head, t, s, a.causal ? t + 1 : e, [] {});
        }
        done += rows;
    }
}

}  // namespace

cudaError_t launch_prompt_rows(const PromptArgs& a, bool bf16, cudaStream_t st) {
    const int64_t want = ((int64_t)a.n * a.k_heads * a.group + kThreads / 32 - 1) / (kThreads / 32), most = 8ll * num_sms();
    auto* kernel = bf16 ? prompt_rows_kernel<true> : prompt_rows_kernel<false>;
    kernel<<<(unsigned)(want < most ? want : most), kThreads, 0, st>>>(a);
    note_launch();
    return cudaGetLastError();
}

}  // namespace soniq
