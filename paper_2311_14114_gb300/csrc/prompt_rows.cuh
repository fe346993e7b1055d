// One row of a prompt's attention by a warp, from its definition: scores from
// products in fp32, softmax in fp32, no weight rounded.
#pragma once

#include "kv_device.cuh"
#include "step_internal.h"

namespace soniq {

// The row of query head `head` at token t, over keys first .. end - 1.
// VEC: rows are whole 16-byte pieces.  Two passes: the largest score; then weights,
// their sum and the output.  Weights are taken in units of 2^spare, the next power
// of two from their number, so that sums of values near the end of bf16's range
// stay in fp32's.  (A score that is NaN makes the row NaN, as do two infinities.)
template <bool BF16, bool VEC>
__device__ __noinline__ void prompt_row(const PromptArgs& a, int head, int t, int first, int end) {
    const int lane = threadIdx.x & 31;
    const int kv = head / a.group;
    const uint16_t* q = a.q.p + t * a.q.token + head * a.q.head;
    auto eight = [](const uint16_t* p, int left, float (&x)[8]) {
        if constexpr (VEC) {
            const uint4 u = *reinterpret_cast<const uint4*>(p);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = kv_load<BF16>((uint16_t)(w[i / 2] >> (16 * (i & 1))));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = i < left ? kv_load<BF16>(p[i]) : 0.0f;
        }
    };
    auto score = [&](int j) {      // a lane's own key
        const uint16_t* k = a.k.p + j * a.k.token + kv * a.k.head;
        float sum = 0.0f;
        for (int c = 0; c < a.D; c += 8) {
            float x[8], y[8];
            eight(q + c, a.D - c, x);
            eight(k + c, a.D - c, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(x[i], y[i], sum);
        }
        return sum;
    };
    float top = -INFINITY;
    bool nan = false;
    for (int j = first + lane; j < end; j += 32) {
        const float s = score(j);
        top = fmaxf(top, s);
        nan = nan || s != s;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    nan = __any_sync(0xffffffffu, nan || top == INFINITY || (top == -INFINITY && end > first));
    const float factor = a.scale * kLog2e;
    const int spare = 32 - __clz(max(end - first - 1, 0));
    float sum = 0.0f, acc[8] = {};
    const int c0 = 8 * lane;
    for (int j0 = first; !nan && j0 < end; j0 += 32) {
        const int j = j0 + lane;
        const float w = j < end ? exp2f((score(j) - top) * factor) : 0.0f;
        sum += w;
        const float part = ldexpf(w, -spare);
        for (int i = 0; i < 32 && j0 + i < end; ++i) {
            const float p = __shfl_sync(0xffffffffu, part, i);
            if (c0 >= a.Dv) continue;
            float x[8];
            eight(a.v.p + (j0 + i) * a.v.token + kv * a.v.head + c0, a.Dv - c0, x);
#pragma unroll
            for (int k = 0; k < 8; ++k) acc[k] = fmaf(p, x[k], acc[k]);
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    const float back = nan ? NAN : ldexpf(1.0f / sum, spare);
    uint16_t* out = a.out + ((int64_t)t * a.k_heads * a.group + head) * a.Dv + c0;
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (c0 + k < a.Dv) out[k] = kv_round<BF16>(acc[k] * back);
}

// A prompt's tokens lie within the batch, and behind those of all before it (`taken`: the end of those within the batch).
__device__ __forceinline__ bool prompt_good(const PromptArgs& a, int s, int e, int taken) { return s >= taken && s <= e && e <= a.n; }

}  // namespace soniq
