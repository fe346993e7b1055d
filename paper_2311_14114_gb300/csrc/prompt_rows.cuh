// One row of a prompt's attention by a warp, from its definition: scores from
// products in fp32, softmax in fp32, no weight rounded.
#pragma once

#include "kv_device.cuh"
#include "step_internal.h"

namespace soniq {

constexpr float kMostScale = 2.3e38f;      // up to here scale * log2(e) is within fp32

// The row of query head `head` at token t, over keys first .. end - 1, 32 at a time.
// VEC: rows are whole 16-byte pieces.  Eight channels to a lane, so the warp takes
// one, two or four keys (and values) at once.  Weights are relative to the largest
// score so far, and what is summed follows it; they are in units of 2^spare, the
// next power of two from their number, so that sums of values near the end of
// bf16's range stay in fp32's.  (A score that is NaN makes the row NaN, as do two
// infinities.)  tick() is called by one lane for every 32 keys.
template <bool BF16, bool VEC, typename Tick>
__device__ __noinline__ void prompt_row(const PromptArgs& a, int head, int t, int first, int end, Tick tick) {
    const int lane = threadIdx.x & 31, kv = head / a.group;
    auto width = [](int pieces) { return pieces <= 8 ? 8 : (pieces <= 16 ? 16 : 32); };
    const int k_pieces = (a.D + 7) / 8, v_pieces = (a.Dv + 7) / 8;
    const int k_wide = width(k_pieces), v_wide = width(v_pieces), k_keys = 32 / k_wide, v_keys = 32 / v_wide;
    const int k_lane = lane & (k_wide - 1), v_lane = lane & (v_wide - 1), k_own = lane / k_wide, v_own = lane / v_wide;
    // eight channels from p on, of which `left` are the row's; and their values, or zeros
    auto fetch = [](const uint16_t* p, int left) {
        if constexpr (VEC) {
            return *reinterpret_cast<const uint4*>(p);
        } else {
            uint32_t x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = i < left ? p[i] : 0u;
            return make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
        }
    };
    auto values_of = [](const uint4& u, bool there, float (&x)[8]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = there ? kv_load<BF16>((uint16_t)(w[i / 2] >> (16 * (i & 1)))) : 0.0f;
    };
    // (lanes without a piece read the first one, and drop it)
    const bool k_there = k_lane < k_pieces, v_there = v_lane < v_pieces;
    const int k_at = k_there ? 8 * k_lane : 0, v_at = v_there ? 8 * v_lane : 0;
    float q[8];
    values_of(fetch(a.q.p + t * a.q.token + head * a.q.head + k_at, a.D - k_at), k_there, q);
    const uint16_t* keys = a.k.p + kv * a.k.head + k_at;
    const uint16_t* values = a.v.p + kv * a.v.head + v_at;
    const int64_t k_token = a.k.token, v_token = a.v.token;
    const int k_left = a.D - k_at, v_left = a.Dv - v_at;
    // (never 0: what is not there, minus infinity, has no weight at any scale; in two steps where one would pass fp32, of which the tiles have none)
    const bool whole = VEC || a.scale <= kMostScale;
    const float factor = whole ? fmaxf(a.scale * kLog2e, 1.4e-45f) : a.scale, rest = whole ? 1.0f : kLog2e;
    const int spare = 32 - __clz(max(end - first - 1, 0));
    float top = -INFINITY, sum = 0.0f, acc[8] = {};
    bool nan = false;
    for (int j0 = first; j0 < end; j0 += 32) {
        if (lane == 0) tick();
        float mine = -INFINITY;        // the score of key j0 + lane
#pragma unroll 1
        for (int i0 = 0; i0 < k_wide; i0 += 4) {
            uint4 raw[4];              // (on their way together)
#pragma unroll
            for (int i = 0; i < 4; ++i) raw[i] = fetch(keys + min(j0 + (i0 + i) * k_keys + k_own, end - 1) * k_token, k_left);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x[8], s = 0.0f;
                values_of(raw[i], k_there, x);
#pragma unroll
                for (int c = 0; c < 8; ++c) s = fmaf(q[c], x[c], s);
#pragma unroll
                for (int d = 16; d; d >>= 1)
                    if (d < k_wide) s += __shfl_xor_sync(0xffffffffu, s, d);
                const float to = __shfl_sync(0xffffffffu, s, (lane & (k_keys - 1)) * k_wide);
                if (lane / k_keys == i0 + i && j0 + lane < end) mine = to;
            }
        }
        float best = mine;
#pragma unroll
        for (int d = 16; d; d >>= 1) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, d));
        best = fmaxf(best, top);
        nan = __any_sync(0xffffffffu, mine != mine) || best == INFINITY;
        if (nan) break;
        // (keys of scores minus infinity alone: no weight, and 0 times a value that is not finite is NaN here too)
        const float from = best == -INFINITY ? 0.0f : best;
        const float down = exp2f((top - from) * factor * rest), w = exp2f((mine - from) * factor * rest), part = ldexpf(w, -spare);
        top = best;
        sum = fmaf(sum, down, w);
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[c] *= down;
#pragma unroll 1
        for (int i0 = 0; i0 < v_wide; i0 += 4) {
            uint4 raw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) raw[i] = fetch(values + min(j0 + (i0 + i) * v_keys + v_own, end - 1) * v_token, v_left);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = (i0 + i) * v_keys + v_own;
                const float p = __shfl_sync(0xffffffffu, part, at);
                float x[8];
                values_of(raw[i], v_there && j0 + at < end, x);
#pragma unroll
                for (int c = 0; c < 8; ++c) acc[c] = fmaf(p, x[c], acc[c]);
            }
        }
    }
    nan = nan || top == -INFINITY;
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (d >= v_wide)
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[c] += __shfl_xor_sync(0xffffffffu, acc[c], d);
    }
    const float back = nan ? NAN : ldexpf(1.0f / sum, spare);
    uint16_t* out = a.out + ((int64_t)t * a.k_heads * a.group + head) * a.Dv + 8 * lane;
#pragma unroll
    for (int c = 0; c < 8; ++c)
        if (8 * lane + c < a.Dv) out[c] = kv_round<BF16>(acc[c] * back);
}

// A prompt's tokens lie within the batch, and behind those of all before it (`taken`: the end of those within the batch).
__device__ __forceinline__ bool prompt_good(const PromptArgs& a, int s, int e, int taken) { return s >= taken && s <= e && e <= a.n; }

}  // namespace soniq
