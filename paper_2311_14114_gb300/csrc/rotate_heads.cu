// Norms of query and key heads, and their rotation by the token's position, in
// one pass over them.
//
//   y = x rsqrt(mean(x^2) + eps) gain
//   pair p of a token at position t: angle = t f_p,
//   (a, b) -> m (a cos - b sin), m (b cos + a sin)
//
// in fp32, rounded once.  Angles are exact: a frequency is held as turns of 2^64
// parts a position, so the product in 64-bit integers, modulo 2^64, is the part of
// a turn that is left at any position, without a division and without the error
// that a float product of a million positions has.  Its upper half goes to
// sincospi.
//
// A warp takes a token, or a share of its heads; each lane keeps the cosines and
// sines of its eight channels for all of the token's heads.  Rows are read and
// written in 16-byte pieces, two rows of 128 channels to a warp; in the half
// layout partners stand in lanes a fixed distance apart and come by shuffles.
// Rows that are no 16-byte pieces, or whose partners are not whole pieces apart,
// take rotate_scalar_kernel, a channel to a lane.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "step_internal.h"

namespace soniq {

namespace {

constexpr int kThreads = 256;

template <bool BF16>
__device__ __forceinline__ float2 load2(uint32_t x) {
    if constexpr (BF16) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
    else return __half22float2(*reinterpret_cast<const __half2*>(&x));
}
template <bool BF16>
__device__ __forceinline__ uint32_t round2(float lo, float hi) {
    if constexpr (BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    } else {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
}

// Cosine and sine of a position's angle for one pair, times the magnitude.
__device__ __forceinline__ float2 turn(const RotateArgs& a, int position, int pair) {
    if (pair >= a.channels / 2) return make_float2(1.0f, 0.0f);
    const uint64_t part = (uint64_t)(int64_t)position * a.turns[pair];
    float s, c;
    sincospif((float)(int32_t)(part >> 32) * 0x1p-31f, &s, &c);
    return make_float2(c * a.magnitude, s * a.magnitude);
}

// Divides a row, N of whose channels each of its LANES lanes holds, by its root
// mean square.  Where the squares' sum leaves fp32 (above; or below, with no eps
// to speak of) the row is brought to about 1 first.
template <int LANES, int N>
__device__ __forceinline__ void normalise(float (&x)[N], const RotateArgs& a) {
    auto squares = [&]() {
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < N; ++k) sum = fmaf(x[k], x[k], sum);
#pragma unroll
        for (int d = LANES / 2; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        return sum;
    };
    const float sum = squares(), mean = sum / (float)a.D + a.eps;
    float f = rsqrtf(mean);
    const bool out = !(sum <= 1e37f && mean >= 1e-30f);
    if (__any_sync(0xffffffffu, out)) {
        float most = 0.0f;
#pragma unroll
        for (int k = 0; k < N; ++k) most = fmaxf(most, fabsf(x[k]));
#pragma unroll
        for (int d = LANES / 2; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        // a power of two, 2^100 at most so that eps stays in range with it; none for rows of zeros or infinities
        const int e = out && most > 0.0f && most < INFINITY ? min(127 - (int)(__float_as_uint(most) >> 23), 100) : 0;
        const float up = __uint_as_float((uint32_t)(max(e, -126) + 127) << 23);
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] *= up;
        const float better = rsqrtf(squares() / (float)a.D + a.eps * up * up);
        if (e != 0) f = better;
    }
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] *= f;
}

// LANES: lanes of a row, eight channels each.
template <bool BF16, int LANES>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const RotateArgs a, const int parts) {
    constexpr int ROWS = 32 / LANES, STEPS = 4;
    const int lane = threadIdx.x & 31, sub = lane / LANES, l = lane % LANES;
    const int64_t task = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const int64_t token = task / parts;
    const int part = (int)(task % parts);
    if (token >= a.n) return;
    const int c0 = 8 * l, half = a.channels / 2;
    const bool in_row = c0 < a.D;
    // ---- this lane's cosines and sines: pairs (c, c + half), or neighbours ----
    float cs[8], sn[8];
    int partner = 0;
    if (half > 0) {
        const int position = a.positions[token];
        if (a.interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 t = turn(a, position, c0 / 2 + i);
                cs[2 * i] = cs[2 * i + 1] = t.x;
                sn[2 * i] = -t.y;
                sn[2 * i + 1] = t.y;
            }
        } else {
            partner = c0 < half ? half / 8 : (c0 < a.channels ? -half / 8 : 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 t = turn(a, position, c0 < half ? c0 + i : (c0 < a.channels ? c0 - half + i : half));
                cs[i] = t.x;
                sn[i] = c0 < half ? -t.y : t.y;
            }
        }
    }
    const int from = sub * LANES + l + partner, turned = a.channels - c0;      // of this lane's channels, the first `turned`
    // ---- the heads: queries, then keys; `parts` warps share a token's groups of rows ----
#pragma unroll 1
    for (int s = 0; s < 2; ++s) {
        const RotateSide& side = a.side[s];
        const int groups = (side.heads + ROWS - 1) / ROWS;
        const int g0 = (int)((int64_t)groups * part / parts), g1 = (int)((int64_t)groups * (part + 1) / parts);
        if (g0 == g1) continue;
        const uint16_t* in = side.in + token * side.in_token + c0;
        uint16_t* out = side.out + token * side.out_token + c0;
        const bool norm = side.gain != nullptr;
        float gain[8] = {};
        if (norm && in_row) {
            const float4 x = *reinterpret_cast<const float4*>(side.gain + c0), y = *reinterpret_cast<const float4*>(side.gain + c0 + 4);
            gain[0] = x.x, gain[1] = x.y, gain[2] = x.z, gain[3] = x.w;
            gain[4] = y.x, gain[5] = y.y, gain[6] = y.z, gain[7] = y.w;
        }
#pragma unroll 1
        for (int g = g0; g < g1; g += STEPS) {
            uint4 raw[STEPS];
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int h = (g + i) * ROWS + sub;
                raw[i] = make_uint4(0, 0, 0, 0);
                if (g + i < g1 && h < side.heads && in_row) raw[i] = *reinterpret_cast<const uint4*>(in + h * side.in_head);
            }
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                if (g + i >= g1) break;
                const int h = (g + i) * ROWS + sub;
                float x[8];
                const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 v = load2<BF16>(w[k]);
                    x[2 * k] = v.x;
                    x[2 * k + 1] = v.y;
                }
                if (norm) {
                    normalise<LANES>(x, a);
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] *= gain[k];
                }
                if (half > 0) {
                    float y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = a.interleaved ? x[k ^ 1] : __shfl_sync(0xffffffffu, x[k], from);
                    // (a channel that is not turned has no partner: 0 times an infinity would not be 0)
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = k < turned ? y[k] : 0.0f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = fmaf(y[k], sn[k], x[k] * cs[k]);
                }
                if (h < side.heads && in_row)
                    *reinterpret_cast<uint4*>(out + h * side.out_head) =
                        make_uint4(round2<BF16>(x[0], x[1]), round2<BF16>(x[2], x[3]), round2<BF16>(x[4], x[5]), round2<BF16>(x[6], x[7]));
            }
        }
    }
}

// A channel to a lane, eight times: any D, channels and strides.
template <bool BF16>
__global__ void __launch_bounds__(kThreads) rotate_scalar_kernel(const RotateArgs a, const int parts) {
    const int lane = threadIdx.x & 31;
    const int64_t task = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const int64_t token = task / parts;
    const int part = (int)(task % parts);
    if (token >= a.n) return;
    const int half = a.channels / 2;
    float cs[8], sn[8];
    int partner[8];
    const int position = half > 0 ? a.positions[token] : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = lane + 32 * i;
        cs[i] = 1.0f, sn[i] = 0.0f, partner[i] = -1;
        if (c >= a.channels) continue;
        const bool first = a.interleaved ? c % 2 == 0 : c < half;
        partner[i] = a.interleaved ? c ^ 1 : (first ? c + half : c - half);
        const float2 t = turn(a, position, a.interleaved ? c / 2 : (first ? c : c - half));
        cs[i] = t.x;
        sn[i] = first ? -t.y : t.y;
    }
    auto value = [](uint16_t x) { return load2<BF16>(x).x; };
#pragma unroll 1
    for (int s = 0; s < 2; ++s) {
        const RotateSide& side = a.side[s];
        const int h0 = (int)((int64_t)side.heads * part / parts), h1 = (int)((int64_t)side.heads * (part + 1) / parts);
#pragma unroll 1
        for (int h = h0; h < h1; ++h) {
            const uint16_t* in = side.in + token * side.in_token + h * side.in_head;
            uint16_t* out = side.out + token * side.out_token + h * side.out_head;
            float x[8], y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = lane + 32 * i;
                x[i] = c < a.D ? value(in[c]) : 0.0f;
                y[i] = partner[i] >= 0 ? value(in[partner[i]]) : 0.0f;
            }
            __syncwarp();       // the whole row is read before any of it is written: out may be in
            if (side.gain != nullptr) {
                normalise<32>(x, a);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = lane + 32 * i;
                    x[i] = c < a.D ? x[i] * side.gain[c] : 0.0f;
                }
                // the lane that holds the partner has its value now
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float p = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float v = __shfl_sync(0xffffffffu, x[j], partner[i] & 31);
                        if (partner[i] >> 5 == j) p = v;
                    }
                    y[i] = p;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = lane + 32 * i;
                if (c < a.D) out[c] = (uint16_t)round2<BF16>(fmaf(y[i], sn[i], x[i] * cs[i]), 0.0f);
            }
            __syncwarp();
        }
    }
}

template <bool BF16>
cudaError_t launch(const RotateArgs& a, bool vectors, cudaStream_t st) {
    const int lanes = !vectors ? 32 : (a.D <= 64 ? 8 : (a.D <= 128 ? 16 : 32)), rows = 32 / lanes;
    const int groups = (a.side[0].heads + rows - 1) / rows + (a.side[1].heads + rows - 1) / rows;
    // a token's heads are shared by warps until there are eight for each scheduler
    const int64_t want = ((int64_t)num_sms() * 32 + a.n - 1) / a.n;
    const int parts = (int)(want < groups ? want : groups);
    const int64_t grid = (a.n * parts + kThreads / 32 - 1) / (kThreads / 32);
    if (grid > 2147483647) return cudaErrorNotSupported;
    auto* kernel = !vectors ? rotate_scalar_kernel<BF16>
                            : (lanes == 8 ? rotate_kernel<BF16, 8> : (lanes == 16 ? rotate_kernel<BF16, 16> : rotate_kernel<BF16, 32>));
    kernel<<<(unsigned)grid, kThreads, 0, st>>>(a, parts);
    note_launch();
    return cudaGetLastError();
}

bool pieces(const void* p, int64_t token, int64_t head, int64_t n, int heads) {
    return (uintptr_t)p % 16 == 0 && (n == 1 || token % 8 == 0) && (heads == 1 || head % 8 == 0);
}

}  // namespace

cudaError_t launch_rotate_heads(const RotateArgs& a, bool bf16, cudaStream_t st) {
    bool vectors = a.D % 8 == 0 && (a.interleaved || a.channels % 16 == 0);
    for (const RotateSide& s : a.side)
        if (s.heads > 0)
            vectors = vectors && pieces(s.in, s.in_token, s.in_head, a.n, s.heads) &&
                      pieces(s.out, s.out_token, s.out_head, a.n, s.heads) && (uintptr_t)s.gain % 16 == 0;
    return bf16 ? launch<true>(a, vectors, st) : launch<false>(a, vectors, st);
}

}  // namespace soniq
