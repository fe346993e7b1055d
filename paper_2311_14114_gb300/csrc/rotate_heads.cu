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
// A warp takes a token, or a share of its heads; its lanes work out the token's
// cosines and sines, and each keeps those of its sixteen channels for all heads.
// Rows are read and written in 16-byte pieces, four rows of 128 channels to a warp.
// Rows that are no 16-byte pieces take rotate_scalar_kernel, a channel to a lane.
//
// Bound by memory where there are many tokens: 16384 tokens x 40 heads of 128, bf16,
// slices of a fused projection, take 67 us (335 MB, 5.0 TB/s; a copy of as many
// bytes takes 56).  Few tokens are bound by the chain position - turns - cosines -
// rows - squares - stores: 8 tokens 6 us, 1001 x 24 heads of 80 8 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "step_internal.h"

namespace soniq {

namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;      // groups of rows, 1 KB each, that a warp has on their way (8: 72 us for 16384 tokens x 40 heads, not 67)

// 16 bytes into shared memory, or zeros; this thread sees them after cp.async.wait_group.
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint32_t read2(uint32_t at) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint4 read16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

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

// 1 / the root mean square of a row, of which each of its LANES lanes holds N
// channels.  Where the squares' sum leaves fp32 (above; or below, with no eps to
// speak of) it is that of the row times *up, a power of two.
template <int LANES, int N>
__device__ __forceinline__ float norm_factor(const float (&x)[N], const RotateArgs& a, float* up) {
    auto over_lanes = [&](float all) {
#pragma unroll
        for (int d = LANES / 2; d; d >>= 1) all += __shfl_xor_sync(0xffffffffu, all, d);
        return all;
    };
    float part[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < N; ++k) part[k & 1] = fmaf(x[k], x[k], part[k & 1]);
    const float sum = over_lanes(part[0] + part[1]), mean = fmaf(sum, a.inverse_D, a.eps);
    float f = rsqrtf(mean);
    const bool out = !(sum <= 1e37f && mean >= 1e-30f);
    if (__any_sync(0xffffffffu, out)) {
        float most = 0.0f, again = 0.0f;
#pragma unroll
        for (int k = 0; k < N; ++k) most = fmaxf(most, fabsf(x[k]));
#pragma unroll
        for (int d = LANES / 2; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        // to about 1; 2^100 at most so that eps stays in range with it; none for rows of zeros or infinities
        const int e = out && most > 0.0f && most < INFINITY ? min(127 - (int)(__float_as_uint(most) >> 23), 100) : 0;
        *up = __uint_as_float((uint32_t)(max(e, -126) + 127) << 23);
#pragma unroll
        for (int k = 0; k < N; ++k) again = fmaf(x[k] * *up, x[k] * *up, again);
        again = over_lanes(again);
        if (e != 0) f = rsqrtf(fmaf(again, a.inverse_D, a.eps * *up * *up));
    }
    return f;
}

enum Pairs { kApart, kNeighbours, kAnywhere };

// LANES: lanes of a row, two pieces of eight channels each.  Where they can a
// pair's two channels are in one lane: apart by whole pieces (kApart), the pieces
// stand half of the turned channels apart; neighbours are in one piece.  Of such a
// pair (x, y) the kernel writes
//   f (x cx + y sx), f (y cy + x sy)
// with the gains in the coefficients; f is the row's norm.  Of pairs that stand
// otherwise (kAnywhere) a lane reads the partners of its channels from the rows in
// shared memory.
template <bool BF16, int LANES, int PAIRS>
__global__ void __launch_bounds__(kThreads, 2) rotate_kernel(const __grid_constant__ RotateArgs a, const int parts) {
    constexpr int ROWS = 32 / LANES;
    const int lane = threadIdx.x & 31, sub = lane / LANES, l = lane % LANES;
    const int64_t task = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const int64_t token = task / parts;
    const int part = (int)(task - token * parts);
    if (token >= a.n) return;
    const int half = a.channels / 2;
    // This lane's pieces: of channels turned in kApart a pair of pieces; else one each of the first and the second half of
    // the row's (of those that are not turned), so that neighbouring lanes have neighbouring pieces.
    const bool turned = PAIRS != kApart || 16 * l < a.channels;
    const int base = PAIRS == kApart ? a.channels : 0, l0 = l - base / 16, pieces = (a.D - base) / 8, upper = (pieces + 1) / 2;
    int c0 = l0 < upper ? base + 8 * l0 : a.D, c1 = l0 < upper && l0 + upper < pieces ? base + 8 * (l0 + upper) : a.D;
    if (PAIRS == kApart && turned) {
        c0 = 8 * l;
        c1 = half + 8 * l;
    }
    const bool in0 = c0 < a.D, in1 = c1 < a.D;
    // `parts` warps share a token's groups of rows
    auto first_of = [&](const RotateSide& side, int p) { return (int)((int64_t)((side.heads + ROWS - 1) / ROWS) * p / parts); };
    // ---- groups of rows on their way: kAhead of them, each lane's pieces in places of its own ----
    extern __shared__ __align__(16) uint8_t ring[];
    const int first0 = first_of(a.side[0], part), n0 = first_of(a.side[0], part + 1) - first0;
    const int first1 = first_of(a.side[1], part), n1 = first_of(a.side[1], part + 1) - first1;
    const uint32_t place = (uint32_t)__cvta_generic_to_shared(ring) + (threadIdx.x >> 5) * (kAhead * 1024) + 16 * lane;
    const uint16_t* next = a.side[0].in + token * a.side[0].in_token + (int64_t)(first0 * ROWS + sub) * a.side[0].in_head;
    int next_left = n0, next_rows = a.side[0].heads - first0 * ROWS - sub;      // groups to come of this side, rows from this lane's on
    bool last_side = false;
    uint32_t put = 0;
    auto fetch = [&]() {
        if (next_left == 0 && !last_side) {
            last_side = true;
            next = a.side[1].in + token * a.side[1].in_token + (int64_t)(first1 * ROWS + sub) * a.side[1].in_head;
            next_left = n1;
            next_rows = a.side[1].heads - first1 * ROWS - sub;
        }
        if (next_left > 0) {
            copy16(place + put, next + (in0 ? c0 : 0), in0 && next_rows > 0);
            copy16(place + put + 512, next + (in1 ? c1 : 0), in1 && next_rows > 0);
            next += ROWS * a.side[last_side ? 1 : 0].in_head;
            next_rows -= ROWS;
            --next_left;
            put = (put + 1024) % (kAhead * 1024);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll 1
    for (int t = 0; t < kAhead; ++t) fetch();
    // ---- the token's cosines and sines, a pair to a lane ----
    __shared__ float2 turns[kThreads / 32][128];
    float2* mine = turns[threadIdx.x >> 5];
    if (half > 0) {
        const int position = a.positions[token];
#pragma unroll 1
        for (int p = lane; p < half; p += 32) mine[p] = turn(a, position, p);
        __syncwarp();
    }
    // what a channel's partner counts for: nothing where it is not turned, even if it is an infinity
    auto pair_of = [&](int i) { return PAIRS == kNeighbours ? (i < 4 ? c0 / 2 + i : c1 / 2 + i - 4) : c0 + i; };
    auto channel = [&](int k) { return k < 8 ? c0 + k : c1 + k - 8; };
    uint32_t counts = 0;       // by pair, or (kAnywhere) by channel
    uint16_t mate[PAIRS == kAnywhere ? 16 : 1];        // where the partner's value stands in the group's 1 KB
    if constexpr (PAIRS == kAnywhere) {
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const int c = channel(k), p = c < half ? c + half : c - half, j = p >> 3;
            counts |= (uint32_t)(c < a.channels) << k;
            mate[k] = (uint16_t)(c < a.channels ? (j < upper ? 16 * (sub * LANES + j) : 512 + 16 * (sub * LANES + j - upper)) + 2 * (p & 7) : 0);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) counts |= (uint32_t)(turned && pair_of(i) < half) << i;
    }
    const bool all = PAIRS != kAnywhere && __all_sync(0xffffffffu, (counts | (in1 ? 0u : 0xf0u)) == 0xffu || !in0);
    // ---- the heads: queries, then keys ----
    uint32_t get = 0;
#pragma unroll 1
    for (int s = 0; s < 2; ++s) {
        const RotateSide& side = a.side[s];
        const int n = s ? n1 : n0, first = s ? first1 : first0;
        if (n == 0) continue;
        const bool norm = side.gain != nullptr;
        float g0[8], g1[8];        // gains of this lane's pieces
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const float4 one = make_float4(1.0f, 1.0f, 1.0f, 1.0f);
            const float4 p = norm && in0 ? *reinterpret_cast<const float4*>(side.gain + c0 + i) : one;
            const float4 q = norm && in1 ? *reinterpret_cast<const float4*>(side.gain + c1 + i) : one;
            g0[i] = p.x, g0[i + 1] = p.y, g0[i + 2] = p.z, g0[i + 3] = p.w;
            g1[i] = q.x, g1[i + 1] = q.y, g1[i + 2] = q.z, g1[i + 3] = q.w;
        }
        // of pairs: (cx, sx) and (cy, sy); of channels: cx and sx of the first eight, cy and sy of the others
        float cx[8], sx[8], cy[8], sy[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (PAIRS == kAnywhere) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int c = channel(8 * h + i);
                    const bool on = c < a.channels, first = c < half;
                    const float2 t = on ? mine[first ? c : c - half] : make_float2(1.0f, 0.0f);
                    const float mates = on && norm ? side.gain[first ? c + half : c - half] : 1.0f;
                    (h ? cy : cx)[i] = t.x * (h ? g1 : g0)[i];
                    (h ? sy : sx)[i] = (first ? -t.y : t.y) * mates;
                }
            } else {
                const float gx = PAIRS == kNeighbours ? (i < 4 ? g0[2 * i] : g1[2 * i - 8]) : g0[i];
                const float gy = PAIRS == kNeighbours ? (i < 4 ? g0[2 * i + 1] : g1[2 * i - 7]) : g1[i];
                const float2 t = counts >> i & 1u ? mine[pair_of(i)] : make_float2(1.0f, 0.0f);
                cx[i] = t.x * gx, sx[i] = -t.y * gy;
                cy[i] = t.x * gy, sy[i] = t.y * gx;
            }
        }
        uint16_t* to = side.out + token * side.out_token + (int64_t)(first * ROWS + sub) * side.out_head;
        const int64_t to_step = ROWS * side.out_head;
        int rows = side.heads - first * ROWS - sub;        // from this lane's on
#pragma unroll 1
        for (int g = 0; g < n; ++g, to += to_step, rows -= ROWS) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
            float mates[PAIRS == kAnywhere ? 16 : 1];
            if constexpr (PAIRS == kAnywhere) {
                __syncwarp();       // all of the group's rows are there
#pragma unroll
                for (int k = 0; k < 16; ++k)
                    mates[k] = counts >> k & 1u ? load2<BF16>(read2(place - 16 * lane + get + mate[k])).x : 0.0f;
            }
            const uint4 p0 = read16(place + get), p1 = read16(place + get + 512);
            get = (get + 1024) % (kAhead * 1024);
            const uint32_t w[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
            float v[16];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float2 pair = load2<BF16>(w[k]);
                v[2 * k] = pair.x;
                v[2 * k + 1] = pair.y;
            }
            if constexpr (PAIRS == kAnywhere) __syncwarp();       // their places are read
            fetch();
            float f = 1.0f, up = 1.0f;
            if (norm) {
                f = norm_factor<LANES>(v, a, &up);
                if (up != 1.0f) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        v[k] *= up;
                        if constexpr (PAIRS == kAnywhere) mates[k] *= up;
                    }
                }
            }
            uint32_t r[8];
            if constexpr (PAIRS == kAnywhere) {
#pragma unroll
                for (int k = 0; k < 16; k += 2) {
                    const float* c = k < 8 ? cx + k : cy + k - 8;
                    const float* d = k < 8 ? sx + k : sy + k - 8;
                    r[k / 2] = round2<BF16>(fmaf(mates[k], d[0], v[k] * c[0]) * f, fmaf(mates[k + 1], d[1], v[k + 1] * c[1]) * f);
                }
            } else {
                float z[8], u[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float x = PAIRS == kNeighbours ? v[2 * k] : v[k], y = PAIRS == kNeighbours ? v[2 * k + 1] : v[8 + k];
                    const bool on = all || (counts >> k & 1u) != 0;
                    z[k] = fmaf(on ? y : 0.0f, sx[k], x * cx[k]) * f;
                    u[k] = fmaf(on ? x : 0.0f, sy[k], y * cy[k]) * f;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    r[k] = PAIRS == kNeighbours ? round2<BF16>(z[k], u[k])
                                                : (k < 4 ? round2<BF16>(z[2 * k], z[2 * k + 1]) : round2<BF16>(u[2 * k - 8], u[2 * k - 7]));
            }
            if (rows > 0 && in0) *reinterpret_cast<uint4*>(to + c0) = make_uint4(r[0], r[1], r[2], r[3]);
            if (rows > 0 && in1) *reinterpret_cast<uint4*>(to + c1) = make_uint4(r[4], r[5], r[6], r[7]);
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// A channel to a lane, eight times: any D, channels and strides.
template <bool BF16>
__global__ void __launch_bounds__(kThreads) rotate_scalar_kernel(const __grid_constant__ RotateArgs a, const int parts) {
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
                float up = 1.0f;
                const float f = norm_factor<32>(x, a, &up);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = lane + 32 * i;
                    x[i] = c < a.D ? x[i] * up * f * side.gain[c] : 0.0f;
                    y[i] = partner[i] >= 0 ? y[i] * up * f * side.gain[partner[i]] : 0.0f;
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

template <bool BF16, int PAIRS>
auto* kernel_of(int lanes) {
    return lanes == 4 ? rotate_kernel<BF16, 4, PAIRS> : (lanes == 8 ? rotate_kernel<BF16, 8, PAIRS> : rotate_kernel<BF16, 16, PAIRS>);
}

template <bool BF16>
cudaError_t launch(const RotateArgs& a, bool vectors, cudaStream_t st) {
    const int lanes = !vectors ? 32 : (a.D <= 64 ? 4 : (a.D <= 128 ? 8 : 16)), rows = 32 / lanes;
    const int groups = (a.side[0].heads + rows - 1) / rows + (a.side[1].heads + rows - 1) / rows;
    // a token's heads are shared by warps as long as all of them are at work at once
    const int64_t want = (int64_t)num_sms() * (2 * kThreads / 32) / a.n;
    const int parts = (int)(want < 1 ? 1 : (want < groups ? want : groups));
    const int64_t grid = (a.n * parts + kThreads / 32 - 1) / (kThreads / 32);
    if (grid > 2147483647) return cudaErrorNotSupported;
    auto* kernel = !vectors ? rotate_scalar_kernel<BF16>
                            : (a.interleaved ? kernel_of<BF16, kNeighbours>(lanes)
                                             : (a.channels % 16 == 0 ? kernel_of<BF16, kApart>(lanes) : kernel_of<BF16, kAnywhere>(lanes)));
    const int smem = vectors ? kThreads / 32 * kAhead * 1024 : 0;
    const cudaError_t e = prefer_max_shared(reinterpret_cast<const void*>(kernel));
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)grid, kThreads, smem, st>>>(a, parts);
    note_launch();
    return cudaGetLastError();
}

bool pieces(const void* p, int64_t token, int64_t head, int64_t n, int heads) {
    return (uintptr_t)p % 16 == 0 && (n == 1 || token % 8 == 0) && (heads == 1 || head % 8 == 0);
}

}  // namespace

cudaError_t launch_rotate_heads(const RotateArgs& a, bool bf16, cudaStream_t st) {
    bool vectors = a.D % 8 == 0;
    for (const RotateSide& s : a.side)
        if (s.heads > 0)
            vectors = vectors && pieces(s.in, s.in_token, s.in_head, a.n, s.heads) &&
                      pieces(s.out, s.out_token, s.out_head, a.n, s.heads) && (uintptr_t)s.gain % 16 == 0;
    return bf16 ? launch<true>(a, vectors, st) : launch<false>(a, vectors, st);
}

}  // namespace soniq
