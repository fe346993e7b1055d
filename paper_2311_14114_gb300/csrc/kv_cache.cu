// Key / value cache: rows quantized as they are written, and read back.
//
// A row is one token's key (or value) of one head.  Per precision group g of
// its channels: s_g = max|x|, j = clamp(rne(x / s_g * 2^(n-1)), -2^(n-1),
// 2^(n-1) - 1) (Eq. (1)), packed in 32-code blocks (layout: soniq.h).
//
// Both directions are bound by bytes (2 per channel on the plain side, n/8 on
// the packed one), so the work per value is kept near that of a copy: a lane
// owns eight packed positions of a (side, head), whose channels it looks up
// once, and goes from token to token; LPR lanes (a power of two) make a row.
// Where the channels of every lane are eight in a row (an ascending group), a
// lane loads or stores them with one 16-byte access; otherwise rows pass
// through shared memory in their own order and are gathered there; rows off the
// 16-byte grid are accessed channel by channel.
// Both maxima of a row are reduced together, as two 16-bit patterns in one word
// (patterns of finite magnitudes order as integers).  The quotient is formed by
// Markstein's correction on the reciprocal, two at a time, which is exact for
// 16-bit inputs at scales in [2^-60, 2^60]; other scales divide.
// Bound by instructions (about 195 for 256 written values, 105 for read ones,
// which is why the loop is compiled once for each way to reach a row) and, when
// reading, by the latency of the packed words.  Measured (GB300, bf16, 8 heads of
// 128 channels, mostly 4 bits): 16384 tokens written 33 us (2.6 TB/s of rows and
// codes), 65536 read 123 us (2.8 TB/s); 777 tokens read 4.8 us.
#include "kv_internal.h"
#include "soniq_device.cuh"

namespace soniq {

namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kStride = 2 * kKvMaxCodes + 24;   // bytes of a staged row, its zero entry included: the rows of a warp start on different banks

__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) { return __vmaxu2(a, b); }

// What a lane owns: eight packed positions of a (side, head).
struct Lane {
    bool valid;          // some block holds them
    int grp, bits, q;    // group, width, eighth of the group's codes
    int ch[8];           // channels; -1: padding
    bool run;            // eight channels in a row, on a 16-byte boundary (or none at all)
};

template <int LPR>
__device__ __forceinline__ Lane make_lane(const KvSide& s, int head) {
    Lane l;
    const int q = threadIdx.x & (LPR - 1), first = 4 * s.nb[0];
    l.valid = q < 4 * (s.nb[0] + s.nb[1]);
    l.grp = q < first ? 0 : 1;
    l.q = l.grp ? q - first : q;
    l.bits = s.bits[l.grp];
    const int32_t* perm = s.perm + head * s.D + (l.grp ? s.count[0] : 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int p = 8 * l.q + i;
        l.ch[i] = l.valid && p < s.count[l.grp] ? __ldg(perm + p) : -1;
    }
    bool run = (l.ch[0] & 7) == 0, none = l.ch[0] < 0;
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        run &= l.ch[i] == l.ch[0] + i;
        none &= l.ch[i] < 0;
    }
    l.run = run || none;
    return l;
}

// 16-bit pattern i of four words of two
__device__ __forceinline__ uint32_t pattern(const uint32_t (&w)[4], int i) { return i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu; }

// Values of another than finite magnitude: NaN as 0, infinities as the largest finite value.
__device__ __forceinline__ uint32_t clean(uint32_t x, uint32_t inf) {
    const uint32_t m = x & 0x7FFFu;
    return m < inf ? x : (m == inf ? (x & 0x8000u) | (inf - 1u) : 0u);
}

// Packed codes of a lane: two words (8 bits), one (4), or the low nibble of each
// byte of one (2).
__device__ __forceinline__ void pack8(const uint32_t (&j)[8], int bits, uint32_t (&w)[2]) {
    const uint32_t lo = __byte_perm(__byte_perm(j[0], j[1], 0x0040), __byte_perm(j[2], j[3], 0x0040), 0x5410);
    const uint32_t hi = __byte_perm(__byte_perm(j[4], j[5], 0x0040), __byte_perm(j[6], j[7], 0x0040), 0x5410);
    if (bits == 4) {
        w[0] = (lo & 0x0F0F0F0Fu) | ((hi & 0x0F0F0F0Fu) << 4);
    } else if (bits == 8) {
        w[0] = lo;
        w[1] = hi;
    } else {
        w[0] = (lo & 0x03030303u) | ((hi & 0x03030303u) << 2);
    }
}

// How a warp reaches its rows; the loop over tokens is compiled for each.
enum { kRun = 0, kStaged = 1, kSingle = 2 };
template <int M>
struct Mode {
    static constexpr int value = M;
};

// A slot as page and place in it; page -1: skipped (reported if beyond the cache).
struct Place {
    int page, in;
};
__device__ __forceinline__ Place place_of(const KvGeom& geo, int64_t slot, bool report, unsigned* err) {
    const bool ok = slot >= 0 && slot < geo.n_pages << geo.page_shift;
    if (slot >= 0 && !ok && report) atomicOr(err, kErrKvIndex);
    return Place{ok ? (int)(slot >> geo.page_shift) : -1, (int)(slot & (geo.page - 1))};
}

// Two values, each rounded once, as 16-bit patterns in one word.
template <bool BF16>
__device__ __forceinline__ uint32_t round2(float lo, float hi) {
    uint32_t r;
    if constexpr (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// ... and back
template <bool BF16>
__device__ __forceinline__ float2 load2(uint32_t x) {
    if constexpr (BF16) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
    else return __half22float2(*reinterpret_cast<const __half2*>(&x));
}

template <int LPR, bool BF16>
__global__ void __launch_bounds__(kThreads, 3) kv_write_kernel(const KvGeom geo, const KvRowsArg k, const KvRowsArg v,
                                                            const int64_t* __restrict__ slots, int64_t n, int per_warp,
                                                            int side0, unsigned* err) {
    constexpr int RPW = 32 / LPR;
    constexpr uint32_t INF = BF16 ? 0x7F80u : 0x7C00u;
    __shared__ __align__(16) uint8_t rows[kWarps][RPW][kStride];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int head = blockIdx.y, side = side0 + blockIdx.z, ql = lane & (LPR - 1);
    const KvSide s = side ? geo.s[1] : geo.s[0];
    const KvRowsArg in = side ? v : k;
    const Lane me = make_lane<LPR>(s, head);
    const bool wide = (((uintptr_t)in.p | (uintptr_t)(2 * in.token_stride) | (uintptr_t)(2 * in.head_stride)) & 15u) == 0 && s.D % 8 == 0;
    const int mode = !wide ? kSingle : (__all_sync(0xffffffffu, me.run) ? kRun : kStaged);
    uint8_t* staged = rows[warp][lane / LPR];
    if (mode == kStaged && ql == 0) *reinterpret_cast<uint16_t*>(staged + 2 * s.D) = 0;      // what padding reads
    const uint16_t* base = in.p + head * in.head_stride;
    const int64_t t_warp = ((int64_t)blockIdx.x * kWarps + warp) * per_warp, t_end = min(n, t_warp + per_warp);
    const float half = (float)(1 << (me.bits - 1)), per_half = 1.0f / half, most = half - 1.0f;
    // where a lane's channels are in the staged row, and its codes and scale in a row of this head
    uint32_t from[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) from[i] = (uint32_t)__cvta_generic_to_shared(staged) + 2 * (me.ch[i] < 0 ? s.D : me.ch[i]);
    uint8_t* codes = s.codes + (int64_t)head * geo.page * s.row_bytes + s.off[me.grp] + me.bits * me.q;
    uint16_t* scales = s.scales + (int64_t)head * geo.page * s.ng + me.grp;
    const uint32_t page_codes = geo.heads * geo.page * s.row_bytes, page_scales = geo.heads * geo.page * s.ng;
    const bool stores = me.valid && !(me.bits == 2 && (me.q & 1));
    // the 16 bytes this lane loads of a row: its channels, or its share of the row
    const int ch16 = mode == kRun ? me.ch[0] : 8 * ql;
    const bool loads = mode != kSingle && ch16 >= 0 && ch16 < s.D;
    auto run = [&](auto mode_c) {
        constexpr int MODE = decltype(mode_c)::value;
        // 32 tokens at a time: t_first .. t_first + count - 1; lane i holds the slot of the i-th
        int64_t slot = t_warp + lane < t_end ? __ldg(slots + t_warp + lane) : -1;
#pragma unroll 1
        for (int64_t t_first = t_warp; t_first < t_end; t_first += 32) {
            const int count = (int)min((int64_t)32, t_end - t_first);
            const Place mine = place_of(geo, slot, head == 0 && side == 0, err);
            slot = t_first + 32 + lane < t_end ? __ldg(slots + t_first + 32 + lane) : -1;      // of the next 32
            // rows are loaded two steps ahead of their use (the loop stays rolled: unrolled four times, with all its
            // loads at the top, it took twice as long, for its instructions)
            const uint16_t* load_at = base + (t_first + lane / LPR) * in.token_stride + ch16;
            int i_load = lane / LPR;
            auto load = [&]() {
                uint4 r = make_uint4(0, 0, 0, 0);
                if (loads && i_load < count) r = __ldg(reinterpret_cast<const uint4*>(load_at));
                load_at += RPW * in.token_stride;
                i_load += RPW;
                return r;
            };
            uint4 ahead0 = load(), ahead1 = load();
#pragma unroll 1
            for (int i0 = 0; i0 < count; i0 += RPW) {
                const int i_tok = i0 + lane / LPR;
                const uint4 raw = ahead0;
                ahead0 = ahead1;
                ahead1 = load();
                const int page = __shfl_sync(0xffffffffu, mine.page, i_tok & 31), in_page = __shfl_sync(0xffffffffu, mine.in, i_tok & 31);
                uint32_t x[4] = {raw.x, raw.y, raw.z, raw.w};
                if constexpr (MODE == kStaged) {
                    __syncwarp();
                    if (loads) {        // rows start on 8-byte boundaries
                        *reinterpret_cast<uint2*>(staged + 2 * ch16) = make_uint2(raw.x, raw.y);
                        *reinterpret_cast<uint2*>(staged + 2 * ch16 + 8) = make_uint2(raw.z, raw.w);
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        uint32_t a, b;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=r"(a) : "r"(from[i]) : "memory");
                        asm volatile("ld.shared.u16 %0, [%1];" : "=r"(b) : "r"(from[i + 1]) : "memory");
                        x[i >> 1] = __byte_perm(a, b, 0x5410);
                    }
                } else if constexpr (MODE == kSingle) {
                    const uint16_t* src = base + (t_first + i_tok) * in.token_stride;
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const uint32_t a = i_tok < count && me.ch[i] >= 0 ? src[me.ch[i]] : 0u;
                        const uint32_t b = i_tok < count && me.ch[i + 1] >= 0 ? src[me.ch[i + 1]] : 0u;
                        x[i >> 1] = a | b << 16;
                    }
                }
                if (!me.valid) x[0] = x[1] = x[2] = x[3] = 0u;
                // both groups' maxima: a lane's, in its group's half word, then over the row
                auto row_max = [&]() {
                    uint32_t m = max2(max2(x[0] & 0x7FFF7FFFu, x[1] & 0x7FFF7FFFu), max2(x[2] & 0x7FFF7FFFu, x[3] & 0x7FFF7FFFu));
                    m = max(m & 0xFFFFu, m >> 16) << (16 * me.grp);
#pragma unroll
                    for (int i = LPR / 2; i; i >>= 1) m = max2(m, __shfl_xor_sync(0xffffffffu, m, i));
                    return m;
                };
                uint32_t m = row_max();
                if (__any_sync(0xffffffffu, (m & 0xFFFFu) >= INF || (m >> 16) >= INF)) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = clean(x[i] & 0xFFFFu, INF) | clean(x[i] >> 16, INF) << 16;
                    m = row_max();
                }
                const uint32_t top = me.grp ? m >> 16 : m & 0xFFFFu;
                const float sc = kv_load<BF16>((uint16_t)top);
                uint32_t j[8];
                if (__all_sync(0xffffffffu, sc == 0.0f || (sc >= 0x1p-60f && sc <= 0x1p60f))) {
                    // t = x r + (x - x r s') r with r = 2^(n-1) / s to about an ulp, s' = s / 2^(n-1).  The correction leaves
                    // about 2^-44 of t: a tie, which is a number of few bits, comes out exactly, and other quotients of 11-bit
                    // numbers are further than 2^-20 from one.
                    float rc;
                    asm("rcp.approx.f32 %0, %1;" : "=f"(rc) : "f"(sc));
                    const float r = sc == 0.0f ? 0.0f : rc * half, sh = -sc * per_half;
                    const float2 r2 = make_float2(r, r), s2 = make_float2(sh, sh);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 y = load2<BF16>(x[i]);
                        const float2 q0 = mul2(y, r2);
                        float2 q = fma2(fma2(q0, s2, y), r2, q0);
                        // the integer in the low bits, rounded half to even
                        q = add2(make_float2(fminf(q.x, most), fminf(q.y, most)), 12582912.0f);
                        j[2 * i] = __float_as_uint(q.x);
                        j[2 * i + 1] = __float_as_uint(q.y);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) j[i] = (uint32_t)weight_code(kv_load<BF16>((uint16_t)pattern(x, i)), sc, half);
                }
                uint32_t w[2] = {0u, 0u};
                pack8(j, me.bits, w);
                const uint32_t other = __shfl_xor_sync(0xffffffffu, w[0], 1);
                if (me.bits == 2) w[0] |= other << 4;      // pairs of lanes share a word
                if (i_tok >= count || page < 0 || !stores) continue;
                uint8_t* dst = codes + (uint64_t)(uint32_t)page * page_codes + in_page * s.row_bytes;
                if (me.bits == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
                else *reinterpret_cast<uint32_t*>(dst) = w[0];
                if (me.q == 0) scales[(uint64_t)(uint32_t)page * page_scales + in_page * s.ng] = (uint16_t)top;
            }
        }
    };
    if (mode == kRun) run(Mode<kRun>{});
    else if (mode == kStaged) run(Mode<kStaged>{});
    else run(Mode<kSingle>{});
}

// Eight codes of a lane as fp32, from its word(s).
__device__ __forceinline__ void unpack8(const uint32_t (&w)[2], int bits, float (&f)[8]) {
    // codes 0..3 and 4..7 as bytes in offset binary; 2^23 + byte is that float's low bits
    const uint32_t flip = 0x01010101u << (bits - 1), mask = bits == 8 ? 0xFFFFFFFFu : (bits == 4 ? 0x0F0F0F0Fu : 0x03030303u);
    const uint32_t lo = (w[0] & mask) ^ flip, hi = ((bits == 8 ? w[1] : w[0] >> bits) & mask) ^ flip;
    const float off = 8388608.0f + (float)(1 << (bits - 1));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = __uint_as_float(__byte_perm(lo, 0x4B000000u, 0x7650 + i)) - off;
        f[4 + i] = __uint_as_float(__byte_perm(hi, 0x4B000000u, 0x7650 + i)) - off;
    }
}

template <int LPR, bool BF16>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(const KvGeom geo, const int64_t* __restrict__ slots, int64_t n,
                                                           int per_warp, int side0, uint16_t* k, uint16_t* v, unsigned* err) {
    constexpr int RPW = 32 / LPR;
    __shared__ __align__(16) uint8_t rows[kWarps][RPW][kStride];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int head = blockIdx.y, side = side0 + blockIdx.z, ql = lane & (LPR - 1);
    const KvSide s = side ? geo.s[1] : geo.s[0];
    uint16_t* out = side ? v : k;
    if (out == nullptr) return;
    const Lane me = make_lane<LPR>(s, head);
    const bool wide = ((uintptr_t)out & 15u) == 0 && s.D % 8 == 0;
    const int mode = !wide ? kSingle : (__all_sync(0xffffffffu, me.run) ? kRun : kStaged);
    uint8_t* staged = rows[warp][lane / LPR];
    const int64_t t_warp = ((int64_t)blockIdx.x * kWarps + warp) * per_warp, t_end = min(n, t_warp + per_warp);
    const float unit = 1.0f / (float)(1 << (me.bits - 1));
    // a lane's codes and scale in a row of this head, and its channels in the staged row
    const uint8_t* codes = s.codes + (int64_t)head * geo.page * s.row_bytes + s.off[me.grp] + (me.bits == 2 ? 4 * (me.q >> 1) : me.bits * me.q);
    const uint16_t* scales = s.scales + (int64_t)head * geo.page * s.ng + me.grp;
    const uint32_t page_codes = geo.heads * geo.page * s.row_bytes, page_scales = geo.heads * geo.page * s.ng;
    uint32_t to[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) to[i] = (uint32_t)__cvta_generic_to_shared(staged) + 2 * (me.ch[i] < 0 ? s.D : me.ch[i]);     // padding: behind the row
    auto run = [&](auto mode_c) {
        constexpr int MODE = decltype(mode_c)::value;
        int64_t slot = t_warp + lane < t_end ? __ldg(slots + t_warp + lane) : -1;
#pragma unroll 1
        for (int64_t t_first = t_warp; t_first < t_end; t_first += 32) {
            const int count = (int)min((int64_t)32, t_end - t_first);
            const Place mine = place_of(geo, slot, head == 0, err);
            slot = t_first + 32 + lane < t_end ? __ldg(slots + t_first + 32 + lane) : -1;      // of the next 32
            // packed words and scales are loaded two steps ahead of their use
            struct Packed {
                uint32_t w0, w1, sc;
            };
            int i_load = lane / LPR;
            auto load = [&]() {
                Packed r{0u, 0u, 0u};
                const int page = __shfl_sync(0xffffffffu, mine.page, i_load & 31), in_page = __shfl_sync(0xffffffffu, mine.in, i_load & 31);
                if (i_load < count && me.valid && page >= 0) {
                    const uint8_t* src = codes + (uint64_t)(uint32_t)page * page_codes + in_page * s.row_bytes;
                    r.w0 = *reinterpret_cast<const uint32_t*>(src);
                    if (me.bits == 8) r.w1 = *reinterpret_cast<const uint32_t*>(src + 4);
                    r.sc = scales[(uint64_t)(uint32_t)page * page_scales + in_page * s.ng];
                }
                i_load += RPW;
                return r;
            };
            Packed ahead0 = load(), ahead1 = load();
            uint16_t* dst = out + ((t_first + lane / LPR) * geo.heads + head) * s.D;
            const int64_t dst_step = (int64_t)RPW * geo.heads * s.D;
#pragma unroll 1
            for (int i0 = 0; i0 < count; i0 += RPW) {
                const int i_tok = i0 + lane / LPR;
                uint32_t w[2] = {ahead0.w0, ahead0.w1};
                const float u = kv_load<BF16>((uint16_t)ahead0.sc) * unit;
                ahead0 = ahead1;
                ahead1 = load();
                if (me.bits == 2) w[0] = w[0] >> (4 * (me.q & 1)) & 0x0F0F0F0Fu;
                float f[8];
                unpack8(w, me.bits, f);
                uint32_t y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 z = mul2(make_float2(f[2 * i], f[2 * i + 1]), make_float2(u, u));
                    y[i] = round2<BF16>(z.x, z.y);
                }
                const bool on = i_tok < count && me.valid;
                if constexpr (MODE == kRun) {
                    if (on && me.ch[0] >= 0) *reinterpret_cast<uint4*>(dst + me.ch[0]) = make_uint4(y[0], y[1], y[2], y[3]);
                } else if constexpr (MODE == kStaged) {
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) asm volatile("st.shared.b16 [%0], %1;" ::"r"(to[i]), "h"((uint16_t)pattern(y, i)) : "memory");
                    __syncwarp();
                    if (i_tok < count && 8 * ql < s.D) {
                        const uint2 a = *reinterpret_cast<const uint2*>(staged + 16 * ql), b = *reinterpret_cast<const uint2*>(staged + 16 * ql + 8);
                        *reinterpret_cast<uint4*>(dst + 8 * ql) = make_uint4(a.x, a.y, b.x, b.y);
                    }
                } else if (on) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (me.ch[i] >= 0) dst[me.ch[i]] = (uint16_t)pattern(y, i);
                }
                dst += dst_step;
            }
        }
    };
    if (mode == kRun) run(Mode<kRun>{});
    else if (mode == kStaged) run(Mode<kStaged>{});
    else run(Mode<kSingle>{});
}

// Lanes to a row, and tokens to a warp: as many warps as the registers leave room
// for at once (reading, 32 on an SM), or two such waves (writing, 24 each), then
// as many tokens to each as there are.  16384 tokens written and read, us: 59 so,
// 68 with twice as many warps, 78 with a wave for writing and two for reading.
struct Shape {
    int lpr, per_warp, side0;
    dim3 grid;
};
int lanes_of(const KvSide& s) {
    int lpr = 4;
    while (lpr < 4 * (s.nb[0] + s.nb[1])) lpr *= 2;
    return lpr;
}
// Keys and values in one launch, or, where their rows take different numbers of
// lanes and there are enough of them to repay it, in one each (20 and 16 lanes, 8
// heads, together and apart, us: 8192 tokens written and read 50 and 54, 16384 93
// and 89, 65536 336 and 290, read alone 134 and 123).
constexpr int64_t kApart = 131072;
int make_shapes(const KvGeom& geo, int64_t n, int warps_per_sm, Shape (&shapes)[2]) {
    const int lpr[2] = {lanes_of(geo.s[0]), lanes_of(geo.s[1])};
    const int launches = lpr[0] != lpr[1] && n * geo.heads >= kApart ? 2 : 1, sides = 2 / launches;
    for (int i = 0; i < launches; ++i) {
        Shape* sh = &shapes[i];
        sh->side0 = i;
        sh->lpr = launches == 2 ? lpr[i] : (lpr[0] > lpr[1] ? lpr[0] : lpr[1]);
        const int64_t rpw = 32 / sh->lpr, steps = (n + rpw - 1) / rpw * geo.heads * sides;
        int64_t iters = (steps + (int64_t)num_sms() * warps_per_sm - 1) / ((int64_t)num_sms() * warps_per_sm);
        iters = iters < 1 ? 1 : (iters > 1024 ? 1024 : iters);
        sh->per_warp = (int)(iters * rpw);
        const int64_t blocks = (n + (int64_t)kWarps * sh->per_warp - 1) / ((int64_t)kWarps * sh->per_warp);
        if (blocks > 2147483647) return 0;
        sh->grid = dim3((unsigned)blocks, (unsigned)geo.heads, (unsigned)sides);
    }
    return launches;
}

template <bool BF16>
void run_write(const Shape& sh, const KvGeom& geo, const KvRowsArg& k, const KvRowsArg& v, const int64_t* slots, int64_t n,
               unsigned* err, cudaStream_t st) {
    if (sh.lpr == 32) kv_write_kernel<32, BF16><<<sh.grid, kThreads, 0, st>>>(geo, k, v, slots, n, sh.per_warp, sh.side0, err);
    else if (sh.lpr == 16) kv_write_kernel<16, BF16><<<sh.grid, kThreads, 0, st>>>(geo, k, v, slots, n, sh.per_warp, sh.side0, err);
    else if (sh.lpr == 8) kv_write_kernel<8, BF16><<<sh.grid, kThreads, 0, st>>>(geo, k, v, slots, n, sh.per_warp, sh.side0, err);
    else kv_write_kernel<4, BF16><<<sh.grid, kThreads, 0, st>>>(geo, k, v, slots, n, sh.per_warp, sh.side0, err);
}
template <bool BF16>
void run_read(const Shape& sh, const KvGeom& geo, const int64_t* slots, int64_t n, uint16_t* k, uint16_t* v, unsigned* err,
              cudaStream_t st) {
    if (sh.lpr == 32) kv_read_kernel<32, BF16><<<sh.grid, kThreads, 0, st>>>(geo, slots, n, sh.per_warp, sh.side0, k, v, err);
    else if (sh.lpr == 16) kv_read_kernel<16, BF16><<<sh.grid, kThreads, 0, st>>>(geo, slots, n, sh.per_warp, sh.side0, k, v, err);
    else if (sh.lpr == 8) kv_read_kernel<8, BF16><<<sh.grid, kThreads, 0, st>>>(geo, slots, n, sh.per_warp, sh.side0, k, v, err);
    else kv_read_kernel<4, BF16><<<sh.grid, kThreads, 0, st>>>(geo, slots, n, sh.per_warp, sh.side0, k, v, err);
}

}  // namespace

cudaError_t launch_kv_write(const KvGeom& geo, const KvRowsArg& k, const KvRowsArg& v, const int64_t* slots, int64_t n,
                            unsigned* err, cudaStream_t st) {
    Shape shapes[2];
    const int launches = make_shapes(geo, n, 48, shapes);
    if (launches == 0) return cudaErrorNotSupported;
    for (int i = 0; i < launches; ++i) {
        if (geo.bf16) run_write<true>(shapes[i], geo, k, v, slots, n, err, st);
        else run_write<false>(shapes[i], geo, k, v, slots, n, err, st);
        note_launch();
    }
    return cudaGetLastError();
}

cudaError_t launch_kv_read(const KvGeom& geo, const int64_t* slots, int64_t n, uint16_t* k, uint16_t* v, unsigned* err,
                           cudaStream_t st) {
    Shape shapes[2];
    const int launches = make_shapes(geo, n, 32, shapes);
    if (launches == 0) return cudaErrorNotSupported;
    for (int i = 0; i < launches; ++i) {
        if (geo.bf16) run_read<true>(shapes[i], geo, slots, n, k, v, err, st);
        else run_read<false>(shapes[i], geo, slots, n, k, v, err, st);
        note_launch();
    }
    return cudaGetLastError();
}

}  // namespace soniq
