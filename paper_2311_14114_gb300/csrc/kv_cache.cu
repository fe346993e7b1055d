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

enum { kRun = 0, kStaged = 1, kSingle = 2 };

template <int LPR, bool BF16>
__global__ void __launch_bounds__(kThreads) kv_write_kernel(const KvGeom geo, const KvRowsArg k, const KvRowsArg v,
                                                            const int64_t* __restrict__ slots, int64_t n, int per_warp,
                                                            unsigned* err) {
    constexpr int RPW = 32 / LPR;
    constexpr uint32_t INF = BF16 ? 0x7F80u : 0x7C00u;
    __shared__ __align__(16) uint8_t rows[kWarps][RPW][kStride];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int head = blockIdx.y, side = blockIdx.z, ql = lane & (LPR - 1);
    const KvSide& s = geo.s[side];
    const KvRowsArg& in = side ? v : k;
    const Lane me = make_lane<LPR>(s, head);
    const bool wide = (((uintptr_t)in.p | (uintptr_t)(2 * in.token_stride) | (uintptr_t)(2 * in.head_stride)) & 15u) == 0 && s.D % 8 == 0;
    const int mode = !wide ? kSingle : (__all_sync(0xffffffffu, me.run) ? kRun : kStaged);
    uint8_t* staged = rows[warp][lane / LPR];
    if (mode == kStaged && ql == 0) *reinterpret_cast<uint16_t*>(staged + 2 * s.D) = 0;      // what padding reads
    const uint16_t* base = in.p + head * in.head_stride;
    // a warp's tokens, at most 32: t_first .. t_first + count - 1; lane i holds the slot of the i-th
    const int64_t t_first = ((int64_t)blockIdx.x * kWarps + warp) * per_warp;
    if (t_first >= n) return;
    const int count = (int)min((int64_t)per_warp, n - t_first);
    const int64_t my_slot = lane < count ? __ldg(slots + t_first + lane) : -1;
    const float half = (float)(1 << (me.bits - 1));
    // the 16 bytes this lane loads of a row: its channels, or its share of the row
    const int ch16 = mode == kRun ? me.ch[0] : 8 * ql;
    const bool loads = mode != kSingle && ch16 >= 0 && ch16 < s.D;
    // rows are loaded four steps ahead of their use (the loop stays rolled: unrolled four times, with all its
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
    uint4 ahead0 = load(), ahead1 = load(), ahead2 = load(), ahead3 = load();
#pragma unroll 1
    for (int i0 = 0; i0 < count; i0 += RPW) {
        const int i_tok = i0 + lane / LPR;
        const int64_t t = t_first + i_tok;
        const uint4 raw = ahead0;
        ahead0 = ahead1;
        ahead1 = ahead2;
        ahead2 = ahead3;
        ahead3 = load();
        const int64_t slot = __shfl_sync(0xffffffffu, my_slot, i_tok & 31);
        uint32_t x[4] = {raw.x, raw.y, raw.z, raw.w};
        if (mode == kStaged) {
            __syncwarp();
            if (loads) {        // rows start on 8-byte boundaries
                *reinterpret_cast<uint2*>(staged + 2 * ch16) = make_uint2(raw.x, raw.y);
                *reinterpret_cast<uint2*>(staged + 2 * ch16 + 8) = make_uint2(raw.z, raw.w);
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const uint32_t a = *reinterpret_cast<const uint16_t*>(staged + 2 * (me.ch[i] < 0 ? s.D : me.ch[i]));
                const uint32_t b = *reinterpret_cast<const uint16_t*>(staged + 2 * (me.ch[i + 1] < 0 ? s.D : me.ch[i + 1]));
                x[i >> 1] = a | b << 16;
            }
        } else if (mode == kSingle) {
            const uint16_t* src = base + t * in.token_stride;
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
            // t = x r + (x - x r s') r with r = 2^(n-1) RN(1 / s), s' = s / 2^(n-1)
            const float r = sc == 0.0f ? 0.0f : __frcp_rn(sc) * half, sh = sc / half;
            const float2 r2 = make_float2(r, r), s2 = make_float2(-sh, -sh);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 y = make_float2(kv_load<BF16>((uint16_t)(x[i] & 0xFFFFu)), kv_load<BF16>((uint16_t)(x[i] >> 16)));
                const float2 q0 = mul2(y, r2);
                float2 q = fma2(fma2(q0, s2, y), r2, q0);
                q.x = fminf(q.x, half - 1.0f);
                q.y = fminf(q.y, half - 1.0f);
                // the integer in the low bits, rounded half to even
                q = add2(q, 12582912.0f);
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
        if (i_tok >= count || slot < 0 || !me.valid) continue;
        if (slot >= geo.n_pages * geo.page) {
            if (ql == 0) atomicOr(err, kErrKvIndex);
            continue;
        }
        const int64_t row = ((slot >> geo.page_shift) * geo.heads + head) * geo.page + (slot & (geo.page - 1));
        uint8_t* dst = s.codes + row * s.row_bytes + s.off[me.grp] + me.bits * me.q;
        if (me.bits == 4) *reinterpret_cast<uint32_t*>(dst) = w[0];
        else if (me.bits == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
        else if ((me.q & 1) == 0) *reinterpret_cast<uint32_t*>(dst) = w[0];
        if (me.q == 0) s.scales[row * s.ng + me.grp] = (uint16_t)top;
    }
}

// Eight codes of a lane as fp32, from its word(s).
__device__ __forceinline__ void unpack8(const uint32_t (&w)[2], int bits, float (&f)[8]) {
    if (bits == 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)(int8_t)(w[i >> 2] >> (8 * (i & 3)));
        return;
    }
    // codes 0..3 and 4..7 as bytes in offset binary; 2^23 + byte is that float's low bits
    const uint32_t flip = bits == 4 ? 0x08080808u : 0x02020202u, mask = bits == 4 ? 0x0F0F0F0Fu : 0x03030303u;
    const uint32_t lo = (w[0] & mask) ^ flip, hi = ((w[0] >> bits) & mask) ^ flip;
    const float off = 8388608.0f + (float)(1 << (bits - 1));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = __uint_as_float(__byte_perm(lo, 0x4B000000u, 0x7650 + i)) - off;
        f[4 + i] = __uint_as_float(__byte_perm(hi, 0x4B000000u, 0x7650 + i)) - off;
    }
}

template <int LPR, bool BF16>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(const KvGeom geo, const int64_t* __restrict__ slots, int64_t n,
                                                           int per_warp, uint16_t* k, uint16_t* v, unsigned* err) {
    constexpr int RPW = 32 / LPR;
    __shared__ __align__(16) uint8_t rows[kWarps][RPW][kStride];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int head = blockIdx.y, side = blockIdx.z, ql = lane & (LPR - 1);
    const KvSide& s = geo.s[side];
    uint16_t* out = side ? v : k;
    if (out == nullptr) return;
    const Lane me = make_lane<LPR>(s, head);
    const bool wide = ((uintptr_t)out & 15u) == 0 && s.D % 8 == 0;
    const int mode = !wide ? kSingle : (__all_sync(0xffffffffu, me.run) ? kRun : kStaged);
    uint8_t* staged = rows[warp][lane / LPR];
    const int64_t t_first = ((int64_t)blockIdx.x * kWarps + warp) * per_warp;
    if (t_first >= n) return;
    const int count = (int)min((int64_t)per_warp, n - t_first);
    const int64_t my_slot = lane < count ? __ldg(slots + t_first + lane) : -1;
    const float unit = 1.0f / (float)(1 << (me.bits - 1));
    const int at = s.off[me.grp] + (me.bits == 2 ? 4 * (me.q >> 1) : me.bits * me.q);
    // packed words and scales are loaded four steps ahead of their use
    struct Packed {
        uint32_t w0, w1, sc;
    };
    int i_load = lane / LPR;
    auto load = [&]() {
        Packed r{0u, 0u, 0u};
        const int64_t slot = __shfl_sync(0xffffffffu, my_slot, i_load & 31);
        if (i_load < count && me.valid && slot >= 0) {
            if (slot >= geo.n_pages * geo.page) {
                if (ql == 0) atomicOr(err, kErrKvIndex);
            } else {
                const int64_t row = ((slot >> geo.page_shift) * geo.heads + head) * geo.page + (slot & (geo.page - 1));
                const uint8_t* src = s.codes + row * s.row_bytes + at;
                r.w0 = *reinterpret_cast<const uint32_t*>(src);
                if (me.bits == 8) r.w1 = *reinterpret_cast<const uint32_t*>(src + 4);
                r.sc = s.scales[row * s.ng + me.grp];
            }
        }
        i_load += RPW;
        return r;
    };
    Packed ahead0 = load(), ahead1 = load(), ahead2 = load(), ahead3 = load();
#pragma unroll 1
    for (int i0 = 0; i0 < count; i0 += RPW) {
        const int i_tok = i0 + lane / LPR;
        const int64_t t = t_first + i_tok;
        uint32_t w[2] = {ahead0.w0, ahead0.w1};
        const float u = kv_load<BF16>((uint16_t)ahead0.sc) * unit;
        ahead0 = ahead1;
        ahead1 = ahead2;
        ahead2 = ahead3;
        ahead3 = load();
        if (me.bits == 2) w[0] = w[0] >> (4 * (me.q & 1)) & 0x0F0F0F0Fu;
        float f[8];
        unpack8(w, me.bits, f);
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 z = mul2(make_float2(f[2 * i], f[2 * i + 1]), make_float2(u, u));
            y[i] = kv_round<BF16>(z.x) | (uint32_t)kv_round<BF16>(z.y) << 16;
        }
        uint16_t* dst = out + (t * geo.heads + head) * s.D;
        const bool on = i_tok < count && me.valid;
        if (mode == kRun) {
            if (on && me.ch[0] >= 0) *reinterpret_cast<uint4*>(dst + me.ch[0]) = make_uint4(y[0], y[1], y[2], y[3]);
        } else if (mode == kStaged) {
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (me.ch[i] >= 0) *reinterpret_cast<uint16_t*>(staged + 2 * me.ch[i]) = (uint16_t)pattern(y, i);
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
    }
}

// Lanes to a row, and tokens to a warp: enough warps for the machine first, then
// runs of tokens that repay looking up the channels.
struct Shape {
    int lpr, per_warp;
    dim3 grid;
};
bool make_shape(const KvGeom& geo, int64_t n, Shape* sh) {
    int eighths = 0;
    for (const KvSide& s : geo.s) eighths = 4 * (s.nb[0] + s.nb[1]) > eighths ? 4 * (s.nb[0] + s.nb[1]) : eighths;
    sh->lpr = 4;
    while (sh->lpr < eighths) sh->lpr *= 2;
    const int64_t rpw = 32 / sh->lpr, steps = (n + rpw - 1) / rpw * geo.heads * 2;
    int64_t iters = steps / ((int64_t)num_sms() * 64);
    sh->per_warp = (int)(iters * rpw < rpw ? rpw : (iters * rpw > 32 ? 32 : iters * rpw));      // a warp holds 32 slots
    const int64_t blocks = (n + (int64_t)kWarps * sh->per_warp - 1) / ((int64_t)kWarps * sh->per_warp);
    if (blocks > 2147483647) return false;
    sh->grid = dim3((unsigned)blocks, (unsigned)geo.heads, 2);
    return true;
}

template <bool BF16>
void run_write(const Shape& sh, const KvGeom& geo, const KvRowsArg& k, const KvRowsArg& v, const int64_t* slots, int64_t n,
               unsigned* err, cudaStream_t st) {
    if (sh.lpr == 32) kv_write_kernel<32, BF16><<<sh.grid, kThreads, 0, st>>>(geo, k, v, slots, n, sh.per_warp, err);
    else if (sh.lpr == 16) kv_write_kernel<16, BF16><<<sh.grid, kThreads, 0, st>>>(geo, k, v, slots, n, sh.per_warp, err);
    else if (sh.lpr == 8) kv_write_kernel<8, BF16><<<sh.grid, kThreads, 0, st>>>(geo, k, v, slots, n, sh.per_warp, err);
    else kv_write_kernel<4, BF16><<<sh.grid, kThreads, 0, st>>>(geo, k, v, slots, n, sh.per_warp, err);
}
template <bool BF16>
void run_read(const Shape& sh, const KvGeom& geo, const int64_t* slots, int64_t n, uint16_t* k, uint16_t* v, unsigned* err,
              cudaStream_t st) {
    if (sh.lpr == 32) kv_read_kernel<32, BF16><<<sh.grid, kThreads, 0, st>>>(geo, slots, n, sh.per_warp, k, v, err);
    else if (sh.lpr == 16) kv_read_kernel<16, BF16><<<sh.grid, kThreads, 0, st>>>(geo, slots, n, sh.per_warp, k, v, err);
    else if (sh.lpr == 8) kv_read_kernel<8, BF16><<<sh.grid, kThreads, 0, st>>>(geo, slots, n, sh.per_warp, k, v, err);
    else kv_read_kernel<4, BF16><<<sh.grid, kThreads, 0, st>>>(geo, slots, n, sh.per_warp, k, v, err);
}

}  // namespace

cudaError_t launch_kv_write(const KvGeom& geo, const KvRowsArg& k, const KvRowsArg& v, const int64_t* slots, int64_t n,
                            unsigned* err, cudaStream_t st) {
    Shape sh;
    if (!make_shape(geo, n, &sh)) return cudaErrorNotSupported;
    if (geo.bf16) run_write<true>(sh, geo, k, v, slots, n, err, st);
    else run_write<false>(sh, geo, k, v, slots, n, err, st);
    note_launch();
    return cudaGetLastError();
}

cudaError_t launch_kv_read(const KvGeom& geo, const int64_t* slots, int64_t n, uint16_t* k, uint16_t* v, unsigned* err,
                           cudaStream_t st) {
    Shape sh;
    if (!make_shape(geo, n, &sh)) return cudaErrorNotSupported;
    if (geo.bf16) run_read<true>(sh, geo, slots, n, k, v, err, st);
    else run_read<false>(sh, geo, slots, n, k, v, err, st);
    note_launch();
    return cudaGetLastError();
}

}  // namespace soniq
