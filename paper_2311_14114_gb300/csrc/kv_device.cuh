// Device helpers and tensor maps shared by the attention kernels.
#pragma once

#include <cuda.h>

#include "kv_internal.h"
#include "tc_ptx.cuh"

namespace soniq {

constexpr float kLog2e = 1.4426950408889634f;
constexpr long long kWaitNs = 2000000000ll;   // bound of a wait for a copy

// Tiled copies of packed rows (x: byte, y: row of the page's heads, z: page) and
// of scales (x: entry of the page's heads, y: page); a page outside the cache
// reads as zeros.
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

__device__ __forceinline__ uint32_t lds16(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}

__device__ __forceinline__ float lds32f(uint32_t a) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float4 lds128f(uint32_t a) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void sts128f(uint32_t a, float x, float y, float z, float w) {
    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(x), "f"(y), "f"(z), "f"(w) : "memory");
}

// d (16 x 8, fp32) += a (16 x 16) b (16 x 8)
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 x 8 transpose of halves over the warp
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// (x & m) ^ f in one instruction (written out, as two constants otherwise make two)
__device__ __forceinline__ uint32_t mask_flip(uint32_t x, uint32_t m, uint32_t f) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(r) : "r"(x), "r"(m), "r"(f));
    return r;
}

__device__ __forceinline__ float scale_of(uint32_t bits16, bool bf16) {
    return bf16 ? __uint_as_float(bits16 << 16) : __half2float(__ushort_as_half((uint16_t)bits16));
}
// A cached value scale.  One that no write leaves (negative, not finite) counts as 0: it may stand behind a token
// that no row sees, and 0 times it would not be 0.
__device__ __forceinline__ float value_scale(uint32_t bits16, bool bf16) {
    const float x = scale_of(bits16, bf16);
    return x >= 0.0f && x < INFINITY ? x : 0.0f;
}
// 1 / a softmax sum; nothing seen: 0; NaN stays.
__device__ __forceinline__ float inverse(float l) { return l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l); }
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127
__device__ __forceinline__ float lg2(float x) {
    float r;
    asm("lg2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// How weights become fp16.  With a row's running maximum m (of scores in units of
// the exponent) a token's weight is p = 2^(score - m); its products with the codes
// carry the value scale s.  A row (and value group) rounds p s 2^-power to fp16 and
// sums outputs in that unit.  The power is a whole number that follows the products
// p s of the tokens that the row sees: it is raised to the largest where that
// exceeds 2^15 of it, and falls by m's raises, in whole steps; the outputs take the
// rest.  (It is -110 at least, where a row begins.)  So a weight of 1 costs its
// scale nothing, and rounding costs a row 2^-11 of each other product, or 2^-25 of
// its largest, whatever stands in tokens that it does not see, or hardly weighs.
// (With a power common to all rows of a block, over all of its scales, one scale of
// 2^16 times the others' cost the rest 2 % of their weights.)
// Finding the largest product takes a pass over the tokens, so it is done only
// where the bound from the largest scale of the block and the row's largest score
// leaves the range.
constexpr float kUnset = -3.402823466e+38f;      // maximum of no token seen
constexpr float kRoom = 15.0f;
constexpr float kLeast = -110.0f;                // smallest power: weights (up to 2^13) times its inverse stay floats

// log2 of the largest value scale of a block, from its bits (none: far below any product), at most 0.09 too large:
// log2(1 + f) is f to f + 0.0861.
__device__ __forceinline__ float scale_bound(uint32_t bits) { return fmaf((float)bits, 0x1p-23f, -126.91f); }
// ... and at most that of the smallest.
__device__ __forceinline__ float scale_floor(uint32_t bits) { return fmaf((float)bits, 0x1p-23f, -127.0f); }
// The factor of a row's scores, whose largest in the block is `best`, that takes them to units of the exponent.
// score * factor - m is one rounding; m is that of a rounded product.  Up to 2^30 the two are within 2^5 of each other,
// which weights have room for, and which the row's lead over m counts.  Beyond, different scores are 2^6 or more apart,
// so any factor of that size leaves one weight, or equal ones: a power of two makes the products exact.  (The next one
// above, so that scores stay in order with those of other blocks.)
__device__ __forceinline__ float exponent_factor(float factor, float best) {
    const float whole = __uint_as_float((__float_as_uint(factor) + 0x007FFFFFu) & 0x7F800000u);
    return fabsf(best * factor) > 0x1p30f ? whole : factor;
}
// Raises a row's maximum to its block's `top` if it is to; returns by how much.
__device__ __forceinline__ float raise(float& m, float top, bool is_to) {
    const float to = is_to ? top : m, by = to - m;
    m = to;
    return by;
}
__device__ __forceinline__ float factor_of(float by) { return by < -126.0f ? 0.0f : pow2((int)by); }      // 2^by, a whole by <= 0
// A raise of the maximum in whole steps, and the factor that is too much.  (Rounded up: the unit never rises but to a
// product, or to stay above the smallest.  From 2^23 on floats are whole.)
__device__ __forceinline__ float whole_steps(float by) { return by < 0x1p23f ? ceilf(by) : by; }
__device__ __forceinline__ float rest_of(float by) { return by < 0x1p23f ? ex2(ceilf(by) - by) : 1.0f; }
// Brings a lowered power up to the smallest; returns the factor of what is summed so far.
__device__ __forceinline__ float floor_power(float& power) {
    const float from = power;
    power = fmaxf(from, kLeast);
    return factor_of(from - power);
}
// Raises a power to the largest product, 2^most, if it is to; returns the factor of what is summed so far.
// (126 at most: products reach 2^128, and both 2^power and its inverse are floats.)
__device__ __forceinline__ float raise_power(float& power, float most, bool is_to) {
    const float to = is_to ? fminf(ceilf(most), 126.0f) : power, by = power - to;
    power = to;
    return factor_of(by);
}
// 2^power, and 2^-power through the integer in a float's low bits.
__device__ __forceinline__ float power_of(float power) { return pow2((int)power); }
__device__ __forceinline__ float unit_of(float power) { return __uint_as_float(__float_as_uint(12582912.0f + 127.0f - power) << 23); }

// Eight codes of a block, its l-th quarter, unpack to four half pairs: which codes
// they are, and the powers of two their places in the word give them.
__device__ __forceinline__ int key_code(int bits, int l, int i, int half) {
    if (bits == 8) return 8 * l + 4 * (i >> 1) + (i & 1) + 2 * half;
    if (bits == 4) return 8 * l + 4 * (i & 1) + (i >> 1) + 2 * half;
    return 16 * (l >> 1) + 4 * i + 2 * (l & 1) + half;
}
__device__ __forceinline__ int place_log2(int bits, int i) { return bits == 8 ? 0 : (bits == 4 ? 4 * (i & 1) : 2 * i); }

// The offsets 1024 + 8 and 1024 + 128 as half pairs, in registers: a logic
// instruction has room for one constant, and the compiler would move the other
// one in before each use.
struct Offsets {
    uint32_t c8, c128;
    __device__ __forceinline__ Offsets() {
        asm volatile("mov.b32 %0, 0x64086408;" : "=r"(c8));
        asm volatile("mov.b32 %0, 0x64806480;" : "=r"(c128));
    }
};

// 4-bit codes of two tokens, 4 from each half of w
__device__ __forceinline__ void nibble_pairs(uint32_t w, const Offsets& f, uint32_t (&x)[4]) {
    x[0] = sub2(mask_flip(w, 0x000F000Fu, f.c8), f.c8);
    x[1] = sub2(mask_flip(w, 0x00F000F0u, f.c128), f.c128);
    w >>= 8;
    x[2] = sub2(mask_flip(w, 0x000F000Fu, f.c8), f.c8);
    x[3] = sub2(mask_flip(w, 0x00F000F0u, f.c128), f.c128);
}


// The cache's tensor maps: keys, values.
struct KvMaps {
    CUtensorMap codes[2], scales[2];
};

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_fn() {
    static const EncodeTiledFn fn = [] {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        const bool ok = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault, &q) ==
                            cudaSuccess && q == cudaDriverEntryPointSuccess;
        return ok ? reinterpret_cast<EncodeTiledFn>(ptr) : nullptr;
    }();
    return fn;
}

// Tensor maps of a side: codes as [pages][rows of all heads][row bytes], in boxes
// of box_rows rows by box_bytes; scales as [pages][entries of all heads].
inline bool encode_side(const KvGeom& geo, const KvSide& s, int box_bytes, int box_rows, CUtensorMapSwizzle swizzle,
                        CUtensorMap* codes, CUtensorMap* scales) {
    const EncodeTiledFn enc = encode_fn();
    if (enc == nullptr) return false;
    const cuuint32_t step[3] = {1, 1, 1};
    const cuuint64_t rows = (cuuint64_t)geo.heads * geo.page;
    const cuuint64_t dims[3] = {(cuuint64_t)s.row_bytes, rows, (cuuint64_t)geo.n_pages};
    const cuuint64_t strides[2] = {(cuuint64_t)s.row_bytes, rows * s.row_bytes};
    const cuuint32_t box[3] = {(cuuint32_t)box_bytes, (cuuint32_t)box_rows, 1};
    if (enc(codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, s.codes, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return false;
    const cuuint64_t sdims[2] = {rows * s.ng, (cuuint64_t)geo.n_pages};
    const cuuint64_t sstrides[1] = {rows * s.ng * 2};
    const cuuint32_t sbox[2] = {(cuuint32_t)(box_rows * s.ng), 1};
    return enc(scales, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, s.scales, sdims, sstrides, sbox, step,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}


}  // namespace soniq
