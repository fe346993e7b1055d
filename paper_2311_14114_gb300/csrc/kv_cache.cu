// Key / value cache: rows quantized as they are written, and read back.
//
// A row is one token's key (or value) of one head.  Per precision group g of
// its channels: s_g = max|x|, j = clamp(rne(x / s_g * 2^(n-1)), -2^(n-1),
// 2^(n-1) - 1) (Eq. (1)), packed in 32-code blocks (layout: soniq.h).
#include "kv_internal.h"
#include "soniq_device.cuh"

namespace soniq {

namespace {

constexpr int kThreads = 256;

// Largest finite value of the cache's type; infinities count as it.
template <bool BF16>
__device__ __forceinline__ float kv_clean(float x) {
    constexpr float top = BF16 ? 0x1.FEp127f : 65504.0f;
    return x != x ? 0.0f : fminf(fmaxf(x, -top), top);
}

// One warp per row; lane i forms code i of each block.
template <bool BF16>
__global__ void __launch_bounds__(kThreads) kv_write_kernel(const KvGeom geo, const KvRowsArg k, const KvRowsArg v,
                                                            const int64_t* __restrict__ slots, int64_t n, unsigned* err) {
    const int lane = threadIdx.x & 31;
    const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
    if (w >= n * geo.heads * 2) return;
    const int side = (int)(w & 1);
    const int head = (int)((w >> 1) % geo.heads);
    const int64_t i = (w >> 1) / geo.heads;
    const KvSide& s = geo.s[side];
    const KvRowsArg& in = side ? v : k;
    const int64_t slot = slots[i];
    if (slot < 0) return;
    if (slot >= geo.n_pages * geo.page) {
        if (lane == 0) atomicOr(err, kErrKvIndex);
        return;
    }
    const int64_t row = ((slot >> geo.page_shift) * geo.heads + head) * geo.page + (slot & (geo.page - 1));
    const uint16_t* x = in.p + i * in.token_stride + head * in.head_stride;
    const int32_t* perm = s.perm + head * s.D;
    int pos = 0;
    for (int g = 0; g < s.ng; ++g) {
        float m = 0.0f;
        for (int p = lane; p < s.count[g]; p += 32) m = fmaxf(m, fabsf(kv_clean<BF16>(kv_load<BF16>(x[perm[pos + p]]))));
        m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
        const float half = (float)(1 << (s.bits[g] - 1));
        for (int b = 0; b < s.nb[g]; ++b) {
            const int p = 32 * b + lane;
            int32_t j = 0;
            if (p < s.count[g]) j = weight_code(kv_clean<BF16>(kv_load<BF16>(x[perm[pos + p]])), m, half);
            const uint32_t word = pack_block_warp((uint32_t)j & ((1u << s.bits[g]) - 1u), s.bits[g]);
            uint32_t* dst = reinterpret_cast<uint32_t*>(s.codes + row * s.row_bytes + s.off[g] + 4 * s.bits[g] * b);
            if (lane < s.bits[g]) dst[lane] = word;
        }
        if (lane == 0) s.scales[row * s.ng + g] = kv_round<BF16>(m);
        pos += s.count[g];
    }
}

// Signed code at position p of the block at src.
__device__ __forceinline__ int kv_code(const uint8_t* src, int bits, int p) {
    const int t = p >> 2, per = 8 / bits;
    const int byte = src[4 * (t / per) + (p & 3)];
    const int u = (byte >> (bits * (t % per))) & ((1 << bits) - 1);
    return (u ^ (1 << (bits - 1))) - (1 << (bits - 1));
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(const KvGeom geo, const int64_t* __restrict__ slots, int64_t n,
                                                           uint16_t* k, uint16_t* v, unsigned* err) {
    const int lane = threadIdx.x & 31;
    const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
    if (w >= n * geo.heads * 2) return;
    const int side = (int)(w & 1);
    const int head = (int)((w >> 1) % geo.heads);
    const int64_t i = (w >> 1) / geo.heads;
    const KvSide& s = geo.s[side];
    uint16_t* out = side ? v : k;
    if (out == nullptr) return;
    out += (i * geo.heads + head) * s.D;
    const int64_t slot = slots[i];
    const bool in = slot >= 0 && slot < geo.n_pages * geo.page;
    if (!in) {
        if (slot >= 0 && lane == 0) atomicOr(err, kErrKvIndex);
        for (int c = lane; c < s.D; c += 32) out[c] = 0;
        return;
    }
    const int64_t row = ((slot >> geo.page_shift) * geo.heads + head) * geo.page + (slot & (geo.page - 1));
    const int32_t* perm = s.perm + head * s.D;
    int pos = 0;
    for (int g = 0; g < s.ng; ++g) {
        const float unit = kv_load<BF16>(s.scales[row * s.ng + g]) / (float)(1 << (s.bits[g] - 1));
        for (int p = lane; p < s.count[g]; p += 32) {
            const uint8_t* block = s.codes + row * s.row_bytes + s.off[g] + 4 * s.bits[g] * (p >> 5);
            out[perm[pos + p]] = kv_round<BF16>(unit * (float)kv_code(block, s.bits[g], p & 31));
        }
        pos += s.count[g];
    }
}

unsigned row_blocks(const KvGeom& geo, int64_t n) {
    const int64_t blocks = (n * geo.heads * 2 * 32 + kThreads - 1) / kThreads;
    return blocks > 2147483647 ? 0u : (unsigned)blocks;
}

}  // namespace

cudaError_t launch_kv_write(const KvGeom& geo, const KvRowsArg& k, const KvRowsArg& v, const int64_t* slots, int64_t n,
                            unsigned* err, cudaStream_t st) {
    const unsigned blocks = row_blocks(geo, n);
    if (blocks == 0) return cudaErrorNotSupported;
    if (geo.bf16) kv_write_kernel<true><<<blocks, kThreads, 0, st>>>(geo, k, v, slots, n, err);
    else kv_write_kernel<false><<<blocks, kThreads, 0, st>>>(geo, k, v, slots, n, err);
    note_launch();
    return cudaGetLastError();
}

cudaError_t launch_kv_read(const KvGeom& geo, const int64_t* slots, int64_t n, uint16_t* k, uint16_t* v, unsigned* err,
                           cudaStream_t st) {
    const unsigned blocks = row_blocks(geo, n);
    if (blocks == 0) return cudaErrorNotSupported;
    if (geo.bf16) kv_read_kernel<true><<<blocks, kThreads, 0, st>>>(geo, slots, n, k, v, err);
    else kv_read_kernel<false><<<blocks, kThreads, 0, st>>>(geo, slots, n, k, v, err);
    note_launch();
    return cudaGetLastError();
}

}  // namespace soniq
