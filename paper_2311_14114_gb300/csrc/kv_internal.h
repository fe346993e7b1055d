// Geometry of a key / value cache as its kernels see it, and their launchers.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "soniq_internal.h"

namespace soniq {

// One side (keys or values): a packed row is [group 0 blocks][group 1 blocks],
// padded to 16 bytes.
struct KvSide {
    int32_t D;
    int32_t ng;
    int32_t count[2];
    int32_t nb[2];       // 32-code blocks of a group
    int32_t bits[2];
    int32_t off[2];      // byte offset of a group in a row
    int32_t row_bytes;
    const int32_t* perm; // [heads][D]
    uint8_t* codes;
    uint16_t* scales;    // [..][ng], the cache's 16-bit type
};

struct KvGeom {
    int32_t heads;
    int32_t page;        // tokens per page, a power of two
    int32_t page_shift;
    int32_t bf16;
    int64_t n_pages;
    KvSide s[2];         // keys, values
};

// Most packed codes of a row (both groups, padded).
constexpr int kKvMaxCodes = 256;

struct KvRowsArg {       // caller tensors [token][head][channel], strides in elements
    const uint16_t* p;
    int64_t token_stride;
    int64_t head_stride;
};

struct KvAttendArgs {
    const uint16_t* Q;
    int64_t q_seq_stride, q_token_stride, q_head_stride;
    const int32_t* table;
    int64_t table_stride;
    int32_t max_pages;
    const int32_t* lengths;
    const uint8_t* mask;      // or null: token t sees tokens 0..t
    int64_t mask_stride;
    int32_t B, T, group;      // group: query heads per key head
    float scale;
    uint16_t* out;
    void* scratch;
    unsigned* err;
    int32_t drop;             // test hook: the first copy is left out
};

soniq_status make_kv_geom(const soniq_kv_cache* c, KvGeom* geo);

cudaError_t launch_kv_write(const KvGeom& geo, const KvRowsArg& k, const KvRowsArg& v, const int64_t* slots, int64_t n,
                            unsigned* err, cudaStream_t st);
cudaError_t launch_kv_read(const KvGeom& geo, const int64_t* slots, int64_t n, uint16_t* k, uint16_t* v, unsigned* err,
                           cudaStream_t st);
cudaError_t launch_kv_attend(const KvGeom& geo, const KvAttendArgs& a, cudaStream_t st);
int64_t kv_attend_scratch(const KvGeom& geo, int64_t B, int64_t T, int64_t group);
// Many query rows per key head (kv_tile.cu).
bool kv_tile_supported(const KvGeom& geo, int64_t T, int64_t group);
int64_t kv_tile_scratch(const KvGeom& geo, int64_t T, int64_t group);
cudaError_t launch_kv_tile(const KvGeom& geo, const KvAttendArgs& a, cudaStream_t st);

#ifdef __CUDACC__
// The cache's 16-bit types as fp32, and back with one rounding.
template <bool BF16>
__device__ __forceinline__ float kv_load(uint16_t x) {
    if constexpr (BF16) return __uint_as_float((uint32_t)x << 16);
    else return __half2float(__ushort_as_half(x));
}
template <bool BF16>
__device__ __forceinline__ uint16_t kv_round(float x) {
    if constexpr (BF16) return __bfloat16_as_ushort(__float2bfloat16_rn(x));
    else return __half_as_ushort(__float2half_rn(x));
}
#endif

}  // namespace soniq
