// Attention of a few query rows per key head over the quantized cache.
//
//   out = sum_p softmax_p(scale q . k_p) v_p,  k_p = s j / 2^(n-1) per group
//
// A decoding step reads every visible row once (about 150 bytes per token and
// head at 4 bits) for a handful of query rows, so bytes bound it; next comes
// unpacking, whose instructions are counted below.  Design:
//  * Work is the list of (sequence, key head, row tile, 32-token chunk), cut in
//    equal contiguous ranges, one per CTA, by lengths read on the device:
//    ragged batches balance and long sequences spread over all SMs.  A CTA's
//    warps take the chunks of a range in turn, each with its own ring of
//    shared-memory stages (cp.async) and its own running maximum, sum and
//    outputs, joined at the end of a range; ranges that share an item leave
//    partial results in scratch, and the last of them joins those in order.
//  * Products run transposed on mma.sync m16n8k16 (fp16, fp32 sums): scores =
//    K (16 tokens x 16 channels) x Q^T (8 rows), outputs = V^T (16 channels x
//    16 tokens) x P^T, so 8 query rows fill the instruction, and codes go
//    straight from packed words to A fragments.
//  * Key codes are used as fp16 subnormals: a code's bits in the low bits of a
//    half are u 2^-24 exactly (u 2^-20 for the nibble above), u = j + 2^(n-1).
//    One logic instruction makes two operands; powers of two are divided out of
//    the staged queries, and the offset's share, 2^(n-1) sum(q), is the
//    accumulators' start value.  Value codes are made signed (one more
//    instruction): their sums run over tokens, where the offset would swamp a
//    small average.
//  * Queries are scaled per row by a power of two to 2^13 (bf16 queries are
//    exact in fp16 then), softmax weights times value scales by a running power
//    of two (the largest scale met), so no range of either type is lost.
#include "kv_internal.h"
#include <type_traits>

#include "tc_ptx.cuh"

namespace soniq {

namespace {

constexpr int kChunk = 32;                   // tokens a warp takes at a time
constexpr int kMergeBytes = 32768;           // outputs of all warps, in as many passes as they need
constexpr float kLog2e = 1.4426950408889634f;

// How a warp copies 16 packed rows of one side into shared rows whose stride is
// an odd multiple of 16 bytes (so that lanes reading one place of eight rows
// meet eight bank groups).  Rows of an odd number of 16-byte pieces go as one
// run; others with 2^shift >= pieces lanes to a row.
struct CopyPlan {
    int stride;          // bytes of a shared row
    int shift;           // -1: one run
    int iters, dst_step, src_step;
    uint32_t page_bytes;         // codes of one page (all heads)
    uint32_t page_scales;        // scales of one page, bytes
};

struct RowsPlan {
    int row_tiles;        // tiles of 8 NT query rows per key head
    int rows;             // query rows per key head: T * group
    int stages;
    int stage_bytes;
    CopyPlan cp[2];
    int v_off, ks_off, vs_off;   // in a stage
    int f_off;            // fp32 scales of a warp's chunk, behind its stages
    int warp_bytes;       // a warp's stages and scales
    int q_off, misc_off;
    int smem;
    int min_chunks;       // fewest chunks worth a CTA
};

__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the newest `newer` groups of this thread have landed.
__device__ __forceinline__ void cp_wait(int newer) {
    if (newer >= 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (newer == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
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

// The key side: a quad's lane l holds 8 codes of a block as four half pairs
// h[0..3].  Codes of h[i] and the powers of two their place gives them:
__device__ __forceinline__ int key_code(int bits, int l, int i, int half) {
    if (bits == 8) return 8 * l + 4 * (i >> 1) + (i & 1) + 2 * half;
    if (bits == 4) return 8 * l + 4 * (i & 1) + (i >> 1) + 2 * half;
    return 16 * (l >> 1) + 4 * i + 2 * (l & 1) + half;
}
__device__ __forceinline__ int place_log2(int bits, int i) { return bits == 8 ? 0 : (bits == 4 ? 4 * (i & 1) : 2 * i); }

// ... as u 2^-24 times the place's power; `at`: the lane's bytes of the block.
template <int BITS>
__device__ __forceinline__ void key_halves(uint32_t at, uint32_t (&h)[4]) {
    if constexpr (BITS == 8) {
        const uint2 w = lds64(at);
        h[0] = (w.x & 0x00FF00FFu) ^ 0x00800080u;
        h[1] = ((w.x >> 8) & 0x00FF00FFu) ^ 0x00800080u;
        h[2] = (w.y & 0x00FF00FFu) ^ 0x00800080u;
        h[3] = ((w.y >> 8) & 0x00FF00FFu) ^ 0x00800080u;
    } else if constexpr (BITS == 4) {
        uint32_t w = lds32(at);
        h[0] = (w & 0x000F000Fu) ^ 0x00080008u;
        h[1] = (w & 0x00F000F0u) ^ 0x00800080u;
        w >>= 8;
        h[2] = (w & 0x000F000Fu) ^ 0x00080008u;
        h[3] = (w & 0x00F000F0u) ^ 0x00800080u;
    } else {
        const uint32_t w = __byte_perm(lds16(at), 0, 0x4140);
        h[0] = (w & 0x00030003u) ^ 0x00020002u;
        h[1] = (w & 0x000C000Cu) ^ 0x00080008u;
        h[2] = (w & 0x00300030u) ^ 0x00200020u;
        h[3] = (w & 0x00C000C0u) ^ 0x00800080u;
    }
}

// The value side: lane group g of a warp holds 4 codes of a block, each as the
// pair (token t, token t + 1), signed, times the place's power; row0, row1: its
// bytes of the block in the two rows.
__device__ __forceinline__ int value_code(int bits, int g, int i) {
    if (bits == 8) return 4 * g + i;
    if (bits == 4) return 8 * (g >> 1) + 2 * (g & 1) + 4 * (i & 1) + (i >> 1);
    return 16 * (g >> 2) + 4 * i + (g & 3);
}

template <int BITS>
__device__ __forceinline__ void value_pairs(uint32_t row0, uint32_t row1, uint32_t (&x)[4]) {
    if constexpr (BITS == 8) {
        const uint32_t a = lds32(row0), b = lds32(row1);
        x[0] = sub2((__byte_perm(a, b, 0x4400) & 0x00FF00FFu) ^ 0x64806480u, 0x64806480u);
        x[1] = sub2((__byte_perm(a, b, 0x5511) & 0x00FF00FFu) ^ 0x64806480u, 0x64806480u);
        x[2] = sub2((__byte_perm(a, b, 0x6622) & 0x00FF00FFu) ^ 0x64806480u, 0x64806480u);
        x[3] = sub2((__byte_perm(a, b, 0x7733) & 0x00FF00FFu) ^ 0x64806480u, 0x64806480u);
    } else if constexpr (BITS == 4) {
        uint32_t w = __byte_perm(lds16(row0), lds16(row1), 0x5410);
        x[0] = sub2((w & 0x000F000Fu) ^ 0x64086408u, 0x64086408u);
        x[1] = sub2((w & 0x00F000F0u) ^ 0x64806480u, 0x64806480u);
        w >>= 8;
        x[2] = sub2((w & 0x000F000Fu) ^ 0x64086408u, 0x64086408u);
        x[3] = sub2((w & 0x00F000F0u) ^ 0x64806480u, 0x64806480u);
    } else {
        const uint32_t w = __byte_perm(lds8(row0), lds8(row1), 0x5410);
        x[0] = sub2((w & 0x00030003u) ^ 0x64026402u, 0x64026402u);
        x[1] = sub2((w & 0x000C000Cu) ^ 0x64086408u, 0x64086408u);
        x[2] = sub2((w & 0x00300030u) ^ 0x64206420u, 0x64206420u);
        x[3] = sub2((w & 0x00C000C0u) ^ 0x64806480u, 0x64806480u);
    }
}

__device__ __forceinline__ float scale_of(uint32_t bits16, bool bf16) {
    return bf16 ? __uint_as_float(bits16 << 16) : __half2float(__ushort_as_half((uint16_t)bits16));
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// Chunks of sequence b; the tokens it shows end at `end`.
__device__ __forceinline__ int64_t seen_end(const KvGeom& geo, const KvAttendArgs& a, int b) {
    const int len = a.lengths[b];
    if (len < 0) return 0;
    const int64_t cap = (int64_t)a.max_pages << geo.page_shift, end = (int64_t)len + a.T;
    return end < cap ? end : cap;
}
// At least one for a present sequence, so that its rows are written.
__device__ __forceinline__ int chunks_of(const KvGeom& geo, const KvAttendArgs& a, int b) {
    if (a.lengths[b] < 0) return 0;
    const int64_t end = seen_end(geo, a, b);
    return end == 0 ? 1 : (int)((end + kChunk - 1) / kChunk);
}

template <int NT, int NVB>
constexpr int min_ctas() { return NT * NVB <= 4 ? 2 : 1; }

// WIDE: group 0 of both sides has 4-bit codes and group 1, where there is one,
// 8-bit codes; otherwise the widths are looked up block by block.
template <int NT, int NVB, bool WIDE>
__global__ void __launch_bounds__(256, (min_ctas<NT, NVB>())) kv_rows_kernel(const KvGeom geo, const KvAttendArgs a,
                                                                          const RowsPlan pl) {
    extern __shared__ __align__(128) uint8_t smem[];
    constexpr int R = 8 * NT;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
    const int g = lane >> 2, l = lane & 3;
    const KvSide &ks = geo.s[0], &vs = geo.s[1];
    const int nkb = ks.nb[0] + ks.nb[1], nvb = vs.nb[0] + vs.nb[1];
    const bool bf16 = geo.bf16 != 0;
    const uint32_t smem0 = tc::smem_u32(smem);
    const uint32_t ring = smem0 + warp * pl.warp_bytes, fsc = ring + pl.f_off;
    float* merge = reinterpret_cast<float*>(smem);       // over the rings, which are empty when it is used
    // misc: per (row, group) start value, per row factor, the warps' statistics, the head's value channels
    float* sm_init = reinterpret_cast<float*>(smem + pl.misc_off);   // [2][R]
    float* sm_fac = sm_init + 2 * R;                                 // [R]
    float* sm_m = sm_fac + R;                                        // [8][R]
    float* sm_l = sm_m + 8 * R;                                      // [8][R]
    int16_t* sm_chan = reinterpret_cast<int16_t*>(sm_l + 8 * R);     // [32 NVB]
    __shared__ long long sm_scan[8];
    __shared__ long long sm_base;
    __shared__ int sm_b, sm_last;

    // ---- this CTA's range of chunks --------------------------------------
    const int hr = geo.heads * pl.row_tiles;
    long long total = 0;
    for (int b = tid; b < a.B; b += blockDim.x) {
        const int n = chunks_of(geo, a, b);
        total += n;
        if (n != 0 && blockIdx.x == 0 && (int64_t)a.lengths[b] + a.T > ((int64_t)a.max_pages << geo.page_shift))
            atomicOr(a.err, kErrKvIndex);
    }
    // outputs of absent sequences
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        if (a.lengths[b] >= 0) continue;
        const int64_t size = (int64_t)a.T * a.group * geo.heads * vs.D;
        for (int64_t i = tid; i < size; i += blockDim.x) a.out[b * size + i] = 0;
    }
    for (int i = 16; i; i >>= 1) total += __shfl_xor_sync(0xffffffffu, total, i);
    if (lane == 0) sm_scan[warp] = total;
    __syncthreads();
    total = 0;
    for (int w = 0; w < n_warps; ++w) total += sm_scan[w];
    total *= hr;
    if (total == 0) return;
    const long long by_size = (total + pl.min_chunks - 1) / pl.min_chunks;
    const long long n_cta = by_size < gridDim.x ? by_size : gridDim.x;
    if (blockIdx.x >= n_cta) return;
    const long long lo = total * blockIdx.x / n_cta, hi = total * (blockIdx.x + 1) / n_cta;
    // the sequence of chunk lo
    {
        long long run = 0;
        for (int b0 = 0; b0 < a.B; b0 += blockDim.x) {
            const int b = b0 + tid;
            const long long mine = b < a.B ? chunks_of(geo, a, b) : 0;
            long long incl = mine;
            for (int i = 1; i < 32; i <<= 1) {
                const long long o = __shfl_up_sync(0xffffffffu, incl, i);
                if (lane >= i) incl += o;
            }
            __syncthreads();
            if (lane == 31) sm_scan[warp] = incl;
            __syncthreads();
            for (int w = 0; w < n_warps; ++w) {
                if (w < warp) incl += sm_scan[w];
            }
            const long long at = (run + incl - mine) * hr;
            if (mine > 0 && at <= lo && lo < at + mine * hr) {
                sm_b = b;
                sm_base = at;
            }
            for (int w = 0; w < n_warps; ++w) run += sm_scan[w];
        }
        __syncthreads();
    }

    // ---- what a lane copies of 16 rows: its first piece, and its bound on piece numbers ----
    uint32_t cp_dst[2];
    int cp_src[2], cp_lim[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const CopyPlan& cp = pl.cp[side];
        const int pr = geo.s[side].row_bytes >> 4;
        if (cp.shift < 0) {
            cp_dst[side] = 16 * lane;
            cp_src[side] = 16 * lane;
            cp_lim[side] = 16 * pr;
        } else {
            const int row = lane >> cp.shift, col = lane & ((1 << cp.shift) - 1);
            cp_dst[side] = row * cp.stride + 16 * col;
            cp_src[side] = (row * pr + col) * 16;
            cp_lim[side] = col < pr ? 32 * cp.iters : 0;
        }
    }

    const int qh = geo.heads * a.group;
    const int n_min = ks.ng == 2 && ks.bits[1] < ks.bits[0] ? ks.bits[1] : ks.bits[0];
    const uint32_t k_lane = g * pl.cp[0].stride + (WIDE ? 4 * l : 0);
    const uint32_t v_lane = pl.v_off + 2 * l * pl.cp[1].stride + (WIDE ? 2 * g : 0);
    int b = sm_b;
    long long base = sm_base;        // first chunk of sequence b
    long long pos = lo;
    while (pos < hi) {
        int nch = chunks_of(geo, a, b);
        while (pos >= base + (long long)nch * hr) {
            base += (long long)nch * hr;
            nch = chunks_of(geo, a, ++b);
        }
        const long long rel = pos - base;
        const int item = (int)(rel / nch);
        const int c_first = (int)(rel % nch);
        const int head = item / pl.row_tiles, rt = item % pl.row_tiles;
        const long long left = hi - pos;
        const int c_end = left < nch - c_first ? c_first + (int)left : nch;
        const int len = a.lengths[b];
        const int end = (int)seen_end(geo, a, b);
        const int row0 = rt * R;
        const int32_t* table = a.table + b * a.table_stride;

        // ---- loads: chunk c into a stage of this warp's ring, as two halves of 16 rows ----
        const uint8_t *src[2], *ssrc[2];       // page 0's rows of this head, this lane's first piece
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const KvSide& s = geo.s[side];
            src[side] = s.codes + (int64_t)head * geo.page * s.row_bytes + cp_src[side];
            ssrc[side] = reinterpret_cast<const uint8_t*>(s.scales) + (int64_t)head * geo.page * 2 * s.ng + 4 * (lane & 15);
        }
        auto page_of = [&](int p) -> int { return p < end ? __ldg(table + (p >> geo.page_shift)) : -1; };
        auto issue = [&](int c, uint32_t st, int pg0, int pg1) {
            const int p0 = c * kChunk;
            bool bad = false;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int pg = half ? pg1 : pg0;
                const bool on = (unsigned)pg < (unsigned)geo.n_pages;
                bad |= !on && p0 + 16 * half < end;
                const int in = (p0 + 16 * half) & (geo.page - 1);
                const uint32_t use = on ? (uint32_t)pg : 0u;
                const int size = on ? 16 : 0;
#pragma unroll
                for (int side = 0; side < 2; ++side) {
                    const CopyPlan& cp = pl.cp[side];
                    const KvSide& s = geo.s[side];
                    const uint8_t* p = src[side] + (uint64_t)use * cp.page_bytes + in * s.row_bytes;
                    uint32_t dst = st + (side ? pl.v_off : 0) + half * 16 * cp.stride + cp_dst[side];
                    int i = lane;
#pragma unroll 2
                    for (int k = 0; k < cp.iters; ++k) {
                        if (i < cp_lim[side])
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(p), "r"(size) : "memory");
                        i += 32;
                        dst += cp.dst_step;
                        p += cp.src_step;
                    }
                    // 16 tokens' scales: 2 or 4 bytes each
                    if (lane < 8 * s.ng)
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(st + (side ? pl.vs_off : pl.ks_off) + (half * 8 * s.ng + lane) * 4),
                                     "l"(ssrc[side] + (uint64_t)use * cp.page_scales + in * 2 * s.ng), "r"(size >> 2)
                                     : "memory");
                }
            }
            if (bad && lane == 0) atomicOr(a.err, kErrKvIndex);
        };
        // page ids are read one issue ahead of their use
        int c_load = c_first + warp, n_pg0 = -1, n_pg1 = -1;
        auto fetch_pages = [&](int c) {
            if (c < c_end) {
                n_pg0 = page_of(c * kChunk);
                n_pg1 = geo.page == 16 ? page_of(c * kChunk + 16) : (c * kChunk + 16 < end ? n_pg0 : -1);
            }
        };
        fetch_pages(c_load);
        for (int s = 0; s < pl.stages - 1; ++s) {
            const int pg0 = n_pg0, pg1 = n_pg1, c = c_load;
            c_load += n_warps;
            fetch_pages(c_load);
            if (c < c_end) issue(c, ring + s * pl.stage_bytes, pg0, pg1);
            cp_commit();
        }

        // ---- queries of the item: fp16, each row scaled to 2^13, in fragment order ----
        {
            uint16_t* qf = reinterpret_cast<uint16_t*>(smem + pl.q_off);
            for (int r = warp; r < R; r += n_warps) {
                const int row = row0 + r;
                const bool on = row < pl.rows;
                const int t = on ? row / a.group : 0, h = head * a.group + (on ? row % a.group : 0);
                const uint16_t* q = a.Q + b * a.q_seq_stride + t * a.q_token_stride + h * a.q_head_stride;
                const int32_t* perm = ks.perm + head * ks.D;
                float x[8];
                uint32_t top = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    x[k] = 0.0f;
                    if (k < nkb) {
                        const int grp = k < ks.nb[0] ? 0 : 1;
                        const int c = key_code(ks.bits[grp], lane >> 3, (lane & 7) >> 1, lane & 1);
                        const int p = 32 * (grp ? k - ks.nb[0] : k) + c;
                        if (on && p < ks.count[grp]) x[k] = scale_of(q[perm[(grp ? ks.count[0] : 0) + p]], bf16);
                        top = max(top, __float_as_uint(x[k]) & 0x7FFFFFFFu);
                    }
                }
                top = __reduce_max_sync(0xffffffffu, top);
                const int e = top == 0 ? 0 : min(13 - ((int)(top >> 23) - 127), 120);   // x 2^e: largest in [2^13, 2^14)
                const float up = a.scale < 0.0f ? -pow2(e) : pow2(e);
                float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (k >= nkb) break;
                    const int grp = k < ks.nb[0] ? 0 : 1, bits = ks.bits[grp];
                    const int i = (lane & 7) >> 1;
                    const int down = place_log2(bits, i);
                    const __half hv = __float2half_rn(x[k] * up * pow2(n_min - bits - down));
                    const float back = __half2float(hv) * pow2(down + bits - 1 - 24);
                    if (grp) sum1 += back;
                    else sum0 += back;
                    // lane group r % 8, quad lane, register i, half
                    qf[(((k * NT + (r >> 3)) * 32 + (r & 7) * 4 + (lane >> 3)) * 4 + i) * 2 + (lane & 1)] = __half_as_ushort(hv);
                }
                for (int i = 16; i; i >>= 1) {
                    sum0 += __shfl_xor_sync(0xffffffffu, sum0, i);
                    sum1 += __shfl_xor_sync(0xffffffffu, sum1, i);
                }
                if (lane == 0) {
                    sm_init[r] = -sum0;
                    sm_init[R + r] = -sum1;
                    // positive, so that it can be applied behind the maximum
                    sm_fac[r] = fmaxf(ldexpf(fabsf(a.scale) * kLog2e, 24 - (n_min - 1) - e), 0x1p-126f);
                }
            }
            for (int p = tid; p < 32 * NVB; p += blockDim.x) {
                const int blk = p >> 5, grp = blk < vs.nb[0] ? 0 : 1;
                const int i = p - (grp ? 32 * vs.nb[0] : 0);
                sm_chan[p] = blk < nvb && i < vs.count[grp]
                                 ? (int16_t)vs.perm[head * vs.D + (grp ? vs.count[0] : 0) + i] : (int16_t)-1;
            }
        }
        __syncthreads();

        // running maximum (of scores before the row's factor), sum and outputs
        float fac[NT][2], m[NT][2], lsum[NT][2];
        float o[NVB][2][NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                fac[nt][r] = sm_fac[8 * nt + 2 * l + r];
                m[nt][r] = -INFINITY;
                lsum[nt][r] = 0.0f;
            }
        }
#pragma unroll
        for (int v = 0; v < NVB; ++v)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[v][u][nt][i] = 0.0f;
        int e0 = -100, e1 = -100;     // running powers of two above the value scales

        const uint32_t qbase = smem0 + pl.q_off + lane * 16;
        const int sure = min(len, end);
        uint32_t st = ring, st_load = ring + (pl.stages - 1) * pl.stage_bytes;
        const uint32_t ring_end = ring + pl.stages * pl.stage_bytes;
        for (int c = c_first + warp; c < c_end; c += n_warps) {
            cp_wait(pl.stages - 2);
            __syncwarp();
            {
                const int pg0 = n_pg0, pg1 = n_pg1, cl = c_load;
                c_load += n_warps;
                fetch_pages(c_load);
                if (cl < c_end) issue(cl, st_load, pg0, pg1);
                cp_commit();
                st_load += pl.stage_bytes;
                if (st_load == ring_end) st_load = ring;
            }
            const int p0 = c * kChunk;
            const bool tail = p0 + kChunk > sure;      // some rows may not see some of it

            // ---- scales: lane = token; as fp32 for all lanes, the values' relative to the running power of two ----
            {
                float k0, k1 = 0.0f, v0, v1 = 0.0f;
                if (ks.ng == 2) {
                    const uint32_t w = lds32(st + pl.ks_off + 4 * lane);
                    k0 = scale_of(w & 0xFFFFu, bf16);
                    k1 = scale_of(w >> 16, bf16);
                } else {
                    k0 = scale_of(lds16(st + pl.ks_off + 2 * lane), bf16);
                }
                if (vs.ng == 2) {
                    const uint32_t w = lds32(st + pl.vs_off + 4 * lane);
                    v0 = scale_of(w & 0xFFFFu, bf16);
                    v1 = scale_of(w >> 16, bf16);
                } else {
                    v0 = scale_of(lds16(st + pl.vs_off + 2 * lane), bf16);
                }
                if (tail && p0 + lane >= end) k0 = k1 = v0 = v1 = 0.0f;
                // positive floats order as integers; the exponent plus one bounds them
                const int n0 = max(e0, min((int)(__reduce_max_sync(0xffffffffu, __float_as_uint(v0)) >> 23) - 126, 126));
                int n1 = e1;
                if (vs.ng == 2) n1 = max(e1, min((int)(__reduce_max_sync(0xffffffffu, __float_as_uint(v1)) >> 23) - 126, 126));
                if (n0 > e0 || n1 > e1) {
                    const float d0 = n0 - e0 > 126 ? 0.0f : pow2(e0 - n0), d1 = n1 - e1 > 126 ? 0.0f : pow2(e1 - n1);
                    e0 = n0;
                    e1 = n1;
#pragma unroll
                    for (int v = 0; v < NVB; ++v)
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int i = 0; i < 4; ++i) o[v][u][nt][i] *= v < vs.nb[0] ? d0 : d1;
                }
                sts128f(fsc + 16 * lane, k0, k1, v0 * pow2(-e0), v1 * pow2(-e1));
                __syncwarp();
            }
            float4 sc[4];      // of tokens g, g + 8, g + 16, g + 24
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[j] = lds128f(fsc + 16 * (8 * j + g));

            // ---- scores ----
            float x[2][NT][4];
            const uint32_t krow = st + k_lane;
            auto key_block = [&](auto width, float(&acc)[2][NT][4], uint32_t at, uint32_t qat) {
                constexpr int BITS = decltype(width)::value;
                uint4 q[NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) q[nt] = lds128(qat + nt * 512);
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    uint32_t h[4], k[4];
                    key_halves<BITS>(at + 16 * mt * pl.cp[0].stride, h);
                    key_halves<BITS>(at + (16 * mt + 8) * pl.cp[0].stride, k);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma(acc[mt][nt], h[0], k[0], h[1], k[1], q[nt].x, q[nt].y);
                        mma(acc[mt][nt], h[2], k[2], h[3], k[3], q[nt].z, q[nt].w);
                    }
                }
            };
            auto key_group = [&](auto width, int grp, float(&acc)[2][NT][4]) {
                constexpr int BITS = decltype(width)::value;
                float init[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 2; ++r) init[nt][r] = sm_init[grp * R + 8 * nt + 2 * l + r];
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[mt][nt][i] = init[nt][i & 1];
                // a quad's lane starts BITS bytes behind the one before; krow has 4 of them where WIDE
                uint32_t at = krow + ks.off[grp] + (WIDE ? (BITS == 8 ? 4 * l : 0) : BITS * l);
                uint32_t qat = qbase + (grp ? ks.nb[0] : 0) * NT * 512;
                for (int blk = 0; blk < ks.nb[grp]; ++blk) {
                    key_block(width, acc, at, qat);
                    at += 4 * BITS;
                    qat += NT * 512;
                }
            };
            auto key_any = [&](int grp, float(&acc)[2][NT][4]) {
                if constexpr (WIDE) {
                    if (grp) key_group(std::integral_constant<int, 8>{}, grp, acc);
                    else key_group(std::integral_constant<int, 4>{}, grp, acc);
                } else {
                    if (ks.bits[grp] == 4) key_group(std::integral_constant<int, 4>{}, grp, acc);
                    else if (ks.bits[grp] == 8) key_group(std::integral_constant<int, 8>{}, grp, acc);
                    else key_group(std::integral_constant<int, 2>{}, grp, acc);
                }
            };
            key_any(0, x);
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[mt][nt][i] *= sc[2 * mt + (i >> 1)].x;
            if (ks.ng == 2) {
                float acc[2][NT][4];
                key_any(1, acc);
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[mt][nt][i] = fmaf(acc[mt][nt][i], sc[2 * mt + (i >> 1)].y, x[mt][nt][i]);
            }

            // ---- softmax ----
            if (tail) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int row = row0 + 8 * nt + 2 * l + r;
                        const int t = row < pl.rows ? row / a.group : a.T - 1;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int p = p0 + 8 * j + g, d = p - len;
                            bool see = p < end;
                            if (see && d >= 0) see = a.mask ? a.mask[b * a.mask_stride + (int64_t)t * a.T + d] != 0 : d <= t;
                            if (!see) x[j >> 1][nt][2 * (j & 1) + r] = -INFINITY;
                        }
                    }
            }
            float top[NT][2];
            bool grows = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float tp = fmaxf(fmaxf(x[0][nt][r], x[0][nt][2 + r]), fmaxf(x[1][nt][r], x[1][nt][2 + r]));
                    tp = fmaxf(tp, __shfl_xor_sync(0xffffffffu, tp, 4));
                    tp = fmaxf(tp, __shfl_xor_sync(0xffffffffu, tp, 8));
                    tp = fmaxf(tp, __shfl_xor_sync(0xffffffffu, tp, 16));
                    grows |= tp > m[nt][r];
                    top[nt][r] = tp;
                }
            if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float mn = fmaxf(m[nt][r], top[nt][r]);
                        const float al = mn == -INFINITY ? 1.0f : ex2((m[nt][r] - mn) * fac[nt][r]);
                        m[nt][r] = mn;
                        lsum[nt][r] *= al;
#pragma unroll
                        for (int v = 0; v < NVB; ++v)
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                o[v][u][nt][r] *= al;
                                o[v][u][nt][2 + r] *= al;
                            }
                    }
            }
            uint32_t w[2][2][NT][2];      // weights as B fragments: [group][16 tokens][row tile][8 tokens]
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float ms0 = m[nt][0] == -INFINITY ? 0.0f : -m[nt][0] * fac[nt][0];
                const float ms1 = m[nt][1] == -INFINITY ? 0.0f : -m[nt][1] * fac[nt][1];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float pa = ex2(fmaf(x[j >> 1][nt][2 * (j & 1)], fac[nt][0], ms0));
                    const float pb = ex2(fmaf(x[j >> 1][nt][2 * (j & 1) + 1], fac[nt][1], ms1));
                    lsum[nt][0] += pa;
                    lsum[nt][1] += pb;
                    w[0][j >> 1][nt][j & 1] = transpose8(pack2(pa * sc[j].z, pb * sc[j].z));
                    if (vs.ng == 2) w[1][j >> 1][nt][j & 1] = transpose8(pack2(pa * sc[j].w, pb * sc[j].w));
                }
            }

            // ---- outputs ----
            const uint32_t vrow = st + v_lane;
            auto value_block = [&](auto width, uint32_t at, const uint32_t(&wg)[2][NT][2], float(&ov)[2][NT][4]) {
                constexpr int BITS = decltype(width)::value;
                const int stride = pl.cp[1].stride;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    uint32_t p[4], q[4];
                    value_pairs<BITS>(at + 16 * kt * stride, at + (16 * kt + 1) * stride, p);
                    value_pairs<BITS>(at + (16 * kt + 8) * stride, at + (16 * kt + 9) * stride, q);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma(ov[0][nt], p[0], p[1], q[0], q[1], wg[kt][nt][0], wg[kt][nt][1]);
                        mma(ov[1][nt], p[2], p[3], q[2], q[3], wg[kt][nt][0], wg[kt][nt][1]);
                    }
                }
            };
#pragma unroll
            for (int v = 0; v < NVB; ++v) {
                if (v < vs.nb[0]) {
                    if constexpr (WIDE) {
                        value_block(std::integral_constant<int, 4>{}, vrow + 16 * v, w[0], o[v]);
                    } else {
                        const int bits = vs.bits[0];
                        const uint32_t at = vrow + 4 * v * bits + (bits * g >> 1);
                        if (bits == 4) value_block(std::integral_constant<int, 4>{}, at, w[0], o[v]);
                        else if (bits == 8) value_block(std::integral_constant<int, 8>{}, at, w[0], o[v]);
                        else value_block(std::integral_constant<int, 2>{}, at, w[0], o[v]);
                    }
                } else if (v < nvb) {
                    if constexpr (WIDE) {
                        value_block(std::integral_constant<int, 8>{}, vrow + 2 * g + vs.off[1] + 32 * (v - vs.nb[0]), w[1], o[v]);
                    } else {
                        const int bits = vs.bits[1];
                        const uint32_t at = vrow + vs.off[1] + 4 * (v - vs.nb[0]) * bits + (bits * g >> 1);
                        if (bits == 4) value_block(std::integral_constant<int, 4>{}, at, w[1], o[v]);
                        else if (bits == 8) value_block(std::integral_constant<int, 8>{}, at, w[1], o[v]);
                        else value_block(std::integral_constant<int, 2>{}, at, w[1], o[v]);
                    }
                }
            }
            st += pl.stage_bytes;
            if (st == ring_end) st = ring;
        }

        // ---- join the warps: statistics in units of the softmax's exponent ----
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float& s = lsum[nt][r];
                s += __shfl_xor_sync(0xffffffffu, s, 4);
                s += __shfl_xor_sync(0xffffffffu, s, 8);
                s += __shfl_xor_sync(0xffffffffu, s, 16);
                m[nt][r] *= fac[nt][r];
                if (g == 0) {
                    sm_m[warp * R + 8 * nt + 2 * l + r] = m[nt][r];
                    sm_l[warp * R + 8 * nt + 2 * l + r] = s;
                }
            }
        __syncthreads();
        float join[NT][2];      // 2^(m - the CTA's m)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float mm = -INFINITY;
                for (int wi = 0; wi < n_warps; ++wi) mm = fmaxf(mm, sm_m[wi * R + 8 * nt + 2 * l + r]);
                join[nt][r] = m[nt][r] == -INFINITY ? 0.0f : ex2(m[nt][r] - mm);
            }
        const bool whole = c_first == 0 && c_end == nch;
        const int segment = pos == lo ? 0 : 1;
        constexpr int PART = R * (32 * NVB + 2);      // floats of a partial result: outputs, then m, then l
        float* parts = reinterpret_cast<float*>(static_cast<uint8_t*>(a.scratch) + SONIQ_KV_SCRATCH_ZERO);
        float* part = parts + (int64_t)(2 * blockIdx.x + segment) * PART;
        // the value blocks of one pass: 8 NT rows x 32 PB outputs of 8 warps in the merge buffer
        constexpr int PB = NT >= 4 ? 1 : (4 / NT < NVB ? 4 / NT : NVB);
        auto store = [&](int r, int p, float v) {
            const int row = row0 + r, ch = sm_chan[p];
            if (row < pl.rows && ch >= 0) {
                const int64_t at = (((int64_t)b * a.T + row / a.group) * qh + head * a.group + row % a.group) * vs.D + ch;
                a.out[at] = bf16 ? kv_round<true>(v) : kv_round<false>(v);
            }
        };
#pragma unroll
        for (int v0 = 0; v0 < NVB; v0 += PB) {
#pragma unroll
            for (int vi = 0; vi < PB; ++vi) {
                const int v = v0 + vi;
                if (v < nvb) {
                    const int grp = v < vs.nb[0] ? 0 : 1, bits = vs.bits[grp], e = grp ? e1 : e0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float back = ldexpf(1.0f, e - (bits - 1) - place_log2(bits, i));
                        const int code = value_code(bits, g, i);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int r = 0; r < 2; ++r)
                                merge[((warp * R + 8 * nt + 2 * l + r) * PB + vi) * 32 + code] =
                                    o[v][i >> 1][nt][2 * (i & 1) + r] * join[nt][r] * back;
                    }
                }
            }
            __syncthreads();
            for (int i = tid; i < R * PB * 32; i += blockDim.x) {
                const int r = i / (PB * 32), p = v0 * 32 + i % (PB * 32);
                if (p >= 32 * nvb) continue;
                float sum = 0.0f;
                for (int wi = 0; wi < n_warps; ++wi) sum += merge[wi * R * PB * 32 + i];
                if (whole) {
                    float mm = -INFINITY, ll = 0.0f;
                    for (int wi = 0; wi < n_warps; ++wi) mm = fmaxf(mm, sm_m[wi * R + r]);
                    for (int wi = 0; wi < n_warps; ++wi) {
                        const float mw = sm_m[wi * R + r];
                        ll += sm_l[wi * R + r] * (mw == -INFINITY ? 0.0f : ex2(mw - mm));
                    }
                    store(r, p, ll > 0.0f ? sum / ll : (ll == 0.0f ? 0.0f : ll));
                } else {
                    part[r * 32 * NVB + p] = sum;
                }
            }
            __syncthreads();
        }
        if (!whole) {
            for (int r = tid; r < R; r += blockDim.x) {
                float mm = -INFINITY, ll = 0.0f;
                for (int wi = 0; wi < n_warps; ++wi) mm = fmaxf(mm, sm_m[wi * R + r]);
                for (int wi = 0; wi < n_warps; ++wi) {
                    const float mw = sm_m[wi * R + r];
                    ll += sm_l[wi * R + r] * (mw == -INFINITY ? 0.0f : ex2(mw - mm));
                }
                part[R * 32 * NVB + r] = mm;
                part[R * 32 * NVB + R + r] = ll;
            }
            // the CTAs that share the item: the last to get here joins their parts in order
            const long long s_first = base + (long long)item * nch, s_last = s_first + nch - 1;
            const int cta0 = (int)(((s_first + 1) * n_cta - 1) / total), cta1 = (int)(((s_last + 1) * n_cta - 1) / total);
            unsigned* counter = static_cast<unsigned*>(a.scratch) + cta0;
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const unsigned n = atomicAdd(counter, 1u);
                sm_last = n == (unsigned)(cta1 - cta0);
                if (sm_last) *counter = 0;
            }
            __syncthreads();
            if (sm_last) {
                __threadfence();
                const int head_seg = total * cta0 / n_cta == s_first ? 0 : 1;
                auto part_of = [&](int c) { return parts + (int64_t)(2 * c + (c == cta0 ? head_seg : 0)) * PART; };
                for (int i = tid; i < R * 32 * nvb; i += blockDim.x) {
                    const int r = i / (32 * nvb), p = i % (32 * nvb);
                    if (row0 + r >= pl.rows) continue;
                    float mm = -INFINITY, acc = 0.0f, ll = 0.0f;
                    for (int c = cta0; c <= cta1; ++c) mm = fmaxf(mm, __ldcg(part_of(c) + R * 32 * NVB + r));
                    for (int c = cta0; c <= cta1; ++c) {
                        const float* q = part_of(c);
                        const float mc = __ldcg(q + R * 32 * NVB + r);
                        const float f = mc == -INFINITY ? 0.0f : ex2(mc - mm);
                        acc += f * __ldcg(q + r * 32 * NVB + p);
                        ll += f * __ldcg(q + R * 32 * NVB + R + r);
                    }
                    store(r, p, ll > 0.0f ? acc / ll : (ll == 0.0f ? 0.0f : ll));
                }
            }
        }
        pos += c_end - c_first;
        __syncthreads();
    }
}

struct RowsLaunch {
    int nt, nvb, warps, ctas_per_sm;
    bool wide;
    RowsPlan pl;
};

constexpr int kMaxSmem = 227 * 1024;

RowsLaunch plan_rows(const KvGeom& geo, int64_t T, int64_t group) {
    RowsLaunch r{};
    const KvSide &ks = geo.s[0], &vs = geo.s[1];
    const int nkb = ks.nb[0] + ks.nb[1], nvb = vs.nb[0] + vs.nb[1];
    const int64_t rows = T * group;
    r.nvb = nvb <= 2 ? 2 : (nvb <= 4 ? 4 : 8);
    r.nt = rows <= 8 ? 1 : (rows <= 16 || r.nvb == 8 ? 2 : 4);
    RowsPlan& p = r.pl;
    const int R = 8 * r.nt;
    p.rows = (int)rows;
    p.row_tiles = (int)((rows + R - 1) / R);
    for (int side = 0; side < 2; ++side) {
        const KvSide& sd = geo.s[side];
        CopyPlan& cp = p.cp[side];
        const int pr = sd.row_bytes / 16;
        if (pr % 2) {
            cp.shift = -1;
            cp.stride = sd.row_bytes;
            cp.iters = (16 * pr + 31) / 32;
            cp.dst_step = cp.src_step = 512;
        } else {
            cp.shift = 1;
            while ((1 << cp.shift) < pr) ++cp.shift;
            cp.stride = sd.row_bytes + 16;
            const int rows_at_once = 32 >> cp.shift;
            cp.iters = 16 / rows_at_once;
            cp.dst_step = rows_at_once * cp.stride;
            cp.src_step = rows_at_once * sd.row_bytes;
        }
        cp.page_bytes = (uint32_t)geo.heads * geo.page * sd.row_bytes;
        cp.page_scales = (uint32_t)geo.heads * geo.page * 2 * sd.ng;
    }
    p.v_off = kChunk * p.cp[0].stride;
    p.ks_off = p.v_off + kChunk * p.cp[1].stride;
    p.vs_off = p.ks_off + kChunk * 2 * ks.ng;
    p.stage_bytes = p.vs_off + kChunk * 2 * vs.ng;
    const int q = nkb * r.nt * 512, scales = 16 * kChunk;
    const int misc = (4 * (3 * R + 16 * R) + 2 * 32 * r.nvb + 15) / 16 * 16;
    const int fixed = q + misc;
    // two stages at least; two CTAs per SM where they and the registers allow it
    r.warps = 8;
    r.ctas_per_sm = r.nt * r.nvb <= 4 && fixed + 8 * (2 * p.stage_bytes + scales) <= kMaxSmem / 2 - 2048 ? 2 : 1;
    const int budget = r.ctas_per_sm == 2 ? kMaxSmem / 2 - 2048 : kMaxSmem - 1024;
    if (fixed + 8 * (2 * p.stage_bytes + scales) > budget) r.warps = 4;
    p.stages = ((budget - fixed) / r.warps - scales) / p.stage_bytes;
    if (p.stages > 4) p.stages = 4;
    p.f_off = p.stages * p.stage_bytes;
    p.warp_bytes = p.f_off + scales;
    p.q_off = r.warps * p.warp_bytes;
    if (p.q_off < kMergeBytes) p.q_off = kMergeBytes;
    p.misc_off = p.q_off + q;
    p.smem = p.misc_off + misc;
    p.min_chunks = 8;
    r.wide = ks.bits[0] == 4 && vs.bits[0] == 4 && ks.bits[1] == 8 && vs.bits[1] == 8;
    return r;
}

template <int NT, int NVB>
cudaError_t run_rows(const KvGeom& geo, const KvAttendArgs& a, const RowsLaunch& r, int grid, cudaStream_t st) {
    auto* kernel = r.wide ? kv_rows_kernel<NT, NVB, true> : kv_rows_kernel<NT, NVB, false>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, r.pl.smem);
    if (e == cudaSuccess) e = prefer_max_shared(reinterpret_cast<const void*>(kernel));
    if (e != cudaSuccess) return e;
    kernel<<<grid, 32 * r.warps, r.pl.smem, st>>>(geo, a, r.pl);
    note_launch();
    return cudaGetLastError();
}

}  // namespace

int64_t kv_attend_scratch(const KvGeom& geo, int64_t B, int64_t T, int64_t group) {
    if (B == 0 || T == 0) return 0;
    const RowsLaunch r = plan_rows(geo, T, group);
    return SONIQ_KV_SCRATCH_ZERO + (int64_t)2 * 2 * num_sms() * 8 * r.nt * (32 * r.nvb + 2) * 4;
}

cudaError_t launch_kv_attend(const KvGeom& geo, const KvAttendArgs& a, cudaStream_t st) {
    const RowsLaunch r = plan_rows(geo, a.T, a.group);
    const int64_t cap = (int64_t)a.max_pages << geo.page_shift;
    const int64_t most = (int64_t)a.B * geo.heads * r.pl.row_tiles * (cap / kChunk + 1);
    const int64_t by_size = (most + r.pl.min_chunks - 1) / r.pl.min_chunks;
    const int64_t full = (int64_t)r.ctas_per_sm * num_sms();
    const int grid = (int)(by_size < full ? by_size : full);
    switch (r.nvb * 8 + r.nt) {
        case 2 * 8 + 1: return run_rows<1, 2>(geo, a, r, grid, st);
        case 2 * 8 + 2: return run_rows<2, 2>(geo, a, r, grid, st);
        case 2 * 8 + 4: return run_rows<4, 2>(geo, a, r, grid, st);
        case 4 * 8 + 1: return run_rows<1, 4>(geo, a, r, grid, st);
        case 4 * 8 + 2: return run_rows<2, 4>(geo, a, r, grid, st);
        case 4 * 8 + 4: return run_rows<4, 4>(geo, a, r, grid, st);
        case 8 * 8 + 1: return run_rows<1, 8>(geo, a, r, grid, st);
        default: return run_rows<2, 8>(geo, a, r, grid, st);
    }
}

}  // namespace soniq
