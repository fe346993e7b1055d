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

struct RowsPlan {
    int row_tiles;        // tiles of 8 NT query rows per key head
    int rows;             // query rows per key head: T * group
    int stages;
    int stage_bytes;
    int k_stride, v_stride;      // shared row strides: odd multiples of 16 bytes (no bank conflicts)
    int v_off, ks_off, vs_off;   // in a stage
    int merge_off, q_off, misc_off;
    int smem;
    int min_chunks;       // fewest chunks worth a CTA
    uint32_t k_magic, v_magic;   // ceil(2^16 / 16-byte pieces of a row): pieces are numbered below 512
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool on) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(on ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the newest `newer` groups of this thread have landed.
__device__ __forceinline__ void cp_wait(int newer) {
    if (newer >= 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (newer == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

__device__ __forceinline__ uint32_t lds16(uint32_t a) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a) : "memory");
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
    if (bits == 8) return 8 * l + 2 * i + half;
    if (bits == 4) return 8 * l + 4 * (i & 1) + (i >> 1) + 2 * half;
    return 16 * (l >> 1) + 4 * i + 2 * (l & 1) + half;
}
__device__ __forceinline__ int place_log2(int bits, int i) { return bits == 8 ? 0 : (bits == 4 ? 4 * (i & 1) : 2 * i); }

// ... as u 2^-24 times the place's power, from the block at shared address `at`.
template <int BITS>
__device__ __forceinline__ void key_halves(uint32_t at, int l, uint32_t (&h)[4]) {
    if constexpr (BITS == 8) {
        uint2 w = lds64(at + 8 * l);
        w.x ^= 0x80808080u;
        w.y ^= 0x80808080u;
        h[0] = __byte_perm(w.x, 0, 0x4140);
        h[1] = __byte_perm(w.x, 0, 0x4342);
        h[2] = __byte_perm(w.y, 0, 0x4140);
        h[3] = __byte_perm(w.y, 0, 0x4342);
    } else if constexpr (BITS == 4) {
        uint32_t w = lds32(at + 4 * l);
        h[0] = (w & 0x000F000Fu) ^ 0x00080008u;
        h[1] = (w & 0x00F000F0u) ^ 0x00800080u;
        w >>= 8;
        h[2] = (w & 0x000F000Fu) ^ 0x00080008u;
        h[3] = (w & 0x00F000F0u) ^ 0x00800080u;
    } else {
        const uint32_t w = __byte_perm(lds16(at + 2 * l), 0, 0x4140);
        h[0] = (w & 0x00030003u) ^ 0x00020002u;
        h[1] = (w & 0x000C000Cu) ^ 0x00080008u;
        h[2] = (w & 0x00300030u) ^ 0x00200020u;
        h[3] = (w & 0x00C000C0u) ^ 0x00800080u;
    }
}

// The value side: lane group g of a warp holds 4 codes of a block, each as the
// pair (token t, token t + 1), signed, times the place's power.
__device__ __forceinline__ int value_code(int bits, int g, int i) {
    if (bits == 8) return 4 * g + i;
    if (bits == 4) return 8 * (g >> 1) + 2 * (g & 1) + 4 * (i & 1) + (i >> 1);
    return 16 * (g >> 2) + 4 * i + (g & 3);
}

template <int BITS>
__device__ __forceinline__ void value_pairs(uint32_t row0, uint32_t row1, int g, uint32_t (&x)[4]) {
    if constexpr (BITS == 8) {
        const uint32_t a = lds32(row0 + 4 * g), b = lds32(row1 + 4 * g);
        x[0] = sub2((__byte_perm(a, b, 0x4400) & 0x00FF00FFu) ^ 0x64806480u, 0x64806480u);
        x[1] = sub2((__byte_perm(a, b, 0x5511) & 0x00FF00FFu) ^ 0x64806480u, 0x64806480u);
        x[2] = sub2((__byte_perm(a, b, 0x6622) & 0x00FF00FFu) ^ 0x64806480u, 0x64806480u);
        x[3] = sub2((__byte_perm(a, b, 0x7733) & 0x00FF00FFu) ^ 0x64806480u, 0x64806480u);
    } else if constexpr (BITS == 4) {
        uint32_t w = __byte_perm(lds16(row0 + 2 * g), lds16(row1 + 2 * g), 0x5410);
        x[0] = sub2((w & 0x000F000Fu) ^ 0x64086408u, 0x64086408u);
        x[1] = sub2((w & 0x00F000F0u) ^ 0x64806480u, 0x64806480u);
        w >>= 8;
        x[2] = sub2((w & 0x000F000Fu) ^ 0x64086408u, 0x64086408u);
        x[3] = sub2((w & 0x00F000F0u) ^ 0x64806480u, 0x64806480u);
    } else {
        const uint32_t w = __byte_perm(lds8(row0 + g), lds8(row1 + g), 0x5410);
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

template <int NT, int NVB>
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
    const uint32_t ring = smem0 + warp * pl.stages * pl.stage_bytes;
    float* merge = reinterpret_cast<float*>(smem + pl.merge_off);
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

    const int qh = geo.heads * a.group;
    const int n_min = ks.ng == 2 && ks.bits[1] < ks.bits[0] ? ks.bits[1] : ks.bits[0];
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

        // ---- loads: chunk c into a stage of this warp's ring ----
        auto page_of = [&](int p) -> int { return p < end ? __ldg(table + (p >> geo.page_shift)) : -1; };
        auto issue = [&](int c, int stage, int pg0, int pg1) {
            const int p0 = c * kChunk;
            const uint32_t st = ring + stage * pl.stage_bytes;
            const bool on0 = pg0 >= 0 && pg0 < geo.n_pages, on1 = pg1 >= 0 && pg1 < geo.n_pages;
            if ((!on0 && p0 < end) || (!on1 && p0 + 16 < end)) {
                if (lane == 0) atomicOr(a.err, kErrKvIndex);
            }
            const int in0 = p0 & (geo.page - 1), in1 = (p0 + 16) & (geo.page - 1);
            const int64_t r0 = on0 ? ((int64_t)pg0 * geo.heads + head) * geo.page + in0 : 0;
            // rows 16.. of the chunk as if it went on from there
            const int64_t r1 = on1 ? ((int64_t)pg1 * geo.heads + head) * geo.page + in1 - 16 : 0;
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                const KvSide& s = side ? vs : ks;
                const int pr = s.row_bytes >> 4;
                const uint32_t magic = side ? pl.v_magic : pl.k_magic;
                const uint8_t* src0 = s.codes + r0 * s.row_bytes;
                const uint8_t* src1 = s.codes + (on1 ? r1 * s.row_bytes : 0);
                const int pad = (side ? pl.v_stride : pl.k_stride) - s.row_bytes;   // 0 or 16
                const uint32_t dst = st + (side ? pl.v_off : 0);
#pragma unroll 4
                for (int k = 0; k < pr; ++k) {
                    const int i = lane + 32 * k;
                    const int row = (int)((uint32_t)i * magic >> 16);
                    const bool second = row >= 16;
                    const bool on = second ? on1 : on0;
                    cp16(dst + 16 * i + pad * row, (second ? src1 : src0) + (on ? 16 * i : 0), on);
                }
                const uint32_t sd = st + (side ? pl.vs_off : pl.ks_off);
                if (s.ng == 2) {
                    const bool second = lane >= 16, on = second ? on1 : on0;
                    cp4(sd + 4 * lane, s.scales + (on ? ((second ? r1 : r0) + lane) * 2 : 0), on);
                } else if (lane < 16) {
                    const bool second = lane >= 8, on = second ? on1 : on0;
                    cp4(sd + 4 * lane, s.scales + (on ? (second ? r1 : r0) + 2 * lane : 0), on);
                }
            }
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
            if (c < c_end) issue(c, s, pg0, pg1);
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
                int code[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    x[k] = 0.0f;
                    code[k] = 0;
                    if (k < nkb) {
                        const int grp = k < ks.nb[0] ? 0 : 1;
                        const int c = key_code(ks.bits[grp], lane >> 3, (lane & 7) >> 1, lane & 1);
                        const int p = 32 * (grp ? k - ks.nb[0] : k) + c;
                        if (on && p < ks.count[grp]) {
                            const uint16_t v = q[perm[(grp ? ks.count[0] : 0) + p]];
                            x[k] = scale_of(v, bf16);
                        }
                        top = max(top, __float_as_uint(x[k]) & 0x7FFFFFFFu);
                    }
                }
                top = __reduce_max_sync(0xffffffffu, top);
                const int e = top == 0 ? 0 : min(13 - ((int)(top >> 23) - 127), 120);   // x 2^e: largest in [2^13, 2^14)
                const float up = pow2(e);
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
                    sm_fac[r] = ldexpf(a.scale * kLog2e, 24 - (n_min - 1) - e);
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

        float init0[NT][2], init1[NT][2], fac[NT][2], m[NT][2], lsum[NT][2];
        float o[NVB][2][NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                init0[nt][r] = sm_init[8 * nt + 2 * l + r];
                init1[nt][r] = sm_init[R + 8 * nt + 2 * l + r];
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
        int stage = 0, load_stage = pl.stages - 1;
        for (int c = c_first + warp; c < c_end; c += n_warps) {
            cp_wait(pl.stages - 2);
            __syncwarp();
            {
                const int pg0 = n_pg0, pg1 = n_pg1, cl = c_load;
                c_load += n_warps;
                fetch_pages(c_load);
                if (cl < c_end) issue(cl, load_stage, pg0, pg1);
                cp_commit();
                if (++load_stage == pl.stages) load_stage = 0;
            }
            const uint32_t st = ring + stage * pl.stage_bytes;
            if (++stage == pl.stages) stage = 0;
            const int p0 = c * kChunk;
            const bool tail = p0 + kChunk > min(len, end);      // some rows may not see some of it

            // ---- scores ----
            float x[2][NT][4];
#pragma unroll
            for (int grp = 0; grp < 2; ++grp) {
                if (grp == 1 && ks.ng == 1) break;
                float acc[2][NT][4];
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[mt][nt][i] = grp ? init1[nt][i & 1] : init0[nt][i & 1];
                const int bits = ks.bits[grp], nb = ks.nb[grp];
                const uint32_t krow = st + g * pl.k_stride + ks.off[grp];
                const uint32_t qb = qbase + (grp ? ks.nb[0] : 0) * NT * 512;
                auto block = [&](auto width, int blk) {
                    constexpr int BITS = decltype(width)::value;
                    uint4 q[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) q[nt] = lds128(qb + (blk * NT + nt) * 512);
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        uint32_t h[4], k[4];
                        const uint32_t at = krow + 16 * mt * pl.k_stride + 4 * BITS * blk;
                        key_halves<BITS>(at, l, h);
                        key_halves<BITS>(at + 8 * pl.k_stride, l, k);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma(acc[mt][nt], h[0], k[0], h[1], k[1], q[nt].x, q[nt].y);
                            mma(acc[mt][nt], h[2], k[2], h[3], k[3], q[nt].z, q[nt].w);
                        }
                    }
                };
                if (bits == 4) {
                    for (int blk = 0; blk < nb; ++blk) block(std::integral_constant<int, 4>{}, blk);
                } else if (bits == 8) {
                    for (int blk = 0; blk < nb; ++blk) block(std::integral_constant<int, 8>{}, blk);
                } else {
                    for (int blk = 0; blk < nb; ++blk) block(std::integral_constant<int, 2>{}, blk);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {      // tokens 8 j + g
                    const int tok = 8 * j + g;
                    float s = scale_of(lds16(st + pl.ks_off + 2 * (tok * ks.ng + grp)), bf16);
                    if (tail && p0 + tok >= end) s = 0.0f;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const float v = acc[j >> 1][nt][2 * (j & 1) + r];
                            float& d = x[j >> 1][nt][2 * (j & 1) + r];
                            d = grp ? fmaf(v, s, d) : v * s;
                        }
                }
            }

            // ---- softmax ----
            float vsc[2][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int tok = 8 * j + g;
                const bool gone = tail && p0 + tok >= end;
                vsc[0][j] = gone ? 0.0f : scale_of(lds16(st + pl.vs_off + 2 * (tok * vs.ng)), bf16);
                vsc[1][j] = gone || vs.ng == 1 ? 0.0f : scale_of(lds16(st + pl.vs_off + 2 * (tok * vs.ng) + 2), bf16);
            }
            float top[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    top[nt][r] = -INFINITY;
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j >> 1][nt][2 * (j & 1) + r] *= fac[nt][r];
                    if (tail) {
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
#pragma unroll
                    for (int j = 0; j < 4; ++j) top[nt][r] = fmaxf(top[nt][r], x[j >> 1][nt][2 * (j & 1) + r]);
                }
            bool grows = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float& tp = top[nt][r];
                    tp = fmaxf(tp, __shfl_xor_sync(0xffffffffu, tp, 4));
                    tp = fmaxf(tp, __shfl_xor_sync(0xffffffffu, tp, 8));
                    tp = fmaxf(tp, __shfl_xor_sync(0xffffffffu, tp, 16));
                    grows |= tp > m[nt][r];
                }
            // the power of two above every value scale so far (positive floats order as integers)
            const uint32_t big0 = __reduce_max_sync(0xffffffffu, max(max(__float_as_uint(vsc[0][0]), __float_as_uint(vsc[0][1])),
                                                                     max(__float_as_uint(vsc[0][2]), __float_as_uint(vsc[0][3]))));
            uint32_t big1 = 0;
            if (vs.ng == 2)
                big1 = __reduce_max_sync(0xffffffffu, max(max(__float_as_uint(vsc[1][0]), __float_as_uint(vsc[1][1])),
                                                          max(__float_as_uint(vsc[1][2]), __float_as_uint(vsc[1][3]))));
            const int n0 = max(e0, min((int)(big0 >> 23) - 126, 126)), n1 = max(e1, min((int)(big1 >> 23) - 126, 126));
            if (__any_sync(0xffffffffu, grows || n0 > e0 || n1 > e1)) {
                const float d0 = n0 - e0 > 126 ? 0.0f : pow2(e0 - n0), d1 = n1 - e1 > 126 ? 0.0f : pow2(e1 - n1);
                e0 = n0;
                e1 = n1;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float mn = fmaxf(m[nt][r], top[nt][r]);
                        const float al = mn == -INFINITY ? 1.0f : ex2(m[nt][r] - mn);
                        m[nt][r] = mn;
                        lsum[nt][r] *= al;
#pragma unroll
                        for (int v = 0; v < NVB; ++v) {
                            const float f = al * (v < vs.nb[0] ? d0 : d1);
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                o[v][u][nt][r] *= f;
                                o[v][u][nt][2 + r] *= f;
                            }
                        }
                    }
            }
            const float f0 = pow2(-e0), f1 = pow2(-e1);
            uint32_t w[2][2][NT][2];      // weights as B fragments: [group][16 tokens][row tile][8 tokens]
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float ms0 = m[nt][0] == -INFINITY ? 0.0f : m[nt][0], ms1 = m[nt][1] == -INFINITY ? 0.0f : m[nt][1];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float pa = ex2(x[j >> 1][nt][2 * (j & 1)] - ms0), pb = ex2(x[j >> 1][nt][2 * (j & 1) + 1] - ms1);
                    lsum[nt][0] += pa;
                    lsum[nt][1] += pb;
                    const float s0 = vsc[0][j] * f0;
                    w[0][j >> 1][nt][j & 1] = transpose8(pack2(pa * s0, pb * s0));
                    if (vs.ng == 2) {
                        const float s1 = vsc[1][j] * f1;
                        w[1][j >> 1][nt][j & 1] = transpose8(pack2(pa * s1, pb * s1));
                    }
                }
            }

            // ---- outputs ----
#pragma unroll
            for (int v = 0; v < NVB; ++v) {
                if (v >= nvb) break;
                const int grp = v < vs.nb[0] ? 0 : 1;
                const int blk = grp ? v - vs.nb[0] : v;
                auto block = [&](auto width) {
                    constexpr int BITS = decltype(width)::value;
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt) {
                        const uint32_t at = st + pl.v_off + (16 * kt + 2 * l) * pl.v_stride + vs.off[grp] + 4 * BITS * blk;
                        uint32_t p[4], q[4];
                        value_pairs<BITS>(at, at + pl.v_stride, g, p);
                        value_pairs<BITS>(at + 8 * pl.v_stride, at + 9 * pl.v_stride, g, q);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint32_t b0 = grp ? w[1][kt][nt][0] : w[0][kt][nt][0];
                            const uint32_t b1 = grp ? w[1][kt][nt][1] : w[0][kt][nt][1];
                            mma(o[v][0][nt], p[0], p[1], q[0], q[1], b0, b1);
                            mma(o[v][1][nt], p[2], p[3], q[2], q[3], b0, b1);
                        }
                    }
                };
                const int bits = vs.bits[grp];
                if (bits == 4) block(std::integral_constant<int, 4>{});
                else if (bits == 8) block(std::integral_constant<int, 8>{});
                else block(std::integral_constant<int, 2>{});
            }
        }

        // ---- join the warps ----
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float& s = lsum[nt][r];
                s += __shfl_xor_sync(0xffffffffu, s, 4);
                s += __shfl_xor_sync(0xffffffffu, s, 8);
                s += __shfl_xor_sync(0xffffffffu, s, 16);
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

int odd16(int bytes) { return (bytes / 16) % 2 ? bytes : bytes + 16; }

struct RowsLaunch {
    int nt, nvb, warps, ctas_per_sm;
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
    p.k_stride = odd16(ks.row_bytes);
    p.v_stride = odd16(vs.row_bytes);
    p.v_off = kChunk * p.k_stride;
    p.ks_off = p.v_off + kChunk * p.v_stride;
    p.vs_off = p.ks_off + kChunk * 2 * ks.ng;
    p.stage_bytes = p.vs_off + kChunk * 2 * vs.ng;
    const int merge = kMergeBytes, q = nkb * r.nt * 512;
    const int misc = 4 * (3 * R + 16 * R) + 2 * 32 * r.nvb;
    const int fixed = merge + q + (misc + 15) / 16 * 16;
    r.warps = 8;
    r.ctas_per_sm = r.nt * r.nvb <= 4 ? 2 : 1;
    // two stages at least; two CTAs per SM where they and the registers allow it
    while (r.ctas_per_sm == 2 && fixed + 8 * 2 * p.stage_bytes > kMaxSmem / 2 - 2048) r.ctas_per_sm = 1;
    const int budget = r.ctas_per_sm == 2 ? kMaxSmem / 2 - 2048 : kMaxSmem - 1024;
    if (fixed + 8 * 2 * p.stage_bytes > budget) r.warps = 4;
    p.stages = (budget - fixed) / (r.warps * p.stage_bytes);
    if (p.stages > 4) p.stages = 4;
    p.merge_off = r.warps * p.stages * p.stage_bytes;
    p.q_off = p.merge_off + merge;
    p.misc_off = p.q_off + q;
    p.smem = p.misc_off + (misc + 15) / 16 * 16;
    p.min_chunks = 8;
    p.k_magic = (65536u + ks.row_bytes / 16 - 1) / (ks.row_bytes / 16);
    p.v_magic = (65536u + vs.row_bytes / 16 - 1) / (vs.row_bytes / 16);
    return r;
}

template <int NT, int NVB>
cudaError_t run_rows(const KvGeom& geo, const KvAttendArgs& a, const RowsLaunch& r, int grid, cudaStream_t st) {
    auto* kernel = kv_rows_kernel<NT, NVB>;
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
