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
//    shared-memory stages and its own running maximum, sum and outputs, joined
//    at the end of a range; ranges that share an item leave partial results in
//    scratch, and the last of them joins those in order.
//  * A chunk's rows and scales come by TMA (four copies, swizzled so that lanes
//    reading one place of eight rows meet different banks).
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
//    exact in fp16 then).  Softmax weights times value scales are rounded to fp16
//    relative to a power of two of the row's own (kv_device.cuh).
//
// Bound by instructions, about 830 for a chunk of 32 tokens (keys 4/8 bits,
// values 4, 128 channels, 8 rows) at 2.5 a cycle, and for short contexts by what
// comes before and after: the split, queries, and the joins take 10 to 20 us.
// Measured (GB300): 131071 tokens of one sequence, 8 key heads: 60 us (2.6 TB/s);
// 64 sequences of up to 8192 tokens: 125 us (2.7 TB/s); 97 tokens: 12 us.
#include <type_traits>

#include "kv_device.cuh"
#include "kv_split.cuh"

namespace soniq {

namespace {

constexpr int kChunk = 32;                   // tokens a warp takes at a time
// An item's queries and results take about as long as this many chunks.  (64 sequences of up to 8192 tokens, us: 8: 141,
// 16: 136, 32: 125, 64: 131.)
constexpr int kLead = 32;

struct RowsPlan {
    int row_tiles;        // tiles of 8 NT query rows per key head
    int rows;             // query rows per key head: T * group
    int stages;
    int box_rows;         // tokens of one copy: 32, or a page of 16
    int scale_bytes;      // of a stage: 128 for each copy of keys' or values' scales
    int warp_bytes;       // a warp's stages
    int s_off, bar_off;   // the warps' scales, barriers
    int q_off, misc_off;
    int smem;
    int min_chunks;       // fewest chunks worth a CTA
};

// A quad's lane l holds 8 keys' codes of a block as four half pairs h[0..3] (key_code),
// ... as u 2^-24 times the place's power; `at`: the lane's bytes of the block.
template <int BITS>
__device__ __forceinline__ void key_halves(uint32_t at, uint32_t (&h)[4]) {
    if constexpr (BITS == 8) {
        uint2 w = lds64(at);
        w.x ^= 0x80808080u;
        w.y ^= 0x80808080u;
        h[0] = w.x & 0x00FF00FFu;
        h[1] = (w.x >> 8) & 0x00FF00FFu;
        h[2] = w.y & 0x00FF00FFu;
        h[3] = (w.y >> 8) & 0x00FF00FFu;
    } else if constexpr (BITS == 4) {
        uint32_t w = lds32(at) ^ 0x88888888u;
        h[0] = w & 0x000F000Fu;
        h[1] = w & 0x00F000F0u;
        w >>= 8;
        h[2] = w & 0x000F000Fu;
        h[3] = w & 0x00F000F0u;
    } else {
        const uint32_t w = __byte_perm(lds16(at) ^ 0xAAAAu, 0, 0x4140);
        h[0] = w & 0x00030003u;
        h[1] = w & 0x000C000Cu;
        h[2] = w & 0x00300030u;
        h[3] = w & 0x00C000C0u;
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
__device__ __forceinline__ void value_pairs(uint32_t row0, uint32_t row1, const Offsets& f, uint32_t (&x)[4]) {
    if constexpr (BITS == 8) {
        const uint32_t a = lds32(row0), b = lds32(row1);
        x[0] = sub2(mask_flip(__byte_perm(a, b, 0x4400), 0x00FF00FFu, f.c128), f.c128);
        x[1] = sub2(mask_flip(__byte_perm(a, b, 0x5511), 0x00FF00FFu, f.c128), f.c128);
        x[2] = sub2(mask_flip(__byte_perm(a, b, 0x6622), 0x00FF00FFu, f.c128), f.c128);
        x[3] = sub2(mask_flip(__byte_perm(a, b, 0x7733), 0x00FF00FFu, f.c128), f.c128);
    } else if constexpr (BITS == 4) {
        nibble_pairs(__byte_perm(lds16(row0), lds16(row1), 0x5410), f, x);
    } else {
        const uint32_t w = __byte_perm(lds8(row0), lds8(row1), 0x5410);
        x[0] = sub2(mask_flip(w, 0x00030003u, 0x64026402u), 0x64026402u);
        x[1] = sub2(mask_flip(w, 0x000C000Cu, f.c8), f.c8);
        x[2] = sub2(mask_flip(w, 0x00300030u, 0x64206420u), 0x64206420u);
        x[3] = sub2(mask_flip(w, 0x00C000C0u, f.c128), f.c128);
    }
}
// Two 4-bit blocks in a row at once: lane group g takes word g of their eight,
// codes 8 g + 4 (i & 1) + (i >> 1) of 64 into x[i], those 2 later into y[i].
__device__ __forceinline__ void value_pairs2(uint32_t row0, uint32_t row1, const Offsets& f, uint32_t (&x)[4], uint32_t (&y)[4]) {
    const uint32_t a = lds32(row0), b = lds32(row1);
    nibble_pairs(__byte_perm(a, b, 0x5410), f, x);
    nibble_pairs(__byte_perm(a, b, 0x7632), f, y);
}
__device__ __forceinline__ int value_code2(int g, int i) { return 8 * g + 4 * (i & 1) + (i >> 1); }

// At least one for a present sequence, so that its rows are written.
__device__ __forceinline__ int chunks_of(const KvGeom& geo, const KvAttendArgs& a, int b) {
    if (a.lengths[b] < 0) return 0;
    const int64_t end = seen_end(geo, a, b);
    return end == 0 ? 1 : (int)((end + kChunk - 1) / kChunk);
}

// Byte `x` of a row in shared memory, rows S bytes long: 16-byte pieces swizzled
// by `sw` (the row's share, swizzle_of), rows of 256 bytes as two tiles of 32
// half rows.
template <int S>
__device__ __forceinline__ uint32_t row_byte(uint32_t x, uint32_t sw) {
    if constexpr (S == 256) return ((x & 0x80u) << 5) + ((x & 0x7Fu) ^ sw);
    else return x ^ sw;
}
template <int S>
__device__ __forceinline__ uint32_t swizzle_of(int row) {
    return S == 64 ? ((row >> 1) & 3) << 4 : (row & 7) << 4;
}
// distance of two rows of a tile
template <int S>
constexpr int kRowStep = S == 256 ? 128 : S;

// Two CTAs per SM where 128 registers do: 8 rows, up to 128 value channels.  (16 rows of 64 channels, two CTAs with
// 432 bytes spilled and one, us: 3 x 13 drafts over 1501 tokens 24.1 and 20.9, 16 sequences over 4096 48.5 and 41.3,
// one over 131071 92.5 and 76.6.)
template <int NT, int NVB>
constexpr int min_ctas() { return NT == 1 && NVB <= 4 ? 2 : 1; }

// KS, VS: bytes of a key and a value row in shared memory.  WIDE: group 0 of
// both sides has 4-bit codes and group 1, where there is one, 8-bit codes;
// otherwise the widths are looked up block by block.
template <int NT, int NVB, int KS, int VS, bool WIDE>
__global__ void __launch_bounds__(256, (min_ctas<NT, NVB>()))
    kv_rows_kernel(const KvGeom geo, const KvAttendArgs a, const RowsPlan pl, const __grid_constant__ KvMaps maps) {
    extern __shared__ __align__(1024) uint8_t smem[];
    constexpr int R = 8 * NT;
    constexpr int KB = kChunk * KS, VB = kChunk * VS;      // bytes of a stage's rows
    constexpr int KR = kRowStep<KS>, VR = kRowStep<VS>;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
    const int g = lane >> 2, l = lane & 3;
    const KvSide &ks = geo.s[0], &vs = geo.s[1];
    const int nkb = ks.nb[0] + ks.nb[1], nvb = vs.nb[0] + vs.nb[1];
    const bool bf16 = geo.bf16 != 0;
    const uint32_t smem0 = tc::smem_u32(smem);
    // a warp's part: key rows of all stages, value rows; elsewhere its scales and, as fp32, those of the chunk in hand
    const uint32_t ring = smem0 + warp * pl.warp_bytes;
    const uint32_t v_ring = ring + pl.stages * KB;
    const uint32_t s_ring = smem0 + pl.s_off + warp * (pl.stages * pl.scale_bytes + 16 * kChunk);
    const uint32_t fsc = s_ring + pl.stages * pl.scale_bytes;
    const uint32_t bars = smem0 + pl.bar_off + warp * 32;
    float* merge = reinterpret_cast<float*>(smem);       // over the rings, which are empty when it is used
    // misc: per (row, group) start value, per row factor, the warps' statistics and the item's, the head's value channels
    float* sm_init = reinterpret_cast<float*>(smem + pl.misc_off);   // [2][R]
    float* sm_fac = sm_init + 2 * R;                                 // [R]
    float* sm_tm = sm_fac + R;                                       // [R]
    float* sm_tl = sm_tm + R;                                        // [R]
    float* sm_m = sm_tl + R;                                         // [8][R]
    float* sm_l = sm_m + 8 * R;                                      // [8][R]
    int16_t* sm_chan = reinterpret_cast<int16_t*>(sm_l + 8 * R);     // [32 NVB]
    uint32_t* sm_scan = reinterpret_cast<uint32_t*>(smem + pl.bar_off + 256);      // [32]
    int& sm_last = reinterpret_cast<int&>(sm_scan[32]);
    int& sm_abort = reinterpret_cast<int&>(sm_scan[33]);
    const uint32_t abort_flag = tc::smem_u32(&sm_abort);

    if (lane == 0) {
        for (int i = 0; i < pl.stages; ++i) tc::mbar_init(bars + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == 0) sm_abort = 0;

    // ---- this CTA's range of chunks --------------------------------------
    check_lengths(geo, a, tid, blockDim.x);
    auto chunks = [&](int b) { return (uint32_t)chunks_of(geo, a, b); };
    Split split;
    if (!split.begin(chunks, a.B, geo.heads * pl.row_tiles, pl.min_chunks, kLead, 2 * n_warps, sm_scan)) return;

    const int qh = geo.heads * a.group;
    const int n_min = ks.ng == 2 && ks.bits[1] < ks.bits[0] ? ks.bits[1] : ks.bits[0];
    const uint32_t k_sw = swizzle_of<KS>(g);                                       // rows 8 i + g
    const uint32_t v_sw0 = swizzle_of<VS>(2 * l), v_sw1 = swizzle_of<VS>(2 * l + 1);   // rows 8 i + 2 l, 8 i + 2 l + 1
    const Offsets offsets;
    // token `lane`'s scales in a stage
    const uint32_t ks_lane = 2 * ks.ng * (lane % pl.box_rows) + 128 * (lane / pl.box_rows);
    const uint32_t vs_lane = pl.scale_bytes / 2 + 2 * vs.ng * (lane % pl.box_rows) + 128 * (lane / pl.box_rows);
    uint32_t phases = 0, flying = 0;    // parity of each stage's next completion; stages with copies in flight
    while (true) {
        const Segment seg = split.segment(chunks);
        const int b = seg.entry, c_first = seg.c_first, c_end = seg.c_end, n_part = seg.n_part;
        const int head = seg.item / pl.row_tiles, rt = seg.item % pl.row_tiles;
        const int len = a.lengths[b];
        const int end = (int)seen_end(geo, a, b);
        const int row0 = rt * R;
        const int32_t* table = a.table + b * a.table_stride;

        // ---- loads of chunk c into stage s ----
        auto page_of = [&](int p) -> int { return p < end ? __ldg(table + (p >> geo.page_shift)) : -1; };
        auto issue = [&](int c, int s, int pg0, int pg1) {
            const int p0 = c * kChunk;
            const int boxes = p0 < end ? (pl.box_rows == kChunk || p0 + 16 >= end ? 1 : 2) : 0;
            const int box = pl.box_rows;
            const uint32_t bar = bars + 8 * s;
            flying |= 1u << s;
            const bool ok0 = (unsigned)pg0 < (unsigned)geo.n_pages, ok1 = (unsigned)pg1 < (unsigned)geo.n_pages;
            if (tc::elect_one()) {
                const int kx = KS == 256 && ks.row_bytes > 128 ? 2 : 1, vx = VS == 256 && vs.row_bytes > 128 ? 2 : 1;
                tc::mbar_arrive_expect_tx(bar, boxes * box * (kx * KR + vx * VR + 2 * (ks.ng + vs.ng)));
                for (int i = 0; i < boxes; ++i) {
                    const bool ok = i ? ok1 : ok0;
                    if (!ok) atomicOr(a.err, kErrKvIndex);
                    const int pg = ok ? (i ? pg1 : pg0) : (int)geo.n_pages;
                    const int row = head * geo.page + ((p0 + 16 * i) & (geo.page - 1));
                    const uint32_t kd = ring + s * KB + i * 16 * KR, vd = v_ring + s * VB + i * 16 * VR;
                    tma_load_3d(kd, &maps.codes[0], 0, row, pg, bar);
                    if (kx == 2) tma_load_3d(kd + KB / 2, &maps.codes[0], 128, row, pg, bar);
                    tma_load_3d(vd, &maps.codes[1], 0, row, pg, bar);
                    if (vx == 2) tma_load_3d(vd + VB / 2, &maps.codes[1], 128, row, pg, bar);
                    tc::tma_load_2d(s_ring + s * pl.scale_bytes + i * 128, &maps.scales[0], row * ks.ng, pg, bar);
                    tc::tma_load_2d(s_ring + s * pl.scale_bytes + pl.scale_bytes / 2 + i * 128, &maps.scales[1], row * vs.ng, pg, bar);
                }
            }
            __syncwarp();
        };
        {
            int pg0[4], pg1[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int c = c_first + warp + s * n_warps;
                pg0[s] = pg1[s] = -1;
                if (s < pl.stages && c < c_end) {
                    pg0[s] = page_of(c * kChunk);
                    pg1[s] = geo.page == 16 ? page_of(c * kChunk + 16) : pg0[s];
                }
            }
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int c = c_first + warp + s * n_warps;
                if (s < pl.stages && c < c_end && !(a.drop && c == 0 && blockIdx.x == 0)) issue(c, s, pg0[s], pg1[s]);
            }
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
                // all channels' numbers, then all queries: two waits for memory
                const int code0 = key_code(ks.bits[0], lane >> 3, (lane & 7) >> 1, lane & 1);
                const int code1 = key_code(ks.bits[1], lane >> 3, (lane & 7) >> 1, lane & 1);
                float x[8];
                int ch[8];
                uint32_t top = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const bool hi_group = k >= ks.nb[0];
                    const int p = hi_group ? 32 * (k - ks.nb[0]) + code1 : 32 * k + code0;
                    const bool in = on && k < nkb && p < (hi_group ? ks.count[1] : ks.count[0]);
                    ch[k] = in ? __ldg(perm + (hi_group ? ks.count[0] : 0) + p) : -1;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = ch[k] >= 0 ? scale_of(q[ch[k]], bf16) : 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(x[k]) & 0x7FFFFFFFu);
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
                    // positive, so that it can be applied behind the maximum; finite where queries are (of scores that
                    // large one takes the whole weight)
                    sm_fac[r] = fminf(fmaxf(ldexpf(fabsf(a.scale) * kLog2e, 24 - (n_min - 1) - e), 0x1p-126f), 0x1p126f);
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

        // A row's running maximum (in units of the exponent), sum, outputs and, for each value group, the power of two that
        // its outputs and weights are relative to, counted from the maximum (kv_device.cuh).
        float fac[NT][2], init[2][NT][2], m[NT][2], lsum[NT][2], power[2][NT][2];
        float o[NVB][2][NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                fac[nt][r] = sm_fac[8 * nt + 2 * l + r];
                init[0][nt][r] = sm_init[8 * nt + 2 * l + r];
                init[1][nt][r] = sm_init[R + 8 * nt + 2 * l + r];
                m[nt][r] = kUnset;
                power[0][nt][r] = power[1][nt][r] = kLeast;
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

        const uint32_t qbase = smem0 + pl.q_off + lane * 16;
        const int sure = min(len, end);
        int stage = 0;
        for (int c = c_first + warp; c < c_end; c += n_warps) {
            // the page ids of the chunk that will take this stage
            const int c_next = c + pl.stages * n_warps;
            int pg0 = -1, pg1 = -1;
            if (c_next < c_end) {
                pg0 = page_of(c_next * kChunk);
                pg1 = geo.page == 16 ? page_of(c_next * kChunk + 16) : pg0;
            }
            const int p0 = c * kChunk;
            const bool tail = p0 + kChunk > sure;      // some rows may not see some of it
            const uint32_t s_at = s_ring + stage * pl.scale_bytes;
            if (!tc::wait_bounded_warp(bars + 8 * stage, (phases >> stage) & 1u, abort_flag, kWaitNs, a.err, kErrWait)) break;
            phases ^= 1u << stage;
            flying &= ~(1u << stage);

            // ---- scales: lane = token; as fp32 for all lanes ----
            float room[2];      // of a row's largest weight over its power, for each value group
            {
                float k0, k1 = 0.0f, v0, v1 = 0.0f;
                if (ks.ng == 2) {
                    const uint32_t w = lds32(s_at + ks_lane);
                    k0 = scale_of(w & 0xFFFFu, bf16);
                    k1 = scale_of(w >> 16, bf16);
                } else {
                    k0 = scale_of(lds16(s_at + ks_lane), bf16);
                }
                if (vs.ng == 2) {
                    const uint32_t w = lds32(s_at + vs_lane);
                    v0 = value_scale(w & 0xFFFFu, bf16);
                    v1 = value_scale(w >> 16, bf16);
                } else {
                    v0 = value_scale(lds16(s_at + vs_lane), bf16);
                }
                if (tail && p0 + lane >= end) k0 = k1 = v0 = v1 = 0.0f;
                room[0] = kRoom - scale_bound(__reduce_max_sync(0xffffffffu, __float_as_uint(v0)));
                room[1] = vs.ng == 2 ? kRoom - scale_bound(__reduce_max_sync(0xffffffffu, __float_as_uint(v1))) : INFINITY;
                __syncwarp();
                sts128f(fsc + 16 * lane, k0, k1, v0, v1);
                __syncwarp();
            }
            float4 sc[4];      // of tokens g, g + 8, g + 16, g + 24
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[j] = lds128f(fsc + 16 * (8 * j + g));

            // ---- scores ----
            float x[2][NT][4];
            const uint32_t krow = ring + stage * KB + g * KR;
            auto key_group = [&](auto width, int grp, float(&acc)[2][NT][4]) {
                constexpr int BITS = decltype(width)::value;
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[mt][nt][i] = init[grp][nt][i & 1];
                uint32_t byte = ks.off[grp] + BITS * l;
                uint32_t qat = qbase + (grp ? ks.nb[0] : 0) * NT * 512;
                for (int blk = 0; blk < ks.nb[grp]; ++blk) {
                    const uint32_t at = krow + row_byte<KS>(byte, k_sw);
                    uint4 q[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) q[nt] = lds128(qat + nt * 512);
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        uint32_t h[4], k[4];
                        key_halves<BITS>(at + 16 * mt * KR, h);
                        key_halves<BITS>(at + (16 * mt + 8) * KR, k);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma(acc[mt][nt], h[0], k[0], h[1], k[1], q[nt].x, q[nt].y);
                            mma(acc[mt][nt], h[2], k[2], h[3], k[3], q[nt].z, q[nt].w);
                        }
                    }
                    byte += 4 * BITS;
                    qat += NT * 512;
                }
            };
            auto key_any = [&](auto grp, float(&acc)[2][NT][4]) {
                constexpr int G = decltype(grp)::value;
                if constexpr (WIDE) {
                    key_group(std::integral_constant<int, G ? 8 : 4>{}, G, acc);
                } else {
                    if (ks.bits[G] == 4) key_group(std::integral_constant<int, 4>{}, G, acc);
                    else if (ks.bits[G] == 8) key_group(std::integral_constant<int, 8>{}, G, acc);
                    else key_group(std::integral_constant<int, 2>{}, G, acc);
                }
            };
            key_any(std::integral_constant<int, 0>{}, x);
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[mt][nt][i] *= sc[2 * mt + (i >> 1)].x;
            if (ks.ng == 2) {
                float acc[2][NT][4];
                key_any(std::integral_constant<int, 1>{}, acc);
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
            float best[NT][2], to_exp[NT][2];       // a row's largest score, and the factor to units of the exponent
            bool grows = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float tp = fmaxf(fmaxf(x[0][nt][r], x[0][nt][2 + r]), fmaxf(x[1][nt][r], x[1][nt][2 + r]));
                    tp = fmaxf(tp, __shfl_xor_sync(0xffffffffu, tp, 4));
                    tp = fmaxf(tp, __shfl_xor_sync(0xffffffffu, tp, 8));
                    tp = fmaxf(tp, __shfl_xor_sync(0xffffffffu, tp, 16));
                    best[nt][r] = tp;
                    to_exp[nt][r] = exponent_factor(fac[nt][r], tp);
                    grows |= tp * to_exp[nt][r] > m[nt][r];
                }
            if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float top = best[nt][r] * to_exp[nt][r], by = raise(m[nt][r], top, top > m[nt][r]);
                        lsum[nt][r] *= ex2(-by);
                        const float rest = rest_of(by), steps = whole_steps(by);
                        power[0][nt][r] -= steps;
                        if (vs.ng == 2) power[1][nt][r] -= steps;
#pragma unroll
                        for (int v = 0; v < NVB; ++v)
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                o[v][u][nt][r] *= rest;
                                o[v][u][nt][2 + r] *= rest;
                            }
                    }
            }
            // where a row's weights times scales might leave fp16: the power that those it sees need; and the least one
            bool over = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float lead = fmaf(best[nt][r], to_exp[nt][r], -m[nt][r]);
                    over |= lead - power[0][nt][r] > room[0] || power[0][nt][r] < kLeast;
                    if (vs.ng == 2) over |= lead - power[1][nt][r] > room[1] || power[1][nt][r] < kLeast;
                }
            if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                for (int grp = 0; grp < 2; ++grp) {
                    if (grp >= vs.ng) break;
                    float down[NT][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            float z = -INFINITY;
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                z = fmaxf(z, fmaf(x[j >> 1][nt][2 * (j & 1) + r], to_exp[nt][r], -m[nt][r]) + lg2(grp ? sc[j].w : sc[j].z));
                            z = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, 4));
                            z = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, 8));
                            z = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, 16));
                            down[nt][r] = floor_power(power[grp][nt][r]);
                            down[nt][r] *= raise_power(power[grp][nt][r], z, z - power[grp][nt][r] > kRoom);
                        }
#pragma unroll
                    for (int v = 0; v < NVB; ++v)
                        if ((v < vs.nb[0]) == (grp == 0))
#pragma unroll
                            for (int u = 0; u < 2; ++u)
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                    for (int i = 0; i < 4; ++i) o[v][u][nt][i] *= down[nt][i & 1];
                }
            }
            uint32_t w[2][2][NT][2];      // weights as B fragments: [group][16 tokens][row tile][8 tokens]
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float a0 = unit_of(power[0][nt][0]), b0 = unit_of(power[0][nt][1]);
                const float a1 = unit_of(power[1][nt][0]), b1 = unit_of(power[1][nt][1]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float pa = ex2(fmaf(x[j >> 1][nt][2 * (j & 1)], to_exp[nt][0], -m[nt][0]));
                    const float pb = ex2(fmaf(x[j >> 1][nt][2 * (j & 1) + 1], to_exp[nt][1], -m[nt][1]));
                    lsum[nt][0] += pa;
                    lsum[nt][1] += pb;
                    w[0][j >> 1][nt][j & 1] = transpose8(pack2(pa * a0 * sc[j].z, pb * b0 * sc[j].z));
                    if (vs.ng == 2) w[1][j >> 1][nt][j & 1] = transpose8(pack2(pa * a1 * sc[j].w, pb * b1 * sc[j].w));
                }
            }

            // ---- outputs ----
            const uint32_t vrow = v_ring + stage * VB + 2 * l * VR;
            auto value_block = [&](auto width, uint32_t byte, const uint32_t(&wg)[2][NT][2], float(&ov)[2][NT][4]) {
                constexpr int BITS = decltype(width)::value;
                byte += BITS * g / 2;
                const uint32_t at0 = vrow + row_byte<VS>(byte, v_sw0);
                const uint32_t at1 = VS == 64 ? at0 + VR : vrow + row_byte<VS>(byte, v_sw1) + VR;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    uint32_t p[4], q[4];
                    value_pairs<BITS>(at0 + 16 * kt * VR, at1 + 16 * kt * VR, offsets, p);
                    value_pairs<BITS>(at0 + (16 * kt + 8) * VR, at1 + (16 * kt + 8) * VR, offsets, q);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma(ov[0][nt], p[0], p[1], q[0], q[1], wg[kt][nt][0], wg[kt][nt][1]);
                        mma(ov[1][nt], p[2], p[3], q[2], q[3], wg[kt][nt][0], wg[kt][nt][1]);
                    }
                }
            };
            auto value_any = [&](int grp, uint32_t blk, const uint32_t(&wg)[2][NT][2], float(&ov)[2][NT][4]) {
                if constexpr (!WIDE) {
                    const int bits = vs.bits[grp];
                    const uint32_t byte = vs.off[grp] + 4 * bits * blk;
                    if (bits == 4) value_block(std::integral_constant<int, 4>{}, byte, wg, ov);
                    else if (bits == 8) value_block(std::integral_constant<int, 8>{}, byte, wg, ov);
                    else value_block(std::integral_constant<int, 2>{}, byte, wg, ov);
                }
            };
            if constexpr (WIDE) {
#pragma unroll
                for (int v = 0; v < NVB; v += 2) {
                    if (v + 1 < vs.nb[0]) {
                        const uint32_t byte = 16 * v + 4 * g;
                        const uint32_t at0 = vrow + row_byte<VS>(byte, v_sw0);
                        const uint32_t at1 = VS == 64 ? at0 + VR : vrow + row_byte<VS>(byte, v_sw1) + VR;
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt) {
                            uint32_t p[4], q[4], p2[4], q2[4];
                            value_pairs2(at0 + 16 * kt * VR, at1 + 16 * kt * VR, offsets, p, p2);
                            value_pairs2(at0 + (16 * kt + 8) * VR, at1 + (16 * kt + 8) * VR, offsets, q, q2);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma(o[v][0][nt], p[0], p[1], q[0], q[1], w[0][kt][nt][0], w[0][kt][nt][1]);
                                mma(o[v][1][nt], p[2], p[3], q[2], q[3], w[0][kt][nt][0], w[0][kt][nt][1]);
                                mma(o[v + 1][0][nt], p2[0], p2[1], q2[0], q2[1], w[0][kt][nt][0], w[0][kt][nt][1]);
                                mma(o[v + 1][1][nt], p2[2], p2[3], q2[2], q2[3], w[0][kt][nt][0], w[0][kt][nt][1]);
                            }
                        }
                    } else {
                        if (v < vs.nb[0]) value_block(std::integral_constant<int, 4>{}, 16 * v, w[0], o[v]);
                        else if (v < nvb) value_block(std::integral_constant<int, 8>{}, vs.off[1] + 32 * (v - vs.nb[0]), w[1], o[v]);
                        if (v + 1 < nvb) value_block(std::integral_constant<int, 8>{}, vs.off[1] + 32 * (v + 1 - vs.nb[0]), w[1], o[v + 1]);
                    }
                }
            } else {
#pragma unroll
                for (int v = 0; v < NVB; ++v) {
                    if (v < vs.nb[0]) value_any(0, v, w[0], o[v]);
                    else if (v < nvb) value_any(1, v - vs.nb[0], w[1], o[v]);
                }
            }
            __syncwarp();
            if (c_next < c_end) issue(c_next, stage, pg0, pg1);
            if (++stage == pl.stages) stage = 0;
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
                if (g == 0) {
                    sm_m[warp * R + 8 * nt + 2 * l + r] = m[nt][r];
                    sm_l[warp * R + 8 * nt + 2 * l + r] = s;
                }
            }
        __syncthreads();
        if (tc::abort_raised(abort_flag)) {
            // a copy did not come: wait for the others of this warp, as long again, and leave
            for (int i = 0; i < pl.stages; ++i) {
                const long long t0 = tc::globaltimer();
                while ((flying >> i & 1u) && !tc::mbar_try_wait(bars + 8 * i, (phases >> i) & 1u) &&
                       tc::globaltimer() - t0 < kWaitNs) {
                }
            }
            return;
        }
        const bool whole = n_part == 1;
        constexpr int PART = R * (32 * NVB + 2);      // floats of a partial result: outputs (divided by l), then m, then l
        float* parts = reinterpret_cast<float*>(static_cast<uint8_t*>(a.scratch) + SONIQ_KV_SCRATCH_ZERO);
        float* part = parts + (int64_t)seg.slot * PART;
        if (tid < R) {
            float mm = kUnset, ll = 0.0f;
            for (int wi = 0; wi < n_warps; ++wi) mm = fmaxf(mm, sm_m[wi * R + tid]);
            for (int wi = 0; wi < n_warps; ++wi) ll += sm_l[wi * R + tid] * ex2(sm_m[wi * R + tid] - mm);
            sm_tm[tid] = mm;
            sm_tl[tid] = inverse(ll);
            if (!whole) {
                part[R * 32 * NVB + tid] = mm;
                part[R * 32 * NVB + R + tid] = ll;
            }
        }
        __syncthreads();
        // 2^(m - the CTA's m) / the CTA's sum: results are averages from here on, which are representable where sums
        // of values near the end of the type's range are not
        float join[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = 8 * nt + 2 * l + r;
                join[nt][r] = ex2(m[nt][r] - sm_tm[row]) * sm_tl[row];
            }
        auto store = [&](int r, int p, float v) {
            const int row = row0 + r, ch = sm_chan[p];
            if (row < pl.rows && ch >= 0) {
                const int64_t at = (((int64_t)b * a.T + row / a.group) * qh + head * a.group + row % a.group) * vs.D + ch;
                a.out[at] = bf16 ? kv_round<true>(v) : kv_round<false>(v);
            }
        };
        // the value blocks of one pass: 8 NT rows x 32 PB outputs of 8 warps in the merge buffer
        constexpr int PB = NT >= 2 || NVB == 2 ? 2 : 4;
#pragma unroll
        for (int v0 = 0; v0 < NVB; v0 += PB) {
#pragma unroll
            for (int vi = 0; vi < PB; ++vi) {
                const int v = v0 + vi;
                if (v < nvb) {
                    const int grp = v < vs.nb[0] ? 0 : 1, bits = vs.bits[grp];
                    const bool paired = WIDE && (v | 1) < vs.nb[0];      // value_pairs2's order
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float back = pow2(1 - bits - place_log2(bits, i));
                        const int code = paired ? value_code2(g, i) - 30 * (v & 1) : value_code(bits, g, i);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int r = 0; r < 2; ++r)
                                merge[((warp * R + 8 * nt + 2 * l + r) * PB + vi) * 32 + code] =
                                    (o[v][i >> 1][nt][2 * (i & 1) + r] * join[nt][r]) * (back * power_of(grp ? power[1][nt][r] : power[0][nt][r]));
                    }
                }
            }
            __syncthreads();
            for (int i = tid; i < R * PB * 32; i += blockDim.x) {
                const int r = i / (PB * 32), p = v0 * 32 + i % (PB * 32);
                if (p >= 32 * nvb) continue;
                float sum = 0.0f;
                for (int wi = 0; wi < n_warps; ++wi) sum += merge[wi * R * PB * 32 + i];
                if (whole) store(r, p, sum);
                else part[r * 32 * NVB + p] = sum;
            }
            __syncthreads();
        }
        if (!whole) {
            // the CTAs that share the item: the last to get here joins their parts in order
            unsigned* counter = static_cast<unsigned*>(a.scratch) + seg.cta0;
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const unsigned n = atomicAdd(counter, 1u);
                sm_last = n == (unsigned)(n_part - 1);
                if (sm_last) *counter = 0;
            }
            __syncthreads();
            if (sm_last) {
                __threadfence();
                auto part_of = [&](int i) { return parts + (int64_t)part_slot(seg, i) * PART; };
                float* fp = merge;                      // [n_part][R]: each part's share of the sum
                for (int i = tid; i < n_part * R; i += blockDim.x) fp[i] = __ldcg(part_of(i / R) + R * 32 * NVB + i % R);
                __syncthreads();
                for (int r = warp; r < R; r += n_warps) {
                    float mm = kUnset, ll = 0.0f;
                    for (int i = lane; i < n_part; i += 32) mm = fmaxf(mm, fp[i * R + r]);
                    for (int i = 16; i; i >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, i));
                    for (int i = lane; i < n_part; i += 32) {
                        const float f = ex2(fp[i * R + r] - mm) * __ldcg(part_of(i) + R * 32 * NVB + R + r);
                        ll += f;
                        fp[i * R + r] = f;
                    }
                    for (int i = 16; i; i >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, i);
                    for (int i = lane; i < n_part; i += 32) fp[i * R + r] *= inverse(ll);
                }
                __syncthreads();
                // four outputs to a thread; parts split over the threads that are left, and joined in order
                const int rows_used = min(R, pl.rows - row0), per_row = 8 * nvb, n_vec = rows_used * per_row;
                const int slices = n_vec < (int)blockDim.x ? (int)blockDim.x / n_vec : 1;
                float4* red = reinterpret_cast<float4*>(fp + (n_part * R + 3) / 4 * 4);
                for (int v0 = 0; v0 < n_vec; v0 += blockDim.x) {
                    const int slice = slices > 1 ? tid / n_vec : 0, v = slices > 1 ? tid % n_vec : v0 + tid;
                    const bool on = slice < slices && v < n_vec;
                    const int r = on ? v / per_row : 0, p = on ? 4 * (v % per_row) : 0;
                    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (on) {
#pragma unroll 8
                        for (int i = slice; i < n_part; i += slices) {
                            const float4 q = __ldcg(reinterpret_cast<const float4*>(part_of(i) + r * 32 * NVB + p));
                            const float f = fp[i * R + r];
                            acc.x = fmaf(f, q.x, acc.x);
                            acc.y = fmaf(f, q.y, acc.y);
                            acc.z = fmaf(f, q.z, acc.z);
                            acc.w = fmaf(f, q.w, acc.w);
                        }
                        red[tid] = acc;
                    }
                    __syncthreads();
                    if (on && slice == 0) {
                        for (int i = 1; i < slices; ++i) {
                            const float4 q = red[tid + i * n_vec];
                            acc.x += q.x;
                            acc.y += q.y;
                            acc.z += q.z;
                            acc.w += q.w;
                        }
                        store(r, p, acc.x);
                        store(r, p + 1, acc.y);
                        store(r, p + 2, acc.z);
                        store(r, p + 3, acc.w);
                    }
                    __syncthreads();
                }
            }
        }
        if (!split.next(seg)) break;
        // the next item's copies land where this one's results were joined
        tc::fence_proxy_async_shared();
        __syncthreads();
    }
}

constexpr int kMaxSmem = 227 * 1024, kHalfSmem = 228 * 1024 / 2 - 1024;

struct RowsLaunch {
    int nt, nvb, ks, vs, warps, ctas_per_sm;
    bool wide;
    RowsPlan pl;
};

RowsLaunch plan_rows(const KvGeom& geo, int64_t T, int64_t group) {
    RowsLaunch r{};
    const KvSide &ks = geo.s[0], &vs = geo.s[1];
    const int nkb = ks.nb[0] + ks.nb[1], nvb = vs.nb[0] + vs.nb[1];
    const int64_t rows = T * group;
    // the smallest of the built shapes that holds the rows
    if (ks.row_bytes <= 64 && vs.row_bytes <= 64 && nvb <= 2) r.nvb = 2, r.ks = 64, r.vs = 64;
    else if (ks.row_bytes <= 128 && vs.row_bytes <= 64 && nvb <= 4) r.nvb = 4, r.ks = 128, r.vs = 64;
    else if (ks.row_bytes <= 128 && vs.row_bytes <= 128 && nvb <= 4) r.nvb = 4, r.ks = 128, r.vs = 128;
    else r.nvb = 8, r.ks = 256, r.vs = 256;
    // (Four tiles of 8 rows to a warp do not fit its registers: 32 rows over 131071 tokens 270 us, as two tiles of 16 158.)
    r.nt = rows <= 8 ? 1 : 2;
    RowsPlan& p = r.pl;
    const int R = 8 * r.nt;
    p.rows = (int)rows;
    p.row_tiles = (int)((rows + R - 1) / R);
    p.box_rows = geo.page < kChunk ? geo.page : kChunk;
    p.scale_bytes = 256 * (kChunk / p.box_rows);
    const int stage = kChunk * (r.ks + r.vs);
    const int q = nkb * r.nt * 512;
    const int misc = (4 * (5 * R + 16 * R) + 2 * 32 * r.nvb + 15) / 16 * 16;
    const int fixed = q + misc + 256 + 192;
    auto warp_bytes = [&](int stages) { return stages * (stage + p.scale_bytes) + 16 * kChunk; };
    // two stages at least; two CTAs per SM where they and the registers allow it
    r.warps = 8;
    r.ctas_per_sm = r.nt == 1 && r.nvb <= 4 && fixed + 8 * warp_bytes(2) <= kHalfSmem ? 2 : 1;
    const int budget = r.ctas_per_sm == 2 ? kHalfSmem : kMaxSmem;
    if (fixed + 8 * warp_bytes(2) > budget) r.warps = 4;
    p.stages = 2;
    while (p.stages < 4 && fixed + r.warps * warp_bytes(p.stages + 1) <= budget) ++p.stages;
    p.warp_bytes = p.stages * stage;
    p.s_off = r.warps * p.warp_bytes;
    p.q_off = p.s_off + r.warps * (p.stages * p.scale_bytes + 16 * kChunk);
    p.misc_off = p.q_off + q;
    p.bar_off = p.misc_off + misc;
    p.smem = p.bar_off + 256 + 192;
    p.min_chunks = 8;
    r.wide = ks.bits[0] == 4 && vs.bits[0] == 4 && ks.bits[1] == 8 && vs.bits[1] == 8;
    return r;
}

template <int NT, int NVB, int KS, int VS>
cudaError_t run_rows(const KvGeom& geo, const KvAttendArgs& a, const RowsLaunch& r, const KvMaps& maps, int grid,
                     cudaStream_t st) {
    auto* kernel = r.wide ? kv_rows_kernel<NT, NVB, KS, VS, true> : kv_rows_kernel<NT, NVB, KS, VS, false>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, r.pl.smem);
    if (e == cudaSuccess) e = prefer_max_shared(reinterpret_cast<const void*>(kernel));
    if (e != cudaSuccess) return e;
    kernel<<<grid, 32 * r.warps, r.pl.smem, st>>>(geo, a, r.pl, maps);
    note_launch();
    return cudaGetLastError();
}

template <int NVB, int KS, int VS>
cudaError_t run_rows(const KvGeom& geo, const KvAttendArgs& a, const RowsLaunch& r, const KvMaps& maps, int grid,
                     cudaStream_t st) {
    if (r.nt == 1) return run_rows<1, NVB, KS, VS>(geo, a, r, maps, grid, st);
    return run_rows<2, NVB, KS, VS>(geo, a, r, maps, grid, st);
}

// Whether the rows of a key head go to the tile kernel: more than 32, where its operands fit.  (This kernel and that
// one, us, key groups of 96 and 32 channels: 16 sequences over up to 4096 tokens 16 rows 51 and 87, 32 rows 80 and 94,
// 48 rows 113 and 95; one over 131071 tokens 32 rows 158 and 175, 48 rows 216 and 179; over 500, 32 rows 22 and 30,
// 64 rows 25 and 31.  One key group, or heads of 64: the same side wins, 32 and 48 rows included, but for 64 channels
// over 131071, 32 rows 154 and 152.)
bool takes_tile(const KvGeom& geo, int64_t T, int64_t group) { return T * group > 32 && kv_tile_supported(geo, T, group); }

}  // namespace

int64_t kv_attend_scratch(const KvGeom& geo, int64_t B, int64_t T, int64_t group) {
    if (B == 0 || T == 0) return 0;
    if (takes_tile(geo, T, group)) return kv_tile_scratch(geo, T, group);
    const RowsLaunch r = plan_rows(geo, T, group);
    return SONIQ_KV_SCRATCH_ZERO + (int64_t)2 * r.ctas_per_sm * num_sms() * 8 * r.nt * (32 * r.nvb + 2) * 4;
}

cudaError_t launch_kv_attend(const KvGeom& geo, const KvAttendArgs& args, cudaStream_t st) {
    KvAttendArgs a = args;
    a.drop = take_drop_arrival();
    if (takes_tile(geo, a.T, a.group)) return launch_kv_tile(geo, a, st);
    const RowsLaunch r = plan_rows(geo, a.T, a.group);
    const int64_t cap = (int64_t)a.max_pages << geo.page_shift;
    const int64_t items = (int64_t)a.B * geo.heads * r.pl.row_tiles, most = items * (cap / kChunk + 1);
    if (most + items * kLead >= 2147483648ll) return cudaErrorNotSupported;      // chunks are numbered in 32 bits
    const int64_t by_size = (most + r.pl.min_chunks - 1) / r.pl.min_chunks;
    const int64_t want = by_size > items ? by_size : items, full = (int64_t)r.ctas_per_sm * num_sms();
    const int grid = (int)(want < full ? want : full);
    KvMaps maps;
    const int shared_row[2] = {r.ks, r.vs};
    for (int side = 0; side < 2; ++side) {
        const int row = shared_row[side];
        if (!encode_side(geo, geo.s[side], row < 128 ? row : 128, r.pl.box_rows,
                         row == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, &maps.codes[side],
                         &maps.scales[side]))
            return cudaErrorUnknown;
    }
    if (r.nvb == 2) return run_rows<2, 64, 64>(geo, a, r, maps, grid, st);
    if (r.nvb == 8) return run_rows<8, 256, 256>(geo, a, r, maps, grid, st);
    if (r.vs == 64) return run_rows<4, 128, 64>(geo, a, r, maps, grid, st);
    return run_rows<4, 128, 128>(geo, a, r, maps, grid, st);
}

}  // namespace soniq
