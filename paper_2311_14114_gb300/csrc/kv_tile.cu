// Attention of many query rows per key head over the quantized cache: drafted
// trees, pieces of prompts.
//
//   S = Q K^T, P = softmax(S), O = P V on tcgen05, accumulators in TMEM.
//
// With 128 rows to a tile the products (4 x 64 x 128 x 128 multiply-adds per 64
// tokens at 128 channels) and the exponentials are the work; the cache's bytes
// are read once per tile of up to 256 rows.  One CTA per SM, 20 warps:
//   warps 0, 3      issue the MMAs, each for one softmax group;
//   warp 1          copies packed rows by TMA;
//   warp 2          turns scales into fp32 and works out the next segment;
//   warps 4-7, 8-11 unpack a block of 64 tokens' keys, and values, into fp16
//                   operand tiles (codes exactly);
//   warps 12-15, 16-19  softmax of two row tiles (a thread per row, its scores from
//                   TMEM), each with its own S, P and O columns.
// (Registers move to the softmax warps: 64 + 2 x 56 + 2 x 152 = 5 x 96 a thread.)
// While one tile's softmax runs, the tensor cores work for the other.  With at
// most 128 rows both softmax groups serve the same tile on alternate blocks,
// as two streams joined at the end.
//
// Numerics.  Queries are fp16, each row scaled by a power of two to 2^13; codes
// are exact in fp16, so S is an exact product summed in fp32, per precision
// group, and gets its scales in fp32.  P times the value scale is rounded to fp16
// relative to a power of two of the row's own, which O is relative to (kv_device.cuh):
// O is rescaled only when a product leaves fp16's range above it.
//
// Values keep their row order (tokens x channels) as the MN-major operand of
// O = P V, so both operand tiles have one layout: 64-code column groups of
// [token][128 bytes], 16-byte pieces swizzled by the token.
//
// Bound by the softmax warps where scores have two buffers: about 3200 cycles for
// 64 tokens of 256 rows, of which the tensor cores work 630.  (2930 before rows had
// powers of two of their own: waits 340, scores times key scales 560, maxima and
// their check 750, exponentials and rounding 900, the rest the loop.)  With two key
// groups TMEM holds one buffer, and the way scores - softmax - outputs - scores is
// one chain of about 4600 cycles, two of which run side by side.  An item costs
// 12000 cycles for its queries and 5000 to 9000 for its results besides, so short
// items count kLead blocks more.
// Measured (GB300): 4 x 64 drafted tokens x 8 heads per key head over 16384
// cached ones 122 us (560 TFLOP/s), 2 x 512 x 4 over 3500 162 us (390), 16 x 24 x
// 4 over up to 4096 99 us.
#include <type_traits>

#include "kv_device.cuh"
#include "kv_flights.h"
#include "kv_split.cuh"
#include "soniq_device.cuh"
#include "tile_ops.cuh"

namespace soniq {

namespace {

constexpr int kTok = 64;                 // tokens of a block
constexpr int kThreads = 640;
constexpr int kAtom = kTok * 128;        // bytes of a 64-code column group of a K or V tile
constexpr int kQAtom = 128 * 128;        // ... of a query tile
constexpr int kSlotCols = 256;           // TMEM columns of a softmax group: S (and P over it), then O
// A row's running maximum may be exceeded by 2^kLazy before it is raised, and O with it.
constexpr float kLazy = 13.0f;
// Columns of a softmax group in front of O: scores (the weights of the first value group go over them), and those
// of the second key group or the weights of the second value group
__host__ __device__ constexpr int s_cols(int k_groups, int v_groups) { return k_groups == 2 ? 2 * kTok : (v_groups == 2 ? kTok + kTok / 2 : kTok); }

struct TilePlan {
    int rows;               // query rows per key head
    int tiles;              // row tiles of one CTA: 2, or 1 with two streams
    int row_units;          // CTA-sized tiles of rows per key head
    int k_atoms, v_atoms, v_atom1;   // column groups; v_atom1: the second precision group's first
    int o_cols;
    int stages, raw_stages, buffers;
    int stage_bytes, raw_bytes, raw_v, raw_s;     // raw_s: scales, 128 bytes or more for each copy
    int box_rows, scale_step[2];
    int ring_off, raw_off, misc_off, smem;
    int out_stride;         // bytes of a staged output row
    int min_chunks;
};

// An item whose parts the join kernel puts together: written by the CTA that has
// the first of them (n_part 0: none), one place per CTA behind the zeroed words
// of the scratch, in front of the parts.
struct JoinItem {
    int entry, item, n_part, cta0, cta0_slot;
};
constexpr int kJoinBytes = 8192;
// An item's queries and results take about as long as this many blocks.  (Blocks, us: 16 x 24 drafted tokens over
// ragged contexts 4: 113, 8: 100, 16: 92; 2 x 512 tokens 4: 161, 8: 162, 16: 177.)
constexpr int kLead = 8;

struct Bars {               // offsets in 8-byte barriers
    static constexpr int raw_full = 0, raw_free = 4, k_ready = 8, v_ready = 12, kv_free = 16, s_full = 20, p_full = 24,
                         pv_done = 28, o_full = 30, q_full = 32, drain = 33;      // s_full, p_full: [group][buffer]
};

// Eight codes as signed halves times their places' powers: of 8 bits ...
__device__ __forceinline__ void bytes8(uint32_t w0, uint32_t w1, const Offsets& f, uint32_t (&x)[4]) {
    x[0] = sub2(mask_flip(w0, 0x00FF00FFu, f.c128), f.c128);
    x[1] = sub2(mask_flip(w0 >> 8, 0x00FF00FFu, f.c128), f.c128);
    x[2] = sub2(mask_flip(w1, 0x00FF00FFu, f.c128), f.c128);
    x[3] = sub2(mask_flip(w1 >> 8, 0x00FF00FFu, f.c128), f.c128);
}
// ... and of 2 bits, from a half word.
__device__ __forceinline__ void crumbs8(uint32_t h, const Offsets& f, uint32_t (&x)[4]) {
    const uint32_t w = __byte_perm(h, 0, 0x4140);
    x[0] = sub2(mask_flip(w, 0x00030003u, 0x64026402u), 0x64026402u);
    x[1] = sub2(mask_flip(w, 0x000C000Cu, f.c8), f.c8);
    x[2] = sub2(mask_flip(w, 0x00300030u, 0x64206420u), 0x64206420u);
    x[3] = sub2(mask_flip(w, 0x00C000C0u, f.c128), f.c128);
}
__device__ __forceinline__ void sts128(uint32_t at, const uint32_t (&x)[4]) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
}
// 16 packed bytes from byte `at` (a multiple of 8) of the row at `row`, whose
// 16-byte pieces are swizzled by sw.
__device__ __forceinline__ uint4 packed16(uint32_t row, uint32_t at, uint32_t sw) {
    if ((at & 8u) == 0) return lds128(row + (at ^ sw));
    const uint2 a = lds64(row + (at ^ sw)), b = lds64(row + ((at + 8) ^ sw));
    return make_uint4(a.x, a.y, b.x, b.y);
}
// The 32-code block at byte `at` of a packed row -> 16-byte pieces p0 .. p0 + 3 of
// the operand row at `to`, swizzled by t8 = token % 8.
template <int BITS>
__device__ __forceinline__ void unpack_block(uint32_t row, uint32_t at, uint32_t sw, uint32_t to, uint32_t p0, uint32_t t8,
                                             const Offsets& f) {
    uint32_t x[4][4];
    if constexpr (BITS == 4) {
        const uint4 w = packed16(row, at, sw);
        nibble_pairs(w.x, f, x[0]);
        nibble_pairs(w.y, f, x[1]);
        nibble_pairs(w.z, f, x[2]);
        nibble_pairs(w.w, f, x[3]);
    } else if constexpr (BITS == 8) {
        const uint4 w = packed16(row, at, sw), v = packed16(row, at + 16, sw);
        bytes8(w.x, w.y, f, x[0]);
        bytes8(w.z, w.w, f, x[1]);
        bytes8(v.x, v.y, f, x[2]);
        bytes8(v.z, v.w, f, x[3]);
    } else {
        const uint2 w = lds64(row + (at ^ sw));
        crumbs8(w.x & 0xFFFFu, f, x[0]);
        crumbs8(w.x >> 16, f, x[1]);
        crumbs8(w.y & 0xFFFFu, f, x[2]);
        crumbs8(w.y >> 16, f, x[3]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sts128(to + (((p0 + i) ^ t8) << 4), x[i]);
}

// Column `col` (of its group's unpacked codes) -> code of the group.
__device__ __forceinline__ int column_code(int bits, int col) {
    return 32 * (col >> 5) + key_code(bits, (col >> 3) & 3, (col & 7) >> 1, col & 1);
}

// KNG, VNG: precision groups of keys and values.  SB: buffers of scores (2 where
// TMEM has room: the next block's scores are there when this one's softmax ends).
template <int KNG, int VNG, int SB>
__global__ void __launch_bounds__(kThreads, 1)
    kv_tile_kernel(const KvGeom geo, const KvAttendArgs a, const TilePlan pl, const __grid_constant__ KvMaps maps) {
    extern __shared__ __align__(1024) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const KvSide &ks = geo.s[0], &vs = geo.s[1];
    const bool bf16 = geo.bf16 != 0;
    const uint32_t smem0 = tc::smem_u32(smem);
    const uint32_t ring = smem0 + pl.ring_off, raw = smem0 + pl.raw_off;
    uint8_t* misc = smem + pl.misc_off;
    const uint32_t bars = smem0 + pl.misc_off;
    uint32_t* words = reinterpret_cast<uint32_t*>(misc + 320);       // [32] for the split, then:
    const uint32_t abort_flag = tc::smem_u32(words + 32);
    uint32_t* tmem_at = words + 33;
    float* sm_fac = reinterpret_cast<float*>(misc + 512);            // [256] factor of a row's scores
    float* sm_m = sm_fac + 256;                                      // [128], of the second stream
    float* sm_l = sm_m + 128;
    int16_t* sm_chan = reinterpret_cast<int16_t*>(sm_l + 128);       // [192] channel of an output column
    float* sm_back = reinterpret_cast<float*>(sm_chan + 192);        // [192] its power of two
    int16_t* sm_col = reinterpret_cast<int16_t*>(sm_back + 192);     // [256] column of a key channel
    Segment* sm_seg = reinterpret_cast<Segment*>(sm_col + 256);      // the next segment, behind a flag that there is one
    int* sm_more = reinterpret_cast<int*>(sm_seg + 1);
    float2* sm_span = reinterpret_cast<float2*>(misc + 4608);        // [4 stages][2]: log2 of the largest and smallest value scale
    float* sm_up = reinterpret_cast<float*>(sm_span + 8);            // [4 stages]: what the keys' scales were divided by
    auto bar = [&](int i) { return bars + 8u * i; };

    if (tid == 0) {
        for (int i = 0; i < 4; ++i) {
            tc::mbar_init(bar(Bars::raw_full + i), 1);
            tc::mbar_init(bar(Bars::raw_free + i), 9);
            tc::mbar_init(bar(Bars::k_ready + i), 5);
            tc::mbar_init(bar(Bars::v_ready + i), 5);
            tc::mbar_init(bar(Bars::kv_free + i), pl.tiles);
            tc::mbar_init(bar(Bars::s_full + i), 1);
            tc::mbar_init(bar(Bars::p_full + i), 4);
        }
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(bar(Bars::pv_done + i), 1);
            tc::mbar_init(bar(Bars::o_full + i), 1);
        }
        tc::mbar_init(bar(Bars::q_full), 8);
        tc::mbar_init(bar(Bars::drain), 2);
        words[32] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }

    // ---- this CTA's share: entries are (sequence, unit of row tiles) ----
    const int unit_rows = 128 * pl.tiles;
    auto last_token = [&](int u) { return (min((u + 1) * unit_rows, pl.rows) - 1) / a.group; };
    auto end_of = [&](int b, int u) {      // tokens that any row of the unit may see
        const int64_t end = seen_end(geo, a, b);
        const int64_t chain = (int64_t)a.lengths[b] + last_token(u) + 1;
        return (int)(a.mask == nullptr && chain < end ? chain : end);
    };
    auto chunks = [&](int e) -> uint32_t {
        const int b = e / pl.row_units;
        if (a.lengths[b] < 0) return 0;
        const int end = end_of(b, e % pl.row_units);
        return end == 0 ? 1 : (end + kTok - 1) / kTok;      // a present sequence's rows are written even if they see nothing
    };
    Split split;
    JoinItem* join = reinterpret_cast<JoinItem*>(static_cast<uint8_t*>(a.scratch) + SONIQ_KV_SCRATCH_ZERO) + blockIdx.x;
    const bool any = split.begin(chunks, a.B * pl.row_units, geo.heads, pl.min_chunks, kLead, 8, words);
    if (tid == 0) join->n_part = 0;
    if (!any) {
        check_lengths(geo, a, tid, kThreads);
        return;
    }

    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(tmem_at)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_at;
    constexpr uint32_t p1_off = kTok;            // the second value group's weights, behind the first scores
    constexpr uint32_t o_off = SB * s_cols(KNG, VNG);     // O's first column in a slot
    const int nkb = ks.nb[0] + ks.nb[1];
    const int pa0 = 32 * ks.nb[0], pa1 = 32 * ks.nb[1], va0 = 32 * vs.nb[0], va1 = 32 * vs.nb[1];

    auto wait = [&](int i, uint32_t parity) {
        return wait_warp(bar(i), parity & 1u, abort_flag, a.err);
    };
    auto wait2 = [&](int i, uint32_t pi, int j, uint32_t pj) {
        return wait_warp2(bar(i), pi & 1u, bar(j), pj & 1u, abort_flag, a.err);
    };
    auto wait3 = [&](int i, uint32_t pi, int j, uint32_t pj, int k, uint32_t pk) {
        return wait_warp3(bar(i), pi & 1u, bar(j), pj & 1u, bar(k), pk & 1u, abort_flag, a.err);
    };
    // where the next segment's blocks begin in the rings; parities of the softmax groups'
    // scores and weights, blocks done and results (bit s), and of the queries'
    Ring kv0, raw0;
    uint32_t s_phase = 0, p_phase = 0, o_phase = 0, q_phase = 0;      // s: bit 2 group + buffer
    bool ok = true, checked = false;

    const Segment first = split.segment(chunks);
    auto work = [&](auto role) {
    constexpr int ROLE = decltype(role)::value;      // 0 softmax, 1 unpacking, 2 MMAs and copies
    Segment seg = first;
    Flights flights;        // of the copying warp
    while (true) {
        const int b = seg.entry / pl.row_units, unit = seg.entry % pl.row_units, head = seg.item;
        const int row0 = unit * unit_rows;
        const int len = a.lengths[b], end = end_of(b, unit);
        const int nblk = seg.c_end - seg.c_first;
        // row tiles at work, or streams: group s takes every block of its tile, or every second block
        const int groups = pl.tiles == 2 ? (row0 + 128 < pl.rows ? 2 : 1) : (nblk > 1 ? 2 : 1);
        const bool streams = pl.tiles == 1;

        if (ROLE == 2 && warp == 1) {
            // ---- copies ----
            const int32_t* table = a.table + b * a.table_stride;
            Ring ring_r = raw0;
#pragma unroll 1
            for (int j = 0; ok && j < nblk; ++j, ring_r.step(pl.raw_stages)) {
                const int r = ring_r.i;
                const int p0 = (seg.c_first + j) * kTok;
                const int boxes = p0 < end ? min(kTok / pl.box_rows, (end - p0 + pl.box_rows - 1) / pl.box_rows) : 0;
                int page = -1;
                if (lane < boxes) page = __ldg(table + ((p0 + lane * pl.box_rows) >> geo.page_shift));
                const bool good = (unsigned)page < (unsigned)geo.n_pages;
                if (lane < boxes && !good) atomicOr(a.err, kErrKvIndex);
                if (!good) page = (int)geo.n_pages;        // reads as zeros
                ok = wait(Bars::raw_free + r, ring_r.phase ^ 1u);
                if (!ok) break;
                if (a.drop && j == 0 && blockIdx.x == 0) continue;
                flights.issue(r, ring_r.phase);
                const uint32_t at = raw + r * pl.raw_bytes, full = bar(Bars::raw_full + r);
                if (tc::elect_one()) tc::mbar_arrive_expect_tx(full, boxes * pl.box_rows * (ks.row_bytes + vs.row_bytes + 2 * (ks.ng + vs.ng)));
#pragma unroll 1
                for (int i = 0; i < boxes; ++i) {
                    const int pg = __shfl_sync(0xffffffffu, page, i);
                    const int row = head * geo.page + ((p0 + i * pl.box_rows) & (geo.page - 1));
                    if (tc::elect_one()) {
                        tma_load_3d(at + i * pl.box_rows * ks.row_bytes, &maps.codes[0], 0, row, pg, full);
                        tma_load_3d(at + pl.raw_v + i * pl.box_rows * vs.row_bytes, &maps.codes[1], 0, row, pg, full);
                        tc::tma_load_2d(at + pl.raw_s + i * pl.scale_step[0], &maps.scales[0], row * ks.ng, pg, full);
                        tc::tma_load_2d(at + pl.raw_s + kTok / pl.box_rows * pl.scale_step[0] + i * pl.scale_step[1],
                                        &maps.scales[1], row * vs.ng, pg, full);
                    }
                }
            }
        } else if (ROLE == 2 && (warp == 0 || warp == 3)) {
            // ---- MMAs of softmax group s ----
            const int s = warp == 0 ? 0 : 1, step = streams ? 2 : 1;
            const int mine = s < groups ? (streams ? (nblk - s + 1) / 2 : nblk) : 0;
            constexpr uint32_t fmt = (1u << 4) | ((128u >> 4) << 24);
            const uint32_t id_s = fmt | ((kTok >> 3) << 17);
            const uint32_t id_o0 = fmt | (1u << 16) | ((uint32_t)(va0 >> 3) << 17), id_o1 = fmt | (1u << 16) | ((uint32_t)(va1 >> 3) << 17);
            const uint32_t t_s = tmem + s * kSlotCols;
            const uint64_t q_tile = tc::sw128_desc(smem0 + (streams ? 0 : s * pl.k_atoms * kQAtom));
            // every lane runs the loops, the elected one issues
            const bool leader = tc::elect_one();
            if (mine > 0) ok = wait(Bars::q_full, q_phase);
            tc::tc_fence_after();
            Ring now = kv0, next = kv0;       // the block whose outputs, and whose scores, come next
            if (streams && s == 1) now.step(pl.stages), next.step(pl.stages);
            auto advance = [&](Ring& r) {
                r.step(pl.stages);
                if (step == 2) r.step(pl.stages);
            };
            uint32_t phases = s_phase >> (2 * s);      // of the weights in each buffer, as of the scores
            // Scores run SB blocks ahead of the outputs.  Where the ring has a place for the next scores' keys that no
            // outputs of this block or later free, one wait covers both.
            const bool early = pl.stages > SB * step;
#pragma unroll 1
            for (int i = -SB; ok && i < mine; ++i) {
                const int buf = SB == 2 ? i & 1 : 0;
                if (i >= 0) {
                    const int nx = i + SB < mine && early ? Bars::k_ready + next.i : Bars::v_ready + now.i;
                    ok = wait3(Bars::p_full + 2 * s + buf, phases >> buf, Bars::v_ready + now.i, now.phase, nx,
                               i + SB < mine && early ? next.phase : now.phase);
                    if (!ok) break;
                    tc::tc_fence_after();
                    phases ^= 1u << buf;
                    uint64_t v = value_desc(ring + now.i * pl.stage_bytes + pl.k_atoms * kAtom, kAtom);
                    uint32_t p = t_s + buf * s_cols(KNG, VNG);
                    const uint32_t d = t_s + o_off;
#pragma unroll 1
                    for (int k = 0; k < kTok / 16; k += 2) {
                        if (leader) {
                            mma_ts(d, p, v, id_o0, i != 0 || k != 0);
                            mma_ts(d, p + 8, v + (2048 >> 4), id_o0, 1);
                            if (VNG == 2) {
                                const uint64_t v1 = v + pl.v_atom1 * (kAtom >> 4);
                                mma_ts(d + va0, p + p1_off, v1, id_o1, i != 0 || k != 0);
                                mma_ts(d + va0, p + p1_off + 8, v1 + (2048 >> 4), id_o1, 1);
                            }
                        }
                        v += 2 * (2048 >> 4);
                        p += 16;
                    }
                    if (leader) {
                        tc::mma_commit(bar(Bars::kv_free + now.i));
                        if (!streams && groups == 1) tc::mma_commit(bar(Bars::kv_free + now.i));     // for the group without rows
                        if (SB == 2) tc::mma_commit(bar(Bars::pv_done + s));
                        if (i == mine - 1) tc::mma_commit(bar(Bars::o_full + s));
                    }
                    __syncwarp();
                    advance(now);
                }
                if (i + SB < mine) {
                    if (i < 0 || !early) {
                        ok = wait(Bars::k_ready + next.i, next.phase);
                        if (!ok) break;
                        tc::tc_fence_after();
                    }
                    uint64_t q = q_tile, k = tc::sw128_desc(ring + next.i * pl.stage_bytes);
                    const uint32_t d = t_s + buf * s_cols(KNG, VNG);
                    // 32-code halves of column groups, two MMAs each
#pragma unroll 1
                    for (int h = 0; h < nkb; ++h) {
                        const bool second = KNG == 2 && h >= ks.nb[0];
                        if (leader) {
                            mma_ss(d + (second ? kTok : 0), q, k, id_s, h != 0 && (KNG == 1 || h != ks.nb[0]));
                            mma_ss(d + (second ? kTok : 0), q + 2, k + 2, id_s, 1);
                        }
                        q += h & 1 ? (kQAtom - 64) >> 4 : 4;
                        k += h & 1 ? (kAtom - 64) >> 4 : 4;
                    }
                    if (leader) tc::mma_commit(bar(Bars::s_full + 2 * s + buf));
                    __syncwarp();
                    advance(next);
                }
            }
        } else if (ROLE == 2 && warp == 2) {
            // ---- the segment after this one, and scales ----
            const bool more = split.next(seg);
            if (more) *sm_seg = split.segment(chunks);
            *sm_more = more;
            // ---- scales as fp32, keys' with 2^-(n-1); two tokens to a lane.  Exact products reach 2^28 before they get
            // their scales, so those above 2^90 are brought down to it with the block, and scores stay in fp32's range where
            // their softmax argument does. ----
            uint32_t from[2][2];        // [side][token]
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                const int ng = side ? VNG : KNG, at0 = pl.raw_s + (side ? kTok / pl.box_rows * pl.scale_step[0] : 0);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int t = lane + 32 * h;
                    from[side][h] = at0 + (t / pl.box_rows) * pl.scale_step[side] + 2 * ng * (t % pl.box_rows);
                }
            }
            Ring kv = kv0, rw = raw0;
#pragma unroll 1
            for (int j = 0; ok && j < nblk; ++j, kv.step(pl.stages), rw.step(pl.raw_stages)) {
                const int st = kv.i, r = rw.i, p0 = (seg.c_first + j) * kTok;
                ok = wait2(Bars::kv_free + st, kv.phase ^ 1u, Bars::raw_full + r, rw.phase);
                if (!ok) break;
                const uint32_t src = raw + r * pl.raw_bytes, to = ring + st * pl.stage_bytes + (pl.k_atoms + pl.v_atoms) * kAtom + 4 * lane;
                auto scale = [&](int side, int grp, int h) {
                    const uint32_t raw16 = lds16(src + from[side][h] + 2 * grp);
                    return p0 + lane + 32 * h >= end ? 0.0f : (side ? value_scale(raw16, bf16) : scale_of(raw16, bf16));
                };
                auto put = [&](int side, int grp, float x0, float x1) {
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + 512 * side + 256 * grp), "f"(x0) : "memory");
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + 512 * side + 256 * grp + 128), "f"(x1) : "memory");
                };
                float k[KNG][2];
                uint32_t top = 0;       // (a token that no row sees may hold anything: not finite, it does not count)
#pragma unroll
                for (int i = 0; i < 2 * KNG; ++i) {
                    k[i >> 1][i & 1] = scale(0, i >> 1, i & 1);
                    const uint32_t mag = __float_as_uint(k[i >> 1][i & 1]) & 0x7FFFFFFFu;
                    top = max(top, mag < 0x7F800000u ? mag : 0u);
                }
                const int by = max((int)ceilf(scale_bound(__reduce_max_sync(0xffffffffu, top))) - 90, 0);
                if (lane == 0) sm_up[st] = pow2(by);
#pragma unroll
                for (int grp = 0; grp < KNG; ++grp) {
                    const float f = pow2(1 - ks.bits[grp] - by);
                    put(0, grp, k[grp][0] * f, k[grp][1] * f);
                }
#pragma unroll
                for (int grp = 0; grp < VNG; ++grp) {
                    const float x0 = scale(1, grp, 0), x1 = scale(1, grp, 1);
                    const uint32_t big = __reduce_max_sync(0xffffffffu, max(__float_as_uint(x0), __float_as_uint(x1)));
                    // (beyond the end: none)
                    const uint32_t a0 = p0 + lane >= end ? big : __float_as_uint(x0), a1 = p0 + lane + 32 >= end ? big : __float_as_uint(x1);
                    const uint32_t least = __reduce_min_sync(0xffffffffu, min(a0, a1));
                    if (lane == 0) sm_span[2 * st + grp] = make_float2(scale_bound(big), scale_floor(least));
                    put(1, grp, x0, x1);
                }
                __syncwarp();
                if (lane == 0) {
                    tc::mbar_arrive(bar(Bars::k_ready + st));
                    tc::mbar_arrive(bar(Bars::v_ready + st));
                    tc::mbar_arrive(bar(Bars::raw_free + r));
                }
            }
            if (!checked) check_lengths(geo, a, lane, 32);
            checked = true;
        } else if constexpr (ROLE == 1) {
            // ---- packed rows -> operand tiles: keys by one warpgroup, values by the other ----
            const int side = warp >= 8 ? 1 : 0, dw = warp & 3, tok = (dw & 1) * 32 + lane;
            const KvSide& sd = geo.s[side];
            const Offsets f;
            const uint32_t raw_sw = sd.row_bytes == 64 ? ((tok >> 1) & 3) << 4 : (sd.row_bytes == 128 ? (tok & 7) << 4 : 0);
            Ring kv = kv0, rw = raw0;
#pragma unroll 1
            for (int j = 0; ok && j < nblk; ++j, kv.step(pl.stages), rw.step(pl.raw_stages)) {
                const int st = kv.i, r = rw.i;
                const uint32_t at = ring + st * pl.stage_bytes, src = raw + r * pl.raw_bytes;
                ok = wait2(Bars::kv_free + st, kv.phase ^ 1u, Bars::raw_full + r, rw.phase);
                if (!ok) break;
                // a lane takes a token, two warps every second block
                const uint32_t base = src + (side ? pl.raw_v : 0) + tok * sd.row_bytes;
                const uint32_t to = at + (side ? pl.k_atoms * kAtom : 0) + tok * 128;
#pragma unroll 1
                for (int blk = dw >> 1; blk < sd.nb[0] + sd.nb[1]; blk += 2) {
                    const int grp = blk < sd.nb[0] ? 0 : 1, bb = grp ? blk - sd.nb[0] : blk, bits = sd.bits[grp];
                    const uint32_t byte = sd.off[grp] + 4 * bits * bb;
                    // keys' groups follow each other, values' start a column group each
                    const int col = side && grp ? 64 * pl.v_atom1 + 32 * bb : 32 * blk;
                    const uint32_t row = to + (col >> 6) * kAtom, p0 = (col >> 3) & 7;
                    if (bits == 4) unpack_block<4>(base, byte, raw_sw, row, p0, tok & 7, f);
                    else if (bits == 8) unpack_block<8>(base, byte, raw_sw, row, p0, tok & 7, f);
                    else unpack_block<2>(base, byte, raw_sw, row, p0, tok & 7, f);
                }
                tc::fence_proxy_async_shared();
                __syncwarp();
                if (lane == 0) {
                    tc::mbar_arrive(bar((side ? Bars::v_ready : Bars::k_ready) + st));
                    tc::mbar_arrive(bar(Bars::raw_free + r));
                }
            }
        } else if constexpr (ROLE == 0) {
            // ---- softmax ----
            const int s = (warp >> 2) - 3, quad = warp & 3, st_id = tid - 384;
            // queries: fp16, each row scaled to 2^13; a lane takes eight channels (of 128) of a row
            {
                const int total = groups == 2 && !streams ? 256 : 128, cols = pa0 + pa1;
                for (int c = st_id; c < cols; c += 256) {
                    const int grp = c < pa0 ? 0 : 1, code = column_code(ks.bits[grp], grp ? c - pa0 : c);
                    if (code < ks.count[grp]) sm_col[__ldg(ks.perm + head * ks.D + (grp ? ks.count[0] : 0) + code)] = (int16_t)c;
                }
                for (int c = st_id; c < pl.o_cols; c += 256) {
                    const int grp = c < va0 ? 0 : 1, code = column_code(vs.bits[grp], grp ? c - va0 : c);
                    sm_chan[c] = code < vs.count[grp] ? (int16_t)__ldg(vs.perm + head * vs.D + (grp ? vs.count[0] : 0) + code) : (int16_t)-1;
                    sm_back[c] = pow2(1 - vs.bits[grp] - place_log2(vs.bits[grp], (c & 7) >> 1));
                }
                const int r_first = (warp - 12) * (total / 8), r_end = r_first + total / 8;
                if (cols != ks.D) {      // columns without a channel
                    for (int i = lane; i < (r_end - r_first) * 8 * pl.k_atoms; i += 32) {
                        const int r = r_first + (i & (total / 8 - 1)), p = i / (total / 8);
                        *reinterpret_cast<uint4*>(smem + ((r >> 7) * pl.k_atoms + (p >> 3)) * kQAtom + (r & 127) * 128 + (p & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                }
                bar_group(1, 256);
                const bool wide = ks.D % 8 == 0 && (((uintptr_t)a.Q | (uintptr_t)(2 * a.q_seq_stride) | (uintptr_t)(2 * a.q_token_stride) |
                                                     (uintptr_t)(2 * a.q_head_stride)) & 15u) == 0;
                const float fac0 = fabsf(a.scale) * kLog2e, sign = a.scale < 0.0f ? -1.0f : 1.0f;
                auto fill = [&](auto halves) {
                    constexpr int H = decltype(halves)::value;      // 128 channels each
                    const int half = lane >> 4, l16 = lane & 15;
                    uint32_t to[8 * H];
                    float down[8 * H];
#pragma unroll
                    for (int k = 0; k < 8 * H; ++k) {
                        const int ch = 128 * (k >> 3) + 8 * l16 + (k & 7);
                        const int col = ch < ks.D ? sm_col[ch] : 0, bits = ks.bits[col < pa0 ? 0 : 1];
                        to[k] = (col >> 6) * kQAtom + ((col & 63) >> 3) * 16 + 2 * (col & 7);
                        down[k] = sign * pow2(-place_log2(bits, (col & 7) >> 1));
                    }
                    // each half of the warp takes every second row: two rows' loads go out while the two before are
                    // scaled and stored
                    int row = row0 + r_first + half, t = row / a.group, hq = row - t * a.group;
                    const uint16_t* q0 = a.Q + b * a.q_seq_stride + (int64_t)head * a.group * a.q_head_stride;
                    auto load = [&](uint4(&v)[2][H]) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint16_t* q = q0 + t * a.q_token_stride + hq * a.q_head_stride + 8 * l16;
                            const bool on = row < pl.rows;
#pragma unroll
                            for (int h = 0; h < H; ++h) {
                                const int left = ks.D - 128 * h - 8 * l16;      // channels from this lane's on
                                v[i][h] = make_uint4(0, 0, 0, 0);
                                if (wide && on && left > 0) {
                                    v[i][h] = *reinterpret_cast<const uint4*>(q + 128 * h);
                                } else if (on && !wide) {
                                    uint32_t x[8];
#pragma unroll
                                    for (int k = 0; k < 8; ++k) x[k] = k < left ? (uint32_t)q[128 * h + k] : 0u;
                                    v[i][h] = make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
                                }
                            }
                            row += 2;
                            hq += 2;
#pragma unroll
                            for (int k = 0; k < 2; ++k)
                                if (hq >= a.group) hq -= a.group, ++t;
                        }
                    };
                    uint4 v[2][H];
                    load(v);
#pragma unroll 1
                    for (int r0 = r_first + half; r0 < r_end; r0 += 4) {
                        uint4 w[2][H];
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int h = 0; h < H; ++h) w[i][h] = v[i][h];
                        if (r0 + 4 < r_end) load(v);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int r = r0 + 2 * i;
                            uint32_t most = 0;      // magnitudes order as their patterns
#pragma unroll
                            for (int h = 0; h < H; ++h)
                                most = __vmaxu2(__vmaxu2(__vmaxu2(most, w[i][h].x & 0x7FFF7FFFu), w[i][h].y & 0x7FFF7FFFu),
                                                __vmaxu2(w[i][h].z & 0x7FFF7FFFu, w[i][h].w & 0x7FFF7FFFu));
#pragma unroll
                            for (int k = 8; k; k >>= 1) most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, k));
                            const uint32_t top = __float_as_uint(scale_of(max(most & 0xFFFFu, most >> 16), bf16));
                            const int e = top == 0 ? 0 : min(13 - ((int)(top >> 23) - 127), 120);
                            const float up = pow2(e);
                            if (l16 == 0) sm_fac[r] = fmaxf(fac0 * pow2(-e), 0x1p-126f);
                            const uint32_t q = smem0 + (r >> 7) * pl.k_atoms * kQAtom + (r & 127) * 128, sw = (r & 7) << 4;
#pragma unroll
                            for (int k = 0; k < 8 * H; ++k) {
                                const uint4& u = w[i][k >> 3];
                                const uint32_t pair = (k >> 1 & 3) == 0 ? u.x : ((k >> 1 & 3) == 1 ? u.y : ((k >> 1 & 3) == 2 ? u.z : u.w));
                                const float x = scale_of(k & 1 ? pair >> 16 : pair & 0xFFFFu, bf16);
                                if (128 * (k >> 3) + 8 * l16 + (k & 7) < ks.D)
                                    asm volatile("st.shared.b16 [%0], %1;" ::"r"(q + (to[k] ^ sw)),
                                                 "h"(__half_as_ushort(__float2half_rn(x * (up * down[k]))))
                                                 : "memory");
                            }
                        }
                    }
                };
                if (ks.D <= 128) fill(std::integral_constant<int, 1>{});
                else fill(std::integral_constant<int, 2>{});
                tc::fence_proxy_async_shared();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(bar(Bars::q_full));
            }
            bar_group(1, 256);      // the rows' factors
            const int r_tile = quad * 32 + lane;                               // row of the tile
            const int row = row0 + (streams ? 0 : 128 * s) + r_tile;
            const int t_row = row < pl.rows ? row / a.group : a.T - 1;
            const float fac = sm_fac[(streams ? 0 : 128 * s) + r_tile];
            const uint32_t lanes = (uint32_t)(quad * 32) << 16;
            const uint32_t t_s = tmem + s * kSlotCols + lanes;
            // the maximum (in units of the exponent), the sum, and each value group's power of two (kv_device.cuh) that
            // weights and outputs are relative to
            float m = kUnset, l = 0.0f, power0 = kLeast, power1 = kLeast;
            const int mine = s < groups ? (streams ? (nblk - s + 1) / 2 : nblk) : 0;
            const int sure = min(len, end);
            Ring kv = kv0;
            if (streams && s == 1) kv.step(pl.stages);
            uint32_t phases = s_phase >> (2 * s), done = p_phase >> s;      // of the score buffers, and of the block's MMAs
            for (int i = 0; ok && i < mine; ++i) {
                const int j = streams ? 2 * i + s : i, st = kv.i, buf = SB == 2 ? i & 1 : 0;
                const int p0 = (seg.c_first + j) * kTok;
                const uint32_t sc = ring + st * pl.stage_bytes + (pl.k_atoms + pl.v_atoms) * kAtom;
                ok = wait3(Bars::s_full + 2 * s + buf, phases >> buf, Bars::k_ready + st, kv.phase, Bars::v_ready + st, kv.phase);
                if (!ok) break;
                phases ^= 1u << buf;
                const uint32_t t_b = t_s + buf * s_cols(KNG, VNG);
                kv.step(pl.stages);
                if (streams) kv.step(pl.stages);
                tc::tc_fence_after();
                const bool tail = p0 + kTok > sure;
                uint32_t seen[2] = {0xffffffffu, 0xffffffffu};      // of the block, by the row
                if (tail) {
                    const uint8_t* mask = a.mask ? a.mask + b * a.mask_stride + (int64_t)t_row * a.T : nullptr;
                    // shown without a look at the mask (a length may be near 2^31)
                    const int upto = (mask ? sure : (int)min((int64_t)end, (int64_t)len + t_row + 1)) - p0;
                    seen[0] = upto >= 32 ? 0xffffffffu : (upto <= 0 ? 0u : (1u << upto) - 1u);
                    seen[1] = upto >= 64 ? 0xffffffffu : (upto <= 32 ? 0u : (1u << (upto - 32)) - 1u);
                    if (mask) {
#pragma unroll 8
                        for (int k = max(upto, 0); k < min(kTok, end - p0); ++k) {
                            const uint32_t shown = mask[p0 + k - len] != 0;
                            if (k < 32) seen[0] |= shown << k;
                            else seen[1] |= shown << (k - 32);
                        }
                    }
                }
                const float2 span0 = sm_span[2 * st], span1 = VNG == 2 ? sm_span[2 * st + 1] : span0;
                float2 x[kTok / 2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t v[2][16];
                    tc::tmem_ld16x2(t_b + 32 * h, t_b + 32 * h + 16, v[0], v[1]);
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        const float4 kk = lds128f(sc + 128 * h + 8 * k);
                        const uint32_t* y = &v[k >> 3][2 * k & 15];
                        x[16 * h + k] = mul2(make_float2(__uint_as_float(y[0]), __uint_as_float(y[1])), make_float2(kk.x, kk.y));
                        x[16 * h + k + 1] = mul2(make_float2(__uint_as_float(y[2]), __uint_as_float(y[3])), make_float2(kk.z, kk.w));
                    }
                    if (KNG == 2) {
                        tc::tmem_ld16x2(t_b + kTok + 32 * h, t_b + kTok + 32 * h + 16, v[0], v[1]);
#pragma unroll
                        for (int k = 0; k < 16; k += 2) {
                            const float4 kk = lds128f(sc + 256 + 128 * h + 8 * k);
                            const uint32_t* y = &v[k >> 3][2 * k & 15];
                            x[16 * h + k] = fma2(make_float2(__uint_as_float(y[0]), __uint_as_float(y[1])), make_float2(kk.x, kk.y), x[16 * h + k]);
                            x[16 * h + k + 1] = fma2(make_float2(__uint_as_float(y[2]), __uint_as_float(y[3])), make_float2(kk.z, kk.w), x[16 * h + k + 1]);
                        }
                    }
                    if (tail) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            if (!(seen[h] >> (2 * k) & 1u)) x[16 * h + k].x = -INFINITY;
                            if (!(seen[h] >> (2 * k + 1) & 1u)) x[16 * h + k].y = -INFINITY;
                        }
                    }
                }
                float tops[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) tops[k] = fmaxf(x[k].x, x[k].y);
#pragma unroll
                for (int k = 8; k < kTok / 2; ++k) tops[k & 7] = fmaxf(fmaxf(tops[k & 7], x[k].x), x[k].y);
                const float best = fmaxf(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), fmaxf(fmaxf(tops[4], tops[5]), fmaxf(tops[6], tops[7])));
                const float to_exp = exponent_factor(fac * sm_up[st], best);
                const float ahead = fmaf(best, to_exp, -m);
                if (__any_sync(0xffffffffu, ahead > kLazy || ahead + span0.x - power0 > kRoom ||
                                                (VNG == 2 && ahead + span1.x - power1 > kRoom))) {
                    const float by = raise(m, best * to_exp, ahead > kLazy), lead = fmaf(best, to_exp, -m);
                    const float rest = rest_of(by), steps = whole_steps(by);
                    power0 -= steps;
                    if (VNG == 2) power1 -= steps;
                    float down0 = rest * floor_power(power0), down1 = rest * floor_power(power1);       // of what is summed so far
                    l *= ex2(-by);
                    bool over0 = lead + span0.x - power0 > kRoom, over1 = VNG == 2 && lead + span1.x - power1 > kRoom;
                    if (__any_sync(0xffffffffu, over0 || over1)) {
                        // Weights times scales might leave fp16: the power becomes that of the largest product that the row
                        // sees, or of its largest weight and the smallest scale where scales are within 2^14 of each other.
                        float most0 = lead + span0.y, most1 = lead + span1.y;
                        if (fmaxf(span0.x - span0.y, span1.x - span1.y) > kRoom - 1.0f) {
                            // (through TMEM, where scores can be indexed by a loop: unrolled over registers, these rare lines
                            // cost the common ones 2 to 5 %)
                            float z0 = 0.0f, z1 = 0.0f;
#pragma unroll
                            for (int c = 0; c < kTok; c += 16) {
                                uint32_t v[16];
#pragma unroll
                                for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(k & 1 ? x[(c + k) / 2].y : x[(c + k) / 2].x);
                                tmem_st16v(t_b + c, v);
                            }
#pragma unroll 1
                            for (int c = 0; c < kTok; c += 8) {
                                uint32_t v[8];
                                tc::tmem_ld8(t_b + c, v);
#pragma unroll
                                for (int k = 0; k < 8; ++k) {
                                    const float p = ex2(fmaf(__uint_as_float(v[k]), to_exp, -m));
                                    z0 = fmaxf(z0, p * lds32f(sc + 512 + 4 * (c + k)));
                                    if (VNG == 2) z1 = fmaxf(z1, p * lds32f(sc + 768 + 4 * (c + k)));
                                }
                            }
                            most0 = lg2(z0);
                            most1 = lg2(z1);
                            over0 = most0 - power0 > kRoom;
                            over1 = VNG == 2 && most1 - power1 > kRoom;
                        }
                        down0 *= raise_power(power0, most0, over0);
                        down1 *= raise_power(power1, most1, over1);
                    }
                    if (i != 0 && __any_sync(0xffffffffu, down0 != 1.0f || down1 != 1.0f)) {
                        // The MMAs that wrote O have to be complete: with one buffer they came before those that wrote
                        // these scores.
                        if (SB == 2) {
                            ok = wait(Bars::pv_done + s, done ^ 1u);
                            if (!ok) break;
                            tc::tc_fence_after();
                        }
#pragma unroll 1
                        for (int c = 0; c < pl.o_cols; c += 16) {
                            uint32_t v[16];
                            tc::tmem_ld16(t_s + o_off + c, v);
                            const float f = c < va0 ? down0 : down1;
#pragma unroll
                            for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * f);
                            tmem_st16v(t_s + o_off + c, v);
                        }
                    }
                }
                // weights, over the scores that are done with: the first value group's from column 0, the second's from
                // the second key group's place
                const float unit0 = unit_of(power0), unit1 = unit_of(power1);
                float2 sums[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t w[16];
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        const float4 vv = lds128f(sc + 512 + 128 * h + 8 * k);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float2& y = x[16 * h + k + j];
                            y = fma2(y, make_float2(to_exp, to_exp), make_float2(-m, -m));
                            y = make_float2(ex2(y.x), ex2(y.y));
                            sums[j] = fma2(y, make_float2(1.0f, 1.0f), sums[j]);
                            const float2 z = mul2(mul2(y, make_float2(unit0, unit0)), j ? make_float2(vv.z, vv.w) : make_float2(vv.x, vv.y));
                            w[k + j] = pack2(z.x, z.y);
                        }
                    }
                    tmem_st16v(t_b + 16 * h, w);
                    if (VNG == 2) {
#pragma unroll
                        for (int k = 0; k < 16; k += 2) {
                            const float4 vv = lds128f(sc + 768 + 128 * h + 8 * k);
                            const float2 y0 = mul2(mul2(x[16 * h + k], make_float2(unit1, unit1)), make_float2(vv.x, vv.y));
                            const float2 y1 = mul2(mul2(x[16 * h + k + 1], make_float2(unit1, unit1)), make_float2(vv.z, vv.w));
                            w[k] = pack2(y0.x, y0.y);
                            w[k + 1] = pack2(y1.x, y1.y);
                        }
                        tmem_st16v(t_b + p1_off + 16 * h, w);
                    }
                }
                l += sums[0].x + sums[0].y + sums[1].x + sums[1].y;
                tc::tc_fence_before();
                __syncwarp();
                // (by buffer: with two, a warp may be a block ahead of the others of its group)
                if (lane == 0) tc::mbar_arrive(bar(Bars::p_full + 2 * s + buf));
                done ^= 1u;
            }
            // ---- results: both groups' MMAs are complete, so queries' and operands' memory is free ----
            for (int g = 0; g < groups; ++g) ok = ok && wait(Bars::o_full + g, o_phase >> g);
            tc::tc_fence_after();
            const bool works = s < (streams ? 1 : groups);          // this group has a tile's results
            const bool whole = seg.n_part == 1;
            // Results are averages from here on, which are representable where sums of values near the end of the type's
            // range are not.
            float inv = inverse(l), other = 0.0f;
            const float unit_power0 = power_of(power0), unit_power1 = power_of(power1);
            float* second = reinterpret_cast<float*>(smem);       // [o_cols][128]: the second stream's outputs
            if (streams && s == 1) {
                sm_m[r_tile] = m;
                sm_l[r_tile] = l;
#pragma unroll 1
                for (int c = 0; ok && mine > 0 && c < pl.o_cols; c += 16) {
                    uint32_t v[16];
                    tc::tmem_ld16(t_s + o_off + c, v);
                    const float f = c < va0 ? unit_power0 : unit_power1;
#pragma unroll
                    for (int k = 0; k < 16; ++k) second[(c + k) * 128 + r_tile] = (__uint_as_float(v[k]) * inv) * (sm_back[c + k] * f);
                }
            }
            bar_group(1, 256);
            if (streams && s == 0 && groups == 2) {
                const float m1 = sm_m[r_tile], mm = fmaxf(m, m1), keep = ex2(m - mm);
                other = ex2(m1 - mm) * sm_l[r_tile];
                l = l * keep + other;
                inv = inverse(l) * keep;
                other *= inverse(l);
                m = mm;
            }
            const int unit_row = (streams ? 0 : 128 * s) + r_tile;
            const int64_t part_floats = (int64_t)unit_rows * (pl.o_cols + 2);
            float* parts = reinterpret_cast<float*>(static_cast<uint8_t*>(a.scratch) + SONIQ_KV_SCRATCH_ZERO + kJoinBytes);
            uint8_t* staged = smem + (streams ? pl.o_cols * 512 : 128 * s * pl.out_stride);
            auto stage_out = [&](int c, float v) {
                const int ch = sm_chan[c];
                if (ch >= 0) *reinterpret_cast<uint16_t*>(staged + r_tile * pl.out_stride + 2 * ch) = bf16 ? kv_round<true>(v) : kv_round<false>(v);
            };
            if (works && ok) {
#pragma unroll 1
                for (int c = 0; c < pl.o_cols; c += 16) {
                    uint32_t v[16];
                    tc::tmem_ld16(t_s + o_off + c, v);
                    const float f = c < va0 ? unit_power0 : unit_power1;
                    float x[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        x[k] = (__uint_as_float(v[k]) * inv) * (sm_back[c + k] * f);
                        if (streams && groups == 2) x[k] = fmaf(second[(c + k) * 128 + r_tile], other, x[k]);
                    }
                    if (whole) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) stage_out(c + k, x[k]);
                    } else {
                        float4* to = reinterpret_cast<float4*>(parts + seg.slot * part_floats) + (int64_t)(c / 4) * unit_rows + unit_row;
#pragma unroll
                        for (int k = 0; k < 4; ++k) to[k * unit_rows] = make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                    }
                }
                if (!whole) {
                    float* st = parts + seg.slot * part_floats + (int64_t)unit_rows * pl.o_cols;
                    st[unit_row] = m;
                    st[unit_rows + unit_row] = l;
                }
            }
            // (thread 0 cleared the place; it and this one are apart by a barrier of all threads)
            if (!whole && seg.c_first == 0 && st_id == 0)
                *join = JoinItem{seg.entry, seg.item, tc::abort_raised(abort_flag) ? 0 : seg.n_part, seg.cta0, seg.cta0_slot};
            __syncwarp();
            if (whole && works && ok) {
                // a warp's 32 rows, each in one run
                const int qh = geo.heads * a.group;
                const bool pairs = vs.D % 2 == 0 && (reinterpret_cast<uintptr_t>(a.out) & 3u) == 0;
                for (int i = 0; i < 32; ++i) {
                    const int r = row0 + (streams ? 0 : 128 * s) + quad * 32 + i;
                    if (r >= pl.rows) break;
                    const uint8_t* from = staged + (quad * 32 + i) * pl.out_stride;
                    uint16_t* to = a.out + (((int64_t)b * a.T + r / a.group) * qh + head * a.group + r % a.group) * vs.D;
                    if (pairs) {
                        for (int c = lane; c < vs.D / 2; c += 32) reinterpret_cast<uint32_t*>(to)[c] = reinterpret_cast<const uint32_t*>(from)[c];
                    } else {
                        for (int c = lane; c < vs.D; c += 32) to[c] = reinterpret_cast<const uint16_t*>(from)[c];
                    }
                }
            }
        }
        kv0.skip(nblk, pl.stages);
        raw0.skip(nblk, pl.raw_stages);
        // each group's number of blocks, and of uses of its score buffers, modulo 2
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t n = s < groups ? (streams ? (nblk - s + 1) / 2 : nblk) : 0;
            p_phase ^= (n & 1u) << s;
            if (SB == 2) s_phase ^= (((n + 1) / 2 & 1u) | (n / 2 & 1u) << 1) << (2 * s);
            else s_phase ^= (n & 1u) << (2 * s);
        }
        o_phase ^= groups == 2 ? 3u : 1u;
        q_phase ^= 1u;
        tc::tc_fence_before();
        __syncthreads();
        tc::tc_fence_after();
        if (tc::abort_raised(abort_flag)) {
            // a copy did not come: let those on their way land, and the MMAs end, within the same bound
            const long long t0 = tc::globaltimer();
            if (warp == 1) {
                flights.land([&](int i, uint32_t parity) { return tc::mbar_try_wait(bar(Bars::raw_full + i), parity); },
                             [&]() { return tc::globaltimer() - t0 < kWaitNs; });
            } else if (warp == 0 || warp == 3) {
                if (tc::elect_one()) tc::mma_commit(bar(Bars::drain));
                while (!tc::mbar_try_wait(bar(Bars::drain), 0) && tc::globaltimer() - t0 < kWaitNs) {
                }
            }
            break;
        }
        if (*sm_more == 0) break;
        seg = *sm_seg;
        __syncthreads();      // read before it is overwritten
    }
    };
    if (warp >= 12) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 152;");
        work(std::integral_constant<int, 0>{});
    } else if (warp >= 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        work(std::integral_constant<int, 1>{});
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        work(std::integral_constant<int, 2>{});
    }
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// Joins the parts of split items, in order: 32 rows of one to a CTA.  (Joined by
// the last CTA of the item to finish, inside the kernel above, five parts of 256
// rows took 33 us.)
constexpr int kJoinThreads = 256;
__global__ void __launch_bounds__(kJoinThreads) kv_join_kernel(const KvGeom geo, const KvAttendArgs a, const TilePlan pl) {
    extern __shared__ __align__(16) uint8_t staged[];      // 32 output rows
    __shared__ int16_t chan[192];
    tc::pdl_wait();
    const uint8_t* scratch = static_cast<const uint8_t*>(a.scratch) + SONIQ_KV_SCRATCH_ZERO;
    const JoinItem it = reinterpret_cast<const JoinItem*>(scratch)[blockIdx.x];
    if (it.n_part == 0) return;
    const KvSide& vs = geo.s[1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int unit_rows = 128 * pl.tiles, unit_row = 32 * blockIdx.y + lane;
    const int b = it.entry / pl.row_units, row0 = it.entry % pl.row_units * unit_rows + 32 * blockIdx.y, head = it.item;
    if (row0 >= pl.rows) return;
    const bool bf16 = geo.bf16 != 0;
    const int va0 = 32 * vs.nb[0];
    for (int c = tid; c < pl.o_cols; c += kJoinThreads) {
        const int grp = c < va0 ? 0 : 1, code = column_code(vs.bits[grp], grp ? c - va0 : c);
        chan[c] = code < vs.count[grp] ? (int16_t)vs.perm[head * vs.D + (grp ? vs.count[0] : 0) + code] : (int16_t)-1;
    }
    const int64_t part_floats = (int64_t)unit_rows * (pl.o_cols + 2);
    auto part = [&](int i) {
        return reinterpret_cast<const float*>(scratch + kJoinBytes) + (int64_t)(2 * (it.cta0 + i) + (i == 0 ? it.cta0_slot : 0)) * part_floats;
    };
    auto m_of = [&](int i) { return part(i)[(int64_t)unit_rows * pl.o_cols + unit_row]; };
    float mm = kUnset, ll = 0.0f;
    // a part's sum in units of the item's maximum
    auto sum_of = [&](int i) { return part(i)[(int64_t)unit_rows * (pl.o_cols + 1) + unit_row] * ex2(m_of(i) - mm); };
#pragma unroll 4
    for (int i = 0; i < it.n_part; ++i) mm = fmaxf(mm, m_of(i));
#pragma unroll 4
    for (int i = 0; i < it.n_part; ++i) ll += sum_of(i);
    const float inv = inverse(ll);
    __syncthreads();
    for (int c = 4 * warp; c < pl.o_cols; c += 4 * (kJoinThreads / 32)) {
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (int i = 0; i < it.n_part; ++i) {
            const float4 q = *(reinterpret_cast<const float4*>(part(i)) + (int64_t)(c / 4) * unit_rows + unit_row);
            const float f = sum_of(i) * inv;
            x.x = fmaf(f, q.x, x.x);
            x.y = fmaf(f, q.y, x.y);
            x.z = fmaf(f, q.z, x.z);
            x.w = fmaf(f, q.w, x.w);
        }
        const float y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int ch = chan[c + k];
            if (ch >= 0) *reinterpret_cast<uint16_t*>(staged + lane * pl.out_stride + 2 * ch) = bf16 ? kv_round<true>(y[k]) : kv_round<false>(y[k]);
        }
    }
    __syncthreads();
    const int qh = geo.heads * a.group;
    for (int i = warp; i < 32 && row0 + i < pl.rows; i += kJoinThreads / 32) {
        const int r = row0 + i;
        uint16_t* to = a.out + (((int64_t)b * a.T + r / a.group) * qh + head * a.group + r % a.group) * vs.D;
        for (int c = lane; c < vs.D; c += 32) to[c] = *reinterpret_cast<const uint16_t*>(staged + i * pl.out_stride + 2 * c);
    }
}

struct TileLaunch {
    bool fits;
    TilePlan pl;
};

TileLaunch plan_tile(const KvGeom& geo, int64_t T, int64_t group) {
    TileLaunch t{};
    TilePlan& p = t.pl;
    const KvSide &ks = geo.s[0], &vs = geo.s[1];
    const int64_t rows = T * group;
    p.rows = (int)rows;
    p.tiles = rows > 128 ? 2 : 1;
    p.row_units = (int)((rows + 128 * p.tiles - 1) / (128 * p.tiles));
    p.k_atoms = (ks.nb[0] + ks.nb[1] + 1) / 2;
    p.v_atom1 = (vs.nb[0] + 1) / 2;
    p.v_atoms = p.v_atom1 + (vs.nb[1] + 1) / 2;
    p.o_cols = 32 * (vs.nb[0] + vs.nb[1]);
    if (s_cols(ks.ng, vs.ng) + p.o_cols > kSlotCols) return t;
    p.box_rows = geo.page < kTok ? geo.page : kTok;
    const int copies = kTok / p.box_rows;
    for (int i = 0; i < 2; ++i) p.scale_step[i] = (p.box_rows * geo.s[i].ng * 2 + 127) / 128 * 128;
    p.raw_v = kTok * ks.row_bytes;
    p.raw_s = p.raw_v + kTok * vs.row_bytes;
    p.raw_bytes = (p.raw_s + copies * (p.scale_step[0] + p.scale_step[1]) + 1023) / 1024 * 1024;     // swizzled tiles start on 1024
    p.stage_bytes = (p.k_atoms + p.v_atoms) * kAtom + 1024;
    p.ring_off = p.tiles * p.k_atoms * kQAtom;
    p.out_stride = (vs.D + 1) / 2 * 4 + 4;
    if (p.out_stride / 4 % 2 == 0) p.out_stride += 4;
    constexpr int misc = 5120, most = 227 * 1024;
    // two tiles share a block and look one ahead, two streams two
    static const int choices[][2] = {{4, 4}, {4, 3}, {4, 2}, {3, 4}, {3, 3}, {3, 2}, {2, 3}, {2, 2}};
    for (const auto& c : choices) {
        if (p.tiles == 2 && c[0] > 3) continue;
        p.stages = c[0];
        p.raw_stages = c[1];
        p.raw_off = p.ring_off + p.stages * p.stage_bytes;
        p.misc_off = p.raw_off + p.raw_stages * p.raw_bytes;
        p.smem = p.misc_off + misc;
        const int results = p.tiles == 2 ? 256 * p.out_stride : p.o_cols * 512 + 128 * p.out_stride;
        if (p.smem <= most && results <= p.raw_off) {
            t.fits = true;
            // (two streams with two buffers each run up to three blocks ahead)
            p.buffers = ks.ng == 1 && vs.ng == 1 && 2 * kTok + p.o_cols <= kSlotCols && p.stages >= (p.tiles == 2 ? 2 : 3) ? 2 : 1;
            break;
        }
    }
    p.min_chunks = 4;
    return t;
}

}  // namespace

bool kv_tile_supported(const KvGeom& geo, int64_t T, int64_t group) { return plan_tile(geo, T, group).fits; }

int64_t kv_tile_scratch(const KvGeom& geo, int64_t T, int64_t group) {
    const TilePlan p = plan_tile(geo, T, group).pl;
    return SONIQ_KV_SCRATCH_ZERO + kJoinBytes + (int64_t)2 * num_sms() * 128 * p.tiles * (p.o_cols + 2) * 4;
}

cudaError_t launch_kv_tile(const KvGeom& geo, const KvAttendArgs& a, cudaStream_t st) {
    const TileLaunch t = plan_tile(geo, a.T, a.group);
    if (!t.fits) return cudaErrorNotSupported;
    const TilePlan& p = t.pl;
    const int64_t cap = (int64_t)a.max_pages << geo.page_shift;
    const int64_t items = (int64_t)a.B * geo.heads * p.row_units, most = items * (cap / kTok + 1);
    if (most + items * kLead >= 2147483648ll) return cudaErrorNotSupported;      // chunks are numbered in 32 bits
    const int64_t by_size = (most + p.min_chunks - 1) / p.min_chunks, want = by_size > items ? by_size : items;
    const int grid = (int)(want < num_sms() ? want : num_sms());
    KvMaps maps;
    for (int side = 0; side < 2; ++side) {
        // rows whose stride would put eight tokens' pieces on one bank group are swizzled
        const int row = geo.s[side].row_bytes;
        const CUtensorMapSwizzle swizzle = row == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : (row == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE);
        if (!encode_side(geo, geo.s[side], row, p.box_rows, swizzle, &maps.codes[side], &maps.scales[side]))
            return cudaErrorUnknown;
    }
    auto* kernel = geo.s[0].ng == 1 ? (geo.s[1].ng == 1 ? (p.buffers == 2 ? kv_tile_kernel<1, 1, 2> : kv_tile_kernel<1, 1, 1>) : kv_tile_kernel<1, 2, 1>)
                                    : (geo.s[1].ng == 1 ? kv_tile_kernel<2, 1, 1> : kv_tile_kernel<2, 2, 1>);
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, p.smem);
    if (e == cudaSuccess) e = prefer_max_shared(reinterpret_cast<const void*>(kernel));
    if (e != cudaSuccess) return e;
    kernel<<<grid, kThreads, p.smem, st>>>(geo, a, p, maps);
    note_launch();
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    e = launch_pdl(kv_join_kernel, dim3((unsigned)grid, 4u * p.tiles), dim3(kJoinThreads), (size_t)(32 * p.out_stride), st, geo, a, p);
    if (e == cudaSuccess) note_launch();
    return e;
}

}  // namespace soniq
