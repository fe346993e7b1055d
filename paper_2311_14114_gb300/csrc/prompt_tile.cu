// Attention of packed prompts on tcgen05:
//
//   S = Q K^T, P = softmax(scale S), O = P V, accumulators in TMEM.
//
// A tile is 128 rows: the query heads of one key head (128 at most) at as many
// neighbouring tokens as fit, so a key block serves all of them.  A CTA works at
// one unit at a time, TILES neighbouring tiles of one prompt and key head, over
// blocks of 128 tokens.  Its warps:
//   warp 0 (and 2)   issue the MMAs, each for one tile;
//   warp 1           copies queries, keys and values by TMA;
//   warp 3           finds the next unit, and looks at the clock for all waits;
//   warps 4-11 and 12-19  softmax of a tile, two threads to a row.
// Weights go over the scores that they come from.  While one tile's softmax runs,
// the tensor cores work for the other; a lone tile has two buffers of scores.
// Keys and values come in pieces of 128 tokens by 128 channels, in the order in
// which the MMAs take them.  Units are handed out by a counter, the longest of a
// prompt first, and one unit's scores begin while the one before leaves its outputs.
//
// Bound by the chain of a tile: scores there - softmax (about 1300 cycles: scores
// 90, maxima 240, exponentials 700, the rest votes, stores and skew) - MMAs (1024
// and 200 to be seen).  Two tiles side by side take 2600 cycles for 128 keys of 256
// rows, of which the tensor cores work 2048; a unit costs 8000 more, where both
// leave outputs and begin anew, in code that is not in the instruction cache.
// Lone tiles (256 channels) have 2048 cycles of MMAs to 1300, and hide the softmax.
// Measured (GB300, bf16, causal, 32 query heads on 8): 16384 tokens of 128 channels
// 1.42 ms (1550 TFLOP/s), 8192 of 64, 128, 256: 275, 320, 609 us (1000, 1720, 1800),
// 16 prompts of 410 to 4096 tokens 675 us (1240), 200 of 0 to 200, 12 heads of 64 in
// fp16, 58 us.
// Taken and not, at 16384 tokens: blocks of 64 with two buffers of scores 1864 us
// (their MMAs, N = 64, read 192 bytes of operands a cycle for 128); a thread to a
// row, 1960; one warp for both tiles' MMAs, 2200, as its instructions between them
// add up; weights in one part, 1530.
//
// Numerics.  Scores are fp32.  A row's weights are 2^(score - m), held at most
// 2^15: m is raised, and O with it, only when a weight would pass that, to where
// the largest is 2^8.  (So fp16 weights have their full 11 bits down to 2^-22 of
// the row's largest.)  Weights are rounded to the type for the product.
//
// What no rounding of that kind holds ends in an output that is not finite: NaN
// and infinities in the values of later tokens, which a row does not see (0 times
// them is not 0), sums that pass fp32, scores so large that their products with
// the exponent's factor are off.  Rows with such an output are done again, from
// the definition, by prompt_row.  So the blocks need no look at what is hidden;
// only what stands behind a prompt, where a buffer's padding may hold anything, is
// cleared in its last block.
#include <atomic>

#include "kv_flights.h"
#include "prompt_rows.cuh"
#include "soniq_device.cuh"
#include "tile_ops.cuh"

namespace soniq {

namespace {

constexpr int kTok = 128;                // tokens of a block
constexpr int kAtom = kTok * 128;        // bytes of a 64-channel column group of a key or value block, or of a query tile
constexpr int kMaxSlots = 12;
constexpr int shared_of(int ctas) { return (ctas == 1 ? 227 : 113) * 1024; }      // (each CTA of an SM's 228 KB has 1 KB that it does not see)
constexpr float kMost = 15.0f, kBegin = 8.0f;      // log2 of the largest weight, and of a row's largest when m is raised

struct PromptPlan {
    int row_heads;           // query heads of a tile
    int tile_tokens;
    int head_parts;          // tiles that share a key head's query heads
    int k_atoms, v_atoms;
    int o_cols;              // Dv rounded up to whole MMA columns
    int slots, slot_bytes;   // of the ring of pieces
    int ring_off, misc_off, smem;
    int wide_rows;           // output rows are whole 32-byte pieces
};

struct PromptMaps {
    CUtensorMap q, k, v;
};

struct Unit {
    int start, len;          // the prompt
    int token;               // first token of the unit, within it; negative: there is no unit
    int kv_head, part;
    int blocks0, blocks1;    // of each tile; 0: the tile is empty
    __device__ __forceinline__ int blocks_of(int s) const { return s ? blocks1 : blocks0; }
    __device__ __forceinline__ int blocks() const { return max(blocks0, blocks1); }
};

struct Bars {                // offsets in 8-byte barriers; the first ones are those of copies (Flights)
    static constexpr int full = 0, q_full = kMaxSlots, free = q_full + 1,
                         q_free = free + kMaxSlots, s_full = q_free + 1, p_full = s_full + 4, pv_done = p_full + 4,
                         o_full = pv_done + 2, o_free = o_full + 2, unit_full = o_free + 2, unit_free = unit_full + 2,
                         turn = unit_free + 2, drain = turn + 2, count = drain + 1;      // s_full: [tile][buffer]; p_full: [tile or buffer][half]
};
constexpr int kMisc = 3 * 1024;
static_assert(8 * Bars::count <= 512, "barriers");

// 64 consecutive TMEM columns of this thread's lane (load + wait in one statement).
__device__ __forceinline__ void tmem_ld64(uint32_t at, uint32_t (&r)[64]) {
#define SONIQ_R4(i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3])
#define SONIQ_R16(i) SONIQ_R4(i), SONIQ_R4(i + 4), SONIQ_R4(i + 8), SONIQ_R4(i + 12)
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%64];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,"
        "%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%65];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : SONIQ_R16(0), SONIQ_R16(16), SONIQ_R16(32), SONIQ_R16(48)
        : "r"(at), "r"(at + 32)
        : "memory");
}
#undef SONIQ_R16
#undef SONIQ_R4
// 16 columns without the wait.
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// MMAs and commits of a whole warp, issued by one of its lanes, which the instruction
// itself elects: control flow stays that of the warp, and what it works out in uniform
// registers.  (Under a branch of one lane each operand is moved there first, and
// waits for the MMA before to have read it: 90 to 130 cycles an MMA.)
__device__ __forceinline__ void warp_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc));
}
__device__ __forceinline__ void warp_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(acc));
}
__device__ __forceinline__ void warp_commit(uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar)
        : "memory");
}
// Arrival of a whole warp as one.
__device__ __forceinline__ void warp_arrive(uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred e;\n\t.reg .b64 st;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e mbarrier.arrive.shared::cta.b64 st, [%0];\n\t}" ::"r"(bar)
        : "memory");
}
// Rounded to the type, values beyond its range to its largest.
template <bool BF16>
__device__ __forceinline__ uint32_t pack_finite(float lo, float hi) {
    uint32_t r;
    if constexpr (BF16) asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// A value that is the same in all lanes, so that the compiler knows.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// CTAS: resident on an SM.  Two of one tile each take turns at the SM's units where prompts are short.
template <bool BF16, int TILES, int CTAS>
__global__ void __launch_bounds__(128 + 256 * TILES, CTAS)
    prompt_tile_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ PromptPlan pl, const __grid_constant__ PromptMaps maps, unsigned* counters, const int drop, const long long wait_ns) {
    extern __shared__ __align__(1024) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
    const uint32_t smem0 = tc::smem_u32(smem), ring = smem0 + pl.ring_off, bars = smem0 + pl.misc_off;
    uint8_t* misc = smem + pl.misc_off;
    Unit* units = reinterpret_cast<Unit*>(misc + 512);                // [2]
    uint32_t* words = reinterpret_cast<uint32_t*>(misc + 640);
    const uint32_t abort_flag = tc::smem_u32(words), progress = abort_flag + 8;
    uint32_t* tmem_at = words + 1;
    float* halves = reinterpret_cast<float*>(misc + 1024);            // [tile][half][128]: what the two threads of a row tell each other
    auto bar = [&](int i) { return bars + 8u * i; };
    const int unit_tokens = TILES * pl.tile_tokens;
    constexpr int SB = TILES * CTAS == 1 ? 2 : 1;       // buffers of scores
    constexpr int tmem_cols = 512 / CTAS, slot_cols = tmem_cols / TILES, o_col = SB * kTok;      // TMEM columns of a tile; where its outputs begin

    if (tid == 0) {
        auto init = [&](int first, int n, int arrivals) {
            for (int i = 0; i < n; ++i) tc::mbar_init(bar(first + i), arrivals);
        };
        init(Bars::full, kMaxSlots + 1, 1);              // and q_full
        init(Bars::free, kMaxSlots + 1, TILES);          // and q_free
        init(Bars::s_full, 4, 1);
        init(Bars::p_full, 4, 8);
        init(Bars::pv_done, 4, 1);                       // and o_full
        init(Bars::o_free, 2, 8);
        init(Bars::unit_full, 2, 1);
        init(Bars::unit_free, 2, 1 + 9 * TILES);
        init(Bars::turn, 2, 1);
        init(Bars::drain, 1, TILES);
        words[0] = words[2] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(tmem_at)), "r"(tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = uniform(*tmem_at);
    // Waits are bounded: the warp that finds units is there until all others have seen the last of them, and raises the
    // abort flag, which every wait looks at, once none of them has got on for `wait_ns`.  (Not before: a role may wait for
    // as long as the others take over a unit, which with prompts of 2^28 tokens, or rows done again, is longer than any
    // limit.)  These say that they get on: the warp that copies, with each piece, and those that do rows again, with
    // each 32 keys.  (A clock in every wait is code at 35 places: 200 short prompts took 62 us, and 64 with the look at
    // whether others get on; now 58.)
    auto tick = [progress]() { asm volatile("red.relaxed.cta.shared::cta.add.u32 [%0], 1;" ::"r"(progress) : "memory"); };
    // (one look at a wait that is over costs 20 cycles, the loop 160)
    auto wait = [&](int i, uint32_t parity) {
        return __all_sync(0xffffffffu, tc::mbar_try_wait(bar(i), parity & 1u)) || wait_watched(bar(i), parity & 1u, abort_flag);
    };

    // The next unit, as the warps of other roles read it; they release it (`done`) when they have gone on.
    auto next_unit = [&](uint32_t n, Unit* u) {
        if (!wait(Bars::unit_full + (n & 1), n >> 1)) return false;
        const Unit x = units[n & 1];
        *u = Unit{uniform(x.start), uniform(x.len), uniform(x.token), uniform(x.kv_head), uniform(x.part), uniform(x.blocks0), uniform(x.blocks1)};
        if (lane == 0) tc::mbar_arrive(bar(Bars::unit_free + (n & 1)));
        return u->token >= 0;
    };

    Flights flights;       // of the copying warp
    // Registers move to the softmax warps: 4 x 104 + 64 = 5 x 96 a thread, of two CTAs 2 x 96 + 48 = 3 x 80.  (All four
    // warps of a group give up theirs, or the others wait for them without end.)
    if (warp < 4) {
        if constexpr (TILES == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if constexpr (CTAS == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == 3) {
        // ---- units: numbered prompt by prompt, later tokens first, key heads side by side ----
        const int per_unit = a.k_heads * pl.head_parts;
        int64_t base = 0;              // units of the prompts before b0
        int b0 = 0, taken = 0;         // and the end of them
        unsigned id = blockIdx.x;
        bool ok = true;
        auto watch = [&](int i, uint32_t parity) {
            return wait_watching(bar(i), parity & 1u, abort_flag, a.err, [&]() { return lds32(progress); }, wait_ns);
        };
        uint32_t last = 0;
        for (uint32_t n = 0;; ++n) {
            // the prompt that holds it: 32 at a time, from the last one on
            int found = -1, s = 0, len = 0;
            int64_t before = 0;
            while (b0 < a.B) {
                const int b = b0 + lane;
                int s_b = b < a.B ? a.starts[b] : 0, e_b = b < a.B ? a.starts[b + 1] : 0;
                // the end of the prompts before: a start that fell leaves out what begins in front of it
                int upmost = b < a.B && prompt_good(a, s_b, e_b, 0) ? e_b : 0;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int x = __shfl_up_sync(0xffffffffu, upmost, d);
                    if (lane >= d) upmost = max(upmost, x);
                }
                const int before_me = __shfl_up_sync(0xffffffffu, upmost, 1);
                if (b < a.B && !prompt_good(a, s_b, e_b, lane ? max(before_me, taken) : taken)) {
                    if (blockIdx.x == 0) atomicOr(a.err, kErrKvIndex);
                    s_b = e_b = 0;
                }
                const int64_t mine = (int64_t)((e_b - s_b + unit_tokens - 1) / unit_tokens) * per_unit;
                int64_t upto = mine;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int64_t x = __shfl_up_sync(0xffffffffu, upto, d);
                    if (lane >= d) upto += x;
                }
                const unsigned in = __ballot_sync(0xffffffffu, (int64_t)id < base + upto);
                if (in != 0) {
                    const int at = __ffs(in) - 1;
                    found = b0 + at;
                    s = __shfl_sync(0xffffffffu, s_b, at);
                    len = __shfl_sync(0xffffffffu, e_b - s_b, at);
                    before = base + __shfl_sync(0xffffffffu, upto - mine, at);
                    break;
                }
                base += __shfl_sync(0xffffffffu, upto, 31);
                taken = max(taken, __shfl_sync(0xffffffffu, upmost, 31));
                b0 += 32;
            }
            ok = watch(Bars::unit_free + (n & 1), (n >> 1) ^ 1u);
            Unit u{};
            u.token = -1;
            if (found >= 0) {
                const int r = (int)(id - before), of = (len + unit_tokens - 1) / unit_tokens;
                const int head = r % per_unit;
                u.start = s;
                u.len = len;
                u.token = (of - 1 - r / per_unit) * unit_tokens;
                u.kv_head = head / pl.head_parts;
                u.part = head % pl.head_parts;
                auto blocks = [&](int first) {
                    const int end = a.causal ? min(first + pl.tile_tokens, len) : len;
                    return first < len ? (end + kTok - 1) / kTok : 0;
                };
                u.blocks0 = blocks(u.token);
                if (TILES == 2) u.blocks1 = blocks(u.token + pl.tile_tokens);
            }
            if (ok && lane == 0) {
                units[n & 1] = u;
                tc::mbar_arrive(bar(Bars::unit_full + (n & 1)));
            }
            __syncwarp();
            if (!ok) break;
            if (found < 0) {
                last = n;
                break;
            }
            if (lane == 0) id = gridDim.x + atomicAdd(counters, 1u);
            id = __shfl_sync(0xffffffffu, id, 0);
        }
        // the last CTA to have asked leaves the counters as it found them
        if (ok && lane == 0) {
            __threadfence();
            if (atomicAdd(counters + 1, 1u) == gridDim.x - 1) {
                counters[0] = 0;
                counters[1] = 0;
            }
        }
        // until all others have seen that there are no more
        __syncwarp();
        if (ok) watch(Bars::unit_free + (last & 1), last >> 1);
    } else if (warp == 1) {
        // ---- copies ----
        Ring kv;
        Unit u;
        bool ok = true;
        for (uint32_t n = 0; ok && next_unit(n, &u); ++n) {
            const int blocks = u.blocks();
            const int head = (u.kv_head * a.group + u.part * pl.row_heads);
            ok = wait(Bars::q_free, n ^ 1u);
            if (!ok) break;
            flights.issue(Bars::q_full, n);
            const int box_bytes = pl.row_heads * pl.tile_tokens * 128, tiles = u.blocks_of(TILES - 1) > 0 ? TILES : 1;
            if (tc::elect_one()) tc::mbar_arrive_expect_tx(bar(Bars::q_full), tiles * pl.k_atoms * box_bytes);
            for (int i = 0; i < tiles * pl.k_atoms; ++i) {
                const int tile = i / pl.k_atoms, atom = i % pl.k_atoms;
                if (tc::elect_one())
                    tma_load_3d(smem0 + i * kAtom, &maps.q, 64 * atom, a.q.head ? head : 0, u.start + u.token + tile * pl.tile_tokens, bar(Bars::q_full));
            }
            // a block's pieces of keys or of values
            auto pieces = [&](int j, int atoms, const CUtensorMap* map, int kv_head) {
#pragma unroll 1
                for (int c = 0; ok && c < atoms; c += 2, kv.step(pl.slots)) {
                    ok = wait(Bars::free + kv.i, kv.phase ^ 1u);
                    if (!ok) break;
                    if (drop && blockIdx.x == 0 && n == 0 && j == 0) continue;
                    flights.issue(Bars::full + kv.i, kv.phase);
                    const uint32_t at = ring + kv.i * pl.slot_bytes;
                    if (tc::elect_one()) {
                        tc::mbar_arrive_expect_tx(bar(Bars::full + kv.i), (c + 1 < atoms ? 2 : 1) * kAtom);
                        tma_load_3d(at, map, 64 * c, kv_head, u.start + j * kTok, bar(Bars::full + kv.i));
                        if (c + 1 < atoms) tma_load_3d(at + kAtom, map, 64 * c + 64, kv_head, u.start + j * kTok, bar(Bars::full + kv.i));
                        tick();
                    }
                    __syncwarp();
                }
            };
#pragma unroll 1
            for (int j = -SB; ok && j < blocks; ++j) {
                if (j >= 0) pieces(j, pl.v_atoms, &maps.v, a.v.head ? u.kv_head : 0);
                if (j + SB < blocks) pieces(j + SB, pl.k_atoms, &maps.k, a.k.head ? u.kv_head : 0);
            }
        }
    } else if (warp == 0 || TILES == 2) {
        // ---- MMAs of tile s ----
        const int s = TILES == 2 ? warp >> 1 : 0;
        constexpr uint32_t fmt = (1u << 4) | (BF16 ? (1u << 7) | (1u << 10) : 0u) | ((128u >> 4) << 24);
        auto columns = [](int n) { return (uint32_t)(n >> 3) << 17; };
        const int steps = (a.D + 15) / 16;      // of 16 channels
        const int k_pieces = (pl.k_atoms + 1) / 2, v_pieces = (pl.v_atoms + 1) / 2;
        bool ok = true;
        // steps of 16 keys in the order in which their weights come: the first quarter of each half, then the second
        auto step_of = [](int h) { return (h & 1) + 4 * (h >> 1 & 1) + 2 * (h >> 2); };
        const uint32_t t_s = tmem + s * slot_cols;
        const uint64_t q_tile = tc::sw128_desc(smem0 + s * pl.k_atoms * kAtom);
        // scores of a block, `keys` of it, whose pieces begin at r
        auto scores = [&](uint32_t buf, int keys, Ring r) {
            const uint32_t d = t_s + buf * kTok, id = fmt | columns(keys);
            uint64_t q = q_tile;
#pragma unroll 1
            for (int c = 0; c < k_pieces; ++c, r.step(pl.slots), q += 2 * (kAtom >> 4)) {
                ok = ok && wait(Bars::full + r.i, r.phase);
                if (!ok) break;
                tc::tc_fence_after();
                const uint64_t k = tc::sw128_desc(ring + r.i * pl.slot_bytes);
                const int some = steps - 8 * c;
                if (some >= 8) {
#pragma unroll
                    for (int h = 0; h < 8; ++h)
                        warp_mma_ss(d, q + (h >> 2) * (kAtom >> 4) + 2 * (h & 3), k + (h >> 2) * (kAtom >> 4) + 2 * (h & 3), id, h == 0 ? c : 1);
                } else {
                    if (some >= 4) {
#pragma unroll
                        for (int h = 0; h < 4; ++h) warp_mma_ss(d, q + 2 * h, k + 2 * h, id, h == 0 ? c : 1);
                    }
#pragma unroll 1
                    for (int h = some >= 4 ? 4 : 0; h < some; ++h)
                        warp_mma_ss(d, q + (h >> 2) * (kAtom >> 4) + 2 * (h & 3), k + (h >> 2) * (kAtom >> 4) + 2 * (h & 3), id, c | h);
                }
                warp_commit(bar(Bars::free + r.i));
            }
            warp_commit(bar(Bars::s_full + 2 * s + buf));
        };
        // outputs over block i, `keys` of it, of which `first` are the prompt's, once weights of the parity are there
        auto outputs = [&](int i, uint32_t buf, uint32_t parity, int keys, int first, Ring r) {
            const uint32_t p = t_s + buf * kTok;
#pragma unroll 1
            for (int c = 0; c < v_pieces; ++c, r.step(pl.slots)) {
                ok = ok && wait(Bars::full + r.i, r.phase) && (c > 0 || wait(Bars::p_full + 2 * (SB == 2 ? buf : s), parity));
                if (!ok) break;
                tc::tc_fence_after();
                const uint32_t values = ring + r.i * pl.slot_bytes, d = t_s + o_col + 128 * c;
                if (keys > first) {
                    // Tokens behind the prompt, whose weights are 0, may hold anything (a buffer's padding): 0 times
                    // that is to be 0.  (The other tile's warp writes the same zeros.)
                    const int n16 = 8 * (keys - first), atoms = min(pl.v_atoms - 2 * c, 2);
                    for (int k = lane; k < atoms * n16; k += 32)
                        sts128f(values + (k >= n16 ? kAtom - 16 * n16 : 0) + 128 * first + 16 * k, 0.0f, 0.0f, 0.0f, 0.0f);
                    tc::fence_proxy_async_shared();
                    __syncwarp();
                }
                const uint64_t v = value_desc(values, kAtom);
                const uint32_t id = fmt | (1u << 16) | columns(min(pl.o_cols - 128 * c, 128));
#pragma unroll
                for (int h = 0; h < kTok / 16; ++h) {
                    const int k = step_of(h);
                    if (c == 0 && h == 4) {
                        ok = ok && wait(Bars::p_full + 2 * (SB == 2 ? buf : s) + 1, parity);
                        tc::tc_fence_after();
                    }
                    if (16 * k < keys) warp_mma_ts(d, p + 8 * k, v + k * (2048 >> 4), id, h == 0 ? i : 1);
                }
                warp_commit(bar(Bars::free + r.i));
            }
            if (SB == 2) warp_commit(bar(Bars::pv_done + s));
        };
        auto skip = [&](Ring& r, int n) {
            for (int i = 0; i < n; ++i) r.step(pl.slots);
        };
        // Pieces that only the other tile uses are released when they are there, so that no release runs ahead.
        auto leave = [&](Ring r, int n) {
            for (int i = 0; ok && i < n; ++i, r.step(pl.slots)) {
                ok = wait(Bars::full + r.i, r.phase);
                if (ok) warp_arrive(bar(Bars::free + r.i));
            }
        };
        const bool plain = k_pieces == 1;
        Ring kv;                                 // the next piece
        uint32_t done = 0, tiles = 0, turns = 0; // blocks, tiles and turns so far
        Unit u;
        for (uint32_t n = 0; ok && next_unit(n, &u); ++n) {
            const int blocks = u.blocks(), mine = u.blocks_of(s);
            // keys of the last block, in whole steps of 16
            const int end = a.causal ? min(u.token + (s + 1) * pl.tile_tokens, u.len) : u.len;
            const int last_keys = (end - (mine - 1) * kTok + 15) / 16 * 16;
            ok = wait(Bars::q_full, n);
            if (mine == 0) warp_arrive(bar(Bars::q_free));
#pragma unroll 1
            for (int i = -SB; ok && i < blocks; ++i) {
                if (TILES == 2 && plain && i == 0 && mine > 1) {
                    // Whole blocks of up to 128 channels, with few questions on the way: the warp's instructions come from the
                    // cache that the softmax warps sweep, some 5 cycles each.
                    ok = wait(Bars::o_free + s, tiles ^ 1u);
                    uint32_t at = kv.i, phase = kv.phase;
#pragma unroll 1
                    for (; ok && i + 1 < mine; ++i) {
                        const uint32_t v_at = at, v_phase = phase;
                        if (++at == (uint32_t)pl.slots) at = 0, phase ^= 1u;
                        const uint32_t k_at = at, k_phase = phase;
                        if (++at == (uint32_t)pl.slots) at = 0, phase ^= 1u;
                        ok = wait(Bars::full + v_at, v_phase) && wait(Bars::full + k_at, k_phase) && wait(Bars::turn + s, turns ^ (s ^ 1u)) &&
                             wait(Bars::p_full + 2 * s, done + i);
                        if (!ok) break;
                        tc::tc_fence_after();
                        const uint64_t v = value_desc(ring + v_at * pl.slot_bytes, kAtom), k = tc::sw128_desc(ring + k_at * pl.slot_bytes);
                        const uint32_t id = fmt | (1u << 16) | columns(pl.o_cols), id_s = fmt | columns(i + 2 == mine ? last_keys : kTok);
#pragma unroll
                        for (int h = 0; h < 8; ++h) {
                            if (h == 4) {
                                ok = wait(Bars::p_full + 2 * s + 1, done + i);
                                tc::tc_fence_after();
                            }
                            warp_mma_ts(t_s + o_col, t_s + 8 * step_of(h), v + step_of(h) * (2048 >> 4), id, h == 0 ? i : 1);
                        }
                        warp_commit(bar(Bars::free + v_at));
                        auto step = [&](int h) {
                            warp_mma_ss(t_s, q_tile + (h >> 2) * (kAtom >> 4) + 2 * (h & 3), k + (h >> 2) * (kAtom >> 4) + 2 * (h & 3), id_s, h != 0);
                        };
                        int h = 0;
                        if (steps >= 4) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) step(e);
                            h = 4;
                        }
                        if (steps == 8) {
#pragma unroll
                            for (int e = 4; e < 8; ++e) step(e);
                        } else {
#pragma unroll 1
                            for (; h < steps; ++h) step(h);
                        }
                        warp_commit(bar(Bars::free + k_at));
                        warp_commit(bar(Bars::s_full + 2 * s));
                        if (i + 2 == mine) warp_commit(bar(Bars::q_free));
                        warp_arrive(bar(Bars::turn + (s ^ 1)));
                        ++turns;
                    }
                    kv.i = at;
                    kv.phase = phase;
                    if (!ok) break;
                }
                if (SB == 2 && i == 0 && mine > 2) {
                    // whole blocks, likewise
                    ok = wait(Bars::o_free, tiles ^ 1u);
                    uint32_t at = kv.i, phase = kv.phase;
                    auto go_on = [&] {
                        if (++at == (uint32_t)pl.slots) at = 0, phase ^= 1u;
                    };
#pragma unroll 1
                    for (; ok && i + 2 < mine; ++i) {
                        const uint32_t b = (done + i) & 1u, t_b = t_s + b * kTok, half_round = (done + i) >> 1;
#pragma unroll 1
                        for (int c = 0; c < v_pieces; ++c) {
                            ok = wait(Bars::full + at, phase) && (c > 0 || wait(Bars::p_full + 2 * b, half_round));
                            if (!ok) break;
                            tc::tc_fence_after();
                            const uint64_t v = value_desc(ring + at * pl.slot_bytes, kAtom);
                            const uint32_t id = fmt | (1u << 16) | columns(min(pl.o_cols - 128 * c, 128));
#pragma unroll
                            for (int h = 0; h < 8; ++h) {
                                if (h == 4 && c == 0) {
                                    ok = wait(Bars::p_full + 2 * b + 1, half_round);
                                    tc::tc_fence_after();
                                }
                                warp_mma_ts(t_s + o_col + 128 * c, t_b + 8 * step_of(h), v + step_of(h) * (2048 >> 4), id, h == 0 ? i : 1);
                            }
                            warp_commit(bar(Bars::free + at));
                            go_on();
                        }
                        if (!ok) break;
                        warp_commit(bar(Bars::pv_done));
                        const uint32_t id_s = fmt | columns(i + 3 == mine ? last_keys : kTok);
#pragma unroll 1
                        for (int c = 0; c < k_pieces; ++c) {
                            ok = wait(Bars::full + at, phase);
                            if (!ok) break;
                            tc::tc_fence_after();
                            const uint64_t k = tc::sw128_desc(ring + at * pl.slot_bytes), q = q_tile + c * 2 * (kAtom >> 4);
                            auto step = [&](int h, uint32_t acc) {
                                warp_mma_ss(t_b, q + (h >> 2) * (kAtom >> 4) + 2 * (h & 3), k + (h >> 2) * (kAtom >> 4) + 2 * (h & 3), id_s, acc);
                            };
                            if (steps - 8 * c >= 8) {
#pragma unroll
                                for (int h = 0; h < 8; ++h) step(h, h == 0 ? c : 1);
                            } else {
#pragma unroll 1
                                for (int h = 0; h < steps - 8 * c; ++h) step(h, c | h);
                            }
                            warp_commit(bar(Bars::free + at));
                            go_on();
                        }
                        if (!ok) break;
                        warp_commit(bar(Bars::s_full + b));
                        if (i + 3 == mine) warp_commit(bar(Bars::q_free));
                    }
                    kv.i = at;
                    kv.phase = phase;
                    if (!ok) break;
                }
                const uint32_t buf = SB == 2 ? (done + (i & 1)) & 1u : 0u, parity = SB == 2 ? (done + i) >> 1 : done + i;
                const bool out = i >= 0 && i < mine, in = i + SB < mine;
                Ring keys_at = kv;
                if (i >= 0) skip(keys_at, v_pieces);
                if (out && i == 0) ok = wait(Bars::o_free + s, tiles ^ 1u);
                // The two tiles take turns: the softmax of one has the time of the other's MMAs.  (Without, the two ran in
                // step, both softmaxes and then both tiles' MMAs: 5200 cycles a block instead of 2700.)
                if (TILES == 2 && i >= 0 && ok) ok = wait(Bars::turn + s, turns ^ (s ^ 1u));
                if (!ok) break;
                if (out) {
                    outputs(i, buf, parity, i == mine - 1 ? last_keys : kTok, u.len - i * kTok, kv);
                    if (i == mine - 1) warp_commit(bar(Bars::o_full + s));
                }
                if (!ok) break;
                if (in) {
                    scores(buf, i + SB == mine - 1 ? last_keys : kTok, keys_at);
                    if (i + SB == mine - 1) warp_commit(bar(Bars::q_free));
                }
                if (TILES == 2 && i >= 0) {
                    warp_arrive(bar(Bars::turn + (s ^ 1)));
                    ++turns;
                }
                if (i >= 0) {
                    if (!out) leave(kv, v_pieces);
                    kv = keys_at;
                }
                if (i + SB < blocks) {
                    if (!in) leave(kv, k_pieces);
                    skip(kv, k_pieces);
                }
            }
            done += mine;
            tiles += mine > 0;
        }
    }
    } else {
        if constexpr (TILES == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        if constexpr (CTAS == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");
        // ---- softmax of tile s: two threads to a row, each with half of a block's keys ----
        const int s = (warp - 4) >> 3, half = ((warp - 4) >> 2) & 1, quad = warp & 3, row = quad * 32 + lane;
        const uint32_t t_s = tmem + s * slot_cols + ((uint32_t)(quad * 32) << 16);
        const int row_token = row / pl.row_heads, row_head = row - row_token * pl.row_heads;
        const int heads = a.k_heads * a.group;
        float* mine_at = halves + (2 * s + half) * 128 + row;
        const float* other_at = halves + (2 * s + 1 - half) * 128 + row;
        // Whether it is so in any row of the two warps that share these 32.  Waits are bounded, but this is not: both have to
        // come to each.  So a warp whose wait was given up goes on to the next one, where both learn of it and leave; and
        // none stands within a loop over a half's columns, of which the other half may have none.
        auto either = [&](bool x) {
            uint32_t r;
            asm volatile(
                "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                : "=r"(r)
                : "r"((uint32_t)x), "r"(1 + 4 * s + quad)
                : "memory");
            return r != 0;
        };
        // (never 0: a score that is masked, minus infinity, has no weight at any scale)
        const float factor = fmaxf(a.scale * kLog2e, 1.4e-45f);
        // this half's share of the outputs' columns
        const int chunks = pl.o_cols / 16, c_first = half ? (chunks + 1) / 2 * 16 : 0, c_end = half ? pl.o_cols : (chunks + 1) / 2 * 16;
        uint32_t done = 0, tiles = 0;
        Unit u;
        bool ok = true;
        for (uint32_t n = 0;; ++n) {
            ok = next_unit(n, &u);
            if (either(!ok)) break;
            const int mine = u.blocks_of(s);
            if (mine == 0) continue;
            const int token = u.token + s * pl.tile_tokens + row_token, head = u.part * pl.row_heads + row_head;
            const bool live = row_token < pl.tile_tokens && token < u.len && head < a.group;
            // keys that the row sees, and those that all of the warp's do (rows of no token do not matter)
            const int end = live && a.causal ? token + 1 : u.len;
            const int sure = __reduce_min_sync(0xffffffffu, end);
            float m = kUnset, l = 0.0f;
#pragma unroll 1
            for (int i = 0; i < mine; ++i, ++done) {
                const uint32_t buf = SB == 2 ? done & 1u : 0u, t_b = t_s + buf * kTok;
                ok = ok && wait(Bars::s_full + 2 * s + buf, SB == 2 ? done >> 1 : done);
                tc::tc_fence_after();
                uint32_t raw[64];
                tmem_ld64(t_b + 64 * half, raw);
                float2 x[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) x[k] = make_float2(__uint_as_float(raw[2 * k]), __uint_as_float(raw[2 * k + 1]));
                if ((i + 1) * kTok > sure) {
                    // (by sixteen keys, most of which all rows of the warp see)
                    const int upto = end - i * kTok - 64 * half;
#pragma unroll
                    for (int k = 0; k < 32; k += 8) {
                        if (i * kTok + 64 * half + 2 * k + 16 <= sure) continue;
#pragma unroll
                        for (int e = k; e < k + 8; ++e) {
                            if (2 * e >= upto) x[e].x = -INFINITY;
                            if (2 * e + 1 >= upto) x[e].y = -INFINITY;
                        }
                    }
                }
                float tops[8];
#pragma unroll
                for (int k = 0; k < 32; ++k) tops[k & 7] = k < 8 ? fmaxf(x[k].x, x[k].y) : fmaxf(fmaxf(tops[k & 7], x[k].x), x[k].y);
                const float best = fmaxf(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), fmaxf(fmaxf(tops[4], tops[5]), fmaxf(tops[6], tops[7])));
                float2 sums[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
                uint32_t w[16];
                // weights of a quarter of the block's keys
                auto weigh = [&](int h) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float2 y = fma2(x[16 * h + k], make_float2(factor, factor), make_float2(-m, -m));
                        y = make_float2(ex2(y.x), ex2(y.y));
                        sums[k & 1] = fma2(y, make_float2(1.0f, 1.0f), sums[k & 1]);
                        w[k] = BF16 ? pack_bf16(y.x, y.y) : pack2(y.x, y.y);
                    }
                };
                auto leave = [&](int h) {
                    tmem_st16(t_b + 32 * half + 16 * h, w);
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                    tc::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(bar(Bars::p_full + 2 * (SB == 2 ? buf : s) + h));
                };
                // (the first quarter as if m stays, which it mostly does: the two warps are not asked before it)
                if (i != 0) weigh(0);
                // Behind this both have read their scores, and weights may go over them.
                if (i == 0 || either(!ok || fmaf(best, factor, -m) > kMost)) {
                    *mine_at = best;
                    if (either(!ok)) {
                        ok = false;
                        break;
                    }
                    const float both = fmaxf(best, *other_at);
                    const bool over = fmaf(both, factor, -m) > kMost;
                    const float to = over ? both * factor - kBegin : m, by = ex2(m - to);
                    m = to;
                    l *= by;
                    // scores whose products are off by their rounding: the row is done again
                    if (over && !(fabsf(fmaf(both, factor, -m) - kBegin) <= 4.0f)) l = NAN;
                    if (i != 0) {
                        // the MMAs that wrote O have to be complete: with one buffer they came before those of these scores
                        if (SB == 2) {
                            ok = wait(Bars::pv_done + s, done ^ 1u);
                            tc::tc_fence_after();
                        }
#pragma unroll 1
                        for (int c = c_first; c < c_end; c += 16) {
                            uint32_t v[16];
                            tc::tmem_ld16(t_s + o_col + c, v);
#pragma unroll
                            for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * by);
                            tmem_st16v(t_s + o_col + c, v);
                        }
                    }
                    sums[0] = sums[1] = make_float2(0.0f, 0.0f);
                    weigh(0);
                }
                leave(0);
                weigh(1);
                leave(1);
                l += sums[0].x + sums[0].y + sums[1].x + sums[1].y;
            }
            // ---- outputs, half of the columns each ----
            ok = ok && wait(Bars::o_full + s, tiles);
            *mine_at = l;
            if (either(!ok)) break;
            tc::tc_fence_after();
            float inv;                     // (sums are 2^8 or more: their reciprocals are normal numbers)
            asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(l + *other_at));
            uint16_t* out = a.out + ((int64_t)(u.start + token) * heads + u.kv_head * a.group + head) * a.Dv;
            // (Rows of their own are 32 of them to an instruction, 32 bytes each.  Four lanes that first exchange pieces, to
            // write 64 bytes of a row together, halve what the memory pipe does but take 300 instructions instead of 120, in
            // all warps at about the same time.)
            float2 odd2 = make_float2(0.0f, 0.0f);
#pragma unroll 1
            for (int c = c_first; c < c_end; c += 16) {
                uint32_t v[16], w[8];
                tc::tmem_ld16(t_s + o_col + c, v);
#pragma unroll
                for (int k = 0; k < 16; k += 2) {
                    const float2 y = mul2(make_float2(__uint_as_float(v[k]), __uint_as_float(v[k + 1])), make_float2(inv, inv));
                    odd2 = fma2(y, make_float2(0.0f, 0.0f), odd2);
                    // (an average of values of the type is not beyond it, though rounded weights may say so)
                    w[k / 2] = pack_finite<BF16>(y.x, y.y);
                }
                if (live) {
                    if (pl.wide_rows) {
                        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + c), "r"(w[0]), "r"(w[1]),
                                     "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                                     : "memory");
                    } else {
                        *reinterpret_cast<uint4*>(out + c) = make_uint4(w[0], w[1], w[2], w[3]);
                        if (c + 8 < a.Dv) *reinterpret_cast<uint4*>(out + c + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                }
            }
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(bar(Bars::o_free + s));
            ++tiles;
            const float odd = odd2.x + odd2.y;      // NaN where an output is not finite
            // rows to be done again, behind both halves' stores
            if (either(live && odd != 0.0f)) {
                *mine_at = odd;
                either(false);
                const bool row_odd = live && (odd != 0.0f || *other_at != 0.0f);
                // (every second one each)
                unsigned again = __ballot_sync(0xffffffffu, row_odd && (lane & 1) == half);
                while (again != 0) {
                    const int from = __ffs(again) - 1;
                    again &= again - 1;
                    const int t = __shfl_sync(0xffffffffu, u.start + token, from), h = __shfl_sync(0xffffffffu, u.kv_head * a.group + head, from);
                    const int e = __shfl_sync(0xffffffffu, end, from);
                    prompt_row<BF16, true>(a, h, t, u.start, u.start + e, tick);
                    __syncwarp();
                }
            }
        }
    }
    __syncthreads();
    if (tc::abort_raised(abort_flag)) {
        // a copy did not come: let those on their way land, and the MMAs end, within the same bound
        const long long t0 = tc::globaltimer();
        if (warp == 1) {
            flights.land([&](int i, uint32_t parity) { return tc::mbar_try_wait(bar(i), parity); },
                         [&]() { return tc::globaltimer() - t0 < kWaitNs; });
        } else if (warp == 0 || (TILES == 2 && warp == 2)) {
            if (tc::elect_one()) tc::mma_commit(bar(Bars::drain));
            while (!tc::mbar_try_wait(bar(Bars::drain), 0) && tc::globaltimer() - t0 < kWaitNs) {
            }
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols) : "memory");
}

// [tokens][heads][channels] in boxes of 64 channels.
bool encode(const PromptSide& x, bool bf16, int64_t n, int heads, int D, int box_heads, int box_tokens, CUtensorMap* map) {
    const EncodeTiledFn enc = encode_fn();
    if (enc == nullptr) return false;
    // (strides of dimensions of one are not used, but have to be some)
    if (x.head == 0) heads = 1;
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)n};
    const cuuint64_t strides[2] = {heads > 1 ? (cuuint64_t)(2 * x.head) : 512, n > 1 ? (cuuint64_t)(2 * x.token) : 512};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens}, step[3] = {1, 1, 1};
    return enc(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<uint16_t*>(x.p), dims, strides,
               box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Rows on 16 bytes, no further apart than a tensor map reaches; a row of all tokens, or (queries) of all heads, has none.
bool mapped(const PromptSide& x, int64_t n, int heads, bool shared_heads) {
    const int64_t far = (int64_t)1 << 39;
    return (uintptr_t)x.p % 16 == 0 && (n == 1 || (x.token > 0 && x.token % 8 == 0 && x.token < far / 2)) &&
           (heads == 1 || (x.head == 0 ? shared_heads : x.head > 0 && x.head % 8 == 0 && x.head < far / 2));
}

// Asks for the shared memory, once per device and kernel (`which`).
cudaError_t prepared(const void* kernel, int which, int shared) {
    static std::atomic<uint32_t> done[64];
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const bool known = device >= 0 && device < 64;
    if (known && (done[device].load(std::memory_order_relaxed) >> which & 1u) != 0) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
    if (e == cudaSuccess) e = prefer_max_shared(kernel);
    if (e == cudaSuccess && known) done[device].fetch_or(1u << which, std::memory_order_relaxed);
    return e;
}

bool make_plan(const PromptArgs& a, int tiles, int ctas, PromptPlan* p) {
    p->row_heads = a.group < 128 ? a.group : 128;
    p->tile_tokens = 128 / p->row_heads;
    p->head_parts = (a.group + p->row_heads - 1) / p->row_heads;
    p->k_atoms = (a.D + 63) / 64;
    p->v_atoms = (a.Dv + 63) / 64;
    p->o_cols = (a.Dv + 15) / 16 * 16;
    p->wide_rows = a.Dv % 16 == 0 && (uintptr_t)a.out % 32 == 0;
    if ((tiles * ctas == 1 ? 2 : 1) * kTok + p->o_cols > 512 / (tiles * ctas)) return false;
    p->slot_bytes = (p->k_atoms > 1 || p->v_atoms > 1 ? 2 : 1) * kAtom;
    p->ring_off = tiles * p->k_atoms * kAtom;
    p->slots = (shared_of(ctas) - kMisc - p->ring_off) / p->slot_bytes;
    if (p->slots > kMaxSlots) p->slots = kMaxSlots;
    p->misc_off = p->ring_off + p->slots * p->slot_bytes;
    p->smem = p->misc_off + kMisc;
    return p->slots >= 3 || (ctas == 2 && p->slots >= 2);
}

}  // namespace

bool prompt_tile_supported(const PromptArgs& a) {
    return a.scale <= kMostScale && a.D % 8 == 0 && a.Dv % 8 == 0 && (uintptr_t)a.out % 16 == 0 && mapped(a.q, a.n, a.k_heads * a.group, false) &&
           mapped(a.k, a.n, a.k_heads, true) && mapped(a.v, a.n, a.k_heads, true);
}

cudaError_t launch_prompt_tile(const PromptArgs& a, bool bf16, unsigned* counters, cudaStream_t st) {
    PromptPlan p{};
    int tiles = 1, ctas = 2;
    // Prompts of 128 rows or less on the average go to two CTAs an SM: the second has the time that the first spends
    // between units.  (200 prompts x 12 heads, us with one / two: 100 tokens of 64 channels 52 / 44, of 128 60 / 58, 120
    // of 128 62 / 63; 160 of 64 79 / 85.)
    const bool small = (int64_t)a.n * (a.group < 128 ? a.group : 128) <= 128 * (int64_t)a.B;
    if (!small || !make_plan(a, 1, 2, &p)) {
        ctas = 1;
        tiles = 2;
        if (!make_plan(a, 2, 1, &p)) {
            tiles = 1;
            if (!make_plan(a, 1, 1, &p)) return cudaErrorNotSupported;
        }
    }
    PromptMaps maps;
    if (!encode(a.q, bf16, a.n, a.k_heads * a.group, a.D, p.row_heads, p.tile_tokens, &maps.q) ||
        !encode(a.k, bf16, a.n, a.k_heads, a.D, 1, kTok, &maps.k) || !encode(a.v, bf16, a.n, a.k_heads, a.Dv, 1, kTok, &maps.v))
        return cudaErrorUnknown;
    // as many units as the prompts can make, each of which ends one
    const int64_t unit_tokens = tiles * p.tile_tokens;
    const int64_t units = ((int64_t)a.n / unit_tokens + (a.B < a.n ? a.B : a.n)) * a.k_heads * p.head_parts;
    if (units > 2000000000) return cudaErrorNotSupported;      // they are numbered in 32 bits
    const int most = ctas * num_sms(), grid = (int)(units < most ? units : most);
    auto* kernel = ctas == 2 ? (bf16 ? prompt_tile_kernel<true, 1, 2> : prompt_tile_kernel<false, 1, 2>)
                             : (tiles == 2 ? (bf16 ? prompt_tile_kernel<true, 2, 1> : prompt_tile_kernel<false, 2, 1>)
                                           : (bf16 ? prompt_tile_kernel<true, 1, 1> : prompt_tile_kernel<false, 1, 1>));
    const cudaError_t e = prepared(reinterpret_cast<const void*>(kernel), 2 * (tiles - 1 + 2 * (ctas - 1)) + bf16, shared_of(ctas));
    if (e != cudaSuccess) return e;
    const long long limit = take_wait_limit();
    kernel<<<grid, 128 + 256 * tiles, p.smem, st>>>(a, p, maps, counters, take_drop_arrival() ? 1 : 0, limit > 0 ? limit : kWaitNs);
    note_launch();
    return cudaGetLastError();
}

}  // namespace soniq
