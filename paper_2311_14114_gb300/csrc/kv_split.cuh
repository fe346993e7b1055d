// How the attention kernels share their work: the list of all chunks (a fixed
// number of cached tokens of one item: a sequence, key head and tile of query
// rows) is cut into ranges, one or more per CTA, from the lengths on the device.
//
// Items come in entries: entry e (a sequence, or a sequence's row tile) stands
// for `mult` items of chunks(e) chunks each.  Few items: each is cut in equal
// parts, a CTA to a part, if that costs no CTA more than `slack` chunks over the
// even split.  Otherwise the list is cut evenly, and a CTA may end one item and
// begin another; there an item counts `lead` units more than its chunks, in front
// of them, for what it costs whatever its length.  CTAs that share an item leave
// partial results, each in a place of its own, which are joined in order, so the
// outputs do not depend on which CTA was first.
#pragma once

#include "kv_internal.h"

namespace soniq {

struct Segment {
    int entry, item;         // item: 0 .. mult - 1 of the entry
    int c_first, c_end;
    int cta0, n_part;        // the CTAs that share the item
    int slot, cta0_slot;     // places of this part and (0 or 1) of the first CTA's
};

struct Split {
    uint32_t part_chunks;              // 0: the even cut
    uint32_t n_cta, per, more, pos, hi, lo, base, mult, lead;
    int entry;

    // shared: 32 words (at most 30 warps).  Every thread of the CTA calls it; false: this CTA has
    // nothing to do.  chunks(e) is 0 for an entry without work.
    template <typename F>
    __device__ __forceinline__ bool begin(F chunks, int n_entries, uint32_t mult_, uint32_t min_chunks, uint32_t lead_,
                                          uint32_t slack, uint32_t* shared) {
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
        mult = mult_;
        lead = lead_;
        part_chunks = lo = hi = 0;
        per = 1;
        more = 0;
        // exclusive prefix sum over the CTA, and the total
        auto scan = [&](uint32_t mine, uint32_t& all) {
            uint32_t incl = mine;
            for (int i = 1; i < 32; i <<= 1) {
                const uint32_t o = __shfl_up_sync(0xffffffffu, incl, i);
                if (lane >= i) incl += o;
            }
            __syncthreads();
            if (lane == 31) shared[warp] = incl;
            __syncthreads();
            all = 0;
            uint32_t before = incl - mine;
            for (int w = 0; w < n_warps; ++w) {
                const uint32_t o = shared[w];
                if (w < warp) before += o;
                all += o;
            }
            return before;
        };
        const bool one_scan = n_entries <= (int)blockDim.x;
        auto units_of = [&](int e) {
            const uint32_t n = chunks(e);
            return n == 0 ? 0u : n + lead;
        };
        uint32_t total, mine = 0, before = 0, items = 0xffffffffu;
        if (one_scan) {
            mine = tid < n_entries ? units_of(tid) : 0;
            items = __syncthreads_count(mine > 0) * mult;
            before = scan(mine, total);
        } else {
            for (int e = tid; e < n_entries; e += blockDim.x) mine += units_of(e);
            scan(mine, total);
        }
        total *= mult;      // below 2^31 (checked on the host)
        if (total == 0) return false;
        if (items <= gridDim.x) {
            const uint32_t free_cta = gridDim.x - min(items, gridDim.x / 2);
            const uint32_t want = max((total - items * lead + free_cta - 1) / free_cta, min_chunks);
            const uint32_t mine_units = mine == 0 ? 0 : (mine - lead + want - 1) / want * mult;
            uint32_t units;
            const uint32_t u0 = scan(mine_units, units);
            if (units <= gridDim.x && want <= total / gridDim.x + slack) {
                part_chunks = want;
                n_cta = units;
                if (u0 <= blockIdx.x && blockIdx.x < u0 + mine_units) {
                    shared[30] = tid;
                    shared[31] = u0;
                }
            }
        }
        if (part_chunks == 0) {
            n_cta = min((total + min_chunks - 1) / min_chunks, gridDim.x);
            // the first `more` CTAs take one chunk more than the others
            per = total / n_cta;
            more = total - per * n_cta;
            if (blockIdx.x < n_cta) {
                lo = range_of(blockIdx.x);
                hi = range_of(blockIdx.x + 1);
            }
            // the entry of chunk lo
            uint32_t run = 0;
            for (int e0 = 0; e0 < n_entries; e0 += blockDim.x) {
                uint32_t all = 0;
                if (!one_scan) {
                    mine = e0 + tid < n_entries ? units_of(e0 + tid) : 0;
                    before = scan(mine, all);
                }
                const uint32_t at = (run + before) * mult;
                if (mine > 0 && at <= lo && lo < at + mine * mult) {
                    shared[30] = e0 + tid;
                    shared[31] = at;
                }
                run += all;
            }
        }
        if (blockIdx.x >= n_cta) return false;
        __syncthreads();
        entry = (int)shared[30];
        base = shared[31];
        pos = lo;
        // a range within an item's lead has no chunks
        return part_chunks != 0 || hi - lo > left_of_lead(lo, chunks(entry) + lead);
    }

    template <typename F>
    __device__ __forceinline__ Segment segment(F chunks) {
        Segment s;
        uint32_t nch = chunks(entry);
        s.slot = 2 * blockIdx.x;
        if (part_chunks != 0) {
            const uint32_t parts = (nch + part_chunks - 1) / part_chunks, unit = blockIdx.x - base;
            s.item = (int)(unit / parts);
            const uint32_t part = unit - s.item * parts;
            s.c_first = (int)((uint64_t)nch * part / parts);
            s.c_end = (int)((uint64_t)nch * (part + 1) / parts);
            s.cta0 = (int)(blockIdx.x - part);
            s.n_part = (int)parts;
            s.cta0_slot = 0;
        } else {
            // (an entry without chunks has no units)
            while (nch == 0 || pos >= base + (nch + lead) * mult) {
                base += nch == 0 ? 0 : (nch + lead) * mult;
                nch = chunks(++entry);
            }
            s.item = (int)((pos - base) / (nch + lead));
            const uint32_t first = base + s.item * (nch + lead) + lead;      // unit of its first chunk
            s.c_first = pos > first ? (int)(pos - first) : 0;
            s.c_end = min((int)(hi - first), (int)nch);
            s.cta0 = (int)owner_of(first);
            s.n_part = (int)owner_of(first + nch - 1) - s.cta0 + 1;
            // a CTA's first range leaves its partial result in the first of its two places
            s.slot += pos == lo ? 0 : 1;
            s.cta0_slot = range_of(s.cta0) + lead >= first ? 0 : 1;
            pos = first + s.c_first;
        }
        s.entry = entry;
        return s;
    }

    // Behind a segment; false: it was the last.
    __device__ __forceinline__ bool next(const Segment& s) {
        pos += s.c_end - s.c_first;
        return part_chunks == 0 && hi > pos + lead;       // a next item's chunks come behind its lead
    }

private:
    // Units from u to the first chunk of its item (0: u is a chunk).
    __device__ __forceinline__ uint32_t left_of_lead(uint32_t u, uint32_t item_units) const {
        const uint32_t at = (u - base) % item_units;
        return at < lead ? lead - at : 0;
    }
    __device__ __forceinline__ uint32_t range_of(uint32_t c) const { return per * c + min(c, more); }
    __device__ __forceinline__ uint32_t owner_of(uint32_t chunk) const {
        const uint32_t cut = more * (per + 1);
        return chunk < cut ? chunk / (per + 1) : more + (chunk - cut) / per;
    }
};

// Place of part i of a segment's item.
__device__ __forceinline__ int part_slot(const Segment& s, int i) { return 2 * (s.cta0 + i) + (i == 0 ? s.cta0_slot : 0); }

// End of the tokens that sequence b shows (0: absent, or nothing within its pages).
__device__ __forceinline__ int64_t seen_end(const KvGeom& geo, const KvAttendArgs& a, int b) {
    const int len = a.lengths[b];
    if (len < 0) return 0;
    const int64_t cap = (int64_t)a.max_pages << geo.page_shift, end = (int64_t)len + a.T;
    return end < cap ? end : cap;
}

// Reports lengths beyond the page table and writes the outputs of absent
// sequences; called by `count` threads of each CTA, `rank` among them.
__device__ __forceinline__ void check_lengths(const KvGeom& geo, const KvAttendArgs& a, int rank, int count) {
    if (blockIdx.x == 0) {
        for (int b = rank; b < a.B; b += count)
            if (a.lengths[b] >= 0 && (int64_t)a.lengths[b] + a.T > ((int64_t)a.max_pages << geo.page_shift))
                atomicOr(a.err, kErrKvIndex);
    }
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        if (a.lengths[b] >= 0) continue;
        const int64_t size = (int64_t)a.T * a.group * geo.heads * geo.s[1].D;
        for (int64_t i = rank; i < size; i += count) a.out[b * size + i] = 0;
    }
}

}  // namespace soniq
