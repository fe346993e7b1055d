// Where the tokens of a step go: pages taken from and given back to the pool,
// slots and positions.
//
//   has = ceil(old / page), to = ceil(goal / page)
//   pages given back are numbered in the order of sequences and tokens, R in all;
//   pages needed likewise.  The k-th that is needed is the k-th that was given
//   back while k < R, then entry n_free - 1 - (k - R) of the pool; what was given
//   back and not needed, numbers k >= taken, becomes entry n_free + R - 1 - k.
//
// So no sequence waits for another one: two prefix sums over the sequences (in
// 64 bits, in every CTA, from 8 bytes a sequence) number all pages, and tokens,
// table entries and pool entries are then written independently, each finding
// its sequence by bisection in shared memory.  What is read is not written: the
// pool's entries below n_free are read, those from n_free on written; a row's
// entries below `has` are read, the others written.  Lengths and the count, which
// may be updated in place, are written by the last CTA to have read them.
//
// Bound by latency: the launch, two dependent reads (lengths, then table entries),
// the prefix sums' barriers, bisections.  Measured, replayed from a graph (GB300): 8
// sequences that decode 6.2 us, 1000 of which some leave 12.3, 32 prompts of up to
// 4000 tokens 10.3.
#include <atomic>

#include "step_internal.h"

namespace soniq {

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;

struct Two {
    int64_t a, b;
};

// Exclusive prefix sums of a pair over the CTA's threads; `total` of all.
__device__ __forceinline__ Two scan(Two x, Two* sums, Two* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Two y = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t a = __shfl_up_sync(0xffffffffu, y.a, d), b = __shfl_up_sync(0xffffffffu, y.b, d);
        if (lane >= d) y.a += a, y.b += b;
    }
    if (lane == 31) sums[warp] = y;
    __syncthreads();
    Two before{0, 0}, all{0, 0};
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        const Two s = sums[w];
        if (w < warp) before.a += s.a, before.b += s.b;
        all.a += s.a, all.b += s.b;
    }
    __syncthreads();
    *total = all;
    return Two{before.a + y.a - x.a, before.b + y.b - x.b};
}

// The last of at[0 .. n], which rise from 0, that is not above x.
__device__ __forceinline__ int last_upto(const int32_t* at, int n, int x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (at[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

struct Grow {
    int old, goal, has, to;      // tokens and pages, before and after; has at most the table's
    __device__ __forceinline__ Grow(const KvPlanArgs& a, int b) {
        const int n = a.lengths[b], t = a.targets[b];
        const int64_t page = (int64_t)1 << a.page_shift;
        old = max(n, 0);
        goal = max(t, 0);
        has = pages(a, old);
        to = (int)((goal + page - 1) >> a.page_shift);
    }
    __device__ __forceinline__ static int pages(const KvPlanArgs& a, int old) {
        return (int)min((old + ((int64_t)1 << a.page_shift) - 1) >> a.page_shift, (int64_t)a.max_pages);
    }
    __device__ __forceinline__ int tokens() const { return max(goal - old, 0); }
    __device__ __forceinline__ int back() const { return max(has - to, 0); }
    __device__ __forceinline__ int need() const { return max(to - has, 0); }
};

__global__ void __launch_bounds__(kThreads) kv_plan_kernel(const KvPlanArgs a) {
    extern __shared__ int32_t mem[];
    __shared__ Two sums[kWarps];
    __shared__ int32_t taken_of[kWarps];
    __shared__ int last;
    const int tid = threadIdx.x, B = a.B;
    int32_t* start = mem;                    // [B + 1] first token, at most max_tokens
    int32_t* back0 = start + B + 1;          // [B + 1] first page given back
    int32_t* need0 = back0 + B + 1;          // [B + 1] first page needed
    int32_t* old_of = need0 + B + 1;         // [B] tokens before
    int32_t* to_of = old_of + B;             // [B] pages after
    uint8_t* served = reinterpret_cast<uint8_t*>(to_of + B);

    // ---- tokens and pages given back, pages needed; a thread takes neighbouring sequences ----
    const int per = (B + kThreads - 1) / kThreads, b0 = min(tid * per, B), b1 = min(b0 + per, B);
    Two mine{0, 0}, total, at;
    for (int b = b0; b < b1; ++b) {
        const Grow g(a, b);
        mine.a += g.tokens();
        mine.b += g.back();
    }
    at = scan(mine, sums, &total);
    const int64_t cap = a.max_tokens, tokens = min(total.a, cap);
    const int64_t R = total.b;
    Two need{0, 0}, need_all;
    for (int b = b0; b < b1; ++b) {
        const Grow g(a, b);
        start[b] = (int32_t)min(at.a, cap);
        back0[b] = (int32_t)at.b;
        old_of[b] = g.old;
        to_of[b] = g.to;
        at.a += g.tokens();
        at.b += g.back();
        const bool fits = g.to <= a.max_pages && at.a <= cap;
        served[b] = fits;
        need.a += fits ? g.need() : 0;
    }
    if (tid == 0) start[B] = (int32_t)tokens, back0[B] = (int32_t)R;
    const Two before = scan(need, sums, &need_all);
    const int n_free = a.count[0];
    const int pool = min(max(n_free, 0), a.n_pages);
    if (n_free != pool && tid == 0) atomicOr(a.err, kErrKvIndex);
    int64_t upto = before.a;
    int32_t taken = 0;
    for (int b = b0; b < b1; ++b) {
        const Grow g(a, b);
        need0[b] = (int32_t)upto;
        const int n = served[b] ? g.need() : 0;
        upto += n;
        served[b] = g.tokens() == 0 || (served[b] && (n == 0 || upto <= pool + R));
        if (served[b] && n > 0) taken = (int32_t)upto;
    }
    if (tid == 0) need0[B] = (int32_t)need_all.a;
    taken = __reduce_max_sync(0xffffffffu, taken);
    if ((tid & 31) == 0) taken_of[tid >> 5] = taken;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) taken = max(taken, taken_of[w]);

    // ---- pages by their numbers ----
    auto checked = [&](int page) {
        if ((unsigned)page >= (unsigned)a.n_pages) atomicOr(a.err, kErrKvIndex);
        return page;
    };
    auto has_of = [&](int b) { return Grow::pages(a, old_of[b]); };
    auto released = [&](int k) {
        const int b = last_upto(back0, B, k);
        return checked(a.table[b * a.table_stride + to_of[b] + k - back0[b]]);
    };
    auto given = [&](int k) { return k < R ? released(k) : checked(a.free_pages[pool - 1 - (k - (int)R)]); };
    const int first = blockIdx.x * kThreads + tid, step = gridDim.x * kThreads;
    for (int k = first; k < taken; k += step) {
        const int b = last_upto(need0, B, k);
        a.table[b * a.table_stride + has_of(b) + k - need0[b]] = given(k);
    }
    for (int64_t k = (int64_t)taken + first; k < R; k += step) {
        const int64_t to = pool + R - 1 - k;
        if (to < a.n_pages) a.free_pages[to] = released((int)k);
        else atomicOr(a.err, kErrKvIndex);
    }
    // ---- slots and positions ----
    for (int64_t t = first; t < cap; t += step) {
        int64_t slot = -1;
        int pos = 0;
        if (t < tokens) {
            // (of the sequences that start at t, the last: the others have no tokens)
            const int b = last_upto(start, B - 1, (int)t);
            pos = old_of[b] + ((int)t - start[b]);
            if (served[b]) {
                const int i = pos >> a.page_shift, has = has_of(b);
                const int page = i < has ? a.table[b * a.table_stride + i] : given(need0[b] + i - has);
                const int64_t size = (int64_t)1 << a.page_shift;
                slot = (unsigned)page < (unsigned)a.n_pages ? page * size + (pos & (size - 1)) : a.n_pages * size;
            }
        }
        a.slots[t] = slot;
        a.positions[t] = pos;
    }
    if (blockIdx.x == 0)
        for (int b = tid; b <= B; b += kThreads) a.starts[b] = start[b];

    // ---- lengths and the count, once every CTA has read them ----
    __syncthreads();
    if (tid == 0) {
        last = 1;
        if (gridDim.x > 1) {
            __threadfence();
            last = atomicAdd(reinterpret_cast<unsigned*>(a.count + 1), 1u) == gridDim.x - 1;
            __threadfence();
            if (last) a.count[1] = 0;
        }
    }
    __syncthreads();
    if (!last) return;
    for (int b = tid; b < B; b += kThreads) {
        const int n = a.lengths[b], t = a.targets[b];
        a.lengths_out[b] = served[b] ? max(t, -1) : n;
    }
    if (tid == 0) a.count_out[0] = (int32_t)min(pool + R - taken, (int64_t)a.n_pages);
}

constexpr int shared_of(int B) { return 12 * (B + 1) + 9 * B; }

// Asks for the shared memory of the largest call, once per device: the limit is the
// function's, so one that each call set to its own size would fail other threads' launches.
cudaError_t prepared() {
    static std::atomic<bool> done[64];
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const bool known = device >= 0 && device < 64;
    if (known && done[device].load(std::memory_order_relaxed)) return cudaSuccess;
    e = cudaFuncSetAttribute(kv_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared_of(kPlanMaxSequences));
    if (e == cudaSuccess) e = prefer_max_shared(reinterpret_cast<const void*>(kv_plan_kernel));
    if (e == cudaSuccess && known) done[device].store(true, std::memory_order_relaxed);
    return e;
}

}  // namespace

cudaError_t launch_kv_plan(const KvPlanArgs& a, cudaStream_t st) {
    const int smem = shared_of(a.B);
    const cudaError_t e = prepared();
    if (e != cudaSuccess) return e;
    // two tokens to a thread, or one sequence, whose pages are not known here, to a warp
    const int64_t by_tokens = ((int64_t)a.max_tokens + 2 * kThreads - 1) / (2 * kThreads), by_pages = (a.B + 15) / 16;
    const int64_t want = by_tokens > by_pages ? by_tokens : by_pages;
    const int grid = (int)(want < 1 ? 1 : (want < num_sms() ? want : num_sms()));
    kv_plan_kernel<<<grid, kThreads, smem, st>>>(a);
    note_launch();
    return cudaGetLastError();
}

}  // namespace soniq
