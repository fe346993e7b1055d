// What the tcgen05 attention kernels share: MMAs on tiles of 16-bit operands,
// rings of stages, and bounded waits of whole warps.
#pragma once

#include "kv_device.cuh"

namespace soniq {

__device__ __forceinline__ void tmem_st16v(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n\t"
        "tcgen05.wait::st.sync.aligned;" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// Values as an MN-major operand: 64-channel column groups `group` bytes apart, 8-token rows of 1024 bytes.
__device__ __forceinline__ uint64_t value_desc(uint32_t at, uint32_t group) {
    uint64_t d = (uint64_t)((at & 0x3FFFFu) >> 4);
    d |= (uint64_t)(group >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc));
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(acc));
}

__device__ __forceinline__ void bar_group(int id, int threads) {
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// Position in a ring of n stages and the parity of its current round.
struct Ring {
    int i = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void step(int n) {
        if (++i == n) {
            i = 0;
            phase ^= 1u;
        }
    }
    __device__ __forceinline__ void skip(int by, int n) {
        const int to = i + by, rounds = to / n;
        i = to - rounds * n;
        phase ^= rounds & 1;
    }
};

// Wait of a whole warp for phase `parity` of `bar`; one result for its lanes:
// false once the CTA gives up, or when the wait is given up after 2 s.  (The
// polling loop is written out: twenty warps' polls took a third of the issue
// slots, and what all roles run has to stay in the instruction cache.  A poll may
// suspend the warp for a time that the hardware sets, so the clock is read every
// 64 of them.)
template <typename F>
__device__ __forceinline__ bool wait_until(F poll, uint32_t abort_flag, unsigned* err) {
    long long t0 = 0;
    while (true) {
        if (__all_sync(0xffffffffu, poll())) return true;
        if (__any_sync(0xffffffffu, tc::abort_raised(abort_flag))) return false;
        const long long t = tc::globaltimer();
        if (t0 == 0) t0 = t;
        if (__any_sync(0xffffffffu, t - t0 > kWaitNs)) {
            tc::set_flag(abort_flag, 1);
            atomicOr(err, kErrWait);
            return false;
        }
    }
}
__device__ __forceinline__ uint32_t poll64(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .u32 n;\n\tmov.u32 n, 64;\n"
        "TRY:\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t@p bra DONE;\n\t"
        "sub.u32 n, n, 1;\n\tsetp.ne.u32 q, n, 0;\n\t@q bra TRY;\n"
        "DONE:\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done;
}
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, uint32_t abort_flag, unsigned* err) {
    return wait_until([&]() { return poll64(bar, parity); }, abort_flag, err);
}
// One that looks at no clock: another warp of the CTA does, for all of them, and raises the flag.
__device__ __forceinline__ bool wait_watched(uint32_t bar, uint32_t parity, uint32_t abort_flag) {
    while (true) {
        if (__all_sync(0xffffffffu, poll64(bar, parity))) return true;
        if (__any_sync(0xffffffffu, tc::abort_raised(abort_flag))) return false;
    }
}
// That warp's: given up after `limit` in which sign(), a word that others change as they get on, stayed the same.
template <typename Sign>
__device__ __forceinline__ bool wait_watching(uint32_t bar, uint32_t parity, uint32_t abort_flag, unsigned* err, Sign sign, long long limit) {
    long long t0 = 0;
    uint32_t seen = 0;
    while (true) {
        if (__all_sync(0xffffffffu, poll64(bar, parity))) return true;
        const long long t = tc::globaltimer();
        const uint32_t now = __shfl_sync(0xffffffffu, sign(), 0);
        if (t0 == 0 || now != seen) {
            t0 = t;
            seen = now;
        }
        if (__any_sync(0xffffffffu, t - t0 > limit)) {
            tc::set_flag(abort_flag, 1);
            atomicOr(err, kErrWait);
            return false;
        }
    }
}
// The same for two or three barriers, whose phases stay complete until this warp has gone
// on.  (One after the other, three waits that were over took 870 cycles of a block's 3550.)
__device__ __forceinline__ bool wait_warp2(uint32_t b0, uint32_t parity0, uint32_t b1, uint32_t parity1, uint32_t abort_flag, unsigned* err) {
    return wait_until([&]() {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p, q;\n\t.reg .u32 n;\n\tmov.u32 n, 64;\n"
            "TRY:\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 q, [%3], %4;\n\t"
            "and.pred p, p, q;\n\t@p bra DONE;\n\t"
            "sub.u32 n, n, 1;\n\tsetp.ne.u32 q, n, 0;\n\t@q bra TRY;\n"
            "DONE:\n\tselp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(b0), "r"(parity0), "r"(b1), "r"(parity1)
            : "memory");
        return done;
    }, abort_flag, err);
}
__device__ __forceinline__ bool wait_warp3(uint32_t b0, uint32_t parity0, uint32_t b1, uint32_t parity1, uint32_t b2, uint32_t parity2,
                                           uint32_t abort_flag, unsigned* err) {
    return wait_until([&]() {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p, q, r;\n\t.reg .u32 n;\n\tmov.u32 n, 64;\n"
            "TRY:\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 q, [%3], %4;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 r, [%5], %6;\n\t"
            "and.pred p, p, q;\n\tand.pred p, p, r;\n\t@p bra DONE;\n\t"
            "sub.u32 n, n, 1;\n\tsetp.ne.u32 q, n, 0;\n\t@q bra TRY;\n"
            "DONE:\n\tselp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(b0), "r"(parity0), "r"(b1), "r"(parity1), "r"(b2), "r"(parity2)
            : "memory");
        return done;
    }, abort_flag, err);
}

}  // namespace soniq
