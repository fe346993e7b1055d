// Copies on their way into a ring of at most 32 stages, each signalled by an
// mbarrier of its own: what a CTA that gives up has to wait for before its
// shared memory may become another's.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define SONIQ_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define SONIQ_HOST_DEVICE inline
#endif

namespace soniq {

struct Flights {
    uint32_t issued = 0, parity = 0;      // by stage: a copy was issued; the parity of the phase that its arrival ends

    SONIQ_HOST_DEVICE void issue(int stage, uint32_t phase) {
        issued |= 1u << stage;
        parity = (parity & ~(1u << stage)) | (phase & 1u) << stage;
    }
    // Waits for the last copy of every stage, while more() allows; false: some did not come.  try_wait(stage, parity)
    // says whether the phase of that parity is over.  Only the phase of the last copy will do: of the two parities one
    // is always over, the running phase's predecessor's.  (Earlier copies of a stage came before its last was issued.)
    template <typename Try, typename More>
    SONIQ_HOST_DEVICE bool land(Try try_wait, More more) const {
        for (int s = 0; issued >> s != 0; ++s) {
            if ((issued >> s & 1u) == 0) continue;
            while (!try_wait(s, parity >> s & 1u))
                if (!more()) return false;
            if (s == 31) break;
        }
        return true;
    }
};

}  // namespace soniq
