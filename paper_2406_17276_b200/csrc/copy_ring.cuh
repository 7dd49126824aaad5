// Which barrier and phase the copies into a ring of stages complete: copy i (counted from the start) goes to stage i % kStages and completes
// phase i / kStages of its barrier.  (No device code, so that the bookkeeping can be run on its own.)
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define OT_RING_FN __host__ __device__ __forceinline__
#else
#define OT_RING_FN inline
#endif

namespace ot {

template <uint32_t kStages> struct CopyRing {
    OT_RING_FN static uint32_t stage(uint32_t i) { return i % kStages; }
    OT_RING_FN static uint32_t parity(uint32_t i) { return i / kStages & 1; }
    // The oldest of `issued` copies that may still be in flight: later copies went to the stages of those before it, which had been taken.
    OT_RING_FN static uint32_t oldest(uint32_t issued) { return issued > kStages ? issued - kStages : 0; }
    // Waits for copies [from, issued) with wait(stage, parity).
    template <class Wait> OT_RING_FN static void drain(uint32_t from, uint32_t issued, Wait wait) {
        for (uint32_t i = from; i < issued; ++i) wait(stage(i), parity(i));
    }
};

}  // namespace ot
