// The order of a warp's copies through a ring of kStages stages, each with a barrier that counts its copies (attn.cu).  Plain
// arithmetic, so that it can be followed on the host.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define DSP_RING_FN __host__ __device__ __forceinline__
#else
#define DSP_RING_FN inline
#endif

namespace dsp {

template <int kStages> struct CopyRing {
    uint32_t phases = 0u;                        // a bit per stage: parity that its barrier's next completion has
    int stage = 0;                               // the next to be used
    DSP_RING_FN void restart() { stage = 0; }    // nothing is under way
    DSP_RING_FN uint32_t parity() const { return (phases >> stage) & 1u; }
    // Where the copy goes that is kStages - 1 after the one in use: the stage used before.
    DSP_RING_FN int before() const { return stage == 0 ? kStages - 1 : stage - 1; }
    // The copy of `stage` has come (or is not waited for any more).
    DSP_RING_FN void used() {
        phases ^= 1u << stage;
        stage = stage == kStages - 1 ? 0 : stage + 1;
    }
    // Copies that are under way when iteration `run` of run, run + step, .. run_end is waited for, `ahead` being the next to be fetched.
    static DSP_RING_FN int under_way(int run, int ahead, int run_end, int step) {
        const int end = ahead < run_end ? ahead : run_end;
        return end > run ? (end - run + step - 1) / step : 0;
    }
};

}  // namespace dsp
