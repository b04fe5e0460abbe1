// What a warp of kv_attend.cu knows of its ring of bulk copies: the parity of each stage's next phase, and whether a wait
// ran out.  Plain C++, so that its steps can be checked without a device.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define LEXI_RING_FN __device__ __forceinline__
#else
#define LEXI_RING_FN inline
#endif

namespace lexi {
namespace kv {

template <int STAGES>
struct RingWaits {
    uint32_t phase = 0;          // one bit for each stage
    bool dead = false;

    // Step k of `steps`, of which k .. k + STAGES - 1 are under way: true once its copies have arrived.  wait(stage, parity) is
    // a bounded wait, the same for the whole warp.  Once one ran out nothing more is started, waited for or used, in later
    // pieces of the CTA neither: a copy that came late would count as another piece's.  Copies that are under way then are
    // waited for once more, so that they do not write what the CTA, or the next one, has in their place.
    template <typename Wait>
    LEXI_RING_FN bool arrived(int k, int steps, Wait wait) {
        if (dead) return false;
        const int stage = k % STAGES;
        dead = !wait(stage, (phase >> stage) & 1u);
        if (!dead) {
            phase ^= 1u << stage;
            return true;
        }
#ifdef __CUDACC__
#pragma unroll 1
#endif
        for (int x = k; x < steps && x < k + STAGES; ++x) wait(x % STAGES, (phase >> (x % STAGES)) & 1u);
        return false;
    }
};

}  // namespace kv
}  // namespace lexi
