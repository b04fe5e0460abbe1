// Attention of single tokens over the pages listed for them (kv_attend_body.cuh has the kernel).
#include "kv_attend_body.cuh"

namespace lexi {
namespace kv {

cudaError_t launch_attend_listed(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    return launch_rows<Reads::Listed>(a.G, a, sm_count, s, launches);
}

}  // namespace kv
}  // namespace lexi
