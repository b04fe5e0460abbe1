// Attention of few query rows over all keys of their requests (kv_attend_body.cuh has the kernel).
#include "kv_attend_body.cuh"

namespace lexi {
namespace kv {

size_t attend_part_floats(int w) { return (size_t)2 * (w == 256 ? 16 : 32) * w; }

cudaError_t launch_attend_rows(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    long long rows = (long long)(a.max_new > 0 ? a.max_new : a.T) * a.G;
    if (a.prompt_rows > 0 && rows > a.prompt_rows) rows = a.prompt_rows;
    return launch_rows<Reads::Every>(rows, a, sm_count, s, launches);
}

}  // namespace kv
}  // namespace lexi
