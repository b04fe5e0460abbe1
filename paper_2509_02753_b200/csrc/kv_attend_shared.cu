// Attention of few query rows over the shared prefix of a group of requests, and over what lies behind it
// (kv_attend_body.cuh has the kernel).
#include "kv_attend_body.cuh"

namespace lexi {
namespace kv {

cudaError_t launch_attend_prefix_rows(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    long long rows = (long long)(a.max_new > 0 ? a.max_new : a.T) * a.G;
    if (a.prompt_rows > 0 && rows > a.prompt_rows) rows = a.prompt_rows;
    return launch_rows<Reads::Prefix>(rows, a, sm_count, s, launches);
}

cudaError_t launch_attend_rest_rows(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    return launch_rows<Reads::Rest>((long long)(a.max_new > 0 ? a.max_new : a.T) * a.G, a, sm_count, s, launches);
}

}  // namespace kv
}  // namespace lexi
