// Attention of many query rows over the shared prefix of a group of requests (kv_prompt_body.cuh has the kernel).
#include "kv_prompt_body.cuh"

namespace lexi {
namespace kv {

cudaError_t launch_attend_prefix_prompt(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) { return launch_prompt<true>(a, sm_count, s, launches); }

}  // namespace kv
}  // namespace lexi
