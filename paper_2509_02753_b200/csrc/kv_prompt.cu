// Attention of prompts over all keys of their requests (kv_prompt_body.cuh has the kernel).
#include "kv_prompt_body.cuh"

namespace lexi {
namespace kv {

size_t prompt_part_floats(int w) { return (size_t)2 * (w == 256 ? 128 : 256) * w; }
size_t prompt_part_rows() { return 2 * 256; }

cudaError_t launch_attend_prompt(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) { return launch_prompt<false>(a, sm_count, s, launches); }

}  // namespace kv
}  // namespace lexi
