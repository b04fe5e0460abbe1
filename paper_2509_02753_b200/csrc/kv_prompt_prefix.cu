// Attention of many query rows over the shared prefix of a group of requests (kv_prompt_body.cuh has the kernel).
#include "kv_prompt_body.cuh"

namespace lexi {
namespace kv {

void prefix_prompt_pieces(AttendArgs &a, int sm_count) {
    const int w = padded_width(a.D);
    a.piece_rows = w == 256 ? kTileRows : 2 * kTileRows;
    a.result_rows = kTileRows;
    a.piece_results = a.dtype == MOE_F32 && w == 128 ? 2 : 1;          // alternating groups have a result each
    a.piece_ctas = sm_count;
}

cudaError_t launch_attend_prefix_prompt(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) { return launch_prompt<true>(a, sm_count, s, launches); }

}  // namespace kv
}  // namespace lexi
