// Attention of few query rows over the shared prefix of a group of requests, and over what lies behind it
// (kv_attend_body.cuh has the kernel).
#include "kv_attend_body.cuh"

namespace lexi {
namespace kv {

void prefix_rows_pieces(AttendArgs &a, int max_ctas) {
    a.piece_rows = a.result_rows = tile_rows(padded_width(a.D), (long long)a.max_new * a.G);
    a.piece_results = 1;
    a.piece_ctas = max_ctas;
}

cudaError_t launch_attend_prefix_rows(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    return launch_rows<Reads::Prefix>((long long)a.max_new * a.G, a, sm_count, s, launches);
}

cudaError_t launch_attend_rest_rows(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    return launch_rows<Reads::Rest>((long long)a.max_new * a.G, a, sm_count, s, launches);
}

}  // namespace kv
}  // namespace lexi
