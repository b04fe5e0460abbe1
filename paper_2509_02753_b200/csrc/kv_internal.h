// Internal declarations of the operators around the 4-bit key/value cache (C ABI: include/moe_kv.h).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "moe_internal.h"
#include "moe_kv.h"

namespace lexi {
namespace kv {

constexpr int kBlockTokens = 16;       // tokens of one block of the cache
constexpr int kMaxRequests = 4096;

// head_dim rounded up to a width the kernels are built for
__host__ __device__ constexpr int padded_width(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }
__host__ __device__ constexpr int block_bytes(int w) { return 18 * w; }
__host__ __device__ constexpr int v_codes_at(int w) { return 8 * w; }
__host__ __device__ constexpr int k_scales_at(int w) { return 16 * w; }
__host__ __device__ constexpr int v_scales_at(int w) { return 17 * w; }
// XOR on the byte offset token * (W/16) inside stretch r of the value codes
__host__ __device__ constexpr int v_turn(int w, int r) {
    return w == 64 ? ((r >> 1) & 1) * 32 : w == 128 ? (r & 1) * 64 : (r & 1) * 16;
}

// a page's bounds of one head: largest and smallest key in 8 bits, the step and 12 bytes of zeros
__host__ __device__ constexpr int summary_bytes(int w) { return 2 * w + 16; }

struct Rows { const void *p; int64_t ts, hs; };

// n / d for every 32-bit n and d >= 1 by one high product (Granlund and Montgomery's division by invariants): the
// kernels of few instructions a thread spent most of them in the compiler's divisions
struct FastDiv {
    uint32_t d, m, s1, s2;
    __host__ __device__ FastDiv() : d(1), m(1), s1(0), s2(0) {}
    __host__ explicit FastDiv(uint32_t by) : d(by) {
        uint32_t l = 0;
        while (l < 32 && (1ull << l) < by) ++l;
        m = (uint32_t)(((1ull << 32) * ((1ull << l) - by)) / by + 1);
        s1 = l < 1 ? l : 1;
        s2 = l < 1 ? 0 : l - 1;
    }
#ifdef __CUDACC__
    __device__ __forceinline__ uint32_t div(uint32_t n) const {
        const uint32_t t = __umulhi(m, n);
        return (t + ((n - t) >> s1)) >> s2;
    }
    __device__ __forceinline__ void split(uint32_t n, uint32_t &q, uint32_t &r) const { q = div(n); r = n - q * d; }
#endif
};

#ifdef __CUDACC__
// A request of a call, as all kernels take it: keys that the tables have room for, first new token, new tokens
struct Request { int i, len, q0, nq; };

// The first request i with f(cu[i + 1], i + 1) > x, where f does not fall; i = n, without rows, if there is none.  By a whole warp, 32
// probes at a time; the last ones bring the lengths along, so that these are not one more read that waits for another.
// T: rows of the call; room: tokens that a row of the table stands for
template <typename F>
__device__ __forceinline__ Request find_request(const int32_t *cu, const int32_t *kv_len, int n, int x, int T, int64_t room, int32_t *status, F f) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = n;
#pragma unroll 1
    while (hi - lo > 32) {
        const int step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step, in = min(at, hi);
        const int before = __popc(__ballot_sync(0xffffffffu, at <= hi && f(cu[in], in) <= x));
        lo = min(lo + before * step, hi);
        hi = min(lo + step, hi);
    }
    const int at = min(lo + lane, n - 1);
    const int c0 = cu[at], c1 = cu[at + 1], l = kv_len[at];
    const int found = __popc(__ballot_sync(0xffffffffu, lo + lane < hi && f(c1, at + 1) <= x));
    Request r{lo + found, max(__shfl_sync(0xffffffffu, l, found & 31), 0), __shfl_sync(0xffffffffu, c0, found & 31), __shfl_sync(0xffffffffu, c1, found & 31)};
    r.nq -= r.q0;
    if (lo + found >= hi) return Request{n, 0, 0, 0};
    const bool bad_rows = r.q0 < 0 || r.nq < 0 || r.q0 > T - r.nq;
    if ((bad_rows || r.len > room) && lane == 0) atomicOr(status, MOE_KV_STATUS_BAD_INDEX);
    if (bad_rows) r.nq = 0;
    r.len = (int)min((int64_t)r.len, room);
    return r;
}
#endif

struct TablesArgs {
    const int32_t *ctx, *fresh_tokens; int n;
    const int32_t *free_pages; int n_free;
    int32_t *table; int width, page_shift;        // a page has 1 << page_shift tokens
    int n_tokens;
    int32_t *kv_len, *cu, *position; int64_t *slot; int32_t *taken;
    int32_t *status;
};
cudaError_t launch_tables(const TablesArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);

struct RopeTableArgs { int n, half; double base, factor, low, high, original, magnitude; int scaling; float2 *table; };
cudaError_t launch_rope_table(const RopeTableArgs &a, cudaStream_t s);

struct Turn {            // rotary positions of a call
    const int32_t *position; const float2 *table; int n_positions, rot, layout, inverse;
};
struct RopeArgs {
    int dtype; Rows x; int T, H, D; Turn turn; void *y; int64_t yts, yhs; int32_t *status;
};
cudaError_t launch_rope(const RopeArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);

struct AppendArgs {
    int dtype; Rows q, k, v; int T, H, Hk, D, page_shift; Turn turn;
    const int64_t *slot; float k_scale, v_scale, k_inv6, v_inv6; void *q_out;
    uint8_t *cache; int64_t n_slots; int32_t *status;
};
cudaError_t launch_append(const AppendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);

struct ReadArgs {
    int dtype; const uint8_t *cache; int64_t n_slots; const int64_t *slot; int T, Hk, D, page_shift;
    float k_scale, v_scale; void *k, *v; int32_t *status;
};
cudaError_t launch_read(const ReadArgs &a, cudaStream_t s, uint64_t *launches);

// summaries of pages and the selection by them
constexpr size_t kSelectSmem = 192 * 1024;       // of scores, at most: 49152 pages of one token
struct SelectArgs {
    int dtype; Rows q; int T; const int32_t *cu, *kv_len; int n; int max_new;
    const int32_t *table; int width; const uint8_t *cache; int n_pages;
    int Hk, G, D, page_shift;                 // a page has 1 << page_shift tokens
    uint8_t *summaries;
    int n_select, first, last; int32_t *selected;
    int room;                                 // scores of a token
    int32_t *status;
};
cudaError_t launch_summarise(const SelectArgs &a, cudaStream_t s, uint64_t *launches);
cudaError_t launch_select(const SelectArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);
struct ReadSummariesArgs {
    const uint8_t *summaries; int n_pages; const int32_t *page; int m, Hk, D; float k_scale; float *high, *low; int32_t *status;
};
cudaError_t launch_read_summaries(const ReadSummariesArgs &a, cudaStream_t s, uint64_t *launches);

struct PrefixArgs {
    const int32_t *groups; int n_groups; const int32_t *cu, *kv_len; int n;
    const int32_t *table; int width, page_shift;        // a page has 1 << page_shift tokens
    int32_t *shared, *start; int32_t *status;
};
cudaError_t launch_prefix(const PrefixArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);

struct AttendArgs {
    int dtype; Rows q; int T; const int32_t *cu, *kv_len; int n; int max_new;
    const int32_t *table; int width; const uint8_t *cache; int n_pages;
    int H, Hk, G, D, page_shift;              // a page has 1 << page_shift blocks of 16 tokens
    float score_scale;                        // softmax_scale * k_scale * log2(e)
    float v_scale; int window, sinks;
    void *out;
    float *part; float2 *part_ml; int32_t *arrived; int max_ctas;   // split over the keys
    FastDiv g_div;                            // by G
    // requests of more query rows per key/value head than this are kv_prompt.cu's; 0: all are the launched kernel's
    int prompt_rows;
    float *prompt_part; float2 *prompt_ml; int32_t *prompt_arrived;
    int32_t *status;
    // Shared prefixes.  Prefix: n groups, group i = requests [groups[i], groups[i + 1]) of n_members, kv_len its shared keys,
    // max_new the largest number of its new tokens.  Rest: request i reads the keys from start[i] on.  A row's sums, reference
    // and denominator over what is behind the prefix lie in own_part [T][H][W] and own_ml [T][H]; those over its prefix
    // in o_part and o_ml likewise, o_pieces being (-1, ...), or in the pieces of
    // its stretch, o_pieces being (first CTA, CTAs, row): that row of prompt_part and prompt_ml in slot 1 of the first CTA and
    // 0 of the others.  A slot has piece_rows rows, results of result_rows each where there are piece_results of them; piece_ctas CTAs
    // have slots
    const int32_t *groups, *member_len; int n_members;       // member_len: the requests' keys
    const int32_t *start;
    float *o_part, *own_part; float2 *o_ml, *own_ml; int4 *o_pieces;
    int piece_rows, result_rows, piece_results, piece_ctas;
    // Selected pages: [T][Hk][n_listed] columns of the request's row of the block table, -1: none
    const int32_t *listed; int n_listed;
    int cluster;                              // CTAs that have a stretch's pieces, 0: no clusters
};
#ifdef __CUDACC__
__device__ __forceinline__ int div_g(const AttendArgs &a, int row) { return (int)a.g_div.div((uint32_t)row); }      // row / G
#endif
// rows of queries that share a key/value head, in the N dimension of mma.sync (kv_attend.cu)
cudaError_t launch_attend_rows(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);
size_t attend_part_floats(int w);          // per CTA of the grid
void prefix_rows_pieces(AttendArgs &a, int max_ctas);          // how the kernel below lays out its pieces
cudaError_t launch_attend_prefix_rows(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);
cudaError_t launch_attend_rest_rows(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);
cudaError_t launch_attend_join(const AttendArgs &a, cudaStream_t s, uint64_t *launches);
cudaError_t launch_attend_listed(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);
// prompts, on tcgen05 (kv_prompt.cu)
cudaError_t launch_attend_prompt(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);
void prefix_prompt_pieces(AttendArgs &a, int sm_count);
cudaError_t launch_attend_prefix_prompt(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);
size_t prompt_part_floats(int w);          // per CTA, of which there is one per SM
size_t prompt_part_rows();

}  // namespace kv
}  // namespace lexi
