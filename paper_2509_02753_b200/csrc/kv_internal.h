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
};
#ifdef __CUDACC__
__device__ __forceinline__ int div_g(const AttendArgs &a, int row) { return (int)a.g_div.div((uint32_t)row); }      // row / G
#endif
// rows of queries that share a key/value head, in the N dimension of mma.sync (kv_attend.cu)
cudaError_t launch_attend_rows(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);
size_t attend_part_floats(int w);          // per CTA of the grid
// prompts, on tcgen05 (kv_prompt.cu)
cudaError_t launch_attend_prompt(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches);
size_t prompt_part_floats(int w);          // per CTA, of which there is one per SM
size_t prompt_part_rows();

}  // namespace kv
}  // namespace lexi
