// Block tables, slots and positions of a step from the requests' lengths, one launch.
//
//   fresh_i = ceil((ctx_i + new_i)/P) - ceil(ctx_i/P),   cu = running sum of new,   first = running sum of fresh
//   token t of request r: position = ctx_r + t - cu_r; its page is entry position/P of the row, which is one of the
//   row's old entries or free_pages[first_r + position/P - ceil(ctx_r/P)]
//
// Bound by latency: a call moves 12 bytes a token, and lengths -> sums -> page -> slot are dependent steps.  Every CTA
// therefore makes the sums over all requests by itself (they come out of the L2; 8 bytes a request) and no CTA waits
// for another: one launch instead of a scan and a fill.  Tokens and fresh table entries find their request by a binary
// search of the sums in shared memory.
#include "kv_internal.h"

namespace lexi {
namespace kv {
namespace {

constexpr int kThreads = 256;
constexpr int kTokensPerCta = kThreads;      // 16384 tokens of 512 requests: 8.1 us with four tokens a thread

// last i with sum[i] <= x (sum[0] = 0 <= x); both sums are non-decreasing
__device__ __forceinline__ int find(const int32_t *sum, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sum[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kThreads) tables_kernel(TablesArgs a) {
    extern __shared__ int32_t sums[];
    int32_t *cu = sums, *first = sums + a.n + 1;
    __shared__ unsigned long long warp_sum[kThreads / 32];
    __shared__ unsigned long long carry_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int bad = 0;
    auto pages = [&](long long tokens) { return (tokens + (1 << a.page_shift) - 1) >> a.page_shift; };

    pdl_trigger();
    pdl_wait();

    // running sums of (fresh pages, new tokens), packed in one 64-bit word, 256 requests at a time
    unsigned long long carry = 0;
    for (int base = 0; base < a.n; base += kThreads) {
        const int i = base + tid;
        unsigned long long mine = 0;
        if (i < a.n) {
            int c = a.ctx[i], m = a.fresh_tokens[i];
            if (c < 0) { c = 0; bad |= MOE_KV_STATUS_BAD_INDEX; }
            if (m < 0) { m = 0; bad |= MOE_KV_STATUS_BAD_INDEX; }
            const long long total = (long long)c + m;
            const unsigned fresh = (unsigned)(pages(total) - pages(c));
            mine = ((unsigned long long)fresh << 32) | (unsigned)m;
            if (blockIdx.x == 0) a.kv_len[i] = total > INT32_MAX ? INT32_MAX : (int32_t)total;
        }
        unsigned long long inc = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long up = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += up;
        }
        if (lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        unsigned long long before = carry;
        for (int w = 0; w < warp; ++w) before += warp_sum[w];
        const unsigned long long at = before + inc - mine;
        if (i < a.n) { cu[i] = (int32_t)(uint32_t)at; first[i] = (int32_t)(at >> 32); }
        if (tid == kThreads - 1) carry_s = before + inc;
        __syncthreads();
        carry = carry_s;
    }
    if (tid == 0) { cu[a.n] = (int32_t)(uint32_t)carry; first[a.n] = (int32_t)(carry >> 32); }
    __syncthreads();
    const int n_new = cu[a.n], n_fresh = first[a.n];

    if (blockIdx.x == 0) {
        for (int i = tid; i <= a.n; i += kThreads) a.cu[i] = cu[i];
        if (tid == 0) {
            a.taken[0] = n_fresh;
            if (n_new > a.n_tokens) bad |= MOE_KV_STATUS_BAD_INDEX;
            if (n_fresh > a.n_free) bad |= MOE_KV_STATUS_NO_PAGES;
        }
    }

    const int stride = gridDim.x * kThreads;
    for (int t = blockIdx.x * kThreads + tid; t < a.n_tokens; t += stride) {
        int position = 0;
        int64_t slot = -1;
        if (t < n_new) {
            const int r = find(cu, a.n, t);
            const int c = max(a.ctx[r], 0);
            position = c + (t - cu[r]);
            const int col = position >> a.page_shift, held = (int)pages(c);
            int page = -1;
            if (col < held) {
                if (col < a.width) page = a.table[(int64_t)r * a.width + col];
            } else {
                const int f = first[r] + col - held;
                if (f < a.n_free && col < a.width) page = a.free_pages[f];
            }
            if (col >= a.width) bad |= MOE_KV_STATUS_NO_PAGES;
            if (page >= 0) slot = ((int64_t)page << a.page_shift) + (position & ((1 << a.page_shift) - 1));
        }
        a.position[t] = position;
        a.slot[t] = slot;
    }
    for (int f = blockIdx.x * kThreads + tid; f < n_fresh; f += stride) {
        const int r = find(first, a.n, f);
        const int held = (int)pages(max(a.ctx[r], 0));
        const long long col = (long long)held + f - first[r];
        if (col < a.width) a.table[(int64_t)r * a.width + col] = f < a.n_free ? a.free_pages[f] : -1;
        else bad |= MOE_KV_STATUS_NO_PAGES;
    }
    if (bad) atomicOr(a.status, bad);
}

}  // namespace

cudaError_t launch_tables(const TablesArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    const size_t smem = (size_t)2 * (a.n + 1) * sizeof(int32_t);      // at most 32 KB
    int grid = (a.n_tokens + kTokensPerCta - 1) / kTokensPerCta;
    grid = grid < 1 ? 1 : grid > 2 * sm_count ? 2 * sm_count : grid;
    ++*launches;
    return launch_chained(tables_kernel, dim3(grid), dim3(kThreads), smem, s, true, a);
}

}  // namespace kv
}  // namespace lexi
