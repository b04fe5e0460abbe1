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
    // running sums: new tokens, fresh pages, and the entries of the block table that these fill
    int32_t *cu = sums, *first = sums + a.n + 1, *entry = sums + 2 * (a.n + 1);
    __shared__ unsigned long long new_sum[kThreads / 32], fresh_sum[kThreads / 32], entry_sum[kThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int bad = 0;
    auto pages = [&](long long tokens) { return (tokens + (1 << a.page_shift) - 1) >> a.page_shift; };

    pdl_trigger();
    pdl_wait();

    // 256 requests at a time, in 64 bits: whatever the lengths are, sums do not wrap, and what does not fit 32 bits stays at
    // their largest value (a bad index in any case).  Entries lie inside the table, so there are at most n * width
    unsigned long long new_carry = 0, fresh_carry = 0, entry_carry = 0;
    auto low = [](unsigned long long x) { return x > INT32_MAX ? INT32_MAX : (int32_t)x; };
    for (int base = 0; base < a.n; base += kThreads) {
        const int i = base + tid;
        unsigned long long tokens = 0, fresh = 0, entries = 0;
        if (i < a.n) {
            int c = a.ctx[i], m = a.fresh_tokens[i];
            if (c < 0) { c = 0; bad |= MOE_KV_STATUS_BAD_INDEX; }
            if (m < 0) { m = 0; bad |= MOE_KV_STATUS_BAD_INDEX; }
            const long long total = (long long)c + m, held = pages(c), wanted = pages(total);
            tokens = (unsigned)m;
            fresh = (unsigned long long)(wanted - held);
            entries = (unsigned long long)(min(wanted, (long long)a.width) - min(held, (long long)a.width));
            if (entries < fresh) bad |= MOE_KV_STATUS_NO_PAGES;
            if (blockIdx.x == 0) a.kv_len[i] = low(total);
        }
        unsigned long long new_inc = tokens, fresh_inc = fresh, entry_inc = entries;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long x = __shfl_up_sync(0xffffffffu, new_inc, o), y = __shfl_up_sync(0xffffffffu, fresh_inc, o),
                                     z = __shfl_up_sync(0xffffffffu, entry_inc, o);
            if (lane >= o) { new_inc += x; fresh_inc += y; entry_inc += z; }
        }
        if (lane == 31) { new_sum[warp] = new_inc; fresh_sum[warp] = fresh_inc; entry_sum[warp] = entry_inc; }
        __syncthreads();
        unsigned long long new_before = new_carry, fresh_before = fresh_carry, entry_before = entry_carry;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w == warp) { new_before = new_carry; fresh_before = fresh_carry; entry_before = entry_carry; }
            new_carry += new_sum[w];
            fresh_carry += fresh_sum[w];
            entry_carry += entry_sum[w];
        }
        if (i < a.n) {
            cu[i] = low(new_before + new_inc - tokens);
            first[i] = low(fresh_before + fresh_inc - fresh);
            entry[i] = low(entry_before + entry_inc - entries);
        }
        __syncthreads();
    }
    if (tid == 0) { cu[a.n] = low(new_carry); first[a.n] = low(fresh_carry); entry[a.n] = low(entry_carry); }
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
            position = low((unsigned long long)c + (t - cu[r]));
            const int col = position >> a.page_shift, held = (int)pages(c);
            const long long f = (long long)first[r] + col - held;          // of the free list, if the page is a fresh one
            int page = -1;
            if (col >= a.width) {
                bad |= MOE_KV_STATUS_NO_PAGES;
            } else if (col < held || f < a.n_free) {
                page = col < held ? a.table[(int64_t)r * a.width + col] : a.free_pages[f];
                if (page < 0) bad |= MOE_KV_STATUS_BAD_INDEX;
            }
            if (page >= 0) slot = ((int64_t)page << a.page_shift) + (position & ((1 << a.page_shift) - 1));
        }
        a.position[t] = position;
        a.slot[t] = slot;
    }
    for (long long e = blockIdx.x * kThreads + tid; e < entry[a.n]; e += stride) {
        const int r = find(entry, a.n, (int)e);
        const long long in = e - entry[r], col = pages(max(a.ctx[r], 0)) + in, f = (long long)first[r] + in;
        if (col < a.width) a.table[(int64_t)r * a.width + col] = f < a.n_free ? a.free_pages[f] : -1;
    }
    if (bad) atomicOr(a.status, bad);
}

}  // namespace

cudaError_t launch_tables(const TablesArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    const size_t smem = (size_t)3 * (a.n + 1) * sizeof(int32_t);      // 48 KB for the most requests, besides the static sums
    if (smem > 40 * 1024) {
        const cudaError_t err = cudaFuncSetAttribute(tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (err != cudaSuccess) return err;
    }
    int grid = (a.n_tokens + kTokensPerCta - 1) / kTokensPerCta;
    grid = grid < 1 ? 1 : grid > 2 * sm_count ? 2 * sm_count : grid;
    ++*launches;
    return launch_chained(tables_kernel, dim3(grid), dim3(kThreads), smem, s, true, a);
}

}  // namespace kv
}  // namespace lexi
