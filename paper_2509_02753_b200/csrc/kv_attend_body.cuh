// Attention of few query rows over the 4-bit cache: single tokens, drafts, and every shape that kv_prompt.cu leaves.
//
//   o_i = sum_j w_ij v_j / sum_j w_ij,   w_ij = 2^(c q_i . k_j - m_i),   c = softmax_scale * k_scale * log2(e)
//
// in one pass over the keys with a running reference m_i.  The rows that share a key/value head - its query heads times
// the new tokens - are the N dimension (8 a tile) of mma.sync.m16n8k16, 16 keys are M, so a key's codes are converted
// once for all rows:
//   S^T[16 keys, 8 rows]  = K[16 keys, W] Q^T          A operand: key rows, converted e2m1 -> f16, times their scales
//   O^T[W, 8 rows]       += V^T[W, 16 keys] P^T        A operand: value columns; two keys' codes of a dimension are put
//                                                      into one byte, so that one conversion makes an operand register
// A value code times its scale has at most 6 significant bits: both operands are exact in f16.  Queries are scaled by a
// power of two per row: bf16 ones are exact in f16 too, fp32 ones are the sum of two f16 parts (22 bits) with products for
// both.  Weights are rounded to f16 for bf16 calls, each by at most 2^-11 where the output itself is rounded by up to 2^-8
// (errors against 64 bits 0.0016 to 0.0017 of the norm, as with weights in 32 bits; single outputs round the other way, 3e-4
// to 8e-4 of the norm), and are two f16 parts for fp32.  Denominators sum them as they are in fp32: the roundings of many
// keys are independent and average out.
//
// Bound by the cache's bytes (9/8 W a key and head for K and V together) as long as a key's conversion, about 1.5 lane
// operations an element, hides behind them; with several N tiles by mma.sync's rate.
//
// Work split: a stretch is what one (request, row block, key/value head) has to read, in blocks of 16 keys.  Where there
// are few stretches each is cut in equal pieces so that every CTA gets one; many short stretches are pieces themselves;
// otherwise the stretches stand in one line that is cut in equal shares, at places that need not be ends of stretches.
// A stretch in several pieces is joined by the last of them to arrive, which adds them in the order of the keys: equal
// calls give equal bits.  Lengths are read on the device; no host knows them.  Warps of a CTA take the blocks of a piece
// two at a time in turn, each with its own ring of bulk copies, and join once per piece.
//
// Five builds of the kernel, by what the rows of a stretch read (Reads below; kv_attend.cu, kv_attend_shared.cu,
// kv_attend_selected.cu):
//   Every   all keys of the request that the row's position and the window let it see
//   Prefix  "requests" are groups of requests and "keys" their shared prefix, which all rows of a group see whole; what
//           comes out is sums, references and denominators as they are, in fp32, of each piece of a stretch
//   Rest    the keys behind the shared prefix; what comes out, again, is sums.  The kernel starts while the one of the prefix
//           runs and shares the SMs with it; only one CTA waits for it, in the end, so that this kernel's end is both kernels'.
//           kv_attend_shared.cu joins the two
//   Listed  a token is a "request" of its own; its blocks are those of the pages listed for it and the head
//   Pieces  the same where stretches are few: all have as many blocks, which the host knows, so the pieces of one are the CTAs
//           of a cluster, which join through one another's shared memory
#pragma once

#include <float.h>

#include <algorithm>
#include <atomic>

#include "kv_codes.cuh"
#include "kv_internal.h"
#include "kv_ring.cuh"
#include "tc_ptx.cuh"

namespace lexi {
namespace kv {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kPair = 2;                       // blocks a warp handles per step
constexpr int kLeast = kWarps * kPair;         // blocks of a piece, at least: a step of every warp
constexpr int kEntry = 16;                     // what a stretch costs besides its blocks, in blocks: counted in the line
constexpr int kBrief = 32;                     // stretches of at most this many blocks are not cut
constexpr float kFloor = -FLT_MAX;             // reference of a row that has seen no key
// Weights are 2^(x - m + kHead + kSlack): m is kSlack above a score that was once the largest, and follows only when a
// score passes it; f16 holds weights up to 2^(kHead + kSlack) and down to 2^-24: one below 2^-20 of its row's largest is
// held in steps of 2^-30 of that
constexpr float kHead = 6.f, kSlack = 8.f;

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ float load_q(const float *p) { return *p; }
__device__ __forceinline__ float load_q(const __nv_bfloat16 *p) { return __bfloat162float(*p); }

template <int W, int NT, bool SPLIT>
struct Shape {
    static constexpr int kRows = 8 * NT;
    static constexpr int kStages = 2;
    static constexpr int kStageBytes = kPair * block_bytes(W);
    static constexpr int kRing = kWarps * kStages * kStageBytes;
    static constexpr int kSteps = W / 16;                     // k16 steps of the scores
    static constexpr int kTiles = W / 16;                     // m16 tiles of the output
    static constexpr int kQ = kRows * W * 2 * (SPLIT ? 2 : 1);
    static constexpr int kJoinTiles = NT >= 8 ? 1 : (kTiles < 8 / NT ? kTiles : 8 / NT);   // m16 tiles joined at a time: 32 KB
    static constexpr int kJoin = kWarps * kRows * kJoinTiles * 16 * 4;
    static_assert(kJoin <= kRing, "the join's buffer is the ring's");
    static constexpr int kRowsBytes = kRows * W * 4;          // a piece's sums, behind that buffer where the CTAs of a cluster join
    static constexpr bool kClusters = kJoin + kRowsBytes <= kRing;
    static constexpr int kSmem = kRing + kQ;                  // plus the line of requests
};

enum class Reads { Every, Prefix, Rest, Listed, Pieces };

template <typename T, int W, int NT, int MINB, Reads R>
__global__ void __launch_bounds__(kThreads, MINB) attend_rows_kernel(AttendArgs a) {
    constexpr bool SPLIT = sizeof(T) == 4;
    constexpr bool kPrefix = R == Reads::Prefix, kRest = R == Reads::Rest, kListed = R == Reads::Listed || R == Reads::Pieces, kPieces = R == Reads::Pieces;
    using S = Shape<W, NT, SPLIT>;
    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t *ring = smem, *q_s = smem + S::kRing;
    int64_t *line = reinterpret_cast<int64_t *>(smem + S::kSmem);      // [n + 1] running sum of blocks
    __shared__ __align__(8) uint64_t full[kWarps * S::kStages];
    __shared__ int32_t row_pos[S::kRows];          // position of a row's token, -1 for a row that is none
    __shared__ float row_scale[S::kRows];          // its factor from the product to the exponent
    __shared__ float2 join_ml[kWarps][S::kRows];   // reference and sum of each warp, then weight of each warp
    __shared__ float2 row_ml[S::kRows];
    __shared__ long long sum_s[kWarps];
    __shared__ int strips_s[kWarps], longest_s[kWarps], len_s[32], q0_s[32], nq_s[32];
    __shared__ int last_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, c = lane & 3;

    if (tid < kWarps * S::kStages) tc::mbar_init(smem_u32(&full[tid]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    // Rest starts once the prefix's kernel lets it, which it does behind its own wait: what came before both is complete
    if (!kPrefix) pdl_trigger();
    if (!kRest) pdl_wait();
    if (kPrefix) pdl_trigger();

    // ---- the line: for request i, row blocks * heads * visible blocks (at least one, which writes the zeros)
    const int page_tokens = kBlockTokens << a.page_shift;
    auto lengths = [&](int i, int &len, int &q0, int &nq) {
        const int64_t room = (int64_t)a.width * page_tokens;
        int i0 = i, i1 = i + 1;
        if (kPrefix) {
            i0 = a.groups[i];
            i1 = a.groups[i + 1];
            if (i0 < 0 || i1 < i0 || i1 > a.n_members) { atomicOr(a.status, MOE_KV_STATUS_BAD_INDEX); i0 = i1 = 0; }
        }
        len = max(a.kv_len[i], 0);
        q0 = a.cu[i0];
        nq = a.cu[i1] - q0;
        const bool bad_rows = q0 < 0 || nq < 0 || q0 > a.T - nq;
        if (bad_rows || len > room) atomicOr(a.status, MOE_KV_STATUS_BAD_INDEX);
        if (kPrefix && len == 0) nq = 0;          // nothing is shared: the other kernel does all of it
        if (bad_rows || (a.prompt_rows > 0 && nq * a.G > a.prompt_rows)) nq = 0;       // many rows: kv_prompt.cu's
        len = (int)min((int64_t)len, room);
    };
    // position of a row's token; of a prefix all rows see the last key
    auto position = [&](int len, int nq, int row) { return kPrefix ? len - 1 : len - nq + div_g(a, row); };
    // Rest: the first key, behind the prefix, which ends in front of the new tokens
    auto begins = [&](int i, int len, int nq) {
        const int s = a.start[i], most = max(len - nq, 0);
        if (s < 0 || s > most) atomicOr(a.status, MOE_KV_STATUS_BAD_INDEX);
        return min(max(s, 0), most);
    };
    // blocks that rows [row0, row1) of a request see: [0, sb) and [wb, nb)
    auto visible = [&](int begin, int len, int nq, int row0, int row1, int &sb, int &wb, int &nb) {
        if (kListed) {
            sb = wb = 0;
            nb = a.n_listed << a.page_shift;
            return;
        }
        const int p0 = position(len, nq, row0), p1 = position(len, nq, row1 - 1);
        nb = p1 < 0 ? 0 : p1 / kBlockTokens + 1;
        wb = kRest ? begin / kBlockTokens : !kPrefix && a.window > 0 ? max(p0 - a.window + 1, 0) / kBlockTokens : 0;
        wb = min(wb, nb);
        sb = R == Reads::Every && a.window > 0 ? min((int)(((int64_t)a.sinks + kBlockTokens - 1) / kBlockTokens), wb) : 0;
    };
    auto units_of = [&](int begin, int len, int nq, int row0) {
        int sb, wb, nb;
        visible(begin, len, nq, row0, min(row0 + S::kRows, nq * a.G), sb, wb, nb);
        return max(sb + nb - wb, 1);
    };

    // ---- how much there is: blocks, stretches, the longest stretch; then how it is cut:
    //   even   stretch by stretch, ceil(units/chunk) pieces each (one piece a CTA where there are few stretches; whole
    //          stretches, several a CTA, where all are brief)
    //   else   the line of all stretches, kEntry and their blocks each, `share` of it a CTA
    // A lane has a request; the row blocks of one with several are summed by the warp.  sum(chunk): chunk 0 counts blocks.
    auto sum = [&](int begin, int len, int nq, int chunk, int &strips, int &longest) {
        const int rows = nq * a.G, many = (rows + S::kRows - 1) / S::kRows;
        long long mine = 0;
        strips = many;
        longest = 0;
        if (many == 1) {
            const int u = units_of(begin, len, nq, 0);
            longest = u;
            mine = chunk ? (u + chunk - 1) / chunk : u + kEntry;
        }
        for (uint32_t todo = __ballot_sync(0xffffffffu, many > 1); todo; todo &= todo - 1) {
            const int src = __ffs(todo) - 1;
            const int l = __shfl_sync(0xffffffffu, len, src), q = __shfl_sync(0xffffffffu, nq, src), m = __shfl_sync(0xffffffffu, many, src);
            const int from = kRest ? __shfl_sync(0xffffffffu, begin, src) : 0;
            long long part = 0;
            int top = 0;
            for (int rb = lane; rb < m; rb += 32) {
                const int u = units_of(from, l, q, rb * S::kRows);
                top = max(top, u);
                part += chunk ? (u + chunk - 1) / chunk : u + kEntry;
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
            top = __reduce_max_sync(0xffffffffu, top);
            if (lane == src) { mine = part; longest = top; }
        }
        return mine * a.Hk;
    };
    bool few = false, even = false;
    int chunk = 0;
    long long share = 0, total = 0;
    const int grid = gridDim.x;
    // ceil(x / by), x >= 0: 32-bit division where x has no more
    auto div_up = [&](long long x, int by) { x += by - 1; return x >> 32 ? x / by : (long long)((uint32_t)x / (uint32_t)by); };
    auto choose = [&](long long blocks, long long stretches, int longest) {       // blocks without the entries
        few = 2 * stretches <= grid;
        even = few || longest <= kBrief;
        // few: sum of ceil(u/chunk) <= blocks/chunk + stretches <= grid
        chunk = few ? (int)max(div_up(blocks, max(grid - (int)stretches, 1)), (long long)kLeast) : even ? kBrief : 0;
        share = max(div_up(blocks + kEntry * stretches, grid), (long long)2 * kLeast);
    };
    // The usual step: up to 32 requests with one strip each.  Every warp does it for itself, in its lanes, without a barrier
    bool simple = false;
    const int strips_of = (a.G + S::kRows - 1) / S::kRows;          // Listed: row blocks of a token
    if constexpr (kListed) {
        // every stretch has the same blocks: no line
        const long long stretches = (long long)a.T * strips_of * a.Hk, units = (long long)a.n_listed << a.page_shift;
        choose(stretches * units, stretches, (int)units);
        if (kPieces) few = even = true;
        total = stretches * (kPieces ? a.cluster : even ? (units + chunk - 1) / chunk : units + kEntry);
        simple = true;
    } else if (a.n <= 32) {
        int len = 0, q0 = 0, nq = 0, begin = 0;
        if (lane < a.n) {
            lengths(lane, len, q0, nq);
            if (kRest) begin = begins(lane, len, nq);
        }
        const int rows = nq * a.G, u = rows > 0 ? units_of(begin, len, nq, 0) : 0;
        const uint32_t sum_u = __reduce_add_sync(0xffffffffu, (uint32_t)u);             // u <= 2^26
        simple = !__any_sync(0xffffffffu, rows > S::kRows) && ((unsigned long long)sum_u + 32 * kEntry) * a.Hk < (1ull << 30);
        if (simple) {
            choose((long long)sum_u * a.Hk, (long long)__popc(__ballot_sync(0xffffffffu, u > 0)) * a.Hk, (int)__reduce_max_sync(0xffffffffu, (uint32_t)u));
            const int weight = u == 0 ? 0 : (even ? (int)((uint32_t)(u + chunk - 1) / (uint32_t)chunk) : u + kEntry) * a.Hk;
            int inc = weight;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += up;
            }
            total = __shfl_sync(0xffffffffu, inc, 31);
            // all warps write the same
            if (lane < a.n) { line[lane] = inc - weight; len_s[lane] = len; q0_s[lane] = q0; nq_s[lane] = nq; }
            __syncwarp();
        }
    }
    // Any other: pass 0 counts, pass 1 weighs and lines up (one copy of the code: an instruction's first run costs more)
#pragma unroll 1
    for (int pass = simple ? 2 : 0; pass < 2; ++pass) {
        long long carry = 0, stretches = 0;
        int most = 0;
#pragma unroll 1
        for (int base = 0; base < a.n; base += kThreads) {
            const int i = base + tid;
            int len = 0, q0, nq = 0, begin = 0, strips, longest;
            if (i < a.n) {
                lengths(i, len, q0, nq);
                if (kRest) begin = begins(i, len, nq);
            }
            const long long mine = sum(begin, len, nq, chunk, strips, longest);
            stretches += strips;
            most = max(most, longest);
            long long inc = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long up = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += up;
            }
            if (lane == 31) sum_s[warp] = inc;
            __syncthreads();
            long long before = carry;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                if (w == warp) before = carry;
                carry += sum_s[w];
            }
            if (i < a.n) line[i] = before + inc - mine;
            __syncthreads();
        }
        total = carry;
        if (pass == 0) {
            stretches = __reduce_add_sync(0xffffffffu, (int)stretches);
            most = __reduce_max_sync(0xffffffffu, most);
            if (lane == 0) { strips_s[warp] = (int)stretches; longest_s[warp] = most; }
            __syncthreads();
            stretches = 0;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) { stretches += strips_s[w]; most = max(most, longest_s[w]); }
            stretches *= a.Hk;
            choose(total - kEntry * stretches, stretches, most);
            if (!even) break;               // the line of blocks is there already
        }
    }
    __syncthreads();          // the barriers are initialised, the line is there
    // even: pieces blockIdx.x, + gridDim.x, ...; else blocks [at, end) of the line
    long long at = even ? (long long)blockIdx.x : share * blockIdx.x;
    const long long end = even ? total : min(at + share, total);
    RingWaits<S::kStages> waits;          // of this warp's ring

    int req = 0, len = 0, q0 = 0, nq = 0, sb = 0, wb = 0, nb = 0, row0 = 0, row1 = 0, units = 0, head = -1, begin = 0;
    long long place = 0;         // where the stretch begins (even: its first piece)
    const int32_t *listed = nullptr;
    auto take = [&]() {
        if (simple) { len = len_s[req]; q0 = q0_s[req]; nq = nq_s[req]; }
        else lengths(req, len, q0, nq);
        if (kRest) begin = begins(req, len, nq);
    };
    auto shape = [&]() {
        row1 = min(row0 + S::kRows, nq * a.G);
        visible(begin, len, nq, row0, row1, sb, wb, nb);
        units = max(sb + nb - wb, 1);
    };
    // Listed: which request token q0 belongs to; its keys up to its own are those it may see.  A token of no request has no row
    auto take_token = [&]() {
        const Request r = find_request(a.cu, a.kv_len, a.n, q0, a.T, (int64_t)a.width * page_tokens, a.status, [](int cu, int) { return cu; });
        const bool here = q0 >= r.q0 && q0 - r.q0 < r.nq;
        req = min(r.i, a.n - 1);
        len = here ? max(r.len - r.nq + q0 - r.q0 + 1, 0) : 0;
        nq = here ? 1 : 0;
    };
    while (at < end) {
        // ---- which stretch `at` lies in: found, or the one behind the last piece's
        if constexpr (kListed) {
            const long long many = ((long long)a.n_listed << a.page_shift), weight = kPieces ? a.cluster : even ? (few ? (many + chunk - 1) / chunk : 1) : many + kEntry;
            const long long stretch = (at | weight) >> 31 ? at / weight : (long long)((uint32_t)at / (uint32_t)weight);
            place = stretch * weight;
            const int per = strips_of * a.Hk, in = (int)(stretch % per);
            q0 = (int)(stretch / per);
            row0 = in / a.Hk * S::kRows;
            head = in % a.Hk;
            units = (int)many;
            listed = a.listed + ((int64_t)q0 * a.Hk + head) * a.n_listed;
        } else if (even || head < 0) {
            int lo = 0, hi = a.n;
#pragma unroll 1
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (line[mid] <= at) lo = mid; else hi = mid;
            }
            long long from = line[lo];
            req = lo;
            take();
            if (even && !few) {              // every stretch is one piece
                const uint32_t x = (uint32_t)(at - from);
                row0 = (int)(x / (uint32_t)a.Hk) * S::kRows;
                head = (int)(x % (uint32_t)a.Hk);
                shape();
                place = at;
            } else {
#pragma unroll 1
                for (row0 = 0;; row0 += S::kRows) {
                    shape();
                    const int weight = even ? (units + chunk - 1) / chunk : units + kEntry;
                    const long long here = (long long)weight * a.Hk;
                    if (at < from + here) {
                        head = (int)((uint32_t)(at - from) / (uint32_t)weight);
                        place = from + (long long)head * weight;
                        break;
                    }
                    from += here;
                }
            }
        } else {
            place = at;
            if (++head == a.Hk) {
                head = 0;
                row0 += S::kRows;
#pragma unroll 1
                while (row0 >= nq * a.G) { ++req; take(); row0 = 0; }          // the line goes on, so there is a request with rows
                shape();
            }
        }
        // blocks [first, last) of the stretch are this piece; cta0..cta1 have its pieces
        const int within = (int)(at - place);
        int first, last, cta0, cta1;
        if (even) {
            const int weight = kPieces ? a.cluster : few ? (units + chunk - 1) / chunk : 1;
            const int each = units / weight, rest = units - each * weight;          // `each` blocks, the first `rest` pieces one more
            first = within * each + min(within, rest);
            last = first + each + (within < rest);
            cta0 = (int)blockIdx.x - within;
            cta1 = cta0 + weight - 1;
            at += gridDim.x;
        } else {
            const long long block0 = place + kEntry;
            first = max(within - kEntry, 0);
            last = (int)min((long long)units, end - block0);
            at = block0 + units;                    // the next stretch
            if (last <= first) continue;
            const bool all = first == 0 && last == units;
            cta0 = all ? (int)blockIdx.x : (int)(block0 / share);
            cta1 = all ? (int)blockIdx.x : (int)((block0 + units - 1) / share);
        }
        // Listed: pages of this warp's first steps, asked for before the token's request is looked up
        auto page_of = [&](int from) {
            const int u = first + (warp + (from + (lane >> 1)) * kWarps) * kPair + (lane & 1);
            return u < last ? listed[u >> a.page_shift] : -1;
        };
        int page_now = 0, page_then = 0;
        if constexpr (kListed) {
            page_now = page_of(0);
            page_then = page_of(16);
            take_token();
            shape();
        }
        const int present = sb + nb - wb;
        const int b1 = min(last, present);             // blocks [first, b1) of the stretch are loaded

        // ---- queries: a warp a row, lane l has dimensions [l W/32, (l+1) W/32).  Asked for before the pages are waited for
        constexpr int kPer = W / 32, kMine = S::kRows / kWarps;
        float q_raw[kMine][kPer];
#pragma unroll
        for (int x = 0; x < kMine; ++x) {
            const int row = row0 + warp + x * kWarps, tok = div_g(a, row);
            const bool real = row < row1;
            const T *src = (const T *)a.q.p + (int64_t)(q0 + (real ? tok : 0)) * a.q.ts + (int64_t)(head * a.G + (real ? row - tok * a.G : 0)) * a.q.hs;
#pragma unroll
            for (int i = 0; i < kPer; ++i) q_raw[x][i] = real && lane * kPer + i < a.D ? load_q(src + lane * kPer + i) : 0.f;
        }

        // ---- this warp's blocks: the first copies start before the queries are read
        const int32_t *table = a.table + (int64_t)(kPrefix ? a.groups[req] : req) * a.width;
        const uint32_t my_ring = smem_u32(ring) + warp * S::kStages * S::kStageBytes, my_bar = smem_u32(&full[warp * S::kStages]);
        const uint8_t *my_ring_p = ring + warp * S::kStages * S::kStageBytes;
        const int steps = b1 > first ? (b1 - first + kPair - 1) / kPair : 0;
        const int mine = steps > warp ? (steps - warp + kWarps - 1) / kWarps : 0;
        auto block_at = [&](int u) { return u < sb ? u : wb + u - sb; };
        // 16 steps at a time: lane l finds the cache block that is block l%2 of step (from + l/2); -1: none
        auto find_blocks = [&](int from, int page, int &b) {
            const int k = from + (lane >> 1), u = first + (warp + k * kWarps) * kPair + (lane & 1);
            b = 0;
            if (k >= mine || u >= b1 || (kListed && nq == 0)) return -1;          // the list of a token of no request says nothing
            b = block_at(u);
            if (kListed) {
                if (page < 0 || page >= a.width) {
                    if (page != -1) atomicOr(a.status, MOE_KV_STATUS_BAD_INDEX);
                    return -1;
                }
                b = (page << a.page_shift) + (u & ((1 << a.page_shift) - 1));
                if (b * kBlockTokens >= len) return -1;          // no key that the token sees
            }
            const int pg = table[b >> a.page_shift];
            if (pg < 0 || pg >= a.n_pages) { atomicOr(a.status, MOE_KV_STATUS_BAD_INDEX); return -1; }
            return ((pg * a.Hk + head) << a.page_shift) + (b & ((1 << a.page_shift) - 1));
        };
        int now_at, then_at;          // which blocks of the request they are
        int now = find_blocks(0, page_now, now_at), then = find_blocks(16, page_then, then_at);
        uint32_t has_now = __ballot_sync(0xffffffffu, now >= 0), has_then = __ballot_sync(0xffffffffu, then >= 0);
        // copies of step (from + d), d < 32: by the two lanes that found its blocks
        auto issue = [&](int d, int stage) {
            const bool later = d >= 16;
            const uint32_t two = ((later ? has_then : has_now) >> (2 * (d & 15))) & 3u;
            const uint32_t bar = my_bar + 8 * stage;
            if (lane == 0) tc::mbar_expect_tx(bar, (uint32_t)__popc(two) * block_bytes(W));
            __syncwarp();
            const int blk = later ? then : now;
            if ((lane >> 1) == (d & 15) && blk >= 0)
                bulk_load(my_ring + stage * S::kStageBytes + (lane & 1) * block_bytes(W), a.cache + (int64_t)blk * block_bytes(W), block_bytes(W), bar);
        };
        for (int k = 0; k < S::kStages && k < mine && !waits.dead; ++k) issue(k, k);

        // ---- queries as operand fragments: [N tile][two k16 steps][lane] 16 bytes
#pragma unroll
        for (int x = 0; x < kMine; ++x) {
            const int n = warp + x * kWarps, row = row0 + n;
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) top = fmaxf(top, fabsf(q_raw[x][i]));
#pragma unroll
            for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const int e = row_exponent(top);
            const float up = power2(10 - e);
            if (lane == 0) {
                row_pos[n] = row < row1 ? position(len, nq, row) : -1;
                row_scale[n] = a.score_scale * power2(e - 10);
            }
#pragma unroll
            for (int i = 0; i < kPer; i += 2) {
                const int d = lane * kPer + i;
                // thread c of a fragment has dimensions [c W/4, (c+1) W/4) of row r, four for each k16 step
                const int fc = d / (W / 4), in = d % (W / 4), step = in / 4, part = (in % 4) / 2;
                uint32_t *dst = reinterpret_cast<uint32_t *>(q_s) + ((((n >> 3) * (S::kSteps / 2) + step / 2) * 32 + (n & 7) * 4 + fc) * 4 + (step & 1) * 2 + part);
                const float u = q_raw[x][i] * up, w = q_raw[x][i + 1] * up;
                const uint32_t h = pack2(u, w);
                *dst = h;
                if (SPLIT) {
                    const float2 f = unpack2(h);
                    dst[S::kRows * W / 2] = pack2(u - f.x, w - f.y);
                }
            }
        }
        __syncthreads();

        constexpr bool kHoldQ = NT == 1 && !SPLIT && W <= 128;         // 8 or 16 registers
        uint4 q_r[kHoldQ ? S::kSteps / 2 : 1];
        if (kHoldQ) {
#pragma unroll
            for (int i = 0; i < S::kSteps / 2; ++i) q_r[i] = *reinterpret_cast<const uint4 *>(q_s + (i * 32 + lane) * 16);
        }
        float m[NT][2], l[NT][2], o[S::kTiles][NT][4], f[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                m[t][j] = kFloor; l[t][j] = 0.f;
                f[t][j] = row_scale[t * 8 + 2 * c + j];
            }
        // blocks of the stretch that every row sees whole: [0, sink_clear) and [clear0, clear1)
        const int p_first = position(len, nq, row0), p_last = position(len, nq, row1 - 1);
        const int whole1 = max(p_first + 1, 0) / kBlockTokens;                                                    // blocks below are complete
        const int whole0 = kRest ? (begin + kBlockTokens - 1) / kBlockTokens :
                           R == Reads::Every && a.window > 0 ? (max(p_last - a.window + 1, 0) + kBlockTokens - 1) / kBlockTokens : 0;   // and from here inside the window
        const int sink_clear = min(sb, min(a.sinks / kBlockTokens, whole1));
        const int clear0 = max(whole0 - wb, 0) + sb, clear1 = whole1 - wb + sb;
#pragma unroll
        for (int t = 0; t < S::kTiles; ++t)
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[t][u][j] = 0.f;

        int from = 0;
        for (int k = 0; k < mine; ++k) {
            if (k - from == 16) {
                from = k;
                now = then; has_now = has_then; now_at = then_at;
                then = find_blocks(from + 16, kListed ? page_of(from + 16) : 0, then_at);
                has_then = __ballot_sync(0xffffffffu, then >= 0);
            }
            const int stage = k % S::kStages;
            // a copy that never ends: nothing more is waited for, the status word tells
            if (!waits.arrived(k, mine, [&](int of, uint32_t parity) { return (bool)__all_sync(0xffffffffu, tc::mbar_wait(my_bar + 8 * of, parity, a.status)); })) break;
            const uint8_t *buf = my_ring_p + stage * S::kStageBytes;
            const int u0 = first + (warp + k * kWarps) * kPair;
            const uint32_t has = (has_now >> (2 * (k - from))) & 3u;
            const bool two = has & 2u;

            // ---- scores of 32 keys: s[block][N tile]
            float s[kPair][NT][4];
#pragma unroll
            for (int b = 0; b < kPair; ++b) {
                constexpr bool kTwo = NT == 1;      // two chains of sums: half the latency of dependent products (more tiles are chains of their own)
                float s2[kTwo ? NT : 1][4];
                if (b == 1 && !two) {
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[b][t][j] = 0.f;
                    continue;
                }
                const uint8_t *blk = buf + b * block_bytes(W);
                constexpr int kBytes = W / 8;               // code bytes of a thread's share of a key
                constexpr int kGroups = W / 64;             // scales of it
                uint32_t sc[2][kGroups];                    // f16 pairs (s, s) of keys r and r + 8
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint8_t *p = blk + k_scales_at(W) + (r + 8 * half) * (W / 16) + c * kGroups;
                    if (W == 64) {
                        sc[half][0] = scales2((uint32_t)*p * 0x101u);
                    } else if (W == 128) {
                        const uint32_t two_s = scales2(*reinterpret_cast<const uint16_t *>(p));
                        sc[half][0] = __byte_perm(two_s, 0, 0x1010);
                        sc[half][kGroups > 1 ? 1 : 0] = __byte_perm(two_s, 0, 0x3232);
                    } else {
                        const uint32_t four = *reinterpret_cast<const uint32_t *>(p);
                        const uint32_t x = scales2(four & 0xffffu), y = scales2(four >> 16);
                        sc[half][0] = __byte_perm(x, 0, 0x1010);
                        sc[half][1 % kGroups] = __byte_perm(x, 0, 0x3232);
                        sc[half][2 % kGroups] = __byte_perm(y, 0, 0x1010);
                        sc[half][3 % kGroups] = __byte_perm(y, 0, 0x3232);
                    }
                }
                // 8 bytes of codes a group: two words, 4 k16 steps
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    const uint2 w0 = *reinterpret_cast<const uint2 *>(blk + r * (W / 2) + c * kBytes + g * 8);
                    const uint2 w1 = *reinterpret_cast<const uint2 *>(blk + (r + 8) * (W / 2) + c * kBytes + g * 8);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t h0[4], h1[4];
                        codes4(i ? w0.y : w0.x, h0);
                        codes4(i ? w1.y : w1.x, h1);
#pragma unroll
                        for (int j = 0; j < 4; ++j) { h0[j] = mul2(h0[j], sc[0][g]); h1[j] = mul2(h1[j], sc[1][g]); }
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            const uint4 q = kHoldQ ? q_r[g * 2 + i] : *reinterpret_cast<const uint4 *>(q_s + ((t * (S::kSteps / 2) + g * 2 + i) * 32 + lane) * 16);
                            if (g + i == 0) mma_first(s[b][t], h0[0], h1[0], h0[1], h1[1], q.x, q.y);
                            else mma(s[b][t], h0[0], h1[0], h0[1], h1[1], q.x, q.y);
                            if (kTwo && g + i == 0) mma_first(s2[kTwo ? t : 0], h0[2], h1[2], h0[3], h1[3], q.z, q.w);
                            else mma(kTwo ? s2[kTwo ? t : 0] : s[b][t], h0[2], h1[2], h0[3], h1[3], q.z, q.w);
                            if (SPLIT) {
                                const uint4 ql = *reinterpret_cast<const uint4 *>(q_s + S::kRows * W * 2 + ((t * (S::kSteps / 2) + g * 2 + i) * 32 + lane) * 16);
                                mma(s[b][t], h0[0], h1[0], h0[1], h1[1], ql.x, ql.y);
                                mma(kTwo ? s2[kTwo ? t : 0] : s[b][t], h0[2], h1[2], h0[3], h1[3], ql.z, ql.w);
                            }
                        }
                    }
                }
                if (kTwo) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[b][0][j] += s2[0][j];
                }
            }

            // ---- exponents, masks, the reference
            bool over = false, clear[kPair];
            int valid[kPair];         // keys of the block that lie in the cache: the rest of its value scales count as 0
#pragma unroll
            for (int b = 0; b < kPair; ++b) {
                const int u = u0 + b;
                const int which = kListed ? __shfl_sync(0xffffffffu, now_at, 2 * (k - from) + b) : 0;
                clear[b] = (has >> b & 1u) && (kListed ? which < whole1 : u < sink_clear || (u >= clear0 && u < clear1));
                valid[b] = kBlockTokens;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[b][t][j] *= f[t][j & 1];
                if (!clear[b]) {
                    const bool here = has >> b & 1u;
                    const int key = (kListed ? which : block_at(u)) * kBlockTokens + r;
                    valid[b] = len - key + r;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            // the query's position less the key's, for keys r and r + 8
                            const int back = row_pos[t * 8 + 2 * c + j] - key;
                            constexpr bool kWindow = R == Reads::Every;
                            const bool see0 = here && back >= 0 && (!kWindow || a.window <= 0 || back < a.window || key < a.sinks) && (!kRest || key >= begin);
                            const bool see8 = here && back >= 8 && (!kWindow || a.window <= 0 || back - 8 < a.window || key + 8 < a.sinks) && (!kRest || key + 8 >= begin);
                            s[b][t][j] = see0 ? s[b][t][j] : -INFINITY;
                            s[b][t][j + 2] = see8 ? s[b][t][j + 2] : -INFINITY;
                        }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) over = over || s[b][t][j] > m[t][j & 1];
            }
            if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float top = kFloor;
#pragma unroll
                        for (int b = 0; b < kPair; ++b) top = fmaxf(top, fmaxf(s[b][t][j], s[b][t][j + 2]));
                        for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                        top = fmaxf(m[t][j], top + kSlack);
                        const float scale = m[t][j] == top ? 1.f : ex2(m[t][j] - top);      // 0 for a row that had seen no key
                        m[t][j] = top;
                        l[t][j] *= scale;
#pragma unroll
                        for (int i = 0; i < S::kTiles; ++i) { o[i][t][j] *= scale; o[i][t][j + 2] *= scale; }
                    }
            }

            // ---- weights and values
#pragma unroll
            for (int b = 0; b < kPair; ++b) {
                if (!(has >> b & 1u)) continue;
                const uint8_t *blk = buf + b * block_bytes(W);
                uint32_t p0[NT], p1[NT], q0l[NT], q1l[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        w[j] = ex2(s[b][t][j] - m[t][j & 1] + (kHead + kSlack));
                        l[t][j & 1] += w[j];
                    }
                    const uint32_t h0 = pack2(w[0], w[1]), h1 = pack2(w[2], w[3]);
                    p0[t] = transpose8(h0);
                    p1[t] = transpose8(h1);
                    if (SPLIT) {
                        const float2 f0 = unpack2(h0), f1 = unpack2(h1);
                        q0l[t] = transpose8(pack2(w[0] - f0.x, w[1] - f0.y));
                        q1l[t] = transpose8(pack2(w[2] - f1.x, w[3] - f1.y));
                    }
                }
                const uint8_t *codes = blk + v_codes_at(W) + r * W;
                constexpr int vb = W / 16;
                constexpr int kWords = vb / 4;              // words of a key's share: 1, 2, 4
                uint32_t ka[kWords], kb[kWords], kc[kWords], kd[kWords];      // keys 2c, 2c+1, 2c+8, 2c+9
                const int turned = v_turn(W, r);
                if (W == 64) {
                    const uint2 x = *reinterpret_cast<const uint2 *>(codes + ((8 * c) ^ turned)), y = *reinterpret_cast<const uint2 *>(codes + ((32 + 8 * c) ^ turned));
                    ka[0] = x.x; kb[0] = x.y; kc[0] = y.x; kd[0] = y.y;
                } else if (W == 128) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(codes + ((16 * c) ^ turned)), y = *reinterpret_cast<const uint4 *>(codes + ((64 + 16 * c) ^ turned));
                    ka[0] = x.x; ka[1 % kWords] = x.y; kb[0] = x.z; kb[1 % kWords] = x.w;
                    kc[0] = y.x; kc[1 % kWords] = y.y; kd[0] = y.z; kd[1 % kWords] = y.w;
                } else {
                    const uint4 x = *reinterpret_cast<const uint4 *>(codes + ((32 * c) ^ turned)), y = *reinterpret_cast<const uint4 *>(codes + ((32 * c + 16) ^ turned));
                    const uint4 z = *reinterpret_cast<const uint4 *>(codes + ((128 + 32 * c) ^ turned)), u = *reinterpret_cast<const uint4 *>(codes + ((128 + 32 * c + 16) ^ turned));
                    ka[0] = x.x; ka[1 % kWords] = x.y; ka[2 % kWords] = x.z; ka[3 % kWords] = x.w;
                    kb[0] = y.x; kb[1 % kWords] = y.y; kb[2 % kWords] = y.z; kb[3 % kWords] = y.w;
                    kc[0] = z.x; kc[1 % kWords] = z.y; kc[2 % kWords] = z.z; kc[3 % kWords] = z.w;
                    kd[0] = u.x; kd[1 % kWords] = u.y; kd[2 % kWords] = u.z; kd[3 % kWords] = u.w;
                }
                // scales of the key pairs (2c, 2c+1) and (2c+8, 2c+9); a key behind the cached ones has none, whatever its bytes
                constexpr int kG = W == 256 ? 2 : 1;
                uint32_t sa[kG], sb2[kG];
#pragma unroll
                for (int g = 0; g < kG; ++g) {
                    const int grp = W == 64 ? r >> 1 : W == 128 ? r : 2 * r + g;
                    const uint8_t *p = blk + v_scales_at(W) + grp * kBlockTokens + 2 * c;
                    sa[g] = scales2(*reinterpret_cast<const uint16_t *>(p));
                    sb2[g] = scales2(*reinterpret_cast<const uint16_t *>(p + 8));
                    if (!clear[b] && valid[b] < kBlockTokens) {
                        const int x = valid[b] - 2 * c;
                        sa[g] = x >= 2 ? sa[g] : x == 1 ? sa[g] & 0xffffu : 0u;
                        sb2[g] = x >= 10 ? sb2[g] : x == 9 ? sb2[g] & 0xffffu : 0u;
                    }
                }
#pragma unroll
                for (int w = 0; w < kWords; ++w) {
                    constexpr uint32_t L = 0x0f0f0f0fu;
                    uint32_t a0[4], a1[4], a2[4], a3[4];
                    codes4((ka[w] & L) | ((kb[w] & L) << 4), a0);
                    codes4(((ka[w] >> 4) & L) | (kb[w] & ~L), a1);
                    codes4((kc[w] & L) | ((kd[w] & L) << 4), a2);
                    codes4(((kc[w] >> 4) & L) | (kd[w] & ~L), a3);
                    const int g = W == 256 ? w >> 1 : 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        a0[i] = mul2(a0[i], sa[g % kG]); a1[i] = mul2(a1[i], sa[g % kG]);
                        a2[i] = mul2(a2[i], sb2[g % kG]); a3[i] = mul2(a3[i], sb2[g % kG]);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            mma(o[w * 4 + i][t], a0[i], a1[i], a2[i], a3[i], p0[t], p1[t]);
                            if (SPLIT) mma(o[w * 4 + i][t], a0[i], a1[i], a2[i], a3[i], q0l[t], q1l[t]);
                        }
                    }
                }
            }
            __syncwarp();
            if (k + S::kStages < mine) issue(k + S::kStages - from, stage);
        }

        // ---- join the warps: o[t][u] holds rows 8u + 2c + {0, 1}, dimensions (W/8) r + 2t + {0, 1}
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                for (int x = 4; x < 32; x <<= 1) l[t][j] += __shfl_xor_sync(0xffffffffu, l[t][j], x);
                if (r == 0) join_ml[warp][t * 8 + 2 * c + j] = make_float2(m[t][j], l[t][j]);
            }
        __syncthreads();       // every warp is done with its ring too
        if (tid < S::kRows) {
            float top = kFloor, sum = 0.f;
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, join_ml[w][tid].x);
            for (int w = 0; w < kWarps; ++w) {
                const float2 ml = join_ml[w][tid];
                const float k = ml.x == top ? 1.f : ex2(ml.x - top);
                sum += k * ml.y;
                join_ml[w][tid].x = k;
            }
            row_ml[tid] = make_float2(top, sum);
        }
        __syncthreads();
        float k_mine[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) k_mine[t][j] = join_ml[warp][t * 8 + 2 * c + j].x;

        const bool whole = first == 0 && last == units;
        // a CTA's first piece may be the end of a stretch, its last piece the beginning of one
        const int my_slot = blockIdx.x * 2 + (first == 0 ? 1 : 0);
        float *part = kPieces ? reinterpret_cast<float *>(ring + S::kJoin) : a.part + (int64_t)my_slot * S::kRows * W;
        float2 *part_ml = a.part_ml + (int64_t)my_slot * S::kRows;
        float2 *buf = reinterpret_cast<float2 *>(ring);
        // row n of the stretch, dimensions d and d + 1: sums v with reference `top` and denominator `sum`
        auto put = [&](int n, int d, float2 v, float top, float sum) {
            const int row = row0 + n;
            if (row >= row1 || d >= a.D) return;
            const int tok = div_g(a, row);
            const int64_t at_row = (int64_t)(q0 + tok) * a.H + head * a.G + row - tok * a.G;
            if (kPrefix) {
                *reinterpret_cast<float2 *>(a.o_part + at_row * W + d) = v;
                if (d == 0) {
                    a.o_ml[at_row] = make_float2(top, sum);
                    a.o_pieces[at_row] = make_int4(-1, 1, 0, 0);
                }
                return;
            }
            if (kRest && begin > 0) {
                *reinterpret_cast<float2 *>(a.own_part + at_row * W + d) = v;
                if (d == 0) a.own_ml[at_row] = make_float2(top, sum);
                return;
            }
            const float k = sum > 0.f || sum != sum ? a.v_scale / sum : 0.f;
            T *dst = (T *)a.out + at_row * a.D + d;
            if (SPLIT) *reinterpret_cast<float2 *>(dst) = make_float2(v.x * k, v.y * k);
            else *reinterpret_cast<__nv_bfloat162 *>(dst) = __floats2bfloat162_rn(v.x * k, v.y * k);
        };
#pragma unroll
        for (int t0 = 0; t0 < S::kTiles; t0 += S::kJoinTiles) {
            if (t0) __syncthreads();
#pragma unroll
            for (int tl = 0; tl < S::kJoinTiles; ++tl)
#pragma unroll
                for (int u = 0; u < NT; ++u)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        buf[((warp * S::kRows + 8 * u + 2 * c + j) * S::kJoinTiles + tl) * 8 + r] =
                            make_float2(o[t0 + tl][u][j] * k_mine[u][j], o[t0 + tl][u][j + 2] * k_mine[u][j]);
            __syncthreads();
#pragma unroll 1
            for (int e = tid; e < S::kRows * S::kJoinTiles * 8; e += kThreads) {
                const int n = e / (S::kJoinTiles * 8), tl = e / 8 % S::kJoinTiles, rr = e % 8;
                float2 v = make_float2(0.f, 0.f);
                for (int w = 0; w < kWarps; ++w) {
                    const float2 x = buf[w * S::kRows * S::kJoinTiles * 8 + e];
                    v.x += x.x; v.y += x.y;
                }
                const int d = rr * (W / 8) + 2 * (t0 + tl);
                if (whole) {
                    put(n, d, v, row_ml[n].x, row_ml[n].y);
                } else {
                    *reinterpret_cast<float2 *>(part + (int64_t)n * W + d) = v;
                }
            }
        }
        if (kPrefix && !whole) {
            // join_kernel adds them: where the row's pieces are
            if (tid < S::kRows) {
                part_ml[tid] = row_ml[tid];
                const int row = row0 + tid;
                if (first == 0 && row < row1) {
                    const int tok = div_g(a, row);
                    a.o_pieces[(int64_t)(q0 + tok) * a.H + head * a.G + row - tok * a.G] = make_int4(cta0, cta1 + 1 - cta0, tid, 0);
                }
            }
        } else if (kPieces) {
            // a share of the rows' dimensions from every CTA's shared memory, in the order of the keys; no CTA leaves before all are done
            asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
            const uint32_t part_at = smem_u32(part), ml_at = smem_u32(row_ml);
#pragma unroll 1
            for (int e = within * kThreads + tid; e < S::kRows * W / 4; e += a.cluster * kThreads) {
                const int n = e / (W / 4), d = e % (W / 4) * 4;
                float top = kFloor, sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
                for (int y = 0; y < a.cluster; ++y) {
                    uint32_t ml_of, part_of;
                    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ml_of) : "r"(ml_at + 8u * n), "r"(y));
                    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(part_of) : "r"(part_at + 16u * e), "r"(y));
                    float m_y, l_y, z[4];
                    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(m_y), "=f"(l_y) : "r"(ml_of) : "memory");
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(z[0]), "=f"(z[1]), "=f"(z[2]), "=f"(z[3]) : "r"(part_of) : "memory");
                    const float to = fmaxf(top, m_y), old = top == to ? 1.f : ex2(top - to), k = m_y == to ? 1.f : ex2(m_y - to);
                    sum = sum * old + l_y * k;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = v[i] * old + z[i] * k;
                    top = to;
                }
                put(n, d, make_float2(v[0], v[1]), top, sum);
                put(n, d + 2, make_float2(v[2], v[3]), top, sum);
            }
            asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        } else if (!whole) {
            if (tid < S::kRows) part_ml[tid] = row_ml[tid];
            __syncthreads();
            if (tid == 0) {
                int before;                         // releases all of the CTA's writes above, by way of the barrier
                asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(a.arrived + cta0) : "memory");
                last_s = before == cta1 - cta0;
                if (last_s) a.arrived[cta0] = 0;             // ready for the next call
            }
            __syncthreads();
            if (last_s) {
                // the pieces in the order of the keys, as many at a time as the ring holds: their latency is paid once for all
                // of these (loaded by the threads that add them, four at a time, 16 pieces took 8 us)
                constexpr int kBytes = S::kRows * W * 4, kAtOnce = S::kRing / (kBytes + S::kRows * 8);
                static_assert(kAtOnce >= 1, "");
                float2 *ml_s = reinterpret_cast<float2 *>(ring + kAtOnce * kBytes);
                constexpr int kOwn = S::kRows * W / 4 / kThreads;              // a thread's quads of dimensions
                float top[kOwn], sum[kOwn], v[kOwn][4];
#pragma unroll
                for (int x = 0; x < kOwn; ++x) { top[x] = kFloor; sum[x] = 0.f; v[x][0] = v[x][1] = v[x][2] = v[x][3] = 0.f; }
#pragma unroll 1
                for (int b0 = cta0; b0 <= cta1; b0 += kAtOnce) {
                    const int m = min(kAtOnce, cta1 + 1 - b0);
#pragma unroll 1
                    for (int e = tid; e < m * (kBytes / 16); e += kThreads) {
                        const int y = e / (kBytes / 16), b = b0 + y;
                        const float *src = a.part + (int64_t)(b * 2 + (b == cta0)) * S::kRows * W + (e % (kBytes / 16)) * 4;
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(ring) + e * 16), "l"(src) : "memory");
                    }
#pragma unroll 1
                    for (int e = tid; e < m * S::kRows; e += kThreads) {
                        const int b = b0 + e / S::kRows;
                        ml_s[e] = __ldcg(&a.part_ml[(int64_t)(b * 2 + (b == cta0)) * S::kRows + e % S::kRows]);
                    }
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    __syncthreads();
#pragma unroll 1
                    for (int y = 0; y < m; ++y)
#pragma unroll
                        for (int x = 0; x < kOwn; ++x) {
                            const int e = tid + x * kThreads;
                            const float2 ml = ml_s[y * S::kRows + e / (W / 4)];
                            const float4 z = *reinterpret_cast<const float4 *>(ring + y * kBytes + e * 16);
                            const float to = fmaxf(top[x], ml.x), old = top[x] == to ? 1.f : ex2(top[x] - to), k = ml.x == to ? 1.f : ex2(ml.x - to);
                            sum[x] = sum[x] * old + ml.y * k;
                            v[x][0] = v[x][0] * old + z.x * k; v[x][1] = v[x][1] * old + z.y * k;
                            v[x][2] = v[x][2] * old + z.z * k; v[x][3] = v[x][3] * old + z.w * k;
                            top[x] = to;
                        }
                    __syncthreads();
                }
#pragma unroll
                for (int x = 0; x < kOwn; ++x) {
                    const int e = tid + x * kThreads, n = e / (W / 4), d = e % (W / 4) * 4;
                    put(n, d, make_float2(v[x][0], v[x][1]), top[x], sum[x]);
                    put(n, d + 2, make_float2(v[x][2], v[x][3]), top[x], sum[x]);
                }
            }
        }
        // the ring and the rows' tables are the next piece's; its copies come after this piece's plain accesses
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
    }
    if (kRest && blockIdx.x == 0) pdl_wait();          // that this kernel is complete means that the prefix's is
}

template <typename T, int W, int NT, int MINB, Reads R>
cudaError_t launch(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    using S = Shape<W, NT, sizeof(T) == 4>;
    auto k = attend_rows_kernel<T, W, NT, MINB, R>;
    // CTAs an SM holds, for up to kFew requests and for the most, asked once per device
    constexpr int kFew = 256;
    static std::atomic<int> held[64][2];
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    const bool many = R != Reads::Listed && a.n > kFew;
    const int smem = S::kSmem + 8 * ((many ? kMaxRequests : kFew) + 1);
    int per_sm = dev < 64 ? held[dev][many].load() : 0;
    if (per_sm == 0) {
        err = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem + 8 * (kMaxRequests + 1));
        if (err != cudaSuccess) return err;
        err = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, k, kThreads, smem);
        if (err != cudaSuccess) return err;
        if (per_sm < 1) return cudaErrorInvalidConfiguration;
        if (dev < 64) held[dev][many].store(per_sm);
    }
    // no more CTAs than pieces: what the block tables can hold bounds the blocks
    const long long strips = (R == Reads::Listed ? (long long)a.T * ((a.G + S::kRows - 1) / S::kRows) : (long long)a.T * a.G / S::kRows + a.n) * a.Hk;
    const double most = (double)strips * ((double)((long long)(R == Reads::Listed ? a.n_listed : a.width) << a.page_shift) / kLeast + 1);
    long long grid = (long long)sm_count * per_sm;
    const long long pieces = most < 1e9 ? (long long)most : grid;
    grid = pieces < grid ? pieces : grid;
    grid = grid > a.max_ctas ? a.max_ctas : grid < 1 ? 1 : grid;
    ++*launches;
    if constexpr (R == Reads::Listed && S::kClusters) {
        // Few stretches: as many pieces of one as there are CTAs for, each a step of every warp at least, up to the eight that a
        // cluster may have; where more would leave a piece below kLong blocks they join through the L2.  In us, so / in clusters:
        // 32/8 heads of 128, 128 blocks: 1 token 11.3 / 7.9, 8 tokens 13.7 / 11.9, 16 tokens 17.4 / 15.9; 7/1 heads, 256 blocks in 32
        // or 8 pieces 12.8 / 9.6; 8/8 heads of 96, fp32, 2 tokens, 480 blocks in 37 or 8 pieces 19.5 / 21.9
        constexpr long long kLong = 40;
        const long long stretches = (long long)a.T * ((a.G + S::kRows - 1) / S::kRows) * a.Hk, units = (long long)a.n_listed << a.page_shift;
        const long long room = std::min((long long)sm_count * per_sm, (long long)a.max_ctas) / std::max(stretches, 1ll);
        const long long most = std::min(room, (units + kLeast - 1) / kLeast), pieces = std::min(most, 8ll);
        if (pieces > 1 && (most == pieces || units <= pieces * kLong)) {
            auto in_clusters = attend_rows_kernel<T, W, NT, MINB, Reads::Pieces>;
            static std::atomic<bool> ready[64];
            if (dev >= 64 || !ready[dev].load()) {
                err = cudaFuncSetAttribute(in_clusters, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem + 8 * (kFew + 1));
                if (err != cudaSuccess) return err;
                if (dev < 64) ready[dev].store(true);
            }
            AttendArgs b = a;
            b.cluster = (int)pieces;
            cudaLaunchConfig_t cfg{};
            cfg.gridDim = dim3((unsigned)(stretches * pieces));
            cfg.blockDim = dim3(kThreads);
            cfg.dynamicSmemBytes = smem;
            cfg.stream = s;
            cudaLaunchAttribute attr[2];
            attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr[0].val.programmaticStreamSerializationAllowed = 1;
            attr[1].id = cudaLaunchAttributeClusterDimension;
            attr[1].val.clusterDim.x = (unsigned)pieces;
            attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 2;
            return cudaLaunchKernelEx(&cfg, in_clusters, b);
        }
    }
    return launch_chained(k, dim3((unsigned)grid), dim3(kThreads), smem, s, true, a);
}

// `rows`: those of a stretch's tokens that share a key/value head, at most
inline int tile_rows(int w, long long rows) { return rows <= 8 ? 8 : w == 256 || rows <= 16 ? 16 : 32; }

template <typename T, int W, Reads R>
cudaError_t by_rows(long long rows, const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    if (tile_rows(W, rows) == 8) return launch<T, W, 1, W == 256 ? 3 : 4, R>(a, sm_count, s, launches);
    if (tile_rows(W, rows) == 16) return launch<T, W, 2, W == 256 ? 2 : 3, R>(a, sm_count, s, launches);
    if constexpr (W < 256) return launch<T, W, 4, 2, R>(a, sm_count, s, launches);
    return cudaErrorInvalidValue;
}

template <Reads R>
cudaError_t launch_rows(long long rows, const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    const int w = padded_width(a.D);
    if (a.dtype == MOE_BF16)
        return w == 64 ? by_rows<__nv_bfloat16, 64, R>(rows, a, sm_count, s, launches) : w == 128 ? by_rows<__nv_bfloat16, 128, R>(rows, a, sm_count, s, launches)
                                                                                          : by_rows<__nv_bfloat16, 256, R>(rows, a, sm_count, s, launches);
    return w == 64 ? by_rows<float, 64, R>(rows, a, sm_count, s, launches) : w == 128 ? by_rows<float, 128, R>(rows, a, sm_count, s, launches)
                                                                               : by_rows<float, 256, R>(rows, a, sm_count, s, launches);
}

}  // namespace
}  // namespace kv
}  // namespace lexi
