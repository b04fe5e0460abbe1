// Attention of prompts over the 4-bit cache: many query rows of a request, on the tcgen05 tensor cores (kv_attend.cu has
// the formula and serves few rows).
//
// A CTA works on 256 query rows of one (request, key/value head) - tokens times the query heads that share it, in two
// tiles of 128 (128 rows for fp32 with W = 128 and for W = 256) - against tiles of 128 keys (64 for W = 256,
// in one stage instead of two for fp32, whose queries take 128 KB: two prompts of 1024 tokens on 4096 keys, 16/4 heads,
// 426 us; 1163 in kv_attend.cu):
//   S_t[128 rows, 128 keys] = Q_t K^T       A, B from shared memory, sums in tensor memory
//   O_t[128 rows, W]       += P_t V         A = the weights in tensor memory (they take S_t's columns), B from shared memory
// A code times its scale is exact in f16, so the codes become f16 operands once per CTA and tile: K rows as they lie,
// V transposed (8 keys of a dimension are 16 bytes), both in the 128-byte swizzle.  Queries are scaled by a power of two
// per row and are exact in f16 too; the weights are rounded to f16 (11 bits, for outputs of 8; kv_attend.cu has the errors).
// For fp32 both are two f16 parts, high and low, and each part has its products.
//
// Roles: two warpgroups of softmax (one for W = 256), one thread a row; one warpgroup that converts; one thread that issues
// products.  The groups alternate: while one's weights are computed the other's products run.  Each has a tile of rows; for
// fp32 with W = 128, whose queries leave room for one, both have that and every other tile of its keys (two prompts of
// 1024 tokens on 4096 keys, 16/4 heads: 212 -> 164 us; the same for bf16 stretches of up to 128 rows loses, 42 -> 55 us
// with 36 rows on 16000 keys, by the second set of results).  A row's scores stay in registers from the search for the
// largest to the weights; its reference lies kSlack above a score that was once the largest, so O is rescaled a few times
// per row, not per tile.
//
// Bounds: 2 x 256 x 128 x W multiply-adds of a key tile take 2048 cycles at W = 128; its 32768 exponentials take 2048
// cycles too on the 16 lanes of the special-function units; conversion 384 issue cycles.
//
// Work split: as in kv_attend.cu, the key tiles of all stretches stand in one line cut evenly over the CTAs, which also
// serves few rows over a long context; a stretch in several pieces is joined by its last CTA in the order of the keys.
#include <float.h>

#include <atomic>

#include "kv_codes.cuh"
#include "kv_internal.h"
#include "tc_ptx.cuh"

namespace lexi {
namespace kv {
namespace {

constexpr int kTileRows = 128;
constexpr int kThreads = 512;
constexpr float kFloor = -FLT_MAX;
constexpr float kTop = 14.f;                     // the largest weight is 2^kTop, as in kv_attend.cu
// What a stretch costs besides its tiles (queries, output, an empty pipeline), in tiles: counted in the line, or a CTA
// with many short stretches would be last by far.  Alternating groups pass a tile in about half the time (with 5 for 3
// there: 333 to 700 tokens of 15/5 heads 52 -> 49 us, 64 tokens on 16000 keys of 16/4 heads 83 -> 77)
constexpr int kEntryTiles = 3, kEntryAlternate = 5;

// T: type of queries and outputs; fp32 queries and weights are two f16 parts each, with products for both.  GROUPS: softmax
// warpgroups, each with its own scores and outputs.  TILES: row tiles of a stretch.  KEYS: keys of a tile
template <typename T, int W, int GROUPS, int TILES, int KEYS>
struct Shape {
    static constexpr int kParts = sizeof(T) == 4 ? 2 : 1;
    static constexpr int kRows = TILES * kTileRows, kPartRows = GROUPS * kTileRows;      // of a stretch; of a piece's results
    static constexpr int kQPart = kTileRows * W * 2, kQTile = kQPart * kParts;          // bytes
    static constexpr int kKTile = KEYS * W * 2, kVTile = KEYS * W * 2;
    static constexpr int kQAt = 0, kKAt = TILES * kQTile;
    static constexpr int kStages = kKAt + 2 * (kKTile + kVTile) <= 196608 ? 2 : 1;       // of keys, of values
    static constexpr int kVAt = kKAt + kStages * kKTile, kLineAt = kVAt + kStages * kVTile;
    static constexpr int kS = 0, kO = GROUPS * 128;           // columns of tensor memory
    static constexpr bool kAlternate = TILES < GROUPS;        // the groups share the rows and take every other key tile
    static_assert((TILES == GROUPS || (TILES == 1 && GROUPS == 2 && kParts == 2)) && kO + GROUPS * W <= 512 && KEYS <= 128 && kLineAt <= 196608, "");
    static_assert(!kAlternate || kStages == 2, "");
    // of the x-th key tile: its stage, and the parity of the stage's use
    static __device__ __forceinline__ int stage(int x) { return x & (kStages - 1); }
    static __device__ __forceinline__ uint32_t turn(int x) { return (uint32_t)(x >> (kStages - 1)) & 1u; }
    // conversion: a thread's dimensions of a key; stretches of dimensions of V, one for KEYS/8 threads
    static constexpr int kKeyDims = W * KEYS / 128, kStretches = 1024 / KEYS, kVDims = W / kStretches;
};
constexpr uint32_t kTmem = 0;                    // where an allocation of all 512 columns begins

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void ld32(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void ld64(uint32_t taddr, uint32_t (&r)[64]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
        "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
          "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
          "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
          "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void st32(uint32_t taddr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// two fp32 numbers in one operation
__device__ __forceinline__ uint64_t pair(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float2 halves(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// D[tmem] (+)= A[tmem] * B[smem]^T, f16
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__host__ __device__ constexpr uint32_t idesc_f16(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24); }

// byte offset of 16-byte chunk c of row r in a swizzled sub-tile of 128-byte rows
__device__ __forceinline__ uint32_t swizzled(int r, int c) { return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)); }

// the lowest n of 32 bits
__device__ __forceinline__ uint32_t below(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

__device__ __forceinline__ void sts16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ void lds16(uint32_t at, uint32_t (&v)[4]) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
}

template <typename T, int W, int GROUPS, int TILES, int KEYS>
__global__ void __launch_bounds__(kThreads, 1) attend_prompt_kernel(AttendArgs a) {
    using S = Shape<T, W, GROUPS, TILES, KEYS>;
    constexpr bool SPLIT = sizeof(T) == 4;
    // The reference lies this far above a score that was once the largest.  fp32: near, so that exponents are small numbers
    // (an exponent of 8 to 16 is rounded to 2^-20, which its weight feels); 2^kTop is then a factor, not part of the exponent
    constexpr float kSlack = SPLIT ? 2.f : 8.f;
    constexpr int kEntry = S::kAlternate ? kEntryAlternate : kEntryTiles;
    constexpr int kTileKeys = KEYS, kTileBlocks = KEYS / kBlockTokens, kStretchRows = S::kRows;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    int64_t *line = reinterpret_cast<int64_t *>(smem + S::kLineAt);
    __shared__ __align__(8) uint64_t bars[15];
    __shared__ uint32_t tmem_slot, absent[4];
    __shared__ long long sum_s[kThreads / 32];
    __shared__ int last_s;
    __shared__ float f_s[kTileRows];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, group = warp >> 2;
    const uint32_t bar = smem_u32(bars);
    // full and empty of two K stages, of two V stages; scores, weights, output and queries of two tiles
    auto k_full = [&](int i) { return bar + 8 * i; };
    auto k_empty = [&](int i) { return bar + 16 + 8 * i; };
    auto v_full = [&](int i) { return bar + 32 + 8 * i; };
    auto v_empty = [&](int i) { return bar + 48 + 8 * i; };
    auto s_full = [&](int t) { return bar + 64 + 8 * t; };
    auto p_full = [&](int t) { return bar + 80 + 8 * t; };
    auto o_full = [&](int t) { return bar + 96 + 8 * t; };
    const uint32_t all_done = bar + 112;          // of the last products, if a wait ran out

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(k_full(i), 4); tc::mbar_init(k_empty(i), 1);
            tc::mbar_init(v_full(i), 4); tc::mbar_init(v_empty(i), 1);
            tc::mbar_init(s_full(i), 1); tc::mbar_init(p_full(i), 4); tc::mbar_init(o_full(i), 1);
        }
        tc::mbar_init(all_done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid < 4) absent[tid] = 0u;
    if (warp == 12) tc::tmem_alloc(smem_u32(&tmem_slot), 512);

    // Maybe ahead of warp 12's allocation.  A dependent that starts early cannot take the tensor memory first: it starts once
    // every CTA of this kernel is there, and each has all 65536 registers of its SM
    pdl_trigger();
    pdl_wait();

    // ---- the line: key tiles of every stretch of prompts
    auto lengths = [&](int i, int &len, int &q0, int &nq) {
        len = max(a.kv_len[i], 0);
        q0 = a.cu[i];
        nq = a.cu[i + 1] - q0;
        if (q0 < 0 || nq < 0 || q0 > a.T - nq) { atomicOr(a.status, MOE_KV_STATUS_BAD_INDEX); nq = 0; }
        const int page_tokens = kBlockTokens << a.page_shift;
        if (len > (int64_t)a.width * page_tokens) { atomicOr(a.status, MOE_KV_STATUS_BAD_INDEX); len = a.width * page_tokens; }
        if ((int64_t)nq * a.G <= a.prompt_rows) nq = 0;       // the other kernel's
    };
    // tiles that rows [row0, row1) see: [0, st) and [wt, nt)
    auto visible = [&](int len, int nq, int row0, int row1, int &st, int &wt, int &nt) {
        const int p0 = len - nq + div_g(a, row0), p1 = len - nq + div_g(a, row1 - 1);
        nt = p1 < 0 ? 0 : p1 / kTileKeys + 1;
        wt = a.window > 0 ? max(p0 - a.window + 1, 0) / kTileKeys : 0;
        wt = min(wt, nt);
        st = a.window > 0 ? min((int)(((int64_t)a.sinks + kTileKeys - 1) / kTileKeys), wt) : 0;
    };
    {
        long long carry = 0;
        for (int base = 0; base < a.n; base += kThreads) {
            const int i = base + tid;
            long long mine = 0;
            if (i < a.n) {
                int len, q0, nq;
                lengths(i, len, q0, nq);
                for (int row0 = 0; row0 < nq * a.G; row0 += kStretchRows) {
                    int st, wt, nt;
                    visible(len, nq, row0, min(row0 + kStretchRows, nq * a.G), st, wt, nt);
                    mine += (long long)(kEntry + max(st + nt - wt, 1)) * a.Hk;
                }
            }
            long long inc = mine;
            for (int o = 1; o < 32; o <<= 1) {
                const long long up = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += up;
            }
            if (lane == 31) sum_s[warp] = inc;
            __syncthreads();
            long long before = carry, all = carry;
            for (int w = 0; w < kThreads / 32; ++w) { if (w < warp) before += sum_s[w]; all += sum_s[w]; }
            if (i < a.n) line[i] = before + inc - mine;
            carry = all;
            __syncthreads();
        }
        if (tid == 0) line[a.n] = carry;
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = kTmem;
    bool dead = tmem_slot != kTmem;          // a wait ran out: nothing more is waited for or issued, the loops run out
    if (dead && tid == 0) atomicOr(a.status, MOE_KV_STATUS_TIMEOUT);
    const long long total = line[a.n], share = max((total + gridDim.x - 1) / (long long)gridDim.x, 1ll);
    const long long at = min(share * blockIdx.x, total);
    const long long end = min(at + share, total);

    // A stretch's place in the line is kEntry (what beginning it costs) and then its tiles.  Every role walks the pieces
    // of the CTA's share by itself: found once, then counted on.
    struct Piece { int req, len, q0, nq, row0, row1, st, wt, present, units, head, first, last, cta0, cta1; long long place; };
    auto shape = [&](Piece &p) {
        p.row1 = min(p.row0 + kStretchRows, p.nq * a.G);
        int nt;
        visible(p.len, p.nq, p.row0, p.row1, p.st, p.wt, nt);
        p.present = p.st + nt - p.wt;
        p.units = max(p.present, 1);
    };
    auto cut = [&](Piece &p) {          // which tiles of the stretch are this CTA's; false: behind the share
        const long long tiles0 = p.place + kEntry;
        p.first = (int)max(at - tiles0, 0ll);
        p.last = (int)min(end - tiles0, (long long)p.units);
        p.cta0 = (int)(tiles0 / share);
        p.cta1 = (int)((tiles0 + p.units - 1) / share);
        return p.place < end;
    };
    auto begin = [&](Piece &p) {
        if (at >= end) return false;
        int lo = 0, hi = a.n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (line[mid] <= at) lo = mid; else hi = mid;
        }
        p.req = lo;
        lengths(lo, p.len, p.q0, p.nq);
        p.place = line[lo];
        for (p.row0 = 0;; p.row0 += kStretchRows) {
            shape(p);
            const long long here = (long long)(kEntry + p.units) * a.Hk;
            if (at < p.place + here) break;
            p.place += here;
        }
        p.head = (int)((at - p.place) / (kEntry + p.units));
        p.place += (long long)p.head * (kEntry + p.units);
        return cut(p);
    };
    auto next = [&](Piece &p) {
        p.place += kEntry + p.units;
        if (p.place >= end) return false;
        if (++p.head == a.Hk) {
            p.head = 0;
            p.row0 += kStretchRows;
            while (p.row0 >= p.nq * a.G) {          // the line goes on, so there is a request with rows
                lengths(++p.req, p.len, p.q0, p.nq);
                p.row0 = 0;
            }
            shape(p);
        }
        return cut(p);
    };
    auto wait = [&](uint32_t b, uint32_t parity) { if (!dead) dead = !tc::mbar_wait(b, parity, a.status); };

    // registers by role: 2 x 184 + 88 + 56 = 512 = 4 x 128, what the block was launched with
    if (group == 2) {
        // ================================================================ conversion
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        const int c8 = tid - 256;                                             // 0..127
        const int key_in = c8 % KEYS, key_part = c8 / KEYS;                   // a thread's key, and which kKeyDims of it
        const int v_sub = KEYS == 128 ? c8 >> 6 : 0, v_c = lane & 7, v_r = (lane >> 3) + 4 * (KEYS == 128 ? (c8 >> 5) & 1 : c8 >> 5);
        constexpr int kCodes = S::kKeyDims / 32;                              // 16-byte words of its codes
        constexpr int kVWords = S::kVDims;                                    // words of 8 keys' share of a stretch
        static_assert(W <= 128 || (W == 256 && KEYS == 64), "");
        uint4 kc[kCodes];
        uint2 ks, vs;
        uint32_t vc[kVWords];
        int it = 0;                                                           // tiles so far, over all pieces
        Piece p;
        for (bool more = begin(p); more; more = next(p)) {
            if (p.last <= p.first) continue;
            const int32_t *table = a.table + (int64_t)p.req * a.width;
            // Of a tile's blocks those that some row of the stretch sees: a tile reaches in front of the window and behind the first
            // tokens, and what lies there may be gone from the table
            const int blocks = (p.len + kBlockTokens - 1) / kBlockTokens, sink_blocks = a.sinks / kBlockTokens + (a.sinks % kBlockTokens > 0);
            const int window_block = a.window > 0 ? max(p.len - p.nq + div_g(a, p.row0) - a.window + 1, 0) / kBlockTokens : 0;
            const int n = min(p.last, p.present) - p.first;
            auto tile_of = [&](int j) { const int u = p.first + j; return u < p.st ? u : p.wt + u - p.st; };
            // cache block of this thread's key (value) share of the j-th tile; -1: absent, -2: seen by no row
            auto find = [&](int j, int in) -> int {
                if (j >= n) return -2;
                const int b = tile_of(j) * kTileBlocks + in;
                if (b >= blocks || (b < window_block && b >= sink_blocks)) return -2;
                const int pg = table[b >> a.page_shift];
                if (pg < 0 || pg >= a.n_pages) { atomicOr(a.status, MOE_KV_STATUS_BAD_INDEX); return -1; }
                return ((pg * a.Hk + p.head) << a.page_shift) + (b & ((1 << a.page_shift) - 1));
            };
            auto fetch_keys = [&](int kb) {
                ks = make_uint2(0u, 0u);
#pragma unroll
                for (int i = 0; i < kCodes; ++i) kc[i] = make_uint4(0u, 0u, 0u, 0u);
                if (kb < 0) return;
                const uint8_t *blk = a.cache + (int64_t)kb * block_bytes(W);
                const int token = key_in & 15;
                const uint8_t *codes = blk + token * (W / 2) + key_part * (S::kKeyDims / 2), *scales = blk + k_scales_at(W) + token * (W / 16) + key_part * (S::kKeyDims / 16);
#pragma unroll
                for (int i = 0; i < kCodes; ++i) kc[i] = __ldg(reinterpret_cast<const uint4 *>(codes + 16 * i));
                if (S::kKeyDims == 128) ks = __ldg(reinterpret_cast<const uint2 *>(scales));
                else ks.x = __ldg(reinterpret_cast<const uint32_t *>(scales));
            };
            auto fetch_values = [&](int vb) {
                vs = make_uint2(0u, 0u);
#pragma unroll
                for (int i = 0; i < kVWords; ++i) vc[i] = 0u;
                if (vb < 0) return;
                const uint8_t *blk = a.cache + (int64_t)vb * block_bytes(W);
                const int half = v_c & 1;
                if (W == 256) {           // half of a stretch of the cache's layout
                    const int r = v_r >> 1;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint2 x = __ldg(reinterpret_cast<const uint2 *>(blk + v_codes_at(W) + r * W + (((half * 8 + i) * 16) ^ v_turn(W, r)) + (v_r & 1) * 8));
                        vc[(2 * i) % kVWords] = x.x; vc[(2 * i + 1) % kVWords] = x.y;
                    }
                } else {
                    const uint4 *src = reinterpret_cast<const uint4 *>(blk + v_codes_at(W) + v_r * W + ((half * (W / 2)) ^ v_turn(W, v_r)));
#pragma unroll
                    for (int i = 0; i < kVWords / 4; ++i) {
                        const uint4 x = __ldg(src + i);
                        vc[4 * i] = x.x; vc[4 * i + 1] = x.y; vc[4 * i + 2] = x.z; vc[4 * i + 3] = x.w;
                    }
                }
                vs = __ldg(reinterpret_cast<const uint2 *>(blk + v_scales_at(W) + (W == 64 ? v_r >> 1 : v_r) * kBlockTokens + half * 8));
            };
            const int k_in = key_in >> 4, v_in = v_sub * 4 + (v_c >> 1);
            // a tile's bytes are asked for as soon as the tile before has left the registers, its pages a tile earlier
            int kb = find(0, k_in), vb = find(0, v_in), kb2 = find(1, k_in), vb2 = find(1, v_in);
            fetch_keys(kb);
            fetch_values(vb);
            for (int j = 0; j < n; ++j, ++it) {
                const int stage = S::stage(it);
                const uint32_t parity = S::turn(it) ^ 1u;
                const int kb_now = kb;
                const int key0 = tile_of(j) * kTileKeys;
                kb = kb2; vb = vb2;
                kb2 = find(j + 2, k_in); vb2 = find(j + 2, v_in);

                // ---- keys: this thread's row
                wait(k_empty(stage), parity);
                {
                    const uint32_t gone = __ballot_sync(0xffffffffu, kb_now == -1);       // lanes 0 and 16: two blocks
                    if (lane == 0) {
                        // 32 keys have a byte of the tile's word; a word is written again four tiles later, when the softmax
                        // groups have long read it
                        const int byte = warp % (KEYS / 32);
                        const uint32_t bits = ((gone & 1u) | ((gone >> 15) & 2u)) << (2 * byte);
                        reinterpret_cast<volatile uint8_t *>(&absent[it & 3])[byte] = (uint8_t)bits;
                    }
                    const uint32_t row = smem_u32(smem + S::kKAt + stage * S::kKTile);
#pragma unroll
                    for (int g = 0; g < S::kKeyDims / 16; ++g) {        // 16 dimensions: 8 bytes of codes, one scale, two chunks
                        const uint4 q = kc[g / 2];
                        const uint32_t w0 = g & 1 ? q.z : q.x, w1 = g & 1 ? q.w : q.y;
                        const uint32_t two = scales2(((g < 4 ? ks.x : ks.y) >> (8 * (g & 3))) & 0xffu);
                        const uint32_t sc = __byte_perm(two, 0, 0x1010);
                        uint32_t h[4], u[4];
                        codes4(w0, h);
                        codes4(w1, u);
                        const uint32_t base = row + (key_part * (S::kKeyDims / 64) + g / 4) * (KEYS * 128);
                        sts16(base + swizzled(key_in, (g & 3) * 2), mul2(h[0], sc), mul2(h[1], sc), mul2(h[2], sc), mul2(h[3], sc));
                        sts16(base + swizzled(key_in, (g & 3) * 2 + 1), mul2(u[0], sc), mul2(u[1], sc), mul2(u[2], sc), mul2(u[3], sc));
                    }
                }
                fence_async();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(k_full(stage));
                fetch_keys(kb);

                // ---- values: 8 keys of a stretch of dimensions, transposed
                wait(v_empty(stage), parity);
                {
                    // a key behind the cached ones has no scale, whatever its bytes
                    const int rest = p.len - (key0 + v_in * kBlockTokens + (v_c & 1) * 8);
                    if (rest < 8) {
                        const uint64_t keep = rest <= 0 ? 0ull : (1ull << (8 * rest)) - 1ull;
                        vs.x &= (uint32_t)keep; vs.y &= (uint32_t)(keep >> 32);
                    }
                    uint32_t sc[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[i] = scales2(((i < 2 ? vs.x : vs.y) >> (16 * (i & 1))) & 0xffffu);
                    const uint32_t base = smem_u32(smem + S::kVAt + stage * S::kVTile) + v_sub * (W * 128);
                    constexpr int kPerKey = S::kVDims / 8;    // words of a key's share: dimensions 8 w .. of the stretch
                    constexpr uint32_t L = 0x0f0f0f0fu;
#pragma unroll
                    for (int w = 0; w < kPerKey; ++w) {
                        uint32_t d[8][4];                     // [dimension][key pair]
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t x = vc[(2 * i) * kPerKey + w], y = vc[(2 * i + 1) * kPerKey + w];
                            uint32_t even[4], odd[4];
                            codes4((x & L) | ((y & L) << 4), even);
                            codes4(((x >> 4) & L) | (y & ~L), odd);
#pragma unroll
                            for (int e = 0; e < 4; ++e) { d[2 * e][i] = mul2(even[e], sc[i]); d[2 * e + 1][i] = mul2(odd[e], sc[i]); }
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            sts16(base + swizzled(v_r * S::kVDims + 8 * w + e, v_c), d[e][0], d[e][1], d[e][2], d[e][3]);
                    }
                }
                fence_async();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(v_full(stage));
                fetch_values(vb);
            }
        }
    } else if (group == 3) {
        // ================================================================ products
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 12) {
            // The warp walks together and one thread issues, so that descriptors are in uniform registers (the whole walk in
            // one thread: 764 us for 710 on four prompts of 2048 tokens)
            const bool one = elect_one();
            int it = 0;
            uint32_t p_phase = 0;                  // bit t
            // a k16 step is 32 bytes inside a 128-byte row (2 in a descriptor's units of 16), 64 elements are a sub-tile
            const uint64_t q_d = tc::make_kmajor_sw128_desc(smem_u32(smem + S::kQAt)), k_d = tc::make_kmajor_sw128_desc(smem_u32(smem + S::kKAt)),
                           v_d = tc::make_kmajor_sw128_desc(smem_u32(smem + S::kVAt));
            auto scores = [&](int t, int stage) {
                const uint64_t da = q_d + (S::kAlternate ? 0 : t) * (S::kQTile / 16), db = k_d + stage * (S::kKTile / 16);
                if (one && !dead) {
#pragma unroll
                    for (int x = 0; x < S::kParts; ++x)
#pragma unroll
                        for (int i = 0; i < W / 16; ++i) {
                            const int part = S::kParts - 1 - x;          // the low part first: sums are cut off at their size so far
                            tc::umma_bf16(kTmem + S::kS + t * KEYS, da + part * (S::kQPart / 16) + (i / 4) * (kTileRows * 128 / 16) + 2 * (i % 4),
                                          db + (i / 4) * (KEYS * 128 / 16) + 2 * (i % 4), idesc_f16(KEYS), x + i > 0);
                        }
                    tc::umma_commit(s_full(t));
                }
                __syncwarp();
            };
            auto outputs = [&](int t, int stage, bool more) {
                const uint64_t db = v_d + stage * (S::kVTile / 16);
                if (one && !dead) {
#pragma unroll
                    for (int part = 0; part < S::kParts; ++part)
#pragma unroll
                        for (int i = 0; i < KEYS / 16; ++i)
                            umma_ts(kTmem + S::kO + t * W, kTmem + S::kS + t * KEYS + part * (KEYS / 2) + 8 * i, db + (i / 4) * (W * 128 / 16) + 2 * (i % 4), idesc_f16(W),
                                    part + i > 0 || more);
                    tc::umma_commit(o_full(t));
                }
                __syncwarp();
            };
            Piece p;
            for (bool go = begin(p); go; go = next(p)) {
                if (p.last <= p.first) continue;
                const int n = __reduce_max_sync(0xffffffffu, min(p.last, p.present) - p.first);        // into a uniform register
                if constexpr (S::kAlternate) {
                    for (int t = 0; t < 2 && t < n; ++t) {
                        const int x = it + t;
                        wait(k_full(S::stage(x)), S::turn(x));
                        wait(p_full(t), (p_phase >> t) & 1u);          // the queries are there
                        p_phase ^= 1u << t;
                        tc::tc_fence_after();
                        scores(t, S::stage(x));
                        if (one && !dead) tc::umma_commit(k_empty(S::stage(x)));
                        __syncwarp();
                    }
#pragma unroll 1
                    for (int j = 0; j < n; ++j, ++it) {
                        const int stage = S::stage(it), t = j & 1;
                        wait(v_full(stage), S::turn(it));
                        wait(p_full(t), (p_phase >> t) & 1u);          // the weights are there, the scores are read
                        p_phase ^= 1u << t;
                        tc::tc_fence_after();
                        outputs(t, stage, j >= 2);
                        if (one && !dead) tc::umma_commit(v_empty(stage));
                        __syncwarp();
                        if (j + 2 < n) {
                            wait(k_full(stage), S::turn(it + 2));
                            tc::tc_fence_after();
                            scores(t, stage);
                            if (one && !dead) tc::umma_commit(k_empty(stage));
                            __syncwarp();
                        }
                    }
                } else {
                    const int tiles = TILES == 1 ? 1 : __reduce_max_sync(0xffffffffu, p.row1 - p.row0 > kTileRows ? 2 : 1);
                    if (n > 0) {
                        wait(k_full(S::stage(it)), S::turn(it));
                        for (int t = 0; t < tiles; ++t) {
                            wait(p_full(t), (p_phase >> t) & 1u);          // the queries are there
                            p_phase ^= 1u << t;
                            tc::tc_fence_after();
                            scores(t, S::stage(it));
                        }
                        if (one && !dead) tc::umma_commit(k_empty(S::stage(it)));
                        __syncwarp();
                    }
#pragma unroll 1
                    for (int j = 0; j < n; ++j, ++it) {
                        const int stage = S::stage(it), other = S::stage(it + 1);
                        wait(v_full(stage), S::turn(it));
                        if (j + 1 < n) wait(k_full(other), S::turn(it + 1));
#pragma unroll
                        for (int t = 0; t < TILES; ++t) {
                            if (t >= tiles) continue;
                            wait(p_full(t), (p_phase >> t) & 1u);          // the weights are there, the scores are read
                            p_phase ^= 1u << t;
                            tc::tc_fence_after();
                            outputs(t, stage, j > 0);
                            if (j + 1 < n) scores(t, other);
                        }
                        if (one && !dead) {
                            tc::umma_commit(v_empty(stage));
                            if (j + 1 < n) tc::umma_commit(k_empty(other));
                        }
                        __syncwarp();
                    }
                }
            }
        }
        __syncwarp();
    } else if (group < GROUPS) {
        // ================================================================ softmax: thread = row of tile `group`
        asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
        const int t = group, row_in = tid & 127, wl = (warp & 3) * 32;
        const uint32_t lanes = (uint32_t)wl << 16;
        const uint32_t s_tmem = tmem + S::kS + t * kTileKeys + lanes, o_tmem = tmem + S::kO + t * W + lanes;
        uint32_t s_phase = 0, o_phase = 0;
        int it = 0;
        Piece p;
        for (bool more = begin(p); more; more = next(p)) {
            if (p.last <= p.first) continue;
            const int n = min(p.last, p.present) - p.first;
            const int tiles = TILES == 1 || p.row1 - p.row0 <= kTileRows ? 1 : 2;
            // alternating groups have all rows and take key tiles t, t + 2, ...; their results are joined as pieces are
            const int n_t = S::kAlternate ? (n - t + 1) / 2 : t < tiles ? n : 0;
            const int tile0 = S::kAlternate ? p.row0 : p.row0 + t * kTileRows;
            const int row = tile0 + row_in;
            const bool real = row < p.row1;
            const int tok = div_g(a, row), pos = real ? p.len - p.nq + tok : -1;
            const int64_t out_row = (int64_t)(p.q0 + tok) * a.H + p.head * a.G + row - tok * a.G;
            float m = kFloor, l = 0.f, f = 0.f;
            if (n_t > 0 && !(S::kAlternate && t == 1)) {
                // ---- queries into their place, 16 bytes a lane; then a row a thread: a power of two makes it f16 (two parts of
                // fp32: 16 raw bytes each lie where a chunk of one part will)
                constexpr int kPerChunk = 16 / (int)sizeof(T), kChunks = W / kPerChunk, kLanes = kChunks < 32 ? kChunks : 32, kAtOnce = 32 / kLanes,
                              kTurns = kChunks / kLanes;
                const bool vec = (reinterpret_cast<uintptr_t>(a.q.p) & 15u) == 0 && ((a.q.ts | a.q.hs) & (kPerChunk - 1)) == 0;
                const int64_t q_row = real ? (int64_t)(p.q0 + tok) * a.q.ts + (int64_t)(p.head * a.G + row - tok * a.G) * a.q.hs : INT64_MIN;
                const uint32_t place = smem_u32(smem + S::kQAt) + t * S::kQTile;
                auto chunk_at = [&](int part, int r, int c) { return place + part * S::kQPart + (c / 8) * (kTileRows * 128) + swizzled(r, c % 8); };
#pragma unroll 4
                for (int x = 0; x < 32 / kAtOnce * kTurns; ++x) {
                    const int r = x / kTurns * kAtOnce + lane / kLanes;    // of the warp's 32 rows
                    const int chunk = x % kTurns * kLanes + lane % kLanes;
                    const int64_t at_row = __shfl_sync(0xffffffffu, q_row, r);
                    const uint32_t to = SPLIT ? chunk_at(chunk & 1, wl + r, chunk >> 1) : chunk_at(0, wl + r, chunk);
                    const T *src = (const T *)a.q.p + at_row + kPerChunk * chunk;
                    if (at_row == INT64_MIN || kPerChunk * chunk >= a.D) sts16(to, 0u, 0u, 0u, 0u);
                    else if (vec) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(src) : "memory");
                    else {
#pragma unroll 1
                        for (int e = 0; e < kPerChunk; ++e) {
                            if (SPLIT) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + 4 * e), "r"(reinterpret_cast<const uint32_t *>(src)[e]) : "memory");
                            else asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + 2 * e), "h"(reinterpret_cast<const uint16_t *>(src)[e]) : "memory");
                        }
                    }
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                __syncwarp();
                auto numbers = [&](int c, float (&v)[8]) {                 // dimensions 8 c .. of this thread's row
                    uint32_t x[4], y[4];
                    lds16(chunk_at(0, row_in, c), x);
                    if (SPLIT) lds16(chunk_at(1, row_in, c), y);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (SPLIT) { v[e] = __uint_as_float(x[e]); v[4 + e] = __uint_as_float(y[e]); }
                        else { v[2 * e] = __uint_as_float(x[e] << 16); v[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u); }
                    }
                };
                float top = 0.f;
#pragma unroll 4
                for (int c = 0; c < W / 8; ++c) {
                    float v[8];
                    numbers(c, v);
#pragma unroll
                    for (int e = 0; e < 8; e += 2) top = max3(top, fabsf(v[e]), fabsf(v[e + 1]));
                }
                const int e2 = row_exponent(top);
                const float up = power2(10 - e2) * (a.score_scale < 0.f ? -1.f : 1.f);
                f = fmaxf(fabsf(a.score_scale) * power2(e2 - 10), 1e-30f);      // not 0, which times a masked -infinity is no number
#pragma unroll 4
                for (int c = 0; c < W / 8; ++c) {
                    float v[8];
                    numbers(c, v);
                    uint32_t h[4], lo[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float u = v[2 * e] * up, w = v[2 * e + 1] * up;
                        h[e] = pack2(u, w);
                        if (SPLIT) { const float2 g = unpack2(h[e]); lo[e] = pack2(u - g.x, w - g.y); }
                    }
                    sts16(chunk_at(0, row_in, c), h[0], h[1], h[2], h[3]);
                    if (SPLIT) sts16(chunk_at(1, row_in, c), lo[0], lo[1], lo[2], lo[3]);
                }
                fence_async();
            }
            if (S::kAlternate && n > 0) {
                if (t == 0) f_s[row_in] = f;
                asm volatile("bar.sync 2, 256;" ::: "memory");
                if (t == 1) f = f_s[row_in];
            }
            if (n_t > 0) {
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(p_full(t));

                const int p_first = p.len - p.nq + div_g(a, tile0);
                const int p_last = p.len - p.nq + div_g(a, min(tile0 + kTileRows, p.row1) - 1);
                for (int jj = 0; jj < n_t; ++jj) {
                    const int j = S::kAlternate ? 2 * jj + t : jj;
                    const int u = p.first + j, key0 = (u < p.st ? u : p.wt + u - p.st) * kTileKeys;
                    wait(s_full(t), s_phase);
                    s_phase ^= 1u;
                    tc::tc_fence_after();
                    const uint32_t gone = reinterpret_cast<volatile uint32_t *>(absent)[(it + j) & 3];
                    const bool clear = key0 + kTileKeys - 1 <= p_first && gone == 0u &&
                                       (a.window <= 0 || p_last - key0 < a.window || key0 + kTileKeys <= a.sinks);
                    // Code size counts: four roles run at once out of one instruction cache.  Masks (of the first and last
                    // tiles only) are a pass of their own over the scores, the weights are one copy of code.
                    if (!clear) {
#pragma unroll 1
                        for (int c = 0; c < kTileKeys / 32; ++c) {
                            uint32_t r[32];
                            ld32(s_tmem + 32 * c, r);
                            tc::tmem_ld_wait();
                            // keys key0 + 32 c + i that the row sees, i = 0..31
                            const int k0 = key0 + 32 * c;
                            uint32_t see = below(pos + 1 - k0);
                            if (a.window > 0) see &= ~below(pos - a.window + 1 - k0) | below(a.sinks - k0);
                            const uint32_t out = (gone >> (10 * c)) & 3u;          // byte c, bits 2c and 2c + 1: blocks that are absent
                            see &= ~((out & 1u ? 0xffffu : 0u) | (out & 2u ? 0xffff0000u : 0u));
#pragma unroll
                            for (int i = 0; i < 32; ++i) r[i] = see >> i & 1u ? r[i] : 0xff800000u;      // -infinity
                            st32(s_tmem + 32 * c, r);
                        }
                        st_wait();
                    }
                    // ---- the row's scores stay in registers from the search for the largest to the weights: a chain of
                    // loads from tensor memory (200 cycles each) would be the longest part of a tile
                    uint32_t r0[64], r1[KEYS == 128 ? 64 : 4];
                    ld64(s_tmem, r0);
                    if constexpr (KEYS == 128) ld64(s_tmem + 64, r1);
                    tc::tmem_ld_wait();
                    float top0 = -INFINITY, top1 = -INFINITY, top2 = -INFINITY, top3 = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 64; i += 4) {
                        top0 = max3(top0, __uint_as_float(r0[i]), __uint_as_float(r0[i + 1]));
                        top1 = max3(top1, __uint_as_float(r0[i + 2]), __uint_as_float(r0[i + 3]));
                        if constexpr (KEYS == 128) {
                            top2 = max3(top2, __uint_as_float(r1[i]), __uint_as_float(r1[i + 1]));
                            top3 = max3(top3, __uint_as_float(r1[i + 2]), __uint_as_float(r1[i + 3]));
                        }
                    }
                    const float top = fmaxf(fmaxf(top0, top1), fmaxf(top2, top3)), reach = top == -INFINITY ? -INFINITY : top * f;
                    if (__any_sync(0xffffffffu, reach > m)) {       // O follows only when a score passes the reference
                        const float to = fmaxf(m, reach == -INFINITY ? kFloor : reach + kSlack);
                        const float scale = m == to ? 1.f : ex2(m - to);
                        if (jj > 0) {
                            wait(o_full(t), o_phase ^ 1u);       // the products of the tile before
                            tc::tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < W / 16; ++c) {
                                uint32_t x[16];
                                tc::tmem_ld16(o_tmem + 16 * c, x);
                                tc::tmem_ld_wait();
#pragma unroll
                                for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * scale);
                                st16(o_tmem + 16 * c, x);
                            }
                        }
                        l *= scale;
                        m = to;
                    }
                    // ---- weights: 32 scores become 16 columns
                    const float away = SPLIT ? -m : kTop - m;
                    const uint64_t f2 = pair(f, f), away2 = pair(away, away);
                    uint64_t sum2 = 0ull, sum2b = 0ull;
                    auto weights = [&](const uint32_t (&r)[64], int at_key) {        // 32 keys become 16 columns
                        uint32_t w[16], lo[SPLIT ? 16 : 1];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float2 x = halves(fma2(pair(__uint_as_float(r[at_key % 64 + 2 * i]), __uint_as_float(r[at_key % 64 + 2 * i + 1])), f2, away2));
                            float e0 = ex2(x.x), e1 = ex2(x.y);
                            if (SPLIT) { e0 *= 16384.f; e1 *= 16384.f; }          // 2^kTop
                            if (SPLIT && (i & 1)) sum2b = add2(sum2b, pair(e0, e1));
                            else sum2 = add2(sum2, pair(e0, e1));
                            w[i] = pack2(e0, e1);
                            if (SPLIT) { const float2 g = unpack2(w[i]); lo[SPLIT ? i : 0] = pack2(e0 - g.x, e1 - g.y); }
                        }
                        st16(s_tmem + at_key / 2, w);
                        if constexpr (SPLIT) st16(s_tmem + KEYS / 2 + at_key / 2, lo);
                    };
                    weights(r0, 0);
                    weights(r0, 32);
                    if constexpr (KEYS == 128) {
                        weights(r1, 64);
                        weights(r1, 96);
                    }
                    if (SPLIT) sum2 = add2(sum2, sum2b);
                    l += halves(sum2).x + halves(sum2).y;
                    st_wait();
                    tc::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(p_full(t));
                    o_phase ^= 1u;
                }
                wait(o_full(t), o_phase ^ 1u);
                tc::tc_fence_after();
            }
            it += max(n, 0);
            // the queries are both groups': their place is free once both have all their scores
            if (S::kAlternate && n > 0) asm volatile("bar.sync 2, 256;" ::: "memory");

            // ---- the rows' outputs, or this piece of them
            const bool whole = p.first == 0 && p.last == p.units && !S::kAlternate;
            const int slot = blockIdx.x * 2 + (p.first == 0 ? 1 : 0);
            if (S::kAlternate || t < tiles) {
                // the rows go through the queries' place in shared memory (their products are done), so that W/8 lanes store
                // 2 W bytes of a row: all of its dimensions as bf16, or half of them as fp32
                constexpr int kLanes = W / 8, kAtOnce = 32 / kLanes, kPass = W / 2;
                const float k = whole ? (l > 0.f || l != l ? a.v_scale / l : 0.f) : 1.f;
                const uint32_t place = smem_u32(smem + S::kQAt) + t * (S::kAlternate ? S::kQPart : S::kQTile);
                const bool wide = SPLIT || !whole;
                auto slot16 = [&](int r, int c) { return place + (c / 8) * (kTileRows * 128) + swizzled(wl + r, c % 8); };
                const int chunk = lane % kLanes;
                const int64_t to_row = real ? out_row * a.D : -1;
                float *part = a.prompt_part + ((int64_t)slot * S::kPartRows + t * kTileRows + wl) * W;
#pragma unroll 1
                for (int pass = 0; pass < (wide ? 2 : 1); ++pass) {
                    __syncwarp();
#pragma unroll 1
                    for (int c = 0; c < (wide ? kPass : W) / 32; ++c) {
                        uint32_t r[32];
                        if (n_t > 0) { ld32(o_tmem + pass * kPass + 32 * c, r); tc::tmem_ld_wait(); }
                        else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) r[i] = 0u;
                        }
                        if (SPLIT) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * k);
                        } else if (whole) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) r[i] = bf2(__uint_as_float(r[2 * i]) * k, __uint_as_float(r[2 * i + 1]) * k);
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (i < 4 || wide) sts16(slot16(lane, (wide ? 8 : 4) * c + i), r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
                    }
                    __syncwarp();
#pragma unroll 4
                    for (int x = 0; x < 32 / kAtOnce; ++x) {
                        const int r = x * kAtOnce + lane / kLanes;
                        const int64_t to = __shfl_sync(0xffffffffu, to_row, r);
                        uint32_t v[4];
                        lds16(slot16(r, chunk), v);
                        if (to == -1) continue;
                        if (!whole) *reinterpret_cast<uint4 *>(part + r * W + pass * kPass + 4 * chunk) = make_uint4(v[0], v[1], v[2], v[3]);
                        else {
                            const int d = SPLIT ? pass * kPass + 4 * chunk : 8 * chunk;
                            if (d < a.D) *reinterpret_cast<uint4 *>((T *)a.out + to + d) = make_uint4(v[0], v[1], v[2], v[3]);
                        }
                    }
                }
                __syncwarp();
                if (!whole && real) a.prompt_ml[(int64_t)slot * S::kPartRows + t * kTileRows + row_in] = make_float2(m, l);
            }
            tc::tc_fence_before();
            if (!whole) {
                __threadfence();
                asm volatile("bar.sync 1, %0;" ::"n"(GROUPS * 128) : "memory");
                if (tid == 0) {
                    last_s = S::kAlternate && p.cta0 == p.cta1;        // the stretch is this CTA's alone
                    if (!last_s) {
                        const int before = atomicAdd(a.prompt_arrived + p.cta0, 1);
                        last_s = before == p.cta1 - p.cta0;
                        if (last_s) a.prompt_arrived[p.cta0] = 0;      // ready for the next call
                    }
                }
                asm volatile("bar.sync 1, %0;" ::"n"(GROUPS * 128) : "memory");
                if (last_s) {
                    __threadfence();
                    // a warp takes every kWarps-th row, a lane W/32 neighbouring dimensions: whole lines, several rows in flight
                    constexpr int kPer = W / 32, kRowsAtOnce = W == 256 ? 4 : 8, kWarps = 4 * GROUPS;
                    const int rows = p.row1 - p.row0;
#pragma unroll 1
                    for (int x0 = warp; x0 < rows; x0 += kWarps * kRowsAtOnce) {
                        float top[kRowsAtOnce], sum[kRowsAtOnce], v[kRowsAtOnce][kPer];
#pragma unroll
                        for (int y = 0; y < kRowsAtOnce; ++y) {
                            top[y] = kFloor; sum[y] = 0.f;
#pragma unroll
                            for (int e = 0; e < kPer; ++e) v[y][e] = 0.f;
                        }
                        constexpr int kOf = S::kAlternate ? 2 : 1;             // results of a piece
#pragma unroll 1
                        for (int h = p.cta0 * kOf; h < (p.cta1 + 1) * kOf; ++h) {
                            const int b = h / kOf;
                            const int64_t at_piece = (int64_t)(b * 2 + (b == p.cta0)) * S::kPartRows + h % kOf * kTileRows;
                            float2 ml[kRowsAtOnce];
                            float d[kRowsAtOnce][kPer];
#pragma unroll
                            for (int y = 0; y < kRowsAtOnce; ++y) {
                                const int64_t at_row = at_piece + min(x0 + kWarps * y, rows - 1);
                                ml[y] = __ldcg(&a.prompt_ml[at_row]);
                                const float *src = a.prompt_part + at_row * W + lane * kPer;
                                if (kPer >= 4) {
#pragma unroll
                                    for (int e = 0; e < kPer; e += 4) {
                                        const float4 z = __ldcg(reinterpret_cast<const float4 *>(src + e));
                                        d[y][e % kPer] = z.x; d[y][(e + 1) % kPer] = z.y; d[y][(e + 2) % kPer] = z.z; d[y][(e + 3) % kPer] = z.w;
                                    }
                                } else {
                                    const float2 z = __ldcg(reinterpret_cast<const float2 *>(src));
                                    d[y][0] = z.x; d[y][1] = z.y;
                                }
                            }
#pragma unroll
                            for (int y = 0; y < kRowsAtOnce; ++y) {
                                const float to = fmaxf(top[y], ml[y].x), old = top[y] == to ? 1.f : ex2(top[y] - to), k = ml[y].x == to ? 1.f : ex2(ml[y].x - to);
                                sum[y] = sum[y] * old + ml[y].y * k;
#pragma unroll
                                for (int e = 0; e < kPer; ++e) v[y][e] = v[y][e] * old + d[y][e] * k;
                                top[y] = to;
                            }
                        }
#pragma unroll
                        for (int y = 0; y < kRowsAtOnce; ++y) {
                            const int x = x0 + kWarps * y;
                            if (x >= rows || lane * kPer >= a.D) continue;
                            const float k = sum[y] > 0.f || sum[y] != sum[y] ? a.v_scale / sum[y] : 0.f;
                            const int r_tok = div_g(a, p.row0 + x);
                            T *dst = (T *)a.out + ((int64_t)(p.q0 + r_tok) * a.H + p.head * a.G + p.row0 + x - r_tok * a.G) * a.D + lane * kPer;
#pragma unroll
                            for (int e = 0; e < kPer; e += 2) {
                                if (SPLIT) *reinterpret_cast<float2 *>(dst + e) = make_float2(v[y][e] * k, v[y][e + 1] * k);
                                else *reinterpret_cast<uint32_t *>(dst + e) = bf2(v[y][e] * k, v[y][e + 1] * k);
                            }
                        }
                    }
                }
                asm volatile("bar.sync 1, %0;" ::"n"(GROUPS * 128) : "memory");       // last_s is the next piece's
            }
        }
    }
    tc::tc_fence_before();
    // The softmax groups wait for the last products; where one gave up, the thread that issued them does, before their operands
    // and sums are another CTA's
    const bool gave_up = __syncthreads_or(dead);
    tc::tc_fence_after();
    if (warp == 12) {
        if (gave_up) {
            if (elect_one()) tc::umma_commit(all_done);
            __syncwarp();
            tc::mbar_wait(all_done, 0u, a.status);
            __syncwarp();
        }
        tc::tmem_dealloc(tmem_slot, 512);
    }
}

template <typename T, int W, int GROUPS, int TILES, int KEYS>
cudaError_t launch(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    using S = Shape<T, W, GROUPS, TILES, KEYS>;
    auto k = attend_prompt_kernel<T, W, GROUPS, TILES, KEYS>;
    static std::atomic<bool> ready[64];
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    const int most = S::kLineAt + 8 * (kMaxRequests + 1) + 1024;
    if (dev >= 64 || !ready[dev].load()) {
        err = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        if (err != cudaSuccess) return err;
        if (dev < 64) ready[dev].store(true);
    }
    ++*launches;
    return launch_chained(k, dim3(sm_count), dim3(kThreads), S::kLineAt + 8 * (a.n + 1) + 1024, s, true, a);
}

}  // namespace

size_t prompt_part_floats(int w) { return (size_t)2 * (w == 256 ? 128 : 256) * w; }
size_t prompt_part_rows() { return 2 * 256; }

cudaError_t launch_attend_prompt(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    const int w = padded_width(a.D);
    if (a.dtype == MOE_BF16)
        return w == 64 ? launch<__nv_bfloat16, 64, 2, 2, 128>(a, sm_count, s, launches) : w == 128 ? launch<__nv_bfloat16, 128, 2, 2, 128>(a, sm_count, s, launches)
                                                                                              : launch<__nv_bfloat16, 256, 1, 1, 64>(a, sm_count, s, launches);
    return w == 64 ? launch<float, 64, 2, 2, 128>(a, sm_count, s, launches) : w == 128 ? launch<float, 128, 2, 1, 128>(a, sm_count, s, launches)
                                                                                       : launch<float, 256, 1, 1, 64>(a, sm_count, s, launches);
}

}  // namespace kv
}  // namespace lexi
