// Attention of prompts over the 4-bit cache: many query rows of a request, on the tcgen05 tensor cores (bf16 queries,
// heads of up to 128 dimensions; kv_attend.cu has the formula and serves the rest).
//
// A CTA works on 256 query rows of one (request, key/value head) - tokens times the query heads that share it, in two
// tiles of 128 - against tiles of 128 keys:
//   S_t[128 rows, 128 keys] = Q_t K^T       A, B from shared memory, sums in tensor memory
//   O_t[128 rows, W]       += P_t V         A = the weights in tensor memory (they take S_t's columns), B from shared memory
// A code times its scale is exact in f16, so the codes become f16 operands once per CTA and tile: K rows as they lie,
// V transposed (8 keys of a dimension are 16 bytes), both in the 128-byte swizzle.  Queries are scaled by a power of two
// per row and are exact in f16 too; the weights are rounded to f16 (11 bits).
//
// Roles: two warpgroups of softmax, one thread a row; one warpgroup that converts; one thread that issues products.  The
// two tiles alternate: while one's weights are computed the other's products run.  A thread computes a row's weights
// with the reference it has, and again only if a score passed it (kSlack above the largest one so far): tensor memory
// is read once a tile and O is rescaled a few times per row.
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

constexpr int kTileKeys = 128, kTileRows = 128, kStretchRows = 2 * kTileRows;
constexpr int kTileBlocks = kTileKeys / kBlockTokens;
constexpr int kThreads = 512;
constexpr float kFloor = -FLT_MAX;
constexpr float kHead = 6.f, kSlack = 8.f;       // as in kv_attend.cu

template <int W>
struct Shape {
    static constexpr int kQTile = kTileRows * W * 2;          // bytes
    static constexpr int kKTile = kTileKeys * W * 2, kVTile = kTileKeys * W * 2;
    static constexpr int kQAt = 0, kKAt = 2 * kQTile, kVAt = kKAt + 2 * kKTile, kLineAt = kVAt + 2 * kVTile;
    static constexpr int kS = 0, kO = 2 * kTileKeys;          // columns of tensor memory
};

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
__device__ __forceinline__ void st32(uint32_t taddr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
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

__device__ __forceinline__ void sts16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

template <int W>
__global__ void __launch_bounds__(kThreads, 1) attend_prompt_kernel(AttendArgs a) {
    using S = Shape<W>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    int64_t *line = reinterpret_cast<int64_t *>(smem + S::kLineAt);
    __shared__ __align__(8) uint64_t bars[14];
    __shared__ uint32_t tmem_slot, absent[4];
    __shared__ long long sum_s[kThreads / 32];
    __shared__ int last_s;
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

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(k_full(i), 4); tc::mbar_init(k_empty(i), 1);
            tc::mbar_init(v_full(i), 4); tc::mbar_init(v_empty(i), 1);
            tc::mbar_init(s_full(i), 1); tc::mbar_init(p_full(i), 4); tc::mbar_init(o_full(i), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) tc::tmem_alloc(smem_u32(&tmem_slot), 512);

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
        const int p0 = len - nq + row0 / a.G, p1 = len - nq + (row1 - 1) / a.G;
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
                    mine += (long long)max(st + nt - wt, 1) * a.Hk;
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
    const uint32_t tmem = tmem_slot;
    const long long total = line[a.n], share = max((total + gridDim.x - 1) / (long long)gridDim.x, 1ll);
    long long at = min(share * blockIdx.x, total);
    const long long end = min(at + share, total);

    struct Piece { int len, q0, nq, req, row0, row1, st, wt, units, present, head, first, last, cta0, cta1; };
    auto piece_at = [&](long long x) {
        Piece p;
        int lo = 0, hi = a.n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (line[mid] <= x) lo = mid; else hi = mid;
        }
        p.req = lo;
        lengths(lo, p.len, p.q0, p.nq);
        long long off = x - line[lo];
        int nt;
        for (p.row0 = 0;; p.row0 += kStretchRows) {
            p.row1 = min(p.row0 + kStretchRows, p.nq * a.G);
            visible(p.len, p.nq, p.row0, p.row1, p.st, p.wt, nt);
            p.units = max(p.st + nt - p.wt, 1);
            const long long here = (long long)p.units * a.Hk;
            if (off < here) break;
            off -= here;
        }
        p.present = p.st + nt - p.wt;
        p.head = (int)(off / p.units);
        p.first = (int)(off - (long long)p.head * p.units);
        p.last = (int)min((long long)p.units, p.first + end - x);
        p.cta0 = (int)((x - p.first) / share);
        p.cta1 = (int)((x - p.first + p.units - 1) / share);
        return p;
    };
    bool dead = false;       // a wait ran out: nothing more is waited for or issued, the loops run out
    auto wait = [&](uint32_t b, uint32_t parity) { if (!dead) dead = !tc::mbar_wait(b, parity, a.status); };

    // registers by role: 2 x 176 + 104 + 56 = 512 = 4 x 128, what the block was launched with
    if (group == 2) {
        // ================================================================ conversion
        asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        const int c8 = tid - 256;                                             // 0..127
        const int v_sub = c8 >> 6, v_c = lane & 7, v_r = (lane >> 3) + 4 * ((c8 >> 5) & 1);
        constexpr int kCodes = W / 32;                                        // 16-byte words of a key's codes
        constexpr int kVWords = W / 8;                                        // words of 8 keys' share of a stretch
        uint4 kc[kCodes], kn[kCodes];
        uint2 ks, ksn, vs, vsn;
        uint32_t vc[kVWords], vn[kVWords];
        int it = 0;                                                           // tiles so far, over all pieces
        while (at < end) {
            const Piece p = piece_at(at);
            const int32_t *table = a.table + (int64_t)p.req * a.width;
            const int blocks = (p.len + kBlockTokens - 1) / kBlockTokens;
            const int n = min(p.last, p.present) - p.first;
            auto tile_of = [&](int j) { const int u = p.first + j; return u < p.st ? u : p.wt + u - p.st; };
            // cache block of this thread's key (value) share of the j-th tile; -1: absent, -2: behind the cached tokens
            auto find = [&](int j, int in) -> int {
                if (j >= n) return -2;
                const int b = tile_of(j) * kTileBlocks + in;
                if (b >= blocks) return -2;
                const int pg = table[b >> a.page_shift];
                if (pg < 0 || pg >= a.n_pages) { atomicOr(a.status, MOE_KV_STATUS_BAD_INDEX); return -1; }
                return ((pg * a.Hk + p.head) << a.page_shift) + (b & ((1 << a.page_shift) - 1));
            };
            auto fetch = [&](int kb, int vb, uint4 (&kd)[kCodes], uint2 &sd, uint32_t (&vd)[kVWords], uint2 &vsd) {
                sd = vsd = make_uint2(0u, 0u);
#pragma unroll
                for (int i = 0; i < kCodes; ++i) kd[i] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int i = 0; i < kVWords; ++i) vd[i] = 0u;
                if (kb >= 0) {
                    const uint8_t *blk = a.cache + (int64_t)kb * block_bytes(W);
                    const int token = c8 & 15;
#pragma unroll
                    for (int i = 0; i < kCodes; ++i) kd[i] = __ldg(reinterpret_cast<const uint4 *>(blk + token * (W / 2) + 16 * i));
                    if (W == 128) sd = __ldg(reinterpret_cast<const uint2 *>(blk + k_scales_at(W) + token * (W / 16)));
                    else sd.x = __ldg(reinterpret_cast<const uint32_t *>(blk + k_scales_at(W) + token * (W / 16)));
                }
                if (vb >= 0) {
                    const uint8_t *blk = a.cache + (int64_t)vb * block_bytes(W);
                    const int half = v_c & 1;
                    const uint4 *src = reinterpret_cast<const uint4 *>(blk + v_codes_at(W) + v_r * W + ((half * (W / 2)) ^ v_turn(W, v_r)));
#pragma unroll
                    for (int i = 0; i < kVWords / 4; ++i) {
                        const uint4 x = __ldg(src + i);
                        vd[4 * i] = x.x; vd[4 * i + 1] = x.y; vd[4 * i + 2] = x.z; vd[4 * i + 3] = x.w;
                    }
                    vsd = __ldg(reinterpret_cast<const uint2 *>(blk + v_scales_at(W) + (W == 128 ? v_r : v_r >> 1) * kBlockTokens + half * 8));
                }
            };
            const int k_in = c8 >> 4, v_in = v_sub * 4 + (v_c >> 1);
            int kb = find(0, k_in), vb = find(0, v_in), kb2 = find(1, k_in), vb2 = find(1, v_in);
            fetch(kb, vb, kc, ks, vc, vs);
            for (int j = 0; j < n; ++j, ++it) {
                const int stage = it & 1;
                const uint32_t parity = ((it >> 1) & 1) ^ 1;
                fetch(kb2, vb2, kn, ksn, vn, vsn);
                const int kb_now = kb;
                const int key0 = tile_of(j) * kTileKeys;
                kb = kb2; vb = vb2;
                kb2 = find(j + 2, k_in); vb2 = find(j + 2, v_in);

                // ---- keys: this thread's row
                wait(k_empty(stage), parity);
                {
                    const uint32_t gone = __ballot_sync(0xffffffffu, kb_now == -1);       // lanes 0 and 16: two blocks
                    if (lane == 0) {
                        const uint32_t bits = ((gone & 1u) | ((gone >> 15) & 2u)) << (2 * (warp & 3));
                        // every warp has its own byte of the tile's word; a word is written again four tiles later, when
                        // both softmax groups have long read it
                        reinterpret_cast<volatile uint8_t *>(&absent[it & 3])[warp & 3] = (uint8_t)bits;
                    }
                    const uint32_t row = smem_u32(smem + S::kKAt + stage * S::kKTile);
#pragma unroll
                    for (int g = 0; g < W / 16; ++g) {        // 16 dimensions: 8 bytes of codes, one scale, two chunks
                        const uint4 q = kc[g / 2];
                        const uint32_t w0 = g & 1 ? q.z : q.x, w1 = g & 1 ? q.w : q.y;
                        const uint32_t two = scales2(((g < 4 ? ks.x : ks.y) >> (8 * (g & 3))) & 0xffu);
                        const uint32_t sc = __byte_perm(two, 0, 0x1010);
                        uint32_t h[4], u[4];
                        codes4(w0, h);
                        codes4(w1, u);
                        const uint32_t base = row + (g / 4) * (kTileKeys * 128);
                        sts16(base + swizzled(c8, (g & 3) * 2), mul2(h[0], sc), mul2(h[1], sc), mul2(h[2], sc), mul2(h[3], sc));
                        sts16(base + swizzled(c8, (g & 3) * 2 + 1), mul2(u[0], sc), mul2(u[1], sc), mul2(u[2], sc), mul2(u[3], sc));
                    }
                }
                fence_async();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(k_full(stage));

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
                    constexpr int kPerKey = W / 64;           // words of a key's share: dimensions 8 w .. of the stretch
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
                            sts16(base + swizzled(v_r * (W / 8) + 8 * w + e, v_c), d[e][0], d[e][1], d[e][2], d[e][3]);
                    }
                }
                fence_async();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(v_full(stage));
#pragma unroll
                for (int i = 0; i < kCodes; ++i) kc[i] = kn[i];
#pragma unroll
                for (int i = 0; i < kVWords; ++i) vc[i] = vn[i];
                ks = ksn; vs = vsn;
            }
            at += p.last - p.first;
        }
    } else if (group == 3) {
        // ================================================================ products
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 12 && lane == 0) {
            int it = 0;
            uint32_t p_phase = 0;                  // bit t
            const uint32_t q_s = smem_u32(smem + S::kQAt);
            auto scores = [&](int t, int stage) {
                if (dead) return;
#pragma unroll
                for (int i = 0; i < W / 16; ++i) {
                    const uint64_t da = tc::make_kmajor_sw128_desc(q_s + t * S::kQTile + (i / 4) * (kTileRows * 128)) + 2 * (i % 4);
                    const uint64_t db = tc::make_kmajor_sw128_desc(smem_u32(smem + S::kKAt) + stage * S::kKTile + (i / 4) * (kTileKeys * 128)) + 2 * (i % 4);
                    tc::umma_bf16(tmem + S::kS + t * kTileKeys, da, db, idesc_f16(kTileKeys), i > 0);
                }
                tc::umma_commit(s_full(t));
            };
            while (at < end) {
                const Piece p = piece_at(at);
                const int n = min(p.last, p.present) - p.first;
                const int tiles = p.row1 - p.row0 > kTileRows ? 2 : 1;
                if (n > 0) {
                    wait(k_full(it & 1), (it >> 1) & 1);
                    for (int t = 0; t < tiles; ++t) {
                        wait(p_full(t), (p_phase >> t) & 1u);          // the queries are there
                        p_phase ^= 1u << t;
                        tc::tc_fence_after();
                        scores(t, it & 1);
                    }
                    if (!dead) tc::umma_commit(k_empty(it & 1));
                }
                for (int j = 0; j < n; ++j, ++it) {
                    const int stage = it & 1, next = stage ^ 1;
                    wait(v_full(stage), (it >> 1) & 1);
                    if (j + 1 < n) wait(k_full(next), ((it + 1) >> 1) & 1);
                    for (int t = 0; t < tiles; ++t) {
                        wait(p_full(t), (p_phase >> t) & 1u);          // the weights are there, the scores are read
                        p_phase ^= 1u << t;
                        tc::tc_fence_after();
                        if (!dead) {
#pragma unroll
                            for (int i = 0; i < kTileKeys / 16; ++i) {
                                const uint64_t db = tc::make_kmajor_sw128_desc(smem_u32(smem + S::kVAt) + stage * S::kVTile + (i / 4) * (W * 128)) + 2 * (i % 4);
                                umma_ts(tmem + S::kO + t * W, tmem + S::kS + t * kTileKeys + 8 * i, db, idesc_f16(W), j > 0 || i > 0);
                            }
                            tc::umma_commit(o_full(t));
                        }
                        if (j + 1 < n) scores(t, next);
                    }
                    if (!dead) {
                        tc::umma_commit(v_empty(stage));
                        if (j + 1 < n) tc::umma_commit(k_empty(next));
                    }
                }
                at += p.last - p.first;
            }
        }
        __syncwarp();
    } else {
        // ================================================================ softmax: thread = row of tile `group`
        asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
        const int t = group, row_in = tid & 127, wl = (warp & 3) * 32;
        const uint32_t lanes = (uint32_t)wl << 16;
        const uint32_t s_tmem = tmem + S::kS + t * kTileKeys + lanes, o_tmem = tmem + S::kO + t * W + lanes;
        uint32_t s_phase = 0, o_phase = 0;
        int it = 0;
        while (at < end) {
            const Piece p = piece_at(at);
            const int n = min(p.last, p.present) - p.first;
            const int tiles = p.row1 - p.row0 > kTileRows ? 2 : 1;
            const int row = p.row0 + t * kTileRows + row_in;
            const bool real = row < p.row1;
            const int tok = row / a.G, pos = real ? p.len - p.nq + tok : -1;
            const int64_t out_row = (int64_t)(p.q0 + tok) * a.H + p.head * a.G + row - tok * a.G;
            float m = kFloor, l = 0.f, f = 0.f;
            if (t < tiles && n > 0) {
                // ---- queries: a power of two per row makes them f16
                const __nv_bfloat16 *src = (const __nv_bfloat16 *)a.q.p + (int64_t)(p.q0 + tok) * a.q.ts + (int64_t)(p.head * a.G + row - tok * a.G) * a.q.hs;
                const bool vec = (reinterpret_cast<uintptr_t>(a.q.p) & 15u) == 0 && ((a.q.ts | a.q.hs) & 7) == 0;
                uint32_t q[W / 2];
                float top = 0.f;
#pragma unroll
                for (int i = 0; i < W / 8; ++i) {
                    uint4 x = make_uint4(0u, 0u, 0u, 0u);
                    if (real && 8 * i < a.D) {
                        if (vec) x = *reinterpret_cast<const uint4 *>(src + 8 * i);
                        else {
                            uint32_t w[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) w[e] = (uint32_t)__bfloat16_as_ushort(src[8 * i + 2 * e]) | (uint32_t)__bfloat16_as_ushort(src[8 * i + 2 * e + 1]) << 16;
                            x = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                    q[4 * i] = x.x; q[4 * i + 1] = x.y; q[4 * i + 2] = x.z; q[4 * i + 3] = x.w;
                }
#pragma unroll
                for (int i = 0; i < W / 2; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(q[i] << 16)), fabsf(__uint_as_float(q[i] & 0xffff0000u))));
                int e = top > 0.f && top <= FLT_MAX ? ilogbf(top) : 0;
                e = max(e, -100);
                const float up = ldexpf(a.score_scale < 0.f ? -1.f : 1.f, 10 - e);
                f = fmaxf(ldexpf(fabsf(a.score_scale), e - 10), 1e-30f);      // not 0, which times a masked -infinity is no number
                const uint32_t dst = smem_u32(smem + S::kQAt) + t * S::kQTile;
#pragma unroll
                for (int i = 0; i < W / 8; ++i) {
                    uint32_t h[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) h[x] = pack2(__uint_as_float(q[4 * i + x] << 16) * up, __uint_as_float(q[4 * i + x] & 0xffff0000u) * up);
                    sts16(dst + (i / 8) * (kTileRows * 128) + swizzled(row_in, i % 8), h[0], h[1], h[2], h[3]);
                }
                fence_async();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(p_full(t));

                const int p_first = p.len - p.nq + (p.row0 + t * kTileRows) / a.G;
                const int p_last = p.len - p.nq + (min(p.row0 + (t + 1) * kTileRows, p.row1) - 1) / a.G;
                for (int j = 0; j < n; ++j) {
                    const int u = p.first + j, key0 = (u < p.st ? u : p.wt + u - p.st) * kTileKeys;
                    wait(s_full(t), s_phase);
                    s_phase ^= 1u;
                    tc::tc_fence_after();
                    const uint32_t gone = reinterpret_cast<volatile uint32_t *>(absent)[(it + j) & 3];
                    const bool clear = key0 + kTileKeys - 1 <= p_first && gone == 0u &&
                                       (a.window <= 0 || p_last - key0 < a.window || key0 + kTileKeys <= a.sinks);
                    uint32_t w[kTileKeys / 2];
                    float sum = 0.f, top = kFloor;
                    auto weights = [&](float mm) {          // P with the reference mm, its sum, the largest exponent
                        float s0 = 0.f, s1 = 0.f;
                        const float away = (kHead + kSlack) - mm;
                        top = -INFINITY;
#pragma unroll
                        for (int c = 0; c < kTileKeys / 32; ++c) {
                            uint32_t r[32];
                            ld32(s_tmem + 32 * c, r);
                            tc::tmem_ld_wait();
                            if (!clear) {
#pragma unroll
                                for (int i = 0; i < 32; ++i) {
                                    const int key = key0 + 32 * c + i;
                                    const bool see = key <= pos && (a.window <= 0 || pos - key < a.window || key < a.sinks) &&
                                                     !(gone >> (((2 * c + i / 16) >> 1) * 8 + ((2 * c + i / 16) >> 1) * 2 + ((2 * c + i / 16) & 1)) & 1u);
                                    if (!see) r[i] = 0xff800000u;      // -infinity
                                }
                            }
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                const float x = __uint_as_float(r[i]), y = __uint_as_float(r[i + 1]);
                                top = fmaxf(top, fmaxf(x, y));
                                const float e0 = ex2(fmaf(x, f, away)), e1 = ex2(fmaf(y, f, away));
                                s0 += e0; s1 += e1;
                                w[16 * c + i / 2] = pack2(e0, e1);
                            }
                        }
                        sum = s0 + s1;
                    };
                    weights(m);
                    const float reach = top == -INFINITY ? -INFINITY : top * f;
                    if (__any_sync(0xffffffffu, reach > m)) {
                        const float to = fmaxf(m, reach == -INFINITY ? kFloor : reach + kSlack);
                        const float scale = m == to ? 1.f : ex2(m - to);
                        if (j > 0) {
                            wait(o_full(t), o_phase ^ 1u);       // the products of the tile before
                            tc::tc_fence_after();
#pragma unroll
                            for (int c = 0; c < W / 32; ++c) {
                                uint32_t r[32];
                                ld32(o_tmem + 32 * c, r);
                                tc::tmem_ld_wait();
#pragma unroll
                                for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * scale);
                                st32(o_tmem + 32 * c, r);
                            }
                        }
                        l *= scale;
                        m = to;
                        weights(m);
                    }
                    l += sum;
                    st32(s_tmem, w);
                    st32(s_tmem + 32, w + 32);
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

            // ---- the rows' outputs, or this piece of them
            const bool whole = p.first == 0 && p.last == p.units;
            const int slot = blockIdx.x * 2 + (p.first == 0 ? 1 : 0);
            const int in_stretch = t * kTileRows + row_in;
            if (t < tiles) {
                const float k = whole ? (l > 0.f || l != l ? a.v_scale / l : 0.f) : 1.f;
                __nv_bfloat16 *dst = (__nv_bfloat16 *)a.out + out_row * a.D;
                float *part = a.prompt_part + ((int64_t)slot * kStretchRows + in_stretch) * W;
#pragma unroll
                for (int c = 0; c < W / 32; ++c) {
                    uint32_t r[32];
                    __syncwarp();
                    if (n > 0) { ld32(o_tmem + 32 * c, r); tc::tmem_ld_wait(); }
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        float v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = n > 0 ? __uint_as_float(r[i + e]) * k : 0.f;
                        if (!real) continue;
                        if (whole) {
                            if (32 * c + i < a.D)
                                *reinterpret_cast<uint4 *>(dst + 32 * c + i) = make_uint4(bf2(v[0], v[1]), bf2(v[2], v[3]), bf2(v[4], v[5]), bf2(v[6], v[7]));
                        } else {
                            *reinterpret_cast<float4 *>(part + 32 * c + i) = make_float4(v[0], v[1], v[2], v[3]);
                            *reinterpret_cast<float4 *>(part + 32 * c + i + 4) = make_float4(v[4], v[5], v[6], v[7]);
                        }
                    }
                }
                if (!whole && real) a.prompt_ml[(int64_t)slot * kStretchRows + in_stretch] = make_float2(m, l);
            }
            tc::tc_fence_before();
            if (!whole) {
                __threadfence();
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (tid == 0) {
                    const int before = atomicAdd(a.prompt_arrived + p.cta0, 1);
                    last_s = before == p.cta1 - p.cta0;
                    if (last_s) a.prompt_arrived[p.cta0] = 0;          // ready for the next call
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (last_s && t < tiles && real) {
                    __threadfence();
                    float top = kFloor, sum = 0.f;
                    for (int b = p.cta0; b <= p.cta1; ++b)
                        top = fmaxf(top, __ldcg(&a.prompt_ml[(int64_t)(b * 2 + (b == p.cta0)) * kStretchRows + in_stretch]).x);
                    for (int b = p.cta0; b <= p.cta1; ++b) {
                        const float2 ml = __ldcg(&a.prompt_ml[(int64_t)(b * 2 + (b == p.cta0)) * kStretchRows + in_stretch]);
                        sum += (ml.x == top ? 1.f : ex2(ml.x - top)) * ml.y;
                    }
                    const float k = sum > 0.f || sum != sum ? a.v_scale / sum : 0.f;
                    __nv_bfloat16 *dst = (__nv_bfloat16 *)a.out + out_row * a.D;
                    for (int d = 0; d < a.D; d += 8) {
                        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                        for (int b = p.cta0; b <= p.cta1; ++b) {
                            const int64_t at_row = (int64_t)(b * 2 + (b == p.cta0)) * kStretchRows + in_stretch;
                            const float mb = __ldcg(&a.prompt_ml[at_row]).x, kb = (mb == top ? 1.f : ex2(mb - top)) * k;
                            const float4 x = __ldcg(reinterpret_cast<const float4 *>(a.prompt_part + at_row * W + d));
                            const float4 y = __ldcg(reinterpret_cast<const float4 *>(a.prompt_part + at_row * W + d + 4));
                            v[0] += kb * x.x; v[1] += kb * x.y; v[2] += kb * x.z; v[3] += kb * x.w;
                            v[4] += kb * y.x; v[5] += kb * y.y; v[6] += kb * y.z; v[7] += kb * y.w;
                        }
                        *reinterpret_cast<uint4 *>(dst + d) = make_uint4(bf2(v[0], v[1]), bf2(v[2], v[3]), bf2(v[4], v[5]), bf2(v[6], v[7]));
                    }
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");       // last_s is the next piece's
            }
            at += p.last - p.first;
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    if (warp == 12) tc::tmem_dealloc(tmem, 512);
}

template <int W>
cudaError_t launch(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    auto k = attend_prompt_kernel<W>;
    static std::atomic<bool> ready[64];
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    const int most = Shape<W>::kLineAt + 8 * (kMaxRequests + 1) + 1024;
    if (dev >= 64 || !ready[dev].load()) {
        err = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        if (err != cudaSuccess) return err;
        if (dev < 64) ready[dev].store(true);
    }
    k<<<sm_count, kThreads, Shape<W>::kLineAt + 8 * (a.n + 1) + 1024, s>>>(a);
    ++*launches;
    return cudaGetLastError();
}

}  // namespace

size_t prompt_part_floats(int w) { return (size_t)2 * kStretchRows * w; }
size_t prompt_part_rows() { return 2 * kStretchRows; }
bool prompt_supported(int dtype, int head_dim) { return dtype == MOE_BF16 && head_dim <= 128; }

cudaError_t launch_attend_prompt(const AttendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    return padded_width(a.D) == 64 ? launch<64>(a, sm_count, s, launches) : launch<128>(a, sm_count, s, launches);
}

}  // namespace kv
}  // namespace lexi
