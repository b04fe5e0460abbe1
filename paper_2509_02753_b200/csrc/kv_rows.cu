// Rotary positions, storing rows in 4 bits, and reading them back.
#include <float.h>
#include <math.h>

#include "kv_internal.h"

namespace lexi {
namespace kv {
namespace {

constexpr int kThreads = 256;

// ------------------------------------------------------------------ angles
// theta_i in 64 bits: at position 10^6 an angle in 32 bits would be off by 0.06.  A program makes the table once: 32768
// positions of 64 pairs take 56 us (3 to write them), by the power that every position computes for itself
__global__ void rope_table_kernel(RopeTableArgs a) {
    const long long total = (long long)a.n * a.half;
    for (long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x; e < total; e += (long long)gridDim.x * blockDim.x) {
        const int i = (int)(e % a.half);
        const double p = (double)(e / a.half), rot = 2.0 * a.half;
        double base = a.base;
        if (a.scaling == MOE_ROPE_BASE && rot > 2) base *= pow(a.factor, rot / (rot - 2.0));
        double theta = pow(base, -2.0 * i / rot);
        const double two_pi = 6.283185307179586476925286766559;
        if (a.scaling == MOE_ROPE_LINEAR) {
            theta /= a.factor;
        } else if (a.scaling == MOE_ROPE_PARTS) {
            // the pair index that turns n times over the original context: rot ln(original/(2 pi n)) / (2 ln base)
            const double k = rot / (2.0 * log(base));
            const double from = fmax(floor(k * log(a.original / (two_pi * a.high))), 0.0);
            const double to = fmin(ceil(k * log(a.original / (two_pi * a.low))), rot - 1.0);
            const double ramp = fmin(fmax((i - from) / fmax(to - from, 1e-3), 0.0), 1.0);
            theta = theta * (1.0 - ramp) + theta / a.factor * ramp;
        } else if (a.scaling == MOE_ROPE_BANDS) {
            const double turns = a.original * theta / two_pi;
            const double keep = fmin(fmax((turns - a.low) / (a.high - a.low), 0.0), 1.0);
            theta = theta * keep + theta / a.factor * (1.0 - keep);
        }
        double sn, cs;
        sincos(p * theta, &sn, &cs);
        a.table[e] = make_float2((float)(cs * a.magnitude), (float)(sn * a.magnitude));
    }
}

// ------------------------------------------------------------------ elements
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }

__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// 8 neighbouring elements; VEC: 16-byte aligned
template <bool VEC>
__device__ __forceinline__ void load8(const float *p, int n, float (&v)[8]) {
    if (VEC) {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
    }
}
template <bool VEC>
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, int n, float (&v)[8]) {
    if (VEC) {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f(p[i]) : 0.f;
    }
}
template <bool VEC>
__device__ __forceinline__ void store8(float *p, int n, const float (&v)[8]) {
    if (VEC) {
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) p[i] = v[i];
    }
}
template <bool VEC>
__device__ __forceinline__ void store8(__nv_bfloat16 *p, int n, const float (&v)[8]) {
    if (VEC) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) p[i] = __float2bfloat16_rn(v[i]);
    }
}

// u cos - w sin, w cos + u sin, each product rounded by itself: keys are quantised from these numbers, and a product
// fused into the sum would round some of them to another 4-bit code than the formula read operation by operation
__device__ __forceinline__ void turn(float &u, float &w, float2 cs) {
    const float a = __fsub_rn(__fmul_rn(u, cs.x), __fmul_rn(w, cs.y));
    w = __fadd_rn(__fmul_rn(w, cs.x), __fmul_rn(u, cs.y));
    u = a;
}

// How the rows of a call are walked, by layout and alignment; a thread has one unit of a row, two stretches of 8
// dimensions where it can (32 bytes of bf16 in flight per head, and the unit of several heads shares the angles):
//   kHalves    half layout, rope_dim/2 a multiple of 8, rows on 16 bytes: stretch u with the one it turns with; behind
//              rope_dim two neighbours
//   kPairs     pairs layout, rows on 16 bytes: two neighbours
//   kPartners  half layout, any rope_dim, rows on 16 bytes, not in place: one stretch; the other ends are read one by one
//   kSingles   everything else: 8 pairs or 8 passing dimensions, one by one
// Both ends of a pair are one thread's except in kPartners, so that the others can work in place.
enum Walk { kHalves, kPairs, kPartners, kSingles };

__host__ __device__ inline int units_of(Walk walk, int D, int rot) {
    switch (walk) {
        case kHalves: return rot / 16 + (D - rot + 15) / 16;
        case kPairs: return (D + 15) / 16;
        case kPartners: return D / 8;
        default: return (rot / 2 + 7) / 8 + (D - rot + 7) / 8;
    }
}

// the angles of pairs i0.. of a row of the table, 1 and 0 behind rope_dim
template <bool VEC>
__device__ __forceinline__ void load_angles(const Turn &tn, int t, int i0, float2 (&cs)[8], bool &turns, int32_t *status) {
    const int half = tn.rot / 2;
    const int p = i0 < half ? tn.position[t] : 0;
    turns = i0 < half && p >= 0 && p < tn.n_positions;
    if (i0 < half && !turns) atomicOr(status, MOE_KV_STATUS_BAD_INDEX);
    const float2 *row = tn.table + (int64_t)p * half + i0;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float4 v = make_float4(1.f, 0.f, 1.f, 0.f);
        if (turns) {
            if (VEC && i0 + i + 2 <= half) v = *reinterpret_cast<const float4 *>(row + i);
            else {
                if (i0 + i < half) { v.x = row[i].x; v.y = row[i].y; }
                if (i0 + i + 1 < half) { v.z = row[i + 1].x; v.w = row[i + 1].y; }
            }
        }
        cs[i] = make_float2(v.x, tn.inverse ? -v.y : v.y);
        cs[i + 1] = make_float2(v.z, tn.inverse ? -v.w : v.w);
    }
}

template <typename T>
__device__ __forceinline__ float turned_at(const T *row, const Turn &tn, const float2 *cs_row, int d);

// Heads a thread takes where there are enough rows: it reads the angles once for them.  8192 tokens x 32 heads of 128
// dimensions, bf16: 35.7, 28.7, 27.6 us with 1, 2, 4
constexpr int kHeads = 4;

// heads h0 .. h0 + n of unit `unit` of token t
template <typename T, int WALK, bool TABLE16>
__device__ __forceinline__ void turn_unit(const T *x, int64_t xhs, T *y, int64_t yhs, int n, int D, const Turn &tn, int t, int unit, int32_t *status) {
    float2 cs[8];
    bool turns;
    const int half = tn.rot / 2;
    if (WALK == kHalves || WALK == kPairs) {
        const int turning = WALK == kHalves ? half / 8 : (D + 15) / 16;
        const bool turner = unit < turning;
        const int d0 = WALK == kPairs ? 16 * unit : turner ? 8 * unit : tn.rot + 16 * (unit - turning);
        const int d1 = WALK == kHalves && turner ? half + d0 : d0 + 8;
        const int pairs = WALK == kPairs ? half - d0 / 2 : 8;          // of the unit's 8, those in front of rope_dim
        // rows are asked for before the angles, which wait for the position
        float a[8], b[8];
        load8<true>(x + d0, 8, a);
        if (d1 < D) load8<true>(x + d1, 8, b);
        load_angles<TABLE16>(tn, t, WALK == kPairs ? d0 / 2 : turner ? d0 : half, cs, turns, status);
        if (!turns && x == y) return;
        for (int h = 0; h < n; ++h) {
            if (turns) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (WALK == kHalves) turn(a[i], b[i], cs[i]);
                    else if (i < pairs) {          // by (1, 0) is not the same: an infinity times 0 is no number
                        if (i < 4) turn(a[2 * i], a[2 * i + 1], cs[i]);
                        else turn(b[2 * i - 8], b[2 * i - 7], cs[i]);
                    }
                }
            }
            store8<true>(y + h * yhs + d0, 8, a);
            if (d1 < D) store8<true>(y + h * yhs + d1, 8, b);
            if (h + 1 < n) {
                load8<true>(x + (h + 1) * xhs + d0, 8, a);
                if (d1 < D) load8<true>(x + (h + 1) * xhs + d1, 8, b);
            }
        }
    } else if (WALK == kPartners) {
        const int d0 = 8 * unit;
        const int p = d0 < tn.rot ? tn.position[t] : 0;
        const bool in = d0 < tn.rot && p >= 0 && p < tn.n_positions;
        if (d0 < tn.rot && !in) atomicOr(status, MOE_KV_STATUS_BAD_INDEX);
        const float2 *row = in ? tn.table + (int64_t)p * half : nullptr;
        for (int h = 0; h < n; ++h) {
            float a[8];
            load8<true>(x + h * xhs + d0, 8, a);
            if (in) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (d0 + i < tn.rot) a[i] = turned_at(x + h * xhs, tn, row, d0 + i);
            }
            store8<true>(y + h * yhs + d0, 8, a);
        }
    } else {
        const int turning = (half + 7) / 8;
        if (unit < turning) {
            const int i0 = 8 * unit, m = min(8, half - i0);
            load_angles<false>(tn, t, i0, cs, turns, status);
            if (!turns && x == y) return;
            const bool two = tn.layout == MOE_ROPE_PAIRS;
            for (int h = 0; h < n; ++h)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < m) {
                        const int d = two ? 2 * (i0 + i) : i0 + i, e = two ? d + 1 : d + half;
                        float u = to_f(x[h * xhs + d]), w = to_f(x[h * xhs + e]);
                        if (turns) turn(u, w, cs[i]);
                        put(y + h * yhs + d, u);
                        put(y + h * yhs + e, w);
                    }
        } else if (x != y) {
            const int d = tn.rot + (unit - turning) * 8;
            for (int h = 0; h < n; ++h)
                for (int i = d; i < min(d + 8, D); ++i) y[h * yhs + i] = x[h * xhs + i];
        }
    }
}

template <typename T, int WALK, bool TABLE16>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs a, FastDiv units, FastDiv groups, int per_group) {
    pdl_trigger();
    pdl_wait();
    uint32_t e = blockIdx.x * kThreads + threadIdx.x, unit, grp, token;
    units.split(e, e, unit);
    groups.split(e, token, grp);
    if (token >= (uint32_t)a.T) return;
    const int64_t t = token;
    const int h0 = (int)grp * per_group;
    turn_unit<T, WALK, TABLE16>((const T *)a.x.p + t * a.x.ts + h0 * a.x.hs, a.x.hs, (T *)a.y + t * a.yts + h0 * a.yhs, a.yhs, min(per_group, a.H - h0), a.D,
                                a.turn, (int)t, (int)unit, a.status);
}

// ------------------------------------------------------------------ 4 bits
__device__ __forceinline__ uint32_t to_e4m3(float v) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(v));
    return r & 0xffu;
}
__device__ __forceinline__ float from_e4m3(uint32_t b) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)b));
    const __half2 v = *reinterpret_cast<const __half2 *>(&h);
    return __low2float(v);
}
__device__ __forceinline__ uint32_t to_e2m1_pair(float lo, float hi) {
    uint32_t r;
    asm("{\n\t.reg .b8 b;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %1, %2;\n\tmov.b32 %0, {b, 0, 0, 0};\n\t}" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 from_e2m1_pair(uint32_t byte) {
    uint32_t h;
    asm("{\n\t.reg .b8 b, u0, u1, u2;\n\tmov.b32 {b, u0, u1, u2}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b;\n\t}" : "=r"(h) : "r"(byte));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

__device__ __forceinline__ float max_or_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Half of a group of 16: its 8 numbers -> 4 bytes of codes, and the group's scale byte; the neighbouring lane has the
// other half
__device__ __forceinline__ uint32_t quantise8(float (&x)[8], float inv6, float scale, uint32_t &s8, int32_t *status) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max_or_nan(top, fabsf(x[i]));
    if (!(top <= FLT_MAX)) {          // a NaN -> 0, an infinity -> the largest number
        atomicOr(status, MOE_KV_STATUS_NONFINITE);
        top = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!(fabsf(x[i]) <= FLT_MAX)) x[i] = x[i] != x[i] ? 0.f : copysignf(FLT_MAX, x[i]);
            top = fmaxf(top, fabsf(x[i]));
        }
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    s8 = to_e4m3(fminf(__fmul_rn(top, inv6), 448.f));
    const float s = __fmul_rn(from_e4m3(s8), scale);
    float inv = s > 0.f ? __frcp_rn(s) : 0.f;
    if (inv > FLT_MAX) {          // s below 2^-128: x and s times 2^64, or a zero times infinity would be stored as a code
        inv = __frcp_rn(__fmul_rn(s, 0x1p64f));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __fmul_rn(x[i], 0x1p64f);
    }
    uint32_t w = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= to_e2m1_pair(__fmul_rn(x[2 * i], inv), __fmul_rn(x[2 * i + 1], inv)) << (8 * i);
    return w;
}

// One element of a row with its head turned
template <typename T>
__device__ __forceinline__ float turned_at(const T *row, const Turn &tn, const float2 *cs_row, int d) {
    float u = to_f(row[d]);
    if (!cs_row || d >= tn.rot) return u;
    const int half = tn.rot / 2;
    const bool second = tn.layout == MOE_ROPE_HALF ? d >= half : d & 1;
    const int i = tn.layout == MOE_ROPE_HALF ? (second ? d - half : d) : d >> 1;
    float w = to_f(row[tn.layout == MOE_ROPE_HALF ? (second ? d - half : d + half) : d ^ 1]);
    float2 cs = cs_row[i];
    if (tn.inverse) cs.y = -cs.y;
    if (second) { turn(w, u, cs); return u; }
    turn(u, w, cs);
    return u;
}

// 8 dimensions d0.. of a row, turned; VEC: rows and the table on 16 bytes.  In two parts, so that the row's bytes are
// asked for before the position is known: a are the dimensions, b what they turn with where that is another stretch of 8
template <typename T, bool VEC>
__device__ __forceinline__ void load_turned8(const T *row, int D, int d0, const Turn &tn, bool turns, float (&a)[8], float (&b)[8]) {
    if (d0 >= D) {
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = 0.f;
        return;
    }
    load8<VEC>(row + d0, D - d0, a);
    const int half = tn.rot / 2;
    if (VEC && turns && d0 < tn.rot && tn.layout == MOE_ROPE_HALF && half % 8 == 0) load8<true>(row + (d0 >= half ? d0 - half : d0 + half), 8, b);
}
template <typename T, bool VEC>
__device__ __forceinline__ void turn8(const T *row, int d0, const Turn &tn, const float2 *cs_row, float (&a)[8], const float (&b)[8]) {
    if (!cs_row || d0 >= tn.rot) return;
    const int half = tn.rot / 2;
    if (VEC && tn.layout == MOE_ROPE_HALF && half % 8 == 0) {
        // as turn(), this thread's end only: own cos -+ other sin, whichever end it is
        const bool second = d0 >= half;
        const float4 *cs = reinterpret_cast<const float4 *>(cs_row + (second ? d0 - half : d0));
        const uint32_t flip = second ? 0u : 0x80000000u;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float4 v = cs[i / 2];
            a[i] = __fadd_rn(__fmul_rn(a[i], v.x), __fmul_rn(b[i], __uint_as_float(__float_as_uint(v.y) ^ flip)));
            a[i + 1] = __fadd_rn(__fmul_rn(a[i + 1], v.z), __fmul_rn(b[i + 1], __uint_as_float(__float_as_uint(v.w) ^ flip)));
        }
    } else if (tn.layout == MOE_ROPE_PAIRS) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (d0 / 2 + i < half) turn(a[2 * i], a[2 * i + 1], cs_row[d0 / 2 + i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d0 + i < tn.rot) a[i] = turned_at(row, tn, cs_row, d0 + i);
    }
}

// Address of a slot's block; nullptr for a slot that is not stored
__device__ __forceinline__ uint8_t *block_of(uint8_t *cache, int64_t slot, int64_t n_slots, int page_shift, int Hk, int h, int W, int32_t *status) {
    if (slot < 0 || slot >= n_slots) {
        if (slot != -1) atomicOr(status, MOE_KV_STATUS_BAD_INDEX);
        return nullptr;
    }
    const int64_t pg = slot >> page_shift;
    const int in = (int)slot & ((1 << page_shift) - 1);
    return cache + ((((pg * Hk + h) << page_shift) + in) >> 4) * (int64_t)block_bytes(W);
}

// One launch, two kinds of CTAs: queries turn as in rope_kernel; keys and values are stored by a thread for 8
// dimensions of both, W/8 neighbouring threads having a row, two of them a group's scale.  Rows are read in whole lines and a
// key's codes leave in one piece; a value's codes leave as W/8 pieces, next to those of its 15 neighbours, which the L2
// puts together (through shared memory, a warp for 16 tokens, it took 1.8 times as long: fewer loads in flight).
template <typename T, int WALK, bool VEC, int W>
__global__ void __launch_bounds__(kThreads, 4) append_kernel(AppendArgs a, uint32_t store_ratio, FastDiv units, FastDiv groups, int per_group, FastDiv heads) {
    constexpr int kLanes = W / 8;
    pdl_trigger();
    pdl_wait();
    // the storing CTAs (29 us by themselves for 8192 tokens: 451 instructions a warp, issue slots 54 % taken, else waits for
    // memory of 28 warps an SM) lie evenly among the turning ones (bound by memory): number f(i) is CTA i
    // where f(i + 1) > f(i), f(i) = i * ratio / 2^32
    const uint32_t store = __umulhi(blockIdx.x, store_ratio);
    if (store_ratio != 0xffffffffu && __umulhi(blockIdx.x + 1, store_ratio) == store) {
        uint32_t e = (blockIdx.x - store) * kThreads + threadIdx.x, unit, grp, token;
        units.split(e, e, unit);
        groups.split(e, token, grp);
        if (token >= (uint32_t)a.T) return;
        const int64_t t = token;
        const int h0 = (int)grp * per_group;
        turn_unit<T, WALK, VEC>((const T *)a.q.p + t * a.q.ts + h0 * a.q.hs, a.q.hs, (T *)a.q_out + (t * a.H + h0) * a.D, a.D, min(per_group, a.H - h0), a.D, a.turn,
                                (int)t, (int)unit, a.status);
        return;
    }
    // a row's lanes are in one warp and go together
    const uint32_t e = (store_ratio != 0xffffffffu ? store : blockIdx.x) * kThreads + threadIdx.x;
    const int c = (int)(e % kLanes);
    uint32_t token_no, head;
    heads.split(e / kLanes, token_no, head);
    const int h = (int)head;
    const int64_t t = token_no;
    const bool real = t < a.T, turns = a.turn.rot > 0;
    const T *k_src = (const T *)a.k.p + t * a.k.ts + h * a.k.hs, *v_src = (const T *)a.v.p + t * a.v.ts + h * a.v.hs;
    float k[8], other[8], v[8];
    int64_t slot = -1;
    int p = 0;
    // all that is read but the angles, before anything waits
    if (real) {
        slot = a.slot[t];
        if (turns) p = a.turn.position[t];
        load_turned8<T, VEC>(k_src, a.D, 8 * c, a.turn, turns, k, other);
        load_turned8<T, VEC>(v_src, a.D, 8 * c, a.turn, false, v, other);
    }
    uint8_t *blk = block_of(a.cache, slot, a.n_slots, a.page_shift, a.Hk, h, W, a.status);
    if (blk) {
        const bool in = p >= 0 && p < a.turn.n_positions;
        if (turns && !in) atomicOr(a.status, MOE_KV_STATUS_BAD_INDEX);
        if (8 * c < a.D) turn8<T, VEC>(k_src, 8 * c, a.turn, turns && in ? a.turn.table + (int64_t)p * (a.turn.rot / 2) : nullptr, k, other);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) k[i] = v[i] = 0.f;          // what is not stored tells nothing of its numbers
    }
    uint32_t ks, vs;
    const uint32_t kc = quantise8(k, a.k_inv6, a.k_scale, ks, a.status), vc = quantise8(v, a.v_inv6, a.v_scale, vs, a.status);
    if (!blk) return;
    constexpr int per = W / 64;                 // chunks of 8 dimensions in a stretch of the layout
    const int token = (int)(slot % kBlockTokens), r = c / per;
    *reinterpret_cast<uint32_t *>(blk + token * (W / 2) + 4 * c) = kc;
    *reinterpret_cast<uint32_t *>(blk + v_codes_at(W) + r * W + ((token * (W / 16)) ^ v_turn(W, r)) + 4 * (c % per)) = vc;
    if (c % 2 == 0) {
        blk[k_scales_at(W) + token * (W / 16) + c / 2] = (uint8_t)ks;
        blk[v_scales_at(W) + c / 2 * kBlockTokens + token] = (uint8_t)vs;
    }
}

// A thread reads 8 dimensions of a key row and of a value row
template <typename T, int W>
__global__ void __launch_bounds__(kThreads) read_kernel(ReadArgs a, FastDiv chunks, FastDiv heads) {
    pdl_trigger();
    pdl_wait();
    uint32_t e = blockIdx.x * kThreads + threadIdx.x, chunk, head, token_no;
    chunks.split(e, e, chunk);
    heads.split(e, token_no, head);
    if (token_no >= (uint32_t)a.T) return;
    const int c = (int)chunk, h = (int)head;
    const int64_t t = token_no;
    const int64_t slot = a.slot[t];
    const uint8_t *blk = block_of(const_cast<uint8_t *>(a.cache), slot, a.n_slots, a.page_shift, a.Hk, h, W, a.status);
    uint32_t kw = 0u, vw = 0u;
    float ks = 0.f, vs = 0.f;
    if (blk) {
        constexpr int per = W / 64;                 // stretches of 8 dimensions in one of the layout's
        const int token = (int)(slot & 15), r = c / per;
        if (a.k) {
            kw = *reinterpret_cast<const uint32_t *>(blk + token * (W / 2) + 4 * c);
            ks = from_e4m3(blk[k_scales_at(W) + token * (W / 16) + c / 2]);
        }
        if (a.v) {
            vw = *reinterpret_cast<const uint32_t *>(blk + v_codes_at(W) + r * W + ((token * (W / 16)) ^ v_turn(W, r)) + 4 * (c % per));
            vs = from_e4m3(blk[v_scales_at(W) + c / 2 * kBlockTokens + token]);
        }
    }
    const int64_t out = (t * a.Hk + h) * a.D + 8 * c;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        T *dst = (T *)(which ? a.v : a.k);
        if (!dst) continue;
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = from_e2m1_pair((which ? vw : kw) >> (8 * i) & 0xffu);
            x[2 * i] = f.x * (which ? vs : ks) * (which ? a.v_scale : a.k_scale);          // code * scale has at most 6 bits: one rounding
            x[2 * i + 1] = f.y * (which ? vs : ks) * (which ? a.v_scale : a.k_scale);
        }
        store8<true>(dst + out, 8, x);
    }
}

bool aligned(const void *p, int64_t ts, int64_t hs, int dtype) {
    const int64_t e = dtype == MOE_BF16 ? 8 : 4;
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ts % e == 0 && hs % e == 0;
}

Walk walk_of(int D, const Turn &tn, bool rows16, bool in_place) {
    if (!rows16 || D % 8) return kSingles;
    if (tn.rot == 0 || tn.layout == MOE_ROPE_PAIRS) return kPairs;
    if (tn.rot % 16 == 0) return kHalves;
    return in_place ? kSingles : kPartners;
}

// Heads that share a thread's angles: kHeads once there are enough threads for the machine without it
int heads_per_thread(long long threads, int sm_count) { return threads >= (long long)kHeads * 2048 * sm_count ? kHeads : 1; }

bool table16(const Turn &tn) { return tn.rot == 0 || ((reinterpret_cast<uintptr_t>(tn.table) & 15u) == 0 && (tn.rot / 2) % 2 == 0); }

template <typename T>
auto rope_of(Walk w, bool t16) {
    switch (w) {
        case kHalves: return t16 ? rope_kernel<T, kHalves, true> : rope_kernel<T, kHalves, false>;
        case kPairs: return t16 ? rope_kernel<T, kPairs, true> : rope_kernel<T, kPairs, false>;
        case kPartners: return rope_kernel<T, kPartners, false>;
        default: return rope_kernel<T, kSingles, false>;
    }
}
// VEC: rows and table on 16 bytes
template <typename T, int W>
auto append_of(Walk w, bool vec) {
    if (!vec) {
        switch (w) {
            case kHalves: return append_kernel<T, kHalves, false, W>;
            case kPairs: return append_kernel<T, kPairs, false, W>;
            case kPartners: return append_kernel<T, kPartners, false, W>;
            default: return append_kernel<T, kSingles, false, W>;
        }
    }
    switch (w) {
        case kHalves: return append_kernel<T, kHalves, true, W>;
        case kPairs: return append_kernel<T, kPairs, true, W>;
        case kPartners: return append_kernel<T, kPartners, true, W>;
        default: return append_kernel<T, kSingles, true, W>;
    }
}
template <typename T>
auto append_of(int width, Walk w, bool vec) { return width == 64 ? append_of<T, 64>(w, vec) : width == 128 ? append_of<T, 128>(w, vec) : append_of<T, 256>(w, vec); }

}  // namespace

cudaError_t launch_rope_table(const RopeTableArgs &a, cudaStream_t s) {
    const long long total = (long long)a.n * a.half;
    if (total == 0) return cudaSuccess;
    const long long grid = (total + kThreads - 1) / kThreads;
    rope_table_kernel<<<(int)(grid > 16384 ? 16384 : grid), kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

// Tokens of one launch: thread numbers have 32 bits (a longer call is several launches)
static int tokens_at_once(long long threads_per_token) {
    const long long most = 0xf0000000ll / (threads_per_token < 1 ? 1 : threads_per_token);
    return most > 0x7fffffff ? 0x7fffffff : (int)most;
}
static const void *moved(const void *p, int64_t elements, int dtype) { return (const uint8_t *)p + elements * (dtype == MOE_BF16 ? 2 : 4); }

cudaError_t launch_rope(const RopeArgs &all, int sm_count, cudaStream_t s, uint64_t *launches) {
    const bool rows16 = aligned(all.x.p, all.x.ts, all.x.hs, all.dtype) && aligned(all.y, all.yts, all.yhs, all.dtype);
    const Walk walk = walk_of(all.D, all.turn, rows16, all.x.p == all.y);
    const int units = units_of(walk, all.D, all.turn.rot);
    const int per = heads_per_thread((long long)all.T * all.H * units, sm_count), groups = (all.H + per - 1) / per;
    const bool t16 = table16(all.turn);
    auto k = all.dtype == MOE_BF16 ? rope_of<__nv_bfloat16>(walk, t16) : rope_of<float>(walk, t16);
    const int step = tokens_at_once((long long)groups * units);
    for (int t0 = 0; t0 < all.T; t0 += step) {
        RopeArgs a = all;
        a.T = all.T - t0 < step ? all.T - t0 : step;
        a.x.p = moved(all.x.p, t0 * all.x.ts, all.dtype);
        a.y = (void *)moved(all.y, t0 * all.yts, all.dtype);
        a.turn.position += t0;
        const cudaError_t err = launch_chained(k, dim3((unsigned)(((long long)a.T * groups * units + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, true, a, FastDiv(units),
                                               FastDiv(groups), per);
        if (err != cudaSuccess) return err;
        ++*launches;
    }
    return cudaSuccess;
}

cudaError_t launch_append(const AppendArgs &all, int sm_count, cudaStream_t s, uint64_t *launches) {
    const bool q16 = !all.q.p || (aligned(all.q.p, all.q.ts, all.q.hs, all.dtype) && aligned(all.q_out, (int64_t)all.H * all.D, all.D, all.dtype));
    const Walk walk = walk_of(all.D, all.turn, q16, all.q.p == all.q_out);
    const int units = units_of(walk, all.D, all.turn.rot);
    const int per = heads_per_thread((long long)all.T * all.H * units, sm_count), groups = (all.H + per - 1) / per;
    // nothing to do where the queries stay as they are, in place
    const bool q_moves = all.q.p && (all.turn.rot || all.q.p != all.q_out);
    const bool vec = table16(all.turn) && aligned(all.k.p, all.k.ts, all.k.hs, all.dtype) && aligned(all.v.p, all.v.ts, all.v.hs, all.dtype);
    const int w = padded_width(all.D);
    auto k = all.dtype == MOE_BF16 ? append_of<__nv_bfloat16>(w, walk, vec) : append_of<float>(w, walk, vec);
    const int step = tokens_at_once((long long)groups * units + 1ll * all.Hk * (w / 8));
    for (int t0 = 0; t0 < all.T; t0 += step) {
        AppendArgs a = all;
        a.T = all.T - t0 < step ? all.T - t0 : step;
        a.k.p = moved(all.k.p, t0 * all.k.ts, all.dtype);
        a.v.p = moved(all.v.p, t0 * all.v.ts, all.dtype);
        a.slot += t0;
        if (a.turn.rot) a.turn.position += t0;
        if (a.q.p) {
            a.q.p = moved(all.q.p, t0 * all.q.ts, all.dtype);
            a.q_out = (void *)moved(all.q_out, (int64_t)t0 * all.H * all.D, all.dtype);
        }
        const long long qc = q_moves ? ((long long)a.T * groups * units + kThreads - 1) / kThreads : 0;
        const long long sc = ((long long)a.T * a.Hk * (w / 8) + kThreads - 1) / kThreads;
        // ceil(2^32 sc / (qc + sc)): f(qc + sc) = sc exactly; all ones where nothing turns
        const uint32_t ratio = qc == 0 ? 0xffffffffu : (uint32_t)((((unsigned long long)sc << 32) + qc + sc - 1) / (qc + sc));
        const cudaError_t err = launch_chained(k, dim3((unsigned)(qc + sc)), dim3(kThreads), 0, s, true, a, ratio, FastDiv(units), FastDiv(groups), per, FastDiv(a.Hk));
        if (err != cudaSuccess) return err;
        ++*launches;
    }
    return cudaSuccess;
}

cudaError_t launch_read(const ReadArgs &all, cudaStream_t s, uint64_t *launches) {
    if (!all.k && !all.v) return cudaSuccess;
    const int chunks = all.D / 8, w = padded_width(all.D);
    auto k = all.dtype == MOE_BF16 ? (w == 64 ? read_kernel<__nv_bfloat16, 64> : w == 128 ? read_kernel<__nv_bfloat16, 128> : read_kernel<__nv_bfloat16, 256>)
                                   : (w == 64 ? read_kernel<float, 64> : w == 128 ? read_kernel<float, 128> : read_kernel<float, 256>);
    const int step = tokens_at_once((long long)all.Hk * chunks);
    for (int t0 = 0; t0 < all.T; t0 += step) {
        ReadArgs a = all;
        a.T = all.T - t0 < step ? all.T - t0 : step;
        a.slot += t0;
        if (a.k) a.k = (void *)moved(all.k, (int64_t)t0 * all.Hk * all.D, all.dtype);
        if (a.v) a.v = (void *)moved(all.v, (int64_t)t0 * all.Hk * all.D, all.dtype);
        const cudaError_t err = launch_chained(k, dim3((unsigned)(((long long)a.T * a.Hk * chunks + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, true, a, FastDiv(chunks),
                                               FastDiv(a.Hk));
        if (err != cudaSuccess) return err;
        ++*launches;
    }
    return cudaSuccess;
}

}  // namespace kv
}  // namespace lexi
