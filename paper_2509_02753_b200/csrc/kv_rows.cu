// Rotary positions, storing rows in 4 bits, and reading them back.
#include <math.h>

#include "kv_internal.h"

namespace lexi {
namespace kv {
namespace {

constexpr int kThreads = 256;

// ------------------------------------------------------------------ angles
// theta_i in 64 bits: at position 10^6 an angle in 32 bits would be off by 0.06
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

// A unit of a row's work: 8 pairs that turn (two stretches of 8 dimensions in the half layout, 16 neighbouring ones in
// the pairs layout), or up to 8 dimensions behind rope_dim that pass.  Both ends of a pair are one thread's, so a call
// can work in place.  The same unit of several heads shares the angles.
struct Units { int turning, passing; };
__host__ __device__ inline Units units_of(int D, int rot) { return Units{(rot / 2 + 7) / 8, (D - rot + 7) / 8}; }

template <typename T, bool VEC>
__device__ __forceinline__ void turn_unit(const T *x, T *y, int D, const Turn &tn, bool turns, int unit,
                                          const Units &un, const float2 (&cs)[8]) {
    const int half = tn.rot / 2;
    float a[8], b[8];
    if (unit < un.turning) {
        const int i0 = unit * 8, n = min(8, half - i0);
        if (tn.layout == MOE_ROPE_HALF) {
            load8<VEC>(x + i0, n, a);
            load8<VEC>(x + half + i0, n, b);
            if (turns) {
#pragma unroll
                for (int i = 0; i < 8; ++i) turn(a[i], b[i], cs[i]);
            }
            store8<VEC>(y + i0, n, a);
            store8<VEC>(y + half + i0, n, b);
        } else {
            load8<VEC>(x + 2 * i0, 2 * n, a);
            load8<VEC>(x + 2 * i0 + 8, 2 * n - 8, b);
            if (turns) {
#pragma unroll
                for (int i = 0; i < 4; ++i) { turn(a[2 * i], a[2 * i + 1], cs[i]); turn(b[2 * i], b[2 * i + 1], cs[i + 4]); }
            }
            store8<VEC>(y + 2 * i0, 2 * n, a);
            store8<VEC>(y + 2 * i0 + 8, 2 * n - 8, b);
        }
    } else if (x != y) {
        const int d = tn.rot + (unit - un.turning) * 8, n = min(8, D - d);
        load8<VEC>(x + d, n, a);
        store8<VEC>(y + d, n, a);
    }
}

// cos and sin of the unit's pairs; false: the position is outside the table (the row then stays unturned)
__device__ __forceinline__ bool unit_angles(const Turn &tn, int t, int unit, const Units &un, float2 (&cs)[8], int32_t *status) {
    if (unit >= un.turning) return false;
    const int p = tn.position[t], half = tn.rot / 2, i0 = unit * 8;
    if (p < 0 || p >= tn.n_positions) { atomicOr(status, MOE_KV_STATUS_BAD_INDEX); return false; }
    const float2 *row = tn.table + (int64_t)p * half + i0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        cs[i] = i0 + i < half ? row[i] : make_float2(1.f, 0.f);
        if (tn.inverse) cs[i].y = -cs[i].y;
    }
    return true;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs a, int groups, int per_group) {
    const Units un = units_of(a.D, a.turn.rot);
    const int nu = un.turning + un.passing;
    const long long e = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (e >= (long long)a.T * groups * nu) return;
    const int unit = (int)(e % nu), grp = (int)(e / nu % groups), t = (int)(e / nu / groups);
    float2 cs[8];
    const bool turns = unit_angles(a.turn, t, unit, un, cs, a.status);
    const int h1 = min(a.H, (grp + 1) * per_group);
    for (int h = grp * per_group; h < h1; ++h)
        turn_unit<T, VEC>((const T *)a.x.p + t * a.x.ts + h * a.x.hs, (T *)a.y + t * a.yts + h * a.yhs, a.D, a.turn, turns, unit, un, cs);
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

// 16 numbers of a group -> 8 bytes of codes and the scale byte
__device__ __forceinline__ uint2 quantise(float (&x)[16], float inv6, float scale, uint32_t &s8, int32_t *status) {
    float top = 0.f;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        if (!(fabsf(x[i]) <= 3.4028234663852886e38f)) {          // NaN -> 0, infinity -> the largest number
            x[i] = x[i] != x[i] ? 0.f : copysignf(3.4028234663852886e38f, x[i]);
            odd = true;
        }
        top = fmaxf(top, fabsf(x[i]));
    }
    if (odd) atomicOr(status, MOE_KV_STATUS_NONFINITE);
    s8 = to_e4m3(fminf(__fmul_rn(top, inv6), 448.f));
    const float s = __fmul_rn(from_e4m3(s8), scale);
    const float inv = s > 0.f ? __frcp_rn(s) : 0.f;
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2] |= to_e2m1_pair(__fmul_rn(x[2 * i], inv), __fmul_rn(x[2 * i + 1], inv)) << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
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
    const float2 cs = cs_row[i];
    if (second) { turn(w, u, cs); return u; }
    turn(u, w, cs);
    return u;
}

// 16 dimensions d0.. of a key row, turned; VEC: every stretch of 8 is aligned and turns or passes as a whole
template <typename T, bool VEC>
__device__ __forceinline__ void key_group(const T *row, int D, int d0, const Turn &tn, const float2 *cs_row, float (&x)[16]) {
    if (VEC) {
        const int half = tn.rot / 2;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const int d = d0 + 8 * part;
            float a[8], b[8];
            if (d >= D) {
#pragma unroll
                for (int i = 0; i < 8; ++i) a[i] = 0.f;
            } else {
                load8<true>(row + d, 8, a);
                if (cs_row && d < tn.rot) {
                    if (tn.layout == MOE_ROPE_HALF) {
                        const bool second = d >= half;
                        const float2 *cs = cs_row + (second ? d - half : d);
                        load8<true>(row + (second ? d - half : d + half), 8, b);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            if (second) turn(b[i], a[i], cs[i]); else turn(a[i], b[i], cs[i]);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) turn(a[2 * i], a[2 * i + 1], cs_row[d / 2 + i]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) x[8 * part + i] = a[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = d0 + i < D ? turned_at(row, tn, cs_row, d0 + i) : 0.f;
    }
}

// Address of a slot's block; nullptr for a slot that is not stored
__device__ __forceinline__ uint8_t *block_of(uint8_t *cache, int64_t slot, int64_t n_slots, int page, int Hk, int h, int W, int32_t *status) {
    if (slot < 0 || slot >= n_slots) {
        if (slot != -1) atomicOr(status, MOE_KV_STATUS_BAD_INDEX);
        return nullptr;
    }
    const int64_t pg = slot / page;
    const int in = (int)(slot - pg * page);
    return cache + ((pg * Hk + h) * (page / kBlockTokens) + in / kBlockTokens) * (int64_t)block_bytes(W);
}

// One launch, three stretches of CTAs: queries turn (units as in rope_kernel), keys turn and are stored, values are
// stored.  A thread stores one group of 16 dimensions: 8 bytes of codes and a scale.  Neighbouring threads take the
// groups of one key row (its codes are neighbours in a block) but the same stretch of 16 tokens' value rows (which are
// neighbours there), so both write whole sectors.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) append_kernel(AppendArgs a, int q_ctas, int k_ctas, int groups, int per_group, int W) {
    const int ng = W / 16;
    if ((int)blockIdx.x < q_ctas) {
        const Units un = units_of(a.D, a.turn.rot);
        const int nu = un.turning + un.passing;
        const long long e = (long long)blockIdx.x * kThreads + threadIdx.x;
        if (e >= (long long)a.T * groups * nu) return;
        const int unit = (int)(e % nu), grp = (int)(e / nu % groups), t = (int)(e / nu / groups);
        float2 cs[8];
        const bool turns = unit_angles(a.turn, t, unit, un, cs, a.status);
        const int h1 = min(a.H, (grp + 1) * per_group);
        for (int h = grp * per_group; h < h1; ++h)
            turn_unit<T, VEC>((const T *)a.q.p + t * a.q.ts + h * a.q.hs, (T *)a.q_out + ((int64_t)t * a.H + h) * a.D, a.D, a.turn, turns, unit, un, cs);
        return;
    }
    const bool key = (int)blockIdx.x < q_ctas + k_ctas;
    const long long e = (long long)(blockIdx.x - q_ctas - (key ? 0 : k_ctas)) * kThreads + threadIdx.x;
    int g, h;
    long long t;
    if (key) {
        g = (int)(e % ng); h = (int)(e / ng % a.Hk); t = e / ng / a.Hk;
    } else {
        const long long u = e / 16;
        g = (int)(u % ng); h = (int)(u / ng % a.Hk); t = u / ng / a.Hk * 16 + e % 16;
    }
    if (t >= a.T) return;
    const int64_t slot = a.slot[t];
    uint8_t *blk = block_of(a.cache, slot, a.n_slots, a.page, a.Hk, h, W, a.status);
    if (!blk) return;
    const int token = (int)(slot % kBlockTokens);
    float x[16];
    uint32_t s8;
    if (key) {
        const float2 *cs_row = nullptr;
        if (a.turn.rot) {
            const int p = a.turn.position[t];
            if (p >= 0 && p < a.turn.n_positions) cs_row = a.turn.table + (int64_t)p * (a.turn.rot / 2);
            else atomicOr(a.status, MOE_KV_STATUS_BAD_INDEX);
        }
        key_group<T, VEC>((const T *)a.k.p + t * a.k.ts + h * a.k.hs, a.D, g * 16, a.turn, cs_row, x);
        const uint2 c = quantise(x, a.k_inv6, a.k_scale, s8, a.status);
        *reinterpret_cast<uint2 *>(blk + token * (W / 2) + g * 8) = c;
        blk[k_scales_at(W) + token * ng + g] = (uint8_t)s8;
    } else {
        Turn still = a.turn;
        still.rot = 0;
        key_group<T, VEC>((const T *)a.v.p + t * a.v.ts + h * a.v.hs, a.D, g * 16, still, nullptr, x);
        const uint2 c = quantise(x, a.v_inv6, a.v_scale, s8, a.status);
        uint8_t *codes = blk + v_codes_at(W);
        const int vb = W / 16;
        if (W == 64) {
            *reinterpret_cast<uint32_t *>(codes + 2 * g * 64 + ((token * 4) ^ v_turn(64, 2 * g))) = c.x;
            *reinterpret_cast<uint32_t *>(codes + (2 * g + 1) * 64 + ((token * 4) ^ v_turn(64, 2 * g + 1))) = c.y;
        } else if (W == 128) {
            *reinterpret_cast<uint2 *>(codes + g * 128 + ((token * vb) ^ v_turn(128, g))) = c;
        } else {
            const int r = g >> 1;
            *reinterpret_cast<uint2 *>(codes + r * 256 + ((token * vb) ^ v_turn(256, r)) + (g & 1) * 8) = c;
        }
        blk[v_scales_at(W) + g * kBlockTokens + token] = (uint8_t)s8;
    }
}

// A thread reads one group of 16 dimensions of a key or value row
template <typename T>
__global__ void __launch_bounds__(kThreads) read_kernel(ReadArgs a, int W) {
    const int ng = (a.D + 15) / 16;
    const long long e = (long long)blockIdx.x * kThreads + threadIdx.x;
    const bool key = blockIdx.y == 0 && a.k != nullptr;
    const int g = (int)(e % ng), h = (int)(e / ng % a.Hk);
    const long long t = e / ng / a.Hk;
    if (t >= a.T) return;
    const int64_t slot = a.slot[t];
    const uint8_t *blk = block_of(const_cast<uint8_t *>(a.cache), slot, a.n_slots, a.page, a.Hk, h, W, a.status);
    uint2 c = make_uint2(0u, 0u);
    float s = 0.f;
    if (blk) {
        const int token = (int)(slot % kBlockTokens), vb = W / 16;
        if (key) {
            c = *reinterpret_cast<const uint2 *>(blk + token * (W / 2) + g * 8);
            s = from_e4m3(blk[k_scales_at(W) + token * (W / 16) + g]);
        } else {
            const uint8_t *codes = blk + v_codes_at(W);
            if (W == 64) {
                c.x = *reinterpret_cast<const uint32_t *>(codes + 2 * g * 64 + ((token * 4) ^ v_turn(64, 2 * g)));
                c.y = *reinterpret_cast<const uint32_t *>(codes + (2 * g + 1) * 64 + ((token * 4) ^ v_turn(64, 2 * g + 1)));
            } else if (W == 128) {
                c = *reinterpret_cast<const uint2 *>(codes + g * 128 + ((token * vb) ^ v_turn(128, g)));
            } else {
                const int r = g >> 1;
                c = *reinterpret_cast<const uint2 *>(codes + r * 256 + ((token * vb) ^ v_turn(256, r)) + (g & 1) * 8);
            }
            s = from_e4m3(blk[v_scales_at(W) + g * kBlockTokens + token]);
        }
    }
    const float scale = key ? a.k_scale : a.v_scale;
    T *out = (T *)(key ? a.k : a.v) + ((int64_t)t * a.Hk + h) * a.D + g * 16;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        const uint32_t w = part ? c.y : c.x;
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = from_e2m1_pair((w >> (8 * i)) & 0xffu);
            x[2 * i] = f.x * s * scale;          // code * s has at most 6 bits: one rounding
            x[2 * i + 1] = f.y * s * scale;
        }
        if (g * 16 + part * 8 < a.D) store8<true>(out + part * 8, 8, x);
    }
}

bool aligned(const void *p, int64_t ts, int64_t hs, int dtype) {
    const int64_t e = dtype == MOE_BF16 ? 8 : 4;
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ts % e == 0 && hs % e == 0;
}

// Stretches of 8 dimensions (8 pairs) that turn or pass as a whole
bool whole_units(int D, int rot) { return rot % 16 == 0 && D % 8 == 0; }

// Heads that share a thread's angles: 4 once there are enough threads for the machine without it
int heads_per_thread(long long threads, int sm_count) { return threads >= 4ll * 2048 * sm_count ? 4 : 1; }

}  // namespace

cudaError_t launch_rope_table(const RopeTableArgs &a, cudaStream_t s) {
    const long long total = (long long)a.n * a.half;
    if (total == 0) return cudaSuccess;
    const long long grid = (total + kThreads - 1) / kThreads;
    rope_table_kernel<<<(int)(grid > 16384 ? 16384 : grid), kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_rope(const RopeArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    const Units un = units_of(a.D, a.turn.rot);
    const int nu = un.turning + un.passing;
    const int per = heads_per_thread((long long)a.T * a.H * nu, sm_count), groups = (a.H + per - 1) / per;
    const long long grid = ((long long)a.T * groups * nu + kThreads - 1) / kThreads;
    if (grid == 0) return cudaSuccess;
    if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
    const bool vec = whole_units(a.D, a.turn.rot) && aligned(a.x.p, a.x.ts, a.x.hs, a.dtype) && aligned(a.y, a.yts, a.yhs, a.dtype);
    auto k = a.dtype == MOE_BF16 ? (vec ? rope_kernel<__nv_bfloat16, true> : rope_kernel<__nv_bfloat16, false>)
                                 : (vec ? rope_kernel<float, true> : rope_kernel<float, false>);
    k<<<(int)grid, kThreads, 0, s>>>(a, groups, per);
    ++*launches;
    return cudaGetLastError();
}

cudaError_t launch_append(const AppendArgs &a, int sm_count, cudaStream_t s, uint64_t *launches) {
    if (a.T == 0) return cudaSuccess;
    const int W = padded_width(a.D), ng = W / 16;
    const Units un = units_of(a.D, a.turn.rot);
    const int nu = un.turning + un.passing;
    const int per = heads_per_thread((long long)a.T * a.H * nu, sm_count), groups = (a.H + per - 1) / per;
    auto ctas = [](long long n) { return (n + kThreads - 1) / kThreads; };
    // nothing to do where the queries stay as they are, in place
    const bool q_moves = a.q.p && (a.turn.rot || a.q.p != a.q_out);
    const long long qc = q_moves ? ctas((long long)a.T * groups * nu) : 0;
    const long long kc = ctas((long long)a.T * a.Hk * ng), vc = ctas((long long)((a.T + 15) / 16 * 16) * a.Hk * ng);
    if (qc + kc + vc > 0x7fffffffll) return cudaErrorInvalidValue;
    bool vec = whole_units(a.D, a.turn.rot) && aligned(a.k.p, a.k.ts, a.k.hs, a.dtype) && aligned(a.v.p, a.v.ts, a.v.hs, a.dtype);
    if (a.q.p) vec = vec && aligned(a.q.p, a.q.ts, a.q.hs, a.dtype) && aligned(a.q_out, (int64_t)a.H * a.D, a.D, a.dtype);
    auto k = a.dtype == MOE_BF16 ? (vec ? append_kernel<__nv_bfloat16, true> : append_kernel<__nv_bfloat16, false>)
                                 : (vec ? append_kernel<float, true> : append_kernel<float, false>);
    k<<<(int)(qc + kc + vc), kThreads, 0, s>>>(a, (int)qc, (int)kc, groups, per, W);
    ++*launches;
    return cudaGetLastError();
}

cudaError_t launch_read(const ReadArgs &a, cudaStream_t s, uint64_t *launches) {
    if (a.T == 0 || (!a.k && !a.v)) return cudaSuccess;
    const long long grid = ((long long)a.T * a.Hk * ((a.D + 15) / 16) + kThreads - 1) / kThreads;
    if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
    auto k = a.dtype == MOE_BF16 ? read_kernel<__nv_bfloat16> : read_kernel<float>;
    k<<<dim3((unsigned)grid, a.k && a.v ? 2 : 1), kThreads, 0, s>>>(a, padded_width(a.D));
    ++*launches;
    return cudaGetLastError();
}

}  // namespace kv
}  // namespace lexi
