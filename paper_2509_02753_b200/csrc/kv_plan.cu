// C ABI of the operators around the 4-bit key/value cache (include/moe_kv.h): plan, checks of arguments, launches.
#include <cmath>
#include <cstring>
#include <new>

#include "kv_internal.h"

using namespace lexi::kv;

struct moe_kv_plan {
    moe_kv_config_t cfg{};
    int device = 0, sm_count = 0;
    uint8_t *base = nullptr;          // one allocation
    uint64_t bytes = 0;
    uint64_t launches = 0;
    int32_t *status = nullptr, *arrived = nullptr;
    float *part = nullptr;
    float2 *part_ml = nullptr;
    float *prompt_part = nullptr;
    float2 *prompt_ml = nullptr;
    int32_t *prompt_arrived = nullptr;
    int32_t *status_host = nullptr;   // pinned
    int max_ctas = 0;
};

namespace {

constexpr int kMaxCtasPerSm = 8;
constexpr int64_t kMaxRows = 1 << 30;         // max_tokens * n_heads
constexpr int64_t kMaxContext = 1 << 30;      // tokens that a row of a block table may stand for
constexpr int kPartRows = 32;         // rows of a piece, at most
constexpr int kPassRows = 32;         // query rows of a pass over the keys in kv_attend.cu

size_t elem_size(int dtype) { return dtype == MOE_BF16 ? 2 : 4; }
bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
// arrays of 32-bit numbers; NULL is aligned
template <typename... P>
bool words(const P *...p) { return (aligned(p, 4) && ...); }

int check_config(const moe_kv_config_t *c) {
    if (!c) return MOE_ERR_INVALID_ARG;
    if (c->n_heads < 1 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads || c->max_requests < 1 || c->max_tokens < 1 ||
        (c->dtype != MOE_F32 && c->dtype != MOE_BF16)) return MOE_ERR_INVALID_ARG;
    if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 || c->n_heads > 1024 || c->max_requests > kMaxRequests ||
        (int64_t)c->max_tokens * c->n_heads > kMaxRows) return MOE_ERR_SHAPE;
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return MOE_ERR_SHAPE;
    return MOE_OK;
}

// rows of a call: the pointer is there and on the type's alignment
int check_rows(const moe_kv_rows_t *r, int dtype) {
    if (!r || !r->data) return MOE_ERR_INVALID_ARG;
    return aligned(r->data, elem_size(dtype)) ? MOE_OK : MOE_ERR_ALIGN;
}

int check_turn(const moe_kv_plan *p, int32_t tokens, const int32_t *position, const float *table, int32_t n_positions, int32_t rope_dim, int32_t layout) {
    if (rope_dim == 0) return MOE_OK;
    if (rope_dim < 0 || rope_dim % 2 || rope_dim > p->cfg.head_dim) return MOE_ERR_SHAPE;
    if (layout != MOE_ROPE_HALF && layout != MOE_ROPE_PAIRS) return MOE_ERR_INVALID_ARG;
    if (tokens == 0) return MOE_OK;
    if (!position || !table || n_positions < 1) return MOE_ERR_INVALID_ARG;
    return aligned(table, 8) && words(position) ? MOE_OK : MOE_ERR_ALIGN;
}

// log2 of a page's blocks
int page_shift(const moe_kv_config_t &c) { return c.page_size == 16 ? 0 : c.page_size == 32 ? 1 : c.page_size == 64 ? 2 : 3; }

bool good_scale(float s) { return s > 0.f && std::isnormal(s); }          // 1/(6 s) is finite

// The plan's device, for as long as it lives; whichever is current otherwise
struct OnDevice {
    int before = -1;
    explicit OnDevice(int device) {
        if (cudaGetDevice(&before) != cudaSuccess || before == device || cudaSetDevice(device) != cudaSuccess) before = -1;
    }
    ~OnDevice() { if (before >= 0) cudaSetDevice(before); }
};

int done(cudaError_t err) {
    if (err == cudaSuccess) return MOE_OK;
    cudaGetLastError();
    return MOE_ERR_CUDA;
}

}  // namespace

extern "C" {

int moe_kv_plan_create(const moe_kv_config_t *cfg, moe_kv_plan_t **out) {
    if (!out) return MOE_ERR_INVALID_ARG;
    *out = nullptr;
    if (const int rc = check_config(cfg)) return rc;
    int dev = 0, major = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        major != 10 || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return MOE_ERR_CUDA;
    }
    moe_kv_plan *p = new (std::nothrow) moe_kv_plan;
    if (!p) return MOE_ERR_WORKSPACE;
    p->cfg = *cfg;
    p->device = dev;
    p->sm_count = sms;
    p->max_ctas = sms * kMaxCtasPerSm;
    const size_t part = (size_t)p->max_ctas * attend_part_floats(padded_width(cfg->head_dim)) * sizeof(float);
    const size_t ml = (size_t)p->max_ctas * 2 * kPartRows * sizeof(float2);
    const size_t arrived = ((size_t)p->max_ctas * sizeof(int32_t) + 255) & ~size_t(255);
    // prompts: two pieces for each SM, whose grid that is
    const size_t ppart = (size_t)sms * prompt_part_floats(padded_width(cfg->head_dim)) * sizeof(float);
    const size_t pml = (size_t)sms * prompt_part_rows() * sizeof(float2);
    const size_t parrived = ((size_t)sms * sizeof(int32_t) + 255) & ~size_t(255);
    p->bytes = part + ml + ppart + pml + arrived + parrived + 256;
    void *mem = nullptr;
    if (cudaMalloc(&mem, p->bytes) != cudaSuccess || cudaMallocHost((void **)&p->status_host, 4) != cudaSuccess) {
        cudaGetLastError();
        if (mem) cudaFree(mem);
        delete p;
        return MOE_ERR_WORKSPACE;
    }
    p->base = (uint8_t *)mem;
    p->part = (float *)mem;
    p->part_ml = (float2 *)(p->base + part);
    p->prompt_part = (float *)(p->base + part + ml);
    p->prompt_ml = (float2 *)(p->base + part + ml + ppart);
    uint8_t *words = p->base + part + ml + ppart + pml;
    p->arrived = (int32_t *)words;
    p->prompt_arrived = (int32_t *)(words + arrived);
    p->status = (int32_t *)(words + arrived + parrived);
    if (cudaMemset(words, 0, arrived + parrived + 256) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
        cudaGetLastError();
        moe_kv_plan_destroy(p);
        return MOE_ERR_CUDA;
    }
    *out = p;
    return MOE_OK;
}

int moe_kv_plan_destroy(moe_kv_plan_t *p) {
    if (!p) return MOE_OK;
    {
        const OnDevice on(p->device);
        cudaDeviceSynchronize();
        cudaFree(p->base);
    }
    cudaFreeHost(p->status_host);
    cudaGetLastError();
    delete p;
    return MOE_OK;
}

uint64_t moe_kv_plan_workspace_bytes(const moe_kv_plan_t *p) { return p ? p->bytes : 0; }
uint64_t moe_kv_plan_launch_count(const moe_kv_plan_t *p) { return p ? p->launches : 0; }

uint64_t moe_kv_page_bytes(const moe_kv_config_t *cfg) {
    if (check_config(cfg) != MOE_OK) return 0;
    return (uint64_t)cfg->n_kv_heads * (cfg->page_size / kBlockTokens) * block_bytes(padded_width(cfg->head_dim));
}

int moe_kv_device_status(moe_kv_plan_t *p, int32_t *bits, void *stream) {
    if (!p) return MOE_ERR_INVALID_ARG;
    const OnDevice on(p->device);          // a stream of NULL is this device's
    cudaStream_t s = (cudaStream_t)stream;
    if (cudaMemcpyAsync(p->status_host, p->status, 4, cudaMemcpyDeviceToHost, s) != cudaSuccess ||
        cudaMemsetAsync(p->status, 0, 4, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
        cudaGetLastError();
        return MOE_ERR_CUDA;
    }
    const int32_t b = *p->status_host;
    if (bits) *bits = b;
    return b & MOE_KV_STATUS_TIMEOUT ? MOE_ERR_TIMEOUT : b ? MOE_ERR_DEVICE_CHECK : MOE_OK;
}

int moe_kv_tables(moe_kv_plan_t *p, const int32_t *ctx_len, const int32_t *new_len, int32_t n, const int32_t *free_pages, int32_t n_free,
                  int32_t *block_table, int32_t width, int32_t n_tokens, int32_t *kv_len, int32_t *cu_new, int32_t *position,
                  int64_t *slot, int32_t *taken, void *stream) {
    if (!p || n < 0 || n > p->cfg.max_requests || n_tokens < 0 || n_tokens > p->cfg.max_tokens || n_free < 0 || width < 0 || !cu_new || !taken)
        return MOE_ERR_INVALID_ARG;
    if (n > 0 && (!ctx_len || !new_len || !kv_len || (width > 0 && !block_table))) return MOE_ERR_INVALID_ARG;
    if ((n_free > 0 && !free_pages) || (n_tokens > 0 && (!position || !slot))) return MOE_ERR_INVALID_ARG;
    if (!words(ctx_len, new_len, free_pages, block_table, kv_len, cu_new, position, taken) || !aligned(slot, 8)) return MOE_ERR_ALIGN;
    TablesArgs a{ctx_len, new_len, n, free_pages, n_free, block_table, width, page_shift(p->cfg) + 4, n_tokens,
                 kv_len, cu_new, position, slot, taken, p->status};
    return done(launch_tables(a, p->sm_count, (cudaStream_t)stream, &p->launches));
}

int moe_rope_table(const moe_rope_config_t *c, int32_t n, float *table, void *stream) {
    if (!c || n < 0 || c->rope_dim < 2 || c->rope_dim % 2 || c->rope_dim > 256 || c->scaling < MOE_ROPE_PLAIN || c->scaling > MOE_ROPE_BANDS ||
        !(c->base > 0) || !(c->factor >= 1) || !(c->magnitude >= 0) || !std::isfinite(c->base) || !std::isfinite(c->factor) || !std::isfinite(c->magnitude))
        return MOE_ERR_INVALID_ARG;
    if (c->scaling >= MOE_ROPE_PARTS && (!(c->low > 0) || !(c->high > c->low) || !std::isfinite(c->high) || !(c->original_context > 0) ||
                                         !std::isfinite(c->original_context) || c->base == 1.0)) return MOE_ERR_INVALID_ARG;
    if (n == 0) return MOE_OK;
    if (!table) return MOE_ERR_INVALID_ARG;
    if (!aligned(table, 8)) return MOE_ERR_ALIGN;
    double magnitude = c->magnitude;
    if (magnitude == 0) magnitude = c->scaling == MOE_ROPE_PARTS ? 0.1 * std::log(c->factor) + 1.0 : 1.0;
    RopeTableArgs a{n, c->rope_dim / 2, c->base, c->factor, c->low, c->high, c->original_context, magnitude, c->scaling, (float2 *)table};
    return done(launch_rope_table(a, (cudaStream_t)stream));
}

int moe_rope(moe_kv_plan_t *p, const moe_kv_rows_t *x, int32_t T, int32_t H, const int32_t *position, const float *table, int32_t n_positions,
             int32_t rope_dim, int32_t layout, int32_t inverse, void *y, int64_t yts, int64_t yhs, void *stream) {
    if (!p || T < 0 || T > p->cfg.max_tokens || H < 1 || H > 1024 || (inverse != 0 && inverse != 1)) return MOE_ERR_INVALID_ARG;
    if (rope_dim < 2) return MOE_ERR_SHAPE;
    if (const int rc = check_turn(p, T, position, table, n_positions, rope_dim, layout)) return rc;
    if (T == 0) return MOE_OK;
    if (const int rc = check_rows(x, p->cfg.dtype)) return rc;
    if (!y) return MOE_ERR_INVALID_ARG;
    if (!aligned(y, elem_size(p->cfg.dtype))) return MOE_ERR_ALIGN;
    RopeArgs a{p->cfg.dtype, Rows{x->data, x->token_stride, x->head_stride}, T, H, p->cfg.head_dim,
               Turn{position, (const float2 *)table, n_positions, rope_dim, layout, inverse}, y, yts, yhs, p->status};
    return done(launch_rope(a, p->sm_count, (cudaStream_t)stream, &p->launches));
}

int moe_kv_append(moe_kv_plan_t *p, const moe_kv_rows_t *q, const moe_kv_rows_t *k, const moe_kv_rows_t *v, int32_t T, const int32_t *position,
                  const float *table, int32_t n_positions, int32_t rope_dim, int32_t layout, const int64_t *slot, float k_scale, float v_scale,
                  void *q_out, void *cache, int32_t n_pages, void *stream) {
    if (!p || T < 0 || T > p->cfg.max_tokens || n_pages < 0 || !good_scale(k_scale) || !good_scale(v_scale)) return MOE_ERR_INVALID_ARG;
    if (const int rc = check_turn(p, T, position, table, n_positions, rope_dim, layout)) return rc;
    if (T == 0) return MOE_OK;
    const moe_kv_config_t &c = p->cfg;
    if (const int rc = check_rows(k, c.dtype)) return rc;
    if (const int rc = check_rows(v, c.dtype)) return rc;
    Rows qr{nullptr, 0, 0};
    if (q && q->data) {
        if (const int rc = check_rows(q, c.dtype)) return rc;
        if (!q_out) return MOE_ERR_INVALID_ARG;
        if (!aligned(q_out, elem_size(c.dtype))) return MOE_ERR_ALIGN;
        qr = Rows{q->data, q->token_stride, q->head_stride};
    }
    if (!slot || !cache) return MOE_ERR_INVALID_ARG;
    if (!aligned(cache, 16) || !aligned(slot, 8)) return MOE_ERR_ALIGN;
    AppendArgs a{c.dtype, qr, Rows{k->data, k->token_stride, k->head_stride}, Rows{v->data, v->token_stride, v->head_stride}, T,
                 c.n_heads, c.n_kv_heads, c.head_dim, page_shift(c) + 4, Turn{position, (const float2 *)table, n_positions, rope_dim, layout, 0},
                 slot, k_scale, v_scale, (float)(1.0 / (6.0 * (double)k_scale)), (float)(1.0 / (6.0 * (double)v_scale)), q_out,
                 (uint8_t *)cache, (int64_t)n_pages * c.page_size, p->status};
    return done(launch_append(a, p->sm_count, (cudaStream_t)stream, &p->launches));
}

int moe_kv_read(moe_kv_plan_t *p, const void *cache, int32_t n_pages, const int64_t *slot, int32_t T, float k_scale, float v_scale,
                void *k, void *v, void *stream) {
    if (!p || T < 0 || T > p->cfg.max_tokens || n_pages < 0 || !good_scale(k_scale) || !good_scale(v_scale)) return MOE_ERR_INVALID_ARG;
    if (T == 0 || (!k && !v)) return MOE_OK;
    if (!slot || !cache) return MOE_ERR_INVALID_ARG;
    if (!aligned(cache, 16) || !aligned(slot, 8) || !aligned(k, 16) || !aligned(v, 16)) return MOE_ERR_ALIGN;
    const moe_kv_config_t &c = p->cfg;
    ReadArgs a{c.dtype, (const uint8_t *)cache, (int64_t)n_pages * c.page_size, slot, T, c.n_kv_heads, c.head_dim, page_shift(c) + 4,
               k_scale, v_scale, k, v, p->status};
    return done(launch_read(a, (cudaStream_t)stream, &p->launches));
}

int moe_kv_attention(moe_kv_plan_t *p, const moe_kv_rows_t *q, int32_t T, const int32_t *cu_new, const int32_t *kv_len, int32_t n, int32_t max_new,
                     const int32_t *block_table, int32_t width, const void *cache, int32_t n_pages, float softmax_scale, float k_scale,
                     float v_scale, int32_t window, int32_t sinks, void *out, void *stream) {
    if (!p || T < 0 || T > p->cfg.max_tokens || n < 0 || n > p->cfg.max_requests || max_new < 0 || width < 0 || n_pages < 0 || window < 0 || sinks < 0 ||
        !std::isfinite(softmax_scale) || !good_scale(k_scale) || !good_scale(v_scale)) return MOE_ERR_INVALID_ARG;
    const moe_kv_config_t &c = p->cfg;
    if ((int64_t)width * c.page_size > kMaxContext) return MOE_ERR_SHAPE;
    if (T == 0 || n == 0) return MOE_OK;
    if (const int rc = check_rows(q, c.dtype)) return rc;
    if (!cu_new || !kv_len || !out || (width > 0 && !block_table) || (n_pages > 0 && !cache)) return MOE_ERR_INVALID_ARG;
    if (!aligned(cache, 16) || !aligned(out, 16) || !words(cu_new, kv_len, block_table)) return MOE_ERR_ALIGN;
    AttendArgs a{};
    a.dtype = c.dtype; a.q = Rows{q->data, q->token_stride, q->head_stride}; a.T = T; a.cu = cu_new; a.kv_len = kv_len; a.n = n; a.max_new = max_new;
    a.table = block_table; a.width = width; a.cache = (const uint8_t *)cache; a.n_pages = n_pages;
    a.H = c.n_heads; a.Hk = c.n_kv_heads; a.G = c.n_heads / c.n_kv_heads; a.D = c.head_dim; a.g_div = FastDiv((uint32_t)a.G); a.page_shift = page_shift(c);
    a.score_scale = (float)((double)softmax_scale * k_scale * 1.4426950408889634);
    a.v_scale = v_scale; a.out = out;
    // no position reaches kMaxContext, and sums of these stay below 2^31
    a.window = window < kMaxContext ? window : (int)kMaxContext; a.sinks = sinks < kMaxContext ? sinks : (int)kMaxContext;
    a.part = p->part; a.part_ml = p->part_ml; a.arrived = p->arrived; a.max_ctas = p->max_ctas; a.status = p->status;
    a.prompt_part = p->prompt_part; a.prompt_ml = p->prompt_ml; a.prompt_arrived = p->prompt_arrived;
    cudaStream_t s = (cudaStream_t)stream;
    // Which kernel.  One pass over the keys serves 32 rows in kv_attend.cu (16 of wide heads); more rows read them again
    // there, while kv_prompt.cu has tiles of 128.  Measured at 8 key/value heads of 128 dimensions, 36 rows each: 16 requests
    // of 2000 keys 69 us there, 57 here; 64 dimensions 46 and 41; 256 dimensions, 36 rows 95 and 102, 64 rows 117 and 106;
    // in fp32, 68 rows, 241 and 156, and one request of 16000 keys 121 and 123.
    // While all of its work is about one step of every warp kv_attend.cu is faster whatever the rows (one request of 500
    // keys, 256 rows: 22 us and 31).
    const int most = max_new > 0 && max_new < T ? max_new : T;
    const long long rows = (long long)most * a.G, strips = (rows + kPassRows - 1) / kPassRows * n * a.Hk;
    const bool one_step = strips * (((long long)width * c.page_size + kBlockTokens - 1) / kBlockTokens) <= 32ll * p->sm_count;
    const int limit = padded_width(c.head_dim) == 256 ? 2 * kPassRows : kPassRows;
    if (rows <= limit || one_step) return done(launch_attend_rows(a, p->sm_count, s, &p->launches));
    // requests of one size, whichever it is, all go to the one kernel; otherwise each to its own
    const bool alike = (long long)n * most == T;
    a.prompt_rows = alike ? 0 : limit;
    const cudaError_t err = launch_attend_prompt(a, p->sm_count, s, &p->launches);
    if (err != cudaSuccess || alike) return done(err);
    return done(launch_attend_rows(a, p->sm_count, s, &p->launches));
}

}  // extern "C"
