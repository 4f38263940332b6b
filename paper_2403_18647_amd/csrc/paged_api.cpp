// Host runtime of the paged cache: handle, workspace layout, argument checks (include/sdsat.h).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <new>
#include <string>

#include "../../include/sdsat.h"
#include "kernels.h"

using namespace sdsat;

struct sdsat_paged {
    sdsat_paged_config cfg;
    PagedPlan plan;
    hipStream_t stream = nullptr;
    int device = 0;
    std::string err = "no error";
    int* err_flag = nullptr;
    float* part = nullptr;
    size_t tile_part = 0;
};

namespace {

int fail(sdsat_paged* p, int code, const std::string& msg) {
    if (!p) return report_error(code, msg);
    p->err = msg;
    return code;
}

int launched(sdsat_paged* p, hipError_t e, const char* what) {
    return e == hipSuccess ? SDSAT_OK : fail(p, SDSAT_EDEVICE, std::string(what) + ": " + hipGetErrorString(e));
}

// The handle's device is the current one while this lives (the caller's may be another).
struct DeviceScope {
    int before = -1;
    explicit DeviceScope(int device) {
        int now = device;
        if (hipGetDevice(&now) == hipSuccess && now != device && hipSetDevice(device) == hipSuccess) before = now;
    }
    ~DeviceScope() { if (before >= 0) (void)hipSetDevice(before); }
};

constexpr int kMaxPagedBatch = 4096, kMaxPagedRows = 1 << 20, kMaxHeads = 1024, kMaxPagedCtx = 1 << 24;

int check_config(const sdsat_paged_config* c, std::string* why) {
    if (!c) { *why = "config is NULL"; return SDSAT_EINVAL; }
    if (c->n_heads < 1 || c->n_kv_heads < 1 || c->n_pages < 1 || c->max_rows < 1 || c->max_batch < 1 || c->max_ctx < 1) {
        *why = "config has a non-positive dimension";
        return SDSAT_EINVAL;
    }
    if (c->n_heads % c->n_kv_heads) { *why = "n_heads must be a multiple of n_kv_heads"; return SDSAT_EINVAL; }
    if (c->dtype != SDSAT_DTYPE_FP32 && c->dtype != SDSAT_DTYPE_BF16) { *why = "dtype must be 0 or 1"; return SDSAT_EINVAL; }
    if (c->head_dim != 64 && c->head_dim != 128) { *why = "head_dim must be 64 or 128"; return SDSAT_EUNSUPPORTED; }
    if (c->n_heads > kMaxHeads || c->max_batch > kMaxPagedBatch || c->max_rows > kMaxPagedRows || c->max_ctx > kMaxPagedCtx ||
        (int64_t)c->max_batch * c->n_kv_heads > kPagedMaxPairs) {
        *why = "n_heads <= 1024, max_batch <= 4096, max_batch * n_kv_heads <= 2^19, max_rows <= 2^20 and max_ctx <= 2^24 are supported";
        return SDSAT_EUNSUPPORTED;
    }
    return SDSAT_OK;
}

size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

// Offsets of the workspace's arrays and its size.
struct Layout { size_t part, bytes, tile_part; PagedPlan plan; };
Layout layout(const sdsat_paged_config& c) {
    Layout l{};
    l.plan = plan_paged(c.n_kv_heads, c.max_batch, c.max_ctx);
    l.part = 256;   // ahead of it the error flags
    l.bytes = l.part + align_up(4 * (4 + paged_part_floats(l.plan, c.n_heads, c.n_kv_heads, c.head_dim, c.max_batch, c.max_rows, &l.tile_part)));
    return l;
}

// A call's sequences, checked as far as the host can.
int check_batch(sdsat_paged* p, const sdsat_paged_batch* b, PagedSeqs* s) {
    const sdsat_paged_config& c = p->cfg;
    if (!b || !b->d_start || !b->d_len || !b->d_pages) return fail(p, SDSAT_EINVAL, "batch, or its d_start, d_len or d_pages, is NULL");
    if (b->batch < 1 || b->rows < 0 || b->max_q < 0 || b->max_len < 0 || b->pages_ld < 1)
        return fail(p, SDSAT_EINVAL, "batch or pages_ld below 1, or rows, max_q or max_len below 0");
    if (b->batch > c.max_batch) return fail(p, SDSAT_ECAPACITY, "batch exceeds max_batch");
    if (b->rows > c.max_rows) return fail(p, SDSAT_ECAPACITY, "rows exceed max_rows");
    if (b->max_len > c.max_ctx) return fail(p, SDSAT_ECAPACITY, "max_len exceeds max_ctx");
    if (b->max_q > b->max_len || b->max_q > b->rows)
        return fail(p, SDSAT_EINVAL, "max_q exceeds max_len (which counts the new tokens) or rows");
    if (b->max_len > (int64_t)b->pages_ld * kPage) return fail(p, SDSAT_ECAPACITY, "max_len exceeds 32 * pages_ld slots");
    *s = PagedSeqs{b->d_start, b->d_len, b->d_pages, b->batch, b->pages_ld, b->rows, b->max_q, b->max_len, c.n_pages, p->err_flag};
    return SDSAT_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

extern "C" {

int sdsat_rope_init(int32_t layout, int32_t rot_dims, double base, int32_t scaling, double factor, double ctx, double low,
                    double high, float mscale, sdsat_rope* out) {
    if (!out) return fail(nullptr, SDSAT_EINVAL, "out is NULL");
    if (layout != SDSAT_ROPE_HALF && layout != SDSAT_ROPE_INTERLEAVED) return fail(nullptr, SDSAT_EINVAL, "bad rotary layout");
    if (rot_dims < 0 || rot_dims > 2 * kMaxPairs || rot_dims % 8) return fail(nullptr, SDSAT_EUNSUPPORTED, "rot_dims must be a multiple of 8, at most 128");
    if (scaling < SDSAT_ROPE_PLAIN || scaling > SDSAT_ROPE_PARTS) return fail(nullptr, SDSAT_EINVAL, "bad rotary scaling");
    if (!(base > 0) || !std::isfinite(base) || !std::isfinite(mscale)) return fail(nullptr, SDSAT_EINVAL, "rotary base must be positive and finite, mscale finite");
    if (scaling != SDSAT_ROPE_PLAIN && (!(factor > 0) || !std::isfinite(factor))) return fail(nullptr, SDSAT_EINVAL, "rotary factor must be positive and finite");
    if (scaling == SDSAT_ROPE_PARTS && (!(ctx > 0) || !std::isfinite(ctx) || !std::isfinite(low) || !std::isfinite(high) || !(high > low)))
        return fail(nullptr, SDSAT_EINVAL, "scaling by parts needs ctx > 0 and high > low");
    std::memset(out, 0, sizeof(*out));
    out->layout = layout;
    out->rot_dims = rot_dims;
    out->mscale = mscale;
    const double two_pi = 6.283185307179586476925;
    if (scaling == SDSAT_ROPE_NTK && rot_dims > 0) base *= std::pow(factor, rot_dims / (rot_dims - 2.0));
    for (int j = 0; j < rot_dims / 2; ++j) {
        double f = std::pow(base, -2.0 * j / rot_dims);
        if (scaling == SDSAT_ROPE_LINEAR) f /= factor;
        if (scaling == SDSAT_ROPE_PARTS) {
            const double keep = std::fmin(std::fmax((ctx * f / two_pi - low) / (high - low), 0.0), 1.0);
            f = f / factor * (1.0 - keep) + f * keep;
        }
        out->turns[j] = f / two_pi;
    }
    return SDSAT_OK;
}

int sdsat_paged_query_sizes(const sdsat_paged_config* cfg, size_t* workspace_bytes) {
    if (!workspace_bytes) return fail(nullptr, SDSAT_EINVAL, "workspace_bytes is NULL");
    std::string why;
    const int rc = check_config(cfg, &why);
    if (rc) return fail(nullptr, rc, why);
    *workspace_bytes = layout(*cfg).bytes;
    return SDSAT_OK;
}

int sdsat_paged_init(const sdsat_paged_config* cfg, void* workspace, size_t workspace_bytes, void* hip_stream, sdsat_paged** out) {
    if (!out) return fail(nullptr, SDSAT_EINVAL, "out is NULL");
    *out = nullptr;
    std::string why;
    const int rc = check_config(cfg, &why);
    if (rc) return fail(nullptr, rc, why);
    if (!workspace || ((uintptr_t)workspace & 255)) return fail(nullptr, SDSAT_EINVAL, "workspace must be non-NULL and 256-byte aligned");
    const Layout l = layout(*cfg);
    if (workspace_bytes < l.bytes) return fail(nullptr, SDSAT_ENOMEM, "workspace smaller than sdsat_paged_query_sizes()");
    sdsat_paged* p = new (std::nothrow) sdsat_paged();
    if (!p) return fail(nullptr, SDSAT_ENOMEM, "host allocation failed");
    p->cfg = *cfg;
    p->plan = l.plan;
    p->stream = (hipStream_t)hip_stream;
    (void)hipGetDevice(&p->device);
    char* w = static_cast<char*>(workspace);
    p->err_flag = reinterpret_cast<int*>(w);
    p->part = reinterpret_cast<float*>(w + l.part);
    p->tile_part = l.tile_part;
    const hipError_t e = launch_fill_i32(p->err_flag, 1, 0, p->stream);
    if (e != hipSuccess || hipStreamSynchronize(p->stream) != hipSuccess) {
        delete p;
        return fail(nullptr, SDSAT_EDEVICE, "clearing the workspace failed");
    }
    *out = p;
    return SDSAT_OK;
}

int sdsat_paged_append(sdsat_paged* p, const sdsat_paged_batch* batch, void* d_k, void* d_v, const void* d_x, int32_t x_dtype,
                       int64_t ld_x, const sdsat_rope* rope, const int32_t* d_pos, const float* d_q_gain, const float* d_k_gain,
                       float eps, void* d_q, int64_t ld_q) {
    if (!p) return fail(nullptr, SDSAT_EINVAL, "paged is NULL");
    const DeviceScope scope(p->device);
    const sdsat_paged_config& c = p->cfg;
    PagedAppendArgs a{};
    const int rc = check_batch(p, batch, &a.seq);
    if (rc) return rc;
    if (!d_k || !d_v || !d_x || !d_q) return fail(p, SDSAT_EINVAL, "d_k, d_v, d_x or d_q is NULL");
    if (x_dtype != SDSAT_DTYPE_FP32 && x_dtype != SDSAT_DTYPE_BF16) return fail(p, SDSAT_EINVAL, "x_dtype must be 0 or 1");
    const int64_t dq = (int64_t)c.n_heads * c.head_dim, dkv = (int64_t)c.n_kv_heads * c.head_dim;
    if (ld_x < dq + 2 * dkv || ld_x % 8 || ld_q < dq || ld_q % 8)
        return fail(p, SDSAT_EINVAL, "ld_x or ld_q shorter than a row, or not a multiple of 8");
    if (!aligned16(d_k) || !aligned16(d_v) || !aligned16(d_x) || !aligned16(d_q))
        return fail(p, SDSAT_EINVAL, "d_k, d_v, d_x and d_q must be 16-byte aligned");
    if (!(eps >= 0.f)) return fail(p, SDSAT_EINVAL, "eps must be >= 0");
    if (rope) {
        if ((rope->layout != SDSAT_ROPE_HALF && rope->layout != SDSAT_ROPE_INTERLEAVED) || rope->rot_dims < 0 || rope->rot_dims % 8 ||
            rope->rot_dims > c.head_dim)
            return fail(p, SDSAT_EINVAL, "bad rotary layout, or rot_dims past head_dim");
        a.interleaved = rope->layout == SDSAT_ROPE_INTERLEAVED;
        a.rot = rope->rot_dims;
        a.mscale = rope->mscale;
        std::memcpy(a.turns, rope->turns, sizeof(a.turns));
    }
    if (!batch->max_q) return launched(p, launch_paged_check(a.seq, p->stream), "paged append");
    a.kp = d_k; a.vp = d_v; a.x = d_x; a.ldx = ld_x; a.qout = d_q; a.ldq = ld_q;
    a.pos = d_pos; a.q_gain = d_q_gain; a.k_gain = d_k_gain; a.eps = eps;
    a.H = c.n_heads; a.Hkv = c.n_kv_heads;
    return launched(p, launch_paged_append(c.dtype, x_dtype, c.head_dim, a, p->stream), "paged append");
}

int sdsat_paged_attention(sdsat_paged* p, const sdsat_paged_batch* batch, const void* d_k, const void* d_v, const void* d_q,
                          int64_t ld_q, const uint64_t* d_mask, int32_t window, float scale, void* d_out, int32_t out_dtype,
                          int64_t ld_out) {
    if (!p) return fail(nullptr, SDSAT_EINVAL, "paged is NULL");
    const DeviceScope scope(p->device);
    const sdsat_paged_config& c = p->cfg;
    PagedAttnArgs a{};
    const int rc = check_batch(p, batch, &a.seq);
    if (rc) return rc;
    if (!d_k || !d_v || !d_q || !d_out) return fail(p, SDSAT_EINVAL, "d_k, d_v, d_q or d_out is NULL");
    if (out_dtype != SDSAT_DTYPE_FP32 && out_dtype != c.dtype) return fail(p, SDSAT_EINVAL, "out_dtype must be fp32 or the cache's");
    const int64_t dq = (int64_t)c.n_heads * c.head_dim;
    if (ld_q < dq || ld_q % 8 || ld_out < dq || ld_out % 8)
        return fail(p, SDSAT_EINVAL, "ld_q or ld_out shorter than a row, or not a multiple of 8");
    if (!aligned16(d_k) || !aligned16(d_v) || !aligned16(d_q) || !aligned16(d_out))
        return fail(p, SDSAT_EINVAL, "d_k, d_v, d_q and d_out must be 16-byte aligned");
    if (window < 0) return fail(p, SDSAT_EINVAL, "window must be >= 0");
    if (d_mask && batch->max_q > 64) return fail(p, SDSAT_EUNSUPPORTED, "masks need max_q <= 64");
    if (d_mask && window) return fail(p, SDSAT_EUNSUPPORTED, "masks and a window cannot be combined");
    if (scale == 0.f) scale = (float)(1.0 / std::sqrt((double)c.head_dim));
    const float in2 = scale * 1.44269504f;   // log2 e
    if (!(in2 > 0.f) || !std::isfinite(in2)) return fail(p, SDSAT_EINVAL, "scale must be positive and finite (0: 1 / sqrt(head_dim))");
    if (!batch->max_q) return launched(p, launch_paged_check(a.seq, p->stream), "paged attention");
    PagedPlan plan = p->plan;
    plan_paged_call(plan, c.n_heads, c.n_kv_heads, batch->batch, batch->rows, batch->max_q, batch->max_len);
    a.kp = d_k; a.vp = d_v; a.q = d_q; a.ldq = ld_q; a.mask = d_mask; a.out = d_out; a.ldo = ld_out;
    a.out_f32 = out_dtype == SDSAT_DTYPE_FP32;
    a.H = c.n_heads; a.Hkv = c.n_kv_heads; a.window = window; a.scale = in2;
    a.part_shift = plan.part_shift; a.max_parts = plan.max_parts; a.tile_wgs = plan.tile_wgs; a.few_wgs = plan.few_wgs; a.few_once = plan.few_once;
    a.part = p->part; a.tile_part = p->tile_part;
    return launched(p, launch_paged_attention(c.dtype, c.head_dim, plan, a, p->stream), "paged attention");
}

int sdsat_paged_status(sdsat_paged* p) {
    if (!p) return fail(nullptr, SDSAT_EINVAL, "paged is NULL");
    const DeviceScope scope(p->device);
    int h = 0;
    hipError_t e = hipMemcpyAsync(&h, p->err_flag, 4, hipMemcpyDeviceToHost, p->stream);
    if (e == hipSuccess) e = hipStreamSynchronize(p->stream);
    if (e != hipSuccess) return launched(p, e, "paged status");
    if (!h) return SDSAT_OK;
    e = launch_fill_i32(p->err_flag, 1, 0, p->stream);
    if (e != hipSuccess) return launched(p, e, "paged status");
    return fail(p, SDSAT_EDATA, h & 4 ? "a sequence's rows or lengths do not fit what the call says of them" : "page out of range");
}

int sdsat_paged_destroy(sdsat_paged* p) {
    if (!p) return SDSAT_OK;
    const DeviceScope scope(p->device);
    (void)hipStreamSynchronize(p->stream);
    delete p;
    return SDSAT_OK;
}

const char* sdsat_paged_last_error(const sdsat_paged* p) { return p ? p->err.c_str() : sdsat_last_error(nullptr); }

}  // extern "C"
