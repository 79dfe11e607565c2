// Rotary positions and the paged key / value cache: the rotary table, and the step that rotates the new rows' queries and keys and appends
// keys and values.
#include "paged.h"

#include <math.h>

namespace atts {

int32_t check_paged(const char* fn, const atts_paged_cache* cache, PagedView* view) {
    if (!cache) return fail(ATTS_ERR_INVALID_ARG, "%s: cache is NULL", fn);
    const atts_paged_cache& c = *cache;
    if (c.dtype != ATTS_DTYPE_F32 && c.dtype != ATTS_DTYPE_BF16) return fail(ATTS_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, c.dtype);
    if (c.n_pages < 1 || c.n_kv_heads < 1 || c.n_seqs < 0 || c.max_pages < 1)
        return fail(ATTS_ERR_INVALID_ARG, "%s: need n_pages, n_kv_heads and max_pages >= 1 and n_seqs >= 0", fn);
    if (c.page_rows < 8 || c.page_rows > 4096 || (c.page_rows & (c.page_rows - 1)))
        return fail(ATTS_ERR_SHAPE, "%s: page_rows = %d is not a power of two in [8, 4096]", fn, c.page_rows);
    if (c.head_dim < 8 || c.head_dim > 256 || c.head_dim % 8) return fail(ATTS_ERR_SHAPE, "%s: head_dim = %d is not a multiple of 8 up to 256", fn, c.head_dim);
    if ((int64_t)c.max_pages * c.page_rows > (1 << 30)) return fail(ATTS_ERR_SHAPE, "%s: max_pages page_rows exceeds 2^30", fn);
    if (!c.k_pages || !c.v_pages || (c.n_seqs > 0 && !c.page_table)) return fail(ATTS_ERR_INVALID_ARG, "%s: NULL in the cache", fn);
    if (((uintptr_t)c.k_pages | (uintptr_t)c.v_pages) & 15) return fail(ATTS_ERR_INVALID_ARG, "%s: the pages must be 16-byte aligned", fn);
    int log = 3;
    while ((1 << log) < c.page_rows) ++log;
    *view = PagedView{c.page_table, c.n_pages, log, c.n_kv_heads, c.head_dim, c.n_seqs, c.max_pages};
    return ATTS_OK;
}

namespace {

struct RotaryScaling {
    int32_t kind, half;
    double log_theta_over_half, factor, original, low, high, magnitude;
};

__global__ void rotary_table_kernel(float2* __restrict__ table, int64_t first, int64_t n, RotaryScaling s) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= n) return;
    const int64_t row = at / s.half;
    const int i = (int)(at - row * s.half);
    double f = exp(-(double)i * s.log_theta_over_half);
    if (s.kind == ATTS_ROTARY_LINEAR) f /= s.factor;
    if (s.kind == ATTS_ROTARY_BY_PARTS) {
        const double turns = s.original * f / 6.283185307179586476925;
        const double g = fmin(fmax((turns - s.low) / (s.high - s.low), 0.0), 1.0);
        f *= g + (1.0 - g) / s.factor;
    }
    double sn, c;
    sincos((double)(first + row) * f, &sn, &c);
    table[at] = make_float2((float)(s.magnitude * c), (float)(s.magnitude * sn));
}

struct AppendArgs {
    const int32_t *positions, *cached, *row_offsets;
    const float2* table;
    int64_t qkv_stride;
    int32_t R, nq, n_positions, half, interleaved;
};

template <typename T>
__global__ __launch_bounds__(256) void rotary_append_kernel(const T* __restrict__ qkv, T* __restrict__ q_out, T* __restrict__ k_pages,
                                                            T* __restrict__ v_pages, PagedView p, AppendArgs a) {
    const int r = blockIdx.x;
    const int seq = sequence_of(a.row_offsets, p.n_seqs, r);
    int page = -1, token = 0;
    if (seq >= 0) {
        const int64_t at = (int64_t)a.cached[seq] + (r - a.row_offsets[seq]);
        if (at >= 0 && at < p.slots()) {
            token = (int)at;
            page = p.page_of(seq, token);
            if (page >= p.n_pages) page = -1;
        }
    }
    const float2* cs = a.table + (int64_t)min(max(a.positions[r], 0), a.n_positions - 1) * a.half;
    const T* src = qkv + (int64_t)r * a.qkv_stride;
    const int hd = p.hd, heads = a.nq + 2 * p.n_kv, rot = 2 * a.half;
    for (int e = threadIdx.x; e < heads * hd; e += 256) {
        const int head = e / hd, i = e - head * hd;
        float y = to_f32(src[e]);
        if (head < a.nq + p.n_kv && i < rot) {
            int pair, other;
            bool second;
            if (a.interleaved) { pair = i >> 1; second = i & 1; other = i ^ 1; }
            else { second = i >= a.half; pair = second ? i - a.half : i; other = second ? i - a.half : i + a.half; }
            const float2 t = cs[pair];
            const float o = to_f32(src[head * hd + other]);
            y = second ? y * t.x + o * t.y : y * t.x - o * t.y;
        }
        if (head < a.nq) q_out[(int64_t)r * a.nq * hd + e] = from_f32<T>(y);
        else if (page >= 0) {
            const int h = head - a.nq;
            if (h < p.n_kv) k_pages[p.key_at(page, h, token) + i] = from_f32<T>(y);
            else v_pages[p.value_at(page, h - p.n_kv, token) + ((int64_t)i << p.page_log)] = from_f32<T>(y);
        }
    }
}

}  // namespace
}  // namespace atts

using namespace atts;

extern "C" {

int32_t atts_rotary_table(int32_t scaling, double theta, int32_t rot_dim, double factor, double original, double low, double high,
                          double magnitude, int64_t first, int64_t rows, float* table, void* hip_stream) {
    const char* fn = "atts_rotary_table";
    if (scaling < ATTS_ROTARY_PLAIN || scaling > ATTS_ROTARY_BY_PARTS) return fail(ATTS_ERR_INVALID_ARG, "%s: unknown scaling %d", fn, scaling);
    if (rot_dim < 2 || rot_dim % 2 || rot_dim > 256) return fail(ATTS_ERR_SHAPE, "%s: rot_dim = %d is not even in [2, 256]", fn, rot_dim);
    if (!(theta > 0.0 && isfinite(theta)) || !isfinite(magnitude)) return fail(ATTS_ERR_INVALID_ARG, "%s: theta and magnitude must be finite, theta > 0", fn);
    if (scaling != ATTS_ROTARY_PLAIN && !(factor > 0.0 && isfinite(factor))) return fail(ATTS_ERR_INVALID_ARG, "%s: factor = %g", fn, factor);
    if (scaling == ATTS_ROTARY_STRETCHED && rot_dim < 4) return fail(ATTS_ERR_SHAPE, "%s: a stretched theta needs rot_dim > 2", fn);
    if (scaling == ATTS_ROTARY_BY_PARTS && !(original > 0.0 && isfinite(original) && isfinite(low) && isfinite(high) && high > low))
        return fail(ATTS_ERR_INVALID_ARG, "%s: need original > 0 and high > low", fn);
    const int64_t most = (int64_t)1 << 30;
    if (first < 0 || rows < 0 || first > most || rows > most) return fail(ATTS_ERR_INVALID_ARG, "%s: first or rows outside [0, 2^30]", fn);
    if (rows == 0) return ATTS_OK;
    if (!table || ((uintptr_t)table & 7)) return fail(ATTS_ERR_INVALID_ARG, "%s: table NULL or not 8-byte aligned", fn);
    RotaryScaling s{scaling, rot_dim / 2, log(theta), factor, original, low, high, magnitude};
    if (scaling == ATTS_ROTARY_STRETCHED) s.log_theta_over_half += log(factor) * rot_dim / (rot_dim - 2);
    s.log_theta_over_half /= s.half;
    const int64_t step = (int64_t)1 << 22;                                        // rows of a launch
    for (int64_t at = 0; at < rows; at += step) {
        const int64_t n = (rows - at < step ? rows - at : step) * s.half;
        hipLaunchKernelGGL(rotary_table_kernel, dim3((unsigned)ceil_div(n, 256)), dim3(256), 0, static_cast<hipStream_t>(hip_stream),
                           reinterpret_cast<float2*>(table) + at * s.half, first + at, n, s);
        ATTS_LAUNCH_CHECK("rotary_table_kernel");
    }
    return ATTS_OK;
}

int32_t atts_rotary_append(const atts_paged_cache* cache, const void* qkv, int64_t qkv_stride, const int32_t* positions, const int32_t* cached,
                           const int32_t* row_offsets, int32_t R, int32_t n_q_heads, const float* table, int32_t n_positions, int32_t rot_dim,
                           int32_t layout, void* q_out, void* hip_stream) {
    const char* fn = "atts_rotary_append";
    PagedView p;
    const int32_t rc = check_paged(fn, cache, &p);
    if (rc != ATTS_OK) return rc;
    if (R < 0 || n_q_heads < 0 || n_q_heads > 4096 || p.n_kv > 4096) return fail(ATTS_ERR_INVALID_ARG, "%s: need R >= 0 and at most 4096 heads", fn);
    if (layout != ATTS_ROTARY_HALF && layout != ATTS_ROTARY_INTERLEAVED) return fail(ATTS_ERR_INVALID_ARG, "%s: unknown layout %d", fn, layout);
    if (rot_dim < 0 || rot_dim % 2 || rot_dim > p.hd) return fail(ATTS_ERR_SHAPE, "%s: rot_dim = %d is not even in [0, head_dim]", fn, rot_dim);
    if (R == 0) return ATTS_OK;
    if (!qkv || !positions || !row_offsets || (p.n_seqs > 0 && !cached) || (n_q_heads > 0 && !q_out)) return fail(ATTS_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if (rot_dim > 0 && (!table || ((uintptr_t)table & 7) || n_positions < 1)) return fail(ATTS_ERR_INVALID_ARG, "%s: table NULL, empty or not 8-byte aligned", fn);
    if (qkv_stride < (int64_t)(n_q_heads + 2 * p.n_kv) * p.hd) return fail(ATTS_ERR_INVALID_ARG, "%s: rows of qkv overlap", fn);
    const AppendArgs a{positions, cached, row_offsets, reinterpret_cast<const float2*>(table), qkv_stride, R, n_q_heads,
                       n_positions < 1 ? 1 : n_positions, rot_dim / 2, layout == ATTS_ROTARY_INTERLEAVED};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (cache->dtype == ATTS_DTYPE_F32)
        hipLaunchKernelGGL(rotary_append_kernel<float>, dim3((unsigned)R), dim3(256), 0, stream, static_cast<const float*>(qkv),
                           static_cast<float*>(q_out), static_cast<float*>(cache->k_pages), static_cast<float*>(cache->v_pages), p, a);
    else
        hipLaunchKernelGGL(rotary_append_kernel<bf16>, dim3((unsigned)R), dim3(256), 0, stream, static_cast<const bf16*>(qkv),
                           static_cast<bf16*>(q_out), static_cast<bf16*>(cache->k_pages), static_cast<bf16*>(cache->v_pages), p, a);
    ATTS_LAUNCH_CHECK("rotary_append_kernel");
    return ATTS_OK;
}

}  // extern "C"
