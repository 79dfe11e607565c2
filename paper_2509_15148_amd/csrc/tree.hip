// Attention of drafted token trees over a paged key / value cache.
#include "paged.h"

#include <math.h>

namespace atts {
namespace {

struct TreeArgs {
    const int32_t *parents, *cached, *row_offsets;
    int32_t R, nq, max_rows, max_cached, window;
    float scale, softcap;
};

// One wavefront per (row, query head): 64 keys at a time, a lane a key; then a lane holds elements lane, lane + 64, ... of the output.
template <typename T>
__global__ __launch_bounds__(64) void tree_rows_kernel(const T* __restrict__ q, const T* __restrict__ k_pages, const T* __restrict__ v_pages,
                                                       T* __restrict__ out, PagedView p, TreeArgs a) {
    const int lane = threadIdx.x, r = blockIdx.x, head = blockIdx.y, kv = head / (a.nq / p.n_kv), hd = p.hd;
    const int seq = sequence_of(a.row_offsets, p.n_seqs, r);
    if (seq < 0) return;
    const int first = a.row_offsets[seq], own = r - first;
    if (own >= a.max_rows || first < 0) return;
    const int L = min(max(a.cached[seq], 0), min(a.max_cached, p.slots()));
    __shared__ uint32_t mine[ATTS_MAX_TREE / 32];         // bit j: row j is the row itself or an ancestor
    if (lane < ATTS_MAX_TREE / 32) mine[lane] = 0;
    __syncthreads();
    if (lane == 0)
        for (int at = own; at >= 0;) {
            mine[at >> 5] |= 1u << (at & 31);
            const int parent = a.parents[first + at];
            at = parent >= 0 && parent < at ? parent : -1;
        }
    __syncthreads();
    int depth = -1;
    for (int w = 0; w < ATTS_MAX_TREE / 32; ++w) depth += __popc(mine[w]);
    const int here = L + depth;
    const T* qr = q + ((int64_t)r * a.nq + head) * hd;
    float m = -INFINITY, l = 0.f, acc[4] = {};
    const int keys = min(L + own + 1, p.slots());
    for (int j0 = 0; j0 < keys; j0 += 64) {
        const int j = j0 + lane;
        bool open = j < keys;
        int at = j;
        if (open && j >= L) {
            const int t = j - L;
            open = mine[t >> 5] >> (t & 31) & 1;
            at = L - 1;
            for (int w = 0; w <= t >> 5; ++w) at += __popc(w < t >> 5 ? mine[w] : mine[w] & (uint32_t)(2ull << (t & 31)) - 1);
        }
        if (a.window && here - at >= a.window) open = false;
        float z = -INFINITY;
        int page = 0;
        if (open) {
            page = p.page_of(seq, j);
            if ((uint32_t)page >= (uint32_t)p.n_pages) page = 0;
            const T* kr = k_pages + p.key_at(page, kv, j);
            z = 0.f;
            for (int d = 0; d < hd; ++d) z += to_f32(qr[d]) * to_f32(kr[d]);
            z *= a.scale;
            if (a.softcap > 0.f) z = a.softcap * tanhf(z / a.softcap);
        }
        float top = z;
#pragma unroll
        for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
        const float next = fmaxf(m, top);
        if (!(next > -INFINITY) && !__any(open)) continue;
        const float keep = m > -INFINITY ? __expf(m - next) : 0.f;
        const float e = open ? __expf(z - next) : 0.f;
        float sum = e;
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d, 64);
        l = l * keep + sum;
        m = next;
        for (int i = 0; i < 4; ++i) acc[i] *= keep;
        for (int t = 0; t < 64; ++t) {
            if (!__shfl((int)open, t, 64)) continue;
            const float w = __shfl(e, t, 64);
            const T* vc = v_pages + p.value_at(__shfl(page, t, 64), kv, j0 + t);
            for (int i = 0; i < 4; ++i)
                if (lane + 64 * i < hd) acc[i] += w * to_f32(vc[(int64_t)(lane + 64 * i) << p.page_log]);
        }
    }
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < hd) out[((int64_t)r * a.nq + head) * hd + lane + 64 * i] = from_f32<T>(acc[i] / l);
}

int32_t check_tree(const char* fn, const atts_paged_cache* cache, int32_t n_q_heads, int32_t R, int32_t max_rows, int32_t max_cached, PagedView* p) {
    const int32_t rc = check_paged(fn, cache, p);
    if (rc != ATTS_OK) return rc;
    if (n_q_heads < 1 || n_q_heads % p->n_kv || n_q_heads > 4096) return fail(ATTS_ERR_SHAPE, "%s: n_q_heads = %d is not a multiple of n_kv_heads = %d up to 4096", fn, n_q_heads, p->n_kv);
    if (R < 0 || R > (1 << 24) || max_cached < 0) return fail(ATTS_ERR_INVALID_ARG, "%s: need 0 <= R <= 2^24 and max_cached >= 0", fn);
    if (max_rows < 0 || max_rows > ATTS_MAX_TREE) return fail(ATTS_ERR_INVALID_ARG, "%s: max_rows = %d outside [0, %d]", fn, max_rows, ATTS_MAX_TREE);
    return ATTS_OK;
}

}  // namespace
}  // namespace atts

using namespace atts;

extern "C" {

int32_t atts_attention_tree_workspace_bytes(const atts_paged_cache* cache, int32_t n_q_heads, int32_t R, int32_t max_rows, int32_t max_cached,
                                            size_t* out_bytes) {
    const char* fn = "atts_attention_tree_workspace_bytes";
    if (!out_bytes) return fail(ATTS_ERR_INVALID_ARG, "%s: out_bytes is NULL", fn);
    PagedView p;
    const int32_t rc = check_tree(fn, cache, n_q_heads, R, max_rows, max_cached, &p);
    if (rc != ATTS_OK) return rc;
    *out_bytes = 0;
    return ATTS_OK;
}

int32_t atts_attention_tree(const atts_paged_cache* cache, const void* q, const int32_t* parents, const int32_t* cached, const int32_t* row_offsets,
                            int32_t R, int32_t n_q_heads, int32_t max_rows, int32_t max_cached, float scale, float softcap, int32_t window, void* out,
                            void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* fn = "atts_attention_tree";
    PagedView p;
    int32_t rc = check_tree(fn, cache, n_q_heads, R, max_rows, max_cached, &p);
    if (rc != ATTS_OK) return rc;
    if (!isfinite(scale) || !(softcap >= 0.f && isfinite(softcap)) || window < 0)
        return fail(ATTS_ERR_INVALID_ARG, "%s: scale = %g, softcap = %g, window = %d", fn, scale, softcap, window);
    if (R == 0 || p.n_seqs == 0 || max_rows == 0) return ATTS_OK;
    if (!q || !parents || !cached || !row_offsets || !out) return fail(ATTS_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if ((uintptr_t)q & 15) return fail(ATTS_ERR_INVALID_ARG, "%s: q must be 16-byte aligned", fn);
    size_t need = 0;
    rc = atts_attention_tree_workspace_bytes(cache, n_q_heads, R, max_rows, max_cached, &need);
    if (rc != ATTS_OK) return rc;
    if (need && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need))
        return fail(ATTS_ERR_WORKSPACE, "%s: workspace NULL, misaligned or smaller than %zu bytes", fn, need);
    const TreeArgs a{parents, cached, row_offsets, R, n_q_heads, max_rows, max_cached, window, scale, softcap};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (cache->dtype == ATTS_DTYPE_F32)
        hipLaunchKernelGGL(tree_rows_kernel<float>, dim3((unsigned)R, (unsigned)n_q_heads), dim3(64), 0, stream, static_cast<const float*>(q),
                           static_cast<const float*>(cache->k_pages), static_cast<const float*>(cache->v_pages), static_cast<float*>(out), p, a);
    else
        hipLaunchKernelGGL(tree_rows_kernel<bf16>, dim3((unsigned)R, (unsigned)n_q_heads), dim3(64), 0, stream, static_cast<const bf16*>(q),
                           static_cast<const bf16*>(cache->k_pages), static_cast<const bf16*>(cache->v_pages), static_cast<bf16*>(out), p, a);
    ATTS_LAUNCH_CHECK("tree_rows_kernel");
    return ATTS_OK;
}

}  // extern "C"
