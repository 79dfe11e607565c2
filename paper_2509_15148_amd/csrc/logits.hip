// The logits of a step under their requests' rules: penalties for tokens that came before, sparse biases, temperature, a grammar mask;
// with the first arg max and the log-sum-exp of the result.
//
//   * A workgroup takes a slice of the vocabulary for the rows of one sequence.  How often each token of the slice came before is
//     counted into LDS from the history (integer atomics: the order does not matter), once for all rows; a row adds the tokens
//     of its own path before its turn and takes them out behind it.  Nothing of the size of the vocabulary is kept between calls.
//   * The results stay in registers for the maximum and the sum of exponentials: one read and one write of the logits.  Every wavefront
//     leaves (maximum, its index, sum) of its part; a second launch joins the parts of a row in a fixed order.
#include "paged.h"

#include <math.h>

namespace atts {
namespace {

constexpr int kThreads = 256, kTokens = 16, kSlice = kThreads * kTokens, kWaves = kThreads / 64;

struct Part {
    float top, sum;          // maximum, sum of exp(x - top); top = -inf: nothing above -inf
    int32_t id, pad;         // first index of the maximum, -1 if none
};

struct LogitsArgs {
    const int32_t* row_offsets;
    const float* params;
    const int32_t *history, *history_offsets, *prompt_lens, *tree_ids, *parents, *bias_ids, *bias_offsets;
    const float* bias_values;
    const uint32_t* mask;
    Part* parts;
    int64_t in_stride, out_stride, mask_words;
    int32_t max_rows, n_history, n_bias, R, V, slices, rows_per_wg;
};

// (top, id, sum) of two parts together; of equal maxima the lower index
__device__ __forceinline__ void join(Part& a, float top, int id, float sum) {
    if (top > a.top) {
        a.sum = (a.top > -INFINITY ? a.sum * __expf(a.top - top) : a.sum) + sum;
        a.top = top;
        a.id = id;
    } else {
        a.sum += top == a.top ? sum : top > -INFINITY ? sum * __expf(top - a.top) : sum;
        if (top == a.top && id >= 0 && (a.id < 0 || id < a.id)) a.id = id;
    }
}

// Steps 1 to 3 on one value.  Every operation is rounded by itself: no products are contracted into sums.
__device__ __forceinline__ float adjust(float x, uint32_t word, const float4& p) {
#pragma clang fp contract(off)
    const uint32_t count = word & 0x7fffffffu;
    if (word) x = x > 0.f ? x / p.x : x * p.x;
    x = x - (float)count * p.y;
    if (count) x = x - p.z;
    return x;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void logits_kernel(const T* __restrict__ logits, T* __restrict__ out, LogitsArgs a) {
    __shared__ uint32_t seen[kSlice];                    // generated count; bit 31: in the prompt
    __shared__ int32_t bias_at[kSlice];                  // 1 + position of the token's last bias entry, 0: none
    __shared__ int16_t parent[ATTS_MAX_TREE];
    const int tid = threadIdx.x, seq = blockIdx.z, v0 = blockIdx.x * kSlice, n_here = min(kSlice, a.V - v0);
    const int first = a.row_offsets[seq], end = min(a.row_offsets[seq + 1], a.R);
    if (first < 0) return;
    const int n = min(end - first, a.max_rows), r0 = blockIdx.y * a.rows_per_wg, r1 = min(r0 + a.rows_per_wg, n);
    if (r0 >= r1) return;
    for (int i = tid; i < kSlice; i += kThreads) {
        seen[i] = 0;
        bias_at[i] = 0;
    }
    const bool paths = a.params && a.tree_ids;
    if (paths)
        for (int i = tid; i < n; i += kThreads) {
            const int up = a.parents[first + i];
            parent[i] = (int16_t)(up >= 0 && up < i ? up : -1);
        }
    __syncthreads();
    if (a.params && a.history) {
        const int h0 = min(max(a.history_offsets[seq], 0), a.n_history), h1 = min(max(a.history_offsets[seq + 1], h0), a.n_history);
        const int64_t split = (int64_t)h0 + (a.prompt_lens ? a.prompt_lens[seq] : 0);
        for (int i = h0 + tid; i < h1; i += kThreads) {
            const int v = a.history[i] - v0;
            if ((uint32_t)v < (uint32_t)n_here) {
                if (i < split) atomicOr(&seen[v], 0x80000000u);
                else atomicAdd(&seen[v], 1u);
            }
        }
    }
    int bias0 = 0;
    if (a.bias_ids) {
        bias0 = min(max(a.bias_offsets[seq], 0), a.n_bias);
        const int b1 = min(max(a.bias_offsets[seq + 1], bias0), a.n_bias);
        for (int i = bias0 + tid; i < b1; i += kThreads) {
            const int v = a.bias_ids[i] - v0;
            if ((uint32_t)v < (uint32_t)n_here) atomicMax(&bias_at[v], i - bias0 + 1);
        }
    }
    const float4 p = a.params ? reinterpret_cast<const float4*>(a.params)[seq] : make_float4(1.f, 0.f, 0.f, 1.f);
    auto path = [&](int row, uint32_t step) {              // the tokens of the row's path, counted (step 1) or taken out again (-1)
        if (tid == 0)
            for (int at = row; at >= 0; at = parent[at]) {
                const int v = a.tree_ids[first + at] - v0;
                if ((uint32_t)v < (uint32_t)n_here) seen[v] += step;
            }
    };
    for (int row = r0; row < r1; ++row) {
        const int64_t r = first + row;
        __syncthreads();
        if (paths) {
            path(row, 1u);
            __syncthreads();
        }
        const T* src = logits + r * a.in_stride + v0;
        T* dst = out + r * a.out_stride + v0;
        float x[kTokens], top = -INFINITY;
        int id = -1;
#pragma unroll
        for (int i = 0; i < kTokens; ++i) {
            const int t = i * kThreads + tid;
            x[i] = -INFINITY;
            if (t < n_here) {
                float y = to_f32(src[t]);
                if (a.params) y = adjust(y, seen[t], p);
                if (a.bias_ids && bias_at[t]) y = y + a.bias_values[bias0 + bias_at[t] - 1];
                if (a.params) y = y / p.w;
                if (a.mask) {
                    const uint32_t v = (uint32_t)(v0 + t);
                    if (!(a.mask[r * a.mask_words + (v >> 5)] >> (v & 31) & 1)) y = -INFINITY;
                }
                dst[t] = from_f32<T>(y);
                x[i] = y;
                if (y > top) { top = y; id = v0 + t; }
            }
        }
        if (a.parts) {
            float best = top;
#pragma unroll
            for (int d = 32; d; d >>= 1) best = fmaxf(best, __shfl_xor(best, d, 64));
            int lowest = top == best && id >= 0 ? id : 0x7fffffff;
#pragma unroll
            for (int d = 32; d; d >>= 1) lowest = min(lowest, __shfl_xor(lowest, d, 64));
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < kTokens; ++i) sum += best > -INFINITY ? x[i] == best ? 1.f : __expf(x[i] - best) : isnan(x[i]) ? x[i] : 0.f;
#pragma unroll
            for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d, 64);
            if ((tid & 63) == 0)
                a.parts[(r * a.slices + blockIdx.x) * kWaves + (tid >> 6)] = Part{best, sum, lowest == 0x7fffffff ? -1 : lowest, 0};
        }
        if (paths) {
            __syncthreads();
            path(row, ~0u);
        }
    }
}

// One wavefront per row: the parts of its slices in slice order, lanes joined by exchanges.
__global__ __launch_bounds__(64) void logits_join_kernel(const Part* __restrict__ parts, const int32_t* __restrict__ row_offsets, int n_seqs, int max_rows,
                                                         int n_parts, int32_t* __restrict__ top_ids, float* __restrict__ lse) {
    const int r = blockIdx.x, lane = threadIdx.x;
    const int seq = sequence_of(row_offsets, n_seqs, r);
    if (seq < 0 || r - row_offsets[seq] >= max_rows || row_offsets[seq] < 0) return;
    Part p{-INFINITY, 0.f, -1, 0};
    for (int i = lane; i < n_parts; i += 64) {
        const Part o = parts[(int64_t)r * n_parts + i];
        join(p, o.top, o.id, o.sum);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const float top = __shfl_xor(p.top, d, 64), sum = __shfl_xor(p.sum, d, 64);
        const int id = __shfl_xor(p.id, d, 64);
        join(p, top, id, sum);
    }
    if (lane) return;
    if (top_ids) top_ids[r] = p.id;
    if (lse) lse[r] = p.top > -INFINITY ? p.top + __logf(p.sum) : isnan(p.sum) ? p.sum : -INFINITY;
}

int64_t slices_of(int32_t V) { return ceil_div(V, kSlice); }

}  // namespace
}  // namespace atts

using namespace atts;

extern "C" {

int32_t atts_logits_adjust_workspace_bytes(int32_t R, int32_t V, size_t* out_bytes) {
    const char* fn = "atts_logits_adjust_workspace_bytes";
    if (!out_bytes) return fail(ATTS_ERR_INVALID_ARG, "%s: out_bytes is NULL", fn);
    if (R < 0 || R > (1 << 24) || V < 1 || V > (1 << 30)) return fail(ATTS_ERR_INVALID_ARG, "%s: R outside [0, 2^24] or V outside [1, 2^30]", fn);
    *out_bytes = align_up((size_t)R * slices_of(V) * kWaves * sizeof(Part), 256);
    return ATTS_OK;
}

int32_t atts_logits_adjust(int32_t dtype, const void* logits, int64_t logits_stride, const int32_t* row_offsets, int32_t n_seqs, int32_t max_rows,
                           const float* params, const int32_t* history, const int32_t* history_offsets, const int32_t* prompt_lens, int32_t n_history,
                           const int32_t* tree_ids, const int32_t* parents, const int32_t* bias_ids, const float* bias_values,
                           const int32_t* bias_offsets, int32_t n_bias, const uint32_t* mask, int32_t R, int32_t V, void* out, int64_t out_stride,
                           int32_t* top_ids, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* fn = "atts_logits_adjust";
    if (dtype != ATTS_DTYPE_F32 && dtype != ATTS_DTYPE_BF16) return fail(ATTS_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
    size_t need = 0;
    const int32_t rc = atts_logits_adjust_workspace_bytes(R, V, &need);
    if (rc != ATTS_OK) return rc;
    if (n_seqs < 0 || n_seqs > 65535 || n_history < 0 || n_bias < 0) return fail(ATTS_ERR_INVALID_ARG, "%s: n_seqs outside [0, 65535], or a negative length", fn);
    if (max_rows < 0 || max_rows > ATTS_MAX_TREE) return fail(ATTS_ERR_INVALID_ARG, "%s: max_rows = %d outside [0, %d]", fn, max_rows, ATTS_MAX_TREE);
    if (R == 0 || n_seqs == 0 || max_rows == 0) return ATTS_OK;
    if (!logits || !out || !row_offsets) return fail(ATTS_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if (n_history == 0 && !history) history_offsets = nullptr;
    if ((n_history > 0 && !history) || (!history != !history_offsets)) return fail(ATTS_ERR_INVALID_ARG, "%s: history and its offsets come together", fn);
    if (!tree_ids != !parents) return fail(ATTS_ERR_INVALID_ARG, "%s: tree_ids and parents come together", fn);
    if (!bias_ids != !bias_offsets || !bias_ids != !bias_values) return fail(ATTS_ERR_INVALID_ARG, "%s: bias_ids, bias_values and bias_offsets come together", fn);
    if (logits_stride < V || out_stride < V) return fail(ATTS_ERR_INVALID_ARG, "%s: rows overlap", fn);
    if ((uintptr_t)params & 15) return fail(ATTS_ERR_INVALID_ARG, "%s: params must be 16-byte aligned", fn);
    const bool decide = top_ids || lse;
    if (decide && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need))
        return fail(ATTS_ERR_WORKSPACE, "%s: workspace NULL, misaligned or smaller than %zu bytes", fn, need);
    LogitsArgs a{row_offsets, params, history, history_offsets, prompt_lens, tree_ids, parents, bias_ids, bias_offsets, bias_values, mask,
                 decide ? static_cast<Part*>(workspace) : nullptr, logits_stride, out_stride, ceil_div(V, 32), max_rows, n_history, n_bias, R, V,
                 (int32_t)slices_of(V), max_rows};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const dim3 grid((unsigned)a.slices, (unsigned)ceil_div(max_rows, a.rows_per_wg), (unsigned)n_seqs);
    if (dtype == ATTS_DTYPE_F32)
        hipLaunchKernelGGL(logits_kernel<float>, grid, dim3(kThreads), 0, stream, static_cast<const float*>(logits), static_cast<float*>(out), a);
    else
        hipLaunchKernelGGL(logits_kernel<bf16>, grid, dim3(kThreads), 0, stream, static_cast<const bf16*>(logits), static_cast<bf16*>(out), a);
    ATTS_LAUNCH_CHECK("logits_kernel");
    if (decide) {
        hipLaunchKernelGGL(logits_join_kernel, dim3((unsigned)R), dim3(64), 0, stream, a.parts, row_offsets, n_seqs, max_rows, a.slices * kWaves, top_ids, lse);
        ATTS_LAUNCH_CHECK("logits_join_kernel");
    }
    return ATTS_OK;
}

}  // extern "C"
