// Products of a few rows with weights in 4 bits:  out = X W^T,  W[n, k] = scale[n, k / G] (code[n, k] - zero[n, k / G]).
#include "common.h"

namespace atts {
namespace {

struct QuantArgs {
    const void* x;
    const uint8_t* codes;
    const void* scales;
    const uint8_t* zeros;
    const float* residual;
    void* out;
    int64_t x_stride;
    int32_t M, N, K, group_log, groups;
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

template <typename T, int EPI>
__device__ __forceinline__ void store(const QuantArgs& a, int m, int n, float y) {
    const int64_t at = (int64_t)m * a.N + n;
    if constexpr (EPI == ATTS_EPILOGUE_RESIDUAL) reinterpret_cast<float*>(a.out)[at] = a.residual[at] + y;
    else if constexpr (EPI == ATTS_EPILOGUE_STORE_F32) reinterpret_cast<float*>(a.out)[at] = y;
    else reinterpret_cast<T*>(a.out)[at] = from_f32<T>(y);
}

__device__ __forceinline__ float silu(float x) { return x / (1.f + __expf(-x)); }

// One wavefront per output feature: lane l takes eight codes at a time, 4 rows of X in one sweep.
template <typename T, int EPI>
__global__ __launch_bounds__(256) void quant_rows_kernel(QuantArgs a) {
    constexpr int kRows = 4, kWide = EPI == ATTS_EPILOGUE_SWIGLU ? 2 : 1;
    const int lane = threadIdx.x & 63;
    const int n = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (n >= a.N) return;
    const T* x = reinterpret_cast<const T*>(a.x);
    const T* scales = reinterpret_cast<const T*>(a.scales);
    for (int m0 = 0; m0 < a.M; m0 += kRows) {
        float acc[kWide][kRows] = {};
        for (int w = 0; w < kWide; ++w) {
            const int64_t row = n + (int64_t)w * a.N;
            for (int k = lane * 8; k < a.K; k += 512) {
                const uint32_t word = *reinterpret_cast<const uint32_t*>(a.codes + row * (a.K / 2) + k / 2);
                const int64_t g = row * a.groups + (k >> a.group_log);
                const float scale = to_f32(scales[g]);
                const float zero = a.zeros ? (float)a.zeros[g] : 8.f;
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    const T* xr = x + (int64_t)min(m0 + r, a.M - 1) * a.x_stride + k;
                    float s = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) s += ((float)((word >> (4 * j)) & 15) - zero) * to_f32(xr[j]);
                    acc[w][r] += scale * s;
                }
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            float y = wave_sum(acc[0][r]);
            if constexpr (EPI == ATTS_EPILOGUE_SWIGLU) y = silu(y) * wave_sum(acc[kWide - 1][r]);
            if (lane == 0 && m0 + r < a.M) store<T, EPI>(a, m0 + r, n, y);
        }
    }
}

template <typename T, int EPI>
int32_t launch_quant(const QuantArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((quant_rows_kernel<T, EPI>), dim3((unsigned)ceil_div(a.N, 4)), dim3(256), 0, stream, a);
    ATTS_LAUNCH_CHECK("quant_rows_kernel");
    return ATTS_OK;
}

template <typename T>
int32_t launch_quant_epi(int32_t epilogue, const QuantArgs& a, hipStream_t stream) {
    switch (epilogue) {
        case ATTS_EPILOGUE_STORE: return launch_quant<T, ATTS_EPILOGUE_STORE>(a, stream);
        case ATTS_EPILOGUE_STORE_F32: return launch_quant<T, ATTS_EPILOGUE_STORE_F32>(a, stream);
        case ATTS_EPILOGUE_RESIDUAL: return launch_quant<T, ATTS_EPILOGUE_RESIDUAL>(a, stream);
        default: return launch_quant<T, ATTS_EPILOGUE_SWIGLU>(a, stream);
    }
}

// Eight lanes a group: each holds group / 8 of its values, their limits are joined by three exchanges.
template <typename T>
__global__ __launch_bounds__(256) void quantize_kernel(const T* __restrict__ w, int64_t n_groups, int group, uint8_t* __restrict__ codes,
                                                       T* __restrict__ scales, uint8_t* __restrict__ zeros) {
    const int64_t g = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3);
    const int part = threadIdx.x & 7, n = group >> 3;                             // 4, 8 or 16 values
    const bool live = g < n_groups;
    const T* src = w + (live ? g : 0) * group + part * n;
    float lo = 0.f, hi = 0.f;
    for (int i = 0; i < n; ++i) {
        const float x = to_f32(src[i]);
        lo = fminf(lo, x);
        hi = fmaxf(hi, x);
    }
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) {
        lo = fminf(lo, __shfl_xor(lo, d, 64));
        hi = fmaxf(hi, __shfl_xor(hi, d, 64));
    }
    if (!live) return;
    const T stored = from_f32<T>(zeros ? (hi - lo) / 15.f : fmaxf(-lo / 8.f, hi / 7.f));
    const float scale = to_f32(stored);
    const float zero = !zeros ? 8.f : scale > 0.f ? fminf(fmaxf(rintf(-lo / scale), 0.f), 15.f) : 0.f;
    if (part == 0) {
        scales[g] = stored;
        if (zeros) zeros[g] = (uint8_t)zero;
    }
    auto code = [&](int i) { return (uint32_t)(scale > 0.f ? fminf(fmaxf(rintf(to_f32(src[i]) / scale) + zero, 0.f), 15.f) : zero); };
    for (int i = 0; i < n; i += 2) codes[(g * group + part * n + i) >> 1] = (uint8_t)(code(i) | code(i + 1) << 4);
}

int32_t check_quant(const char* fn, int32_t dtype, int32_t N, int32_t Kdim, int32_t group) {
    if (dtype != ATTS_DTYPE_F32 && dtype != ATTS_DTYPE_BF16) return fail(ATTS_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
    if (N < 1 || Kdim < 1) return fail(ATTS_ERR_INVALID_ARG, "%s: need N and Kdim >= 1", fn);
    if ((group != 32 && group != 64 && group != 128) || Kdim % group)
        return fail(ATTS_ERR_SHAPE, "%s: group = %d is not 32, 64 or 128, or does not divide Kdim = %d", fn, group, Kdim);
    if (N > (1 << 29) || Kdim > (1 << 29)) return fail(ATTS_ERR_SHAPE, "%s: N or Kdim exceeds 2^29", fn);
    return ATTS_OK;
}

}  // namespace
}  // namespace atts

using namespace atts;

extern "C" {

int32_t atts_gemm_nt_quant(int32_t dtype, const void* x, int64_t x_stride, const uint8_t* codes, const void* scales, const uint8_t* zeros,
                           int32_t group, const float* residual, void* out, int32_t M, int32_t N, int32_t Kdim, int32_t epilogue,
                           void* hip_stream) {
    const char* fn = "atts_gemm_nt_quant";
    const int32_t rc = check_quant(fn, dtype, N, Kdim, group);
    if (rc != ATTS_OK) return rc;
    if (epilogue < ATTS_EPILOGUE_STORE || epilogue > ATTS_EPILOGUE_SWIGLU) return fail(ATTS_ERR_INVALID_ARG, "%s: unknown epilogue %d", fn, epilogue);
    if (M < 0) return fail(ATTS_ERR_INVALID_ARG, "%s: M = %d < 0", fn, M);
    if (M == 0) return ATTS_OK;
    if (!x || !codes || !scales || !out || (epilogue == ATTS_EPILOGUE_RESIDUAL && !residual)) return fail(ATTS_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if (x_stride < Kdim) return fail(ATTS_ERR_INVALID_ARG, "%s: rows of x overlap", fn);
    if (((uintptr_t)x | (uintptr_t)codes | ((uint64_t)x_stride * dtype_size(dtype))) & 15)
        return fail(ATTS_ERR_INVALID_ARG, "%s: x, its rows and codes must be 16-byte aligned", fn);
    const QuantArgs a{x, codes, scales, zeros, residual, out, x_stride, M, N, Kdim, group == 32 ? 5 : group == 64 ? 6 : 7, Kdim / group};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return dtype == ATTS_DTYPE_F32 ? launch_quant_epi<float>(epilogue, a, stream) : launch_quant_epi<bf16>(epilogue, a, stream);
}

int32_t atts_quantize_rows(int32_t dtype, const void* w, int32_t N, int32_t Kdim, int32_t group, uint8_t* codes, void* scales, uint8_t* zeros,
                           void* hip_stream) {
    const char* fn = "atts_quantize_rows";
    const int32_t rc = check_quant(fn, dtype, N, Kdim, group);
    if (rc != ATTS_OK) return rc;
    if (!w || !codes || !scales) return fail(ATTS_ERR_INVALID_ARG, "%s: NULL argument", fn);
    const int64_t n_groups = (int64_t)N * (Kdim / group), wgs = ceil_div(n_groups, 32);
    if (wgs > 0x7fffffff) return fail(ATTS_ERR_SHAPE, "%s: the matrix has more than 2^36 groups", fn);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (dtype == ATTS_DTYPE_F32)
        hipLaunchKernelGGL(quantize_kernel<float>, dim3((unsigned)wgs), dim3(256), 0, stream, static_cast<const float*>(w), n_groups, group, codes,
                           static_cast<float*>(scales), zeros);
    else
        hipLaunchKernelGGL(quantize_kernel<bf16>, dim3((unsigned)wgs), dim3(256), 0, stream, static_cast<const bf16*>(w), n_groups, group, codes,
                           static_cast<bf16*>(scales), zeros);
    ATTS_LAUNCH_CHECK("quantize_kernel");
    return ATTS_OK;
}

}  // extern "C"
