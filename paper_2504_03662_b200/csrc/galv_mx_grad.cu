// Gradients that read a layer's input where it was kept in 8 bits: activation functions and norms.

#include "galv_mx.cuh"

namespace {

constexpr int kThreads = 256;

// f'(x) of the activation functions, 0 or 1 from |x| = 100 on (a NaN passes both comparisons).
template <int ACT>
__device__ __forceinline__ float act_slope(float x)
{
    x = x > 100.f ? 100.f : x < -100.f ? -100.f : x;
    if (ACT == GALV_ACT_GELU) {
        // Phi(x) + x phi(x)
        return 0.5f * (1.f + erff(x * 0.70710678118654752f)) + x * expf(-0.5f * x * x) * 0.39894228040143268f;
    } else if (ACT == GALV_ACT_GELU_TANH) {
        const float k = 0.79788456080286536f, x2 = x * x;
        const float t = tanhf(k * x * (1.f + 0.044715f * x2));
        return 0.5f * (1.f + t) + 0.5f * x * (1.f - t * t) * k * (1.f + 3.f * 0.044715f * x2);
    } else {
        const float s = 1.f / (1.f + expf(-x));
        return s * (1.f + x * (1.f - s));
    }
}

template <typename T, int ACT, bool VEC>
__global__ void __launch_bounds__(kThreads) mx_act_kernel(long long rows, long long cols, long long nb, long long pieces, long long per_row,
                                                          const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const T* dy,
                                                          long long dy_stride, T* dx, long long dx_stride)
{
    const long long step = (long long)gridDim.x * kThreads, dr = step / pieces, dc = step % pieces;
    const long long first = (long long)blockIdx.x * kThreads + threadIdx.x;
    long long row = first / pieces, c = first % pieces;
    for (long long item = first; item < rows * pieces; item += step) {
        float x[8], g[8];
        mx_restore8<GALV_MX8>(codes, scales, row, c, nb, per_row, x);
        mx_load8<T, VEC>(dy + row * dy_stride, c * 8, cols, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] *= act_slope<ACT>(x[i]);
        mx_store8<T, VEC>(dx + row * dx_stride, c * 8, cols, g);
        row += dr;
        c += dc;
        if (c >= pieces) { c -= pieces; ++row; }
    }
}

__device__ __forceinline__ float block_sum(float v, float* red)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) s += red[w];
    return s;
}

// One CTA a row: statistics, the two means of the gradient, dx; mean and 1/sqrt(var + eps) stay for the column sums.
template <typename T, bool LAYER>
__global__ void __launch_bounds__(kThreads) mx_norm_rows_kernel(long long rows, long long cols, long long nb, long long pitch, float eps,
                                                                const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const T* dy,
                                                                long long dy_stride, const T* __restrict__ weight, T* dx, long long dx_stride, float2* stats)
{
    __shared__ float red[kThreads / 32];
    const long long pieces = (cols + 7) / 8;
    const float inv_n = 1.f / (float)cols;
    for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
        float mean = 0.f;
        float x[8], g[8], w[8];
        if (LAYER) {
            float s = 0.f;
            for (long long c = threadIdx.x; c < pieces; c += kThreads) {
                mx_restore8<GALV_MX8>(codes, scales, row, c, nb, pitch, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) s += x[i];
            }
            mean = block_sum(s, red) * inv_n;
        }
        float s = 0.f;
        for (long long c = threadIdx.x; c < pieces; c += kThreads) {
            mx_restore8<GALV_MX8>(codes, scales, row, c, nb, pitch, x);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c * 8 + i < cols) s += (x[i] - mean) * (x[i] - mean);
        }
        const float rstd = 1.f / sqrtf(block_sum(s, red) * inv_n + eps);
        float sg = 0.f, sgx = 0.f;
        for (long long c = threadIdx.x; c < pieces; c += kThreads) {
            mx_restore8<GALV_MX8>(codes, scales, row, c, nb, pitch, x);
            mx_load8<T, false>(dy + row * dy_stride, c * 8, cols, g);
            if (weight) mx_load8<T, false>(weight, c * 8, cols, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float gw = weight ? g[i] * w[i] : g[i];
                sg += gw;
                sgx += gw * ((x[i] - mean) * rstd);
            }
        }
        const float mg = LAYER ? block_sum(sg, red) * inv_n : 0.f, mgx = block_sum(sgx, red) * inv_n;
        for (long long c = threadIdx.x; c < pieces; c += kThreads) {
            mx_restore8<GALV_MX8>(codes, scales, row, c, nb, pitch, x);
            mx_load8<T, false>(dy + row * dy_stride, c * 8, cols, g);
            if (weight) mx_load8<T, false>(weight, c * 8, cols, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = rstd * ((weight ? g[i] * w[i] : g[i]) - mg - (x[i] - mean) * rstd * mgx);
            mx_store8<T, false>(dx + row * dx_stride, c * 8, cols, g);
        }
        if (threadIdx.x == 0) stats[row] = make_float2(mean, rstd);
    }
}

// One thread a column, rows in order.  Launched before the rows' kernel, which may write dx over dy.
template <typename T>
__global__ void __launch_bounds__(kThreads) mx_norm_cols_kernel(long long rows, long long cols, long long nb, long long pitch, const uint8_t* __restrict__ codes,
                                                                const uint8_t* __restrict__ scales, const T* __restrict__ dy, long long dy_stride,
                                                                const float2* __restrict__ stats, float* dweight, float* dbias)
{
    const long long c = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (c >= cols) return;
    float dw = 0.f, db = 0.f, x[8];
    for (long long row = 0; row < rows; ++row) {
        const float2 st = stats[row];
        const float g = mx_float(dy[row * dy_stride + c]);
        mx_restore8<GALV_MX8>(codes, scales, row, c >> 3, nb, pitch, x);
        float xv = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i == (c & 7)) xv = x[i];
        dw += g * ((xv - st.x) * st.y);
        db += g;
    }
    if (dweight) dweight[c] = dw;
    if (dbias) dbias[c] = db;
}

template <bool LAYER>
__global__ void __launch_bounds__(kThreads) mx_norm_stats_kernel(long long rows, long long cols, long long nb, long long pitch, float eps,
                                                                 const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, float2* stats)
{
    __shared__ float red[kThreads / 32];
    const long long pieces = (cols + 7) / 8;
    const float inv_n = 1.f / (float)cols;
    for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
        float mean = 0.f, x[8], s = 0.f;
        if (LAYER) {
            for (long long c = threadIdx.x; c < pieces; c += kThreads) {
                mx_restore8<GALV_MX8>(codes, scales, row, c, nb, pitch, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) s += x[i];
            }
            mean = block_sum(s, red) * inv_n;
        }
        s = 0.f;
        for (long long c = threadIdx.x; c < pieces; c += kThreads) {
            mx_restore8<GALV_MX8>(codes, scales, row, c, nb, pitch, x);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c * 8 + i < cols) s += (x[i] - mean) * (x[i] - mean);
        }
        const float rstd = 1.f / sqrtf(block_sum(s, red) * inv_n + eps);
        if (threadIdx.x == 0) stats[row] = make_float2(mean, rstd);
    }
}

}  // namespace

extern "C" int galv_mx_act_backward(galv_ctx* ctx, int64_t rows, int64_t cols, int32_t act, const uint8_t* codes, const uint8_t* scales, const void* dy,
                                    int64_t dy_stride, void* dx, int64_t dx_stride, int32_t dtype, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!mx_size_ok(rows, cols) || !mx_dtype_ok(dtype) || act < GALV_ACT_GELU || act > GALV_ACT_SILU)
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_act_backward: sizes, type or function outside the limits");
    if (rows == 0) return GALV_OK;
    if (!mx_matrix_ok(dy, dy_stride, cols, dtype) || !mx_matrix_ok(dx, dx_stride, cols, dtype) || !codes || !scales || !mx_aligned(codes, 16) || !mx_aligned(scales, 16))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_act_backward: NULL or misaligned pointer, or a row stride below cols");
    if (dx == dy && dx_stride != dy_stride)
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_act_backward: dx may be dy with the same stride only");
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    const long long nb = mx_blocks(cols), pieces = (cols + 7) / 8, pitch = mx_pitch8(cols);
    const bool vec = mx_rows16(dy, dy_stride, dtype) && mx_rows16(dx, dx_stride, dtype);
    const long long blocks = (rows * pieces + kThreads - 1) / kThreads, most = (long long)ctx->num_sms * 32;
    const int grid = (int)(blocks < most ? blocks : most);
    cudaStream_t st = (cudaStream_t)stream;
#define MX_ACT(ACT)                                                                                                                                        \
    MX_DISPATCH_TYPE(dtype, if (vec) mx_act_kernel<T, ACT, true><<<grid, kThreads, 0, st>>>(rows, cols, nb, pieces, pitch, codes, scales, (const T*)dy, dy_stride, (T*)dx, dx_stride); \
                     else mx_act_kernel<T, ACT, false><<<grid, kThreads, 0, st>>>(rows, cols, nb, pieces, pitch, codes, scales, (const T*)dy, dy_stride, (T*)dx, dx_stride))
    if (act == GALV_ACT_GELU) MX_ACT(GALV_ACT_GELU);
    else if (act == GALV_ACT_GELU_TANH) MX_ACT(GALV_ACT_GELU_TANH);
    else MX_ACT(GALV_ACT_SILU);
#undef MX_ACT
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}

extern "C" size_t galv_mx_norm_workspace_bytes(const galv_ctx* ctx, int64_t rows, int64_t cols)
{
    if (!ctx || !mx_size_ok(rows, cols)) return 0;
    return ((size_t)rows * sizeof(float2) + 255) & ~(size_t)255;
}

extern "C" int galv_mx_norm_backward(galv_ctx* ctx, int64_t rows, int64_t cols, int32_t kind, float eps, const uint8_t* codes, const uint8_t* scales,
                                     const void* dy, int64_t dy_stride, const void* weight, void* dx, int64_t dx_stride, int32_t dtype, float* dweight,
                                     float* dbias, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!mx_size_ok(rows, cols) || !mx_dtype_ok(dtype) || (kind != GALV_NORM_LAYER && kind != GALV_NORM_RMS) || !(eps >= 0.f))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_norm_backward: sizes, type, kind or eps outside the limits");
    if (kind == GALV_NORM_RMS && dbias) return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_norm_backward: GALV_NORM_RMS has no bias");
    if ((dweight && !mx_aligned(dweight, 4)) || (dbias && !mx_aligned(dbias, 4)))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_norm_backward: misaligned dweight or dbias");
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    if (rows == 0) {
        e = dweight ? cudaMemsetAsync(dweight, 0, cols * 4, st) : cudaSuccess;
        if (e == cudaSuccess && dbias) e = cudaMemsetAsync(dbias, 0, cols * 4, st);
        return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
    }
    if (!mx_matrix_ok(dy, dy_stride, cols, dtype) || !mx_matrix_ok(dx, dx_stride, cols, dtype) || !codes || !scales || !mx_aligned(codes, 16) ||
        !mx_aligned(scales, 16) || (weight && !mx_aligned(weight, mx_size_of(dtype))))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_norm_backward: NULL or misaligned pointer, or a row stride below cols");
    if (dx == dy && dx_stride != dy_stride)
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_norm_backward: dx may be dy with the same stride only");
    if (!workspace || !mx_aligned(workspace, 256) || workspace_bytes < galv_mx_norm_workspace_bytes(ctx, rows, cols))
        return galv_set_error(ctx, GALV_ERR_WORKSPACE, "galv_mx_norm_backward: workspace NULL, misaligned or too small");
    const long long nb = mx_blocks(cols), pitch = mx_pitch8(cols), most = (long long)ctx->num_sms * 8;
    const int grid = (int)(rows < most ? rows : most), cgrid = (int)((cols + kThreads - 1) / kThreads);
    float2* stats = reinterpret_cast<float2*>(workspace);
    if (kind == GALV_NORM_LAYER) mx_norm_stats_kernel<true><<<grid, kThreads, 0, st>>>(rows, cols, nb, pitch, eps, codes, scales, stats);
    else mx_norm_stats_kernel<false><<<grid, kThreads, 0, st>>>(rows, cols, nb, pitch, eps, codes, scales, stats);
    MX_DISPATCH_TYPE(dtype,
        if (dweight || dbias) mx_norm_cols_kernel<T><<<cgrid, kThreads, 0, st>>>(rows, cols, nb, pitch, codes, scales, (const T*)dy, dy_stride, stats, dweight, dbias);
        if (kind == GALV_NORM_LAYER) mx_norm_rows_kernel<T, true><<<grid, kThreads, 0, st>>>(rows, cols, nb, pitch, eps, codes, scales, (const T*)dy, dy_stride, (const T*)weight, (T*)dx, dx_stride, stats);
        else mx_norm_rows_kernel<T, false><<<grid, kThreads, 0, st>>>(rows, cols, nb, pitch, eps, codes, scales, (const T*)dy, dy_stride, (const T*)weight, (T*)dx, dx_stride, stats));
    e = cudaGetLastError();
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}
