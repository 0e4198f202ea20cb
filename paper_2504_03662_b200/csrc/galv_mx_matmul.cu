// Product of two tensors held in 4 bits.

#include "galv_mx.cuh"

namespace {

constexpr int kTile = 64, kDeep = 16, kThreads = 256;

// 64 x 64 outputs a CTA, 4 x 4 a thread, fp32 sums in order of the summed index.
__device__ __forceinline__ void tile_step(const float (*a)[kTile + 4], const float (*b)[kTile + 4], int ty, int tx, float (&acc)[4][4])
{
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
        float u[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { u[i] = a[k][ty * 4 + i]; v[i] = b[k][tx * 4 + i]; }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(u[i], v[j], acc[i][j]);
    }
}

// The elements of 16 columns are multiplied as they are and the sum takes the two blocks' powers of two at once: a held value alone may pass fp32's
// range (6 * 2^126 is one) where the product does not.
template <typename T>
__global__ void __launch_bounds__(kThreads) mx_matmul_simple_kernel(long long m, long long n, long long nb, const uint8_t* __restrict__ ac, const uint8_t* __restrict__ as,
                                                                    const uint8_t* __restrict__ bc, const uint8_t* __restrict__ bs, const T* __restrict__ bias,
                                                                    T* __restrict__ y, long long y_stride)
{
    __shared__ float a[kDeep][kTile + 4], b[kDeep][kTile + 4];
    __shared__ int sc[2][kTile];
    const long long m0 = (long long)blockIdx.y * kTile, n0 = (long long)blockIdx.x * kTile, tiles = (nb + 3) / 4;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    for (long long p0 = 0; p0 < nb * 4; p0 += kDeep / 8) {
        __syncthreads();
        const int which = threadIdx.x / 128, r = threadIdx.x % 128 / 2, p = threadIdx.x % 2;
        const long long row = (which ? n0 : m0) + r;
        float v[8] = {};
        int byte = 0;
        if (row < (which ? n : m)) {
            mx_from4(*reinterpret_cast<const uint32_t*>((which ? bc : ac) + row * nb * 16 + (p0 + p) * 4), v);
            byte = (which ? bs : as)[mx_scale_at<GALV_MX4>(row, p0 >> 2, tiles)];
        }
        if (p == 0) sc[which][r] = byte;
#pragma unroll
        for (int i = 0; i < 8; ++i) (which ? b : a)[p * 8 + i][r] = byte == 255 ? __uint_as_float(0x7fc00000u) : v[i];
        __syncthreads();
        float part[4][4] = {};
        tile_step(a, b, ty, tx, part);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] += ldexpf(part[i][j], sc[0][ty * 4 + i] + sc[1][tx * 4 + j] - 254);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long long r = m0 + ty * 4 + i, c = n0 + tx * 4 + j;
            if (r < m && c < n) y[r * y_stride + c] = mx_round<T>(bias ? acc[i][j] + mx_float(bias[c]) : acc[i][j]);
        }
}

}  // namespace

extern "C" size_t galv_mx_matmul_workspace_bytes(const galv_ctx* ctx, int64_t m, int64_t n, int64_t k)
{
    if (!ctx || !mx_size_ok(m, k) || !mx_size_ok(n, k)) return 0;
    return 0;
}

extern "C" int galv_mx_matmul(galv_ctx* ctx, int64_t m, int64_t n, int64_t k, const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes,
                              const uint8_t* b_scales, const void* bias, void* y, int64_t y_stride, int32_t dtype, void* workspace, size_t workspace_bytes,
                              void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!mx_size_ok(m, n) || !mx_size_ok(n, k) || n < 1 || !mx_dtype_ok(dtype))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_matmul: sizes or type outside the limits");
    if (m == 0) return GALV_OK;
    if (!a_codes || !a_scales || !b_codes || !b_scales || !mx_aligned(a_codes, 16) || !mx_aligned(a_scales, 16) || !mx_aligned(b_codes, 16) ||
        !mx_aligned(b_scales, 16) || !mx_matrix_ok(y, y_stride, n, dtype) || (bias && !mx_aligned(bias, mx_size_of(dtype))))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_matmul: NULL or misaligned pointer, or a row stride below n");
    const size_t need = galv_mx_matmul_workspace_bytes(ctx, m, n, k);
    if (need && (!workspace || !mx_aligned(workspace, 256) || workspace_bytes < need))
        return galv_set_error(ctx, GALV_ERR_WORKSPACE, "galv_mx_matmul: workspace NULL, misaligned or too small");
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    cudaStream_t st = (cudaStream_t)stream;
    const dim3 grid((unsigned)((n + kTile - 1) / kTile), (unsigned)((m + kTile - 1) / kTile));
    MX_DISPATCH_TYPE(dtype, mx_matmul_simple_kernel<T><<<grid, kThreads, 0, st>>>(m, n, mx_blocks(k), a_codes, a_scales, b_codes, b_scales, (const T*)bias, (T*)y, y_stride));
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}
