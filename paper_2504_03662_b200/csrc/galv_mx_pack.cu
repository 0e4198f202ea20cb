// Microscaled blocks: packing and restoring a matrix.
//
// One pass over the data; a thread has 8 columns (16 bytes of 16-bit numbers), four threads a block of 32, whose largest magnitude they
// find with two shuffles.  The pass is bound by memory: what is read and written once, 2 + 33/32 bytes an element from 16 bits to 8.

#include "galv_mx.cuh"

namespace {

constexpr int kThreads = 256;

// Pieces of 8 columns, row by row; a row has `pieces` of them, up to the last scale byte that has to be written.
struct PieceWalk {
    long long row;
    long long c;
    __device__ PieceWalk(long long item, long long pieces) : row(item / pieces), c(item % pieces) {}
    __device__ void step(long long dr, long long dc, long long pieces)
    {
        row += dr;
        c += dc;
        if (c >= pieces) { c -= pieces; ++row; }
    }
};

template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(kThreads) mx_pack_kernel(long long rows, long long rows_out, long long cols, long long nb, long long pieces, long long per_row,
                                                           const T* __restrict__ x, long long stride, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales)
{
    const long long step = (long long)gridDim.x * kThreads, dr = step / pieces, dc = step % pieces;
    PieceWalk at((long long)blockIdx.x * kThreads + threadIdx.x, pieces);
    // a row has a multiple of 4 pieces, so the four threads of a block agree; a warp leaves as a whole
    for (long long item = (long long)blockIdx.x * kThreads + threadIdx.x; item - threadIdx.x % 32 < rows_out * pieces; item += step, at.step(dr, dc, pieces)) {
        const bool in = at.row < rows && at.c < nb * 4;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
        if (in) mx_load8<T, VEC>(x + at.row * stride, at.c * 8, cols, v);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const int byte = mx_scale_byte<FMT>(m);
        const float inv = byte == 255 ? 0.f : mx_inverse(byte);
        if (in) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = byte == 255 ? 0.f : v[i] * inv;
            if (FMT == GALV_MX8) {
                uint2 w;
                w.x = mx_to8(v[0], v[1], v[2], v[3]);
                w.y = mx_to8(v[4], v[5], v[6], v[7]);
                *reinterpret_cast<uint2*>(codes + (at.row * nb * 32 + at.c * 8)) = w;
            } else {
                *reinterpret_cast<uint32_t*>(codes + (at.row * nb * 16 + at.c * 4)) = mx_to4(v);
            }
        }
        if ((at.c & 3) == 0 && at.row < rows_out) scales[mx_scale_at<FMT>(at.row, at.c >> 2, per_row)] = (uint8_t)byte;      // zero outside the matrix
    }
}

template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(kThreads) mx_unpack_kernel(long long rows, long long cols, long long nb, long long pieces, long long per_row,
                                                             const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, T* __restrict__ x, long long stride)
{
    const long long step = (long long)gridDim.x * kThreads, dr = step / pieces, dc = step % pieces;
    PieceWalk at((long long)blockIdx.x * kThreads + threadIdx.x, pieces);
    for (long long item = (long long)blockIdx.x * kThreads + threadIdx.x; item < rows * pieces; item += step, at.step(dr, dc, pieces)) {
        float v[8];
        mx_restore8<FMT>(codes, scales, at.row, at.c, nb, per_row, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = mx_held<T>(v[i]);
        mx_store8<T, VEC>(x + at.row * stride, at.c * 8, cols, v);
    }
}

int pass_grid(const galv_ctx* ctx, long long items)
{
    const long long blocks = (items + kThreads - 1) / kThreads, most = (long long)ctx->num_sms * 32;
    return (int)(blocks < most ? blocks : most);
}

}  // namespace

extern "C" size_t galv_mx_codes_bytes(int64_t rows, int64_t cols, int32_t fmt)
{
    if (!mx_size_ok(rows, cols) || (fmt != GALV_MX8 && fmt != GALV_MX4)) return 0;
    return (size_t)rows * mx_blocks(cols) * (fmt == GALV_MX8 ? 32 : 16);
}

extern "C" size_t galv_mx_scales_bytes(int64_t rows, int64_t cols, int32_t fmt)
{
    if (!mx_size_ok(rows, cols) || (fmt != GALV_MX8 && fmt != GALV_MX4)) return 0;
    if (fmt == GALV_MX8) return (size_t)rows * mx_pitch8(cols);
    return (size_t)((rows + 127) / 128) * ((mx_blocks(cols) + 3) / 4) * 512;
}

extern "C" int galv_mx_pack(galv_ctx* ctx, int64_t rows, int64_t cols, const void* x, int64_t x_stride, int32_t dtype, int32_t fmt, uint8_t* codes,
                            uint8_t* scales, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!mx_size_ok(rows, cols) || !mx_dtype_ok(dtype) || (fmt != GALV_MX8 && fmt != GALV_MX4))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_pack: sizes, type or format outside the limits");
    if (rows == 0) return GALV_OK;
    if (!mx_matrix_ok(x, x_stride, cols, dtype) || !codes || !scales || !mx_aligned(codes, 16) || !mx_aligned(scales, 16))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_pack: NULL or misaligned pointer, or a row stride below cols");
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    const long long nb = mx_blocks(cols);
    const bool vec = mx_rows16(x, x_stride, dtype);
    // every scale byte is written, those behind the rows and blocks too
    const long long rows_out = fmt == GALV_MX8 ? rows : (rows + 127) / 128 * 128;
    const long long pieces = fmt == GALV_MX8 ? mx_pitch8(cols) * 4 : (nb + 3) / 4 * 16, per_row = fmt == GALV_MX8 ? mx_pitch8(cols) : (nb + 3) / 4;
    const int grid = pass_grid(ctx, rows_out * pieces);
    cudaStream_t st = (cudaStream_t)stream;
#define MX_PACK(FMT)                                                                                                                                         \
    MX_DISPATCH_TYPE(dtype, if (vec) mx_pack_kernel<T, FMT, true><<<grid, kThreads, 0, st>>>(rows, rows_out, cols, nb, pieces, per_row, (const T*)x, x_stride, codes, scales); \
                     else mx_pack_kernel<T, FMT, false><<<grid, kThreads, 0, st>>>(rows, rows_out, cols, nb, pieces, per_row, (const T*)x, x_stride, codes, scales))
    if (fmt == GALV_MX8) MX_PACK(GALV_MX8);
    else MX_PACK(GALV_MX4);
#undef MX_PACK
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}

extern "C" int galv_mx_unpack(galv_ctx* ctx, int64_t rows, int64_t cols, int32_t fmt, const uint8_t* codes, const uint8_t* scales, void* x, int64_t x_stride,
                              int32_t dtype, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!mx_size_ok(rows, cols) || !mx_dtype_ok(dtype) || (fmt != GALV_MX8 && fmt != GALV_MX4))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_unpack: sizes, type or format outside the limits");
    if (rows == 0) return GALV_OK;
    if (!mx_matrix_ok(x, x_stride, cols, dtype) || !codes || !scales || !mx_aligned(codes, 16) || !mx_aligned(scales, 16))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_unpack: NULL or misaligned pointer, or a row stride below cols");
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    const long long nb = mx_blocks(cols), pieces = (cols + 7) / 8, per_row = fmt == GALV_MX8 ? mx_pitch8(cols) : (nb + 3) / 4;
    const bool vec = mx_rows16(x, x_stride, dtype);
    const int grid = pass_grid(ctx, rows * pieces);
    cudaStream_t st = (cudaStream_t)stream;
#define MX_UNPACK(FMT)                                                                                                                         \
    MX_DISPATCH_TYPE(dtype, if (vec) mx_unpack_kernel<T, FMT, true><<<grid, kThreads, 0, st>>>(rows, cols, nb, pieces, per_row, codes, scales, (T*)x, x_stride); \
                     else mx_unpack_kernel<T, FMT, false><<<grid, kThreads, 0, st>>>(rows, cols, nb, pieces, per_row, codes, scales, (T*)x, x_stride))
    if (fmt == GALV_MX8) MX_UNPACK(GALV_MX8);
    else MX_UNPACK(GALV_MX4);
#undef MX_UNPACK
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}

cudaError_t galv_mx_map(CUtensorMap* map, CUtensorMapDataType type, const void* base, uint64_t rows, uint64_t cols, uint64_t pitch, uint32_t box_rows, uint32_t box_cols,
                        bool swizzle)
{
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode fn = [] {                          // looked up once a process
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess) { (void)cudaGetLastError(); p = nullptr; }
        else if (q != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<Encode>(p);
    }();
    if (!fn) return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {pitch};
    const cuuint32_t box[2] = {box_cols, box_rows}, one[2] = {1, 1};
    const CUresult r = fn(map, type, 2, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}
