// Microscaled blocks: packing and restoring a matrix.
//
// One pass over the data; a piece of 8 columns is 16 bytes of 16-bit numbers, four threads a block of 32, whose largest magnitude they find with two
// shuffles (two numbers at a time: magnitudes order like their bits).  Bound by memory, what is read and written once, 2 + 33/32 bytes an element from 16
// bits to 8: 8192 x 8192 in bf16 is packed in 37.6 us (5.4 TB/s, 79 % of the issue slots busy; to 4 bits 39) and restored in 32.6 (6.2 TB/s; 29 from 4).

#include "galv_mx.cuh"

namespace {

// Rows up to rows_out and pieces up to `pieces` have a scale byte to write; rows and nb * 4 pieces lie in the matrix.
template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(kMxThreads) mx_pack_kernel(const MxSpread spread, unsigned rows, unsigned rows_out, int cols, unsigned nb, unsigned pieces, int per_row,
                                                             const T* __restrict__ x, long long stride, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales)
{
    for (long long block = blockIdx.x; block < spread.blocks; block += gridDim.x) {
        const MxPlace at = mx_place(spread, block);
        constexpr int U = MxEach<T>::count;
        MxPiece<T> raw[U];
        const T* from = x + at.row * stride;
        uint8_t* to = codes + ((long long)at.row * nb * 4 + at.c) * FMT;
#pragma unroll
        for (int h = 0; h < U; ++h, from += spread.dr * stride) {
            const unsigned row = at.row + h * spread.dr, c = at.c + h * spread.dc;
            if (row < rows && c < nb * 4) {
                raw[h] = mx_fetch8<T, VEC>(from, (int)c * 8, cols, spread.log >= 5);
            } else {
#pragma unroll
                for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[h].q[i] = make_uint4(0, 0, 0, 0);
            }
        }
#pragma unroll
        for (int h = 0; h < U; ++h, to += ((long long)spread.dr * nb * 4 + spread.dc) * FMT) {
            const unsigned row = at.row + h * spread.dr, c = at.c + h * spread.dc;
            uint32_t m = mx_most<T>(raw[h]);
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));            // the four threads of a block lie next to one another
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
            const int byte = mx_scale_byte<FMT>(m);
            if (row < rows && c < nb * 4) {
                const float inv = mx_inverse(byte);
                float v[8];
                mx_floats(raw[h], v);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= inv;
                if (FMT == GALV_MX8) {
                    uint2 w;
                    w.x = mx_to8(v[0], v[1], v[2], v[3]);
                    w.y = mx_to8(v[4], v[5], v[6], v[7]);
                    if (byte == 255) w = make_uint2(0, 0);
                    *reinterpret_cast<uint2*>(to) = w;
                } else {
                    *reinterpret_cast<uint32_t*>(to) = byte == 255 ? 0 : mx_to4(v);
                }
            }
            if ((c & 3) == 0 && row < rows_out && c < pieces) scales[mx_scale_at<FMT>(row, c >> 2, per_row)] = (uint8_t)byte;      // zero outside the matrix
        }
    }
}

constexpr int kUnpackEach = 4;                            // pieces a thread, of any type: what is read is small
template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(kMxThreads) mx_unpack_kernel(const MxSpread spread, unsigned rows, int cols, unsigned nb, unsigned pieces, int per_row,
                                                               const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, T* __restrict__ x, long long stride)
{
    __shared__ __align__(16) T buf[VEC ? 1 : kMxThreads / 32][256 + 8];
    for (long long block = blockIdx.x; block < spread.blocks; block += gridDim.x) {
        const MxPlace at = mx_place(spread, block);
        constexpr int U = kUnpackEach;
        uint2 code[U];
        int byte[U];
        const uint8_t* held = codes + ((long long)at.row * nb * 4 + at.c) * FMT;
#pragma unroll
        for (int h = 0; h < U; ++h, held += ((long long)spread.dr * nb * 4 + spread.dc) * FMT) {
            const unsigned row = at.row + h * spread.dr, c = at.c + h * spread.dc;
            if (row < rows && c < pieces) {
                if (FMT == GALV_MX8) code[h] = __ldg(reinterpret_cast<const uint2*>(held));
                else code[h].x = __ldg(reinterpret_cast<const uint32_t*>(held));
                byte[h] = __ldg(scales + mx_scale_at<FMT>(row, c >> 2, per_row));
            }
        }
        T* to = x + at.row * stride;
#pragma unroll
        for (int h = 0; h < U; ++h, to += spread.dr * stride) {
            const unsigned row = at.row + h * spread.dr, c = at.c + h * spread.dc;
            const bool in = row < rows && c < pieces;
            if (VEC && !in) continue;
            if (!VEC && !in) { code[h] = make_uint2(0, 0); byte[h] = 0; }
            float v[8];
            if (FMT == GALV_MX8) {
                mx_from8(code[h].x, v);
                mx_from8(code[h].y, v + 4);
            } else {
                mx_from4(code[h].x, v);
            }
            const float s = mx_scale(byte[h]);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= s;
            if (VEC) mx_store8<T, true>(to, (int)c * 8, cols, mx_piece_held<T>(v));
            else mx_store_spread<T>(buf[threadIdx.x / 32], to, c, row < rows, x, stride, spread, at, h, rows, cols, mx_piece_held<T>(v));
        }
    }
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
    const int nb = (int)mx_blocks(cols);
    const bool vec = mx_rows16(x, x_stride, dtype);
    // every scale byte is written, those behind the rows and blocks too
    const unsigned rows_out = (unsigned)(fmt == GALV_MX8 ? rows : (rows + 127) / 128 * 128);
    const int per_row = fmt == GALV_MX8 ? (int)mx_pitch8(cols) : (nb + 3) / 4;
    const int pieces = fmt == GALV_MX8 ? per_row * 4 : per_row * 16;
    const MxSpread spread(rows_out, pieces, dtype == GALV_F32 ? MxEach<float>::count : MxEach<__half>::count);
    const int grid = spread.grid();
    cudaStream_t st = (cudaStream_t)stream;
#define MX_PACK(FMT)                                                                                                                                         \
    MX_DISPATCH_TYPE(dtype, if (vec) mx_pack_kernel<T, FMT, true><<<grid, kMxThreads, 0, st>>>(spread, (unsigned)rows, rows_out, (int)cols, nb, pieces, per_row, (const T*)x, x_stride, codes, scales); \
                     else mx_pack_kernel<T, FMT, false><<<grid, kMxThreads, 0, st>>>(spread, (unsigned)rows, rows_out, (int)cols, nb, pieces, per_row, (const T*)x, x_stride, codes, scales))
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
    const int nb = (int)mx_blocks(cols), pieces = (int)((cols + 7) / 8);
    const int per_row = fmt == GALV_MX8 ? (int)mx_pitch8(cols) : (nb + 3) / 4;
    const bool vec = mx_rows16(x, x_stride, dtype);
    const MxSpread spread(rows, pieces, kUnpackEach);
    const int grid = spread.grid();
    cudaStream_t st = (cudaStream_t)stream;
#define MX_UNPACK(FMT)                                                                                                                         \
    MX_DISPATCH_TYPE(dtype, if (vec) mx_unpack_kernel<T, FMT, true><<<grid, kMxThreads, 0, st>>>(spread, (unsigned)rows, (int)cols, nb, pieces, per_row, codes, scales, (T*)x, x_stride); \
                     else mx_unpack_kernel<T, FMT, false><<<grid, kMxThreads, 0, st>>>(spread, (unsigned)rows, (int)cols, nb, pieces, per_row, codes, scales, (T*)x, x_stride))
    if (fmt == GALV_MX8) MX_UNPACK(GALV_MX8);
    else MX_UNPACK(GALV_MX4);
#undef MX_UNPACK
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}

namespace {

cudaError_t encode(CUtensorMap* map, CUtensorMapDataType type, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box, bool swizzle)
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
    const cuuint32_t one[3] = {1, 1, 1};
    const CUresult r = fn(map, type, rank, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace

cudaError_t galv_mx_map(CUtensorMap* map, CUtensorMapDataType type, const void* base, uint64_t rows, uint64_t cols, uint64_t pitch, uint32_t box_rows, uint32_t box_cols,
                        bool swizzle)
{
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {pitch};
    const cuuint32_t box[2] = {box_cols, box_rows};
    return encode(map, type, 2, base, dims, strides, box, swizzle);
}

cudaError_t galv_map_3d(CUtensorMap* map, CUtensorMapDataType type, const void* base, uint64_t matrices, uint64_t rows, uint64_t cols, uint64_t pitch, uint32_t box_rows, uint32_t box_cols)
{
    const cuuint64_t dims[3] = {cols, rows, matrices}, strides[2] = {pitch, rows * pitch};
    const cuuint32_t box[3] = {box_cols, box_rows, 1};
    return encode(map, type, 3, base, dims, strides, box, true);
}
