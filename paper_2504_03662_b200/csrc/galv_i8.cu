// Rows of 8-bit integers with one scale each: packing and restoring a matrix.
//
// A row's scale needs all of the row before its first code: up to 32768 columns stay in the registers of the threads that read them, what lies
// behind is read twice (from L2).  A code is the whole number nearest to the exact quotient x / s: x * (1 / s) is off by some units of its last place, so
// the remainder x - q s, which an fp32 multiply-add has exactly, decides next to a half.
// Bound by memory and issue slots, what is read and written once, 3 bytes an element from 16 bits: 4096 x 8192 in bf16 is packed in 22 us (4.5 TB/s; 15 instructions an element), 8192 x 4096 in fp32 in
// 29 (5.7 TB/s).  With 8 pieces a thread in place of 4 (two CTAs an SM for five) the first took 41.

#include "galv_i8.cuh"
#include "galv_tc.cuh"

namespace {

// The numbers nearest to v / s in the low bytes of t, ties to even; inv is 1 / s rounded, half is s / 2.  With |v / s| < 127.5 the sum v * inv + 1.5 * 2^23 is
// rounded to a whole number q off by one at most, and only where the remainder r = v - q s has left [-half, half].  r is a multiple of a quarter of s's last
// place and not above it by more than its rounding can tell (at q = 1 and v just below half the rounded |r| may be half itself: q goes to 0 then, which is right).
__device__ __forceinline__ uint2 codes_of(const float (&v)[8], float s, float inv, float half)
{
    constexpr float magic = 12582912.f;
    float q[8], r[8], most = 0.f;
    uint32_t t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float w = fmaf(v[i], inv, magic);
        t[i] = __float_as_uint(w);
        q[i] = w - magic;
        r[i] = fmaf(-q[i], s, v[i]);
        most = fmaxf(most, fabsf(r[i]));
    }
    if (most >= half) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = fabsf(r[i]);
            if (a > half || (a == half && (t[i] & 1))) t[i] += r[i] > 0.f ? 1 : -1;
        }
    }
    uint2 w;
    w.x = __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
    w.y = __byte_perm(__byte_perm(t[4], t[5], 0x0040), __byte_perm(t[6], t[7], 0x0040), 0x5410);
    return w;
}

// WARPS of a CTA's (8, or all of 16 or 32) have a row, of which a thread keeps 4 pieces of 8 columns in registers.
constexpr int kPieces = 4;
template <int WARPS> constexpr int kWarps = WARPS < 8 ? 8 : WARPS;
template <typename T, bool VEC, int WARPS>
__global__ void __launch_bounds__(kWarps<WARPS> * 32, (sizeof(T) == 2 ? 40 : 32) / kWarps<WARPS>)
i8_pack_kernel(long long rows, int cols, int pieces, const T* __restrict__ x, long long stride, int8_t* __restrict__ codes, float* __restrict__ scales)
{
    constexpr int threads = WARPS * 32, rows_each = kWarps<WARPS> / WARPS, P = kPieces;
    __shared__ uint32_t found[2][kWarps<WARPS>];
    const int t = threadIdx.x % threads, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    int turn = 0;
    tc::before_is_over();
    tc::next_may_start();                                 // behind the wait: the product that reads the codes takes it that all before this kernel is over
    for (long long row0 = (long long)blockIdx.x * rows_each; row0 < rows; row0 += (long long)gridDim.x * rows_each, turn ^= 1) {
        const long long row = row0 + warp / WARPS;
        const bool in = row < rows;
        const T* from = x + row * stride;
        MxPiece<T> raw[P];
        uint32_t m = 0;
        if (in) {
#pragma unroll
            for (int h = 0; h < P; ++h) {
                const unsigned c = t + h * threads;       // pieces of a row reach 2^28, and some more in the last step
                if (c < (unsigned)pieces) raw[h] = mx_fetch8<T, VEC>(from, (int)(c * 8), cols);
            }
#pragma unroll
            for (int h = 0; h < P; ++h)
                if (t + h * threads < (unsigned)pieces) m = max(m, mx_most<T>(raw[h]));
            for (unsigned c = t + P * threads; c < (unsigned)pieces; c += threads) m = max(m, mx_most<T>(mx_fetch8<T, VEC>(from, (int)(c * 8), cols)));
        }
        m = __reduce_max_sync(0xffffffffu, m);
        if (WARPS > 1) {                                  // the row's warps meet at a barrier of theirs
            if (lane == 0) found[turn][warp] = m;
            asm volatile("bar.sync %0, %1;" :: "r"(1 + warp / WARPS), "n"(threads) : "memory");
#pragma unroll
            for (int w = 0; w < WARPS; ++w) m = max(m, found[turn][warp / WARPS * WARPS + w]);
        }
        if (!in) continue;
        const bool bad = m >= 0x7f800000u;
        const float s = __fdiv_rn(fmaxf(__uint_as_float(bad ? 0u : m), kI8Least), 127.f), inv = __fdiv_rn(1.f, s), half = s * 0.5f;
        int8_t* to = codes + row * ((long long)pieces * 8);
        auto put = [&](unsigned c, const MxPiece<T>& p) {
            float v[8];
            mx_floats(p, v);
            *reinterpret_cast<uint2*>(to + c * 8ll) = bad ? make_uint2(0, 0) : codes_of(v, s, inv, half);
        };
#pragma unroll
        for (int h = 0; h < P; ++h)
            if (t + h * threads < (unsigned)pieces) put(t + h * threads, raw[h]);
        for (unsigned c = t + P * threads; c < (unsigned)pieces; c += threads) put(c, mx_fetch8<T, VEC>(from, (int)(c * 8), cols));
        if (t == 0) scales[row] = bad ? __uint_as_float(0x7fc00000u) : s;
    }
}

constexpr int kEach = 4;
constexpr float kMostNumber = 3.402823466e38f;
template <typename T, bool VEC>
__global__ void __launch_bounds__(kMxThreads) i8_unpack_kernel(const MxSpread spread, unsigned rows, int cols, long long pitch, const int8_t* __restrict__ codes, const float* __restrict__ scales,
                                                               T* __restrict__ x, long long stride)
{
    __shared__ __align__(16) T buf[VEC ? 1 : kMxThreads / 32][256 + 8];
    const unsigned pieces = (unsigned)((cols + 7ll) / 8);
    for (long long block = blockIdx.x; block < spread.blocks; block += gridDim.x) {
        const MxPlace at = mx_place(spread, block);
        uint2 code[kEach];
        float s[kEach];
#pragma unroll
        for (int h = 0; h < kEach; ++h) {
            const unsigned row = at.row + h * spread.dr, c = at.c + h * spread.dc;
            code[h] = make_uint2(0, 0);
            s[h] = 0.f;
            if (row < rows && c < pieces) {
                code[h] = __ldg(reinterpret_cast<const uint2*>(codes + row * pitch + c * 8ll));
                s[h] = __ldg(scales + row);
            }
        }
#pragma unroll
        for (int h = 0; h < kEach; ++h) {
            const unsigned row = at.row + h * spread.dr, c = at.c + h * spread.dc;
            const bool in = row < rows && c < pieces;
            if (VEC && !in) continue;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = (float)(int8_t)((i < 4 ? code[h].x : code[h].y) >> (i % 4 * 8)) * s[h];
                if (isinf(v[i])) v[i] = copysignf(kMostNumber, v[i]);      // 127 times a scale that was rounded up
            }
            T* to = x + row * stride;
            if (VEC) mx_store8<T, true>(to, (int)c * 8, cols, mx_piece_held<T>(v));
            else mx_store_spread<T>(buf[threadIdx.x / 32], to, c, row < rows, x, stride, spread, at, h, rows, cols, mx_piece_held<T>(v));
        }
    }
}

template <typename T, bool VEC, int WARPS>
void launch_pack(int num_sms, int64_t rows, int64_t cols, const T* x, int64_t stride, int8_t* codes, int64_t pitch, float* scales, cudaStream_t st)
{
    constexpr int each = kWarps<WARPS> / WARPS;
    const int64_t ctas = (rows + each - 1) / each, most = (int64_t)num_sms * 32;
    tc::Launch l((unsigned)(ctas < most ? ctas : most), kWarps<WARPS> * 32, 0, 0, true, st);
    cudaLaunchKernelEx(&l.cfg, i8_pack_kernel<T, VEC, WARPS>, (long long)rows, (int)cols, (int)(pitch / 8), x, (long long)stride, codes, scales);
}

// As many warps a row as keep all of it in registers (up to 32768 columns), and 8 where there are few rows.
template <typename T, bool VEC>
void pack_by_size(int num_sms, int64_t rows, int64_t cols, const T* x, int64_t stride, int8_t* codes, int64_t pitch, float* scales, cudaStream_t st)
{
    if (cols > 16384) launch_pack<T, VEC, 32>(num_sms, rows, cols, x, stride, codes, pitch, scales, st);
    else if (cols > 8192) launch_pack<T, VEC, 16>(num_sms, rows, cols, x, stride, codes, pitch, scales, st);
    else if (cols > 4096 || (cols > 256 && rows <= 2 * num_sms)) launch_pack<T, VEC, 8>(num_sms, rows, cols, x, stride, codes, pitch, scales, st);
    else if (cols > 2048) launch_pack<T, VEC, 4>(num_sms, rows, cols, x, stride, codes, pitch, scales, st);
    else if (cols > 1024) launch_pack<T, VEC, 2>(num_sms, rows, cols, x, stride, codes, pitch, scales, st);
    else launch_pack<T, VEC, 1>(num_sms, rows, cols, x, stride, codes, pitch, scales, st);
}

}  // namespace

cudaError_t galv_i8_pack_launch(int num_sms, int64_t rows, int64_t cols, const void* x, int64_t stride, int32_t dtype, int8_t* codes, int64_t pitch, float* scales, cudaStream_t st)
{
    MX_DISPATCH_TYPE(dtype, if (mx_rows16(x, stride, dtype)) pack_by_size<T, true>(num_sms, rows, cols, (const T*)x, stride, codes, pitch, scales, st);
                     else pack_by_size<T, false>(num_sms, rows, cols, (const T*)x, stride, codes, pitch, scales, st));
    return cudaGetLastError();
}

extern "C" size_t galv_i8_codes_bytes(int64_t rows, int64_t cols) { return mx_size_ok(rows, cols) ? (size_t)rows * i8_pitch(cols) : 0; }

extern "C" int galv_i8_pack(galv_ctx* ctx, int64_t rows, int64_t cols, const void* x, int64_t x_stride, int32_t dtype, int8_t* codes, float* scales, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!mx_size_ok(rows, cols) || !mx_dtype_ok(dtype)) return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_i8_pack: sizes or type outside the limits");
    if (rows == 0) return GALV_OK;
    if (!mx_matrix_ok(x, x_stride, cols, dtype) || !codes || !scales || !mx_aligned(codes, 16) || !mx_aligned(scales, 4))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_i8_pack: NULL or misaligned pointer, or a row stride below cols");
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    const cudaError_t e = galv_i8_pack_launch(ctx->num_sms, rows, cols, x, x_stride, dtype, codes, i8_pitch(cols), scales, (cudaStream_t)stream);
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}

extern "C" int galv_i8_unpack(galv_ctx* ctx, int64_t rows, int64_t cols, const int8_t* codes, const float* scales, void* x, int64_t x_stride, int32_t dtype, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!mx_size_ok(rows, cols) || !mx_dtype_ok(dtype)) return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_i8_unpack: sizes or type outside the limits");
    if (rows == 0) return GALV_OK;
    if (!mx_matrix_ok(x, x_stride, cols, dtype) || !codes || !scales || !mx_aligned(codes, 16) || !mx_aligned(scales, 4))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_i8_unpack: NULL or misaligned pointer, or a row stride below cols");
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    const MxSpread spread(rows, (cols + 7) / 8, kEach);
    MX_DISPATCH_TYPE(dtype, if (mx_rows16(x, x_stride, dtype)) i8_unpack_kernel<T, true><<<spread.grid(), kMxThreads, 0, (cudaStream_t)stream>>>(spread, (unsigned)rows, (int)cols, i8_pitch(cols), codes, scales, (T*)x, x_stride);
                     else i8_unpack_kernel<T, false><<<spread.grid(), kMxThreads, 0, (cudaStream_t)stream>>>(spread, (unsigned)rows, (int)cols, i8_pitch(cols), codes, scales, (T*)x, x_stride));
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}
