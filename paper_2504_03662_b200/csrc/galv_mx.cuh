// Microscaled blocks: conversions and row access shared by the kernels that pack, restore and use them.
// The format is described in include/galv.h.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "galv_internal.h"

// Calls run on the context's device, whichever is current.
struct MxDevice {
    int old = -1;
    cudaError_t err;
    explicit MxDevice(const galv_ctx* ctx)
    {
        err = cudaGetDevice(&old);
        if (err == cudaSuccess && old != ctx->device) err = cudaSetDevice(ctx->device);
        else old = -1;
    }
    ~MxDevice() { if (old >= 0) cudaSetDevice(old); }
};

constexpr int64_t kMxMost = (int64_t(1) << 31) - 128;      // rows and columns stay below this

inline bool mx_size_ok(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 1 && rows < kMxMost && cols < kMxMost; }
inline bool mx_dtype_ok(int32_t t) { return t == GALV_F32 || t == GALV_BF16 || t == GALV_F16; }
inline int mx_size_of(int32_t t) { return t == GALV_F32 ? 4 : 2; }
inline bool mx_aligned(const void* p, int a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
// a matrix of numbers: present, aligned to its element, rows that do not overlap
inline bool mx_matrix_ok(const void* p, int64_t stride, int64_t cols, int32_t t) { return p && mx_aligned(p, mx_size_of(t)) && stride >= cols && stride < (int64_t(1) << 40); }
// its rows can be read in 16-byte pieces
inline bool mx_rows16(const void* p, int64_t stride, int32_t t) { return mx_aligned(p, 16) && stride * mx_size_of(t) % 16 == 0; }
inline int64_t mx_blocks(int64_t cols) { return (cols + 31) / 32; }
inline int64_t mx_pitch8(int64_t cols) { return (mx_blocks(cols) + 15) / 16 * 16; }      // bytes of a row of GALV_MX8 scales

// Whether a wait of a product has run out on the device since the context last looked.
inline bool mx_ran_out(galv_ctx* ctx)
{
    const unsigned seen = ctx->mx_timeouts_seen;
    ctx->mx_timeouts_seen = *(volatile unsigned*)ctx->mx_timeouts;
    return ctx->mx_timeouts_seen != seen;
}
// Whether a product may be launched.
inline int mx_may_run(galv_ctx* ctx, const char* refused, const char* ran_out)
{
    if (!ctx->mx_timeouts_at) return galv_set_error(ctx, GALV_ERR_CUDA, refused);
    return mx_ran_out(ctx) ? galv_set_error(ctx, GALV_ERR_TIMEOUT, ran_out) : GALV_OK;
}

template <int T> struct MxType;
template <> struct MxType<GALV_F32> { using type = float; };
template <> struct MxType<GALV_BF16> { using type = __nv_bfloat16; };
template <> struct MxType<GALV_F16> { using type = __half; };

__device__ __forceinline__ float mx_float(float v) { return v; }
__device__ __forceinline__ float mx_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float mx_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T mx_round(float v);
template <> __device__ __forceinline__ float mx_round<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 mx_round<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half mx_round<__half>(float v) { return __float2half_rn(v); }
template <typename T> __device__ __forceinline__ T mx_zero() { return mx_round<T>(0.f); }
// what was held as a finite number stays one in fp16 (a NaN passes both comparisons)
template <typename T> __device__ __forceinline__ float mx_held(float v) { return v; }
template <> __device__ __forceinline__ float mx_held<__half>(float v) { return v > 65504.f ? 65504.f : v < -65504.f ? -65504.f : v; }

// How a pass over a matrix's pieces of 8 columns is spread: a CTA of 256 threads has `each` pieces a thread, 256 * each of a row, or whole short rows (the
// width of a row is then a power of two of threads).  One division a CTA.  A thread's pieces are all loaded before the first is used: with two
// 16-byte loads under way a thread the pass reached 3.7 TB/s, with four 5 and more.
constexpr int kMxThreads = 256;
template <typename T> struct MxEach { static constexpr int count = sizeof(T) == 2 ? 4 : 2; };
struct MxSpread {
    int log;          // threads along a row: 1 << log
    int each;
    unsigned segs;    // CTAs along a row
    int dr, dc;       // from one of a thread's pieces to the next
    long long blocks; // CTAs in all
    MxSpread(long long rows, long long pieces, int each_) : log(0), each(each_)
    {
        while (log < 8 && (1ll << log) < pieces) ++log;
        const int rpc = kMxThreads >> log;
        const bool along = log == 8;
        segs = along ? (unsigned)((pieces + each * kMxThreads - 1) / (each * kMxThreads)) : 1;
        dr = along ? 0 : rpc;
        dc = along ? kMxThreads : 0;
        blocks = (along ? rows : (rows + each * rpc - 1) / (each * rpc)) * (long long)segs;
    }
    int grid() const { return (int)(blocks < (1ll << 30) ? blocks : (1ll << 30)); }
};
struct MxPlace { unsigned row, c; };                      // either may pass the matrix by what a CTA has: up to 2^31 + 1024 rows, 8 * (2^28 + 1024) columns
__device__ __forceinline__ MxPlace mx_place(const MxSpread& s, long long block)
{
    const unsigned rows = (unsigned)(block / s.segs), seg = (unsigned)(block - (long long)rows * s.segs);
    MxPlace p;
    p.row = (s.dr ? rows * s.each * s.dr : rows) + (threadIdx.x >> s.log);
    p.c = seg * s.each * kMxThreads + (threadIdx.x & ((1 << s.log) - 1));
    return p;
}

// 8 elements of a row as one piece: 16 bytes of 16-bit numbers, 32 of fp32.
template <typename T> struct MxPiece { uint4 q[sizeof(T) / 2]; };

// 16 bytes from `at` bytes (a multiple of 2) behind the start of the 32 in a and b.
__device__ __forceinline__ uint4 mx_shifted(const uint4& a, const uint4& b, uint32_t at)
{
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (at & 8) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (at & 4) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    const uint32_t bits = (at & 2) * 8;
    return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}

// As they lie in memory, zeros behind `cols`.  VEC: the row starts on a 16-byte boundary (c0 is a multiple of 8).  Else a piece inside its row is taken from the
// aligned 16 bytes around it, which lie in the row too; the first and the last pieces go element by element, and so do short rows (`pieces` false), where a
// warp would take both ways.
template <typename T, bool VEC>
__device__ __forceinline__ MxPiece<T> mx_fetch8(const T* row, int c0, int cols, bool pieces = true)
{
    MxPiece<T> p;
    if (VEC && c0 + 8 <= cols) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) p.q[i] = reinterpret_cast<const uint4*>(row + c0)[i];
    } else if (!VEC && pieces && c0 >= 8 && c0 + 16 <= cols) {
        const uintptr_t from = reinterpret_cast<uintptr_t>(row + c0);
        const uint32_t at = from & 15;
        const uint4* g = reinterpret_cast<const uint4*>(from - at);
        uint4 w[sizeof(T) / 2 + 1];
#pragma unroll
        for (int i = 0; i <= (int)sizeof(T) / 2; ++i) w[i] = g[i];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) p.q[i] = mx_shifted(w[i], w[i + 1], at);
    } else {
        T* e = reinterpret_cast<T*>(&p);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = c0 + i < cols ? row[c0 + i] : mx_zero<T>();
    }
    return p;
}
template <typename T> __device__ __forceinline__ void mx_floats(const MxPiece<T>& p, float (&v)[8])
{
    const T* e = reinterpret_cast<const T*>(&p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = mx_float(e[i]);
}

template <typename T> __device__ __forceinline__ MxPiece<T> mx_piece(const float (&v)[8])
{
    MxPiece<T> p;
    T* e = reinterpret_cast<T*>(&p);
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = mx_round<T>(v[i]);
    return p;
}
template <> __device__ __forceinline__ MxPiece<__nv_bfloat16> mx_piece<__nv_bfloat16>(const float (&v)[8])      // two numbers an instruction
{
    MxPiece<__nv_bfloat16> p;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p.q[0].x) : "f"(v[1]), "f"(v[0]));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p.q[0].y) : "f"(v[3]), "f"(v[2]));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p.q[0].z) : "f"(v[5]), "f"(v[4]));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p.q[0].w) : "f"(v[7]), "f"(v[6]));
    return p;
}
template <> __device__ __forceinline__ MxPiece<__half> mx_piece<__half>(const float (&v)[8])
{
    MxPiece<__half> p;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(p.q[0].x) : "f"(v[1]), "f"(v[0]));
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(p.q[0].y) : "f"(v[3]), "f"(v[2]));
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(p.q[0].z) : "f"(v[5]), "f"(v[4]));
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(p.q[0].w) : "f"(v[7]), "f"(v[6]));
    return p;
}

// What was held as a finite number stays one in fp16.
template <typename T> __device__ __forceinline__ MxPiece<T> mx_piece_held(const float (&v)[8]) { return mx_piece<T>(v); }
template <> __device__ __forceinline__ MxPiece<__half> mx_piece_held<__half>(const float (&v)[8])
{
    MxPiece<__half> p;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(p.q[0].x) : "f"(v[1]), "f"(v[0]));
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(p.q[0].y) : "f"(v[3]), "f"(v[2]));
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(p.q[0].z) : "f"(v[5]), "f"(v[4]));
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(p.q[0].w) : "f"(v[7]), "f"(v[6]));
    return p;
}

template <typename T, bool VEC>
__device__ __forceinline__ void mx_store8(T* __restrict__ row, int c0, int cols, const MxPiece<T>& p)
{
    if (VEC && c0 + 8 <= cols) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(row + c0)[i] = p.q[i];
    } else {
        const T* e = reinterpret_cast<const T*>(&p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c0 + i < cols) row[c0 + i] = e[i];
    }
}

// Rows that do not start on 16-byte boundaries: a warp whose 32 pieces lie next to one another in a row writes them through shared memory, so that
// aligned 16 bytes leave at a time (single elements of lanes in turn took five times as long).  start: lane 0's first element; n of them exist from there.
// buf has room for 256 elements, and 16 bytes behind them can be read.
template <typename T>
__device__ __forceinline__ void mx_scatter_run(T* buf, T* start, int n, const MxPiece<T>& p)
{
    constexpr int G = 16 / (int)sizeof(T);                // elements of 16 bytes
    const int lane = threadIdx.x % 32;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(buf + lane * 8)[i] = p.q[i];
    __syncwarp();
    n = min(n, 256);
    const int ahead = (int)(reinterpret_cast<uintptr_t>(start) & 15) / (int)sizeof(T), lead = (G - ahead) % G;      // elements from the boundary before to the start, and to the one behind
    const uint32_t at = lead * (int)sizeof(T);            // of each 16 bytes, in shared memory
#pragma unroll
    for (int k = 0; k < 256 / G; k += 32) {
        const int first = lead + (k + lane) * G;
        if (first + G <= n) {
            const uint4* from = reinterpret_cast<const uint4*>(buf) + (k + lane);
            *reinterpret_cast<uint4*>(start + first) = mx_shifted(from[0], from[1], at);
        } else if (first + G <= 256) {                    // the row's end
#pragma unroll 1
            for (int i = first; i < n; ++i) start[i] = buf[i];
        }
    }
    const int edge = lane < lead ? lane : 256 - G + lane; // before the first boundary, behind the last
    if (ahead && lane < G && edge < n) start[edge] = buf[edge];
}
// ... of pieces in several rows: 32 elements next to one another at a time.  place(l, n): lane l's first element, n of which exist.
template <typename T, typename Place>
__device__ __forceinline__ void mx_scatter8(T* buf, const Place& place, const MxPiece<T>& p)
{
    const int lane = threadIdx.x % 32, e = lane % 8;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(buf + lane * 8)[i] = p.q[i];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int l = i * 4 + lane / 8;
        int n;
        T* to = place(l, n);
        if (e < n) to[e] = buf[l * 8 + e];
    }
}
// The pieces of a spread pass, h-th of a thread: where lane l of this warp has its own.
template <typename T>
struct MxPlaces {
    T* x;
    long long stride;
    unsigned row0, c0, log, rows, cols;
    __device__ __forceinline__ MxPlaces(T* x_, long long stride_, const MxSpread& s, const MxPlace& at, int h, unsigned rows_, unsigned cols_)
        : x(x_), stride(stride_), row0(at.row - (threadIdx.x >> s.log) + h * s.dr), c0(at.c - (threadIdx.x & ((1 << s.log) - 1)) + h * s.dc), log(s.log), rows(rows_), cols(cols_) {}
    __device__ __forceinline__ T* operator()(int l, int& n) const
    {
        const unsigned t = (threadIdx.x & ~31) + l, row = row0 + (t >> log), c = (c0 + (t & ((1 << log) - 1))) * 8;
        n = row < rows && c < cols ? (int)min(8u, cols - c) : 0;
        return x + ((long long)row * stride + c);
    }
};
// A spread pass's piece c of a row (`row`: its start; exists: whether it is one) to rows that do not start on 16-byte boundaries.
template <typename T>
__device__ __forceinline__ void mx_store_spread(T* buf, T* row, unsigned c, bool exists, T* x, long long stride, const MxSpread& s, const MxPlace& at, int h, unsigned rows, unsigned cols,
                                                const MxPiece<T>& p)
{
    if (s.log >= 5) {                                     // the warp's pieces lie in one row
        const unsigned c0 = (c - threadIdx.x % 32) * 8;
        mx_scatter_run<T>(buf, row + c0, exists && c0 < cols ? (int)min(256u, cols - c0) : 0, p);
    } else {
        mx_scatter8<T>(buf, MxPlaces<T>(x, stride, s, at, h, rows, cols), p);
    }
}

// Scale byte of a block whose largest magnitude has these bits: the smallest exponent under which it does not pass the largest element,
// 448 = 1.75 * 2^8 or 6 = 1.5 * 2^2.  Whole numbers only, so exact; 255 for an infinity or a NaN.
template <int FMT>
__device__ __forceinline__ int mx_scale_byte(uint32_t amax_bits)
{
    constexpr int top = FMT == GALV_MX8 ? 8 : 2;
    constexpr uint32_t mant = FMT == GALV_MX8 ? 0x600000u : 0x400000u;
    if (amax_bits >= 0x7f800000u) return 255;
    const int b = (int)(amax_bits >> 23) - top + ((amax_bits & 0x7fffffu) > mant ? 1 : 0);
    return b < 0 ? 0 : b;
}
// 2^(127 - byte); bytes up to 253 occur
__device__ __forceinline__ float mx_inverse(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }
// 2^(byte - 127), NaN for 255
__device__ __forceinline__ float mx_scale(int byte) { return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fc00000u : (uint32_t)byte << 23); }

// Bits (fp32) of the largest magnitude among 8 numbers.  Magnitudes order like their bits, infinities and NaN above all numbers.
__device__ __forceinline__ uint32_t mx_pairs_most(const uint4& q)
{
    const uint32_t k = 0x7fff7fffu, m = __vimax3_u16x2(__vmaxu2(q.x & k, q.y & k), q.z & k, q.w & k);
    return max(m & 0xffffu, m >> 16);
}
template <typename T> __device__ __forceinline__ uint32_t mx_most(const MxPiece<T>& p);
template <> __device__ __forceinline__ uint32_t mx_most<__nv_bfloat16>(const MxPiece<__nv_bfloat16>& p) { return mx_pairs_most(p.q[0]) << 16; }
template <> __device__ __forceinline__ uint32_t mx_most<__half>(const MxPiece<__half>& p) { return __float_as_uint(__half2float(__ushort_as_half((unsigned short)mx_pairs_most(p.q[0])))); }
template <> __device__ __forceinline__ uint32_t mx_most<float>(const MxPiece<float>& p)
{
    const uint32_t k = 0x7fffffffu;
    return max(max(max(p.q[0].x & k, p.q[0].y & k), max(p.q[0].z & k, p.q[0].w & k)), max(max(p.q[1].x & k, p.q[1].y & k), max(p.q[1].z & k, p.q[1].w & k)));
}

// Four numbers to four 8-bit elements, to nearest even (the conversion saturates; nothing here passes 448).
__device__ __forceinline__ uint32_t mx_to8(float a, float b, float c, float d)
{
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | (uint32_t)hi << 16;
}
// Eight numbers to eight 4-bit elements, element 0 lowest.
__device__ __forceinline__ uint32_t mx_to4(const float (&v)[8])
{
    uint32_t r;
    asm("{\n.reg .b8 a, b, c, d;\n"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
        "mov.b32 %0, {a, b, c, d};\n}" : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
__device__ __forceinline__ void mx_from8(uint32_t w, float* v)
{
    uint32_t lo, hi;
    asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %2;\ncvt.rn.f16x2.e4m3x2 %0, l;\ncvt.rn.f16x2.e4m3x2 %1, h;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}
__device__ __forceinline__ void mx_from4(uint32_t w, float (&v)[8])
{
    uint32_t h[4];
    asm("{\n.reg .b8 a, b, c, d;\nmov.b32 {a, b, c, d}, %4;\n"
        "cvt.rn.f16x2.e2m1x2 %0, a;\ncvt.rn.f16x2.e2m1x2 %1, b;\ncvt.rn.f16x2.e2m1x2 %2, c;\ncvt.rn.f16x2.e2m1x2 %3, d;\n}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
}

// Where the scale byte of (row, block) lies.
template <int FMT>
__device__ __forceinline__ long long mx_scale_at(unsigned row, unsigned b, int per_row)      // per_row: bytes a row (MX8), tiles a row of tiles (MX4)
{
    if (FMT == GALV_MX8) return (long long)row * per_row + b;
    return ((long long)(row >> 7) * per_row + (b >> 2)) * 512 + ((row & 31) * 16 + ((row >> 5) & 3) * 4 + (b & 3));
}

// The 8 values held in GALV_MX8 of piece c (columns 8c .. 8c+7) of a row.
__device__ __forceinline__ void mx_restore8(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, long long row, int c, long long nb, long long per_row, float (&v)[8])
{
    const uint2 w = __ldg(reinterpret_cast<const uint2*>(codes + (row * nb * 32 + c * 8ll)));
    mx_from8(w.x, v);
    mx_from8(w.y, v + 4);
    const float s = mx_scale(__ldg(scales + row * per_row + (c >> 2)));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= s;
}

#define MX_DISPATCH_TYPE(dtype, ...)                                                                                  \
    do {                                                                                                              \
        if ((dtype) == GALV_F32) { using T = float; __VA_ARGS__; }                                                    \
        else if ((dtype) == GALV_BF16) { using T = __nv_bfloat16; __VA_ARGS__; }                                      \
        else { using T = __half; __VA_ARGS__; }                                                                       \
    } while (0)

// Tensor map of a matrix [rows][cols] whose rows are `pitch` bytes apart, read in boxes [box_rows][box_cols]; swizzle: rows of 128 bytes, their
// 16-byte pieces exchanged by row % 8.
cudaError_t galv_mx_map(CUtensorMap* map, CUtensorMapDataType type, const void* base, uint64_t rows, uint64_t cols, uint64_t pitch, uint32_t box_rows,
                        uint32_t box_cols, bool swizzle);
