// Tiles of fp32 sums from tensor memory to a matrix in memory, for the kernels whose tiles lie as the matrix does.
#pragma once

#include "galv_mx.cuh"
#include "galv_tc.cuh"

namespace tile_out {

template <typename O> struct Four;
template <> struct Four<float> { using type = float4; };
template <> struct Four<__nv_bfloat16> { using type = uint2; };
template <> struct Four<__half> { using type = uint2; };
template <typename O> __device__ __forceinline__ float2 two(uint32_t w);
template <> __device__ __forceinline__ float2 two<__nv_bfloat16>(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
template <> __device__ __forceinline__ float2 two<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
template <typename O> __device__ __forceinline__ uint32_t join(float a, float b);
template <> __device__ __forceinline__ uint32_t join<__nv_bfloat16>(float a, float b) { const __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
template <> __device__ __forceinline__ uint32_t join<__half>(float a, float b) { const __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
template <typename Q, typename O> struct AddFour {
    static __device__ __forceinline__ void to(float (&v)[4], const Q& q)
    {
        const float2 a = two<O>(q.x), b = two<O>(q.y);
        v[0] += a.x; v[1] += a.y; v[2] += b.x; v[3] += b.y;
    }
};
template <typename O> struct AddFour<float4, O> { static __device__ __forceinline__ void to(float (&v)[4], const float4& q) { v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w; } };
template <typename Q, typename O> struct RoundFour { static __device__ __forceinline__ Q of(const float (&v)[4]) { return make_uint2(join<O>(v[0], v[1]), join<O>(v[2], v[3])); } };
template <typename O> struct RoundFour<float4, O> { static __device__ __forceinline__ float4 of(const float (&v)[4]) { return make_float4(v[0], v[1], v[2], v[3]); } };

// A warp's 32 x 128 sums in tensor memory, a row a lane, to a matrix with rows k apart: 16 columns at a time go through the warp's shared memory
// (rows of 64 bytes, their 16-byte pieces exchanged by row / 2 % 4), so that lanes next to one another write next to one another.  base and out point to
// the thread's first place; `rows` and `cols` of them exist.  All loads of a round come before its first store: out may be base.
template <typename O>
__device__ __forceinline__ void move_out(uint32_t tmem, uint32_t mine, const O* base, O* out, long long k, int rows, int cols, bool vec)
{
    const int lane = threadIdx.x % 32;
    using Q = typename Four<O>::type;
    // vec: a lane has 4 columns of rows lane / 4 + 8 i, k is a multiple of 4; else one column of rows lane / 16 + 2 i
    const uint32_t from = vec ? mine + lane / 4 * 64 + ((lane % 4) ^ (lane >> 3 & 3)) * 16 : mine + lane / 16 * 64 + lane % 4 * 4, piece = lane % 16 / 4;
    rows -= vec ? lane / 4 : lane / 16;
    cols -= vec ? lane % 4 * 4 : lane % 16;
#pragma unroll 1
    for (int j = 0; j < 128; j += 16) {
        uint32_t s[16];
        tc::tmem_load16(tmem + j, s);
        tc::tmem_wait_load();
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 4; ++q)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(mine + lane * 64 + (q ^ (lane >> 1 & 3)) * 16), "r"(s[4 * q]), "r"(s[4 * q + 1]), "r"(s[4 * q + 2]), "r"(s[4 * q + 3]) : "memory");
        __syncwarp();
        const bool in = j < cols;
        if (vec) {
            float v[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[i][0]), "=f"(v[i][1]), "=f"(v[i][2]), "=f"(v[i][3]) : "r"(from + i * 512));
            if (base) {
                Q q[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (in && i * 8 < rows) q[i] = *reinterpret_cast<const Q*>(base + i * 8 * k + j);
#pragma unroll
                for (int i = 0; i < 4; ++i) AddFour<Q, O>::to(v[i], q[i]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (in && i * 8 < rows) *reinterpret_cast<Q*>(out + i * 8 * k + j) = RoundFour<Q, O>::of(v[i]);
        } else {
#pragma unroll
            for (int h = 0; h < 32; h += 16) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v[i]) : "r"(from + (h + 2 * i) * 64 + (piece ^ (i & 3)) * 16));
                if (base) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (in && h + 2 * i < rows) v[i] += mx_float(base[(h + 2 * i) * k + j]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (in && h + 2 * i < rows) out[(h + 2 * i) * k + j] = mx_round<O>(v[i]);
            }
        }
    }
}

}  // namespace tile_out
