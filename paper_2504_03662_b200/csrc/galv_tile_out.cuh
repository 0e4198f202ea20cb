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
// the thread's first place; `rows` and `cols` of them exist.  Without `sums` they count as zeros and tensor memory is not read.  All loads of a round come before its first store: out may be base.
template <typename O>
__device__ __forceinline__ void move_out(uint32_t tmem, uint32_t mine, const O* base, O* out, long long k, int rows, int cols, bool vec, bool sums = true)
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
        if (sums) {
            tc::tmem_load16(tmem + j, s);
            tc::tmem_wait_load();
        } else {
#pragma unroll
            for (int q = 0; q < 16; ++q) s[q] = 0;
        }
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

// The same for rows that do not start on 16-byte boundaries; base and out point to the warp's first place and `mine` has 4096 bytes.  In shared memory a row is a ring of 128 bytes of
// results and a round adds 64; four lanes write the 64 that end at such a boundary in memory, in pieces of 16 bytes, each cut from two of the ring by the bits of where it begins.  Bound by
// instructions and by lines a store: a column a lane, two rows a store, took 54 us for 7 gradients of 2731 x 1365 in fp16 where this takes 41, and 3513 for 64 of 2048 x 4090 onto fp32
// where this takes 1490 (1040 and 690 without base; where all of it stays in L2, 33 to 67 MB, up to 7 us more).  base only beside fp32: 16-bit results are rounded on their way in.
template <typename O>
__device__ __forceinline__ void move_out_odd(uint32_t tmem, uint32_t mine, const O* base, O* out, long long k, int rows, int cols, bool sums)
{
    constexpr int size = sizeof(O), each = 64 / size;     // columns a round
    const int lane = threadIdx.x % 32, bytes = cols * size;
    int first[4];                                         // rows lane / 4 + 8 i: where the lane's piece in round 0 begins, in bytes from the row's first, from -62 on
    uint32_t from[4][2], cut[4];
    unsigned char* to[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = lane / 4 + 8 * i;
        to[i] = reinterpret_cast<unsigned char*>(out + row * k);
        first[i] = lane % 4 * 16 - (int)(reinterpret_cast<uintptr_t>(to[i]) & 63);
        to[i] += first[i];
#pragma unroll
        for (int e = 0; e < 2; ++e) from[i][e] = mine + row * 128 + (((first[i] >> 4) + e + row) & 7) * 16;
        cut[i] = first[i] & 15;
        if (row >= rows) first[i] = 1 << 20;              // no piece of it is inside
    }
    const bool alike = base && ((reinterpret_cast<uintptr_t>(base) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    const long long apart = reinterpret_cast<const unsigned char*>(base) - reinterpret_cast<const unsigned char*>(out);
    // In 16 bits a row's ends, before its first whole piece and behind its last, an element a lane: eight stores a side (a row a lane took as long as it gained).
    auto ends = [&](bool last) {
#pragma unroll
        for (int r = 0; r < 32; r += 4) {
            const int row = r + lane / 8, x = last ? bytes - 16 + lane % 8 * 2 : lane % 8 * 2;
            unsigned char* const p = reinterpret_cast<unsigned char*>(out + row * k);
            const int before = (int)(-reinterpret_cast<uintptr_t>(p) & 15), behind = (int)(reinterpret_cast<uintptr_t>(p + bytes) & 15);
            if (row < rows && (last ? before <= bytes && x >= bytes - behind : x < before && x < bytes)) {
                unsigned short v;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(mine + row * 128 + (((x >> 4) + row) & 7) * 16 + (x & 15)));
                *reinterpret_cast<unsigned short*>(p + x) = v;
            }
        }
    };
#pragma unroll 1
    for (int j = 0; j <= 128 * size && j < bytes + 63; j += 64) {
        const uint32_t turn = j & 64;
        if (j < 128 * size) {
            uint32_t w[16];
            if (!sums) {
#pragma unroll
                for (int q = 0; q < 16; ++q) w[q] = 0;
            } else if constexpr (size == 2) {
                uint32_t s[each];
                tc::tmem_load32(tmem + j / size, s);
                tc::tmem_wait_load();
#pragma unroll
                for (int q = 0; q < 16; ++q) w[q] = join<O>(__uint_as_float(s[2 * q]), __uint_as_float(s[2 * q + 1]));
            } else {
                tc::tmem_load16(tmem + j / size, w);
                tc::tmem_wait_load();
            }
            __syncwarp();
#pragma unroll
            for (int q = 0; q < 4; ++q)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(mine + lane * 128 + (((q + lane) & 7) * 16 ^ turn)), "r"(w[4 * q]), "r"(w[4 * q + 1]), "r"(w[4 * q + 2]), "r"(w[4 * q + 3]) : "memory");
        }
        __syncwarp();
        if (size == 2 && j == 0) ends(false);
        if (size == 2 && j < bytes && j + 64 >= bytes) ends(true);
        uint32_t o[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 2; ++e)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4 * e]), "=r"(w[4 * e + 1]), "=r"(w[4 * e + 2]), "=r"(w[4 * e + 3]) : "r"(from[i][e] ^ turn));
#pragma unroll
            for (int q = 0; q < 6; ++q) w[q] = cut[i] & 8 ? w[q + 2] : w[q];
#pragma unroll
            for (int q = 0; q < 5; ++q) w[q] = cut[i] & 4 ? w[q + 1] : w[q];
#pragma unroll
            for (int q = 0; q < 4; ++q) o[i][q] = size == 2 ? __funnelshift_r(w[q], w[q + 1], (cut[i] & 2) * 8) : w[q];
        }
        if (size == 4 && base) {                          // all loads of a round before its first store: out may be base
            uint32_t b[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = first[i] + j;
                const unsigned char* const p = to[i] + j + apart;
                if (alike && t >= 0 && t + 16 <= bytes) {
                    const uint4 all = *reinterpret_cast<const uint4*>(p);
                    b[i][0] = all.x; b[i][1] = all.y; b[i][2] = all.z; b[i][3] = all.w;
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q) b[i][q] = t + q * 4 >= 0 && t + q * 4 < bytes ? reinterpret_cast<const uint32_t*>(p)[q] : 0u;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) o[i][q] = __float_as_uint(__uint_as_float(o[i][q]) + __uint_as_float(b[i][q]));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = first[i] + j;
            unsigned char* const p = to[i] + j;
            if (t >= 0 && t + 16 <= bytes) {
                *reinterpret_cast<uint4*>(p) = make_uint4(o[i][0], o[i][1], o[i][2], o[i][3]);
            } else if (size == 4 && t > -16 && t < bytes) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (t + q * 4 >= 0 && t + q * 4 < bytes) reinterpret_cast<uint32_t*>(p)[q] = o[i][q];
            }
        }
    }
}

}  // namespace tile_out
