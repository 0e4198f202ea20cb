// Rows sorted by expert: which tiles there are, found on the device from where each expert's rows end.
#pragma once

#include "galv_mx.cuh"

constexpr int kExpertsMost = 1024;

// In shared memory, by one warp: begin[e] is expert e's first row, begin[experts] the end of all.  Ends count as they would if each were clamped between the
// one before it and the rows there are.  ends NULL: one expert has all rows.
__device__ __forceinline__ void experts_begin(const int32_t* __restrict__ ends, int experts, long long rows, int* begin)
{
    const int lane = threadIdx.x % 32;
    int last = 0;
    for (int b = 0; b < experts; b += 32) {
        const int e = b + lane;
        int end = e >= experts ? 0 : ends ? (int)min(max((long long)__ldg(ends + e), 0ll), rows) : (int)rows;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int other = __shfl_up_sync(0xffffffffu, end, o);
            if (lane >= o) end = max(end, other);
        }
        end = max(end, last);
        int first = __shfl_up_sync(0xffffffffu, end, 1);
        if (lane == 0) first = last;
        if (e < experts) begin[e] = first;
        last = __shfl_sync(0xffffffffu, end, 31);
    }
    if (lane == 0) begin[experts] = last;
}

// Rows of an expert's tiles where none has more than `most` (a multiple of 32): as many as it needs, of one size, a multiple of 32 again.
__device__ __forceinline__ int experts_tiles(int rows, int most) { return (int)(((unsigned)rows + most - 1) / most); }
__device__ __forceinline__ int experts_tile(int rows, int tiles) { return tiles ? (int)((((unsigned)rows + tiles - 1) / tiles + 31) & ~31u) : 0; }

// What the tiles of at most `most` rows would take, by one warp: the rounds of `pairs` of CTAs that they make, each by `across` tiles of weights' rows, times their mean cost.
// A tile of r rows takes fixed + r for each chunk of the summed index.
__device__ __forceinline__ float experts_price(const int* begin, int experts, int most, int across, int pairs, float fixed)
{
    float tiles = 0.f, cost = 0.f;
    for (int e = threadIdx.x % 32; e < experts; e += 32) {
        const int rows = begin[e + 1] - begin[e], mine = experts_tiles(rows, most);
        tiles += mine;
        cost += mine * (fixed + experts_tile(rows, mine));
    }
#pragma unroll
    for (int o = 16; o; o /= 2) {
        tiles += __shfl_xor_sync(0xffffffffu, tiles, o);
        cost += __shfl_xor_sync(0xffffffffu, cost, o);
    }
    return tiles > 0.f ? ceilf(tiles * across / pairs) * (cost / tiles) : 0.f;
}

// before[e]: how many tiles the experts before e have, before[experts] all, by one warp.
__device__ __forceinline__ void experts_before(const int* begin, int experts, int most, int* before)
{
    const int lane = threadIdx.x % 32;
    int tiles = 0;
    for (int b = 0; b < experts; b += 32) {
        const int e = b + lane, mine = e < experts ? experts_tiles(begin[e + 1] - begin[e], most) : 0;
        int sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int other = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += other;
        }
        if (e < experts) before[e] = tiles + sum - mine;
        tiles += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) before[experts] = tiles;
}

// The nth (from 0) of the tiles of `most` rows that the experts have, to shared memory by one warp: whose it is, its first row and how many; -1, 0, 0 where there are fewer.
// And where the rows that belong to none begin.
__device__ __forceinline__ void experts_nth(const int32_t* __restrict__ ends, int experts, long long rows, int most, int nth, int* found)
{
    const int lane = threadIdx.x % 32;
    if (lane < 3) found[lane] = lane == 0 ? -1 : 0;
    __syncwarp();
    int last = 0, before = 0;
    for (int b = 0; b < experts; b += 32) {
        const int e = b + lane;
        int end = e >= experts ? 0 : ends ? (int)min(max((long long)__ldg(ends + e), 0ll), rows) : (int)rows;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int other = __shfl_up_sync(0xffffffffu, end, o);
            if (lane >= o) end = max(end, other);
        }
        end = max(end, last);
        int first = __shfl_up_sync(0xffffffffu, end, 1);
        if (lane == 0) first = last;
        const int mine = experts_tiles(end - first, most);
        int sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int other = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += other;
        }
        const int tile = nth - (before + sum - mine);
        if (tile >= 0 && tile < mine) {
            found[0] = e;
            found[1] = first + tile * most;
            found[2] = min(most, end - found[1]);
        }
        before += __shfl_sync(0xffffffffu, sum, 31);
        last = __shfl_sync(0xffffffffu, end, 31);
    }
    if (lane == 0) found[3] = last;
}

// Matrices whose rows bulk copies cannot take (not on 16-byte boundaries) into rows that they can, zeros behind their ends (galv_mx_wgrad.cu).
// They are placed on whole lines, short ones on whole sectors: bulk copies of rows that start in the middle of a sector took up to a third longer (8192 rows x 4096 x 1000, input gradient: 87 us,
// 70 in whole sectors, 62 in whole lines).
inline int64_t galv_aligned_pitch(int64_t cols) { return cols >= 512 ? (cols + 63) / 64 * 64 : (cols + 15) / 16 * 16; }
void galv_align_rows(const galv_ctx* ctx, int64_t rows, int64_t cols, const void* x, int64_t stride, void* out, int64_t pitch, cudaStream_t st);
