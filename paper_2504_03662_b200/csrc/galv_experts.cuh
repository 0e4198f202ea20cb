// Rows sorted by expert: which tiles there are, found on the device from where each expert's rows end.
#pragma once

#include "galv_mx.cuh"

constexpr int kExpertsMost = 1024, kTileRows = 256;

// In shared memory, by one warp: begin[e] is expert e's first row and before[e] how many tiles of kTileRows rows the experts before e have; [experts]: the
// end and the count of all.  Ends count as they would if each were clamped between the one before it and the rows there are.  ends NULL: one expert has all rows.
__device__ __forceinline__ void experts_scan(const int32_t* __restrict__ ends, int experts, long long rows, int* begin, int* before)
{
    const int lane = threadIdx.x % 32;
    int last = 0, tiles = 0;
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
        const int mine = (int)(((unsigned)(end - first) + kTileRows - 1) / kTileRows);
        int sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int other = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += other;
        }
        if (e < experts) {
            begin[e] = first;
            before[e] = tiles + sum - mine;
        }
        last = __shfl_sync(0xffffffffu, end, 31);
        tiles += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) {
        begin[experts] = last;
        before[experts] = tiles;
    }
}

// The nth (from 0) of the experts that have rows, to shared memory by one warp: which it is, its first row and how many; -1, 0, 0 where there are fewer.  And
// where the rows that belong to none begin.
__device__ __forceinline__ void experts_nth(const int32_t* __restrict__ ends, int experts, long long rows, int nth, int* found)
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
        const unsigned some = __ballot_sync(0xffffffffu, end > first);
        if (end > first && before + __popc(some & ((1u << lane) - 1)) == nth) {
            found[0] = e;
            found[1] = first;
            found[2] = end - first;
        }
        before += __popc(some);
        last = __shfl_sync(0xffffffffu, end, 31);
    }
    if (lane == 0) found[3] = last;
}

// Matrices whose rows bulk copies cannot take (not on 16-byte boundaries) into rows that they can, zeros behind their ends (galv_mx_wgrad.cu).
void galv_align_rows(const galv_ctx* ctx, int64_t rows, int64_t cols, const void* x, int64_t stride, void* out, int64_t pitch, cudaStream_t st);
