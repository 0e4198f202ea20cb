// Product of two matrices held in 4 bits: y[i][j] = sum_k a[i][k] b[j][k] + bias[j].
//
// The tensor cores take the elements as they are held and the blocks' powers of two beside them (tcgen05.mma kind::mxf4 with block scales), so
// nothing is restored.  A pair of CTAs owns a tile of 256 x 256 of y: each stages 128 rows of a and of b, 256 columns (128 bytes a row) at a time, its own
// rows' scales of a and all 256 rows' scales of b; the scales lie in memory in the order in which they go to tensor memory (galv.h).
// Tensor memory: two accumulators of 256 columns that share 48 of them, and 24 columns of scales.  The warps that move a tile out begin with
// the shared columns, after which the next tile's sums may start.
//
// 4096 x 32768 x 8192 into bf16 take 375 us (5.9 PFLOP/s; without copies 323, also without the copies of scales to tensor memory 308, without stores 365).  Five stages: four
// take 385, six 391.

#include <mutex>

#include "galv_mx.cuh"
#include "galv_tc.cuh"

namespace {

constexpr int kStages = 5, kTile = 256, kHalf = kTile / 2, kChunkBytes = 128, kChunkBlocks = 8;      // 256 columns a chunk
constexpr int kRowsBytes = kHalf * kChunkBytes, kScaleA = 1024, kScaleB = 2048;
constexpr int kStageBytes = 2 * kRowsBytes + kScaleA + kScaleB;
constexpr int kOutBytes = 8 * 2048;
constexpr int kSmem = 1024 + kStages * kStageBytes + kOutBytes + 256;
constexpr int kThreads = 384;
constexpr int kSecond = 208, kScalesAt = kSecond + kTile;                                            // columns of tensor memory
constexpr int kGroup = 16;                                // tiles along m whose rows of a stay in L2 while their n runs (8: 388 us)

struct MatmulArgs {
    long long m, n, stride;
    int blocks, groups;                                   // of 32 columns; of 4 blocks
    int tiles_m, tiles_n, splits, chunks;
    const uint8_t* a_scales;
    const uint8_t* b_scales;
    const void* bias;
    void* y;
    float* partial;                                       // [splits][m][n], or NULL
    int vec;                                              // four results of a row can be moved at once
    unsigned* timeouts;                                   // host memory: CTAs that have given up a wait
};

struct Unit { int tm, tn, split, c0, c1; };
__device__ __forceinline__ Unit unit_of(const MatmulArgs& a, int u)
{
    Unit w;
    const int tile = u / a.splits, per = kGroup * a.tiles_n, first = tile / per * kGroup;
    const int size = min(kGroup, a.tiles_m - first);
    w.split = u % a.splits;
    w.tm = first + tile % per % size;
    w.tn = tile % per / size;
    w.c0 = (int)((long long)w.split * a.chunks / a.splits);
    w.c1 = (int)((long long)(w.split + 1) * a.chunks / a.splits);
    return w;
}

template <typename O> struct Four;
template <> struct Four<float> {
    using type = float4;
    static __device__ __forceinline__ float4 of(const float (&v)[4]) { return make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Four<__nv_bfloat16> {
    using type = uint2;
    static __device__ __forceinline__ uint32_t two(float a, float b) { const __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
    static __device__ __forceinline__ uint2 of(const float (&v)[4]) { return make_uint2(two(v[0], v[1]), two(v[2], v[3])); }
};
template <> struct Four<__half> {
    using type = uint2;
    static __device__ __forceinline__ uint32_t two(float a, float b) { const __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
    static __device__ __forceinline__ uint2 of(const float (&v)[4]) { return make_uint2(two(v[0], v[1]), two(v[2], v[3])); }
};

// 16 columns of a warp's 32 rows of sums to y, through the warp's shared memory (rows of 64 bytes, their 16-byte pieces exchanged by row / 2 % 4).
// bias and out point to the thread's first place of these columns; `rows` and `cols` of them exist from there.
template <typename O>
__device__ __forceinline__ void move_out(uint32_t tmem, uint32_t mine, const O* bias, O* out, long long stride, int rows, int cols, bool vec)
{
    const int lane = threadIdx.x % 32;
    uint32_t s[16];
    tc::tmem_load16(tmem, s);
    tc::tmem_wait_load();
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 4; ++q)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(mine + lane * 64 + (q ^ (lane >> 1 & 3)) * 16), "r"(s[4 * q]), "r"(s[4 * q + 1]), "r"(s[4 * q + 2]), "r"(s[4 * q + 3]) : "memory");
    __syncwarp();
    if (vec) {
        float v[4][4], b[4] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[i][0]), "=f"(v[i][1]), "=f"(v[i][2]), "=f"(v[i][3])
                         : "r"(mine + lane / 4 * 64 + ((lane % 4) ^ (lane >> 3 & 3)) * 16 + i * 512));
        if (bias && cols > 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = mx_float(bias[j]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] += b[j];
            if (cols > 0 && i * 8 < rows) *reinterpret_cast<typename Four<O>::type*>(out + i * 8 * stride) = Four<O>::of(v[i]);
        }
    } else {
        const float b = bias && cols > 0 ? mx_float(bias[0]) : 0.f;
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v[i]) : "r"(mine + lane / 16 * 64 + lane % 4 * 4 + (h + 2 * i) * 64 + ((lane % 16 / 4) ^ (i & 3)) * 16));
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (cols > 0 && h + 2 * i < rows) out[(h + 2 * i) * stride] = mx_round<O>(v[i] + b);
        }
    }
}

template <typename O>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
mx_matmul_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map, const __grid_constant__ MatmulArgs a)
{
    extern __shared__ unsigned char raw[];
    const uint32_t base = (tc::smem_at(raw) + 1023) & ~1023u;
    const uint32_t a_at = base, b_at = a_at + kStages * kRowsBytes, sa_at = b_at + kStages * kRowsBytes, sb_at = sa_at + kStages * kScaleA, out_at = sb_at + kStages * kScaleB,
                   bars = out_at + kOutBytes;
    const uint32_t full = bars, other = full + 8 * kStages, empty = other + 8 * kStages, acc_full = empty + 8 * kStages, acc_free = acc_full + 16, drain = acc_free + 8, slot = drain + 8;
    __shared__ int failed;

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = tc::cluster_rank();
    const int units = a.tiles_m * a.tiles_n * a.splits, first = blockIdx.x / 2, stride = gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc::bar_init(full + 8 * s, 1);
            tc::bar_init(other + 8 * s, 1);
            tc::bar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) tc::bar_init(acc_full + 8 * b, 1);
        tc::bar_init(acc_free, 16);
        tc::bar_init(drain, 1);
        tc::bar_init_done();
        failed = 0;
        tc::prefetch_map(&a_map);
        tc::prefetch_map(&b_map);
    }
    if (warp == 2) tc::tmem_alloc<2>(slot, 512);
    tc::fence_before();
    __syncthreads();
    tc::cluster_sync();                                   // the pair's barriers exist
    tc::fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(slot));

    auto waited = [&](uint32_t bar, uint32_t parity) {
        if (tc::bar_wait(bar, parity)) return true;
        *(volatile int*)&failed = 1;
        return false;
    };
    // All lanes of a warp go the same way, also where the limit ends between two lanes' tries: what follows takes whole warps.
    auto warp_waited = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, waited(bar, parity)) != 0; };

    if (warp == 0) {
        if (tc::elect()) {
            int it = 0;
            bool ok = true;
            for (int u = first; u < units && ok; u += stride) {
                const Unit w = unit_of(a, u);
                const int m0 = w.tm * kTile + rank * kHalf, n0 = w.tn * kTile + rank * kHalf;
                // tiles of scales: rows of this CTA of a, all rows of the pair of b; those behind the last row do not exist
                const bool a_in = m0 < a.m, b_in = w.tn * kTile + kHalf < a.n;
                const uint8_t* sa = a.a_scales + (long long)(m0 / 128) * a.groups * 512;
                const uint8_t* sb = a.b_scales + (long long)(w.tn * 2) * a.groups * 512;
                for (int c = w.c0; c < w.c1; ++c, ++it) {
                    const int s = it % kStages;
                    const uint32_t bar = full + 8 * s, bytes = min(2, a.groups - 2 * c) * 512;
                    if (!(ok = waited(empty + 8 * s, (it / kStages & 1) ^ 1))) break;
                    tc::bar_expect(bar, 2 * kRowsBytes + bytes * (1 + a_in + b_in));
                    tc::load_2d(a_at + s * kRowsBytes, &a_map, c * kChunkBytes, m0, bar);
                    tc::load_2d(b_at + s * kRowsBytes, &b_map, c * kChunkBytes, n0, bar);
                    if (a_in) tc::load_bytes(sa_at + s * kScaleA, sa + (long long)c * 1024, bytes, bar);
                    tc::load_bytes(sb_at + s * kScaleB, sb + (long long)c * 1024, bytes, bar);
                    if (b_in) tc::load_bytes(sb_at + s * kScaleB + 1024, sb + ((long long)a.groups * 512 + (long long)c * 1024), bytes, bar);
                }
            }
            if (*(volatile int*)&failed)                  // copies still in flight
                for (int i = it < kStages ? 0 : it - kStages; i < it; ++i) tc::bar_wait(full + 8 * (i % kStages), i / kStages & 1);
        }
    } else if (warp == 1 && rank == 1) {                  // tells the first CTA that this one's rows are there
        if (tc::elect()) {
            int it = 0;
            bool ok = true;
            for (int u = first; u < units && ok; u += stride) {
                const Unit w = unit_of(a, u);
                for (int c = w.c0; c < w.c1; ++c, ++it) {
                    if (!(ok = waited(full + 8 * (it % kStages), it / kStages & 1))) break;
                    tc::bar_arrive_cluster(tc::in_cta(other + 8 * (it % kStages), 0));
                }
            }
        }
    } else if (warp == 1) {
        if (tc::elect()) {
            // e2m1 by e2m1, scales that are powers of two, 256 x 256; bits 4 and 29: which pair of a scale column's four bytes
            constexpr uint32_t what = 1u << 7 | 1u << 10 | (uint32_t)(kTile >> 3) << 17 | 1u << 23 | (uint32_t)(kTile >> 4) << 24;
            const uint32_t sa = tmem + kScalesAt, sb = sa + 8;
            int it = 0, done = 0;
            bool ok = true;
            for (int u = first; u < units && ok; u += stride, ++done) {
                const Unit w = unit_of(a, u);
                const uint32_t d = tmem + (done & 1) * kSecond;
                if (done > 0 && !(ok = waited(acc_free, (done - 1) & 1))) break;
                tc::fence_after();
                for (int c = w.c0; c < w.c1; ++c, ++it) {
                    const int s = it % kStages;
                    if (!(ok = waited(full + 8 * s, it / kStages & 1) && waited(other + 8 * s, it / kStages & 1))) break;
                    tc::fence_after();
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        tc::copy_scales<2>(sa + g * 4, tc::operand_plain(sa_at + s * kScaleA + g * 512));
                        tc::copy_scales<2>(sb + g * 8, tc::operand_plain(sb_at + s * kScaleB + g * 512));
                        tc::copy_scales<2>(sb + g * 8 + 4, tc::operand_plain(sb_at + s * kScaleB + 1024 + g * 512));
                    }
                    const int steps = min(4, (a.blocks - c * kChunkBlocks + 1) / 2);      // of 64 columns
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < steps) {
                            const uint32_t pick = (j & 1) * 2;
                            tc::mma_mx4<2>(d, tc::operand(a_at + s * kRowsBytes + j * 32, 16, 1024), tc::operand(b_at + s * kRowsBytes + j * 32, 16, 1024), what | pick << 4 | pick << 29,
                                           sa + j / 2 * 4, sb + j / 2 * 8, c > w.c0 || j > 0);
                        }
                    tc::mma_commit<2>(empty + 8 * s);
                }
                if (ok) tc::mma_commit<2>(acc_full + 8 * (done & 1));
            }
            if (*(volatile int*)&failed) {
                tc::mma_commit<2>(drain);
                tc::bar_wait(drain, 0);
            }
        }
    } else if (warp >= 4) {
        const int quad = warp % 4, half = (warp - 4) / 4;  // 32 rows, every other 16 columns
        const uint32_t mine = out_at + (warp - 4) * 2048, lanes = (uint32_t)quad * 32 << 16;
        int done = 0;
        for (int u = first; u < units; u += stride, ++done) {
            const Unit w = unit_of(a, u);
            const uint32_t buf = done & 1;
            if (!warp_waited(acc_full + 8 * buf, done / 2 & 1)) break;
            tc::fence_after();
            const int lr = a.vec ? lane / 4 : lane / 16, lc = a.vec ? lane % 4 * 4 : lane % 16;
            const long long r0 = (long long)w.tm * kTile + rank * kHalf + quad * 32, c0 = (long long)w.tn * kTile;
            const int rows = (int)max(-64ll, min(32ll, a.m - r0)) - lr, cols = (int)min(256ll, a.n - c0) - lc;
            const long long at = (r0 + lr) * a.stride + c0 + lc, pat = w.split * a.m * a.n + (r0 + lr) * a.n + c0 + lc;
#pragma unroll 1
            for (int i = 0; i < 8; ++i) {
                // the columns that both accumulators have come first: the last 48 of the one, the first of the other
                const int col = ((2 * i + half) * 16 + (buf ? 0 : kSecond)) % kTile;
                const uint32_t from = tmem + buf * kSecond + col + lanes;
                if (a.partial) move_out<float>(from, mine, nullptr, a.partial + pat + col, a.n, rows, cols - col, a.vec);
                else move_out<O>(from, mine, a.bias ? (const O*)a.bias + c0 + lc + col : nullptr, (O*)a.y + at + col, a.stride, rows, cols - col, a.vec);
                if (i == 1) {                             // four pieces of 16: 48 shared columns and 16 more
                    tc::fence_before();
                    __syncwarp();
                    if (lane == 0) tc::bar_arrive_cluster(tc::in_cta(acc_free, 0));
                }
            }
        }
    }
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    tc::cluster_sync();                                   // neither CTA's memory is read by the other any more
    if (threadIdx.x == 0 && failed) atomicAdd_system(a.timeouts, 1u);
    if (warp == 2) tc::tmem_free<2>(tmem, 512);
}

// y = the splits' sums, in order, and the bias.
template <typename O>
__global__ void __launch_bounds__(256) mx_matmul_join_kernel(long long m, long long n, int splits, const float* __restrict__ partial, const O* __restrict__ bias, O* __restrict__ y, long long stride)
{
    const long long count = m * n;
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < count; e += (long long)gridDim.x * 256) {
        float v = partial[e];
        for (int s = 1; s < splits; ++s) v += partial[s * count + e];
        const long long r = e / n, c = e - r * n;
        y[r * stride + c] = mx_round<O>(bias ? v + mx_float(bias[c]) : v);
    }
}

// ---- few rows of a
//
// Up to 64 rows of a: reading b is all there is.  b's rows take the tensor cores' 128 rows and a's the columns (16 to 64 of them), a CTA has 128 rows
// of b, and the CTAs of a cluster share the summed index, so that about one CTA an SM streams b.  Each sends its sums' slices of a's rows
// to the CTA of the cluster that has them, which adds them in order: no second kernel, no memory between.  With 8192 x 8192 of b, 7 rows of a take 10.1 us
// (17.0 in the kernel above and its second one), 64 rows 14.8 (17.2); 128 would take 21.1 (20.0), so they do not come here.  (Calls one behind the other:
// 8.8 and 13.6 us where b stays in L2, 10.8 and 16.0 where it comes from memory.)

constexpr int kFewThreads = 256;
template <int N> struct Few {                             // N: rows of a, rounded up
    static constexpr int stages = 6;
    static constexpr int rows_b = 128 * kChunkBytes, rows_a = N * kChunkBytes, scales = 1024;
    static constexpr int stage = rows_b + rows_a + 2 * scales;
    static constexpr int inbox = N * 128 * 4;
    static constexpr int smem = 1024 + stages * stage + inbox + 256;
};

template <typename O, int N>
__global__ void __launch_bounds__(kFewThreads, 1)
mx_matmul_few_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map, const __grid_constant__ MatmulArgs a)
{
    using F = Few<N>;
    extern __shared__ unsigned char raw[];
    const uint32_t base = (tc::smem_at(raw) + 1023) & ~1023u;
    const uint32_t b_at = base, a_at = b_at + F::stages * F::rows_b, sb_at = a_at + F::stages * F::rows_a, sa_at = sb_at + F::stages * F::scales,
                   inbox = sa_at + F::stages * F::scales, bars = inbox + F::inbox;
    const uint32_t full = bars, empty = full + 8 * F::stages, acc_full = empty + 8 * F::stages, slot = acc_full + 8;
    __shared__ int failed;

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, ranks = a.splits;
    const uint32_t rank = tc::cluster_rank();
    const int tile = blockIdx.x / ranks, n0 = tile * 128;
    const int c0 = (int)((long long)rank * a.chunks / ranks), c1 = (int)((long long)(rank + 1) * a.chunks / ranks);

    if (threadIdx.x == 0) {
        for (int s = 0; s < F::stages; ++s) {
            tc::bar_init(full + 8 * s, 1);
            tc::bar_init(empty + 8 * s, 1);
        }
        tc::bar_init(acc_full, 1);
        tc::bar_init_done();
        failed = 0;
        tc::prefetch_map(&a_map);
        tc::prefetch_map(&b_map);
    }
    constexpr uint32_t columns = N <= 32 ? 64 : 128, scales_at = N < 32 ? 32 : N;
    if (warp == 2) tc::tmem_alloc<1>(slot, columns);
    tc::fence_before();
    __syncthreads();
    tc::cluster_started();                                // waited for before the first store to another CTA
    tc::fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(slot));

    auto waited = [&](uint32_t bar, uint32_t parity) {
        if (tc::bar_wait(bar, parity)) return true;
        *(volatile int*)&failed = 1;
        return false;
    };
    // All lanes of a warp go the same way, also where the limit ends between two lanes' tries: what follows takes whole warps.
    auto warp_waited = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, waited(bar, parity)) != 0; };

    if (warp == 0) {
        if (tc::elect()) {
            const uint8_t* sb = a.b_scales + (long long)tile * a.groups * 512;
            int it = 0;
            for (int c = c0; c < c1; ++c, ++it) {
                const int s = it % F::stages;
                const uint32_t bar = full + 8 * s, bytes = min(2, a.groups - 2 * c) * 512;
                if (!waited(empty + 8 * s, (it / F::stages & 1) ^ 1)) break;
                tc::bar_expect(bar, F::rows_b + F::rows_a + 2 * bytes);
                tc::load_2d(b_at + s * F::rows_b, &b_map, c * kChunkBytes, n0, bar);
                tc::load_2d(a_at + s * F::rows_a, &a_map, c * kChunkBytes, 0, bar);
                tc::load_bytes(sb_at + s * F::scales, sb + (long long)c * 1024, bytes, bar);
                tc::load_bytes(sa_at + s * F::scales, a.a_scales + (long long)c * 1024, bytes, bar);
            }
            if (*(volatile int*)&failed)                  // copies still in flight
                for (int i = it < F::stages ? 0 : it - F::stages; i < it; ++i) tc::bar_wait(full + 8 * (i % F::stages), i / F::stages & 1);
        }
    } else if (warp == 1) {
        if (tc::elect()) {
            constexpr uint32_t what = 1u << 7 | 1u << 10 | (uint32_t)(N >> 3) << 17 | 1u << 23 | (uint32_t)(128 >> 4) << 24;
            const uint32_t sb = tmem + scales_at, sa = sb + 8;
            int it = 0;
            for (int c = c0; c < c1; ++c, ++it) {
                const int s = it % F::stages;
                if (!waited(full + 8 * s, it / F::stages & 1)) break;
                tc::fence_after();
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    tc::copy_scales<1>(sb + g * 4, tc::operand_plain(sb_at + s * F::scales + g * 512));
                    tc::copy_scales<1>(sa + g * 4, tc::operand_plain(sa_at + s * F::scales + g * 512));
                }
                const int steps = min(4, (a.blocks - c * kChunkBlocks + 1) / 2);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < steps) {
                        const uint32_t pick = (j & 1) * 2;
                        tc::mma_mx4<1>(tmem, tc::operand(b_at + s * F::rows_b + j * 32, 16, 1024), tc::operand(a_at + s * F::rows_a + j * 32, 16, 1024), what | pick << 4 | pick << 29,
                                       sb + j / 2 * 4, sa + j / 2 * 4, c > c0 || j > 0);
                    }
                tc::mma_commit<1>(empty + 8 * s);
            }
            tc::mma_commit<1>(acc_full);                  // also after a wait that ran out: nothing may be in flight when the memory goes
            tc::bar_wait(acc_full, 0);
        }
    }
    __syncwarp();
    tc::cluster_wait();                                   // the CTAs that the sums go to run
    const int quad = warp - 4, row = quad * 32 + lane, mine = N / ranks;      // a thread has one row of b; this CTA finishes `mine` rows of a
    bool ok = true;
    if (warp >= 4) {
        ok = warp_waited(acc_full, 0);
        tc::fence_after();
        if (ok) {
#pragma unroll 1
            for (int j = 0; j < N; j += 16) {
                uint32_t v[16];
                tc::tmem_load16(tmem + j + ((uint32_t)quad * 32 << 16), v);
                tc::tmem_wait_load();
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int col = j + i, to = col / mine;
                    const uint32_t at = inbox + (((rank * mine) + col % mine) * 128 + row) * 4;
                    asm volatile("st.shared::cluster.b32 [%0], %1;" :: "r"(tc::in_cta(at, to)), "r"(v[i]) : "memory");
                }
            }
        }
    }
    tc::fence_before();
    __syncthreads();
    tc::cluster_sync();                                   // every slice is where it belongs
    if (warp >= 4 && ok && n0 + row < a.n) {
        const float b = a.bias ? mx_float(((const O*)a.bias)[n0 + row]) : 0.f;
        for (int j = 0; j < mine; ++j) {
            const int col = rank * mine + j;
            if (col >= a.m) break;
            float sum = 0.f;
            for (int r = 0; r < ranks; ++r) {
                float v;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(inbox + ((r * mine + j) * 128 + row) * 4));
                sum = r ? sum + v : v;
            }
            ((O*)a.y)[col * a.stride + n0 + row] = mx_round<O>(a.bias ? sum + b : sum);
        }
    }
    if (threadIdx.x == 0 && failed) atomicAdd_system(a.timeouts, 1u);
    if (warp == 2) tc::tmem_free<1>(tmem, columns);
}

struct MatmulPlan { int few, tiles_m, tiles_n, splits, chunks, clusters; size_t partial; };

MatmulPlan plan_of(const galv_ctx* ctx, int64_t m, int64_t n, int64_t k)
{
    MatmulPlan p;
    const int most = ctx->num_sms / 2;
    p.tiles_m = (int)((m + kTile - 1) / kTile);
    p.tiles_n = (int)((n + kTile - 1) / kTile);
    p.chunks = (int)((mx_blocks(k) + kChunkBlocks - 1) / kChunkBlocks);
    p.few = m <= 16 ? 16 : m <= 32 ? 32 : m <= 64 ? 64 : 0;
    if (p.few) {                                          // clusters along the summed index, two chunks a CTA at least
        p.tiles_m = 1;
        p.tiles_n = (int)((n + 127) / 128);
        p.splits = 1;
        while (p.splits < 8 && (int64_t)p.tiles_n * p.splits * 2 <= ctx->num_sms && p.chunks >= p.splits * 4) p.splits *= 2;
        p.clusters = p.tiles_n;
        p.partial = 0;
        return p;
    }
    const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
    p.splits = 1;
    if (tiles < most && p.chunks >= 8) {
        p.splits = (int)(most / tiles);
        if (p.splits > p.chunks / 4) p.splits = p.chunks / 4;
    }
    const int64_t units = tiles * p.splits;
    p.clusters = (int)(units < most ? units : most);
    p.partial = p.splits > 1 ? (((size_t)p.splits * m * n * 4 + 255) & ~(size_t)255) : 0;
    return p;
}

template <typename O, int N>
cudaError_t launch_few(const MatmulPlan& p, const CUtensorMap& am, const CUtensorMap& bm, const MatmulArgs& a, cudaStream_t st)
{
    cudaError_t e = cudaFuncSetAttribute(mx_matmul_few_kernel<O, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, Few<N>::smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.tiles_n * p.splits));
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = Few<N>::smem;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)p.splits;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, mx_matmul_few_kernel<O, N>, am, bm, a);
}

template <typename O>
cudaError_t launch(const galv_ctx* ctx, const MatmulPlan& p, const CUtensorMap& am, const CUtensorMap& bm, const MatmulArgs& a, cudaStream_t st)
{
    if (p.few == 16) return launch_few<O, 16>(p, am, bm, a, st);
    if (p.few == 32) return launch_few<O, 32>(p, am, bm, a, st);
    if (p.few == 64) return launch_few<O, 64>(p, am, bm, a, st);
    cudaError_t e = cudaFuncSetAttribute(mx_matmul_kernel<O>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    mx_matmul_kernel<O><<<p.clusters * 2, kThreads, kSmem, st>>>(am, bm, a);
    if (a.partial) mx_matmul_join_kernel<O><<<ctx->num_sms * 8, 256, 0, st>>>(a.m, a.n, a.splits, a.partial, (const O*)a.bias, (O*)a.y, a.stride);
    return cudaGetLastError();
}

}  // namespace

extern "C" size_t galv_mx_matmul_workspace_bytes(const galv_ctx* ctx, int64_t m, int64_t n, int64_t k)
{
    if (!ctx || !mx_size_ok(m, k) || !mx_size_ok(n, k) || m == 0 || n == 0) return 0;
    return plan_of(ctx, m, n, k).partial;
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
    const MatmulPlan p = plan_of(ctx, m, n, k);
    if (p.partial && (!workspace || !mx_aligned(workspace, 256) || workspace_bytes < p.partial))
        return galv_set_error(ctx, GALV_ERR_WORKSPACE, "galv_mx_matmul: workspace NULL, misaligned or too small");
    const int may = mx_may_run(ctx, "galv_mx_matmul: the library's host memory could not be registered", "galv_mx_matmul: a bounded wait of an earlier microscaled product ran out");
    if (may != GALV_OK) return may;
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    CUtensorMap am, bm;
    const uint64_t pitch = mx_blocks(k) * 16;
    cudaError_t e = galv_mx_map(&am, CU_TENSOR_MAP_DATA_TYPE_UINT8, a_codes, m, pitch, pitch, p.few ? p.few : kHalf, kChunkBytes, true);
    if (e == cudaSuccess) e = galv_mx_map(&bm, CU_TENSOR_MAP_DATA_TYPE_UINT8, b_codes, n, pitch, pitch, kHalf, kChunkBytes, true);
    if (e != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, "galv_mx_matmul: tensor map");
    MatmulArgs a;
    a.m = m; a.n = n; a.stride = y_stride;
    a.blocks = (int)mx_blocks(k); a.groups = (a.blocks + 3) / 4;
    a.tiles_m = p.tiles_m; a.tiles_n = p.tiles_n; a.splits = p.splits; a.chunks = p.chunks;
    a.a_scales = a_scales; a.b_scales = b_scales; a.bias = bias; a.y = y; a.timeouts = ctx->mx_timeouts_at;
    a.partial = p.partial ? reinterpret_cast<float*>(workspace) : nullptr;
    a.vec = p.partial ? n % 4 == 0 : n % 4 == 0 && y_stride % 4 == 0 && mx_aligned(y, 4 * mx_size_of(dtype));
    MX_DISPATCH_TYPE(dtype, e = launch<T>(ctx, p, am, bm, a, (cudaStream_t)stream));
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}

// Waits that have run out are counted in host memory, a line of 64 bytes a device, so that they can be read without waiting for anything.  The
// memory is the process's own and only registered with CUDA: it outlives a device that is reset.  Where it cannot be registered, only the products are refused.
void galv_mx_configure(galv_ctx* ctx)
{
    constexpr int most = 64, words = 16;
    alignas(4096) static unsigned counts[most * words];
    static unsigned none = 0;
    static std::mutex registering;
    const bool in = ctx->device >= 0 && ctx->device < most;
    ctx->mx_timeouts = in ? counts + ctx->device * words : &none;
    ctx->mx_timeouts_at = nullptr;
    std::lock_guard<std::mutex> lock(registering);
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;         // another thread may be capturing
    if (in && cudaThreadExchangeStreamCaptureMode(&mode) == cudaSuccess) {
        void* at = nullptr;
        const cudaError_t e = cudaHostRegister(counts, sizeof(counts), cudaHostRegisterMapped | cudaHostRegisterPortable);
        if ((e == cudaSuccess || e == cudaErrorHostMemoryAlreadyRegistered) && cudaHostGetDevicePointer(&at, ctx->mx_timeouts, 0) == cudaSuccess)
            ctx->mx_timeouts_at = static_cast<unsigned*>(at);
        cudaThreadExchangeStreamCaptureMode(&mode);
    }
    (void)cudaGetLastError();                             // what went wrong here is not the next call's
    ctx->mx_timeouts_seen = *(volatile unsigned*)ctx->mx_timeouts;
}

extern "C" uint32_t* galv_mx_timeouts(const galv_ctx* ctx) { return ctx ? ctx->mx_timeouts : nullptr; }

extern "C" int galv_mx_status(galv_ctx* ctx, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    const cudaError_t e = cudaStreamSynchronize((cudaStream_t)stream);
    if (e != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
    return mx_ran_out(ctx) ? galv_set_error(ctx, GALV_ERR_TIMEOUT, "galv_mx_status: a bounded wait of a microscaled product ran out") : GALV_OK;
}
