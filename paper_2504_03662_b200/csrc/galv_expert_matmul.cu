// Products of tokens and weights, each token by its expert's: y[r][j] = sum_c x[r][c] w[e][j][c] + bias[e][j] for the rows r of expert e, in 16 bits or in 8-bit
// integers, and the gradient of x; one expert that has all rows is a plain product.
//
// Rows are sorted by expert, where they end is known on the device alone.  So each CTA finds the tiles there are (a scan over the experts), and a grid that
// fills the card walks through them.  The weights' rows take the tensor cores' 256 rows of a pair of CTAs, the tokens their columns, as many as an expert's last
// tile has (a multiple of 32): what ragged sizes waste is less than 32 tokens an expert, and a few tokens cost little more than reading the weights.
// A column of sums depends on its own token alone: a tile's copy of tokens may run into the next expert's, whose sums nobody takes, whatever they are.
// Per CTA: a thread that starts bulk tensor copies (128 bytes of the summed index a chunk: 128 rows of weights, half of the tile's tokens; both CTAs' tell the
// first one's barrier), one (in the first) that issues the matrix instructions for the pair, eight warps that move
// sums from the tensor memory to y while the next are made (two accumulators fill it).
//
// Bound by the tensor cores at the clock that the card's power allows: 16384 rows over 8 experts, 8192 x 2048 in bf16, take 366 to 380 us (1.45 to 1.5 PFLOP/s, tensor pipe active 93 % of the cycles),
// 429 in a loop of seconds (a library product of that size 416); 4096 x 8192 x 32768 in 8-bit integers 622 us (3.5 POP/s, 98 %), 745 in such a loop (763).  The input gradient of 8192 rows over 16 experts,
// 4096 x 2048: 106 to 119 us (78 %: five rounds of tiles where four and a half would do).

#include <stdio.h>

#include "galv_experts.cuh"
#include "galv_i8.cuh"
#include "galv_tc.cuh"

namespace {

enum Kind { kForward, kInputGrad, kWhole };               // 16 bits, summed along the weights' rows; across them; 8-bit integers

constexpr int kTile = 256, kHalf = kTile / 2, kChunkBytes = 128;
constexpr int kRowsBytes = kHalf * kChunkBytes;
// The ring of chunks: 6 of full tiles, up to 10 of smaller ones, whose matrix instructions are over sooner and whose copies are to be as far ahead.
constexpr int kRing = 12 * kRowsBytes, kStagesMost = 10;
constexpr int kOutBytes = 8 * 2048;
constexpr int kBox = 64, kPart = 16;                      // tokens of a copy, and of one where fewer are left
constexpr int kThreads = 384;
// What a chunk costs besides its tokens, in tokens.  Measured at 256, 160, 128 and 64 tokens of every tile (2048 x 8192): 396, 285, 257 and 213 ns in 16 bits, 425, 306, 272 and 237 in 8-bit integers.
constexpr float kFixed = 160.f;
constexpr int kGroup = 16;                                // tiles of tokens that stay in L2 while their tiles of weights run

struct ProductArgs {
    long long rows, n, stride;                            // tokens, columns of y, from one row of y to the next
    int experts, tiles_m, chunks, last_steps;             // last_steps: of 32 bytes in the last chunk
    uint32_t what;                                        // the matrix instruction without its sizes (the second kernel's: without its number of tokens)
    const int32_t* ends;
    const float* x_scales;
    const float* w_scales;
    const void* bias;
    void* y;
    int vec;                                              // 16 bytes of a row of y can be moved at once
    int in_front;                                         // the kernel before this one in the stream puts the tokens into 8-bit integers: all before it is over
    unsigned* timeouts;                                   // host memory: CTAs that have given up a wait
};

// A walk through the tiles: units of 256 weights' rows by up to 256 tokens, those of an expert next to one another.
struct Walk {
    const int* begin;
    const int* before;
    int tiles_m, expert = -1, from = 0, all = 0, each = 0;      // the expert's first tile of tokens, how many it has and of how many rows
    int tm, row0, count;                                  // tile of weights' rows; first token and number of tokens
    __device__ __forceinline__ Walk(const int* begin_, const int* before_, int tiles_m_) : begin(begin_), before(before_), tiles_m(tiles_m_) {}
    __device__ __forceinline__ void to(int u)             // units in rising order
    {
        if (u >= (from + all) * tiles_m) {
            do {
                ++expert;
                from += all;
                all = before[expert + 1] - from;
            } while (u >= (from + all) * tiles_m);
            each = experts_tile(begin[expert + 1] - begin[expert], all);
        }
        const int local = u - from * tiles_m, per = kGroup * tiles_m, first = local / per * kGroup, size = min(kGroup, all - first), in = local % per;
        row0 = begin[expert] + (first + in % size) * each;
        tm = in / size;
        count = min(each, begin[expert + 1] - row0);
    }
    __device__ __forceinline__ int columns() const { return (count + 31) & ~31; }
};

// 16 tokens' sums of a warp's 32 channels, a channel a lane, as numbers.
template <int K>
__device__ __forceinline__ float number(uint32_t sum, float x_scale, float w_scale, float bias)
{
    if (K == kWhole) return fmaf((float)(int)sum, x_scale * w_scale, bias);
    return __uint_as_float(sum) + bias;
}

template <int K, typename O>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
expert_product_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap part_map,
                      const __grid_constant__ ProductArgs a)
{
    extern __shared__ unsigned char raw[];
    const uint32_t base = (tc::smem_at(raw) + 1023) & ~1023u;
    const uint32_t out_at = base + kRing, bars = out_at + kOutBytes;
    const uint32_t full = bars, empty = full + 8 * kStagesMost, acc_full = empty + 8 * kStagesMost, acc_empty = acc_full + 16, drain = acc_empty + 16,
                   slot = drain + 8;
    int* const begin = reinterpret_cast<int*>(raw + (bars + 256 - tc::smem_at(raw)));
    int* const before = begin + a.experts + 1;
    __shared__ int failed;
    __shared__ float prices[8];
    __shared__ int most;                                  // tokens of a tile

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = tc::cluster_rank();
    const int first = blockIdx.x / 2, stride = gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStagesMost; ++s) {
            tc::bar_init(full + 8 * s, 1);
            tc::bar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            tc::bar_init(acc_full + 8 * b, 1);
            tc::bar_init(acc_empty + 8 * b, 16);
        }
        tc::bar_init(drain, 1);
        tc::bar_init_done();
        failed = 0;
        tc::prefetch_map(&w_map);
        tc::prefetch_map(&x_map);
        tc::prefetch_map(&part_map);
    }
    if (warp == 2) tc::tmem_alloc<2>(slot, 512);
    const bool in_front = K == kWhole && a.in_front;
    if (!in_front) tc::before_is_over();
    tc::next_may_start();
    if (warp == 3) experts_begin(a.ends, a.experts, a.rows, begin);
    __syncthreads();
    if (warp >= 4) {                                      // a size of tiles each: 256, 224 .. 32 rows
        const float price = experts_price(begin, a.experts, kTile - (warp - 4) * 32, a.tiles_m, stride, kFixed);
        if (lane == 0) prices[warp - 4] = price;
    }
    __syncthreads();
    if (warp == 3) {                                      // the cheapest, of equals the largest
        int best = 0;
        for (int i = 1; i < 8; ++i)
            if (prices[i] < prices[best]) best = i;
        experts_before(begin, a.experts, kTile - best * 32, before);
        if (lane == 0) most = kTile - best * 32;
    }
    tc::fence_before();
    __syncthreads();
    tc::cluster_sync();                                   // the pair's barriers exist
    tc::fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(slot));
    const int units = before[a.experts] * a.tiles_m, stage = kRowsBytes + most / 2 * kChunkBytes, stages = min(kStagesMost, kRing / stage);

    auto waited = [&](uint32_t bar, uint32_t parity) {
        if (tc::bar_wait_asleep<true>(bar, parity)) return true;
        *(volatile int*)&failed = 1;
        return false;
    };
    // One lane of a warp waits: eight warps of 32 asking all the time slow the issuing thread's own questions (tiles of 64 tokens: 263 ns a chunk for 213).
    auto warp_waited = [&](uint32_t bar, uint32_t parity) { return __shfl_sync(0xffffffffu, (int)(lane == 0 && waited(bar, parity)), 0) != 0; };
    Walk w(begin, before, a.tiles_m);

    if (warp == 0) {
        if (tc::elect()) {
            constexpr int elements = K == kWhole ? kChunkBytes : kChunkBytes / 2;
            int s = 0;
            uint32_t turn = 1;
            bool ok = true, over = !in_front;
            for (int u = first; u < units && ok; u += stride) {
                w.to(u);
                const int m0 = w.tm * kTile + rank * kHalf, half = w.columns() / 2, r0 = w.row0 + rank * half;
                auto weights = [&](int s, int c) {
                    const uint32_t bar = tc::in_cta(full + 8 * s, 0), to = base + s * stage;
                    if (rank == 0) tc::bar_expect(full + 8 * s, 2 * (kRowsBytes + half * kChunkBytes));      // of both CTAs
                    if (K == kInputGrad) {                // 64 rows of weights, 64 columns a copy
                        tc::load_3d_pair(to, &w_map, m0, c * elements, w.expert, bar);
                        tc::load_3d_pair(to + kRowsBytes / 2, &w_map, m0 + 64, c * elements, w.expert, bar);
                    } else {
                        tc::load_3d_pair(to, &w_map, c * elements, m0, w.expert, bar);
                    }
                };
                int ahead = 0;
                if (!over) {                              // the kernel in front may still be putting the tokens into 8-bit integers: the weights do not wait for it
                    for (ahead = 0; ahead < min(stages, a.chunks); ++ahead) weights(ahead, ahead);
                    tc::before_is_over();
                    over = true;
                }
                for (int c = 0; c < a.chunks; ++c) {
                    if (c >= ahead) {
                        if (!(ok = waited(empty + 8 * s, turn))) break;
                        weights(s, c);
                    }
                    const uint32_t bar = tc::in_cta(full + 8 * s, 0), to = base + s * stage + kRowsBytes;
                    int i = 0;
                    for (; i + kBox <= half; i += kBox) tc::load_2d_pair(to + i * kChunkBytes, &x_map, c * elements, r0 + i, bar);
                    for (; i < half; i += kPart) tc::load_2d_pair(to + i * kChunkBytes, &part_map, c * elements, r0 + i, bar);
                    if (++s == stages) s = 0, turn ^= 1;
                }
            }
            if (*(volatile int*)&failed) tc::settle();
        }
    } else if (warp == 1 && rank == 0) {
        if (tc::elect()) {
            int s = 0, done = 0;
            uint32_t turn = 0;
            bool ok = true;
            for (int u = first; u < units && ok; u += stride, ++done) {
                w.to(u);
                const uint32_t buf = done & 1, d = tmem + buf * kTile, what = a.what | (uint32_t)(w.columns() >> 3) << 17;
                if (!(ok = waited(acc_empty + 8 * buf, (done / 2 & 1) ^ 1))) break;
                tc::fence_after();
                for (int c = 0; c < a.chunks; ++c) {
                    const int steps = c + 1 < a.chunks ? 4 : a.last_steps;
                    const uint32_t ws = base + s * stage, xs = ws + kRowsBytes;
                    if (!(ok = waited(full + 8 * s, turn))) break;
                    tc::fence_after();
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < steps) {
                            const uint64_t wo = K == kInputGrad ? tc::operand(ws + j * 2048, kRowsBytes / 2, 1024) : tc::operand(ws + j * 32, 16, 1024), xo = tc::operand(xs + j * 32, 16, 1024);
                            if (K == kWhole) tc::mma_i8<2>(d, wo, xo, what, c > 0 || j > 0);
                            else tc::mma_f16<2>(d, wo, xo, what, c > 0 || j > 0);
                        }
                    tc::mma_commit<2>(empty + 8 * s);
                    if (++s == stages) s = 0, turn ^= 1;
                }
                if (ok) tc::mma_commit<2>(acc_full + 8 * buf);
            }
            if (*(volatile int*)&failed) {
                tc::mma_commit<2>(drain);
                tc::bar_wait(drain, 0);
            }
        }
    } else if (warp >= 4) {
        constexpr int pieces = 32 * (int)sizeof(O) / 16;  // 16-byte pieces of a token's 32 channels
        const int quad = warp % 4, half = (warp - 4) / 4;  // 32 channels, every other 16 tokens
        const uint32_t mine = out_at + (warp - 4) * 2048, lanes = (uint32_t)quad * 32 << 16;
        O* const y = (O*)a.y;
        int done = 0;
        if (in_front) tc::before_is_over();
        for (int u = first; u < units; u += stride, ++done) {
            w.to(u);
            const uint32_t buf = done & 1;
            const long long c0 = (long long)w.tm * kTile + rank * kHalf + quad * 32, ch = c0 + lane, at = w.expert * a.n + ch;
            const float bias = a.bias && ch < a.n ? mx_float(((const O*)a.bias)[at]) : 0.f, w_scale = K == kWhole && ch < a.n ? a.w_scales[at] : 0.f;
            if (!warp_waited(acc_full + 8 * buf, done / 2 & 1)) break;
            tc::fence_after();
            for (int j = half * 16; j < w.count; j += 32) {
                const int tokens = min(16, w.count - j);
                const long long r0 = (long long)w.row0 + j;
                uint32_t s[16];
                float x_scale = 0.f;
                if (K == kWhole && lane < tokens) x_scale = a.x_scales[r0 + lane];
                tc::tmem_load16(tmem + buf * kTile + j + lanes, s);
                tc::tmem_wait_load();
                if (a.vec) {
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const O v = mx_round<O>(number<K>(s[i], K == kWhole ? __shfl_sync(0xffffffffu, x_scale, i) : 0.f, w_scale, bias));
                        const uint32_t to = mine + (i * 32 + lane) * (int)sizeof(O);
                        if (sizeof(O) == 2) asm volatile("st.shared.b16 [%0], %1;" :: "r"(to), "h"(*reinterpret_cast<const uint16_t*>(&v)) : "memory");
                        else asm volatile("st.shared.b32 [%0], %1;" :: "r"(to), "r"(*reinterpret_cast<const uint32_t*>(&v)) : "memory");
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 16 * pieces; i += 32) {
                        const int p = i + lane, token = p / pieces, piece = p % pieces;
                        uint4 q;
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(mine + p * 16));
                        const long long col = c0 + piece * (16 / (int)sizeof(O));
                        if (token < tokens && col < a.n) *reinterpret_cast<uint4*>(y + (r0 + token) * a.stride + col) = q;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float v = number<K>(s[i], K == kWhole ? __shfl_sync(0xffffffffu, x_scale, i) : 0.f, w_scale, bias);
                        if (i < tokens && ch < a.n) y[(r0 + i) * a.stride + ch] = mx_round<O>(v);
                    }
                }
            }
            tc::fence_before();
            __syncwarp();
            if (lane == 0) tc::bar_arrive_cluster(tc::in_cta(acc_empty + 8 * buf, 0));
        }
        // rows of no expert
        for (long long r = begin[a.experts] + (long long)blockIdx.x * 8 + warp - 4; r < a.rows; r += gridDim.x * 8ll)
            for (long long c = lane; c < a.n; c += 32) y[r * a.stride + c] = mx_zero<O>();
    }
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    tc::cluster_sync();                                   // neither CTA's memory is read by the other any more
    if (threadIdx.x == 0 && failed) atomicAdd_system(a.timeouts, 1u);
    if (warp == 2) tc::tmem_free<2>(tmem, 512);
}

// ---- few rows
//
// Up to 64 rows in all: reading the weights of the experts that have some is all there is.  (And more rows of so few results that tiles of 256 would leave most SMs without one: the rows go
// in tiles of 64 then.)  A CTA has 128 of an expert's weights' rows, so that two fit an SM and one starts while the other runs; the CTAs of a cluster share the summed index, so that about two an SM stream.  Each sends its sums' slices of the tokens
// to the CTA of the cluster that has them, which adds them in order: no second kernel, no memory between.  Which tile of rows a cluster has is found on the device; clusters
// are launched for as many as there could be, those that are too many end at once.  The weights' first copies
// start before the kernel in front, which puts the tokens into 8-bit integers, is over.  1 x 8192 x 8192 in 8-bit integers takes 15.8 us with packing in front (67 MB: 6.4 TB/s for 10.4 us; the rest
// is the start and, for 2 us, joining; in the kernel above 21.6 alone), 48 x 2048 x 8192 10, 64 rows over 64 experts of 4096 x 2048 52 (280 MB, 5.4 TB/s).

constexpr int kFewThreads = 256, kFewRows = 64, kFewStages = 6;
constexpr int kFewRing = 6 * (128 + kPart) * kChunkBytes;      // shared memory of chunks and of what other CTAs send: 6 chunks for up to 16 tokens, 4 for 64; 5 and 3 in a cluster
constexpr int kFewSmem = 1024 + kFewRing + 256;

template <int K, typename O>
__global__ void __launch_bounds__(kFewThreads, 2)
expert_few_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap part_map, const __grid_constant__ ProductArgs a, int tiles, int ranks)
{
    extern __shared__ unsigned char raw[];
    const uint32_t base = (tc::smem_at(raw) + 1023) & ~1023u;
    const uint32_t bars = base + kFewRing, full = bars, empty = full + 8 * kFewStages, acc_full = empty + 8 * kFewStages, slot = acc_full + 8;
    __shared__ float x_scales[kFewRows];
    __shared__ int failed, mine[4];                       // expert (or -1), its first row, how many; where rows of no expert begin

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = tc::cluster_rank();
    const int unit = blockIdx.x / ranks, tile = unit % tiles, nth = unit / tiles;
    const long long n0 = tile * 128ll;
    const int c0 = (int)((long long)rank * a.chunks / ranks), c1 = (int)((long long)(rank + 1) * a.chunks / ranks);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kFewStages; ++s) {
            tc::bar_init(full + 8 * s, 1);
            tc::bar_init(empty + 8 * s, 1);
        }
        tc::bar_init(acc_full, 1);
        tc::bar_init_done();
        failed = 0;
        tc::prefetch_map(&w_map);
        tc::prefetch_map(&part_map);
    }
    constexpr uint32_t columns = kFewRows;
    if (warp == 2) tc::tmem_alloc<1>(slot, columns);
    if (K != kWhole || !a.in_front) tc::before_is_over();
    tc::next_may_start();
    if (warp == 3) experts_nth(a.ends, a.experts, a.rows, kFewRows, nth, mine);
    tc::fence_before();
    __syncthreads();
    const int expert = mine[0], row0 = mine[1], count = mine[2];
    if (expert < 0 && nth > 0) {                          // there are not so many: the whole cluster ends
        tc::before_is_over();
        if (warp == 2) {
            uint32_t tmem;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(slot));
            tc::tmem_free<1>(tmem, columns);
        }
        return;
    }
    tc::cluster_started();                                // waited for before the first store to another CTA
    tc::fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(slot));

    auto waited = [&](uint32_t bar, uint32_t parity) {
        if (tc::bar_wait_asleep<false>(bar, parity)) return true;
        *(volatile int*)&failed = 1;
        return false;
    };

    const int boxes = (count + kPart - 1) / kPart, tokens = boxes * kPart;      // copies of tokens; none where nobody has rows
    const int stage = (128 + tokens) * kChunkBytes, sent = ranks > 1 ? tokens * 512 : 0, stages = min(kFewStages, (kFewRing - sent) / stage), chunks = boxes ? c1 - c0 : 0;
    const uint32_t inbox = base + kFewRing - sent;
    if (warp == 0) {
        if (tc::elect()) {
            constexpr int elements = K == kWhole ? kChunkBytes : kChunkBytes / 2;
            const int ahead = min(stages, chunks);
            auto weights = [&](int s, int it) {
                tc::bar_expect(full + 8 * s, stage);
                if (K == kInputGrad) {
                    tc::load_3d(base + s * stage, &w_map, (int)n0, (c0 + it) * elements, expert, full + 8 * s);
                    tc::load_3d(base + s * stage + kRowsBytes / 2, &w_map, (int)n0 + 64, (c0 + it) * elements, expert, full + 8 * s);
                } else {
                    tc::load_3d(base + s * stage, &w_map, (c0 + it) * elements, (int)n0, expert, full + 8 * s);
                }
            };
            for (int it = 0; it < ahead; ++it) weights(it, it);
            tc::before_is_over();
            int it = 0, s = 0;
            uint32_t turn = 1;
            for (; it < chunks; ++it) {
                if (it >= ahead) {
                    if (!waited(empty + 8 * s, turn)) break;
                    weights(s, it);
                }
                for (int i = 0; i < boxes; ++i)
                    tc::load_2d(base + s * stage + (128 + i * kPart) * kChunkBytes, &part_map, (c0 + it) * elements, row0 + i * kPart, full + 8 * s);
                if (++s == stages) s = 0, turn ^= 1;
            }
            if (*(volatile int*)&failed) tc::settle();
        }
    } else if (warp == 1) {
        if (tc::elect()) {
            const uint32_t what = a.what | (uint32_t)(tokens >> 3) << 17 | (uint32_t)(128 >> 4) << 24;
            int s = 0;
            uint32_t turn = 0;
            for (int it = 0; it < chunks; ++it) {
                const int steps = c0 + it + 1 < a.chunks ? 4 : a.last_steps;
                const uint32_t ws = base + s * stage, xs = ws + kRowsBytes;
                if (!waited(full + 8 * s, turn)) break;
                tc::fence_after();
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < steps) {
                        const uint64_t wo = K == kInputGrad ? tc::operand(ws + j * 2048, kRowsBytes / 2, 1024) : tc::operand(ws + j * 32, 16, 1024), xo = tc::operand(xs + j * 32, 16, 1024);
                        if (K == kWhole) tc::mma_i8<1>(tmem, wo, xo, what, it > 0 || j > 0);
                        else tc::mma_f16<1>(tmem, wo, xo, what, it > 0 || j > 0);
                    }
                tc::mma_commit<1>(empty + 8 * s);
                if (++s == stages) s = 0, turn ^= 1;
            }
            tc::mma_commit<1>(acc_full);                  // also after a wait that ran out: nothing may be in flight when the memory goes
            tc::bar_wait_asleep<false>(acc_full, 0);
        }
    }
    __syncwarp();
    tc::before_is_over();
    tc::cluster_wait();                                   // the CTAs that the sums go to run
    const int quad = warp - 4, row = quad * 32 + lane, each = tokens / ranks;      // a thread has one row of weights; this CTA finishes `each` tokens
    const long long ch = n0 + row, at = expert * a.n + ch;
    const bool has = warp >= 4 && expert >= 0 && ch < a.n;
    const float bias = a.bias && has ? mx_float(((const O*)a.bias)[at]) : 0.f, w_scale = K == kWhole && has ? a.w_scales[at] : 0.f;
    O* const y = (O*)a.y + ch;
    auto put = [&](int token, uint32_t sum) { y[(long long)(row0 + token) * a.stride] = mx_round<O>(number<K>(sum, K == kWhole ? x_scales[token] : 0.f, w_scale, bias)); };
    if (K == kWhole && warp >= 4) {                       // the tokens' scales, on their way while the sums are
        if (row < count) x_scales[row] = a.x_scales[row0 + row];
        asm volatile("bar.sync 1, 128;" ::: "memory");
    }
    bool ok = true;
    if (warp >= 4) {
        ok = __shfl_sync(0xffffffffu, (int)(lane == 0 && waited(acc_full, 0)), 0) != 0;
        tc::fence_after();
        if (ok) {
            // sums of token `to * each + j` to the `to`-th CTA: its [ranks][each] rows of 128 sums
            int to = 0, j = 0;
            uint32_t there = tc::in_cta(inbox + (rank * each * 128 + row) * 4, 0);
#pragma unroll 1
            for (int col = 0; col < tokens; col += 16) {
                uint32_t v[16];
                tc::tmem_load16(tmem + col + ((uint32_t)quad * 32 << 16), v);
                tc::tmem_wait_load();
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (ranks > 1) {
                        asm volatile("st.shared::cluster.b32 [%0], %1;" :: "r"(there), "r"(v[i]) : "memory");
                        there += 512;
                        if (++j == each) {
                            j = 0;
                            ++to;
                            there = tc::in_cta(inbox + (rank * each * 128 + row) * 4, to < ranks ? to : 0);
                        }
                    } else if (has && col + i < count) {
                        put(col + i, v[i]);
                    }
                }
            }
        }
    }
    tc::fence_before();
    __syncthreads();
    if (ranks > 1) {
        tc::cluster_sync();                               // every slice is where it belongs
        if (has && ok)
            for (int j = 0; j < each; ++j) {
                const int col = rank * each + j;
                if (col >= count) break;
                uint32_t v[8], sum = 0;
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < ranks) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v[r]) : "r"(inbox + ((r * each + j) * 128 + row) * 4));
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < ranks) sum = r == 0 ? v[r] : K == kWhole ? sum + v[r] : __float_as_uint(__uint_as_float(sum) + __uint_as_float(v[r]));
                put(col, sum);
            }
    }
    if (nth == 0 && warp >= 4 && ch < a.n)                // rows of no expert
        for (long long r = mine[3] + (int)rank; r < a.rows; r += ranks) y[r * a.stride] = mx_zero<O>();
    if (threadIdx.x == 0 && failed) atomicAdd_system(a.timeouts, 1u);
    if (warp == 2) tc::tmem_free<1>(tmem, columns);
}

size_t up(size_t x) { return (x + 255) & ~(size_t)255; }
int smem_of(int experts) { return 1024 + kRing + kOutBytes + 256 + 8 * (experts + 1); }

// Where the operands of a product in 16 bits that bulk copies cannot take as they are go in the workspace.
struct AlignPlan { size_t x, w, total; };
AlignPlan align_plan(int64_t rows, int64_t x_cols, const void* x, int64_t x_stride, int64_t experts, int64_t n, int64_t k, const void* w, int64_t w_stride)
{
    AlignPlan p;
    p.x = mx_rows16(x, x_stride, GALV_BF16) && x_stride * 2 < ((int64_t)1 << 40) ? 0 : up((size_t)rows * galv_aligned_pitch(x_cols) * 2);
    p.w = mx_rows16(w, w_stride, GALV_BF16) && n * w_stride * 2 < ((int64_t)1 << 40) ? 0 : up((size_t)experts * n * galv_aligned_pitch(k) * 2);
    p.total = p.x + p.w;
    return p;
}

// Tiles of 64 rows there can be, whatever the ends say, times tiles of 128 weights' rows.
int64_t few_units(const ProductArgs& a) { return (a.rows / kFewRows + (a.rows < a.experts ? a.rows : a.experts)) * ((a.n + 127) / 128); }

// Few rows; or a long sum for few results: clusters of 8 with four chunks a CTA or more, all at once on the card (100 rows x 32768 x 16 in 8-bit integers with packing: 60 us in the kernel above, 26 here).
bool is_few(const galv_ctx* ctx, const ProductArgs& a) { return a.rows <= kFewRows || (a.chunks >= 32 && few_units(a) * 8 <= 2 * ctx->num_sms); }

template <int K, typename O>
cudaError_t launch_few(const galv_ctx* ctx, const CUtensorMap& wm, const CUtensorMap& pm, const ProductArgs& a, cudaStream_t st)
{
    const cudaError_t e = cudaFuncSetAttribute(expert_few_kernel<K, O>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
    if (e != cudaSuccess) return e;
    const int tiles = (int)((a.n + 127) / 128);
    const int64_t units = a.rows <= kFewRows ? tiles * (int64_t)(a.rows < a.experts ? a.rows : a.experts) : few_units(a);
    int ranks = 1;                                        // two CTAs an SM at most, two chunks a CTA at least
    while (ranks < 8 && units * ranks <= ctx->num_sms && a.chunks >= ranks * 4) ranks *= 2;
    tc::Launch l((unsigned)(units * ranks), kFewThreads, kFewSmem, (unsigned)ranks, true, st);
    return cudaLaunchKernelEx(&l.cfg, expert_few_kernel<K, O>, wm, pm, a, tiles, ranks);
}

template <int K, typename O>
cudaError_t launch(const galv_ctx* ctx, const CUtensorMap& wm, const CUtensorMap& xm, const CUtensorMap& pm, ProductArgs& a, cudaStream_t st)
{
    if (is_few(ctx, a)) return launch_few<K, O>(ctx, wm, pm, a, st);
    const int smem = smem_of(a.experts);
    const cudaError_t e = cudaFuncSetAttribute(expert_product_kernel<K, O>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_of(kExpertsMost));
    if (e != cudaSuccess) return e;
    a.what |= (uint32_t)(kTile >> 4) << 24;
    const long long most = (a.rows / 32 + (a.rows < a.experts ? a.rows : a.experts)) * a.tiles_m;      // units, whatever the ends say and their size is
    const int pairs = (int)(most < ctx->num_sms / 2 ? most : ctx->num_sms / 2);
    // Beside the kernel before it where that puts its tokens into 8-bit integers, or where one round of tiles is all there is: starting early is 2 us of 18 there.  Of many rounds it
    // gained nothing (a training step of 16 experts: 433 and 439 us).
    tc::Launch l((unsigned)pairs * 2, kThreads, smem, 0, a.in_front || most <= ctx->num_sms / 2, st);
    return cudaLaunchKernelEx(&l.cfg, expert_product_kernel<K, O>, wm, xm, pm, a);
}

bool units_fit(int64_t rows, int64_t experts, int64_t n) { return (rows / 32 + experts) * ((n + kTile - 1) / kTile) < (int64_t)1 << 31; }

// y = x w^T or x w by expert, both in 16 bits.  across: w [experts][cols of x][n], summed across its rows.
int product16(galv_ctx* ctx, const char* name, bool across, int64_t rows, int32_t experts, int64_t n, int64_t k, const int32_t* ends, const void* x, int64_t x_stride, const void* w,
              int64_t w_stride, const void* bias, void* y, int64_t y_stride, int32_t dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    const int64_t w_rows = across ? k : n, w_cols = across ? n : k;
    auto wrong = [&](int code, const char* what) {
        char text[160];
        snprintf(text, sizeof(text), "%s: %s", name, what);
        return galv_set_error(ctx, code, text);
    };
    if (!mx_size_ok(rows, n) || !mx_size_ok(rows, k) || experts < 1 || experts > kExpertsMost || (!ends && experts != 1) || (dtype != GALV_BF16 && dtype != GALV_F16) ||
        !units_fit(rows, experts, n))
        return wrong(GALV_ERR_INVALID_ARG, "sizes, number of experts or type outside the limits");
    if (rows == 0) return GALV_OK;
    if (!mx_matrix_ok(x, x_stride, k, dtype) || !mx_matrix_ok(w, w_stride, w_cols, dtype) || !mx_matrix_ok(y, y_stride, n, dtype) || (bias && !mx_aligned(bias, 2)) ||
        (ends && !mx_aligned(ends, 4)))
        return wrong(GALV_ERR_INVALID_ARG, "NULL or misaligned pointer, or a row stride below the row's length");
    const AlignPlan p = align_plan(rows, k, x, x_stride, experts, w_rows, w_cols, w, w_stride);
    if (p.total && (!workspace || !mx_aligned(workspace, 256) || workspace_bytes < p.total)) return wrong(GALV_ERR_WORKSPACE, "workspace NULL, misaligned or too small");
    const int may = mx_may_run(ctx, "experts' product: the library's host memory could not be registered", "experts' product: a bounded wait of an earlier product ran out");
    if (may != GALV_OK) return may;
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    cudaStream_t st = (cudaStream_t)stream;
    int64_t w_pitch = w_stride;
    if (p.x) {
        galv_align_rows(ctx, rows, k, x, x_stride, workspace, galv_aligned_pitch(k), st);
        x = workspace;
        x_stride = galv_aligned_pitch(k);
    }
    if (p.w) {
        void* const to = (char*)workspace + p.x;
        w_pitch = galv_aligned_pitch(w_cols);
        galv_align_rows(ctx, (int64_t)experts * w_rows, w_cols, w, w_stride, to, w_pitch, st);
        w = to;
    }
    const CUtensorMapDataType type = dtype == GALV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    CUtensorMap wm, xm = {}, pm;                          // xm is not read where there are few rows
    cudaError_t e = galv_map_3d(&wm, type, w, experts, w_rows, w_cols, w_pitch * 2, across ? 64 : kHalf, 64);
    if (e == cudaSuccess && rows > kFewRows) e = galv_mx_map(&xm, type, x, rows, k, x_stride * 2, kBox, 64, true);
    if (e == cudaSuccess) e = galv_mx_map(&pm, type, x, rows, k, x_stride * 2, kPart, 64, true);
    if (e != cudaSuccess) return wrong(GALV_ERR_CUDA, "tensor map");
    ProductArgs a;
    a.rows = rows; a.n = n; a.stride = y_stride; a.experts = experts; a.tiles_m = (int)((n + kTile - 1) / kTile);
    a.in_front = 0;
    a.chunks = (int)((k + 63) / 64); a.last_steps = (int)((k - (a.chunks - 1) * 64ll + 15) / 16);
    const uint32_t t = dtype == GALV_BF16 ? 1u : 0u;      // fp32 sums, both operands of this type, the weights' summed index along or across their rows
    a.what = 1u << 4 | t << 7 | t << 10 | (across ? 1u << 15 : 0u);
    a.ends = ends; a.x_scales = a.w_scales = nullptr; a.bias = bias; a.y = y; a.timeouts = ctx->mx_timeouts_at;
    a.vec = n % 8 == 0 && y_stride % 8 == 0 && mx_aligned(y, 16);
    if (dtype == GALV_BF16) e = across ? launch<kInputGrad, __nv_bfloat16>(ctx, wm, xm, pm, a, st) : launch<kForward, __nv_bfloat16>(ctx, wm, xm, pm, a, st);
    else e = across ? launch<kInputGrad, __half>(ctx, wm, xm, pm, a, st) : launch<kForward, __half>(ctx, wm, xm, pm, a, st);
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}

bool whole_sizes_ok(int64_t rows, int32_t experts, int64_t n, int64_t k, const int32_t* ends, int32_t dtype)
{
    return mx_size_ok(rows, n) && mx_size_ok(rows, k) && k <= GALV_I8_MOST && experts >= 1 && experts <= kExpertsMost && (ends || experts == 1) && mx_dtype_ok(dtype) &&
           units_fit(rows, experts, n);
}
bool whole_pointers_ok(int64_t n, const int32_t* ends, const int8_t* w_codes, const float* w_scales, const void* bias, const void* y, int64_t y_stride, int32_t dtype)
{
    return w_codes && w_scales && mx_aligned(w_codes, 16) && mx_aligned(w_scales, 4) && mx_matrix_ok(y, y_stride, n, dtype) && (!bias || mx_aligned(bias, mx_size_of(dtype))) &&
           (!ends || mx_aligned(ends, 4));
}

int whole_launch(galv_ctx* ctx, const char* name, int64_t rows, int32_t experts, int64_t n, int64_t k, const int32_t* ends, const int8_t* x_codes, int64_t x_pitch,
                 const float* x_scales, const int8_t* w_codes, const float* w_scales, const void* bias, void* y, int64_t y_stride, int32_t dtype, bool in_front, cudaStream_t st)
{
    CUtensorMap wm, xm = {}, pm;
    cudaError_t e = galv_map_3d(&wm, CU_TENSOR_MAP_DATA_TYPE_UINT8, w_codes, experts, n, k, i8_pitch(k), kHalf, kChunkBytes);
    if (e == cudaSuccess && rows > kFewRows) e = galv_mx_map(&xm, CU_TENSOR_MAP_DATA_TYPE_UINT8, x_codes, rows, k, x_pitch, kBox, kChunkBytes, true);
    if (e == cudaSuccess) e = galv_mx_map(&pm, CU_TENSOR_MAP_DATA_TYPE_UINT8, x_codes, rows, k, x_pitch, kPart, kChunkBytes, true);
    if (e != cudaSuccess) {
        char text[100];
        snprintf(text, sizeof(text), "%s: tensor map", name);
        return galv_set_error(ctx, GALV_ERR_CUDA, text);
    }
    ProductArgs a;
    a.rows = rows; a.n = n; a.stride = y_stride; a.experts = experts; a.tiles_m = (int)((n + kTile - 1) / kTile);
    a.in_front = in_front;
    a.chunks = (int)((k + kChunkBytes - 1) / kChunkBytes); a.last_steps = (int)((k - (a.chunks - 1) * (int64_t)kChunkBytes + 31) / 32);
    a.what = 2u << 4 | 1u << 7 | 1u << 10;      // 32-bit whole sums of signed 8-bit operands
    a.ends = ends; a.x_scales = x_scales; a.w_scales = w_scales; a.bias = bias; a.y = y; a.timeouts = ctx->mx_timeouts_at;
    const int per = 16 / mx_size_of(dtype);
    a.vec = n % per == 0 && y_stride % per == 0 && mx_aligned(y, 16);
    MX_DISPATCH_TYPE(dtype, e = (launch<kWhole, T>(ctx, wm, xm, pm, a, st)));
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}

int whole_may(galv_ctx* ctx) { return mx_may_run(ctx, "8-bit product: the library's host memory could not be registered", "8-bit product: a bounded wait of an earlier product ran out"); }

}  // namespace

extern "C" int64_t galv_expert_pitch(int64_t cols) { return mx_size_ok(0, cols) ? galv_aligned_pitch(cols) : 0; }

extern "C" size_t galv_expert_matmul_workspace_bytes(const galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, int64_t k, const void* x, int64_t x_stride, const void* w,
                                                     int64_t w_stride)
{
    if (!ctx || !mx_size_ok(rows, n) || !mx_size_ok(rows, k) || rows == 0 || experts < 1 || experts > kExpertsMost) return 0;
    return align_plan(rows, k, x, x_stride, experts, n, k, w, w_stride).total;
}

extern "C" int galv_expert_matmul(galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, int64_t k, const int32_t* ends, const void* x, int64_t x_stride, const void* w, int64_t w_stride,
                                  const void* bias, void* y, int64_t y_stride, int32_t dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    return product16(ctx, "galv_expert_matmul", false, rows, experts, n, k, ends, x, x_stride, w, w_stride, bias, y, y_stride, dtype, workspace, workspace_bytes, stream);
}

extern "C" size_t galv_expert_input_grad_workspace_bytes(const galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, int64_t k, const void* dy, int64_t dy_stride, const void* w,
                                                         int64_t w_stride)
{
    if (!ctx || !mx_size_ok(rows, n) || !mx_size_ok(rows, k) || rows == 0 || experts < 1 || experts > kExpertsMost) return 0;
    return align_plan(rows, n, dy, dy_stride, experts, n, k, w, w_stride).total;
}

extern "C" int galv_expert_input_grad(galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, int64_t k, const int32_t* ends, const void* dy, int64_t dy_stride, const void* w, int64_t w_stride,
                                      void* dx, int64_t dx_stride, int32_t dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    return product16(ctx, "galv_expert_input_grad", true, rows, experts, k, n, ends, dy, dy_stride, w, w_stride, nullptr, dx, dx_stride, dtype, workspace, workspace_bytes, stream);
}

extern "C" int galv_i8_matmul(galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, int64_t k, const int32_t* ends, const int8_t* x_codes, const float* x_scales, const int8_t* w_codes,
                              const float* w_scales, const void* bias, void* y, int64_t y_stride, int32_t dtype, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!whole_sizes_ok(rows, experts, n, k, ends, dtype)) return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_i8_matmul: sizes, number of experts or type outside the limits");
    if (rows == 0) return GALV_OK;
    if (!x_codes || !x_scales || !mx_aligned(x_codes, 16) || !mx_aligned(x_scales, 4) || !whole_pointers_ok(n, ends, w_codes, w_scales, bias, y, y_stride, dtype))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_i8_matmul: NULL or misaligned pointer, or a row stride below n");
    const int may = whole_may(ctx);
    if (may != GALV_OK) return may;
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    return whole_launch(ctx, "galv_i8_matmul", rows, experts, n, k, ends, x_codes, i8_pitch(k), x_scales, w_codes, w_scales, bias, y, y_stride, dtype, false, (cudaStream_t)stream);
}

extern "C" size_t galv_i8_linear_workspace_bytes(int64_t rows, int64_t k) { return mx_size_ok(rows, k) ? up((size_t)rows * i8_pitch_within(k)) + up((size_t)rows * 4) : 0; }

extern "C" int galv_i8_linear(galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, int64_t k, const int32_t* ends, const void* x, int64_t x_stride, const int8_t* w_codes,
                              const float* w_scales, const void* bias, void* y, int64_t y_stride, int32_t dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!whole_sizes_ok(rows, experts, n, k, ends, dtype)) return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_i8_linear: sizes, number of experts or type outside the limits");
    if (rows == 0) return GALV_OK;
    if (!mx_matrix_ok(x, x_stride, k, dtype) || !whole_pointers_ok(n, ends, w_codes, w_scales, bias, y, y_stride, dtype))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_i8_linear: NULL or misaligned pointer, or a row stride below the row's length");
    if (!workspace || !mx_aligned(workspace, 256) || workspace_bytes < galv_i8_linear_workspace_bytes(rows, k))
        return galv_set_error(ctx, GALV_ERR_WORKSPACE, "galv_i8_linear: workspace NULL, misaligned or too small");
    const int may = whole_may(ctx);
    if (may != GALV_OK) return may;
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    int8_t* const codes = (int8_t*)workspace;
    float* const scales = (float*)(codes + up((size_t)rows * i8_pitch_within(k)));
    const cudaError_t e = galv_i8_pack_launch(ctx->num_sms, rows, k, x, x_stride, dtype, codes, i8_pitch_within(k), scales, (cudaStream_t)stream);
    if (e != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
    return whole_launch(ctx, "galv_i8_linear", rows, experts, n, k, ends, codes, i8_pitch_within(k), scales, w_codes, w_scales, bias, y, y_stride, dtype, true, (cudaStream_t)stream);
}
