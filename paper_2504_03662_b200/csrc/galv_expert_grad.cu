// Gradients of experts' weights and biases: dw[e][j][c] = base[e][j][c] + sum of dy[r][j] x[r][c], db[e][j] = sum of dy[r][j], over the rows r of expert e.
//
// As in the weight gradient of one layer a pair of CTAs owns a tile of 256 x 256 of dw and both operands lie with tokens along their rows, read as they are
// stored.  An expert's rows end anywhere: its last chunk of 64 holds rows of the next expert (or of none, which may be anything).  Of those the matrix
// instructions take no steps of 16 rows that are not needed, and what is left of the last step is set to zero in shared memory, in both operands, since
// zero times what lies there could be NaN.
// Per CTA: a thread that starts bulk tensor copies (both CTAs' tell the first one's barrier, those of a chunk with such rows their own), a warp that sets such rows to zero and then tells the
// first one's barrier, a thread (of the first) that issues the matrix instructions for the pair, eight warps that take sums from the tensor memory while the next are made and move results out.
//
// Bound by the loop of copies and matrix instructions: 8192 rows over 16 experts, 4096 x 2048 into bf16, take 126 us (1.1 PFLOP/s; the matrix instructions alone 79, with copies 99: shared
// memory and L2 have both at a time); 16384 rows over 8 experts, 2048 x 8192 onto an fp32 base, 468 us (1.17 PFLOP/s, 3.0 TB/s); 300 rows over 24 experts, 1365 x 2048 into fp16, 38.3 to 39.8 us,
// which is what the card writes (3.5 TB/s; zeros of this size go at 3.7).

#include "galv_experts.cuh"
#include "galv_tc.cuh"
#include "galv_tile_out.cuh"

namespace {

constexpr int kStages = 5, kTokens = 64, kTile = 256, kHalf = kTile / 2;
constexpr int kBox = kTokens * 128;                       // 64 rows of 64 columns
constexpr int kOperand = 2 * kBox, kStageBytes = 2 * kOperand;
constexpr int kOutBytes = 8 * 4096;                       // 32 rows of 128 bytes of each warp that moves results out
constexpr int kThreads = 384;
// A tensor core's sum is cut at every addition: 4.8e-7 of the result over 512 rows, 1.0e-6 over 1024 (the cuts go one way, so the error grows with the length).  So after this many chunks
// the sum goes to fp32 registers, rounded additions.  (Onto an fp32 base, 2048 rows an expert, 8192 x 2048: 460 us with 16 chunks, 472 with 12, 491 with 8.)
constexpr int kSegment = 12;
constexpr int kGroup = 8;                                 // tiles along n whose columns of dy stay in L2 while their k runs

struct GradArgs {
    long long rows, n, k;
    int experts, splits, tiles_n, tiles_k;                // splits: of each expert's rows, with a result of their own each
    uint32_t what;
    const int32_t* ends;
    const void* base;
    void* dw;
    int boxes;                                            // base and dw are moved by bulk copies
    unsigned* timeouts;
};

struct Unit { int part, tn, tk, row0, count; };           // part: expert * splits + split
__device__ __forceinline__ Unit unit_of(const GradArgs& a, const int* begin, int u)
{
    Unit w;
    const int each = a.tiles_n * a.tiles_k, tile = u % each, per = kGroup * a.tiles_k, first = tile / per * kGroup, size = min(kGroup, a.tiles_n - first);
    w.part = u / each;
    w.tn = first + tile % per % size;
    w.tk = tile % per / size;
    const int expert = w.part / a.splits, rows = begin[expert + 1] - begin[expert];
    const int len = a.splits == 1 ? rows : (int)((((unsigned)rows + a.splits - 1) / a.splits + kTokens - 1) / kTokens * kTokens), skip = (int)min((long long)(w.part % a.splits) * len, (long long)rows);
    w.row0 = begin[expert] + skip;
    w.count = min(len, rows - skip);
    return w;
}

// Zeros in the rows of an operand's last step that are not the expert's: `count` rows of the chunk are.
__device__ __forceinline__ void clear_rows(uint32_t at, int count)
{
    const int rows = (-count) & 15, lane = threadIdx.x % 32;      // up to the next step
    for (int i = lane; i < rows * 32; i += 32) {          // four boxes, 8 pieces of 16 bytes a row
        const int box = i / (rows * 8), piece = i % (rows * 8);
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" :: "r"(at + box * kBox + count * 128 + piece * 16), "r"(0) : "memory");
    }
}

// 16 bytes of results: sums, and what base has there
__device__ __forceinline__ uint4 four_words(const uint32_t* v, const uint4* base, float)
{
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
    if (base) {
        f[0] += __uint_as_float(base->x); f[1] += __uint_as_float(base->y); f[2] += __uint_as_float(base->z); f[3] += __uint_as_float(base->w);
    }
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <typename O>
__device__ __forceinline__ uint4 four_words(const uint32_t* v, const uint4* base, O)
{
    MxPiece<O> p;
    float f[8], b[8];
    if (base) {
        p.q[0] = *base;
        mx_floats(p, b);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = base ? b[i] + __uint_as_float(v[i]) : __uint_as_float(v[i]);
    return mx_piece<O>(f).q[0];
}

template <typename O>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
expert_grad_kernel(const __grid_constant__ CUtensorMap dy_map, const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap base_map,
                   const __grid_constant__ CUtensorMap dw_map, const __grid_constant__ GradArgs a)
{
    extern __shared__ unsigned char raw[];
    const uint32_t base = (tc::smem_at(raw) + 1023) & ~1023u;
    const uint32_t out_at = base + kStages * kStageBytes, bars = out_at + kOutBytes;
    const uint32_t full = bars, own = full + 8 * kStages, empty = own + 8 * kStages, acc_full = empty + 8 * kStages, acc_empty = acc_full + 16, drain = acc_empty + 16,
                   base_full = drain + 8, slot = base_full + 64;
    int* const begin = reinterpret_cast<int*>(raw + (bars + 256 - tc::smem_at(raw)));
    __shared__ int failed;

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = tc::cluster_rank();
    const int units = a.experts * a.splits * a.tiles_n * a.tiles_k, first = blockIdx.x / 2, stride = gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc::bar_init(full + 8 * s, 2);                // the producer twice, or what both CTAs' warps say that set rows to zero
            tc::bar_init(own + 8 * s, 1);
            tc::bar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            tc::bar_init(acc_full + 8 * b, 1);
            tc::bar_init(acc_empty + 8 * b, 16);
        }
        tc::bar_init(drain, 1);
        for (int b = 0; b < 8; ++b) tc::bar_init(base_full + 8 * b, 1);
        tc::bar_init_done();
        failed = 0;
        if (a.rows > 0) {                                 // else there are none
            tc::prefetch_map(&dy_map);
            tc::prefetch_map(&x_map);
        }
    }
    if (warp == 2) tc::tmem_alloc<2>(slot, 512);
    if (warp == 0) experts_begin(a.ends, a.experts, a.rows, begin);
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
    // Every lane waits and may read what is written; all go the same way, also where the limit ends between two lanes' tries: what follows takes whole warps.
    auto warp_waited = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, waited(bar, parity)) != 0; };

    if (warp == 0) {
        if (tc::elect()) {
            int it = 0;
            bool ok = true;
            for (int u = first; u < units && ok; u += stride) {
                const Unit w = unit_of(a, begin, u);
                const int n0 = w.tn * kTile + rank * kHalf, k0 = w.tk * kTile + rank * kHalf;
                for (int r = 0; r < w.count; r += kTokens, ++it) {
                    const int s = it % kStages;
                    if (!(ok = waited(empty + 8 * s, (it / kStages & 1) ^ 1))) break;
                    const bool ragged = w.count - r < kTokens && w.count % 16 != 0;
                    const uint32_t at = base + s * kStageBytes;
                    const int row = w.row0 + r;
                    if (ragged) {                         // zeros come in between: each CTA's own barrier
                        const uint32_t bar = own + 8 * s;
                        tc::bar_expect(bar, kStageBytes);
                        tc::load_2d(at, &dy_map, n0, row, bar);
                        tc::load_2d(at + kBox, &dy_map, n0 + 64, row, bar);
                        tc::load_2d(at + kOperand, &x_map, k0, row, bar);
                        tc::load_2d(at + kOperand + kBox, &x_map, k0 + 64, row, bar);
                    } else {
                        const uint32_t bar = tc::in_cta(full + 8 * s, 0);
                        if (rank == 0) {                  // both CTAs' copies
                            tc::bar_expect(full + 8 * s, 2 * kStageBytes);
                            tc::bar_arrive(full + 8 * s);
                        }
                        tc::load_2d_pair(at, &dy_map, n0, row, bar);
                        tc::load_2d_pair(at + kBox, &dy_map, n0 + 64, row, bar);
                        tc::load_2d_pair(at + kOperand, &x_map, k0, row, bar);
                        tc::load_2d_pair(at + kOperand + kBox, &x_map, k0 + 64, row, bar);
                    }
                }
            }
            if (*(volatile int*)&failed) tc::settle();
        }
    } else if (warp == 3) {                               // sets to zero what is not the expert's in the last step of its last chunk, and says so
        int it = 0;
        uint32_t turns = 0;                               // of each stage's barrier: bit s
        for (int u = first; u < units; u += stride) {
            const Unit w = unit_of(a, begin, u);
            const int chunks = (w.count + kTokens - 1) / kTokens, s = (it + chunks - 1) % kStages;
            it += chunks;
            if (w.count % 16 == 0) continue;
            if (!warp_waited(own + 8 * s, turns >> s & 1)) break;
            turns ^= 1u << s;
            clear_rows(base + s * kStageBytes, w.count - (chunks - 1) * kTokens);
            tc::fence_async();
            __syncwarp();
            if (lane == 0) tc::bar_arrive_cluster(tc::in_cta(full + 8 * s, 0));
        }
    } else if (warp == 1 && rank == 0) {
        if (tc::elect()) {
            int it = 0, done = 0;
            bool ok = true;
            for (int u = first; u < units && ok; u += stride) {
                const Unit w = unit_of(a, begin, u);
                for (int r = 0; r < w.count && ok; ++done) {
                    const uint32_t buf = done & 1, d = tmem + buf * kTile;
                    const int end = r + min(kSegment * kTokens, w.count - r);
                    if (!(ok = waited(acc_empty + 8 * buf, (done / 2 & 1) ^ 1))) break;
                    tc::fence_after();
                    for (bool add = false; r < end; r += kTokens, ++it, add = true) {
                        const int s = it % kStages, steps = min(kTokens / 16, (w.count - r + 15) / 16);
                        const uint32_t at = base + s * kStageBytes;
                        if (!(ok = waited(full + 8 * s, it / kStages & 1))) break;
                        tc::fence_after();
#pragma unroll
                        for (int j = 0; j < kTokens / 16; ++j)
                            if (j < steps) tc::mma_f16<2>(d, tc::operand(at + j * 2048, kBox, 1024), tc::operand(at + kOperand + j * 2048, kBox, 1024), a.what, add || j > 0);
                        tc::mma_commit<2>(empty + 8 * s);
                    }
                    if (ok) tc::mma_commit<2>(acc_full + 8 * buf);
                }
            }
            if (*(volatile int*)&failed) {
                tc::mma_commit<2>(drain);
                tc::bar_wait(drain, 0);
            }
        }
    } else if (warp >= 4) {
        constexpr int piece = 128 / (int)sizeof(O);        // columns of a copy
        const int quad = warp % 4, half = (warp - 4) / 4;  // 32 rows, 128 columns
        const uint32_t mine = out_at + (warp - 4) * 4096, from = tmem + half * 128 + ((uint32_t)quad * 32 << 16), base_bar = base_full + 8 * (warp - 4);
        int done = 0;
        uint32_t phase = 0;
        bool ok = true, fetched = false;
        auto release = [&](uint32_t acc) {                 // it may be summed into again
            tc::fence_before();
            __syncwarp();
            if (lane == 0) tc::bar_arrive_cluster(tc::in_cta(acc_empty + 8 * acc, 0));
        };
        for (int u = first; u < units && ok; u += stride) {
            const Unit w = unit_of(a, begin, u);
            const unsigned r0 = (unsigned)w.tn * kTile + rank * kHalf + quad * 32, c0 = (unsigned)w.tk * kTile + half * 128;      // may pass 2^31
            const bool some = r0 < a.n && c0 < a.k;
            auto fetch = [&](int c) {                      // base's piece, once the copy before has read this memory
                fetched = true;
                if (lane == 0) {
                    tc::stores_read();
                    tc::bar_expect(base_bar, 4096);
                    tc::load_3d(mine, &base_map, (int)c0 + c, (int)r0, w.part, base_bar);
                }
            };
            if (a.boxes && a.base && some) fetch(0);
            uint32_t acc = done & 1;
            if (w.count > kSegment * kTokens) {           // earlier segments are taken up here, the last one is added where it lies
                float sum[128];
#pragma unroll
                for (int i = 0; i < 128; ++i) sum[i] = 0.f;
                for (int left = w.count; left > 0; left -= kSegment * kTokens) {
                    acc = done & 1;
                    if (!(ok = warp_waited(acc_full + 8 * acc, done / 2 & 1))) break;
                    tc::fence_after();
#pragma unroll
                    for (int j = 0; j < 128; j += 16) {
                        uint32_t v[16];
                        tc::tmem_load16(from + acc * kTile + j, v);
                        tc::tmem_wait_load();
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[j + i] += __uint_as_float(v[i]);
                    }
                    if (left > kSegment * kTokens) {      // this accumulator may be summed into again
                        release(acc);
                        ++done;
                    }
                }
                if (!ok) break;
#pragma unroll
                for (int j = 0; j < 128; j += 16) tc::tmem_store16(from + acc * kTile + j, sum + j);
                tc::tmem_wait_store();
            } else if (w.count > 0) {
                if (!(ok = warp_waited(acc_full + 8 * acc, done / 2 & 1))) break;
                tc::fence_after();
            }
            const int rows = (int)max(-64ll, min(32ll, a.n - r0)), cols = (int)max(-128ll, min(128ll, a.k - c0));
            if (a.boxes) {
                if (some)
#pragma unroll 1
                    for (int c = 0; c < cols; c += piece) {
                        uint32_t v[piece];
                        if (a.base && c > 0) fetch(c);
                        if (w.count > 0) {
#pragma unroll
                            for (int i = 0; i < piece; i += 32) tc::tmem_load32(from + acc * kTile + c + i, v + i);
                            tc::tmem_wait_load();
                            if (c + piece >= cols) release(acc);
                        } else {
#pragma unroll
                            for (int i = 0; i < piece; ++i) v[i] = 0;
                        }
                        if (a.base) {
                            if (!(ok = warp_waited(base_bar, phase))) break;
                            phase ^= 1;
                            fetched = false;
                        } else {
                            if (lane == 0) tc::stores_read();
                            __syncwarp();
                        }
#pragma unroll
                        for (int q = 0; q < 8; ++q) {      // a lane has a row; its 16-byte pieces are exchanged by row % 8
                            const uint32_t at = mine + lane * 128 + ((q ^ (lane & 7)) * 16);
                            uint4 b;
                            if (a.base) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "r"(at));
                            const uint4 o = four_words(v + q * (16 / (int)sizeof(O)), a.base ? &b : nullptr, O());
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(at), "r"(o.x), "r"(o.y), "r"(o.z), "r"(o.w) : "memory");
                        }
                        tc::fence_async();
                        __syncwarp();
                        if (lane == 0) {
                            tc::store_3d(&dw_map, (int)c0 + c, (int)r0, w.part, mine);
                            tc::stores_end();
                        }
                    }
            } else {
                const long long at = w.part * a.n * a.k + r0 * a.k + c0;
                const O* const b = a.base ? (const O*)a.base + at : nullptr;
                if (sizeof(O) == 4 || !b) {
                    tile_out::move_out_odd<O>(from + acc * kTile, mine, b, (O*)a.dw + at, a.k, rows, cols, w.count > 0);
                } else {                                  // base is added before the rounding, a column a lane
                    const long long own = lane / 16 * a.k + lane % 16;
                    tile_out::move_out<O>(from + acc * kTile, mine, b + own, (O*)a.dw + at + own, a.k, rows, cols, false, w.count > 0);
                }
            }
            if (!ok) break;
            if (w.count > 0) {
                if (!a.boxes || !some) release(acc);
                ++done;
            }
        }
        if (fetched) tc::bar_wait(base_bar, phase);       // after a wait that ran out: a copy still in flight
        if (lane == 0) tc::stores_read();
    }
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    tc::cluster_sync();                                   // neither CTA's memory is read by the other any more
    if (threadIdx.x == 0 && failed) atomicAdd_system(a.timeouts, 1u);
    if (warp == 2) tc::tmem_free<2>(tmem, 512);
}

// dw = base + the splits' sums, in order.
template <typename O>
__global__ void __launch_bounds__(256) expert_grad_join_kernel(long long each, long long count, int splits, const float* __restrict__ partial, const O* base, O* dw)
{
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < count; i += (long long)gridDim.x * 256) {
        const float* const p = partial + (i / each * splits * each + i % each);
        float v = p[0];
        for (int s = 1; s < splits; ++s) v += p[s * each];
        dw[i] = mx_round<O>(base ? mx_float(base[i]) + v : v);
    }
}

// ---- bias
//
// A cluster of 8 CTAs has 128 columns of one expert, a warp every 64th of its rows, a lane 4 columns; the warps' sums are added in their order, then the
// CTAs'.  Bound by reading dy once.

constexpr int kBiasColumns = 128, kBiasCtas = 8;

template <typename T> __device__ __forceinline__ void add_row(const T* row, int cols, bool vec, float (&sum)[4])
{
    if (vec) {
        if (cols > 0) {
            const uint2 q = __ldg(reinterpret_cast<const uint2*>(row));
            const T* e = reinterpret_cast<const T*>(&q);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += mx_float(e[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < cols) sum[i] += mx_float(row[i]);
    }
}

template <typename T, typename O>
__global__ void __cluster_dims__(kBiasCtas, 1, 1) __launch_bounds__(256)
expert_bias_grad_kernel(long long rows, int experts, long long n, const int32_t* __restrict__ ends, const T* __restrict__ dy, long long stride, int vec, O* __restrict__ db)
{
    extern __shared__ int begin[];
    __shared__ float part[8][kBiasColumns], sums[kBiasCtas][kBiasColumns];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = tc::cluster_rank();
    if (warp == 0) experts_begin(ends, experts, rows, begin);
    tc::cluster_sync();                                   // the first CTA runs, sums can be sent to it
    const long long blocks = (n + kBiasColumns - 1) / kBiasColumns, all = blocks * experts;
    for (long long b = blockIdx.x / kBiasCtas; b < all; b += gridDim.x / kBiasCtas) {
        const int e = (int)(b / blocks);
        const long long c0 = (b - e * blocks) * kBiasColumns + lane * 4;
        const int cols = (int)max(0ll, min(4ll, n - c0));
        const long long end = begin[e + 1];
        float sum[4] = {};
#pragma unroll 4
        for (long long r = begin[e] + (long long)rank * 8 + warp; r < end; r += kBiasCtas * 8) add_row(dy + r * stride + c0, cols, vec, sum);
#pragma unroll
        for (int i = 0; i < 4; ++i) part[warp][lane * 4 + i] = sum[i];
        __syncthreads();
        if (threadIdx.x < kBiasColumns) {
            float v = part[0][threadIdx.x];
#pragma unroll
            for (int w = 1; w < 8; ++w) v += part[w][threadIdx.x];
            asm volatile("st.shared::cluster.f32 [%0], %1;" :: "r"(tc::in_cta(tc::smem_at(&sums[rank][threadIdx.x]), 0)), "f"(v) : "memory");
        }
        tc::cluster_sync();
        const long long c = (b - e * blocks) * kBiasColumns + threadIdx.x;
        if (rank == 0 && threadIdx.x < kBiasColumns && c < n) {
            float v = sums[0][threadIdx.x];
#pragma unroll
            for (int r = 1; r < kBiasCtas; ++r) v += sums[r][threadIdx.x];
            db[e * n + c] = mx_round<O>(v);
        }
        tc::cluster_sync();                               // the sums have been read
    }
}

size_t up(size_t x) { return (x + 255) & ~(size_t)255; }
int smem_of(int experts) { return 1024 + kStages * kStageBytes + kOutBytes + 256 + 4 * (experts + 1); }

struct GradPlan { size_t dy, x, partial, total; int splits; };
GradPlan plan_of(const galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, int64_t k, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride)
{
    auto moved = [&](const void* p, int64_t stride, int64_t cols) {
        return mx_rows16(p, stride, GALV_BF16) && stride * 2 < ((int64_t)1 << 40) ? 0 : up((size_t)rows * galv_aligned_pitch(cols) * 2);
    };
    GradPlan p;
    p.dy = moved(dy, dy_stride, n);
    p.x = moved(x, x_stride, k);
    // Fewer tiles than half of the pairs and long experts: each expert's rows are split, 256 a split or more (one expert of 16384 rows, 100 x 100: 158 us as one tile, 43 split in 16 and
    // joined; at 1700 rows an expert the second kernel costs what the splits give).
    const int64_t units = ((n + kTile - 1) / kTile) * ((k + kTile - 1) / kTile) * experts, pairs = ctx->num_sms / 2;
    p.splits = 1;
    if (units * 2 <= pairs && rows >= experts * (int64_t)2048) {
        const int64_t most = pairs / units, worth = rows / (experts * (int64_t)256);
        p.splits = (int)(most < worth ? most : worth);
        if (p.splits > 16) p.splits = 16;
    }
    p.partial = p.splits > 1 ? up((size_t)p.splits * experts * n * k * 4) : 0;
    p.total = p.dy + p.x + p.partial;
    return p;
}

template <typename O>
cudaError_t launch(const galv_ctx* ctx, const CUtensorMap& dm, const CUtensorMap& xm, CUtensorMapDataType type, GradArgs& a, cudaStream_t st)
{
    CUtensorMap bm = {}, wm = {};
    a.boxes = mx_rows16(a.dw, a.k, sizeof(O) == 4 ? GALV_F32 : GALV_BF16) && mx_aligned(a.base, 16);
    if (a.boxes) {
        cudaError_t e = galv_map_3d(&wm, type, a.dw, (int64_t)a.experts * a.splits, a.n, a.k, a.k * sizeof(O), 32, 128 / sizeof(O));
        if (e == cudaSuccess && a.base) e = galv_map_3d(&bm, type, a.base, a.experts, a.n, a.k, a.k * sizeof(O), 32, 128 / sizeof(O));
        if (e != cudaSuccess) return e;
    }
    const cudaError_t e = cudaFuncSetAttribute(expert_grad_kernel<O>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_of(kExpertsMost));
    if (e != cudaSuccess) return e;
    const long long units = (long long)a.experts * a.splits * a.tiles_n * a.tiles_k;
    const int pairs = (int)(units < ctx->num_sms / 2 ? units : ctx->num_sms / 2);
    expert_grad_kernel<O><<<pairs * 2, kThreads, smem_of(a.experts), st>>>(dm, xm, bm, wm, a);
    return cudaGetLastError();
}

bool sizes_ok(int64_t rows, int32_t experts, int64_t n, int64_t k, const int32_t* ends, int32_t dtype, int32_t out_dtype)
{
    return mx_size_ok(rows, n) && mx_size_ok(rows, k) && experts >= 1 && experts <= kExpertsMost && (ends || experts == 1) && (dtype == GALV_BF16 || dtype == GALV_F16) &&
           (out_dtype == dtype || out_dtype == GALV_F32) && ((n + kTile - 1) / kTile) * ((k + kTile - 1) / kTile) * experts < (int64_t)1 << 31;
}

}  // namespace

extern "C" size_t galv_expert_weight_grad_workspace_bytes(const galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, int64_t k, const void* dy, int64_t dy_stride, const void* x,
                                                          int64_t x_stride)
{
    if (!ctx || !mx_size_ok(rows, n) || !mx_size_ok(rows, k) || rows == 0 || experts < 1 || experts > kExpertsMost) return 0;
    return plan_of(ctx, rows, experts, n, k, dy, dy_stride, x, x_stride).total;
}

extern "C" int galv_expert_weight_grad(galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, int64_t k, const int32_t* ends, const void* dy, int64_t dy_stride, const void* x,
                                       int64_t x_stride, int32_t dtype, const void* base, void* dw, int32_t dw_dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!sizes_ok(rows, experts, n, k, ends, dtype, dw_dtype))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_expert_weight_grad: sizes, number of experts or types outside the limits");
    if (!mx_matrix_ok(dw, k, k, dw_dtype) || (base && !mx_aligned(base, mx_size_of(dw_dtype))) || (ends && !mx_aligned(ends, 4)))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_expert_weight_grad: NULL or misaligned dw, base or ends");
    if (rows > 0 && (!mx_matrix_ok(dy, dy_stride, n, dtype) || !mx_matrix_ok(x, x_stride, k, dtype)))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_expert_weight_grad: NULL or misaligned pointer, or a row stride below the row's length");
    const size_t need = galv_expert_weight_grad_workspace_bytes(ctx, rows, experts, n, k, dy, dy_stride, x, x_stride);
    if (need && (!workspace || !mx_aligned(workspace, 256) || workspace_bytes < need))
        return galv_set_error(ctx, GALV_ERR_WORKSPACE, "galv_expert_weight_grad: workspace NULL, misaligned or too small");
    const int may = mx_may_run(ctx, "galv_expert_weight_grad: the library's host memory could not be registered", "galv_expert_weight_grad: a bounded wait of an earlier product ran out");
    if (may != GALV_OK) return may;
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    cudaStream_t st = (cudaStream_t)stream;
    GradArgs a;
    a.rows = rows; a.n = n; a.k = k; a.experts = experts; a.splits = 1;
    a.tiles_n = (int)((n + kTile - 1) / kTile); a.tiles_k = (int)((k + kTile - 1) / kTile);
    const uint32_t t = dtype == GALV_BF16 ? 1u : 0u;      // fp32 sums, both operands of this type with the summed index across their rows, 256 x 256
    a.what = 1u << 4 | t << 7 | t << 10 | 1u << 15 | 1u << 16 | (uint32_t)(kTile >> 3) << 17 | (uint32_t)(kTile >> 4) << 24;
    a.ends = ends; a.base = base; a.dw = dw; a.timeouts = ctx->mx_timeouts_at;
    CUtensorMap dm = {}, xm = {};
    float* partial = nullptr;
    if (rows > 0) {
        const GradPlan p = plan_of(ctx, rows, experts, n, k, dy, dy_stride, x, x_stride);
        a.splits = p.splits;
        if (p.partial) partial = (float*)((char*)workspace + p.dy + p.x);
        if (p.dy) {
            galv_align_rows(ctx, rows, n, dy, dy_stride, workspace, galv_aligned_pitch(n), st);
            dy = workspace;
            dy_stride = galv_aligned_pitch(n);
        }
        if (p.x) {
            void* const to = (char*)workspace + p.dy;
            galv_align_rows(ctx, rows, k, x, x_stride, to, galv_aligned_pitch(k), st);
            x = to;
            x_stride = galv_aligned_pitch(k);
        }
        const CUtensorMapDataType type = dtype == GALV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
        cudaError_t e = galv_mx_map(&dm, type, dy, rows, n, dy_stride * 2, kTokens, 64, true);
        if (e == cudaSuccess) e = galv_mx_map(&xm, type, x, rows, k, x_stride * 2, kTokens, 64, true);
        if (e != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, "galv_expert_weight_grad: tensor map");
    }
    // without rows no copy is made: the maps are not read
    cudaError_t e;
    if (partial) {
        a.base = nullptr;
        a.dw = partial;
        e = launch<float>(ctx, dm, xm, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, a, st);
        if (e == cudaSuccess) {
            const int64_t count = experts * n * k, ctas = (count + 255) / 256, most = (int64_t)ctx->num_sms * 8;
            MX_DISPATCH_TYPE(dw_dtype, expert_grad_join_kernel<T><<<(int)(ctas < most ? ctas : most), 256, 0, st>>>(n * k, count, a.splits, partial, (const T*)base, (T*)dw));
            e = cudaGetLastError();
        }
    } else if (dw_dtype == GALV_F32) e = launch<float>(ctx, dm, xm, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, a, st);
    else if (dw_dtype == GALV_BF16) e = launch<__nv_bfloat16>(ctx, dm, xm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, a, st);
    else e = launch<__half>(ctx, dm, xm, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, a, st);
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}

extern "C" int galv_expert_bias_grad(galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, const int32_t* ends, const void* dy, int64_t dy_stride, int32_t dtype, void* db, int32_t db_dtype,
                                     void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!sizes_ok(rows, experts, n, 1, ends, dtype, db_dtype)) return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_expert_bias_grad: sizes, number of experts or types outside the limits");
    if (!db || !mx_aligned(db, mx_size_of(db_dtype)) || (ends && !mx_aligned(ends, 4)) || (rows > 0 && !mx_matrix_ok(dy, dy_stride, n, dtype)))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_expert_bias_grad: NULL or misaligned pointer, or a row stride below n");
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    const int64_t clusters = (n + kBiasColumns - 1) / kBiasColumns * experts, most = ctx->num_sms;
    const int grid = (int)(clusters < most ? clusters : most) * kBiasCtas, smem = 4 * (experts + 1);
    const int vec = n % 4 == 0 && dy_stride % 4 == 0 && mx_aligned(dy, 8);
    cudaStream_t st = (cudaStream_t)stream;
    using B = __nv_bfloat16;
    if (dtype == GALV_BF16 && db_dtype == GALV_F32) expert_bias_grad_kernel<B, float><<<grid, 256, smem, st>>>(rows, experts, n, ends, (const B*)dy, dy_stride, vec, (float*)db);
    else if (dtype == GALV_BF16) expert_bias_grad_kernel<B, B><<<grid, 256, smem, st>>>(rows, experts, n, ends, (const B*)dy, dy_stride, vec, (B*)db);
    else if (db_dtype == GALV_F32) expert_bias_grad_kernel<__half, float><<<grid, 256, smem, st>>>(rows, experts, n, ends, (const __half*)dy, dy_stride, vec, (float*)db);
    else expert_bias_grad_kernel<__half, __half><<<grid, 256, smem, st>>>(rows, experts, n, ends, (const __half*)dy, dy_stride, vec, (__half*)db);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}

namespace {

// What the three gradients need one after the other: dy in rows that bulk copies can take, read by all, and behind it what any of them needs for itself.
struct BackwardPlan { size_t dy, total; int64_t stride; };
BackwardPlan backward_plan(const galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, int64_t k, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const void* w,
                           int64_t w_stride)
{
    BackwardPlan p;
    p.dy = plan_of(ctx, rows, experts, n, k, dy, dy_stride, x, x_stride).dy;
    p.stride = p.dy ? galv_aligned_pitch(n) : dy_stride;
    const void* const at = p.dy ? nullptr : dy;           // moved rows lie on 256 bytes
    const size_t a = w ? galv_expert_input_grad_workspace_bytes(ctx, rows, experts, n, k, at, p.stride, w, w_stride) : 0;
    const size_t b = x ? galv_expert_weight_grad_workspace_bytes(ctx, rows, experts, n, k, at, p.stride, x, x_stride) : 0;
    p.total = p.dy + (a > b ? a : b);
    return p;
}

}  // namespace

extern "C" size_t galv_expert_backward_workspace_bytes(const galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, int64_t k, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride,
                                                       const void* w, int64_t w_stride)
{
    if (!ctx || !mx_size_ok(rows, n) || !mx_size_ok(rows, k) || rows == 0 || experts < 1 || experts > kExpertsMost) return 0;
    return backward_plan(ctx, rows, experts, n, k, dy, dy_stride, x, x_stride, w, w_stride).total;
}

extern "C" int galv_expert_backward(galv_ctx* ctx, int64_t rows, int32_t experts, int64_t n, int64_t k, const int32_t* ends, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride,
                                    const void* w, int64_t w_stride, int32_t dtype, void* dx, int64_t dx_stride, void* dw, void* db, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!sizes_ok(rows, experts, n, k, ends, dtype, dtype)) return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_expert_backward: sizes, number of experts or type outside the limits");
    if (rows > 0 && (!mx_matrix_ok(dy, dy_stride, n, dtype) || (dw && !x) || (dx && !w)))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_expert_backward: NULL or misaligned pointer, or a row stride below the row's length");
    char* ws = (char*)workspace;
    if (rows > 0) {
        const BackwardPlan p = backward_plan(ctx, rows, experts, n, k, dy, dy_stride, dw ? x : nullptr, x_stride, dx ? w : nullptr, w_stride);
        if (p.total && (!workspace || !mx_aligned(workspace, 256) || workspace_bytes < p.total))
            return galv_set_error(ctx, GALV_ERR_WORKSPACE, "galv_expert_backward: workspace NULL, misaligned or too small");
        if (p.dy) {
            MxDevice dev(ctx);
            if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
            galv_align_rows(ctx, rows, n, dy, dy_stride, workspace, p.stride, (cudaStream_t)stream);
            const cudaError_t e = cudaGetLastError();
            if (e != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
            dy = workspace;
            dy_stride = p.stride;
            ws += p.dy;
            workspace_bytes -= p.dy;
        }
    }
    int rc = GALV_OK;
    if (dx) rc = galv_expert_input_grad(ctx, rows, experts, n, k, ends, dy, dy_stride, w, w_stride, dx, dx_stride, dtype, ws, workspace_bytes, stream);
    if (rc == GALV_OK && dw) rc = galv_expert_weight_grad(ctx, rows, experts, n, k, ends, dy, dy_stride, x, x_stride, dtype, nullptr, dw, dtype, ws, workspace_bytes, stream);
    if (rc == GALV_OK && db) rc = galv_expert_bias_grad(ctx, rows, experts, n, ends, dy, dy_stride, dtype, db, dtype, stream);
    return rc;
}
