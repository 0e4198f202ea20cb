// Weight gradient of a layer whose input was kept in 8 bits: dw[n][k] = base[n][k] + sum_t dy[t][n] x[t][k].
//
// The sum runs over tokens, along which the blocks' powers of two change, so they cannot be taken out of it: the kept values are restored to
// dy's 16-bit type on their way to the tensor cores, exactly (4 significant bits and a power of two).  A pair of CTAs owns a tile of 256 x 256 of dw
// (tcgen05.mma over both, M = N = 256): each stages 128 columns of dy and restores 128 columns of x, so every restored value is used 256 times.
// Per CTA: two threads that start bulk tensor copies (64 tokens of dy; of codes and scales), twelve warps that restore (8 bits in, 16 bits out into
// the swizzled rows the tensor cores read), one thread that issues the matrix instructions for the pair, eight warps that take
// sums from the tensor memory while the next are made (two accumulators of 256 columns fill it) and move results out.
// Both operands lie with tokens along their rows ("MN-major"): dy and the codes are read as they are stored, nothing is transposed.
//
// 4096 tokens x 8192 x 8192 in bf16 take 412 to 500 us by the card's power state (1100 to 1335 TFLOP/s; a plain library product of 16-bit inputs 1590), in
// fp16, where restoring is four instructions for four elements in place of nine, 390 to 460.  The loop of matrix instructions alone runs at 1772 TFLOP/s; what
// is left is restored rows that come late (698 cycles a chunk for 512 of matrix instructions) and the power limit.
// Every value is restored once for each 256 columns of dy.  Restoring x to a matrix of its own first (2 bytes an element more) and multiplying that by the
// library is the faster way for large shapes: 4096 x 8192 x 32768 into bf16 1600 us sustained and 1900 here, 4096 x 8192 x 8192 412 and 483, 2048^3 21.5 and 22.5.

#include <atomic>
#include <type_traits>

#include "galv_mx.cuh"
#include "galv_tc.cuh"

namespace {

constexpr int kTokens = 64, kTile = 256, kHalf = kTile / 2;
// Rings of chunks of 64 tokens, each held only while it is needed: dy from its copy to its product, restored x from restoring to the product, codes and
// scales from their copy to restoring.  One ring of five chunks of all of them left the tensor cores waiting a third of the time.
constexpr int kDyRing = 5, kXRing = 5, kCodeRing = 5;
constexpr int kDyBytes = kTokens * kHalf * 2, kCodeBytes = kTokens * kHalf, kScaleBytes = kTokens * 16, kXBytes = kTokens * kHalf * 2;
constexpr int kOutBytes = 8 * 2048;                       // 32 x 16 sums of each warp that moves them out
constexpr int kSmem = 1024 + kDyRing * kDyBytes + kXRing * kXBytes + kCodeRing * (kCodeBytes + kScaleBytes) + kOutBytes + 512;
constexpr int kThreads = 768, kRestoreWarps = 4, kRestoreGroups = 3;      // warps: 4 for copies and matrix instructions, 8 for sums, three groups of 4 that restore
// Registers of a thread of each: 128 * 24 + 256 * 168 + 384 * 40 = 768 * 80, what the block is launched with.
constexpr int kRegsIssue = 24, kRegsSum = 168, kRegsRestore = 40;
// A tensor core's sum is cut at every addition: over 4096 tokens it is 1.6e-6 of the result off, over 1000 half of that (the error grows with the
// root of the length).  So after this many chunks (1024 tokens) the sum goes to fp32 registers, rounded additions.
constexpr int kSegment = 16;
constexpr int kGroup = 8;                                 // tiles along n whose columns of dy stay in L2 while their k runs (4 and 16 the same, 32 slower)

struct WgradArgs {
    long long tokens, n, k;
    int tiles_n, tiles_k, splits, chunks;
    const void* base;
    void* dw;
    float* partial;                                       // [splits][n][k], or NULL
    int vec;                                              // four results of a row can be moved at once
    unsigned* timeouts;                                   // host memory: CTAs that have given up a wait
};

struct Unit { int tn, tk, split, c0, c1; };
__device__ __forceinline__ Unit unit_of(const WgradArgs& a, int u)
{
    Unit w;
    const int tile = u / a.splits, per = kGroup * a.tiles_k, first = tile / per * kGroup;
    const int size = min(kGroup, a.tiles_n - first);
    w.split = u % a.splits;
    w.tn = first + tile % per % size;
    w.tk = tile % per / size;
    w.c0 = (int)((long long)w.split * a.chunks / a.splits);
    w.c1 = (int)((long long)(w.split + 1) * a.chunks / a.splits);
    return w;
}

// Four 8-bit elements times 2^(byte - 127) as two pairs of 16-bit numbers.  common: the shorter way holds for this byte.
template <typename T> struct Restore;
template <> struct Restore<__nv_bfloat16> {
    // An element's exponent and mantissa moved four bits down lie where a bf16 has its own: the value times 2^-120.  One product with 2^(120 + s)
    // restores it exactly (below bf16's normal numbers rounded once); from s = 8 on that factor leaves the type and two take its place.
    __device__ __forceinline__ static bool common(uint32_t byte) { return byte <= 134; }
    __device__ __forceinline__ static uint32_t factor(uint32_t byte) { return (byte + 120 << 7) * 0x10001u; }
    __device__ __forceinline__ static uint32_t mul(uint32_t a, uint32_t b)
    {
        uint32_t r;
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ __forceinline__ static void bits(uint32_t w, uint32_t& lo, uint32_t& hi)
    {
        const uint32_t top = (w & 0x80808080u) | (w >> 4 & 0x07070707u), low = w << 4 & 0xf0f0f0f0u;
        lo = __byte_perm(low, top, 0x5140);
        hi = __byte_perm(low, top, 0x7362);
    }
    __device__ __forceinline__ static void four(uint32_t w, uint32_t f, uint32_t& lo, uint32_t& hi)
    {
        bits(w, lo, hi);
        lo = mul(lo, f);
        hi = mul(hi, f);
    }
    __device__ __forceinline__ static void four_any(uint32_t w, uint32_t byte, uint32_t& lo, uint32_t& hi)
    {
        if (common(byte)) { four(w, factor(byte), lo, hi); return; }
        const uint32_t f = byte == 255 ? 0x7fc07fc0u : (byte << 7) * 0x10001u;
        bits(w, lo, hi);
        lo = mul(mul(lo, (247u << 7) * 0x10001u), f);
        hi = mul(mul(hi, (247u << 7) * 0x10001u), f);
    }
};
template <> struct Restore<__half> {
    // 2^s in fp16 where that and the largest element under it are normal numbers, else through fp32, saturating.
    __device__ __forceinline__ static bool common(uint32_t byte) { return byte >= 113 && byte <= 134; }
    __device__ __forceinline__ static uint32_t factor(uint32_t byte) { return (byte - 112 << 10) * 0x10001u; }
    __device__ __forceinline__ static void four(uint32_t w, uint32_t f, uint32_t& lo, uint32_t& hi)
    {
        uint32_t a, b;
        asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %2;\ncvt.rn.f16x2.e4m3x2 %0, l;\ncvt.rn.f16x2.e4m3x2 %1, h;\n}" : "=r"(a), "=r"(b) : "r"(w));
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(f));
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(f));
    }
    __device__ __forceinline__ static uint32_t clip(float a, float b)
    {
        const __half2 h = __floats2half2_rn(mx_held<__half>(a), mx_held<__half>(b));
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    __device__ __forceinline__ static void four_any(uint32_t w, uint32_t byte, uint32_t& lo, uint32_t& hi)
    {
        float v[4];
        const float s = mx_scale((int)byte);
        mx_from8(w, v);
        lo = clip(v[0] * s, v[1] * s);
        hi = clip(v[2] * s, v[3] * s);
    }
};

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

template <int N> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(N)); }
template <int N> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(N)); }

template <typename T, typename O>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
mx_wgrad_kernel(const __grid_constant__ CUtensorMap dy_map, const __grid_constant__ CUtensorMap code_map, const __grid_constant__ CUtensorMap scale_map,
                const __grid_constant__ WgradArgs a)
{
    extern __shared__ unsigned char raw[];
    const uint32_t base = (tc::smem_at(raw) + 1023) & ~1023u;
    const uint32_t dy_at = base, x_at = dy_at + kDyRing * kDyBytes, code_at = x_at + kXRing * kXBytes, scale_at = code_at + kCodeRing * kCodeBytes;
    const uint32_t out_at = scale_at + kCodeRing * kScaleBytes, bars = out_at + kOutBytes;
    const uint32_t dy_full = bars, dy_other = dy_full + 8 * kDyRing, dy_empty = dy_other + 8 * kDyRing, x_full = dy_empty + 8 * kDyRing, x_empty = x_full + 8 * kXRing,
                   code_full = x_empty + 8 * kXRing, code_empty = code_full + 8 * kCodeRing, acc_full = code_empty + 8 * kCodeRing, acc_empty = acc_full + 16, drain = acc_empty + 16,
                   slot = drain + 8;
    __shared__ int failed;

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = tc::cluster_rank();
    const int units = a.tiles_n * a.tiles_k * a.splits, first = blockIdx.x / 2, stride = gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kDyRing; ++s) {
            tc::bar_init(dy_full + 8 * s, 1);
            tc::bar_init(dy_other + 8 * s, 1);
            tc::bar_init(dy_empty + 8 * s, 1);
        }
        for (int s = 0; s < kXRing; ++s) {
            tc::bar_init(x_full + 8 * s, 2 * kRestoreWarps);
            tc::bar_init(x_empty + 8 * s, 1);
        }
        for (int s = 0; s < kCodeRing; ++s) {
            tc::bar_init(code_full + 8 * s, 1);
            tc::bar_init(code_empty + 8 * s, kRestoreWarps);
        }
        for (int b = 0; b < 2; ++b) {
            tc::bar_init(acc_full + 8 * b, 1);
            tc::bar_init(acc_empty + 8 * b, 16);
        }
        tc::bar_init(drain, 1);
        tc::bar_init_done();
        failed = 0;
        tc::prefetch_map(&dy_map);
        tc::prefetch_map(&code_map);
        tc::prefetch_map(&scale_map);
    }
    if (warp == 2) tc::tmem_alloc<2>(slot, 512);
    tc::fence_before();
    __syncthreads();
    tc::cluster_sync();                                   // the pair's barriers exist
    tc::fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(slot));

    // every wait is bounded; who gives up says so, the others run into their own bound
    auto waited = [&](uint32_t bar, uint32_t parity) {
        if (tc::bar_wait(bar, parity)) return true;
        *(volatile int*)&failed = 1;
        return false;
    };

    if (warp < 4) fewer_registers<kRegsIssue>();
    if (warp == 0) {                                      // copies of codes and scales
        if (tc::elect()) {
            int it = 0;
            bool ok = true;
            for (int u = first; u < units && ok; u += stride) {
                const Unit w = unit_of(a, u);
                const int k0 = w.tk * kTile + rank * kHalf;
                for (int c = w.c0; c < w.c1; ++c, ++it) {
                    const int s = it % kCodeRing;
                    if (!(ok = waited(code_empty + 8 * s, (it / kCodeRing & 1) ^ 1))) break;
                    tc::bar_expect(code_full + 8 * s, kCodeBytes + kScaleBytes);
                    tc::load_2d(code_at + s * kCodeBytes, &code_map, k0, c * kTokens, code_full + 8 * s);
                    tc::load_2d(scale_at + s * kScaleBytes, &scale_map, k0 / 32 & ~15, c * kTokens, code_full + 8 * s);
                }
            }
            if (*(volatile int*)&failed)                  // copies still in flight
                for (int i = it < kCodeRing ? 0 : it - kCodeRing; i < it; ++i) tc::bar_wait(code_full + 8 * (i % kCodeRing), i / kCodeRing & 1);
        }
    } else if (warp == 3) {                               // copies of dy
        if (tc::elect()) {
            int it = 0;
            bool ok = true;
            for (int u = first; u < units && ok; u += stride) {
                const Unit w = unit_of(a, u);
                const int n0 = w.tn * kTile + rank * kHalf;
                for (int c = w.c0; c < w.c1; ++c, ++it) {
                    const int s = it % kDyRing;
                    if (!(ok = waited(dy_empty + 8 * s, (it / kDyRing & 1) ^ 1))) break;
                    tc::bar_expect(dy_full + 8 * s, kDyBytes);
                    tc::load_2d(dy_at + s * kDyBytes, &dy_map, n0, c * kTokens, dy_full + 8 * s);
                    tc::load_2d(dy_at + s * kDyBytes + kDyBytes / 2, &dy_map, n0 + 64, c * kTokens, dy_full + 8 * s);
                }
            }
            if (*(volatile int*)&failed)
                for (int i = it < kDyRing ? 0 : it - kDyRing; i < it; ++i) tc::bar_wait(dy_full + 8 * (i % kDyRing), i / kDyRing & 1);
        }
    } else if (warp == 1 && rank == 1) {                  // tells the first CTA that this one's dy is there
        if (tc::elect()) {
            int it = 0;
            bool ok = true;
            for (int u = first; u < units && ok; u += stride) {
                const Unit w = unit_of(a, u);
                for (int c = w.c0; c < w.c1; ++c, ++it) {
                    const int s = it % kDyRing;
                    if (!(ok = waited(dy_full + 8 * s, it / kDyRing & 1))) break;
                    tc::bar_arrive_cluster(tc::in_cta(dy_other + 8 * s, 0));
                }
            }
        }
    } else if (warp == 1) {
        if (tc::elect()) {
            // fp32 sums, A and B of type T with the summed index across the rows, 256 x 256
            constexpr uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
            constexpr uint32_t what = 1u << 4 | type << 7 | type << 10 | 1u << 15 | 1u << 16 | (uint32_t)(kTile >> 3) << 17 | (uint32_t)(kTile >> 4) << 24;
            int it = 0, done = 0;
            bool ok = true;
            for (int u = first; u < units && ok; u += stride) {
                const Unit w = unit_of(a, u);
                for (int c = w.c0; c < w.c1 && ok; ++done) {
                    const uint32_t buf = done & 1, d = tmem + buf * 256;
                    const int end = min(c + kSegment, w.c1);
                    if (!(ok = waited(acc_empty + 8 * buf, (done / 2 & 1) ^ 1))) break;
                    tc::fence_after();
                    for (bool add = false; c < end; ++c, ++it, add = true) {
                        const int s = it % kDyRing, x = it % kXRing;
                        if (!(ok = waited(dy_full + 8 * s, it / kDyRing & 1) && waited(dy_other + 8 * s, it / kDyRing & 1) && waited(x_full + 8 * x, it / kXRing & 1))) break;
                        tc::fence_after();
#pragma unroll
                        for (int j = 0; j < kTokens / 16; ++j)
                            tc::mma_f16(d, tc::operand(dy_at + s * kDyBytes + j * 2048, 8192, 1024), tc::operand(x_at + x * kXBytes + j * 2048, 8192, 1024), what, add || j > 0);
                        tc::mma_commit<2>(dy_empty + 8 * s);
                        tc::mma_commit<2>(x_empty + 8 * x);
                    }
                    if (ok) tc::mma_commit<2>(acc_full + 8 * buf);
                }
            }
            if (*(volatile int*)&failed) {
                tc::mma_commit<2>(drain);
                tc::bar_wait(drain, 0);
            }
        }
    } else if (warp >= 4 && warp < 12) {
        more_registers<kRegsSum>();
        const int quad = warp % 4, half = (warp - 4) / 4;  // 32 rows, 128 columns
        const uint32_t mine = out_at + (warp - 4) * 2048, from = tmem + half * 128 + ((uint32_t)quad * 32 << 16);
        int done = 0;
        bool ok = true;
        for (int u = first; u < units && ok; u += stride) {
            const Unit w = unit_of(a, u);
            uint32_t buf = done & 1;
            if (w.c1 - w.c0 > kSegment) {                 // earlier segments are taken up here, the last one is added where it lies
                float sum[128];
#pragma unroll
                for (int i = 0; i < 128; ++i) sum[i] = 0.f;
                for (int c = w.c0; c < w.c1; c += kSegment) {
                    buf = done & 1;
                    if (!(ok = waited(acc_full + 8 * buf, done / 2 & 1))) break;
                    tc::fence_after();
#pragma unroll
                    for (int j = 0; j < 128; j += 16) {
                        uint32_t v[16];
                        tc::tmem_load16(from + buf * 256 + j, v);
                        tc::tmem_wait_load();
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[j + i] += __uint_as_float(v[i]);
                    }
                    if (c + kSegment < w.c1) {            // this accumulator may be summed into again
                        tc::fence_before();
                        __syncwarp();
                        if (lane == 0) tc::bar_arrive_cluster(tc::in_cta(acc_empty + 8 * buf, 0));
                        ++done;
                    }
                }
#pragma unroll
                for (int j = 0; j < 128; j += 16) tc::tmem_store16(from + buf * 256 + j, sum + j);
                tc::tmem_wait_store();
            } else if ((ok = waited(acc_full + 8 * buf, done / 2 & 1))) {
                tc::fence_after();
            }
            if (!ok) break;
            const long long r0 = (long long)w.tn * kTile + rank * kHalf + quad * 32, c0 = (long long)w.tk * kTile + half * 128;
            const int rows = (int)min(32ll, a.n - r0), cols = (int)min(128ll, a.k - c0);
            const long long at = (r0 + (a.vec ? lane / 4 : lane / 16)) * a.k + c0 + (a.vec ? lane % 4 * 4 : lane % 16);
            if (a.partial) move_out<float>(from + buf * 256, mine, nullptr, a.partial + (w.split * a.n * a.k + at), a.k, rows, cols, a.vec);
            else move_out<O>(from + buf * 256, mine, a.base ? (const O*)a.base + at : nullptr, (O*)a.dw + at, a.k, rows, cols, a.vec);
            tc::fence_before();
            __syncwarp();
            if (lane == 0) tc::bar_arrive_cluster(tc::in_cta(acc_empty + 8 * buf, 0));
            ++done;
        }
    } else if (warp >= 12) {
        fewer_registers<kRegsRestore>();
        // The groups of warps take chunks in turn.  A thread restores four pieces of 16 elements: columns c*16.. and (c+4)*16.. of rows r and r + 8.  Eight
        // lanes are eight rows: both the codes' and the restored rows' 16-byte pieces are exchanged by row % 8, so the eight meet all banks.
        const int t = threadIdx.x % 128, c = t % 32 / 8, r = t / 32 * 16 + t % 8, group = (warp - 12) / 4;
        int it = 0;
        bool ok = true;
        for (int u = first; u < units && ok; u += stride) {
            const Unit w = unit_of(a, u);
            const uint32_t scale_from = scale_at + r * 16 + (w.tk * kTile + rank * kHalf) / 32 % 16 + c / 2;
            for (int ch = w.c0; ch < w.c1; ++ch, ++it) {
                if (it % kRestoreGroups != group) continue;
                const int s = it % kCodeRing, x = it % kXRing;
                if (!(ok = waited(code_full + 8 * s, it / kCodeRing & 1) && waited(x_empty + 8 * x, (it / kXRing & 1) ^ 1))) break;
                uint32_t byte[2][2], from[2], to[2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) asm volatile("ld.shared.u8 %0, [%1];" : "=r"(byte[i][h]) : "r"(scale_from + s * kScaleBytes + i * 128 + h * 2));
#pragma unroll
                for (int h = 0; h < 2; ++h) {             // 64 columns a restored row
                    from[h] = code_at + s * kCodeBytes + r * 128 + ((c + 4 * h) ^ (r & 7)) * 16;
                    to[h] = x_at + x * kXBytes + h * 8192 + r * 128 + ((2 * c) ^ (r & 7)) * 16;
                }
                const bool common = Restore<T>::common(byte[0][0]) && Restore<T>::common(byte[0][1]) && Restore<T>::common(byte[1][0]) && Restore<T>::common(byte[1][1]);
                auto piece = [&](int i, int h, auto four) {
                    uint32_t q[4], o[8];
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]) : "r"(from[h] + i * 1024));
#pragma unroll
                    for (int j = 0; j < 4; ++j) four(q[j], o[2 * j], o[2 * j + 1]);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(to[h] + i * 1024), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"((to[h] ^ 16) + i * 1024), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]) : "memory");
                };
                if (__all_sync(0xffffffffu, common)) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t f = Restore<T>::factor(byte[i][h]);
                            piece(i, h, [f](uint32_t v, uint32_t& lo, uint32_t& hi) { Restore<T>::four(v, f, lo, hi); });
                        }
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t b = byte[i][h];
                            piece(i, h, [b](uint32_t v, uint32_t& lo, uint32_t& hi) { Restore<T>::four_any(v, b, lo, hi); });
                        }
                }
                tc::fence_async();
                __syncwarp();
                if (lane == 0) {
                    tc::bar_arrive(code_empty + 8 * s);
                    tc::bar_arrive_cluster(tc::in_cta(x_full + 8 * x, 0));
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

// dw = base + the splits' sums, in order.
template <typename O>
__global__ void __launch_bounds__(256) mx_wgrad_join_kernel(long long count, int splits, const float* __restrict__ partial, const O* base, O* dw)
{
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < count; e += (long long)gridDim.x * 256) {
        float v = partial[e];
        for (int s = 1; s < splits; ++s) v += partial[s * count + e];
        dw[e] = mx_round<O>(base ? mx_float(base[e]) + v : v);
    }
}

template <typename O>
__global__ void __launch_bounds__(256) mx_fill_kernel(long long count, const O* base, O* dw)
{
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < count; e += (long long)gridDim.x * 256) dw[e] = base ? base[e] : mx_round<O>(0.f);
}

// Rows that bulk copies cannot take (not on 16-byte boundaries) into rows that they can, zeros behind their ends.
__global__ void __launch_bounds__(256) mx_align_kernel(long long rows, int cols, const __half* __restrict__ x, long long stride, __half* __restrict__ out, long long pitch)
{
    for (long long r = blockIdx.x; r < rows; r += gridDim.x)
        for (unsigned c = threadIdx.x * 8; c < (unsigned)cols; c += 2048)             // may pass 2^31
            *reinterpret_cast<uint4*>(out + r * pitch + c) = mx_fetch8<__half, false>(x + r * stride, (int)c, cols).q[0];
}

struct WgradPlan { int tiles_n, tiles_k, splits, chunks, clusters; size_t aligned, partial, total; };

WgradPlan plan_of(const galv_ctx* ctx, int64_t tokens, int64_t n, int64_t k, const void* dy, int64_t dy_stride)
{
    WgradPlan p;
    const int most = ctx->num_sms / 2;
    p.tiles_n = (int)((n + kTile - 1) / kTile);
    p.tiles_k = (int)((k + kTile - 1) / kTile);
    p.chunks = (int)((tokens + kTokens - 1) / kTokens);
    const int64_t tiles = (int64_t)p.tiles_n * p.tiles_k;
    p.splits = 1;
    if (tiles < most && p.chunks >= 8) {
        p.splits = (int)(most / tiles);
        if (p.splits > p.chunks / 4) p.splits = p.chunks / 4;
    }
    const int64_t units = tiles * p.splits;
    p.clusters = (int)(units < most ? units : most);
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    p.aligned = mx_rows16(dy, dy_stride, GALV_BF16) && dy_stride * 2 < ((int64_t)1 << 40) ? 0 : up((size_t)tokens * ((n + 7) / 8 * 8) * 2);
    p.partial = p.splits > 1 ? up((size_t)p.splits * n * k * 4) : 0;
    p.total = p.aligned + p.partial;
    return p;
}

template <typename T, typename O>
cudaError_t launch(const galv_ctx* ctx, const WgradPlan& p, const CUtensorMap& dy, const CUtensorMap& codes, const CUtensorMap& scales, const WgradArgs& a, cudaStream_t st)
{
    // the registers that the kernel hands round are those it was built with: any other build would wait for what it never had
    static std::atomic<int> known{0};
    int regs = known.load(std::memory_order_relaxed);
    if (!regs) {
        cudaFuncAttributes f;
        const cudaError_t e = cudaFuncGetAttributes(&f, mx_wgrad_kernel<T, O>);
        if (e != cudaSuccess) return e;                   // of this call only: the next one asks again
        known.store(regs = f.numRegs, std::memory_order_relaxed);
    }
    if (regs * kThreads < 128 * kRegsIssue + 256 * kRegsSum + 128 * kRestoreGroups * kRegsRestore) return cudaErrorInvalidDeviceFunction;
    cudaError_t e = cudaFuncSetAttribute(mx_wgrad_kernel<T, O>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    mx_wgrad_kernel<T, O><<<p.clusters * 2, kThreads, kSmem, st>>>(dy, codes, scales, a);
    if (a.partial) mx_wgrad_join_kernel<O><<<ctx->num_sms * 8, 256, 0, st>>>(a.n * a.k, a.splits, a.partial, (const O*)a.base, (O*)a.dw);
    return cudaGetLastError();
}

}  // namespace

extern "C" size_t galv_mx_weight_grad_workspace_bytes(const galv_ctx* ctx, int64_t tokens, int64_t n, int64_t k, const void* dy, int64_t dy_stride)
{
    if (!ctx || !mx_size_ok(tokens, n) || !mx_size_ok(tokens, k) || tokens == 0) return 0;
    return plan_of(ctx, tokens, n, k, dy, dy_stride).total;
}

extern "C" int galv_mx_weight_grad(galv_ctx* ctx, int64_t tokens, int64_t n, int64_t k, const void* dy, int64_t dy_stride, int32_t dtype, const uint8_t* codes,
                                   const uint8_t* scales, const void* base, void* dw, int32_t dw_dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!mx_size_ok(tokens, n) || !mx_size_ok(tokens, k) || (dtype != GALV_BF16 && dtype != GALV_F16) || (dw_dtype != dtype && dw_dtype != GALV_F32))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_weight_grad: sizes or types outside the limits");
    if (!mx_matrix_ok(dw, k, k, dw_dtype) || (base && !mx_aligned(base, mx_size_of(dw_dtype))))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_weight_grad: NULL or misaligned dw or base");
    if (tokens > 0 && (!mx_matrix_ok(dy, dy_stride, n, dtype) || !codes || !scales || !mx_aligned(codes, 16) || !mx_aligned(scales, 16)))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_weight_grad: NULL or misaligned pointer, or a row stride below n");
    const size_t need = galv_mx_weight_grad_workspace_bytes(ctx, tokens, n, k, dy, dy_stride);
    if (need && (!workspace || !mx_aligned(workspace, 256) || workspace_bytes < need))
        return galv_set_error(ctx, GALV_ERR_WORKSPACE, "galv_mx_weight_grad: workspace NULL, misaligned or too small");
    const int may = mx_may_run(ctx, "galv_mx_weight_grad: the library's host memory could not be registered", "galv_mx_weight_grad: a bounded wait of an earlier microscaled product ran out");
    if (may != GALV_OK) return may;
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = cudaSuccess;
    if (tokens == 0) {
        if (dw != base) {
            if (dw_dtype == GALV_F32) mx_fill_kernel<float><<<ctx->num_sms * 8, 256, 0, st>>>(n * k, (const float*)base, (float*)dw);
            else mx_fill_kernel<__half><<<ctx->num_sms * 8, 256, 0, st>>>(n * k, (const __half*)base, (__half*)dw);
            e = cudaGetLastError();
        }
    } else {
        const WgradPlan p = plan_of(ctx, tokens, n, k, dy, dy_stride);
        const void* rows = dy;
        int64_t stride = dy_stride;
        if (p.aligned) {
            stride = (n + 7) / 8 * 8;
            mx_align_kernel<<<(int)(tokens < ctx->num_sms * 16 ? tokens : ctx->num_sms * 16), 256, 0, st>>>(tokens, (int)n, (const __half*)dy, dy_stride, (__half*)workspace, stride);
            rows = workspace;
        }
        CUtensorMap dm, cm, sm;
        const CUtensorMapDataType type = dtype == GALV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
        e = galv_mx_map(&dm, type, rows, tokens, n, stride * 2, kTokens, 64, true);
        if (e == cudaSuccess) e = galv_mx_map(&cm, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, tokens, mx_blocks(k) * 32, mx_blocks(k) * 32, kTokens, kHalf, true);
        if (e == cudaSuccess) e = galv_mx_map(&sm, CU_TENSOR_MAP_DATA_TYPE_UINT8, scales, tokens, mx_pitch8(k), mx_pitch8(k), kTokens, 16, false);
        if (e != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, "galv_mx_weight_grad: tensor map");
        WgradArgs a;
        a.tokens = tokens; a.n = n; a.k = k;
        a.tiles_n = p.tiles_n; a.tiles_k = p.tiles_k; a.splits = p.splits; a.chunks = p.chunks;
        a.base = base; a.dw = dw;
        a.timeouts = ctx->mx_timeouts_at;
        a.partial = p.partial ? reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + p.aligned) : nullptr;
        const int four = p.partial ? 16 : 4 * mx_size_of(dw_dtype);
        a.vec = k % 4 == 0 && (p.partial || (mx_aligned(dw, four) && mx_aligned(base, four)));
        if (dtype == GALV_BF16) e = dw_dtype == GALV_F32 ? launch<__nv_bfloat16, float>(ctx, p, dm, cm, sm, a, st) : launch<__nv_bfloat16, __nv_bfloat16>(ctx, p, dm, cm, sm, a, st);
        else e = dw_dtype == GALV_F32 ? launch<__half, float>(ctx, p, dm, cm, sm, a, st) : launch<__half, __half>(ctx, p, dm, cm, sm, a, st);
    }
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}
