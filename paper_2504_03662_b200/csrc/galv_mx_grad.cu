// Gradients that read a layer's input where it was kept in 8 bits: activation functions and norms.

#include "galv_mx.cuh"
#include "galv_tc.cuh"

namespace {

__device__ __forceinline__ float exp2_fast(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }      // within 2^-22 of the value
__device__ __forceinline__ float inverse_fast(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }   // within 1 step
__device__ __forceinline__ float clamped(float x, float most)      // a NaN stays one
{
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(most));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(-most));
    return x;
}

// f'(x) of the activation functions, within 4e-7 (gelu_tanh 1e-6) of the largest slope: the pass has some twenty instructions an element at the memory's
// rate, and the exact functions take fifty.  From the bounds of x on, the slopes are 0 and 1 to 32 bits.
template <int ACT>
__device__ __forceinline__ float act_slope(float x)
{
    if (ACT == GALV_ACT_GELU) {
        // Phi(x) + x phi(x).  Abramowitz and Stegun 7.1.26: erfc(u) = t (a1 + t (a2 + t (a3 + t (a4 + t a5)))) exp(-u^2), t = 1 / (1 + p u), to 1.5e-7 for u >= 0;
        // with u = |x| / sqrt(2) the exponential is phi's.
        x = clamped(x, 30.f);
        const float e = exp2_fast(x * x * -0.72134752f);               // exp(-x^2 / 2)
        const float t = inverse_fast(fmaf(fabsf(x), 0.3275911f * 0.70710678f, 1.f));
        float q = fmaf(t, 1.061405429f, -1.453152027f);
        q = fmaf(t, q, 1.421413741f);
        q = fmaf(t, q, -0.284496736f);
        q = fmaf(t, q, 0.254829592f);
        q *= 0.5f * t * e;                                             // Phi(-|x|)
        return fmaf(x * 0.39894228f, e, x >= 0.f ? 1.f - q : q);
    } else if (ACT == GALV_ACT_GELU_TANH) {
        // (1 + tanh z) / 2 = 1 / (1 + exp(-2 z)) = s and its slope 2 z' exp(-2 z) s^2, without a difference of near numbers
        x = clamped(x, 10.f);
        const float x2 = x * x;
        const float e = exp2_fast(x * fmaf(x2, -2.f * 0.79788456f * 0.044715f * 1.44269504f, -2.f * 0.79788456f * 1.44269504f));
        const float s = inverse_fast(1.f + e);
        return fmaf(x * fmaf(x2, 6.f * 0.79788456f * 0.044715f, 2.f * 0.79788456f), e * s * s, s);
    } else {
        x = clamped(x, 80.f);
        const float e = exp2_fast(x * -1.44269504f), s = inverse_fast(1.f + e);
        return fmaf(x * e * s, s, s);
    }
}

// A held value is one of 256 elements under one of few powers of two, so a slope can be looked up: [32 scales][256 codes] of fp32 in shared memory, made by
// each CTA, which then stays for its share of the matrix.  Five instructions an element in place of twenty; scales outside the table (a block's
// largest below 448 * 2^-22 or above 448 * 2^9) are computed.
constexpr int kTableFirst = 127 - 22, kTableScales = 32, kTableBytes = kTableScales * 256 * 4;

template <typename T, int ACT, bool VEC, bool TABLE>
__global__ void __launch_bounds__(kMxThreads) mx_act_kernel(const MxSpread spread, unsigned rows, int cols, int nb, unsigned pieces, int per_row,
                                                            const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const T* dy,
                                                            long long dy_stride, T* dx, long long dx_stride)
{
    __shared__ __align__(16) T buf[VEC ? 1 : kMxThreads / 32][256 + 8];
    extern __shared__ float table[];
    if (TABLE) {
        float x[4];
        for (int e = threadIdx.x; e < kTableScales * 64; e += kMxThreads) {
            mx_from8((uint32_t)(e % 64) * 0x04040404u + 0x03020100u, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) table[e * 4 + i] = act_slope<ACT>(x[i] * mx_scale(kTableFirst + e / 64));
        }
        __syncthreads();
    }
    const uint32_t table_at = TABLE ? (uint32_t)__cvta_generic_to_shared(table) : 0;
    for (long long block = blockIdx.x; block < spread.blocks; block += gridDim.x) {
        const MxPlace at = mx_place(spread, block);
        constexpr int U = MxEach<T>::count;
        uint2 code[U];
        int byte[U];
        MxPiece<T> raw[U];
        const T* from = dy + at.row * dy_stride;
        const uint8_t* held = codes + ((long long)at.row * nb * 32 + at.c * 8ll);
        const uint8_t* power = scales + ((long long)at.row * per_row + (at.c >> 2));
#pragma unroll
        for (int h = 0; h < U; ++h) {
            const unsigned row = at.row + h * spread.dr, c = at.c + h * spread.dc;
            if (row < rows && c < pieces) {
                code[h] = __ldg(reinterpret_cast<const uint2*>(held));
                byte[h] = __ldg(power);
                raw[h] = mx_fetch8<T, VEC>(from, (int)c * 8, cols, spread.log >= 5 && dx != dy);      // in place, a neighbour may write meanwhile
            } else if (!VEC) {
                code[h] = make_uint2(0, 0);
                byte[h] = 0;
#pragma unroll
                for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[h].q[i] = make_uint4(0, 0, 0, 0);
            }
            from += spread.dr * dy_stride;
            held += (long long)spread.dr * nb * 32 + spread.dc * 8;
            power += (long long)spread.dr * per_row + spread.dc / 4;
        }
        T* to = dx + at.row * dx_stride;
#pragma unroll
        for (int h = 0; h < U; ++h, to += spread.dr * dx_stride) {
            const unsigned row = at.row + h * spread.dr, c = at.c + h * spread.dc;
            if (VEC && (row >= rows || c >= pieces)) continue;
            float x[8], g[8];
            mx_floats(raw[h], g);
            const int line = byte[h] - kTableFirst;
            if (TABLE && (unsigned)line < (unsigned)kTableScales) {
                const uint32_t from = table_at + line * 1024;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x[i]) : "r"(from + __byte_perm(i < 4 ? code[h].x : code[h].y, 0, 0x4440 + i % 4) * 4));
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] *= x[i];
            } else {
                mx_from8(code[h].x, x);
                mx_from8(code[h].y, x + 4);
                const float s = mx_scale(byte[h]);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] *= act_slope<ACT>(x[i] * s);
            }
            if (VEC) mx_store8<T, true>(to, (int)c * 8, cols, mx_piece<T>(g));
            else mx_store_spread<T>(buf[threadIdx.x / 32], to, c, row < rows, dx, dx_stride, spread, at, h, rows, cols, mx_piece<T>(g));
        }
    }
}

// ---- norms
//
// One pass: a row's codes and gradient are read once, its statistics and the two means of the gradient come from registers, and the column sums stay with
// the thread that has the column, over all rows that its CTA takes (where a thread has two pieces of 8 columns, dweight's in shared memory: with both sums in
// registers only half as many threads fit, and the pass took twice as long).  The next rows are on their way into shared memory
// meanwhile, each thread's pieces its own, so that only the rows' sums need a barrier.  2048 x 12288 in bf16 take 52.0 us for a layer norm and 41.5 for an
// rms norm (2.4 and 3.1 TB/s): 38 instructions an element at 59 % of the issue slots, the rest waits for shuffles, shared memory and the row's sums.

constexpr int kBlockThreads = 1024;
constexpr int kWarpColumns = 1024;                        // up to here a warp has a row to itself, and no barrier

struct NormArgs {
    long long rows, cols, nb, pitch, dy_stride, dx_stride;
    float eps;
    const uint8_t* codes;
    const uint8_t* scales;
    const void* dy;
    const void* weight;
    bool weight16;                                        // on a 16-byte boundary
    void* dx;
    float* part;                                          // [parts][2][cols]: dweight, dbias
    int ranks;                                            // CTAs of the one cluster that finishes dweight and dbias itself, or 0
    int share, span;                                      // SPLIT: CTAs of a cluster that share a row, pieces of it that each has (a multiple of 16)
    float* dweight;
    float* dbias;
};

template <typename T> struct Raw8 { uint4 q[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ float raw_at(const Raw8<T>& r, int i);
template <> __device__ __forceinline__ float raw_at<float>(const Raw8<float>& r, int i) { return __uint_as_float((&r.q[i / 4].x)[i % 4]); }
template <> __device__ __forceinline__ float raw_at<__nv_bfloat16>(const Raw8<__nv_bfloat16>& r, int i)
{
    const uint32_t w = (&r.q[0].x)[i / 2];
    return __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
}
template <> __device__ __forceinline__ float raw_at<__half>(const Raw8<__half>& r, int i)
{
    const uint32_t w = (&r.q[0].x)[i / 2];
    const __half2 h = *reinterpret_cast<const __half2*>(&w);
    return i % 2 ? __high2float(h) : __low2float(h);
}

template <int N> __device__ __forceinline__ void copy_async(uint32_t to, const void* from, int bytes)      // zeros behind `bytes`
{
    if (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to), "l"(from), "r"(bytes) : "memory");
    else if (N == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" :: "r"(to), "l"(from), "r"(bytes) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(to), "l"(from), "r"(bytes) : "memory");
}

// Sums of four values over a warp: each exchange halves the values a lane still has, so that lanes 8 g .. 8 g + 7 end with value g's.
__device__ __forceinline__ float warp_sums(const float4& v)
{
    const int lane = threadIdx.x % 32;
    float a = lane & 16 ? v.z : v.x, b = lane & 16 ? v.w : v.y;
    a += __shfl_xor_sync(0xffffffffu, lane & 16 ? v.x : v.z, 16);
    b += __shfl_xor_sync(0xffffffffu, lane & 16 ? v.y : v.w, 16);
    float c = lane & 8 ? b : a;
    c += __shfl_xor_sync(0xffffffffu, lane & 8 ? a : b, 8);
#pragma unroll
    for (int o = 4; o; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
    return c;
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Sums over the threads that share a row: a warp, a CTA (one barrier; `red` is another one in turn) or a cluster's CTAs (SPLIT: each warp's sums go to all of
// them).  SQUARES: x is the mean of the warp's values in every lane, w a sum of squares around it, z one of products with numbers whose sum is y.  x
// becomes the sum of all values, w and z those around the mean of all (the distances between the means, their squares times the values behind them and
// themselves times y, are added), so that mean and deviation take one barrier, not two (2048 x 12288 in fp32, shared by two CTAs: 104 us and 114; no
// difference within one CTA).  A product sum around zero, from which the mean's part came off afterwards, lost three digits where a row's values are nearly
// equal.  counts: values of each warp, and a 32nd of that (the warp's sum of x is 32 times x, exactly).
template <int W, bool SPLIT, bool SQUARES>
__device__ __forceinline__ float4 row_sums(const float4& v, float4* red, const float2* counts, float inv_n, int share, int rank)
{
    float c = warp_sums(v);
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, entries = (SPLIT ? share : 1) * (W / 32);
    if (W > 32) {
        float* to = reinterpret_cast<float*>(red + (SPLIT ? rank * (W / 32) : 0) + warp) + lane / 8;
        if (SPLIT) {
            if (lane % 8 < share) asm volatile("st.shared::cluster.f32 [%0], %1;" :: "r"(tc::in_cta(tc::smem_at(to), lane % 8)), "f"(c) : "memory");
            __syncwarp();
            tc::cluster_sync();
        } else {
            if (lane % 8 == 0) *to = c;
            __syncthreads();
        }
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int e = lane; e < entries; e += 32) {
            const float4 o = red[e];
            sum.x = SQUARES ? fmaf(o.x, counts[e].y, sum.x) : sum.x + o.x;
            sum.y += o.y;
            if (!SQUARES) sum.z += o.z;
        }
        c = warp_sums(sum);
    }
    float4 r;
    r.x = __shfl_sync(0xffffffffu, c, 0);
    r.y = __shfl_sync(0xffffffffu, c, 8);
    r.w = 0.f;
    if (W > 32 && SQUARES) {
        float products = 0.f;
        for (int e = lane; e < entries; e += 32) {
            const float4 o = red[e];
            const float apart = o.x * (1.f / 32.f) - r.x * inv_n;
            r.w += fmaf(apart * apart, counts[e].x, o.w);
            products += fmaf(apart, o.y, o.z);
        }
        float both = lane & 16 ? products : r.w;           // lanes 0 .. 15 end with the squares
        both += __shfl_xor_sync(0xffffffffu, lane & 16 ? r.w : products, 16);
#pragma unroll
        for (int o = 8; o; o >>= 1) both += __shfl_xor_sync(0xffffffffu, both, o);
        r.w = __shfl_sync(0xffffffffu, both, 0);
        r.z = __shfl_sync(0xffffffffu, both, 16);
    } else {
        r.z = __shfl_sync(0xffffffffu, c, 16);
        if (W == 32) r.w = __shfl_sync(0xffffffffu, c, 24);
    }
    return r;
}

constexpr int kMostShare = 4;                             // CTAs that share a row

template <typename T> struct NormStage {
    static constexpr int count = 2;
    static constexpr int piece = 8 * (int)sizeof(T) + 8 + 4;               // bytes: dy, codes, the word that has the scale byte
};

// W: threads that share a row (32: a warp, eight rows a CTA; else the CTA); PP: pieces of 8 columns a thread; SPLIT: the row is shared by a cluster's CTAs.
template <typename T, bool LAYER, bool VEC, int W, int PP, bool SPLIT>
__global__ void __launch_bounds__(W == 32 ? 256 : W, W == 32 ? (PP < 4 ? 2 : 1) : W <= 256 ? 4 : W <= 512 ? 2 : 1) mx_norm_kernel(const __grid_constant__ NormArgs a)
{
    constexpr bool WARP = W == 32;
    constexpr int NS = NormStage<T>::count, kDy = 8 * (int)sizeof(T);
    extern __shared__ __align__(16) unsigned char raw[];
    constexpr bool kShared = !WARP && PP > 1;             // dweight's sums lie in shared memory
    constexpr int kEntries = W / 32 * (SPLIT ? kMostShare : 1);
    __shared__ float4 red[2][kEntries];
    __shared__ float2 counts[kEntries];
    constexpr int teams = WARP ? 8 : 1, width = W, slots = W * PP;
    const int team = WARP ? threadIdx.x / 32 : 0, lane = WARP ? threadIdx.x % 32 : threadIdx.x;
    const int share = SPLIT ? a.share : 1, rank = SPLIT ? (int)tc::cluster_rank() : 0, lead = SPLIT ? rank * a.span * 8 : 0;      // lead: this CTA's first column
    const int cols = SPLIT ? max(0, min((int)a.cols - lead, a.span * 8)) : (int)a.cols, pieces = (cols + 7) / 8;
    const T* weight = (const T*)a.weight + lead;
    const float inv_n = 1.f / (float)a.cols;
    // weights [slots][8], then each team's stages of dy [slots][8], codes [slots][8 bytes], scale words [slots], then sums [2][slots][4]
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(raw), mine = base + slots * kDy + team * NS * slots * NormStage<T>::piece;
    const uint32_t sums = mine + NS * slots * NormStage<T>::piece;
    // rows off 16-byte boundaries are not staged: the first stage's place of dy is where a warp's results are put together
    T* const buf = reinterpret_cast<T*>(raw + (mine - base) + (WARP ? 0 : (threadIdx.x & ~31) * kDy));
    for (int c = threadIdx.x * 8; c < slots * 8; c += (WARP ? 256 : W) * 8) {
        MxPiece<T> piece;
        if (a.weight && c < cols) {
            piece = a.weight16 ? mx_fetch8<T, true>(weight, c, cols) : mx_fetch8<T, false>(weight, c, cols);
        } else {
            const float ones[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
            piece = mx_piece<T>(ones);
        }
#pragma unroll
        for (int i = 0; i < kDy / 16; ++i) *reinterpret_cast<uint4*>(raw + c * (int)sizeof(T) + i * 16) = piece.q[i];
    }
    // pieces behind the row's end stay zeros
    for (int e = lane; e < NS * slots * NormStage<T>::piece / 4; e += W) asm volatile("st.shared.b32 [%0], %1;" :: "r"(mine + e * 4), "r"(0) : "memory");
    if (LAYER && !WARP && threadIdx.x < share * (W / 32)) {
        const int r = threadIdx.x / (W / 32), w = threadIdx.x % (W / 32), there = SPLIT ? max(0, min((int)a.cols - r * a.span * 8, a.span * 8)) : cols;
        int n = 0;
#pragma unroll
        for (int p = 0; p < PP; ++p) n += max(0, min(256, there - (w * 32 + p * width) * 8));
        counts[threadIdx.x] = make_float2((float)n, (float)n * (1.f / 32.f));
    }
    if (SPLIT) tc::cluster_sync();
    else __syncthreads();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const float mine_n = LAYER && !WARP ? counts[rank * (W / 32) + threadIdx.x / 32].x : 0.f, inv_warp = WARP ? inv_n : mine_n > 0.f ? 1.f / mine_n : 0.f;

    float dw[kShared ? 8 : PP * 8] = {}, db[LAYER ? PP * 8 : 1] = {};
    auto sums_load = [&](int p) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(dw[4 * i]), "=f"(dw[4 * i + 1]), "=f"(dw[4 * i + 2]), "=f"(dw[4 * i + 3]) : "r"(sums + (i * slots + lane + p * width) * 16));
    };
    auto sums_store = [&](int p) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" :: "r"(sums + (i * slots + lane + p * width) * 16), "f"(dw[4 * i]), "f"(dw[4 * i + 1]), "f"(dw[4 * i + 2]), "f"(dw[4 * i + 3]) : "memory");
    };
    if (kShared) {
#pragma unroll
        for (int p = 0; p < PP; ++p) sums_store(p);
    }
    const long long first = (long long)(blockIdx.x / share) * teams + team, step = (long long)(gridDim.x / share) * teams;
    const uint8_t* codes = a.codes + first * a.nb * 32 + lead + lane * 8;
    const uint8_t* scales = a.scales + first * a.pitch + lead / 32;
    const T* dy = (const T*)a.dy + first * a.dy_stride + lead + lane * 8;
    T* dx = (T*)a.dx + first * a.dx_stride + lead;
    long long ahead = first;
    auto fetch = [&](int stage) {
        if (ahead < a.rows) {
            const uint32_t to = mine + stage * slots * NormStage<T>::piece;
#pragma unroll
            for (int p = 0; p < PP; ++p) {
                const int at = lane + p * width;
                if (at < pieces) {
                    if (VEC) {
                        const int left = (cols - at * 8) * (int)sizeof(T);
                        copy_async<16>(to + at * kDy, dy + p * width * 8, min(16, left));
                        if (kDy == 32) copy_async<16>(to + at * kDy + 16, left > 16 ? dy + p * width * 8 + 4 : dy, min(16, max(0, left - 16)));
                    }
                    copy_async<8>(to + slots * kDy + at * 8, codes + p * width * 8, 8);
                    copy_async<4>(to + slots * (kDy + 8) + at * 4, scales + (at >> 4) * 4, 4);
                }
            }
            ahead += step;
            codes += step * a.nb * 32;
            scales += step * a.pitch;
            dy += step * a.dy_stride;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int n = 0; n < NS - 1; ++n) fetch(n);
    int turn = 0, stage = 0;
    for (long long row = first; row < a.rows; row += step, turn ^= 1, dx += step * a.dx_stride) {
        fetch((stage + NS - 1) % NS);
        asm volatile("cp.async.wait_group %0;" :: "n"(NS - 1) : "memory");
        const uint32_t from = mine + stage * slots * NormStage<T>::piece;
        stage = (stage + 1) % NS;
        float x[PP * 8], s[PP];
        Raw8<T> d[PP];
        auto weights = [&](int p) {
            Raw8<T> w;
#pragma unroll
            for (int i = 0; i < kDy / 16; ++i)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.q[i].x), "=r"(w.q[i].y), "=r"(w.q[i].z), "=r"(w.q[i].w) : "r"(base + (lane + p * width) * kDy + i * 16));
            return w;
        };
        // RMS: x is the sum of squares, z that of dy * weight * x.  LAYER: x is the warp's mean, w and z the sums of squares and of dy * weight * x around it,
        // y that of dy * weight.
        float4 m = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int p = 0; p < PP; ++p) {
            const int at = lane + p * width;
            uint2 code;
            uint32_t word;
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(code.x), "=r"(code.y) : "r"(from + slots * kDy + at * 8));
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(word) : "r"(from + slots * (kDy + 8) + at * 4));
            if (VEC) {
#pragma unroll
                for (int i = 0; i < kDy / 16; ++i)
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(d[p].q[i].x), "=r"(d[p].q[i].y), "=r"(d[p].q[i].z), "=r"(d[p].q[i].w) : "r"(from + at * kDy + i * 16));
            } else {
                const MxPiece<T> piece = mx_fetch8<T, false>((const T*)a.dy + row * a.dy_stride + lead, at * 8, cols);
#pragma unroll
                for (int i = 0; i < kDy / 16; ++i) d[p].q[i] = piece.q[i];
            }
            mx_from8(code.x, x + 8 * p);
            mx_from8(code.y, x + 8 * p + 4);
            s[p] = mx_scale((int)(word >> (at >> 2 & 3) * 8 & 255));
            float sx = 0.f, sgx = 0.f;                    // before the block's power of two
            if (LAYER) {
#pragma unroll
                for (int i = 0; i < 8; ++i) sx += x[8 * p + i];
                m.x = fmaf(sx, s[p], m.x);
            } else {
                const Raw8<T> w = weights(p);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float v = x[8 * p + i];
                    sx = fmaf(v, v, sx);
                    sgx = fmaf(raw_at<T>(d[p], i) * raw_at<T>(w, i), v, sgx);
                }
                m.x = fmaf(sx * s[p], s[p], m.x);
                m.z = fmaf(sgx, s[p], m.z);
            }
        }
        float near = 0.f;
        if (LAYER) {                                      // the values around the warp's mean
            m.x = near = warp_sum(m.x) * inv_warp;
#pragma unroll
            for (int p = 0; p < PP; ++p) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[8 * p + i] = fmaf(x[8 * p + i], s[p], -near);
                const int left = cols - (lane + p * width) * 8;
                if (left < 8) {                           // behind the row's end
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i >= left) x[8 * p + i] = 0.f;
                }
                const Raw8<T> w = weights(p);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float v = x[8 * p + i], gw = raw_at<T>(d[p], i) * raw_at<T>(w, i);
                    m.w = fmaf(v, v, m.w);
                    m.y += gw;
                    m.z = fmaf(gw, v, m.z);
                }
            }
        }
        m = row_sums<W, SPLIT, LAYER>(m, red[turn], counts, inv_n, share, rank);
        const float sgx = m.z;
        float sq = m.x, mg = 0.f, shift = 0.f;
        if (LAYER) {
            const float mean = WARP ? near : m.x * inv_n;
            mg = m.y * inv_n;
            sq = m.w;
            shift = mean - near;
        }
        const float r = 1.f / sqrtf(sq * inv_n + a.eps), c = -sgx * inv_n * r * r * r, mr = -mg * r;
#pragma unroll
        for (int p = 0; p < PP; ++p) {
            const Raw8<T> w = weights(p);
            float v[8];
            if (kShared) sums_load(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = raw_at<T>(d[p], i), yr = y * r, xv = !LAYER ? x[8 * p + i] * s[p] : WARP ? x[8 * p + i] : x[8 * p + i] - shift;
                v[i] = fmaf(yr, raw_at<T>(w, i), LAYER ? fmaf(c, xv, mr) : c * xv);
                float& sum = dw[kShared ? i : 8 * p + i];
                sum = fmaf(yr, xv, sum);
                if (LAYER) db[8 * p + i] += y;
            }
            if (kShared) sums_store(p);
            if (VEC) {
                mx_store8<T, true>(dx, (lane + p * width) * 8, cols, mx_piece<T>(v));
            } else {
                const int c = ((lane & ~31) + p * width) * 8;
                mx_scatter_run<T>(buf, dx + c, cols - c, mx_piece<T>(v));
            }
        }
    }
    // this CTA's column sums
    const int pitch = SPLIT ? (int)((a.cols + 7) / 8 * 8) : pieces * 8;
    float* part = a.part + (long long)(blockIdx.x / share) * 2 * pitch + lead;
    float* joined = reinterpret_cast<float*>(raw);        // over what is not read any more: [2][apart] (a warp a row: [team][2][apart])
    const int apart = WARP ? slots * 8 : pitch;
    if (WARP || a.ranks) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
    }
    if (WARP) {
#pragma unroll
        for (int p = 0; p < PP; ++p)
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                float* to = joined + team * 2 * apart + (lane + p * 32) * 8 + i;
                const int k = 8 * p + i;
                *reinterpret_cast<float4*>(to) = make_float4(dw[k], dw[k + 1], dw[k + 2], dw[k + 3]);
                if (LAYER) *reinterpret_cast<float4*>(to + apart) = make_float4(db[k], db[k + 1], db[k + 2], db[k + 3]);
            }
        __syncthreads();
        for (int c = threadIdx.x; c < (LAYER ? 2 : 1) * apart; c += 256) {      // the warps' in order
            float sum = joined[c];
#pragma unroll
            for (int t = 1; t < 8; ++t) sum += joined[t * 2 * apart + c];
            if (a.ranks) joined[c] = sum;
            else if (c % apart < pitch) part[c / apart * pitch + c % apart] = sum;
        }
    } else {
        float* to = a.ranks ? joined : part;
#pragma unroll
        for (int p = 0; p < PP; ++p) {
            const int at = lane + p * width;
            if (at >= pieces) continue;
            if (kShared) sums_load(p);
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const int k = (kShared ? 0 : 8 * p) + i;
                *reinterpret_cast<float4*>(to + at * 8 + i) = make_float4(dw[k], dw[k + 1], dw[k + 2], dw[k + 3]);
                if (LAYER) *reinterpret_cast<float4*>(to + pitch + at * 8 + i) = make_float4(db[8 * p + i], db[8 * p + i + 1], db[8 * p + i + 2], db[8 * p + i + 3]);
            }
        }
    }
    if (a.ranks) {                                        // few rows: the grid is one cluster, each CTA adds its share of the columns, the CTAs' sums in order
        __syncwarp();
        tc::cluster_sync();
        for (int e = blockIdx.x * blockDim.x + threadIdx.x; e < (LAYER ? 2 : 1) * cols; e += a.ranks * blockDim.x) {
            const int c = e < cols ? e : e - cols;
            const uint32_t at = base + ((e < cols ? 0 : apart) + c) * 4;
            float sum = 0.f;
            for (int r = 0; r < a.ranks; ++r) {
                float v;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(tc::in_cta(at, r)) : "memory");
                sum = r ? sum + v : v;
            }
            float* out = e < cols ? a.dweight : a.dbias;
            if (out) out[c] = sum;
        }
        __syncwarp();
        tc::cluster_sync();                               // no CTA leaves while its sums are read
    }
}

// dweight and dbias: the CTAs' sums in a fixed order, 32 columns a CTA, 32 threads a column that take every 32nd.  It is launched while the kernel before it
// still runs (once each of that one's CTAs has allowed it or ended), and waits for that one's end: about 1 us less
// (16384 x 512: 16.1 us, 16.9 one after the other).  The sums are written while this kernel runs, so they are read by plain loads that stay behind the
// wait: neither the read-only path nor a compiler that may move them is for such data.
__device__ __forceinline__ float load_behind(const float* p)
{
    float v;
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p) : "memory");
    return v;
}
__global__ void __launch_bounds__(1024) mx_norm_join_kernel(long long cols, long long pitch, int parts, const float* part, float* dweight, float* dbias)
{
    __shared__ float sum[32][33];
    const int x = threadIdx.x % 32, k = threadIdx.x / 32, which = blockIdx.y;
    const long long c = (long long)blockIdx.x * 32 + x;
    float v = 0.f;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (c < cols) {
#pragma unroll 4
        for (int p = k; p < parts; p += 32) v += load_behind(part + (((long long)p * 2 + which) * pitch + c));
    }
    sum[k][x] = v;
    __syncthreads();
    v = sum[x][k];                                        // now a warp has a column
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    float* out = which ? dbias : dweight;
    const long long mine = (long long)blockIdx.x * 32 + k;
    if (x == 0 && mine < cols && out) out[mine] = v;
}

__device__ __forceinline__ float block_sum(float v, float* red)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    float s = 0.f;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) s += red[w];
    return s;
}

// Rows too long for a cluster's registers: a CTA goes over its row four times (the first reads it, the others find it in the caches).  Mean and 1/sqrt(var + eps) stay for
// the column sums, which come first where dx may be dy: this kernel runs without dx before them and with it after them.
template <typename T, bool LAYER, bool VEC>
__global__ void __launch_bounds__(512) mx_norm_wide_kernel(const NormArgs a, float2* stats, bool last)
{
    __shared__ float red[16];
    const long long pieces = (a.cols + 7) / 8;
    const float inv_n = 1.f / (float)a.cols;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* dy = (const T*)a.dy + row * a.dy_stride;
        T* dx = (T*)a.dx + row * a.dx_stride;
        float x[8], g[8], w[8];
        if (!last) {
            float mean = 0.f, s = 0.f;
            if (LAYER) {
                for (long long c = threadIdx.x; c < pieces; c += 512) {
                    mx_restore8(a.codes, a.scales, row, (int)c, a.nb, a.pitch, x);
#pragma unroll
                    for (int i = 0; i < 8; ++i) s += x[i];
                }
                mean = block_sum(s, red) * inv_n;
            }
            s = 0.f;
            for (long long c = threadIdx.x; c < pieces; c += 512) {
                mx_restore8(a.codes, a.scales, row, (int)c, a.nb, a.pitch, x);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c * 8 + i < a.cols) s = fmaf(x[i] - mean, x[i] - mean, s);
            }
            const float rstd = 1.f / sqrtf(block_sum(s, red) * inv_n + a.eps);
            if (threadIdx.x == 0) stats[row] = make_float2(mean, rstd);
            continue;
        }
        const float mean = stats[row].x, rstd = stats[row].y;
        float sg = 0.f, sgx = 0.f;
        for (long long c = threadIdx.x; c < pieces; c += 512) {
            mx_restore8(a.codes, a.scales, row, (int)c, a.nb, a.pitch, x);
            mx_floats(mx_fetch8<T, VEC>(dy, (int)c * 8, (int)a.cols, false), g);
            if (a.weight) mx_floats(mx_fetch8<T, false>((const T*)a.weight, (int)c * 8, (int)a.cols), w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float gw = a.weight ? g[i] * w[i] : g[i];
                sg += gw;
                sgx = fmaf(gw, x[i] - mean, sgx);
            }
        }
        const float mg = LAYER ? block_sum(sg, red) * inv_n : 0.f, m = block_sum(sgx, red) * inv_n * rstd * rstd;
        for (long long c = threadIdx.x; c < pieces; c += 512) {
            mx_restore8(a.codes, a.scales, row, (int)c, a.nb, a.pitch, x);
            mx_floats(mx_fetch8<T, VEC>(dy, (int)c * 8, (int)a.cols, false), g);
            if (a.weight) mx_floats(mx_fetch8<T, false>((const T*)a.weight, (int)c * 8, (int)a.cols), w);
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = rstd * ((a.weight ? g[i] * w[i] : g[i]) - mg - (x[i] - mean) * m);
            mx_store8<T, VEC>(dx, (int)c * 8, (int)a.cols, mx_piece<T>(g));
        }
    }
}

// ... and their column sums: a thread has a piece of 8 columns and every gridDim.y-th row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(128) mx_norm_columns_kernel(const NormArgs a, const float2* __restrict__ stats)
{
    const long long c = (long long)blockIdx.x * 128 + threadIdx.x;
    if (c * 8 >= a.cols) return;
    float dw[8] = {}, db[8] = {}, x[8], g[8];
    for (long long row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float2 st = stats[row];
        mx_restore8(a.codes, a.scales, row, (int)c, a.nb, a.pitch, x);
        mx_floats(mx_fetch8<T, VEC>((const T*)a.dy + row * a.dy_stride, (int)c * 8, (int)a.cols, false), g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dw[i] = fmaf(g[i], (x[i] - st.x) * st.y, dw[i]);
            db[i] += g[i];
        }
    }
    const long long pitch = (a.cols + 7) / 8 * 8;
    float* part = a.part + (long long)blockIdx.y * 2 * pitch + c * 8;
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
        *reinterpret_cast<float4*>(part + i) = make_float4(dw[i], dw[i + 1], dw[i + 2], dw[i + 3]);
        *reinterpret_cast<float4*>(part + pitch + i) = make_float4(db[i], db[i + 1], db[i + 2], db[i + 3]);
    }
}

struct NormPlan { bool warp, wide; int pp, threads, grid, parts, smem, ranks, share, span; size_t stats, total; };

NormPlan norm_plan(const galv_ctx* ctx, int64_t rows, int64_t cols, int32_t dtype)
{
    NormPlan p;
    const int64_t pieces = (cols + 7) / 8;
    const bool four = dtype == GALV_F32;
    const int stages = four ? NormStage<float>::count : NormStage<__half>::count, piece = four ? NormStage<float>::piece : NormStage<__half>::piece;
    p.stats = 0;
    p.share = 1;
    p.span = 0;
    p.wide = false;
    p.warp = cols <= kWarpColumns;
    if (p.warp) {
        p.pp = pieces <= 32 ? 1 : pieces <= 64 ? 2 : 4;
        p.threads = 256;
        const int64_t most = ctx->num_sms * (p.pp == 4 ? 1 : 2), need = (rows + 7) / 8;
        p.parts = p.grid = (int)(need < most ? need : most);
        p.smem = 32 * p.pp * (piece - 12 + 8 * stages * piece);
        if (p.smem < 8 * 2 * 32 * p.pp * 8 * 4) p.smem = 8 * 2 * 32 * p.pp * 8 * 4;
    } else {
        p.pp = pieces <= kBlockThreads ? 1 : 2;
        const int64_t need = (pieces + p.pp - 1) / p.pp;
        p.threads = p.pp == 1 ? (need <= 256 ? 256 : need <= 512 ? 512 : 1024) : need <= 768 ? 768 : 1024;
        if (need > kBlockThreads) p.threads = kBlockThreads + 1;
        const int64_t smem = (int64_t)p.threads * p.pp * (piece - 12 + stages * piece + (p.pp > 1 ? 32 : 0));
        p.wide = p.threads > kBlockThreads || smem > ctx->smem_optin - 2048 || (four && p.pp > 1);
        const int64_t most = ctx->num_sms * (p.threads <= 256 ? 4 : p.threads <= 512 ? 2 : 1);
        p.parts = p.grid = (int)(rows < most ? rows : most);
        p.smem = (int)smem;
    }
    // A row that one CTA cannot hold is shared by two of a cluster, which exchange its sums over a cluster barrier, up to 16384 columns of fp32 and 32768
    // of 16 bits, or four, up to 65536: 2048 x 12288 in fp32 takes 104 us for a layer norm, 300 with the kernels for wide rows; 1024 x 32768 in bf16
    // 100 and 173; 512 x 49152 81 and 128.  What one CTA holds it keeps (2048 x 12288 in bf16: 53 us, shared by two 90), and fp32 shared by four
    // is no faster than the wide kernels (1024 x 32768: 220 to 275 us and 233).  With four, 32 clusters run at once, not 37.
    const int64_t most_pieces = four ? 1024 : 2048;       // of a CTA
    const int clusters = four || pieces <= 2 * most_pieces ? 2 : 4;
    if (p.wide && pieces <= clusters * most_pieces) {
        p.wide = false;
        p.share = clusters;
        p.pp = four ? 1 : 2;
        p.span = (int)((pieces + p.share - 1) / p.share + 15) / 16 * 16;
        p.threads = p.span <= 768 * p.pp ? 768 : 1024;
        p.smem = p.threads * p.pp * (piece - 12 + stages * piece + (p.pp > 1 ? 32 : 0));
        const int64_t most = (p.share == 2 ? ctx->num_sms : ctx->num_sms * 7 / 8) / p.share;
        p.parts = (int)(rows < most ? rows : most);
        p.grid = p.parts * p.share;
    }
    if (p.wide) {
        p.threads = 512;
        p.grid = (int)(rows < ctx->num_sms * 4 ? rows : ctx->num_sms * 4);
        p.parts = (int)(rows < 8 ? rows : 8);
        p.stats = ((size_t)rows * sizeof(float2) + 255) & ~(size_t)255;
    }
    // Few rows: one cluster of eight CTAs that needs no second kernel and no workspace (33 x 2048, rms: a call takes 16 us in place of 22, the
    // kernel 7.0 in place of two of 5.5 together).
    const int64_t rounds = (rows + 8 * (p.warp ? 8 : 1) - 1) / (8 * (p.warp ? 8 : 1));
    p.ranks = !p.wide && p.share == 1 && pieces <= 512 && rounds <= 5 ? 8 : 0;
    if (p.ranks) {
        const int64_t teams = p.warp ? 8 : 1, need = (rows + teams - 1) / teams;
        p.ranks = need >= 5 ? 8 : need >= 3 ? 4 : (int)need;
        p.parts = p.grid = p.ranks;
        p.total = 0;
        return p;
    }
    p.total = p.stats + (((size_t)p.parts * 2 * pieces * 8 * 4 + 255) & ~(size_t)255);
    return p;
}

template <typename T, bool LAYER, bool VEC, int W, int PP, bool SPLIT = false>
void norm_start(const NormPlan& p, const NormArgs& a, cudaStream_t st)
{
    const auto kernel = mx_norm_kernel<T, LAYER, VEC, W, PP, SPLIT>;
    if (p.smem > 48 * 1024) cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, p.smem);
    if (p.ranks || SPLIT) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(p.grid);
        cfg.blockDim = dim3(p.threads);
        cfg.dynamicSmemBytes = p.smem;
        cfg.stream = st;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)(SPLIT ? p.share : p.ranks);
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        cudaLaunchKernelEx(&cfg, kernel, a);
        return;
    }
    kernel<<<p.grid, p.threads, p.smem, st>>>(a);
}

template <typename T, bool LAYER, bool VEC>
void norm_launch(const NormPlan& p, const NormArgs& a, float2* stats, bool sums, cudaStream_t st)
{
    if (p.wide) {
        mx_norm_wide_kernel<T, LAYER, VEC><<<p.grid, 512, 0, st>>>(a, stats, false);
        if (sums) mx_norm_columns_kernel<T, VEC><<<dim3((unsigned)((a.cols + 1023) / 1024), p.parts), 128, 0, st>>>(a, stats);
        mx_norm_wide_kernel<T, LAYER, VEC><<<p.grid, 512, 0, st>>>(a, stats, true);
    } else if (p.share > 1) {
        constexpr int PP = sizeof(T) == 4 ? 1 : 2;
        if (p.threads == 768) norm_start<T, LAYER, VEC, 768, PP, true>(p, a, st);
        else norm_start<T, LAYER, VEC, 1024, PP, true>(p, a, st);
    } else if (p.warp) {
        if (p.pp == 1) norm_start<T, LAYER, VEC, 32, 1>(p, a, st);
        else if (p.pp == 2) norm_start<T, LAYER, VEC, 32, 2>(p, a, st);
        else norm_start<T, LAYER, VEC, 32, 4>(p, a, st);
    } else if (p.pp == 1) {
        if (p.threads == 256) norm_start<T, LAYER, VEC, 256, 1>(p, a, st);
        else if (p.threads == 512) norm_start<T, LAYER, VEC, 512, 1>(p, a, st);
        else norm_start<T, LAYER, VEC, 1024, 1>(p, a, st);
    } else if constexpr (sizeof(T) == 2) {                // (of fp32 a CTA holds no two pieces a thread)
        if (p.threads == 768) norm_start<T, LAYER, VEC, 768, 2>(p, a, st);
        else norm_start<T, LAYER, VEC, 1024, 2>(p, a, st);
    }
}

}  // namespace

extern "C" int galv_mx_act_backward(galv_ctx* ctx, int64_t rows, int64_t cols, int32_t act, const uint8_t* codes, const uint8_t* scales, const void* dy,
                                    int64_t dy_stride, void* dx, int64_t dx_stride, int32_t dtype, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!mx_size_ok(rows, cols) || !mx_dtype_ok(dtype) || act < GALV_ACT_GELU || act > GALV_ACT_SILU)
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_act_backward: sizes, type or function outside the limits");
    if (rows == 0) return GALV_OK;
    if (!mx_matrix_ok(dy, dy_stride, cols, dtype) || !mx_matrix_ok(dx, dx_stride, cols, dtype) || !codes || !scales || !mx_aligned(codes, 16) || !mx_aligned(scales, 16))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_act_backward: NULL or misaligned pointer, or a row stride below cols");
    if (dx == dy && dx_stride != dy_stride)
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_act_backward: dx may be dy with the same stride only");
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    const int nb = (int)mx_blocks(cols), pitch = (int)mx_pitch8(cols), pieces = (int)((cols + 7) / 8);
    const bool vec = mx_rows16(dy, dy_stride, dtype) && mx_rows16(dx, dx_stride, dtype);
    const MxSpread spread(rows, pieces, dtype == GALV_F32 ? MxEach<float>::count : MxEach<__half>::count);
    // A table pays for 16-bit numbers (fp32 is at the memory's rate without) where each CTA has four rounds or more: 4096 x 32768 in bf16 takes 123 us with
    // it and 153 without for gelu, 120 and 130 for gelu_tanh; 115 without and 118 with for silu, which goes without.  Four CTAs fit an SM.
    const long long resident = (long long)ctx->num_sms * 4;
    const bool table = dtype != GALV_F32 && act != GALV_ACT_SILU && spread.blocks >= 4 * resident;
    const int grid = table ? (int)resident : spread.grid();
    cudaStream_t st = (cudaStream_t)stream;
#define MX_ACT_START(ACT, VEC, TABLE, SMEM) \
    mx_act_kernel<T, ACT, VEC, TABLE><<<grid, kMxThreads, SMEM, st>>>(spread, (unsigned)rows, (int)cols, nb, pieces, pitch, codes, scales, (const T*)dy, dy_stride, (T*)dx, dx_stride)
#define MX_ACT(ACT)                                                                                                          \
    MX_DISPATCH_TYPE(dtype,                                                                                                  \
        constexpr bool can = sizeof(T) == 2 && ACT != GALV_ACT_SILU;                                                                            \
        if (can && table) { if (vec) MX_ACT_START(ACT, true, can, kTableBytes); else MX_ACT_START(ACT, false, can, kTableBytes); } \
        else { if (vec) MX_ACT_START(ACT, true, false, 0); else MX_ACT_START(ACT, false, false, 0); })
    if (act == GALV_ACT_GELU) MX_ACT(GALV_ACT_GELU);
    else if (act == GALV_ACT_GELU_TANH) MX_ACT(GALV_ACT_GELU_TANH);
    else MX_ACT(GALV_ACT_SILU);
#undef MX_ACT
#undef MX_ACT_START
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}

extern "C" size_t galv_mx_norm_workspace_bytes(const galv_ctx* ctx, int64_t rows, int64_t cols)
{
    if (!ctx || !mx_size_ok(rows, cols) || rows == 0) return 0;
    const size_t a = norm_plan(ctx, rows, cols, GALV_F32).total, b = norm_plan(ctx, rows, cols, GALV_F16).total;
    return a > b ? a : b;
}

extern "C" int galv_mx_norm_backward(galv_ctx* ctx, int64_t rows, int64_t cols, int32_t kind, float eps, const uint8_t* codes, const uint8_t* scales,
                                     const void* dy, int64_t dy_stride, const void* weight, void* dx, int64_t dx_stride, int32_t dtype, float* dweight,
                                     float* dbias, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!mx_size_ok(rows, cols) || !mx_dtype_ok(dtype) || (kind != GALV_NORM_LAYER && kind != GALV_NORM_RMS) || !(eps >= 0.f))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_norm_backward: sizes, type, kind or eps outside the limits");
    if (kind == GALV_NORM_RMS && dbias) return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_norm_backward: GALV_NORM_RMS has no bias");
    if ((dweight && !mx_aligned(dweight, 4)) || (dbias && !mx_aligned(dbias, 4)))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_norm_backward: misaligned dweight or dbias");
    MxDevice dev(ctx);
    if (dev.err != cudaSuccess) return galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(dev.err));
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    if (rows == 0) {
        e = dweight ? cudaMemsetAsync(dweight, 0, cols * 4, st) : cudaSuccess;
        if (e == cudaSuccess && dbias) e = cudaMemsetAsync(dbias, 0, cols * 4, st);
        return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
    }
    if (!mx_matrix_ok(dy, dy_stride, cols, dtype) || !mx_matrix_ok(dx, dx_stride, cols, dtype) || !codes || !scales || !mx_aligned(codes, 16) ||
        !mx_aligned(scales, 16) || (weight && !mx_aligned(weight, mx_size_of(dtype))))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_norm_backward: NULL or misaligned pointer, or a row stride below cols");
    if (dx == dy && dx_stride != dy_stride)
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_mx_norm_backward: dx may be dy with the same stride only");
    const size_t bytes = galv_mx_norm_workspace_bytes(ctx, rows, cols);
    if (bytes && (!workspace || !mx_aligned(workspace, 256) || workspace_bytes < bytes))
        return galv_set_error(ctx, GALV_ERR_WORKSPACE, "galv_mx_norm_backward: workspace NULL, misaligned or too small");
    const NormPlan p = norm_plan(ctx, rows, cols, dtype);
    NormArgs a;
    a.rows = rows; a.cols = cols; a.nb = mx_blocks(cols); a.pitch = mx_pitch8(cols); a.dy_stride = dy_stride; a.dx_stride = dx_stride;
    a.eps = eps; a.codes = codes; a.scales = scales; a.dy = dy; a.weight = weight; a.weight16 = mx_aligned(weight, 16); a.dx = dx;
    a.part = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + p.stats);
    a.ranks = p.ranks; a.share = p.share; a.span = p.span; a.dweight = dweight; a.dbias = dbias;
    float2* stats = reinterpret_cast<float2*>(workspace);
    const bool vec = mx_rows16(dy, dy_stride, dtype) && mx_rows16(dx, dx_stride, dtype), layer = kind == GALV_NORM_LAYER, sums = dweight || dbias;
    MX_DISPATCH_TYPE(dtype,
        if (layer) { if (vec) norm_launch<T, true, true>(p, a, stats, sums, st); else norm_launch<T, true, false>(p, a, stats, sums, st); }
        else { if (vec) norm_launch<T, false, true>(p, a, stats, sums, st); else norm_launch<T, false, false>(p, a, stats, sums, st); });
    if (sums && !p.ranks) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)((cols + 31) / 32), dbias ? 2 : 1);
        cfg.blockDim = dim3(1024);
        cfg.stream = st;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        cudaLaunchKernelEx(&cfg, mx_norm_join_kernel, (long long)cols, (long long)((cols + 7) / 8 * 8), p.parts, (const float*)a.part, dweight, dbias);
    }
    e = cudaGetLastError();
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}
