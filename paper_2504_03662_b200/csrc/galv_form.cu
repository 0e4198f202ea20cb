// What a strategy gains and pays when its layers keep their inputs in 8 bits or multiply in 4: added to the cost model's doubles, then quantised
// again.  Compiled with -fmad=false like the cost model itself, so that any IEEE host computes the same doubles.  Elementwise, bound by launch
// latency at the planner's sizes.

#include "galv_internal.h"
#include "galv_quant.cuh"

namespace {

__device__ __forceinline__ bool form_ok(const galv_form_desc& f)
{
    return (f.keep_bits == 0 || f.keep_bits == 8) && (f.mul_bits == 0 || f.mul_bits == 4) && f.keep_s_per_byte >= 0.0 && f.keep_s_per_byte < INFINITY && f.mul_speed > 0.0 &&
           f.mul_speed < INFINITY;
}

__global__ void __launch_bounds__(256) form_cost_kernel(int B, int Lmax, int S, const int32_t* __restrict__ L, const galv_layer_desc* __restrict__ layers, long long layer_stride_B,
                                                        const galv_strategy_desc* __restrict__ strat, const galv_inst_params* __restrict__ inst,
                                                        const galv_form_desc* __restrict__ forms, const double* __restrict__ time_s, const double* __restrict__ mem_bytes,
                                                        int32_t* __restrict__ time_q, int32_t* __restrict__ mem_q)
{
    const long long n = (long long)B * Lmax * S;
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < n; e += (long long)gridDim.x * 256) {
        const int s = (int)(e % S);
        const long long il = e / S;
        const int l = (int)(il % Lmax), i = (int)(il / Lmax);
        const int Li = L[i];
        if (Li < 1 || Li > Lmax || l >= Li || time_q[e] < 0) continue;      // layers that are none, instances that the cost model has flagged
        const galv_form_desc f = forms[s];
        if (!form_ok(f)) {
            time_q[e] = -1;
            mem_q[e] = -1;
            continue;
        }
        if (f.keep_bits == 0 && f.mul_bits == 0) continue;
        const galv_layer_desc ly = layers[i * layer_stride_B + l];
        const galv_strategy_desc sd = strat[s];
        const galv_inst_params in = inst[i];
        const double tp = (double)sd.tp, bq = in.b / sd.batch_div, sbh = ly.seq * bq * ly.h;
        double t = time_s[e], m = mem_bytes[e];
        if (f.keep_bits == 8) {
            // What the model counts as kept layer inputs (bytes); attention scores and parameters stay as they are.  They are bytes of 16-bit numbers whatever
            // bytes_per_elem says (that is what moves between GPUs), so an element is two of them, and 33/32 in 8 bits.
            double act;
            if (sd.ckpt) act = sd.sp ? 2.0 * sbh / tp : 2.0 * sbh;
            else if (sd.sp) act = sbh * (ly.act_rep + ly.act_tp) / tp;
            else act = sbh * (ly.act_rep + ly.act_tp / tp);
            m = m - in.act_mult * (act - act * 1.03125 / 2.0);
            t = t + act * f.keep_s_per_byte;
        }
        if (f.mul_bits == 4) {
            const double fwd = ly.c_lin * bq * ly.seq * ly.h * ly.h * (1.0 + (double)sd.ckpt) / tp / in.flops_rate;
            t = t - (fwd - fwd / f.mul_speed);
        }
        time_q[e] = quant_time(t, in.time_unit_ns);
        mem_q[e] = quant_mem(m, in.bin_bytes);
    }
}

}  // namespace

extern "C" int galv_add_form_cost(galv_ctx* ctx, const galv_shape* sh, const int32_t* L, const galv_layer_desc* layers, int64_t layer_stride_B, const galv_strategy_desc* strat,
                                  const galv_inst_params* inst, const galv_form_desc* forms, const double* time_s, const double* mem_bytes, int32_t* time_q, int32_t* mem_q, void* stream)
{
    if (!ctx) return GALV_ERR_INVALID_ARG;
    if (!sh || sh->B < 1 || sh->Lmax < 1 || sh->Lmax > 65535 || sh->S < 1 || sh->S > 256 || (layer_stride_B != 0 && layer_stride_B < sh->Lmax))
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_add_form_cost: shape outside limits, or layer_stride_B neither 0 nor >= Lmax");
    if (!L || !layers || !strat || !inst || !forms || !time_s || !mem_bytes || !time_q || !mem_q)
        return galv_set_error(ctx, GALV_ERR_INVALID_ARG, "galv_add_form_cost: NULL pointer");
    const long long n = (long long)sh->B * sh->Lmax * sh->S, need = (n + 255) / 256, most = (long long)ctx->num_sms * 16;
    form_cost_kernel<<<(int)(need < most ? need : most), 256, 0, (cudaStream_t)stream>>>(sh->B, sh->Lmax, sh->S, L, layers, layer_stride_B, strat, inst, forms, time_s, mem_bytes, time_q, mem_q);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? GALV_OK : galv_set_error(ctx, GALV_ERR_CUDA, cudaGetErrorString(e));
}
