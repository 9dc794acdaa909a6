// target_probs.cu -- logits to the target's probabilities: penalties for repeated
// tokens, biases, a grammar's mask, temperature, softmax.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "host_common.h"

namespace logo {
namespace {

constexpr int kTpThreads = 1024;

struct TpParams {
    const void* logits;
    const float *temperature, *penalty;
    const int32_t *history, *hist_len, *n_prompt, *draft, *bias_tok;
    const float* bias_val;
    const uint32_t* allowed;
    float* p;
    int B, m1, V, H, K;
    bool half;
};

__device__ __forceinline__ float block_reduce(float x, bool want_max, float* sh)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int round = 0; round < 2; ++round) {
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            const float y = __shfl_xor_sync(0xffffffffu, x, d);
            x = want_max ? fmaxf(x, y) : x + y;
        }
        if (round == 0) {
            __syncthreads();
            if (lane == 0) sh[warp] = x;
            __syncthreads();
            x = sh[lane];
        }
    }
    return x;
}

// A CTA a row; p holds the adjusted logits until the last pass.
__global__ void __launch_bounds__(kTpThreads) target_probs_kernel(TpParams a)
{
    __shared__ float sh[32];
    __shared__ int sh_first, sh_nan;
    const int64_t row = blockIdx.x;
    const int b = row / a.m1, i = row % a.m1, tid = threadIdx.x, V = a.V;
    float* p = a.p + row * V;
    if (tid == 0) sh_first = V, sh_nan = 0;
    for (int v = tid; v < V; v += kTpThreads)
        p[v] = a.half ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(a.logits)[row * V + v]) << 16)
                      : static_cast<const float*>(a.logits)[row * V + v];
    __syncthreads();
    if (a.penalty) {
        const int old = a.history ? max(0, min(a.hist_len[b], a.H)) : 0;
        const int prompt = max(a.n_prompt ? a.n_prompt[b] : 0, old - LOGO_PROBS_MAX_COUNTED);
        const int n = old + (a.draft ? i : 0);
        const int32_t* hist = a.history + static_cast<int64_t>(b) * a.H;
        const int32_t* draft = a.draft + static_cast<int64_t>(b) * (a.m1 - 1);
        const float rep = a.penalty[3 * b], freq = a.penalty[3 * b + 1], pres = a.penalty[3 * b + 2];
        for (int j = tid; j < n; j += kTpThreads) {
            const int t = j < old ? hist[j] : draft[j - old];
            if (t < 0 || t >= V) continue;
            bool first = true;
            int count = 0;
            for (int k = 0; k < n; ++k) {
                if ((k < old ? hist[k] : draft[k - old]) != t) continue;
                first &= k >= j;
                count += k >= prompt;
            }
            if (!first) continue;
            float x = p[t];
            x = x > 0.f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
            if (count) x = __fsub_rn(x, __fadd_rn(__fmul_rn(static_cast<float>(count), freq), pres));
            p[t] = x;
        }
        __syncthreads();
    }
    for (int j = tid; j < a.K; j += kTpThreads) {
        const int32_t* tok = a.bias_tok + static_cast<int64_t>(b) * a.K;
        const int t = tok[j];
        if (t < 0 || t >= V) continue;
        bool first = true;
        float sum = 0.f;
        for (int k = 0; k < a.K; ++k) {
            if (tok[k] != t) continue;
            first &= k >= j;
            sum = __fadd_rn(sum, a.bias_val[static_cast<int64_t>(b) * a.K + k]);
        }
        if (first) p[t] = __fadd_rn(p[t], sum);
    }
    __syncthreads();
    const float T = a.temperature ? a.temperature[b] : 1.f;
    const uint32_t* allowed = a.allowed ? a.allowed + row * ((V + 31) / 32) : nullptr;
    float top = -INFINITY;
    for (int v = tid; v < V; v += kTpThreads) {
        float x = p[v];
        if (T != 0.f) x = __fdiv_rn(x, T);
        if (allowed && !(allowed[v >> 5] >> (v & 31) & 1)) x = -INFINITY;
        if (x != x) sh_nan = 1;
        p[v] = x;
        top = fmaxf(top, x);
    }
    top = block_reduce(top, true, sh);
    __syncthreads();
    const bool none = top == -INFINITY && !sh_nan;
    float sum = 0.f;
    for (int v = tid; v < V; v += kTpThreads) {
        const float x = p[v];
        sum += none ? 0.f : expf(x - top);
        if (x == top && !none) atomicMin(&sh_first, v);
    }
    sum = block_reduce(sum, false, sh);
    __syncthreads();
    for (int v = tid; v < V; v += kTpThreads) {
        const bool out = none || (allowed && !(allowed[v >> 5] >> (v & 31) & 1));
        float x = T == 0.f ? (v == sh_first ? 1.f : 0.f) : __fdiv_rn(expf(p[v] - top), sum);
        if (sh_nan) x = NAN;
        p[v] = out ? 0.f : x;
    }
}

}  // namespace
}  // namespace logo

using namespace logo;

extern "C" int logo_target_probs(const void* logits, int logits_bf16, const float* temperature, const float* penalty,
                                 const int32_t* history, const int32_t* hist_len, const int32_t* n_prompt,
                                 const int32_t* draft, const int32_t* bias_tok, const float* bias_val,
                                 const int32_t* allowed, float* p, int B, int m1, int V, int H, int K, void* stream)
{
    if (B < 1 || m1 < 1 || V < 1 || H < 0 || K < 0 || !logits || !p) return LOGO_ERR_INVALID_ARG;
    if ((history != nullptr) != (hist_len != nullptr) || (n_prompt && !history) || (!history && H > 0) ||
        (history && H < 1) || ((history || draft) && !penalty) || (draft && m1 < 2))
        return LOGO_ERR_INVALID_ARG;
    if ((bias_tok != nullptr) != (K > 0) || (bias_val != nullptr) != (K > 0)) return LOGO_ERR_INVALID_ARG;
    if (V > LOGO_PROBS_MAX_VOCAB || m1 > 1024 || K > 4096 || static_cast<int64_t>(B) * m1 > (1 << 24) ||
        static_cast<int64_t>(B) * H > (1ll << 40))
        return LOGO_ERR_UNSUPPORTED;
    if (!aligned16(logits) || !aligned16(p) || (logits_bf16 && logits == p)) return LOGO_ERR_UNSUPPORTED;
    const TpParams a{logits, temperature, penalty, history, hist_len, n_prompt, draft, bias_tok, bias_val,
                     reinterpret_cast<const uint32_t*>(allowed), p, B, m1, V, H, K, logits_bf16 != 0};
    target_probs_kernel<<<static_cast<unsigned>(B) * m1, kTpThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
    return cudaGetLastError() == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}
