// verify_draft.cu -- speculative sampling: accepts or rejects drafted tokens
// against the target's probabilities and draws the next token from given
// random numbers.
//
// The next token is drawn by a race of exponential clocks: with e_v ~ Exp(1),
// v wins (largest r_v / e_v) with probability r_v / sum r.  So r need not be
// normalised, one pass over the row suffices, and the result is a maximum:
// exact, and the same whatever order the row is read in.
#include <cstdint>

#include "host_common.h"
#include "logo_status.cuh"

namespace logo {
namespace {

constexpr int kVdThreads = 1024;

struct VdParams {
    const int32_t* draft;
    const float *q, *p, *u, *noise;
    const int32_t* draft_len;
    int32_t *tokens, *n_accept;
    int B, m, V;
};

// A candidate as one comparable word: the score's bits (a non-negative float
// orders as its bits), then the lower index first.  0: no candidate.
__device__ __forceinline__ unsigned long long race_key(float r, float e, int v)
{
    if (!(r > 0.f)) return 0ull;
    float s = __fdiv_rn(r, e);
    if (!(s > 0.f)) s = 0.f;  // underflowed, or not a clock: behind all others
    return (static_cast<unsigned long long>(__float_as_uint(s)) << 32) | (0xffffffffu - static_cast<uint32_t>(v));
}

__global__ void __launch_bounds__(kVdThreads) verify_kernel(VdParams p)
{
    __shared__ unsigned long long sh_best[2][32];
    __shared__ int sh_a;
    const int b = blockIdx.x, tid = threadIdx.x;
    const int m = p.draft_len ? max(0, min(p.draft_len[b], p.m)) : p.m;
    if (tid == 0) {
        int a = 0;
        for (; a < m; ++a) {
            const int64_t row = static_cast<int64_t>(b) * p.m + a;
            const int d = p.draft[row];
            if (d < 0 || d >= p.V) break;
            const float pd = p.p[(static_cast<int64_t>(b) * (p.m + 1) + a) * p.V + d];
            const float qd = p.q[row * p.V + d];
            if (!(pd > 0.f && __fmul_rn(p.u[row], qd) <= pd)) break;
        }
        sh_a = a;
    }
    __syncthreads();
    const int a = sh_a;
    const float* pr = p.p + (static_cast<int64_t>(b) * (p.m + 1) + a) * p.V;
    const float* qr = a < m ? p.q + (static_cast<int64_t>(b) * p.m + a) * p.V : nullptr;
    const float* e = p.noise + static_cast<int64_t>(b) * p.V;
    unsigned long long best = 0, best_p = 0;  // of the residual, and of p itself should the residual be empty
    for (int v = tid; v < p.V; v += kVdThreads) {
        const float pv = pr[v], ev = e[v];
        const unsigned long long kp = race_key(pv, ev, v);
        best_p = kp > best_p ? kp : best_p;
        if (qr) {
            const unsigned long long kr = race_key(__fsub_rn(pv, qr[v]), ev, v);
            best = kr > best ? kr : best;
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const unsigned long long x = __shfl_xor_sync(0xffffffffu, best, o), y = __shfl_xor_sync(0xffffffffu, best_p, o);
        best = x > best ? x : best;
        best_p = y > best_p ? y : best_p;
    }
    if ((tid & 31) == 0) {
        sh_best[0][tid >> 5] = best;
        sh_best[1][tid >> 5] = best_p;
    }
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kVdThreads / 32; ++w) {
            best = sh_best[0][w] > best ? sh_best[0][w] : best;
            best_p = sh_best[1][w] > best_p ? sh_best[1][w] : best_p;
        }
        const unsigned long long k = best ? best : best_p;
        p.n_accept[b] = a;
        int32_t* out = p.tokens + static_cast<int64_t>(b) * (p.m + 1);
        for (int i = 0; i < a; ++i) out[i] = p.draft[static_cast<int64_t>(b) * p.m + i];
        out[a] = k ? static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(k)) : 0;
        for (int i = a + 1; i <= p.m; ++i) out[i] = -1;
    }
}

bool verify_sizes_ok(int B, int m, int V)
{
    return B >= 1 && m >= 0 && V >= 1 && static_cast<int64_t>(B) * (static_cast<int64_t>(m) + 1) <= (1ll << 24);
}

}  // namespace
}  // namespace logo

using namespace logo;

extern "C" size_t logo_verify_draft_workspace_size(int B, int m, int V) { return verify_sizes_ok(B, m, V) ? 256 : 0; }

extern "C" int logo_verify_draft(const int32_t* draft, const float* q_draft, const float* p_target, const float* u,
                                 const float* noise, const int32_t* draft_len, int32_t* tokens, int32_t* n_accept,
                                 int B, int m, int V, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!verify_sizes_ok(B, m, V)) return LOGO_ERR_INVALID_ARG;
    if (!p_target || !noise || !tokens || !n_accept) return LOGO_ERR_INVALID_ARG;
    if (m > 0 && (!draft || !q_draft || !u)) return LOGO_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < logo_verify_draft_workspace_size(B, m, V) || !aligned16(workspace))
        return LOGO_ERR_WORKSPACE;
    VdParams p{draft, q_draft, p_target, u, noise, draft_len, tokens, n_accept, B, m, V};
    verify_kernel<<<B, kVdThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return cudaGetLastError() == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}
