// verify_draft.cu -- speculative sampling: accepts or rejects drafted tokens
// against the target's probabilities and draws the next token from given
// random numbers.
//
// The next token is drawn by a race of exponential clocks: with e_v ~ Exp(1),
// v wins (largest r_v / e_v) with probability r_v / sum r.  So r need not be
// normalised, one pass over the row suffices, and the result is a maximum:
// exact, and the same whatever order the row is read in.
//
// Bound by HBM: three rows of V floats a sequence (p, q and the clocks); 256 x 7
// drafts, V = 50021: 151 MB in 32.9 us a call in a graph (34.8 call by call), 4.6
// TB/s, of which 5 us are the start, the verdict on the drafts and the exchange.  A
// thread-block cluster takes a sequence, each of its CTAs an equal stretch of
// the row (as many CTAs as the batch leaves SMs for), and the CTAs' maxima meet
// in distributed shared memory: one launch, no scratch, no counters.
#include <cuda_runtime.h>

#include <cstdint>

#include "cluster.cuh"
#include "host_common.h"
#include "logo_status.cuh"

namespace logo {
namespace {

constexpr int kVdThreads = 512;
constexpr int kVdAt = 8;           // loads of each row in flight per thread
constexpr int kVdMaxCluster = 8;   // portable cluster size

struct VdParams {
    const int32_t* draft;
    const float *q, *p, *u, *noise;
    const int32_t* draft_len;
    int32_t *tokens, *n_accept;
    int B, m, V;
};

__device__ __forceinline__ unsigned long long max64(unsigned long long a, unsigned long long b) { return a > b ? a : b; }

// A candidate (r > 0) against the best so far, as one comparable word: the
// score's bits (a non-negative float orders as its bits), then the lower index
// first.  0: no candidate.  The exact quotient is formed only where the fast one
// (off by 2 units in the last place; 0 for e above 2^126, and flushed where it is
// not a normal number) does not rule it out.
__device__ __forceinline__ void race(float r, float e, int v, unsigned long long& best)
{
    if (!(r > 0.f)) return;
    const float top = __uint_as_float(static_cast<uint32_t>(best >> 32));
    if (top > 1.0e-30f && __fdividef(r, e) * 1.000002f < top && e < 8.0e37f) return;
    float s = __fdiv_rn(r, e);
    if (!(s > 0.f)) s = 0.f;  // underflowed, or not a clock: behind all others
    best = max64(best, (static_cast<unsigned long long>(__float_as_uint(s)) << 32) |
                           (0xffffffffu - static_cast<uint32_t>(v)));
}

// The best candidate of the row p (or p - q) over the whole cluster, in every CTA.
template <bool RESIDUAL>
__device__ __forceinline__ unsigned long long race_row(const float* __restrict__ p, const float* __restrict__ q,
                                                       const float* __restrict__ e, int v0, int v1,
                                                       unsigned long long* sh, unsigned long long* sh_best)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned long long best = 0;
    for (int v = v0 + tid; v < v1; v += kVdAt * kVdThreads) {
        float pv[kVdAt], qv[kVdAt], ev[kVdAt];
#pragma unroll
        for (int k = 0; k < kVdAt; ++k) {
            const int i = v + k * kVdThreads;
            const bool in = i < v1;
            pv[k] = in ? __ldcs(p + i) : 0.f;
            qv[k] = RESIDUAL && in ? __ldcs(q + i) : 0.f;
            ev[k] = in ? __ldcs(e + i) : 1.f;
        }
#pragma unroll
        for (int k = 0; k < kVdAt; ++k)
            race(RESIDUAL ? __fsub_rn(pv[k], qv[k]) : pv[k], ev[k], v + k * kVdThreads, best);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) best = max64(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (lane == 0) sh[warp] = best;
    __syncthreads();
    if (warp == 0) {
        best = lane < kVdThreads / 32 ? sh[lane] : 0;
#pragma unroll
        for (int o = 16; o; o >>= 1) best = max64(best, __shfl_xor_sync(0xffffffffu, best, o));
        if (lane == 0) *sh_best = best;
    }
    cluster_sync();
    const uint32_t n = cluster_size();
    unsigned long long of[kVdMaxCluster];
#pragma unroll
    for (uint32_t c = 0; c < kVdMaxCluster; ++c) of[c] = c < n ? cluster_read(sh_best, c) : 0;
    best = 0;
#pragma unroll
    for (uint32_t c = 0; c < kVdMaxCluster; ++c) best = max64(best, of[c]);
    return best;
}

__global__ void __launch_bounds__(kVdThreads, 2) verify_kernel(VdParams p)
{
    __shared__ unsigned long long sh[kVdThreads / 32], sh_best[2];
    __shared__ int sh_a;
    const uint32_t cs = cluster_size(), rank = cluster_rank();
    const int b = blockIdx.x / cs, tid = threadIdx.x;
    const int m = p.draft_len ? max(0, min(p.draft_len[b], p.m)) : p.m;
    if (tid < 32) {  // drafts accepted before the first rejection, 32 at a time
        int a = 0;
        for (int i0 = 0; i0 < m; i0 += 32) {
            bool ok = false;
            const int i = i0 + tid;
            if (i < m) {
                const int64_t row = static_cast<int64_t>(b) * p.m + i;
                const int d = p.draft[row];
                if (d >= 0 && d < p.V) {
                    const float pd = p.p[(static_cast<int64_t>(b) * (p.m + 1) + i) * p.V + d];
                    const float qd = p.q[row * p.V + d];
                    ok = pd > 0.f && __fmul_rn(p.u[row], qd) <= pd;
                }
            }
            const uint32_t bad = ~__ballot_sync(0xffffffffu, ok);
            const int n = bad ? __ffs(bad) - 1 : 32;
            a += n;
            if (n < 32) break;
        }
        if (tid == 0) sh_a = a;
    }
    __syncthreads();
    const int a = sh_a;
    const float* pr = p.p + (static_cast<int64_t>(b) * (p.m + 1) + a) * p.V;
    const float* e = p.noise + static_cast<int64_t>(b) * p.V;
    const int v0 = static_cast<int>(static_cast<int64_t>(p.V) * rank / cs);
    const int v1 = static_cast<int>(static_cast<int64_t>(p.V) * (rank + 1) / cs);
    unsigned long long best = 0;
    if (a < m) best = race_row<true>(pr, p.q + (static_cast<int64_t>(b) * p.m + a) * p.V, e, v0, v1, sh, sh_best);
    // no draft rejected, or (the same in every CTA) nothing left of p - q
    if (best == 0) {
        __syncthreads();
        best = race_row<false>(pr, nullptr, e, v0, v1, sh, sh_best + 1);
    }
    if (rank == 0) {
        int32_t* out = p.tokens + static_cast<int64_t>(b) * (p.m + 1);
        for (int i = tid; i <= p.m; i += kVdThreads) {
            const int32_t drawn = best ? static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(best)) : 0;
            out[i] = i < a ? p.draft[static_cast<int64_t>(b) * p.m + i] : i == a ? drawn : -1;
        }
        if (tid == 0) p.n_accept[b] = a;
    }
    cluster_sync();  // no CTA leaves while another may read its maximum
}

bool verify_sizes_ok(int B, int m, int V)
{
    return B >= 1 && m >= 0 && V >= 1 && V <= (1 << 30) && static_cast<int64_t>(B) * (static_cast<int64_t>(m) + 1) <= (1ll << 24);
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
    // CTAs per sequence: the largest cluster of which all are resident at once (two
    // CTAs an SM, less what clusters of this size leave free in a group of SMs), with
    // stretches of a few loads a thread at least.  Measured (us) with 1 to 7: 57
    // sequences, V = 60000 28.7 18.9 16.4 14.4 13.1 20.0 20.4; 40, V = 100000 42 26 20
    // 18.5 16.1 15.2 22.3; 96, V = 60000 29.2 21.8 17.3 25.5.
    constexpr int kFill[] = {100, 95, 95, 95, 95, 91, 83, 95};  // per cent
    static_assert(sizeof kFill / sizeof *kFill == kVdMaxCluster, "a share for each cluster size");
    const int64_t places = 2ll * device_sm_count();
    int cs = 1;
    for (int c = 2; c <= kVdMaxCluster && V / c >= 2 * kVdThreads; ++c)
        if (B <= places * kFill[c - 1] / 100 / c) cs = c;
    cudaLaunchAttribute attr{};
    const cudaLaunchConfig_t cfg = cluster_config(static_cast<unsigned>(B) * cs, kVdThreads, cs, 0,
                                                  static_cast<cudaStream_t>(stream), &attr);
    return cudaLaunchKernelEx(&cfg, verify_kernel, p) == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}
