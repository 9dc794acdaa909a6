// prefix_attn.cu -- one serving step of the global branch (Eq. 8) for a batch
// that shares a long prefix: packed rows of n_new tokens per sequence attend
// the shared prefix and their own sequence's cache, and the attention weight
// that every own cache row receives is added up.
#include <cuda_bf16.h>

#include <cstdint>

#include "attn_common.cuh"
#include "host_common.h"
#include "logo_status.cuh"
#include "sm100.cuh"

namespace logo {
namespace {

struct PaParams {
    const logo_bf16 *q, *kp, *vp, *kc, *vc;
    const int32_t *seq_len, *pos, *cu_q, *n_sel;
    logo_bf16* o;
    float* lse;       // [Hq, cap] natural log
    const float* mass_in;
    float* mass_out;
    int B, L, Hq, Hkv, n_new, P, cap;
    float scale_log2;
};

// Own cache rows that token i of a sequence with len tokens sees.
__device__ __forceinline__ int own_visible(int len, int n_new, int i) { return min(len, max(0, len - n_new + i + 1)); }

// A block is one (packed row, query head); a warp takes every fourth key, its
// lanes split the head dimension; each warp keeps an online softmax.
template <int D>
__global__ void __launch_bounds__(128) pa_rows_kernel(PaParams p)
{
    constexpr int E = D / 32;
    __shared__ float sh_o[4][D], sh_m[4], sh_l[4];
    const int r = blockIdx.x, h = blockIdx.y;
    if (r >= *p.n_sel) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int kvh = h / (p.Hq / p.Hkv);
    const int b = seq_of_row(p.cu_q, p.B, r);
    const int len = max(0, min(p.seq_len[b], p.L));
    const int vis = own_visible(len, p.n_new, p.pos[r]);
    const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(p.q) +
                             ((static_cast<int64_t>(b) * p.n_new + p.pos[r]) * p.Hq + h) * D;
    float qv[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        qv[e] = __bfloat162float(q[e * 32 + lane]);
        o[e] = 0.f;
    }
    for (int64_t s = warp; s < static_cast<int64_t>(p.P) + vis; s += 4) {
        const bool pre = s < p.P;
        const int64_t row = pre ? s : static_cast<int64_t>(b) * p.L + (s - p.P);
        const __nv_bfloat16* k = reinterpret_cast<const __nv_bfloat16*>(pre ? p.kp : p.kc) + (row * p.Hkv + kvh) * D;
        const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(pre ? p.vp : p.vc) + (row * p.Hkv + kvh) * D;
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) x += qv[e] * __bfloat162float(k[e * 32 + lane]);
#pragma unroll
        for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        x *= p.scale_log2;
        const float m_new = fmaxf(m, x);
        const float a = m == -INFINITY ? 0.f : exp2f(m - m_new);
        const float w = m_new == -INFINITY ? 0.f : exp2f(x - m_new);
        l = l * a + w;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * a + w * __bfloat162float(v[e * 32 + lane]);
        m = m_new;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) sh_o[warp][e * 32 + lane] = o[e];
    if (lane == 0) {
        sh_m[warp] = m;
        sh_l[warp] = l;
    }
    __syncthreads();
    float M = -INFINITY, Lsum = 0.f;
    for (int w = 0; w < 4; ++w) M = fmaxf(M, sh_m[w]);
    for (int w = 0; w < 4; ++w) Lsum += sh_m[w] == -INFINITY ? 0.f : exp2f(sh_m[w] - M) * sh_l[w];
    if (threadIdx.x < D) {
        float acc = 0.f;
        for (int w = 0; w < 4; ++w) acc += sh_m[w] == -INFINITY ? 0.f : exp2f(sh_m[w] - M) * sh_o[w][threadIdx.x];
        reinterpret_cast<__nv_bfloat16*>(p.o)[(static_cast<int64_t>(r) * p.Hq + h) * D + threadIdx.x] =
            __float2bfloat16_rn(Lsum > 0.f ? acc / Lsum : 0.f);
    }
    if (threadIdx.x == 0) p.lse[static_cast<int64_t>(h) * p.cap + r] = (M + log2f(Lsum)) * kLn2;
}

// The weight of every own cache row: a warp per (sequence, KV head, row).
template <int D>
__global__ void __launch_bounds__(128) pa_mass_kernel(PaParams p)
{
    constexpr int E = D / 32;
    const int b = blockIdx.z, kvh = blockIdx.y, G = p.Hq / p.Hkv;
    const int len = max(0, min(p.seq_len[b], p.L));
    const int lane = threadIdx.x & 31;
    for (int s = blockIdx.x * 4 + (threadIdx.x >> 5); s < len; s += gridDim.x * 4) {
        const __nv_bfloat16* k = reinterpret_cast<const __nv_bfloat16*>(p.kc) +
                                 ((static_cast<int64_t>(b) * p.L + s) * p.Hkv + kvh) * D;
        float kv[E];
#pragma unroll
        for (int e = 0; e < E; ++e) kv[e] = __bfloat162float(k[e * 32 + lane]);
        const int64_t at = (static_cast<int64_t>(b) * p.Hkv + kvh) * p.L + s;
        float acc = 0.f;  // what this call adds: summed first, so that the old weight takes one rounding
        for (int r = p.cu_q[b]; r < p.cu_q[b + 1]; ++r) {
            if (s >= own_visible(len, p.n_new, p.pos[r])) continue;
            for (int g = 0; g < G; ++g) {
                const int h = kvh * G + g;
                const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(p.q) +
                                         ((static_cast<int64_t>(b) * p.n_new + p.pos[r]) * p.Hq + h) * D;
                float x = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) x += kv[e] * __bfloat162float(q[e * 32 + lane]);
#pragma unroll
                for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
                acc += exp2f(x * p.scale_log2 - p.lse[static_cast<int64_t>(h) * p.cap + r] * kLog2e);
            }
        }
        if (lane == 0) p.mass_out[at] = (s < len - p.n_new ? p.mass_in[at] : 0.f) + acc;
    }
}

int check_prefix(const logo_dims& d, int n_new, int P)
{
    int rc = check_dims(d);
    if (rc != LOGO_OK) return rc;
    if (n_new < 1 || P < 0) return LOGO_ERR_INVALID_ARG;
    if (static_cast<int64_t>(d.B) * n_new > (1ll << 24)) return LOGO_ERR_UNSUPPORTED;
    return LOGO_OK;
}

// the rows' lse (kept here when the caller does not want it)
size_t prefix_ws_bytes(const logo_dims& d, int n_new)
{
    return round_up(static_cast<size_t>(d.Hq) * d.B * n_new * sizeof(float), 256);
}

template <int D>
int launch_prefix(const PaParams& p, cudaStream_t st)
{
    pa_rows_kernel<D><<<dim3(p.cap, p.Hq), 128, 0, st>>>(p);
    if (p.mass_out) pa_mass_kernel<D><<<dim3((p.L + 63) / 64, p.Hkv, p.B), 128, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}

}  // namespace

int prefix_attn_tu_status(int clear) { return read_tu_status(clear); }

}  // namespace logo

using namespace logo;

extern "C" size_t logo_decode_prefix_workspace_size(logo_dims dims, int n_new, int prefix_len, int with_mass)
{
    (void)with_mass;
    if (check_prefix(dims, n_new, prefix_len) != LOGO_OK) return 0;
    return prefix_ws_bytes(dims, n_new);
}

extern "C" int logo_decode_prefix_attn(const logo_bf16* q, const logo_bf16* k_prefix, const logo_bf16* v_prefix,
                                       const logo_bf16* k_cache, const logo_bf16* v_cache, const int32_t* seq_len,
                                       const int32_t* pos, const int32_t* cu_q, const int32_t* n_sel_total,
                                       logo_bf16* o_c, float* lse_c, const float* mass_in, float* mass_out,
                                       logo_dims dims, int n_new, int prefix_len, float scale, void* workspace,
                                       size_t workspace_bytes, void* stream)
{
    int rc = check_prefix(dims, n_new, prefix_len);
    if (rc != LOGO_OK) return rc;
    if (!q || !k_cache || !v_cache || !seq_len || !pos || !cu_q || !n_sel_total || !o_c) return LOGO_ERR_INVALID_ARG;
    if (prefix_len > 0 && (!k_prefix || !v_prefix)) return LOGO_ERR_INVALID_ARG;
    if (mass_out && !mass_in) return LOGO_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o_c) ||
        (prefix_len > 0 && (!aligned16(k_prefix) || !aligned16(v_prefix))))
        return LOGO_ERR_UNSUPPORTED;
    if (!(scale >= 0.0f)) return LOGO_ERR_INVALID_ARG;
    if (scale == 0.0f) scale = 1.0f / sqrtf(static_cast<float>(dims.D));
    const size_t need = prefix_ws_bytes(dims, n_new);
    if (!workspace || workspace_bytes < need || !aligned16(workspace)) return LOGO_ERR_WORKSPACE;
    PaParams p{};
    p.q = q;
    p.kp = k_prefix;
    p.vp = v_prefix;
    p.kc = k_cache;
    p.vc = v_cache;
    p.seq_len = seq_len;
    p.pos = pos;
    p.cu_q = cu_q;
    p.n_sel = n_sel_total;
    p.o = o_c;
    p.lse = lse_c ? lse_c : static_cast<float*>(workspace);
    p.mass_in = mass_in;
    p.mass_out = mass_out;
    p.B = dims.B;
    p.L = dims.T;
    p.Hq = dims.Hq;
    p.Hkv = dims.Hkv;
    p.n_new = n_new;
    p.P = prefix_len;
    p.cap = dims.B * n_new;
    p.scale_log2 = scale * kLog2e;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dims.D == 128 ? launch_prefix<128>(p, st) : launch_prefix<64>(p, st);
}
