// cache4_attn.cu -- attention of new tokens over a cache held in 4 bits.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "cache4.cuh"
#include "host_common.h"

namespace logo {
namespace {

constexpr int kCaWarps = 4;

struct CaParams {
    const uint16_t* q;
    const uint8_t *k, *v, *ks, *vs;
    const int32_t *len, *pos, *cu_q, *n_sel;
    uint16_t* o;
    float* lse;
    int B, n, Hq, Hkv, L;
    float scale;
};

// Channels lane * C ... of a row, as floats.
template <int C>
__device__ __forceinline__ void row_values(const uint8_t* codes, const uint8_t* scales, int64_t row, int lane, float (&x)[C])
{
    const uint8_t* c = codes + (row * 32 + lane) * (C / 2);
    const float s = c4_scale(scales[row * (2 * C) + lane * C / kC4Group]);
#pragma unroll
    for (int j = 0; j < C / 2; ++j) {
        uint32_t h[4];
        c4_decode(c[j], h);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[0]));
        x[2 * j] = f.x * s, x[2 * j + 1] = f.y * s;
    }
}

// One CTA per packed row and query head, one cache row per warp at a time.
template <int D>
__global__ void __launch_bounds__(32 * kCaWarps) cache4_attn_kernel(CaParams p)
{
    constexpr int C = D / 32;
    __shared__ float sh_o[kCaWarps][D], sh_m[kCaWarps], sh_l[kCaWarps];
    const int hq = blockIdx.x % p.Hq, r = blockIdx.x / p.Hq;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (r >= min(*p.n_sel, p.B * p.n)) return;
    int b = 0;
    for (int hi = p.B - 1; b < hi;) {  // the last b with cu_q[b] <= r
        const int mid = (b + hi + 1) / 2;
        if (p.cu_q[mid] <= r) b = mid;
        else hi = mid - 1;
    }
    const int i = max(0, min(p.pos[r], p.n - 1));
    const int len = max(0, min(p.len[b], p.L));
    const int vis = min(len, max(0, len - p.n + i + 1));
    const int64_t head = (static_cast<int64_t>(b) * p.Hkv + hq / (p.Hq / p.Hkv)) * p.L;
    float q[C], o[C], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const uint16_t w = p.q[((static_cast<int64_t>(b) * p.n + i) * p.Hq + hq) * D + lane * C + c];
        q[c] = __uint_as_float(static_cast<uint32_t>(w) << 16);
        o[c] = 0.f;
    }
    for (int s = warp; s < vis; s += kCaWarps) {
        float x[C], dot = 0.f;
        row_values<C>(p.k, p.ks, head + s, lane, x);
#pragma unroll
        for (int c = 0; c < C; ++c) dot = fmaf(q[c], x[c], dot);
#pragma unroll
        for (int d = 16; d; d >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, d);
        dot *= p.scale;
        const float top = fmaxf(m, dot);
        const float keep = m == -INFINITY ? 0.f : expf(m - top), e = expf(dot - top);
        m = top;
        l = l * keep + e;
        row_values<C>(p.v, p.vs, head + s, lane, x);
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] = fmaf(e, x[c], o[c] * keep);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) sh_o[warp][lane * C + c] = o[c];
    if (lane == 0) sh_m[warp] = m, sh_l[warp] = l;
    __syncthreads();
    float top = -INFINITY, total = 0.f;
    for (int w = 0; w < kCaWarps; ++w) top = fmaxf(top, sh_m[w]);
    for (int w = 0; w < kCaWarps; ++w) total += sh_l[w] == 0.f ? 0.f : sh_l[w] * expf(sh_m[w] - top);
    if (threadIdx.x < D) {
        float sum = 0.f;
        for (int w = 0; w < kCaWarps; ++w)
            if (sh_l[w] != 0.f) sum += sh_o[w][threadIdx.x] * expf(sh_m[w] - top);
        const float out = vis ? sum / total : 0.f;
        p.o[(static_cast<int64_t>(r) * p.Hq + hq) * D + threadIdx.x] = __bfloat16_as_ushort(__float2bfloat16_rn(out));
    }
    if (threadIdx.x == 0 && p.lse) p.lse[static_cast<int64_t>(hq) * p.B * p.n + r] = vis ? top + logf(total) : -INFINITY;
}

int check_cache4_attn(const logo_dims& d, int n_new)
{
    if (n_new < 1) return LOGO_ERR_INVALID_ARG;
    const int rc = check_dims(d);
    if (rc != LOGO_OK) return rc;
    if (static_cast<int64_t>(d.B) * n_new > (1 << 24) || d.Hkv > (1 << 16) ||
        static_cast<int64_t>(n_new) * (d.Hq / d.Hkv) > 8192 || static_cast<int64_t>(d.B) * n_new * d.Hq > (1 << 30))
        return LOGO_ERR_UNSUPPORTED;
    return LOGO_OK;
}

}  // namespace
}  // namespace logo

using namespace logo;

extern "C" size_t logo_decode_cache4_workspace_size(logo_dims dims, int n_new)
{
    return check_cache4_attn(dims, n_new) == LOGO_OK ? 256 : 0;
}

extern "C" int logo_decode_cache4_attn(const logo_bf16* q, logo_cache4 cache, const int32_t* seq_len,
                                       const int32_t* pos, const int32_t* cu_q, const int32_t* n_sel_total,
                                       logo_bf16* o_c, float* lse_c, logo_dims dims, int n_new, float scale,
                                       void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check_cache4_attn(dims, n_new);
    if (rc != LOGO_OK) return rc;
    if (!q || !cache.k || !cache.v || !cache.k_scale || !cache.v_scale || !seq_len || !pos || !cu_q || !n_sel_total ||
        !o_c || !(scale >= 0.f) || std::isinf(scale))
        return LOGO_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(cache.k) || !aligned16(cache.v) || !aligned16(cache.k_scale) ||
        !aligned16(cache.v_scale) || !aligned16(o_c))
        return LOGO_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < logo_decode_cache4_workspace_size(dims, n_new) || !aligned16(workspace))
        return LOGO_ERR_WORKSPACE;
    CaParams p{q, cache.k, cache.v, cache.k_scale, cache.v_scale, seq_len, pos, cu_q, n_sel_total, o_c, lse_c,
               dims.B, n_new, dims.Hq, dims.Hkv, dims.T, scale > 0.f ? scale : 1.f / sqrtf(static_cast<float>(dims.D))};
    const unsigned blocks = static_cast<unsigned>(dims.B) * n_new * dims.Hq;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dims.D == 128) cache4_attn_kernel<128><<<blocks, 32 * kCaWarps, 0, st>>>(p);
    else cache4_attn_kernel<64><<<blocks, 32 * kCaWarps, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}
