// cache4.cu -- the 4-bit cache: new tokens quantised into it, rows read back.
#include <cuda_runtime.h>

#include <cstdint>

#include "cache4.cuh"
#include "host_common.h"

namespace logo {
namespace {

constexpr int kC4Threads = 256;

struct C4Params {
    const uint16_t *k_in, *v_in;   // append: [B, n, H, D]
    uint16_t *k_out, *v_out;       // read: [B, n, H, D]
    uint8_t *k, *v, *ks, *vs;      // [B, H, L, D/2], [B, H, L, D/16]
    const int32_t *len, *n_valid, *rows;
    int B, n, H, L;
};

// The largest magnitude of 16 bf16 channels, as bf16 bits.
__device__ __forceinline__ uint32_t amax16(const uint32_t (&a)[4], const uint32_t (&b)[4])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m = max(m, max((a[i] & 0x7fffu) , (a[i] >> 16) & 0x7fffu));
        m = max(m, max((b[i] & 0x7fffu) , (b[i] >> 16) & 0x7fffu));
    }
    return m;
}

__device__ __forceinline__ void load16(const uint16_t* p, uint32_t (&a)[4], uint32_t (&b)[4])
{
    const uint4 x = __ldg(reinterpret_cast<const uint4*>(p)), y = __ldg(reinterpret_cast<const uint4*>(p) + 1);
    a[0] = x.x, a[1] = x.y, a[2] = x.z, a[3] = x.w;
    b[0] = y.x, b[1] = y.y, b[2] = y.z, b[3] = y.w;
}

// One group of 16 channels of one (sequence, KV head, token) a thread.
template <int D>
__global__ void __launch_bounds__(kC4Threads) append_kernel(C4Params p)
{
    constexpr int NG = D / kC4Group;
    const int64_t unit = (static_cast<int64_t>(blockIdx.x) * kC4Threads + threadIdx.x);
    const int g = unit % NG;
    const int64_t tok = unit / NG;  // (b, i, h)
    if (tok >= static_cast<int64_t>(p.B) * p.n * p.H) return;
    const int h = tok % p.H;
    const int i = tok / p.H % p.n;
    const int b = tok / p.H / p.n;
    const int nv = p.n_valid ? max(0, min(p.n_valid[b], p.n)) : p.n;
    const int64_t row = static_cast<int64_t>(p.len[b]) - nv + i;
    if (i >= nv || row < 0 || row >= p.L) return;
    const int64_t dst = (static_cast<int64_t>(b) * p.H + h) * p.L + row;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        uint32_t lo[4], hi[4];
        load16((side ? p.v_in : p.k_in) + tok * D + g * kC4Group, lo, hi);
        const uint32_t code = c4_scale_code(amax16(lo, hi));
        const float inv = c4_inverse(code);
        reinterpret_cast<uint2*>((side ? p.v : p.k) + dst * (D / 2))[g] = make_uint2(c4_codes(lo, inv), c4_codes(hi, inv));
        ((side ? p.vs : p.ks) + dst * NG)[g] = code;
    }
}

template <int D>
__global__ void __launch_bounds__(kC4Threads) read_kernel(C4Params p)
{
    constexpr int NG = D / kC4Group;
    const int64_t unit = (static_cast<int64_t>(blockIdx.x) * kC4Threads + threadIdx.x);
    const int g = unit % NG;
    const int64_t tok = unit / NG;  // (b, i, h)
    if (tok >= static_cast<int64_t>(p.B) * p.n * p.H) return;
    const int h = tok % p.H;
    const int i = tok / p.H % p.n;
    const int b = tok / p.H / p.n;
    const int row = p.rows ? p.rows[static_cast<int64_t>(b) * p.n + i] : i;
    const bool held = row >= 0 && row < min(p.len[b], p.L);
    const int64_t src = (static_cast<int64_t>(b) * p.H + h) * p.L + row;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (held) {
            const uint2 c = reinterpret_cast<const uint2*>((side ? p.v : p.k) + src * (D / 2))[g];
            const uint32_t s = c4_scale_f16(((side ? p.vs : p.ks) + src * NG)[g]) * 0x10001u;
            uint32_t x[4];
            c4_decode(c.x, x);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = c4_to_bf16x2(h2_mul(x[j], s));
            c4_decode(c.y, x);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[4 + j] = c4_to_bf16x2(h2_mul(x[j], s));
        }
        uint4* out = reinterpret_cast<uint4*>((side ? p.v_out : p.k_out) + tok * D + g * kC4Group);
        out[0] = make_uint4(w[0], w[1], w[2], w[3]);
        out[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

int check_cache4(const logo_cache4& c, const logo_dims& d, int n)
{
    if (n < 1) return LOGO_ERR_INVALID_ARG;
    const logo_dims kv{d.B, d.T, d.Hkv, d.Hkv, d.D};
    const int rc = check_dims(kv);
    if (rc != LOGO_OK) return rc;
    if (!c.k || !c.v || !c.k_scale || !c.v_scale) return LOGO_ERR_INVALID_ARG;
    if (!aligned16(c.k) || !aligned16(c.v) || !aligned16(c.k_scale) || !aligned16(c.v_scale)) return LOGO_ERR_UNSUPPORTED;
    // rows of the new tokens or of the list: a thread a group has to be countable by the grid
    if (static_cast<int64_t>(d.B) * n > (1ll << 30) || d.Hkv > (1 << 16) ||
        static_cast<int64_t>(d.B) * n * d.Hkv > (1ll << 34))
        return LOGO_ERR_UNSUPPORTED;
    return LOGO_OK;
}

int64_t c4_blocks(const C4Params& p, int D)
{
    return (static_cast<int64_t>(p.B) * p.n * p.H * (D / kC4Group) + kC4Threads - 1) / kC4Threads;
}

}  // namespace
}  // namespace logo

using namespace logo;

extern "C" int logo_cache4_append(logo_cache4 cache, const logo_bf16* k_new, const logo_bf16* v_new,
                                  const int32_t* seq_len, const int32_t* n_valid, logo_dims dims, int n_new,
                                  void* stream)
{
    const int rc = check_cache4(cache, dims, n_new);
    if (rc != LOGO_OK) return rc;
    if (!k_new || !v_new || !seq_len) return LOGO_ERR_INVALID_ARG;
    if (!aligned16(k_new) || !aligned16(v_new)) return LOGO_ERR_UNSUPPORTED;
    C4Params p{};
    p.k_in = k_new, p.v_in = v_new, p.k = cache.k, p.v = cache.v, p.ks = cache.k_scale, p.vs = cache.v_scale;
    p.len = seq_len, p.n_valid = n_valid, p.B = dims.B, p.n = n_new, p.H = dims.Hkv, p.L = dims.T;
    const unsigned blocks = static_cast<unsigned>(c4_blocks(p, dims.D));
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dims.D == 128) append_kernel<128><<<blocks, kC4Threads, 0, st>>>(p);
    else append_kernel<64><<<blocks, kC4Threads, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}

extern "C" int logo_cache4_read(logo_cache4 cache, const int32_t* seq_len, const int32_t* rows, logo_bf16* k,
                                logo_bf16* v, logo_dims dims, int m, void* stream)
{
    const int rc = check_cache4(cache, dims, m);
    if (rc != LOGO_OK) return rc;
    if (!k || !v || !seq_len) return LOGO_ERR_INVALID_ARG;
    if (!aligned16(k) || !aligned16(v)) return LOGO_ERR_UNSUPPORTED;
    C4Params p{};
    p.k_out = k, p.v_out = v, p.k = cache.k, p.v = cache.v, p.ks = cache.k_scale, p.vs = cache.v_scale;
    p.len = seq_len, p.rows = rows, p.B = dims.B, p.n = m, p.H = dims.Hkv, p.L = dims.T;
    const unsigned blocks = static_cast<unsigned>(c4_blocks(p, dims.D));
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dims.D == 128) read_kernel<128><<<blocks, kC4Threads, 0, st>>>(p);
    else read_kernel<64><<<blocks, kC4Threads, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}
