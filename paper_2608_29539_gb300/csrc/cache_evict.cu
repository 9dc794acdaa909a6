// cache_evict.cu -- cuts a sequence's cache back to its budget by accumulated
// attention weight.
//
// One block per (sequence, KV head).  Every cache row has a 33-bit rank key:
// rows inside the recent window above all others, then the order-preserving
// image of the fp32 weight; equal keys go to the lower row.  A radix select
// finds the key of the last row that stays; one ordered pass then lists the
// holes (rows below `end` that go) and the movers (rows at or above `end` that
// stay) in rising order, and mover i is copied into hole i.  No mover's source
// is any mover's destination, so the copies need no order.
#include <cuda_bf16.h>

#include <cstdint>

#include "host_common.h"
#include "logo_status.cuh"

namespace logo {
namespace {

constexpr int kEvThreads = 1024;

struct EvParams {
    logo_bf16 *k, *v;
    const float* mass;
    const int32_t *slot_pos, *seq_len, *n_seen;
    float* mass_out;
    int32_t *pos_out, *new_len;
    int32_t* lists;  // [B * Hkv][L]: holes from the front, movers from the back
    int B, L, Hkv, D, budget, recent;
};

// Larger key: stays longer.  0xffffffff: inside the recent window; a float's
// image is below that; NaN: 0.
__device__ __forceinline__ uint32_t evict_key(float mass, int pos, int first_recent)
{
    if (pos >= first_recent) return 0xffffffffu;
    if (mass != mass) return 0u;
    const uint32_t u = __float_as_uint(mass + 0.0f);  // -0 -> +0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Exclusive sums over the block's 1024 threads of two counts below 2^16 each, packed.
__device__ __forceinline__ uint32_t block_excl_scan(uint32_t v, uint32_t* total, uint32_t* sh)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) sh[warp] = x;
    __syncthreads();
    if (warp == 0) {
        const uint32_t w0 = sh[lane];
        uint32_t w = w0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += y;
        }
        sh[lane] = w - w0;
        if (lane == 31) sh[32] = w;
    }
    __syncthreads();
    const uint32_t r = sh[warp] + x - v;
    *total = sh[32];
    __syncthreads();
    return r;
}

__global__ void __launch_bounds__(kEvThreads) evict_kernel(EvParams p)
{
    __shared__ uint32_t hist[256];
    __shared__ uint32_t sh_scan[33];
    __shared__ uint32_t sh_prefix;
    __shared__ int sh_need;
    const int bh = blockIdx.x, b = bh / p.Hkv, h = bh % p.Hkv;
    const int tid = threadIdx.x;
    const int len = max(0, min(p.seq_len[b], p.L));
    const int end = min(len, p.budget);
    const int64_t base = static_cast<int64_t>(bh) * p.L;
    const float* mass = p.mass + base;
    const int32_t* pos = p.slot_pos + base;
    if (h == 0 && tid == 0) p.new_len[b] = end;
    if (len <= p.budget) {
        for (int s = tid; s < len; s += kEvThreads) {
            const float m = mass[s];
            const int q = pos[s];
            p.mass_out[base + s] = m;
            p.pos_out[base + s] = q;
        }
        return;
    }
    const int first_recent = p.n_seen[b] - p.recent;
    // radix select: the key of the end-th largest, and how many rows with it stay
    uint32_t prefix = 0;
    int need = end;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int s = tid; s < len; s += kEvThreads) {
            const uint32_t k = evict_key(mass[s], pos[s], first_recent);
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            int d = 255, n = need;
            while (d > 0 && static_cast<int>(hist[d]) < n) n -= hist[d--];
            sh_prefix = prefix | (static_cast<uint32_t>(d) << shift);
            sh_need = n;
        }
        __syncthreads();
        prefix = sh_prefix;
        need = sh_need;
    }
    // ordered pass: ties, then holes and movers
    int32_t* lists = p.lists + base;
    uint32_t ties = 0, n_hole = 0, n_move = 0;
    for (int s0 = 0; s0 < len; s0 += kEvThreads) {
        const int s = s0 + tid;
        const uint32_t k = s < len ? evict_key(mass[s], pos[s], first_recent) : 0u;
        const bool tie = s < len && k == prefix;
        uint32_t total;
        const uint32_t tie_rank = ties + block_excl_scan(tie ? 1u : 0u, &total, sh_scan);
        ties += total;
        const bool keep = s < len && (k > prefix || (tie && tie_rank < static_cast<uint32_t>(need)));
        const bool hole = s < end && !keep, mover = s >= end && keep;
        const uint32_t r = block_excl_scan((hole ? 1u : 0u) | (mover ? 0x10000u : 0u), &total, sh_scan);
        if (hole) lists[n_hole + (r & 0xffffu)] = s;
        if (mover) lists[p.L - 1 - (n_move + (r >> 16))] = s;
        n_hole += total & 0xffffu;
        n_move += total >> 16;
        if (s < end && keep) {
            p.mass_out[base + s] = mass[s];
            p.pos_out[base + s] = pos[s];
        }
    }
    __syncthreads();  // the lists are written
    const int warp = tid >> 5, lane = tid & 31, vecs = p.D / 8;
    for (uint32_t i = warp; i < n_hole; i += kEvThreads / 32) {
        const int dst = lists[i], src = lists[p.L - 1 - i];
        if (lane < vecs) {
            const int64_t sr = ((static_cast<int64_t>(b) * p.L + src) * p.Hkv + h) * vecs + lane;
            const int64_t dr = ((static_cast<int64_t>(b) * p.L + dst) * p.Hkv + h) * vecs + lane;
            reinterpret_cast<uint4*>(p.k)[dr] = reinterpret_cast<const uint4*>(p.k)[sr];
            reinterpret_cast<uint4*>(p.v)[dr] = reinterpret_cast<const uint4*>(p.v)[sr];
        }
        if (lane == 0) {
            p.mass_out[base + dst] = mass[src];
            p.pos_out[base + dst] = pos[src];
        }
    }
}

int check_evict(const logo_dims& d)
{
    if (d.B < 1 || d.T < 1 || d.Hkv < 1 || d.D < 1) return LOGO_ERR_INVALID_ARG;
    if (d.D != 64 && d.D != 128) return LOGO_ERR_UNSUPPORTED;
    if (static_cast<int64_t>(d.B) * d.T > (1ll << 30)) return LOGO_ERR_UNSUPPORTED;
    if (static_cast<int64_t>(d.B) * d.Hkv > (1ll << 24)) return LOGO_ERR_UNSUPPORTED;
    return LOGO_OK;
}

size_t evict_ws_bytes(const logo_dims& d)
{
    return round_up(static_cast<size_t>(d.B) * d.Hkv * d.T * sizeof(int32_t), 256);
}

}  // namespace
}  // namespace logo

using namespace logo;

extern "C" size_t logo_cache_evict_workspace_size(logo_dims dims)
{
    if (check_evict(dims) != LOGO_OK) return 0;
    return evict_ws_bytes(dims);
}

extern "C" int logo_cache_evict(logo_bf16* k_cache, logo_bf16* v_cache, const float* mass, const int32_t* slot_pos,
                                const int32_t* seq_len, const int32_t* n_seen, float* mass_out,
                                int32_t* slot_pos_out, int32_t* new_len, logo_dims dims, int budget, int recent,
                                void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check_evict(dims);
    if (rc != LOGO_OK) return rc;
    if (!k_cache || !v_cache || !mass || !slot_pos || !seq_len || !n_seen || !mass_out || !slot_pos_out || !new_len)
        return LOGO_ERR_INVALID_ARG;
    if (new_len == seq_len) return LOGO_ERR_INVALID_ARG;
    if (budget < 1 || budget > dims.T || recent < 0 || recent > budget) return LOGO_ERR_INVALID_ARG;
    if (!aligned16(k_cache) || !aligned16(v_cache)) return LOGO_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < evict_ws_bytes(dims) || !aligned16(workspace)) return LOGO_ERR_WORKSPACE;
    EvParams p{};
    p.k = k_cache;
    p.v = v_cache;
    p.mass = mass;
    p.slot_pos = slot_pos;
    p.seq_len = seq_len;
    p.n_seen = n_seen;
    p.mass_out = mass_out;
    p.pos_out = slot_pos_out;
    p.new_len = new_len;
    p.lists = static_cast<int32_t*>(workspace);
    p.B = dims.B;
    p.L = dims.T;
    p.Hkv = dims.Hkv;
    p.D = dims.D;
    p.budget = budget;
    p.recent = recent;
    evict_kernel<<<dims.B * dims.Hkv, kEvThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return cudaGetLastError() == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}
