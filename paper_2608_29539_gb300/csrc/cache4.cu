// cache4.cu -- the 4-bit cache: new tokens quantised into it, rows read back.
//
// HBM bounds both: 2 bytes a channel on one side, 0.5625 on the other.  Tokens come in as
// [tokens][KV heads][D] and lie in the cache as [KV heads][rows][D], so a warp takes one
// head of 512 / D consecutive tokens: pieces of 2 D bytes on the one side, 256 bytes of
// codes and 32 of scales in a row on the other.  Writing and reading back 8 x 8187 tokens of
// 8 heads, D = 128: 98 us, 94% of the copy rate (groups of 16 channels in the tokens' order,
// which write 8 bytes here and there: 124); 32 x 2048 rows by number: 68 us, as a row's 8
// bytes of scales cost a sector of 32.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "cache4.cuh"
#include "host_common.h"

namespace logo {
namespace {

constexpr int kC4Threads = 256;
constexpr int kC4Warps = kC4Threads / 32;
constexpr int kC4Take = 2;   // pieces of a warp at a time

struct C4Params {
    const uint16_t *k_in, *v_in;   // append: [B, n, H, D]
    uint16_t *k_out, *v_out;       // read: [B, n, H, D]
    uint8_t *k, *v, *ks, *vs;      // [B, H, L, D/2], [B, H, L, D/16]
    const int32_t *len, *n_valid, *rows;
    int B, n, H, L;
    int tiles;                     // of tokens, a sequence
    int pieces;                    // of a tile: a head of 512 / D tokens each
};

// Tokens of a warp's piece.
template <int D>
constexpr int kC4Tokens = 512 / D;

// The largest magnitude of 16 bf16 channels, as bf16 bits.
__device__ __forceinline__ uint32_t amax16(const uint4& a, const uint4& b)
{
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i] & 0x7fff7fffu));
    return max(m & 0xffffu, m >> 16);
}

// A piece's first token and head.
template <int D>
__device__ __forceinline__ int2 piece_of(const C4Params& p, int tile, int piece)
{
    const int quad = piece / p.H;
    return make_int2(tile * (p.pieces / p.H) * kC4Tokens<D> + quad * kC4Tokens<D>, piece - quad * p.H);
}

// A thread a group of 16 channels of a token, K and V.
template <int D>
__global__ void __launch_bounds__(kC4Threads) append_kernel(C4Params p)
{
    constexpr int NG = D / kC4Group;
    const int b = blockIdx.x / p.tiles, tile = blockIdx.x - b * p.tiles;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane % NG;
    const int nv = p.n_valid ? max(0, min(p.n_valid[b], p.n)) : p.n;
    const int64_t base = static_cast<int64_t>(p.len[b]) - nv;  // the cache row of token 0
#pragma unroll 1
    for (int piece0 = warp; piece0 < p.pieces; piece0 += kC4Warps * kC4Take) {
        uint4 w[kC4Take][2][2];
        int64_t to[kC4Take];  // -1: nothing
#pragma unroll
        for (int t = 0; t < kC4Take; ++t) {
            const int2 at = piece_of<D>(p, tile, piece0 + t * kC4Warps);
            const int i = at.x + lane / NG;
            const int64_t row = base + i;
            const bool in = piece0 + t * kC4Warps < p.pieces && i < nv && row >= 0 && row < p.L;
            to[t] = in ? (static_cast<int64_t>(b) * p.H + at.y) * p.L + row : -1;
            const int64_t from = ((static_cast<int64_t>(b) * p.n + i) * p.H + at.y) * D + g * kC4Group;
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                const uint4* src = reinterpret_cast<const uint4*>((side ? p.v_in : p.k_in) + (in ? from : 0));
                w[t][side][0] = in ? __ldcs(src) : make_uint4(0, 0, 0, 0);
                w[t][side][1] = in ? __ldcs(src + 1) : make_uint4(0, 0, 0, 0);
            }
        }
#pragma unroll
        for (int t = 0; t < kC4Take; ++t) {
            if (to[t] < 0) continue;
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                const uint4 x = w[t][side][0], y = w[t][side][1];
                const uint32_t code = c4_scale_code(amax16(x, y));
                const float inv = c4_inverse(code);
                const uint32_t lo[4] = {x.x, x.y, x.z, x.w}, hi[4] = {y.x, y.y, y.z, y.w};
                reinterpret_cast<uint2*>((side ? p.v : p.k) + to[t] * (D / 2))[g] = make_uint2(c4_codes(lo, inv), c4_codes(hi, inv));
                ((side ? p.vs : p.ks) + to[t] * NG)[g] = static_cast<uint8_t>(code);
            }
        }
    }
}

// A thread eight channels of two tokens of the piece, K and V.
template <int D>
__global__ void __launch_bounds__(kC4Threads) read_kernel(C4Params p)
{
    constexpr int NE = D / 8;  // threads a token
    const int b = blockIdx.x / p.tiles, tile = blockIdx.x - b * p.tiles;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane % NE;
    const int len = min(p.len[b], p.L);
#pragma unroll 1
    for (int piece = warp; piece < p.pieces; piece += kC4Warps) {
        const int2 at = piece_of<D>(p, tile, piece);
        uint32_t code[2][2], scale[2][2];
        int i[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            i[t] = at.x + lane / NE + t * (32 / NE);
            int row = -1;
            if (i[t] < p.n) row = p.rows ? p.rows[static_cast<int64_t>(b) * p.n + i[t]] : i[t];
            const bool held = row >= 0 && row < len;
            const int64_t src = (static_cast<int64_t>(b) * p.H + at.y) * p.L + row;
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                code[t][side] = held ? reinterpret_cast<const uint32_t*>((side ? p.v : p.k) + src * (D / 2))[c] : 0;
                scale[t][side] = held ? ((side ? p.vs : p.ks) + src * (D / 16))[c / 2] : 0;
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if (i[t] >= p.n) continue;
            const int64_t to = ((static_cast<int64_t>(b) * p.n + i[t]) * p.H + at.y) * D + c * 8;
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                uint32_t x[4];
                c4_decode(code[t][side], x);
                const uint32_t s = scale[t][side] * 0x800080u;  // the scale's f16 twice
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = c4_to_bf16x2(h2_mul(x[j], s));
                *reinterpret_cast<uint4*>((side ? p.v_out : p.k_out) + to) = make_uint4(x[0], x[1], x[2], x[3]);
            }
        }
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
    // the tiles of the new tokens or of the list have to be countable by the grid
    if (static_cast<int64_t>(d.B) * n > (1ll << 30) || d.Hkv > (1 << 16) ||
        static_cast<int64_t>(d.B) * n * d.Hkv > (1ll << 34))
        return LOGO_ERR_UNSUPPORTED;
    return LOGO_OK;
}

// Cuts each sequence's tokens into tiles of about `want` pieces, at least; the grid.
int64_t c4_tiles(C4Params& p, int D, int want)
{
    const int tokens = 512 / D, quads = (p.n + tokens - 1) / tokens;  // a piece's tokens, pieces of a head
    const int per = std::max(1, std::min(quads, want / p.H));
    p.tiles = (quads + per - 1) / per;
    p.pieces = per * p.H;
    return static_cast<int64_t>(p.B) * p.tiles;
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
    const unsigned blocks = static_cast<unsigned>(c4_tiles(p, dims.D, kC4Warps * kC4Take));
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
    const size_t bytes = static_cast<size_t>(dims.B) * m * dims.Hkv * dims.D * sizeof(logo_bf16);
    if (overlap(k, bytes, v, bytes)) return LOGO_ERR_INVALID_ARG;
    C4Params p{};
    p.k_out = k, p.v_out = v, p.k = cache.k, p.v = cache.v, p.ks = cache.k_scale, p.vs = cache.v_scale;
    p.len = seq_len, p.rows = rows, p.B = dims.B, p.n = m, p.H = dims.Hkv, p.L = dims.T;
    const unsigned blocks = static_cast<unsigned>(c4_tiles(p, dims.D, kC4Warps));
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dims.D == 128) read_kernel<128><<<blocks, kC4Threads, 0, st>>>(p);
    else read_kernel<64><<<blocks, kC4Threads, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}
