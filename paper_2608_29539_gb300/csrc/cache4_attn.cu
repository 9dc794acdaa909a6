// cache4_attn.cu -- attention of new tokens over a cache held in 4 bits.
//
// For the new tokens' rows r of a sequence (packed rows times the query heads of a KV
// head) and its cache rows s:  x_rs = scale q_r.k_s,  o_r = sum_s e^(x_rs - m_r) v_s /
// sum_s e^(x_rs - m_r), one pass with a running maximum.
//
// The work is the bytes: 0.5625 D a cache row, K and V each, read once for all rows of
// a KV head.  At the HBM rate an SM has to turn 40 codes a clock into operands, so what
// bounds the kernel is instructions: everything is laid out so that a code costs one
// conversion (two codes) and one product with its scale (two codes).
//   - Warp-level MMA m16n8k16 with the keys (S^T = K Q^T) and the channels (O^T = V^T
//     P^T) as the 16 rows and 8 query rows as the columns: few query rows leave little
//     of a tile empty, and the softmax's work is spread over the keys.
//   - The order of a product's terms is free, so a thread takes for its fragments of K
//     32 consecutive channels of a key (one 16-byte load) and for V one scale's group of
//     4 keys (one 8-byte load a key).  V's pairs along the keys are made by exchanging
//     nibbles of two keys' words, before the conversion.
//   - code * scale is exact in fp16.  Queries go through fp16 scaled by a power of two
//     a row.  P is rounded to fp16; it comes out of S^T's fragments by a transposition
//     in registers.
// The batch's (sequence, KV head, 32 rows, 128 keys) units form a line, sequences
// without a selected row left out; each CTA takes an equal stretch of it, its four warps
// 32 keys of a unit each through a ring of their own in shared memory (cp.async; no warp
// waits for another before a stretch of one run ends).  A run (sequence, KV head, rows)
// that spans several CTAs is joined by a second launch from their parts, in order.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "cache4.cuh"
#include "host_common.h"
#include "sm100.cuh"

namespace logo {
namespace {

constexpr int kCaWarps = 4;
constexpr int kCaThreads = 32 * kCaWarps;
constexpr int kCaKeys = 32;                   // keys of a warp's step
constexpr int kCaUnit = kCaKeys * kCaWarps;   // keys of a unit
constexpr int kCaStages = 2;
constexpr float kCaSlack = 8.f;               // a maximum may grow by 2^8 before what is summed is rescaled
constexpr int kCaMaxTiles = 4;                // tiles of 8 rows that a warp holds

struct CaParams {
    const uint16_t* q;
    const uint8_t *k, *v, *ks, *vs;
    const int32_t *len, *pos, *cu_q, *n_sel;
    uint16_t* o;
    float* lse;
    float* parts;   // [2 * grid][rows * D, then rows of (max, sum)]
    int4* table;    // [grid]: (sequence or -1, KV head, row block, last CTA) of the run that goes on past a CTA's end
    int B, n, Hq, Hkv, G, L;
    float scale2;   // scale * log2(e)
};

template <int D, int NT>
struct CaShape {
    static constexpr int kRows = 8 * NT;
    static constexpr int kCodes = kCaKeys * D / 2, kScales = kCaKeys * D / 16;  // bytes a step, K or V
    static constexpr int kStage = 2 * (kCodes + kScales);
    static constexpr int kSteps = D / 16;                      // k steps of S^T, m tiles of O^T
    static constexpr int kRowBytes = 4 * D + 16;               // a row of the warps' results (padded for the banks)
    static constexpr int kRing = kCaWarps * kCaStages * kStage;
    static constexpr int kQ = NT * kSteps * 32 * 8;            // fragments of Q
    static constexpr int kMerge = kCaWarps * kRows * kRowBytes;
    static constexpr int kSmem = kRing + kQ + kMerge + kCaWarps * kRows * 8 + kRows * 8;
    static constexpr int kPart = kRows * (D + 2);              // floats of a part
    static constexpr int kCtas = NT == 1 ? 4 : NT == 2 ? 3 : 2;  // an SM
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

template <int N>
__device__ __forceinline__ void cp_async_small(uint32_t dst, const void* src, uint32_t bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(N), "r"(bytes) : "memory");
}

__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }

template <int N>
__device__ __forceinline__ void cp_async_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ uint2 ld_shared_v2(uint32_t addr)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
    return v;
}

__device__ __forceinline__ uint32_t ld_shared_u16(uint32_t addr)
{
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr));
    return v;
}

__device__ __forceinline__ uint32_t ld_shared_u8(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ uint32_t dup16(uint32_t x) { return __byte_perm(x, 0, 0x1010); }

// Where byte `at` (a multiple of 4) of a step's key row lies: the 16-byte pieces of
// 128-byte lines exchanged so that both kinds of loads below meet every bank once.
template <int D>
__device__ __forceinline__ uint32_t piece(uint32_t key, uint32_t at)
{
    const uint32_t x = key * (D / 2) + at, line = x >> 7;
    const uint32_t f = D == 128 ? ((line & 1) << 1) | ((line & 2) << 1) : (line & 1) << 2;
    return x ^ (f << 4);
}

// A run: the units of one (sequence, KV head, row block), in the line's order.
struct CaRun {
    int b, h, rb;
    int nrb, units, len, r0, cnt;   // of the sequence
};

// Whether sequence b has selected rows; its part of the run's description.
__device__ __forceinline__ bool ca_sequence(const CaParams& p, int b, int rows, CaRun& r)
{
    const int n_sel = *p.n_sel;
    r.r0 = p.cu_q[b];
    r.cnt = min(min(p.cu_q[b + 1], n_sel) - r.r0, p.n);
    if (r.cnt <= 0) return false;
    r.b = b;
    r.len = max(0, min(p.len[b], p.L));
    r.units = max(1, (r.len + kCaUnit - 1) / kCaUnit);
    r.nrb = (r.cnt * p.G + rows - 1) / rows;
    return true;
}

__device__ __forceinline__ void ca_next(const CaParams& p, int rows, CaRun& r)
{
    if (++r.rb < r.nrb) return;
    r.rb = 0;
    if (++r.h < p.Hkv) return;
    r.h = 0;
    for (int b = r.b + 1; b < p.B; ++b)
        if (ca_sequence(p, b, rows, r)) return;
    r.units = 0;  // the line's end
}

__device__ __forceinline__ long long ca_weight(const CaParams& p, int b, int rows)
{
    CaRun r;
    return b < p.B && ca_sequence(p, b, rows, r) ? static_cast<long long>(r.units) * r.nrb * p.Hkv : 0;
}

// The line's length and, for a place x on it that depends on the length, the sequence
// that holds it and where its units begin.  All threads of the CTA.
struct CaLine {
    long long total, x0, x1, base;
    int b;
};

__device__ __forceinline__ void ca_line(const CaParams& p, int rows, CaLine& at, long long* sh)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long w = 0;
    for (int b = threadIdx.x; b < p.B; b += kCaThreads) w += ca_weight(p, b, rows);
#pragma unroll
    for (int d = 16; d; d >>= 1) w += __shfl_xor_sync(0xffffffffu, w, d);
    if (lane == 0) sh[warp] = w;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int i = 0; i < kCaWarps; ++i) total += sh[i];
    const long long ctas = min(static_cast<long long>(gridDim.x), total);
    at.total = total;
    at.x0 = at.x1 = 0;
    if (blockIdx.x >= ctas) return;
    at.x0 = total * blockIdx.x / ctas;
    at.x1 = total * (blockIdx.x + 1) / ctas;
    long long base = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {  // every warp for itself
        const long long mine = ca_weight(p, b0 + lane, rows);
        long long upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += y;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, base + upto > at.x0);
        if (past) {
            const int k = __ffs(past) - 1;
            at.b = b0 + k;
            at.base = base + __shfl_sync(0xffffffffu, upto - mine, k);
            return;
        }
        base += __shfl_sync(0xffffffffu, upto, 31);
    }
}

template <int D, int NT>
__global__ void __launch_bounds__(kCaThreads, CaShape<D, NT>::kCtas) cache4_attn_kernel(CaParams p)
{
    using S = CaShape<D, NT>;
    constexpr int NS = S::kSteps;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long sh_line[kCaWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t ring = smem_u32(smem) + warp * (kCaStages * S::kStage);
    uint2* const q_frag = reinterpret_cast<uint2*>(smem + S::kRing);
    uint8_t* const merge = smem + S::kRing + S::kQ;
    float2* const stats = reinterpret_cast<float2*>(merge + S::kMerge);  // [warp][row] (max, sum)
    int* const row_vis = reinterpret_cast<int*>(stats + kCaWarps * S::kRows);
    float* const row_mul = reinterpret_cast<float*>(row_vis + S::kRows);

    CaLine at;
    ca_line(p, S::kRows, at, sh_line);
    int4 goes_on = make_int4(-1, 0, 0, 0);
    if (at.x0 < at.x1) {
        const long long ctas = min(static_cast<long long>(gridDim.x), at.total);
        CaRun run{};
        ca_sequence(p, at.b, S::kRows, run);
        long long off = at.x0 - at.base;
        run.h = static_cast<int>(off / (static_cast<long long>(run.units) * run.nrb));
        off -= static_cast<long long>(run.h) * run.units * run.nrb;
        run.rb = static_cast<int>(off / run.units);
        int unit = static_cast<int>(off - static_cast<long long>(run.rb) * run.units);

        // ---- loads: a cursor of its own, kCaStages - 1 units ahead
        CaRun ahead = run;
        int ahead_unit = unit;
        long long ahead_left = at.x1 - at.x0;
        uint32_t fill = 0;
        auto issue = [&] {
            if (ahead_left > 0) {
                const int key0 = ahead_unit * kCaUnit + warp * kCaKeys;
                if (key0 < ahead.len) {
                    const uint32_t st = ring + fill * S::kStage;
                    const int64_t row0 = (static_cast<int64_t>(ahead.b) * p.Hkv + ahead.h) * p.L + key0;
                    const int rows = ahead.len - key0;  // rows past the end are written as zeros
#pragma unroll
                    for (int i = 0; i < S::kCodes / 512; ++i) {
                        const uint32_t x = (i * 32 + lane) * 16, key = x / (D / 2);
                        const bool in = static_cast<int>(key) < rows;
                        const uint32_t to = st + piece<D>(key, x % (D / 2));
                        const int64_t from = in ? row0 * (D / 2) + x : 0;
                        cp_async16(to, p.k + from, in ? 16 : 0);
                        cp_async16(to + S::kCodes, p.v + from, in ? 16 : 0);
                    }
                    const bool in = lane < rows;
                    const int64_t from = in ? (row0 + lane) * (D / 16) : 0;
                    const uint32_t to = st + 2 * S::kCodes + lane * (D / 16);
                    cp_async_small<D / 16>(to, p.ks + from, in ? D / 16 : 0);
                    cp_async_small<D / 16>(to + S::kScales, p.vs + from, in ? D / 16 : 0);
                }
                --ahead_left;
                if (++ahead_unit == ahead.units) {
                    ahead_unit = 0;
                    if (ahead_left > 0) ca_next(p, S::kRows, ahead);
                }
            }
            cp_async_commit();
            fill = fill + 1 == kCaStages ? 0 : fill + 1;
        };
#pragma unroll
        for (int i = 0; i < kCaStages - 1; ++i) issue();

        uint32_t use = 0;
        for (long long left = at.x1 - at.x0; left > 0;) {
            // ---- a stretch of one run
            const int first = unit, last = static_cast<int>(min(static_cast<long long>(run.units), unit + left));
            const int row0 = run.rb * S::kRows, nrow = min(S::kRows, run.cnt * p.G - row0);
            const int tiles = NT == 1 ? 1 : (nrow + 7) / 8;
            __syncthreads();  // the rows of the stretch before are no longer read
            for (int r = warp; r < S::kRows; r += kCaWarps) {
                uint2 w = make_uint2(0, 0);
                int vis = 0;
                if (r < nrow) {
                    const int i = max(0, min(p.pos[run.r0 + (row0 + r) / p.G], p.n - 1));
                    const int64_t at_q = ((static_cast<int64_t>(run.b) * p.n + i) * p.Hq + run.h * p.G + (row0 + r) % p.G) * D;
                    if (lane < D / 4) w = __ldg(reinterpret_cast<const uint2*>(p.q + at_q) + lane);
                    vis = min(run.len, max(0, run.len - p.n + i + 1));
                }
                // the row times 2^(140 - e), e the largest exponent: below 2^14
                uint32_t top = 0;
                uint32_t bits[4] = {w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t e = bits[j] >> 23 & 0xff;
                    if (e != 0xff) top = max(top, e);
                }
                top = max(16u, __reduce_max_sync(0xffffffffu, top));
                const float up = __uint_as_float((267u - top) << 23);
                float f[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    f[j] = (bits[j] >> 23 & 0xff) == 0xff ? __uint_as_float(0x7fc00000u) : __uint_as_float(bits[j]) * up;
                if (lane < D / 4)  // channels 4 lane ... 4 lane + 3: of thread lane / NS, step lane % NS
                    q_frag[((r >> 3) * NS + lane % NS) * 32 + (r & 7) * 4 + lane / NS] =
                        make_uint2(pack_f16(f[0], f[1]), pack_f16(f[2], f[3]));
                if (lane == 0) {
                    row_vis[r] = vis;
                    // (2^(top - 140) alone may not be a normal number)
                    row_mul[r] = fmaxf(ldexpf(p.scale2, static_cast<int>(top) - 140), 1.2e-38f);
                }
            }
            __syncthreads();
            float mul[NT][2], m[NT][2], l[NT][2], o[NT][NS][4];
            int vis[NT][2], vis_min = run.len;
            uint2 q1[NS];
            if (NT == 1)
#pragma unroll
                for (int ks = 0; ks < NS; ++ks) q1[ks] = q_frag[ks * 32 + lane];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int r = nt * 8 + 2 * t + j;
                    mul[nt][j] = row_mul[r], vis[nt][j] = row_vis[r];
                    m[nt][j] = -INFINITY, l[nt][j] = 0.f;
#pragma unroll
                    for (int i = 0; i < NS; ++i) o[nt][i][j] = o[nt][i][j + 2] = 0.f;
                }
            for (int r = lane; r < nrow; r += 32) vis_min = min(vis_min, row_vis[r]);
            vis_min = __reduce_min_sync(0xffffffffu, vis_min);

            for (; unit < last; ++unit, --left) {
                cp_async_wait<kCaStages - 2>();
                __syncwarp();
                issue();
                const uint32_t st = ring + use * S::kStage;
                use = use + 1 == kCaStages ? 0 : use + 1;
                const int key0 = unit * kCaUnit + warp * kCaKeys;
                if (key0 >= run.len) continue;
                // ---- S^T: row g of a tile is key (g >> 1) + 4 (g & 1), row g + 8 that plus 8
                float s[2][NT][4];
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[mt][nt][j] = 0.f;
                {
                    uint32_t kw[2][2][NS / 2], sc[2][2];
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t key = 16 * mt + 8 * e + (g >> 1) + 4 * (g & 1);
                            const uint32_t sa = st + 2 * S::kCodes + key * (D / 16);
                            if (D == 128) {
                                const uint4 x = ld_shared_v4(st + piece<D>(key, 16 * t));
                                kw[mt][e][0] = x.x, kw[mt][e][1] = x.y, kw[mt][e][2 % (NS / 2)] = x.z;
                                kw[mt][e][3 % (NS / 2)] = x.w;
                                sc[mt][e] = ld_shared_u16(sa + 2 * t);
                            } else {
                                const uint2 x = ld_shared_v2(st + piece<D>(key, 8 * t));
                                kw[mt][e][0] = x.x, kw[mt][e][1] = x.y;
                                sc[mt][e] = ld_shared_u8(sa + t);
                            }
                        }
#pragma unroll
                    for (int w = 0; w < NS / 2; ++w) {
                        uint32_t h[2][2][4];
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                c4_decode(kw[mt][e][w], h[mt][e]);
                                const uint32_t code = D == 128 && w >= NS / 4 ? sc[mt][e] >> 8 : sc[mt][e] & 0xff;
                                const uint32_t f = dup16(c4_scale_f16(code));
#pragma unroll
                                for (int j = 0; j < 4; ++j) h[mt][e][j] = h2_mul(h[mt][e][j], f);
                            }
#pragma unroll
                        for (int half = 0; half < 2; ++half)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                if (NT > 1 && nt >= tiles) break;
                                const uint2 qf = NT == 1 ? q1[2 * w + half] : q_frag[(nt * NS + 2 * w + half) * 32 + lane];
#pragma unroll
                                for (int mt = 0; mt < 2; ++mt) {
                                    const uint32_t a[4] = {h[mt][0][2 * half], h[mt][1][2 * half], h[mt][0][2 * half + 1],
                                                           h[mt][1][2 * half + 1]};
                                    mma_f16(s[mt][nt], a, qf.x, qf.y);
                                }
                            }
                    }
                }
                // ---- what a row does not see; softmax
                const bool cut = key0 + kCaKeys > vis_min;
                const bool drafts = cut && vis_min < run.len;  // keys that some rows see and some do not
                uint32_t pb[2][NT][2];
                uint32_t vb[2][NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    if (NT > 1 && nt >= tiles) break;
                    if (cut) {
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt) {
                            const int key = key0 + 16 * mt + (g >> 1) + 4 * (g & 1);
                            bool in[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                in[j] = key + 8 * (j >> 1) < vis[nt][j & 1];
                                if (!in[j]) s[mt][nt][j] = -INFINITY;
                            }
                            vb[mt][nt][0] = (in[0] ? 0x3c00u : 0u) | (in[1] ? 0x3c000000u : 0u);
                            vb[mt][nt][1] = (in[2] ? 0x3c00u : 0u) | (in[3] ? 0x3c000000u : 0u);
                        }
                    }
                    float top[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        top[j] = fmaxf(fmaxf(s[0][nt][j], s[0][nt][j + 2]), fmaxf(s[1][nt][j], s[1][nt][j + 2])) * mul[nt][j];
                    if (__any_sync(0xffffffffu, top[0] > m[nt][0] + kCaSlack || top[1] > m[nt][1] + kCaSlack)) {
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], d));
                            const float now = fmaxf(m[nt][j], top[j]);
                            const float keep = m[nt][j] == -INFINITY ? 0.f : ex2_approx(m[nt][j] - now);
                            // (a sum that is NaN stays so; nothing but zeros is summed where m is -infinity)
                            l[nt][j] = m[nt][j] == -INFINITY ? l[nt][j] : l[nt][j] * keep;
#pragma unroll
                            for (int i = 0; i < NS; ++i) {
                                o[nt][i][j] *= keep;
                                o[nt][i][j + 2] *= keep;
                            }
                            m[nt][j] = now;
                        }
                    }
                    const float mu[2] = {m[nt][0] == -INFINITY ? 0.f : m[nt][0], m[nt][1] == -INFINITY ? 0.f : m[nt][1]};
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        float e[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            e[j] = ex2_approx(fmaf(s[mt][nt][j], mul[nt][j & 1], -mu[j & 1]));
                            l[nt][j & 1] += e[j];
                        }
                        pb[mt][nt][0] = transpose8(pack_f16(e[0], e[1]));
                        pb[mt][nt][1] = transpose8(pack_f16(e[2], e[3]));
                    }
                }
                // ---- O^T: columns 2t, 2t + 1, 2t + 8, 2t + 9 of a tile are keys t, t + 4, t + 8, t + 12
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    uint32_t vw[4][NS / 4], f[2];
                    {
                        uint32_t code[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t key = 16 * mt + 4 * j + t;
                            const uint32_t va = st + S::kCodes;
                            if (D == 128) {
                                const uint2 x = ld_shared_v2(va + piece<D>(key, 8 * g));
                                vw[j][0] = x.x, vw[j][1 % (NS / 4)] = x.y;
                            } else {
                                vw[j][0] = ld_shared_u32(va + piece<D>(key, 4 * g));
                            }
                            code[j] = ld_shared_u8(st + 2 * S::kCodes + S::kScales + key * (D / 16) + (D == 128 ? g : g >> 1));
                        }
                        f[0] = (code[0] << 7) | (code[1] << 23);
                        f[1] = (code[2] << 7) | (code[3] << 23);
                    }
                    if (drafts) {
                        // a value that is not finite counts for the rows that see it alone: its product is
                        // left out, and the rows that see it are found by a product of their own
                        uint32_t bad[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const uint32_t lo = (f[j] & 0x7c00u) == 0x7c00u ? 0xffffu : 0u;
                            const uint32_t hi = (f[j] & 0x7c000000u) == 0x7c000000u ? 0xffff0000u : 0u;
                            bad[j] = lo | hi;
                            f[j] &= ~bad[j];
                        }
                        if (__any_sync(0xffffffffu, (bad[0] | bad[1]) != 0)) {
                            const uint32_t a[4] = {bad[0] & 0x3c003c00u, 0u, bad[1] & 0x3c003c00u, 0u};
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                if (NT > 1 && nt >= tiles) break;
                                float seen[4] = {0.f, 0.f, 0.f, 0.f};
                                mma_f16(seen, a, transpose8(vb[mt][nt][0]), transpose8(vb[mt][nt][1]));
#pragma unroll
                                for (int i = 0; i < NS; ++i)
#pragma unroll
                                    for (int j = 0; j < 4; ++j)
                                        if (seen[j & 1] > 0.f) o[nt][i][j] = __uint_as_float(0x7fc00000u);
                            }
                        }
                    }
#pragma unroll
                    for (int w = 0; w < NS / 4; ++w) {
                        uint32_t h[2][2][4];  // [keys 0 1 | 2 3][even | odd channel]
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t a = vw[2 * e][w], b = vw[2 * e + 1][w];
                            c4_decode((a & 0x0f0f0f0fu) | ((b << 4) & 0xf0f0f0f0u), h[e][0]);
                            c4_decode(((a >> 4) & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u), h[e][1]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                h[e][0][j] = h2_mul(h[e][0][j], f[e]);
                                h[e][1][j] = h2_mul(h[e][1][j], f[e]);
                            }
                        }
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            if (NT > 1 && nt >= tiles) break;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t a[4] = {h[0][0][i], h[0][1][i], h[1][0][i], h[1][1][i]};
                                mma_f16(o[nt][4 * w + i], a, pb[mt][nt][0], pb[mt][nt][1]);
                            }
                        }
                    }
                }
            }

            // ---- the four warps' results of the stretch
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) l[nt][j] += __shfl_xor_sync(0xffffffffu, l[nt][j], d);
                    if (g == 0) stats[warp * S::kRows + nt * 8 + 2 * t + j] = make_float2(m[nt][j], l[nt][j]);
                }
            __syncthreads();
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int r = nt * 8 + 2 * t + j;
                    float top = -INFINITY;
#pragma unroll
                    for (int w = 0; w < kCaWarps; ++w) top = fmaxf(top, stats[w * S::kRows + r].x);
                    const float keep = m[nt][j] == -INFINITY ? 1.f : ex2_approx(m[nt][j] - top);
                    if (r < nrow) {
                        float2* to = reinterpret_cast<float2*>(merge + (warp * S::kRows + r) * S::kRowBytes);
#pragma unroll
                        for (int i = 0; i < NS; ++i) to[i * 8 + g] = make_float2(o[nt][i][j] * keep, o[nt][i][j + 2] * keep);
                    }
                }
            __syncthreads();
            const bool whole = first == 0 && last == run.units;
            float* part = p.parts + (2ll * blockIdx.x + (first == 0)) * S::kPart;
            for (int x = tid; x < nrow * (D / 2); x += kCaThreads) {
                const int r = x / (D / 2), y = x % (D / 2);
                // whole: channels 2y, 2y + 1; a part: in the fragments' order
                const int slot = whole ? (y & (NS - 1)) * 8 + y / NS : y;
                float2 sum = make_float2(0.f, 0.f);
                float top = -INFINITY, total = 0.f;
#pragma unroll
                for (int w = 0; w < kCaWarps; ++w) {
                    const float2 v = reinterpret_cast<const float2*>(merge + (w * S::kRows + r) * S::kRowBytes)[slot];
                    sum.x += v.x, sum.y += v.y;
                    top = fmaxf(top, stats[w * S::kRows + r].x);
                }
#pragma unroll
                for (int w = 0; w < kCaWarps; ++w) {
                    const float2 st2 = stats[w * S::kRows + r];
                    total += st2.x == -INFINITY ? st2.y : st2.y * ex2_approx(st2.x - top);
                }
                if (!whole) {
                    reinterpret_cast<float2*>(part)[x] = sum;
                    if (y == 0) reinterpret_cast<float2*>(part + S::kRows * D)[r] = make_float2(top, total);
                    continue;
                }
                const int pr = run.r0 + (row0 + r) / p.G, hq = run.h * p.G + (row0 + r) % p.G;
                const bool any = row_vis[r] > 0;
                const float inv = 1.f / total;
                reinterpret_cast<uint32_t*>(p.o + (static_cast<int64_t>(pr) * p.Hq + hq) * D)[y] =
                    any ? cvt_bf16x2(sum.x * inv, sum.y * inv) : 0u;
                if (y == 0 && p.lse)
                    p.lse[static_cast<int64_t>(hq) * p.B * p.n + pr] = any ? (top + log2f(total)) * 0.693147181f : -INFINITY;
            }
            if (last < run.units && first == 0) {
                const long long end = at.x1 + run.units - last;  // the unit after the run's last
                goes_on = make_int4(run.b, run.h, run.rb, static_cast<int>((end * ctas - 1) / at.total));
            }
            if (last == run.units) {
                unit = 0;
                if (left > 0) ca_next(p, S::kRows, run);
            }
        }
    }
    cp_async_wait<0>();
    if (tid == 0) p.table[blockIdx.x] = goes_on;
}

// Joins the parts of the run that goes on past CTA blockIdx.x of the first launch:
// one row a CTA.
template <int D, int NT>
__global__ void __launch_bounds__(kCaThreads) cache4_join_kernel(CaParams p)
{
    using S = CaShape<D, NT>;
    const int4 e = p.table[blockIdx.x];
    if (e.x < 0) return;
    CaRun run{};
    ca_sequence(p, e.x, S::kRows, run);
    const int row0 = e.z * S::kRows, r = blockIdx.y, tid = threadIdx.x;
    if (r >= min(S::kRows, run.cnt * p.G - row0)) return;
    const int first = blockIdx.x, n = e.w - first + 1;
    auto slot = [&](int i) { return p.parts + (2ll * (first + i) + (i == 0)) * S::kPart; };
    float top = -INFINITY;
    for (int i = 0; i < n; ++i) top = fmaxf(top, slot(i)[S::kRows * D + 2 * r]);
    float total = 0.f;
    float2 sum = make_float2(0.f, 0.f);
    for (int i = 0; i < n; ++i) {
        const float2 st = reinterpret_cast<const float2*>(slot(i) + S::kRows * D)[r];
        const float keep = st.x == -INFINITY ? 1.f : ex2_approx(st.x - top);
        total += st.y * keep;
        if (tid < D / 2) {
            const float2 v = reinterpret_cast<const float2*>(slot(i))[r * (D / 2) + tid];
            sum.x += v.x * keep, sum.y += v.y * keep;
        }
    }
    const int pr = run.r0 + (row0 + r) / p.G, hq = e.y * p.G + (row0 + r) % p.G;
    const int i = max(0, min(p.pos[pr], p.n - 1));
    const bool any = min(run.len, max(0, run.len - p.n + i + 1)) > 0;
    if (tid < D / 2) {
        const int y = (tid & 7) * S::kSteps + tid / 8;  // fragment (i, g) holds channels 2 (g * steps + i), + 1
        const float inv = 1.f / total;
        reinterpret_cast<uint32_t*>(p.o + (static_cast<int64_t>(pr) * p.Hq + hq) * D)[y] =
            any ? cvt_bf16x2(sum.x * inv, sum.y * inv) : 0u;
    }
    if (tid == 0 && p.lse)
        p.lse[static_cast<int64_t>(hq) * p.B * p.n + pr] = any ? (top + log2f(total)) * 0.693147181f : -INFINITY;
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

// Tiles of 8 rows that a warp holds: as many as a sequence's rows of a KV head can need.
int ca_tiles(const logo_dims& d, int n_new)
{
    return static_cast<int>(std::min<int64_t>(kCaMaxTiles, (static_cast<int64_t>(n_new) * (d.Hq / d.Hkv) + 7) / 8));
}

template <typename F>
int ca_dispatch(int D, int tiles, F f)
{
    switch ((D == 128) * 4 + tiles - 1) {
        case 0: return f(CaShape<64, 1>());
        case 1: return f(CaShape<64, 2>());
        case 2: return f(CaShape<64, 3>());
        case 3: return f(CaShape<64, 4>());
        case 4: return f(CaShape<128, 1>());
        case 5: return f(CaShape<128, 2>());
        case 6: return f(CaShape<128, 3>());
        default: return f(CaShape<128, 4>());
    }
}

template <int D, int NT>
int ca_grid(CaShape<D, NT>)
{
    return device_sm_count() * CaShape<D, NT>::kCtas;
}

template <int D, int NT>
int ca_launch(CaShape<D, NT> s, CaParams& p, cudaStream_t st)
{
    using S = CaShape<D, NT>;
    static OncePerDevice once;
    if (once([] { return set_smem_limit(cache4_attn_kernel<D, NT>, S::kSmem); }) != cudaSuccess) return LOGO_ERR_CUDA;
    const unsigned grid = ca_grid(s);
    cache4_attn_kernel<D, NT><<<grid, kCaThreads, S::kSmem, st>>>(p);
    cache4_join_kernel<D, NT><<<dim3(grid, S::kRows), kCaThreads, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}

}  // namespace
}  // namespace logo

using namespace logo;

extern "C" size_t logo_decode_cache4_workspace_size(logo_dims dims, int n_new)
{
    if (check_cache4_attn(dims, n_new) != LOGO_OK) return 0;
    size_t bytes = 0;
    ca_dispatch(dims.D, ca_tiles(dims, n_new), [&](auto s) {
        using S = decltype(s);
        const size_t grid = ca_grid(s);
        bytes = round_up(grid * sizeof(int4), 256) + 2 * grid * S::kPart * sizeof(float);
        return 0;
    });
    return bytes;
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
    CaParams p{};
    p.q = q, p.k = cache.k, p.v = cache.v, p.ks = cache.k_scale, p.vs = cache.v_scale;
    p.len = seq_len, p.pos = pos, p.cu_q = cu_q, p.n_sel = n_sel_total, p.o = o_c, p.lse = lse_c;
    p.B = dims.B, p.n = n_new, p.Hq = dims.Hq, p.Hkv = dims.Hkv, p.G = dims.Hq / dims.Hkv, p.L = dims.T;
    p.scale2 = (scale > 0.f ? scale : 1.f / sqrtf(static_cast<float>(dims.D))) * 1.44269504f;
    return ca_dispatch(dims.D, ca_tiles(dims, n_new), [&](auto s) {
        p.table = static_cast<int4*>(workspace);
        p.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + round_up(ca_grid(s) * sizeof(int4), 256));
        return ca_launch(s, p, static_cast<cudaStream_t>(stream));
    });
}
