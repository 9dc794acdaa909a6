// prefix_attn.cu -- one serving step of the global branch (Eq. 8) for a batch
// that shares a long prefix: the packed rows of n_new tokens per sequence
// attend the shared prefix and their own sequence's cache, and the attention
// weight that every own cache row receives is added up.
//
// Mathematics.  A segment is the prefix (rows: every packed row) or one
// sequence's cache (rows: that sequence's packed rows).  For KV head h the
// rows of a segment are (packed row, query head of the group): all of them
// read the same keys.  Softmax over a union of key sets joins exactly: with
// m = max x, l = sum 2^(x - m), O = sum 2^(x - m) v of each part (log2 units),
//   M = max m,  L = sum 2^(m - M) l,  o = sum 2^(m - M) O / L.
// So the key range of every segment is cut into pieces at will, a piece leaves
// (m, l, O), and a second launch joins each row's pieces.
//
// pa_rows_kernel: one persistent CTA per SM walks an equal share of all key
//   tiles (128 keys of a segment and KV head).  A producer warp keeps a ring of
//   K and V tiles in flight (TMA, 192 KB); eight warps do the products
//   with warp-level MMA (decoding has a group's few heads per sequence as rows,
//   mostly padding for a tcgen05 tile, and HBM bounds it: a tile's 64 KB take
//   2790 clocks at an SM's share of it), each on its own 16 keys of every tile
//   with its own running maximum and sum, so that no warp waits for another.
//   More than 32 rows: two groups of four warps take 32 rows each.
// More than 64 rows of the prefix per KV head are bound by the products and go
// to the tcgen05 kernel of the prefill's global branch instead, in tiles of 128
// rows and shares of the prefix (pa_wide_prep_kernel lays them out, on the
// device as the count of rows is known only there; pa_wide_join_kernel joins
// the shares).
// pa_finish_kernel: joins each (row, head)'s pieces, and adds up the weights
//   exp(x - lse) of every own cache row from the logits that pa_rows_kernel
//   wrote down (4 bytes a row and key, against 4 D bytes of K and V a key for
//   all rows; reading K again would cost half of the cache traffic).
#include <cuda_bf16.h>

#include <algorithm>
#include <cstdint>

#include "attn_common.cuh"
#include "host_common.h"
#include "logo_status.cuh"
#include "sm100.cuh"

namespace logo {
namespace {

constexpr int kPaWarps = 8;                        // consumer warps; one more loads
constexpr int kPaThreads = 384;                    // two warpgroups of consumers, one to load (one warp of it)
constexpr uint32_t kPaRegsRows = 216, kPaRegsLoad = 72;
static_assert(128 * (2 * kPaRegsRows + kPaRegsLoad) <= kPaThreads * 168, "register split exceeds the launch allocation");
constexpr int kPaTile = 128;                       // keys per tile
constexpr int kPaRows = 64;                        // rows of a piece at most
constexpr int kPaFinThreads = 256;
constexpr int kPaWideUnits = 1216;                 // (share, KV head) units that the wide prefix is cut into at most

template <int D>
struct PaCfg {
    static constexpr int kTileBytes = kPaTile * D * 2;      // one K or V tile
    static constexpr int kHalfBytes = kPaTile * 128;        // its 64-column half (128-byte rows)
    static constexpr int kStages = D == 128 ? 6 : 12;       // K and V tiles in turn: 192 KB
    static constexpr int kQHalf = kPaRows * 128;
    static constexpr int kQBytes = kPaRows * D * 2;
    static constexpr int kOffRing = 2 * kQBytes;            // after two Q tiles
    static constexpr int kSmemBytes = kOffRing + kStages * kTileBytes + 1024;
};

// All tiles of a call lie on one line: the prefix's (KV head, tile), then the
// own caches' (sequence, KV head, row tile, tile).  CTA c of n takes the tiles
// [total c / n, total (c + 1) / n).
struct PaSched {
    long long K;      // Hkv * PT: length of the prefix part
    long long total;  // length of the line
    int N, PT, n, pad;
};

// What the join needs to know of a sequence.
struct PaSeq {
    long long base;  // its first tile on the line
    int row0, n, len, tiles, rts, pad;
};

struct PaParams {
    CUtensorMap tm_kp, tm_vp;  // prefix [1, P, Hkv, D]
    CUtensorMap tm_kc, tm_vc;  // own caches [B, L, Hkv, D]
    const logo_bf16 *q, *kp, *vp;
    const int32_t *seq_len, *pos, *cu_q, *n_sel;
    logo_bf16* o;
    float* lse;  // [Hq, cap] natural log, or NULL
    const float* mass_in;
    float* mass_out;
    // workspace
    PaSched* sched;
    PaSeq* seqs;            // [B]
    int32_t* row_seq;       // [cap]: sequence of each packed row
    float *o_pre, *ml_pre;  // prefix pieces: [slot][w_pre][D], [slot][w_pre][2]
    float *o_own, *ml_own;
    // wide prefix (more than kPaRows rows per KV head): row M = r * G + g
    logo_bf16* wq;          // [rows + 128, Hkv, D]
    int32_t* wpos;          // [rows]
    GlobalTile* wtiles;
    int32_t* wcount;        // tiles, next item, shares, row tiles
    float *wo_part, *wm_part, *wl_part;  // shares, as the tcgen05 kernel leaves them
    float *wo, *wml;        // joined: [M][Hkv][D], [M][Hkv][2]
    float* logits;  // [B, Hkv, L, R] log2 units, R = n_new * G
    int B, L, Hq, Hkv, G, n_new, P, cap, R, rt_own_max, w_pre, w_own, nCta;
    int wpr, row_blocks;  // finish: warps per (row, head), blocks that join rows
    float scale_log2;
};

// Own cache rows that token i of a sequence with len tokens sees.
__device__ __forceinline__ int own_visible(int len, int n_new, int i) { return min(len, max(0, len - n_new + i + 1)); }

// A piece of nrows rows leaves one (m, l, O) per warp that shared its keys.
__device__ __forceinline__ int piece_reps(int nrows) { return nrows <= 32 ? 8 : 4; }

struct OwnSeq {
    int row0, n, len, tiles, rts;  // first packed row, rows, tokens, key tiles, row tiles
};

__device__ __forceinline__ OwnSeq own_seq(const PaParams& p, int b)
{
    OwnSeq o;
    o.row0 = __ldg(p.cu_q + b);
    const int row1 = __ldg(p.cu_q + b + 1);
    o.n = row1 - o.row0;
    o.len = max(0, min(__ldg(p.seq_len + b), p.L));
    o.tiles = o.rts = 0;
    if (o.n > 0) {
        o.tiles = (own_visible(o.len, p.n_new, __ldg(p.pos + row1 - 1)) + kPaTile - 1) / kPaTile;
        o.rts = (o.n * p.G + kPaRows - 1) / kPaRows;
    }
    return o;
}

__device__ __forceinline__ long long share_start(const PaSched& s, int c) { return s.total * c / s.n; }

// The CTA whose share holds tile u: the last c with floor(total c / n) <= u
// (n <= total: no share is empty).
__device__ __forceinline__ int share_owner(const PaSched& s, long long u)
{
    return static_cast<int>(((u + 1) * s.n - 1) / s.total);
}

// One piece: key tiles [t0, t1) of a segment for one row tile and KV head.
struct PaPiece {
    bool own;
    int b, kvh, row0, nrows;  // own: sequence; rows row0 .. of the segment's (row, head) list
    int seg_row0;             // first packed row of the segment
    int t0, t1, len;          // len: keys of the segment
    int64_t slot;
};

struct PaIter {
    long long u, u1, base;  // position, end, first tile of sequence b
    int c, b;

    __device__ __forceinline__ bool next(const PaParams& p, const PaSched& s, PaPiece* it)
    {
        if (u >= u1) return false;
        if (u < s.K) {
            it->own = false;
            it->b = 0;
            it->kvh = static_cast<int>(u / s.PT);
            it->t0 = static_cast<int>(u % s.PT);
            it->t1 = static_cast<int>(min(static_cast<long long>(s.PT), it->t0 + (u1 - u)));
            it->row0 = 0;
            it->nrows = s.N * p.G;
            it->seg_row0 = 0;
            it->len = p.P;
            it->slot = it->kvh + c;
            u += it->t1 - it->t0;
            return true;
        }
        OwnSeq o = own_seq(p, b);
        long long units = static_cast<long long>(o.tiles) * o.rts * p.Hkv;
        while (u - base >= units) {  // ends: u < u1 <= the line's length
            base += units;
            ++b;
            o = own_seq(p, b);
            units = static_cast<long long>(o.tiles) * o.rts * p.Hkv;
        }
        const int run = static_cast<int>((u - base) / o.tiles);
        it->own = true;
        it->b = b;
        it->kvh = run / o.rts;
        const int r = run % o.rts;
        it->t0 = static_cast<int>((u - base) % o.tiles);
        it->t1 = static_cast<int>(min(static_cast<long long>(o.tiles), it->t0 + (u1 - u)));
        it->row0 = r * kPaRows;
        it->nrows = min(kPaRows, o.n * p.G - it->row0);
        it->seg_row0 = o.row0;
        it->len = o.len;
        it->slot = (static_cast<int64_t>(b) * p.Hkv + it->kvh) * p.rt_own_max + r + c;
        u += it->t1 - it->t0;
        return true;
    }
};

// A warp's share of one piece: MT blocks of 16 rows from row 32 * rg on, and in
// every tile the STEPS blocks of 16 keys from key kg * 16 * STEPS on.
struct PaWarp {
    uint32_t sQ, sRing, kv_full, kv_empty;  // kv_*: the first barrier, the others 8 bytes on
    volatile int* abort_flag;
    int lane, rg, kg, n;  // n: tiles consumed, K and V counted
};

template <int D, int MT, int STEPS>
__device__ __forceinline__ bool pa_warp_piece(const PaParams& p, const PaPiece& it, PaWarp& w)
{
    using C = PaCfg<D>;
    constexpr int NT = D / 8;
    const int lane = w.lane, gid = lane >> 2, tig = lane & 3, mi = lane >> 3, rr = lane & 7;
    const bool with_logits = it.own && p.mass_out != nullptr;
    // this lane's rows: row_of(mt, i) = 32 rg + 16 mt + 8 i + gid
    int vis[MT][2];
    float m_run[MT][2], l_run[MT][2], oc[MT][NT][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = 32 * w.rg + 16 * mt + 8 * i + gid;
            vis[mt][i] = it.len;
            if (it.own && row < it.nrows)
                vis[mt][i] = own_visible(it.len, p.n_new, __ldg(p.pos + it.seg_row0 + (it.row0 + row) / p.G));
            m_run[mt][i] = -INFINITY;
            l_run[mt][i] = 0.f;
        }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) oc[mt][nt][i] = 0.f;

    for (int t = it.t0; t < it.t1; ++t) {
        const int stK = w.n % C::kStages, fK = w.n / C::kStages;
        const int stV = (w.n + 1) % C::kStages, fV = (w.n + 1) / C::kStages;
        w.n += 2;
        const uint32_t sK = w.sRing + stK * C::kTileBytes, sV = w.sRing + stV * C::kTileBytes;
        bool ok = mbar_wait(w.kv_full + 8 * stK, fK & 1, w.abort_flag);
        if (!__all_sync(0xffffffffu, ok)) return false;  // the warp leaves together
        const int k0 = w.kg * 16 * STEPS;  // this warp's first key of the tile
#pragma unroll 1
        for (int st = 0; st < STEPS; ++st) {
            uint32_t pa[MT][4];
            // ---- S = Q K^T over 16 keys (two 8-key blocks)
            float sc[MT][2][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[mt][nt][i] = 0.f;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                const int half = ks / 4, ch0 = (ks % 4) * 2;
                uint32_t b0, b1, b2, b3;
                ldsm_x4(sK + half * C::kHalfBytes + sw128_offset(k0 + st * 16 + (mi >> 1) * 8 + rr, ch0 + (mi & 1)), b0,
                        b1, b2, b3);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    // A fragment: rows (mi & 1) * 8 + rr, 16-byte chunk ch0 + (mi >> 1)
                    uint32_t a[4];
                    ldsm_x4(w.sQ + half * C::kQHalf +
                                sw128_offset(32 * w.rg + 16 * mt + (mi & 1) * 8 + rr, ch0 + (mi >> 1)),
                            a[0], a[1], a[2], a[3]);
                    mma_bf16_16816(sc[mt][0], a, b0, b1);
                    mma_bf16_16816(sc[mt][1], a, b2, b3);
                }
            }
            // ---- online softmax; keys at and past `vis` are not seen (their K may
            //      be anything, NaN included)
            const int key0 = t * kPaTile + k0 + st * 16 + 2 * tig;
            bool grow = false;
            float mx[MT][2];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                mx[mt][0] = mx[mt][1] = -INFINITY;
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = sc[mt][nt][i] * p.scale_log2;
                        sc[mt][nt][i] = key0 + nt * 8 + (i & 1) < vis[mt][i >> 1] ? x : -INFINITY;
                        mx[mt][i >> 1] = fmaxf(mx[mt][i >> 1], sc[mt][nt][i]);
                    }
                if (with_logits) {
                    float* lg = p.logits + ((static_cast<int64_t>(it.b) * p.Hkv + it.kvh) * p.L + key0) * p.R +
                                it.row0 + 32 * w.rg + 16 * mt + gid;
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (32 * w.rg + 16 * mt + 8 * (i >> 1) + gid < it.nrows &&
                                key0 + nt * 8 + (i & 1) < it.len)
                                lg[static_cast<int64_t>(nt * 8 + (i & 1)) * p.R + 8 * (i >> 1)] = sc[mt][nt][i];
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    mx[mt][i] = fmaxf(mx[mt][i], __shfl_xor_sync(0xffffffffu, mx[mt][i], 1));
                    mx[mt][i] = fmaxf(mx[mt][i], __shfl_xor_sync(0xffffffffu, mx[mt][i], 2));
                    // O is rescaled only when the maximum has grown by more than 2^8:
                    // until then l and O hold values up to 2^8 times larger, which fp32
                    // takes without loss (and bf16's P: its precision is relative)
                    grow |= mx[mt][i] > m_run[mt][i] + 8.0f;
                }
            }
            if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    float alpha[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        alpha[i] = 1.f;
                        if (mx[mt][i] > m_run[mt][i] + 8.0f) {
                            alpha[i] = ex2_approx(m_run[mt][i] - mx[mt][i]);  // 0 while nothing was seen
                            m_run[mt][i] = mx[mt][i];
                            l_run[mt][i] *= alpha[i];
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        oc[mt][nt][0] *= alpha[0];
                        oc[mt][nt][1] *= alpha[0];
                        oc[mt][nt][2] *= alpha[1];
                        oc[mt][nt][3] *= alpha[1];
                    }
                }
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const float m0 = m_run[mt][0] == -INFINITY ? 0.f : m_run[mt][0];
                const float m1 = m_run[mt][1] == -INFINITY ? 0.f : m_run[mt][1];
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        sc[mt][nt][i] = ex2_approx(sc[mt][nt][i] - (i < 2 ? m0 : m1));
                        l_run[mt][i >> 1] += sc[mt][nt][i];  // this lane's keys; the quad's are added at the end
                    }
                // P as the A fragment: rows = rows, k = the 16 keys
                pa[mt][0] = pack_bf16x2(sc[mt][0][0], sc[mt][0][1]);
                pa[mt][1] = pack_bf16x2(sc[mt][0][2], sc[mt][0][3]);
                pa[mt][2] = pack_bf16x2(sc[mt][1][0], sc[mt][1][1]);
                pa[mt][3] = pack_bf16x2(sc[mt][1][2], sc[mt][1][3]);
            }
            if (st == STEPS - 1) {
                __syncwarp();
                if (lane == 0) mbar_arrive(w.kv_empty + 8 * stK);
            }
            if (st == 0) {
                ok = mbar_wait(w.kv_full + 8 * stV, fV & 1, w.abort_flag);
                if (!__all_sync(0xffffffffu, ok)) return false;
                const int end = it.len - t * kPaTile;  // rows of the tile that hold a token
                if (it.own && end < k0 + 16 * STEPS) {
                    // a cache row past the length may hold anything: zero its V, so
                    // that P = 0 keeps it out of the product
                    for (int i = lane; i < 16 * STEPS * (D / 8); i += 32) {
                        const int row = k0 + i / (D / 8), ch = i % (D / 8);
                        if (row >= end)
                            st_shared_v4(sV + (ch >> 3) * C::kHalfBytes + sw128_offset(row, ch & 7), 0u, 0u, 0u, 0u);
                    }
                    fence_proxy_async_smem();  // ordered before the stage's next TMA write
                    __syncwarp();
                }
            }
            // ---- O += P V over the 16 keys
#pragma unroll
            for (int np = 0; np < NT / 2; ++np) {
                const int col = np * 16 + (mi >> 1) * 8;
                uint32_t b0, b1, b2, b3;
                ldsm_x4_trans(sV + (col / 64) * C::kHalfBytes +
                                  sw128_offset(k0 + st * 16 + (mi & 1) * 8 + rr, (col % 64) / 8),
                              b0, b1, b2, b3);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    mma_bf16_16816(oc[mt][2 * np], pa[mt], b0, b1);
                    mma_bf16_16816(oc[mt][2 * np + 1], pa[mt], b2, b3);
                }
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(w.kv_empty + 8 * stV);
    }
    // ---- (m, l, O) of this warp's keys
    const int64_t at = it.slot * (it.own ? p.w_own : p.w_pre) + w.kg * it.nrows;
    float* o_part = (it.own ? p.o_own : p.o_pre) + at * D;
    float2* ml = reinterpret_cast<float2*>(it.own ? p.ml_own : p.ml_pre) + at;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float l = l_run[mt][i];
            l += __shfl_xor_sync(0xffffffffu, l, 1);
            l += __shfl_xor_sync(0xffffffffu, l, 2);
            const int row = 32 * w.rg + 16 * mt + 8 * i + gid;
            if (row < it.nrows) {
                if (tig == 0) ml[row] = make_float2(m_run[mt][i], l);
                float* dst = o_part + static_cast<int64_t>(row) * D + 2 * tig;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    *reinterpret_cast<float2*>(dst + nt * 8) =
                        make_float2(oc[mt][nt][2 * i], oc[mt][nt][2 * i + 1]);
            }
        }
    return true;
}

template <int D>
__global__ void __launch_bounds__(kPaThreads, 1) pa_rows_kernel(const __grid_constant__ PaParams p)
{
    using C = PaCfg<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ __align__(8) uint64_t bar_q_full[2], bar_q_empty[2], bar_kv_full[C::kStages], bar_kv_empty[C::kStages];
    __shared__ long long sh_scan[kPaThreads / 32], sh_base;
    __shared__ int sh_b0;
    __shared__ volatile int abort_flag;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    const uint32_t sQ = smem_u32(smem), sRing = smem_u32(smem + C::kOffRing);
    if (tid == 0) {
        abort_flag = 0;
        sh_b0 = 0;
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(smem_u32(&bar_kv_full[s]), 1);
            mbar_init(smem_u32(&bar_kv_empty[s]), kPaWarps);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_u32(&bar_q_full[s]), 1);
            mbar_init(smem_u32(&bar_q_empty[s]), kPaWarps);
        }
        fence_mbar_init();
    }

    // ---- the line, the same in every CTA
    const int N = *p.n_sel;
    const int per = (p.B + kPaThreads - 1) / kPaThreads;  // sequences per thread
    const int tb0 = min(p.B, tid * per), tb1 = min(p.B, tb0 + per);
    long long mine = 0;
    for (int b = tb0; b < tb1; ++b) {
        const OwnSeq o = own_seq(p, b);
        mine += static_cast<long long>(o.tiles) * o.rts * p.Hkv;
    }
    __syncwarp();
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) sh_scan[warp] = incl;
    __syncthreads();
    PaSched s;
    s.N = N;
    s.PT = (p.P + kPaTile - 1) / kPaTile;
    s.K = N > 0 && N * p.G <= kPaRows ? static_cast<long long>(p.Hkv) * s.PT : 0;
    long long excl = s.K + incl - mine;
    s.total = s.K;
    for (int k = 0; k < kPaThreads / 32; ++k) {
        if (k < warp) excl += sh_scan[k];
        s.total += sh_scan[k];
    }
    s.n = static_cast<int>(min(static_cast<long long>(p.nCta), s.total));
    s.pad = 0;
    PaIter iter;
    iter.c = cta;
    iter.u = cta < s.n ? share_start(s, cta) : 0;
    iter.u1 = cta < s.n ? share_start(s, cta + 1) : 0;
    if (tid == 0) sh_base = s.K;
    __syncthreads();
    // the sequence that the share starts in (a share that starts in the prefix
    // meets its sequences from the first one on)
    if (iter.u < iter.u1 && iter.u >= excl && iter.u < excl + mine) {
        long long base = excl;
        int b = tb0;
        for (; b < tb1; ++b) {
            const OwnSeq o = own_seq(p, b);
            const long long units = static_cast<long long>(o.tiles) * o.rts * p.Hkv;
            if (iter.u < base + units) break;
            base += units;
        }
        sh_b0 = b;
        sh_base = base;
    }
    if (cta == 0) {  // for the join
        if (tid == 0) *p.sched = s;
        long long base = excl;
        for (int b = tb0; b < tb1; ++b) {
            const OwnSeq o = own_seq(p, b);
            p.seqs[b] = PaSeq{base, o.row0, o.n, o.len, o.tiles, o.rts, 0};
            base += static_cast<long long>(o.tiles) * o.rts * p.Hkv;
            for (int i = 0; i < o.n; ++i) p.row_seq[o.row0 + i] = b;
        }
    }
    __syncwarp();
    __syncthreads();
    __syncwarp();
    iter.b = sh_b0;
    iter.base = sh_base;
    PaPiece it;

    if (warp >= kPaWarps) {
        // ------------------------------------------------------ loader
        setmaxnreg_dec<kPaRegsLoad>();
        if (warp > kPaWarps) return;
        const uint64_t pol = policy_evict_first();
        int n = 0, piece = 0;
        bool ok = true;
        while (ok && iter.next(p, s, &it)) {
            // Q of the piece: rows past nrows keep whatever is there (a row of S
            // depends on its own row of Q alone)
            const int qb = piece & 1;
            ok = mbar_wait(smem_u32(&bar_q_empty[qb]), ((piece >> 1) & 1) ^ 1, &abort_flag);
            if (!(ok = __all_sync(0xffffffffu, ok))) break;
            constexpr int kChunks = D / 8;  // 16-byte chunks of a row
            const uint32_t qbase = sQ + qb * C::kQBytes;
            for (int i0 = 0; i0 < it.nrows * kChunks; i0 += 32 * 4) {
                uint4 v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int i = i0 + k * 32 + lane;
                    v[k] = make_uint4(0u, 0u, 0u, 0u);
                    if (i < it.nrows * kChunks) {
                        const int m = it.row0 + i / kChunks, r = it.seg_row0 + m / p.G, g = m % p.G;
                        const int b = it.own ? it.b : seq_of_row(p.cu_q, p.B, r);
                        const int64_t row =
                            (static_cast<int64_t>(b) * p.n_new + __ldg(p.pos + r)) * p.Hq + it.kvh * p.G + g;
                        v[k] = __ldg(reinterpret_cast<const uint4*>(p.q + row * D) + i % kChunks);
                    }
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int i = i0 + k * 32 + lane, row = i / kChunks, ch = i % kChunks;
                    if (i < it.nrows * kChunks)
                        st_shared_v4(qbase + (ch >> 3) * C::kQHalf + sw128_offset(row, ch & 7), v[k].x, v[k].y, v[k].z,
                                     v[k].w);
                }
            }
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_u32(&bar_q_full[qb]));
                const CUtensorMap* tk = it.own ? &p.tm_kc : &p.tm_kp;
                const CUtensorMap* tv = it.own ? &p.tm_vc : &p.tm_vp;
                for (int t = it.t0; t < it.t1 && ok; ++t) {
                    for (int kv = 0; kv < 2; ++kv, ++n) {
                        const int st = n % C::kStages, f = n / C::kStages;
                        if (!(ok = mbar_wait(smem_u32(&bar_kv_empty[st]), (f & 1) ^ 1, &abort_flag))) break;
                        const uint32_t bar = smem_u32(&bar_kv_full[st]);
                        mbar_arrive_expect_tx(bar, C::kTileBytes);
                        for (int h = 0; h < D / 64; ++h)
                            tma_load_4d(sRing + st * C::kTileBytes + h * C::kHalfBytes, kv ? tv : tk, bar, 64 * h, it.kvh,
                                        t * kPaTile, it.b, pol);
                    }
                }
            }
            ok = __all_sync(0xffffffffu, ok);
            ++piece;
        }
        if (!ok && lane == 0) {  // let copies already issued land before the CTA exits
            for (int k = max(0, n - C::kStages); k < n; ++k)
                mbar_wait_drain(smem_u32(&bar_kv_full[k % C::kStages]), (k / C::kStages) & 1);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------ products
        setmaxnreg_inc<kPaRegsRows>();
        PaWarp w;
        w.sRing = sRing;
        w.kv_full = smem_u32(&bar_kv_full[0]);
        w.kv_empty = smem_u32(&bar_kv_empty[0]);
        w.abort_flag = &abort_flag;
        w.lane = lane;
        w.n = 0;
        bool ok = true;
        for (int piece = 0; ok && iter.next(p, s, &it); ++piece) {
            const int qb = piece & 1;
            ok = mbar_wait(smem_u32(&bar_q_full[qb]), (piece >> 1) & 1, &abort_flag);
            if (!(ok = __all_sync(0xffffffffu, ok))) break;
            w.sQ = sQ + qb * C::kQBytes;
            if (it.nrows <= 32) {
                w.rg = 0;
                w.kg = warp;
                ok = it.nrows <= 16 ? pa_warp_piece<D, 1, 1>(p, it, w) : pa_warp_piece<D, 2, 1>(p, it, w);
            } else {
                w.rg = warp >> 2;
                w.kg = warp & 3;
                ok = pa_warp_piece<D, 2, 2>(p, it, w);
            }
            __syncwarp();
            if (ok && lane == 0) mbar_arrive(smem_u32(&bar_q_empty[qb]));
        }
    }
}

// --------------------------------------------------------------- wide prefix
// Rows, positions and tiles of the wide prefix.  Block 0 picks the number of
// shares that each row tile's key range is cut into: the least time of the
// busiest SM, an item (row tile, share, KV head) counted with 6 key blocks for
// its start and its join.  Items lie share by share, so that the SMs work on
// the same keys at the same time.
template <int D>
__global__ void __launch_bounds__(256) pa_wide_prep_kernel(const __grid_constant__ PaParams p, int n_sm)
{
    __shared__ unsigned int sh_best;
    const int N = *p.n_sel, rows = N * p.G, tid = threadIdx.x;
    if (rows <= kPaRows) {
        if (blockIdx.x == 0 && tid < 4) p.wcount[tid] = 0;
        return;
    }
    const int nRT = (rows + 127) / 128, blocks = (p.P + 127) / 128;
    if (blockIdx.x == 0) {
        const int most = max(1, min(min(blocks, kPaWideUnits / (nRT * p.Hkv)), 255));
        if (tid == 0) sh_best = ~0u;
        __syncthreads();
        if (tid < most) {
            const int n = tid + 1;
            const long long items = static_cast<long long>(nRT) * p.Hkv * n;
            const long long cost = (items + n_sm - 1) / n_sm * ((blocks + n - 1) / n + 6);
            atomicMin(&sh_best, static_cast<unsigned int>(min(cost, 0xffffffll) << 8) | static_cast<unsigned int>(n));
        }
        __syncthreads();
        const int ns = sh_best & 255;
        for (int e = tid; e < nRT * ns; e += blockDim.x) {
            const int sh = e / nRT, rt = e % nRT;
            GlobalTile g{};
            g.row0 = rt * 128;
            g.nrows = min(128, rows - g.row0);
            g.b = 0;
            g.min_pos = g.max_pos = p.P - 1;
            g.blk_lo = static_cast<int>(static_cast<long long>(blocks) * sh / ns);
            g.blk_hi = static_cast<int>(static_cast<long long>(blocks) * (sh + 1) / ns) - 1;
            g.slot = e;
            g.cost = g.blk_hi - g.blk_lo + 1;
            p.wtiles[e] = g;
        }
        if (tid == 0) {
            p.wcount[0] = nRT * ns;
            p.wcount[1] = 0;
            p.wcount[2] = ns;
            p.wcount[3] = nRT;
        }
    }
    const int vecs = p.Hkv * (D / 8);
    for (int M = blockIdx.x; M < nRT * 128; M += gridDim.x) {
        uint4* dst = reinterpret_cast<uint4*>(p.wq + static_cast<int64_t>(M) * p.Hkv * D);
        if (M >= rows) {  // the last tile's idle rows: finite
            for (int v = tid; v < vecs; v += blockDim.x) dst[v] = make_uint4(0u, 0u, 0u, 0u);
            continue;
        }
        const int r = M / p.G, g = M % p.G, b = seq_of_row(p.cu_q, p.B, r);
        const uint4* src =
            reinterpret_cast<const uint4*>(p.q + (static_cast<int64_t>(b) * p.n_new + p.pos[r]) * p.Hq * D);
        for (int v = tid; v < vecs; v += blockDim.x)
            dst[v] = src[(v / (D / 8) * p.G + g) * (D / 8) + v % (D / 8)];
        if (tid == 0) p.wpos[M] = p.P - 1;
    }
}

// The shares of each (row, KV head) joined: a block takes 128 rows and 8
// columns of a row tile and KV head.
template <int D>
__global__ void __launch_bounds__(128) pa_wide_join_kernel(const __grid_constant__ PaParams p)
{
    const int ns = p.wcount[2], nRT = p.wcount[3], rows = *p.n_sel * p.G, i = threadIdx.x;
    const int units = nRT * p.Hkv * (D / 8);
    for (int un = blockIdx.x; un < units; un += gridDim.x) {
        const int col = un % (D / 8), h = un / (D / 8) % p.Hkv, rt = un / (D / 8) / p.Hkv;
        const int M = rt * 128 + i;
        if (M >= rows) continue;
        const int64_t unit0 = static_cast<int64_t>(rt) * p.Hkv + h, step = static_cast<int64_t>(nRT) * p.Hkv;
        float mx = -INFINITY;
        for (int s = 0; s < ns; ++s) mx = fmaxf(mx, p.wm_part[(unit0 + s * step) * 128 + i]);
        float l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < ns; ++s) {
            const int64_t unit = unit0 + s * step;
            const float m = p.wm_part[unit * 128 + i];
            const float w = m == -INFINITY ? 0.f : ex2_approx(m - mx);
            l += w * p.wl_part[unit * 128 + i];
            const float* src = p.wo_part + (unit * D + col * 8) * 128 + i;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += w * src[e * 128];
        }
        const int64_t at = static_cast<int64_t>(M) * p.Hkv + h;
        float4* dst = reinterpret_cast<float4*>(p.wo + at * D + col * 8);
        dst[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        dst[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
        if (col == 0) *reinterpret_cast<float2*>(p.wml + at * 2) = make_float2(mx, l);
    }
}

// ------------------------------------------------------------------- finish
// The pieces of one (row, head): those of the prefix, then those of its own
// cache; entry e is one copy of the row in one piece.
struct PaParts {
    const float2 *ml_pre, *ml_own;
    const float *o_pre, *o_own;
    int n_pre, n_own, reps_pre, reps_own, nr_pre, nr_own;  // entries; copies; rows of the tile
    int w_pre, w_own;

    __device__ __forceinline__ int count() const { return n_pre + n_own; }
    __device__ __forceinline__ float2 ml(int e) const
    {
        if (e < n_pre) return __ldg(ml_pre + (e / reps_pre) * static_cast<int64_t>(w_pre) + (e % reps_pre) * nr_pre);
        e -= n_pre;
        return __ldg(ml_own + (e / reps_own) * static_cast<int64_t>(w_own) + (e % reps_own) * nr_own);
    }
    template <int D>
    __device__ __forceinline__ const float* o(int e) const
    {
        if (e < n_pre) return o_pre + ((e / reps_pre) * static_cast<int64_t>(w_pre) + (e % reps_pre) * nr_pre) * D;
        e -= n_pre;
        return o_own + ((e / reps_own) * static_cast<int64_t>(w_own) + (e % reps_own) * nr_own) * D;
    }
};

template <int D>
__device__ __forceinline__ PaParts pa_parts(const PaParams& p, const PaSched& s, const PaSeq& q, int r, int b, int kvh,
                                            int g)
{
    PaParts x;
    x.w_pre = p.w_pre;
    x.w_own = p.w_own;
    x.n_pre = x.n_own = 0;
    x.reps_pre = x.reps_own = x.nr_pre = x.nr_own = 1;
    x.ml_pre = x.ml_own = nullptr;
    x.o_pre = x.o_own = nullptr;
    if (s.K > 0) {
        x.nr_pre = s.N * p.G;
        x.reps_pre = piece_reps(x.nr_pre);
        const long long u0 = static_cast<long long>(kvh) * s.PT;
        const int c0 = share_owner(s, u0), c1 = share_owner(s, u0 + s.PT - 1);
        x.n_pre = (c1 - c0 + 1) * x.reps_pre;
        const int64_t at = static_cast<int64_t>(kvh + c0) * p.w_pre + r * p.G + g;
        x.ml_pre = reinterpret_cast<const float2*>(p.ml_pre) + at;
        x.o_pre = p.o_pre + at * D;
    }
    if (s.K == 0 && s.PT > 0) {  // wide: joined already
        const int64_t at = (static_cast<int64_t>(r) * p.G + g) * p.Hkv + kvh;
        x.n_pre = 1;
        x.ml_pre = reinterpret_cast<const float2*>(p.wml) + at;
        x.o_pre = p.wo + at * D;
    }
    if (q.tiles > 0) {
        const int M = (r - q.row0) * p.G + g, rt = M / kPaRows, i = M % kPaRows;
        x.nr_own = min(kPaRows, q.n * p.G - rt * kPaRows);
        x.reps_own = piece_reps(x.nr_own);
        const long long u0 = q.base + (static_cast<long long>(kvh) * q.rts + rt) * q.tiles;
        const int c0 = share_owner(s, u0), c1 = share_owner(s, u0 + q.tiles - 1);
        x.n_own = (c1 - c0 + 1) * x.reps_own;
        const int64_t at = ((static_cast<int64_t>(b) * p.Hkv + kvh) * p.rt_own_max + rt + c0) * p.w_own + i;
        x.ml_own = reinterpret_cast<const float2*>(p.ml_own) + at;
        x.o_own = p.o_own + at * D;
    }
    return x;
}

// (M, L) of a (row, head) over its pieces, by a warp.
__device__ __forceinline__ float2 pa_join_ml(const PaParts& x, int lane)
{
    const int n = x.count();
    float M = -INFINITY, Ls = 0.f;
    for (int e = lane; e < n; e += 32) {
        const float2 v = x.ml(e);
        if (v.x == -INFINITY) continue;
        const float m = fmaxf(M, v.x);
        Ls = Ls * ex2_approx(M - m) + v.y * ex2_approx(v.x - m);
        M = m;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, M, o), l2 = __shfl_xor_sync(0xffffffffu, Ls, o);
        const float m = fmaxf(M, m2);
        if (m != -INFINITY) Ls = Ls * ex2_approx(M - m) + l2 * ex2_approx(m2 - m);
        M = m;
    }
    return make_float2(M, Ls);
}

// Blocks below row_blocks: p.wpr warps join the pieces of one (row, head).
// The others: the weights of 256 cache rows of one (sequence, KV head).
template <int D>
__global__ void __launch_bounds__(kPaFinThreads) pa_finish_kernel(const __grid_constant__ PaParams p)
{
    constexpr int E = D / 32;
    constexpr int kWarps = kPaFinThreads / 32;
    __shared__ float sh_o[kWarps][D];
    __shared__ float sh_lse2[128];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const PaSched s = *p.sched;
    if (blockIdx.x < p.row_blocks) {
        const int sub = warp % p.wpr;
        const long long task = static_cast<long long>(blockIdx.x) * (kWarps / p.wpr) + warp / p.wpr;
        const int r = static_cast<int>(task / p.Hq), h = static_cast<int>(task % p.Hq);
        const bool active = r < s.N;
        float acc[E];
#pragma unroll
        for (int i = 0; i < E; ++i) acc[i] = 0.f;
        float2 ml = make_float2(-INFINITY, 0.f);
        if (active) {
            const int b = p.row_seq[r];
            const PaSeq q = p.seqs[b];
            const PaParts x = pa_parts<D>(p, s, q, r, b, h / p.G, h % p.G);
            ml = pa_join_ml(x, lane);
            const int n = x.count();
            if (ml.x != -INFINITY) {
#pragma unroll 4
                for (int e = sub; e < n; e += p.wpr) {
                    const float w = ex2_approx(x.ml(e).x - ml.x);
                    const float* src = x.o<D>(e) + lane * E;
                    float v[E];
                    if constexpr (E == 4) {
                        const float4 t = __ldg(reinterpret_cast<const float4*>(src));
                        v[0] = t.x, v[1] = t.y, v[2] = t.z, v[3] = t.w;
                    } else {
                        const float2 t = __ldg(reinterpret_cast<const float2*>(src));
                        v[0] = t.x, v[1] = t.y;
                    }
                    // a piece whose keys the row does not see has weight 0 and an O of zeros
#pragma unroll
                    for (int i = 0; i < E; ++i) acc[i] += w * v[i];
                }
            }
        }
        if (p.wpr > 1) {
#pragma unroll
            for (int i = 0; i < E; ++i) sh_o[warp][lane * E + i] = acc[i];
            __syncthreads();
            if (sub == 0) {
                for (int w = 1; w < p.wpr; ++w)
#pragma unroll
                    for (int i = 0; i < E; ++i) acc[i] += sh_o[warp + w][lane * E + i];
            }
        }
        if (active && sub == 0) {
            const float inv = ml.y > 0.f ? 1.0f / ml.y : 0.f;
            uint32_t* dst = reinterpret_cast<uint32_t*>(p.o + (static_cast<int64_t>(r) * p.Hq + h) * D + lane * E);
#pragma unroll
            for (int i = 0; i < E; i += 2) dst[i / 2] = cvt_bf16x2(acc[i] * inv, acc[i + 1] * inv);
            if (p.lse && lane == 0) p.lse[static_cast<int64_t>(h) * p.cap + r] = (ml.x + log2f(ml.y)) * kLn2;
        }
        return;
    }
    const int chunks = (p.L + kPaFinThreads - 1) / kPaFinThreads;
    const int id = blockIdx.x - p.row_blocks;
    const int bh = id / chunks, b = bh / p.Hkv, kvh = bh % p.Hkv;
    const int key = (id % chunks) * kPaFinThreads + tid;
    const PaSeq q = p.seqs[b];
    if ((id % chunks) * kPaFinThreads >= q.len) return;
    const int n_keys = min(q.len, q.tiles * 128);  // keys with logits
    float add = 0.f;
    for (int m0 = 0; m0 < q.n * p.G; m0 += 128) {
        const int nm = min(128, q.n * p.G - m0);
        for (int i = warp; i < nm; i += kWarps) {
            const int m = m0 + i;
            const PaParts x = pa_parts<D>(p, s, q, q.row0 + m / p.G, b, kvh, m % p.G);
            const float2 ml = pa_join_ml(x, lane);
            // a row that sees no key has logits -inf only: weight 0
            if (lane == 0) sh_lse2[i] = ml.x == -INFINITY ? INFINITY : ml.x + log2f(ml.y);
        }
        __syncthreads();
        if (key < n_keys) {
            const float* lg = p.logits + (static_cast<int64_t>(bh) * p.L + key) * p.R + m0;
            for (int i = 0; i < nm; ++i) add += exp2f(lg[i] - sh_lse2[i]);  // exp2f: no weight is flushed to zero
        }
        __syncthreads();
    }
    if (key < q.len) {
        const int64_t at = static_cast<int64_t>(bh) * p.L + key;
        p.mass_out[at] = (key < q.len - p.n_new ? p.mass_in[at] : 0.f) + add;
    }
}

// ---------------------------------------------------------------------- host
int check_prefix(const logo_dims& d, int n_new, int P)
{
    int rc = check_dims(d);
    if (rc != LOGO_OK) return rc;
    if (n_new < 1 || P < 0) return LOGO_ERR_INVALID_ARG;
    if (static_cast<int64_t>(d.B) * n_new > (1ll << 24)) return LOGO_ERR_UNSUPPORTED;
    if (static_cast<int64_t>(d.B) * n_new * (d.Hq / d.Hkv) > (1ll << 30)) return LOGO_ERR_UNSUPPORTED;
    return LOGO_OK;
}

// Fills the sizes of a call and lays out its workspace; returns its bytes.
size_t prefix_layout(const logo_dims& d, int n_new, int P, bool with_mass, char* base, PaParams* p)
{
    const int64_t G = d.Hq / d.Hkv, cap = static_cast<int64_t>(d.B) * n_new, R = n_new * G;
    const int64_t rt_own = (R + kPaRows - 1) / kPaRows;
    const int64_t tiles = d.Hkv * ((P + kPaTile - 1) / kPaTile) +
                          static_cast<int64_t>(d.B) * d.Hkv * rt_own * ((d.T + kPaTile - 1) / kPaTile);
    const int64_t ctas = std::max<int64_t>(1, std::min<int64_t>(tiles, device_sm_count()));
    // (m, l, O) sets of a piece: copies x rows, at most 8 x 32 or 4 x 64
    const int64_t w_pre = std::min<int64_t>(256, 8 * cap * G), w_own = std::min<int64_t>(256, 8 * R);
    const int64_t slots_pre = P > 0 ? d.Hkv + ctas : 0;
    const int64_t slots_own = d.B * d.Hkv * rt_own + ctas;
    const bool wide = P > 0 && cap * G > kPaRows;
    const int64_t w_rows = wide ? cap * G : 0, w_rt = (w_rows + 127) / 128;
    const int64_t w_units = wide ? std::max<int64_t>(w_rt * d.Hkv, kPaWideUnits) : 0;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = round_up(off + bytes, 256);
        return base + at;
    };
    char* sched = take(sizeof(PaSched));
    char* seqs = take(d.B * sizeof(PaSeq));
    char* row_seq = take(cap * sizeof(int32_t));
    char* ml_pre = take(slots_pre * w_pre * 8);
    char* o_pre = take(slots_pre * w_pre * d.D * 4);
    char* ml_own = take(slots_own * w_own * 8);
    char* o_own = take(slots_own * w_own * d.D * 4);
    char* wq = take(wide ? (w_rt + 1) * 128 * d.Hkv * d.D * 2 : 0);
    char* wpos = take(w_rows * sizeof(int32_t));
    char* wtiles = take(w_units * sizeof(GlobalTile));
    char* wcount = take(4 * sizeof(int32_t));
    char* wo_part = take(w_units * 128 * d.D * 4);
    char* wm_part = take(w_units * 128 * 4);
    char* wl_part = take(w_units * 128 * 4);
    char* wo = take(w_rows * d.Hkv * d.D * 4);
    char* wml = take(w_rows * d.Hkv * 8);
    char* logits = take(with_mass ? static_cast<size_t>(d.B) * d.Hkv * d.T * R * 4 : 0);
    if (p) {
        p->sched = reinterpret_cast<PaSched*>(sched);
        p->seqs = reinterpret_cast<PaSeq*>(seqs);
        p->row_seq = reinterpret_cast<int32_t*>(row_seq);
        p->ml_pre = reinterpret_cast<float*>(ml_pre);
        p->o_pre = reinterpret_cast<float*>(o_pre);
        p->ml_own = reinterpret_cast<float*>(ml_own);
        p->o_own = reinterpret_cast<float*>(o_own);
        p->wq = reinterpret_cast<logo_bf16*>(wq);
        p->wpos = reinterpret_cast<int32_t*>(wpos);
        p->wtiles = reinterpret_cast<GlobalTile*>(wtiles);
        p->wcount = reinterpret_cast<int32_t*>(wcount);
        p->wo_part = reinterpret_cast<float*>(wo_part);
        p->wm_part = reinterpret_cast<float*>(wm_part);
        p->wl_part = reinterpret_cast<float*>(wl_part);
        p->wo = reinterpret_cast<float*>(wo);
        p->wml = reinterpret_cast<float*>(wml);
        p->logits = reinterpret_cast<float*>(logits);
        p->B = d.B;
        p->L = d.T;
        p->Hq = d.Hq;
        p->Hkv = d.Hkv;
        p->G = static_cast<int>(G);
        p->n_new = n_new;
        p->P = P;
        p->cap = static_cast<int>(cap);
        p->R = static_cast<int>(R);
        p->rt_own_max = static_cast<int>(rt_own);
        p->w_pre = static_cast<int>(w_pre);
        p->w_own = static_cast<int>(w_own);
        p->nCta = static_cast<int>(ctas);
    }
    return off;
}

template <int D>
int launch_prefix(PaParams& p, cudaStream_t st)
{
    using C = PaCfg<D>;
    static bool attr_done = false;  // benign race: setting the attribute twice is harmless
    if (!attr_done) {
        if (set_smem_limit(pa_rows_kernel<D>, C::kSmemBytes) != cudaSuccess) return LOGO_ERR_CUDA;
        attr_done = true;
    }
    if (p.P > 0 && static_cast<long long>(p.cap) * p.G > kPaRows) {
        const int n_sm = device_sm_count();
        const int64_t rows = static_cast<int64_t>(p.cap) * p.G, rts = (rows + 127) / 128;
        pa_wide_prep_kernel<D><<<static_cast<int>(std::min<int64_t>(rts * 128, 4 * n_sm)), 256, 0, st>>>(p, n_sm);
        TileShares t{};
        t.q = p.wq;
        t.k = p.kp;
        t.v = p.vp;
        t.pos = p.wpos;
        t.tiles = p.wtiles;
        t.n_tiles = p.wcount;
        t.next_item = p.wcount + 1;
        t.o_part = p.wo_part;
        t.m_part = p.wm_part;
        t.l_part = p.wl_part;
        t.q_rows = (rts + 1) * 128;
        t.T = p.P;
        t.Hkv = p.Hkv;
        t.n_items = static_cast<int>(std::min<int64_t>(std::max<int64_t>(rts * p.Hkv, kPaWideUnits), 1 << 30));
        t.scale_log2 = p.scale_log2;
        const int rc = launch_tile_shares(t, D, st);
        if (rc != LOGO_OK) return rc;
        pa_wide_join_kernel<D><<<4 * n_sm, 128, 0, st>>>(p);
    }
    pa_rows_kernel<D><<<p.nCta, kPaThreads, C::kSmemBytes, st>>>(p);
    // few (row, head) pairs have many pieces each: eight warps a pair then
    const long long pairs = static_cast<long long>(p.cap) * p.Hq;
    p.wpr = pairs < 2048 ? 8 : 1;
    const long long row_blocks = (pairs * p.wpr + 7) / 8;
    const long long mass_blocks =
        p.mass_out ? static_cast<long long>(p.B) * p.Hkv * ((p.L + kPaFinThreads - 1) / kPaFinThreads) : 0;
    if (row_blocks + mass_blocks > 0x7fffffffll) return LOGO_ERR_UNSUPPORTED;
    p.row_blocks = static_cast<int>(row_blocks);
    pa_finish_kernel<D><<<static_cast<unsigned>(row_blocks + mass_blocks), kPaFinThreads, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}

}  // namespace

int prefix_attn_tu_status(int clear) { return read_tu_status(clear); }

}  // namespace logo

using namespace logo;

extern "C" size_t logo_decode_prefix_workspace_size(logo_dims dims, int n_new, int prefix_len, int with_mass)
{
    if (check_prefix(dims, n_new, prefix_len) != LOGO_OK) return 0;
    return prefix_layout(dims, n_new, prefix_len, with_mass != 0, nullptr, nullptr);
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
    const size_t need = prefix_layout(dims, n_new, prefix_len, mass_out != nullptr, nullptr, nullptr);
    if (!workspace || workspace_bytes < need || !aligned16(workspace)) return LOGO_ERR_WORKSPACE;
    PaParams p{};
    prefix_layout(dims, n_new, prefix_len, mass_out != nullptr, static_cast<char*>(workspace), &p);
    if (!encode_bf16_4d(&p.tm_kc, k_cache, dims.D, dims.Hkv, dims.T, dims.B, 64, 128) ||
        !encode_bf16_4d(&p.tm_vc, v_cache, dims.D, dims.Hkv, dims.T, dims.B, 64, 128))
        return LOGO_ERR_CUDA;
    if (prefix_len > 0 && (!encode_bf16_4d(&p.tm_kp, k_prefix, dims.D, dims.Hkv, prefix_len, 1, 64, 128) ||
                           !encode_bf16_4d(&p.tm_vp, v_prefix, dims.D, dims.Hkv, prefix_len, 1, 64, 128)))
        return LOGO_ERR_CUDA;
    p.q = q;
    p.kp = k_prefix;
    p.vp = v_prefix;
    p.seq_len = seq_len;
    p.pos = pos;
    p.cu_q = cu_q;
    p.n_sel = n_sel_total;
    p.o = o_c;
    p.lse = lse_c;
    p.mass_in = mass_in;
    p.mass_out = mass_out;
    p.scale_log2 = scale * kLog2e;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dims.D == 128 ? launch_prefix<128>(p, st) : launch_prefix<64>(p, st);
}
