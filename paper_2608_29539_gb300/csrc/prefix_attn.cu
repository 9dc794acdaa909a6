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
// (m, l, O), and a later launch joins each row's pieces.
//
// pa_rows_kernel: one persistent CTA per SM walks an equal share of all key
//   tiles (128 keys of a segment and KV head).  One warp keeps a ring of K and
//   V tiles in flight (TMA, 160 KB), two lay out the next pieces and their rows
//   of Q, and eight do the products with warp-level MMA: decoding has a group's
//   few heads per sequence as rows, mostly padding for a tcgen05 tile, and HBM
//   bounds it (a tile's 64 KB take 2790 clocks at an SM's share of it).  Each
//   warp takes its own keys with its own running maximum and sum, so that none
//   waits for another inside a piece.  8 sequences, 16 heads, D = 128, own caches
//   of up to 16384: 566 MB in 92 us, 6.2 TB/s.  Caches of 1000 to 2000 rows are read
//   at 2.6 to 4.5 TB/s: their runs are short, and start, Q and joins are latency.
// Many rows of a long prefix per KV head are bound by the products and go to the
//   tcgen05 kernel of the prefill's global branch instead ("wide" below), in tiles
//   of 128 rows and shares of the prefix (pa_rows_kernel lays them out first, on the
//   device as the count of rows is known only there).
// pa_finish_kernel (or pa_join_kernel, then pa_mass_kernel): joins each (row,
//   head)'s pieces, and adds up the weights exp(x - lse) of every own cache row from
//   the logits that pa_rows_kernel wrote down (4 bytes a row and key, written and
//   read; reading K again, and multiplying again, would be 2 D bytes a key for all
//   rows: fewer from D / 4 rows a sequence and KV head on, a form that was not
//   built).  11 us of that call, latency most of it.
#include <cuda_bf16.h>

#include <algorithm>
#include <cstdint>

#include "attn_common.cuh"
#include "host_common.h"
#include "logo_status.cuh"
#include "prefix_sched.h"
#include "sm100.cuh"

namespace logo {
namespace {

constexpr int kPaWarps = 8;      // warps that do the products; then the TMA warp, then the planners
constexpr int kPaPlanners = 2;
constexpr int kPaThreads = 384;  // three warpgroups, for the register split
constexpr uint32_t kPaRegsRows = 184, kPaRegsLoad = 136;
static_assert(128 * (2 * kPaRegsRows + kPaRegsLoad) <= kPaThreads * 168, "register split exceeds the launch allocation");
constexpr int kPaTile = 128;         // keys per tile
constexpr int kPaBox = 32;           // rows of an own cache that a copy brings: a warp's keys of a tile
constexpr int kPaRows = 32;          // rows of a piece at most
constexpr int kPaWideUnits = 1216;   // (row tile, share, KV head) units that the wide prefix is cut into, or one share
constexpr int kPaMassThreads = 256;
// A prefix is read again for each 32 rows by pa_rows_kernel up to this many units
// (see PaSched) an SM, as counted at run time, and the tcgen05 kernel is not
// launched where no selection can pass the second number.  Call times, read again
// against tcgen05: 22 row tiles, 4 KV heads, 2 keys 41.1 us, 51.1; 16, 16 and 500
// keys (10 units) 51.4, 62.0.  With all and with half of the rows selected: 16 row
// tiles, 8 KV heads, 2000 keys (15 units) 43.5 and 33.1, against 41.3 and 37.7; 10
// row tiles, 4 KV heads, 8000 keys (17 units) 40.8 and 31.5, against 39.4 and 36.8.
constexpr int kPaNarrow = 8, kPaNarrowCap = 18;
constexpr int kPaMaxR = 8192;        // n_new * (Hq / Hkv) at most (the weights' row statistics in shared memory)

template <int D>
struct PaCfg {
    static constexpr int kTileBytes = kPaTile * D * 2;  // one K or V tile
    static constexpr int kHalfBytes = kPaTile * 128;    // its 64-column half (128-byte rows)
    static constexpr int kStages = D == 128 ? 5 : 10;   // K and V tiles in turn: 160 KB
    static constexpr int kQHalf = kPaRows * 128;
    static constexpr int kQBytes = kPaRows * D * 2;
    static constexpr int kOffRing = 2 * kQBytes;  // after two Q tiles
    static constexpr int kOffMerge = kOffRing + kStages * kTileBytes;
    static constexpr int kMergeBytes = kPaWarps * 16 * (64 + 8) * 4;  // the warps' 16 rows of O, 64 columns at a time
    static constexpr int kSmemBytes = kOffMerge + kMergeBytes + 1024;
};

// What the weights need to know of a sequence (base: its first unit on the line).
struct PaSeq {
    int row0, n, len, tiles, base;
};

// ... and the join of a packed row: where its sequence's parts are.
struct alignas(16) PaRow {
    int row0, base, tiles;  // tiles 0: none of its sequence's keys is seen
    uint32_t b_rts;         // sequence, row tiles - 1 (B <= 2^24, kPaMaxR / kPaRows row tiles at most)
    __device__ __forceinline__ int b() const { return static_cast<int>(b_rts & 0xffffffu); }
    __device__ __forceinline__ int rts() const { return static_cast<int>(b_rts >> 24) + 1; }
};
static_assert(kPaMaxR / kPaRows <= 256, "PaRow holds eight bits");

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
    PaSeq* seqs;               // [B]
    PaRow* rows;               // [cap]
    float *o_pre, *ml_pre;     // prefix pieces: [slot][w_pre][D], [slot][w_pre][2]
    float *o_own, *ml_own;
    float* lse2;               // [Hkv][cap * G] log2 units; +infinity for a row without a key
    // wide prefix: row M = r * G + g
    logo_bf16* wq;  // [rows + 128, Hkv, D]
    int32_t* wpos;  // [rows]
    GlobalTile* wtiles;
    int32_t* wcount;  // tiles, next item, shares, row tiles
    float *wo_part, *wm_part, *wl_part;
    float* logits;  // [B, Hkv, R, Lp] log2 units, R = n_new * G, Lp = L up to a multiple of 4
    int B, L, Lp, Hq, Hkv, G, n_new, P, cap, R, rt_own_max, w_pre, w_own, nCta;
    int n_sm, rt_narrow;  // rt_narrow: row tiles of the prefix up to which it is not wide
    float scale_log2;
};

// Own cache rows that token i of a sequence with len tokens sees.
__device__ __forceinline__ int own_visible(int len, int n_new, int i) { return min(len, max(0, len - n_new + i + 1)); }

// Token of packed row r among its sequence's new ones (no load on the way to
// the keys when there is one only).
__device__ __forceinline__ int token_of(const PaParams& p, int r) { return p.n_new == 1 ? 0 : __ldg(p.pos + r); }

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
        o.tiles = (own_visible(o.len, p.n_new, token_of(p, row1 - 1)) + kPaTile - 1) / kPaTile;
        o.rts = (o.n * p.G + kPaRows - 1) / kPaRows;
    }
    return o;
}

// The same from shared memory, where the batch fits there (seqs, else NULL): the
// loads of one are two round trips, for every sequence that a share passes, and a
// batch of which few are selected has many to pass.
__device__ __forceinline__ OwnSeq seq_at(const PaParams& p, const OwnSeq* seqs, int b)
{
    return seqs ? seqs[b] : own_seq(p, b);
}

// Sequence of packed row r.
__device__ __forceinline__ int seq_of(const PaParams& p, const OwnSeq* seqs, int r)
{
    if (!seqs) return seq_of_row(p.cu_q, p.B, r);
    int lo = 0, hi = p.B - 1;  // the last one that starts at or before r
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (seqs[mid].row0 <= r) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Units of a sequence on the line.
__device__ __forceinline__ int own_units(const PaParams& p, const OwnSeq& o)
{
    return o.tiles > 0 ? (kRunCost + o.tiles) * o.rts * p.Hkv : 0;
}

// One piece: key tiles [t0, t1) of a segment for one row tile and KV head.
struct PaPiece {
    int own;
    int b, kvh, row0, nrows;  // own: sequence; rows row0 .. of the segment's (row, head) list
    int seg_row0;             // first packed row of the segment
    int t0, t1, len;          // len: keys of the segment
    int slot;
};

struct PaIter {
    int u, u1, base, c, b;  // position, end, first unit of sequence b, share, b

    __device__ __forceinline__ bool next(const PaParams& p, const PaSched& s, const OwnSeq* seqs, PaPiece* it)
    {
        for (;;) {
            if (u >= u1) return false;
            int tiles, first;  // of the run: tiles, first unit
            if (u < s.K) {
                tiles = s.PT;
                const int k = u / (kRunCost + tiles);
                first = k * (kRunCost + tiles);
                it->own = 0;
                it->b = 0;
                it->kvh = k / s.rt_pre;
                it->row0 = k % s.rt_pre * kPaRows;
                it->nrows = min(kPaRows, s.N * p.G - it->row0);
                it->seg_row0 = 0;
                it->len = p.P;
                it->slot = k + c;
            } else {
                OwnSeq o = seq_at(p, seqs, b);
                int units = own_units(p, o);
                while (u - base >= units) {  // ends: u < u1 <= the line's length
                    base += units;
                    ++b;
                    o = seq_at(p, seqs, b);
                    units = own_units(p, o);
                }
                tiles = o.tiles;
                const int k = (u - base) / (kRunCost + tiles);
                first = base + k * (kRunCost + tiles);
                it->own = 1;
                it->b = b;
                it->kvh = k / o.rts;
                const int r = k % o.rts;
                it->row0 = r * kPaRows;
                it->nrows = min(kPaRows, o.n * p.G - it->row0);
                it->seg_row0 = o.row0;
                it->len = o.len;
                const int id = (b * p.Hkv + it->kvh) * p.rt_own_max + r;
                it->slot = id + c;
            }
            it->t0 = max(0, u - first - kRunCost);
            u = min(u1, first + kRunCost + tiles);
            it->t1 = max(0, u - first - kRunCost);
            if (it->t1 > it->t0) return true;  // else the share ends in the run's overhead
        }
    }
};

// What a warp of the products keeps from piece to piece.
struct PaWarp {
    uint32_t sQ, sRing, kv_full, kv_empty;  // kv_*: the first barrier, the others 8 bytes on
    volatile int* abort_flag;
    float* merge;     // [warp][16][64 + 8]
    float2* sh_ml;    // [warp][16]
    const int* vis;   // [kPaRows] keys that each row of the piece sees
    int warp, lane, n;  // n: tiles consumed, K and V counted
};

// All 256 threads of the products: true if every thread's `ok` is.
__device__ __forceinline__ bool products_sync_and(bool ok)
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.and.pred q, 1, 256, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}\n"
        : "=r"(r)
        : "r"(ok ? 1u : 0u)
        : "memory");
    return r != 0;
}

__device__ __forceinline__ void products_sync() { asm volatile("barrier.cta.sync 1, 256;" ::: "memory"); }

// acc + 0 x for two packed bf16: stays 0 unless one is infinite or NaN.
__device__ __forceinline__ uint32_t add_zero_times_bf16x2(uint32_t acc, uint32_t x)
{
    asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(x), "r"(0u));
    return acc;
}

// One piece, by the eight warps in two groups of four, a warp taking 32 keys of a
// tile.  More than 16 rows: each group takes 16 rows, of every tile.  Up to 16:
// the groups take the tiles in turn.  Either way a warp has two independent
// blocks of 16 keys in flight, and fetches fragments a batch ahead of the
// products that use them, as two warps a scheduler hide little of each other's
// latency; and there is one code path (a second one, met by a few SMs only, cost
// them 8 us of instruction fetches).  16 sequences of up to 8192 keys, 8 KV heads,
// 32 rows: 49.8 us a call, 271 MB at 80% of the measured HBM rate.  Then the warps' results are joined in shared memory.
// Returns false, to all warps, if a wait of any gave up.
template <int D, bool DRAFTS>
__device__ __forceinline__ bool pa_piece(const PaParams& p, const PaPiece& it, PaWarp& w, bool ok)
{
    using C = PaCfg<D>;
    constexpr int NT = D / 8, KS = D / 16;
    const int lane = w.lane, gid = lane >> 2, tig = lane & 3, mi = lane >> 3, rr = lane & 7;
    const bool with_logits = it.own && p.mass_out != nullptr;
    const bool split_rows = it.nrows > 16;
    const int group = split_rows ? 4 : 8;  // warps that share the rows' keys
    const int rg = split_rows ? w.warp >> 2 : 0, k0 = (w.warp & 3) * 32;  // row group, first key of a tile
    // this lane's rows: 16 rg + 8 i + gid
    int vis[2];
    float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f}, oc[NT][4];
    uint32_t qa[KS][4];
#pragma unroll
    for (int i = 0; i < 2; ++i) vis[i] = ok ? w.vis[16 * rg + 8 * i + gid] : 0;
    const int vis_all = __shfl_sync(0xffffffffu, vis[0], 0);  // keys that every row of the group sees (later rows see more)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) oc[nt][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
        ldsm_x4(w.sQ + (ks / 4) * C::kQHalf + sw128_offset(16 * rg + (mi & 1) * 8 + rr, (ks % 4) * 2 + (mi >> 1)), qa[ks][0],
                qa[ks][1], qa[ks][2], qa[ks][3]);

    for (int t = it.t0; t < it.t1 && ok; ++t) {
        const int stK = w.n % C::kStages, fK = w.n / C::kStages;
        const int stV = (w.n + 1) % C::kStages, fV = (w.n + 1) / C::kStages;
        w.n += 2;
        const uint32_t sK = w.sRing + stK * C::kTileBytes, sV = w.sRing + stV * C::kTileBytes;
        ok = mbar_wait(w.kv_full + 8 * stK, fK & 1, w.abort_flag);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;  // the warp leaves together
        const int end = it.len - t * kPaTile;  // rows of the tile that hold a token
        if ((!split_rows && ((t - it.t0) & 1) != w.warp >> 2) || end <= k0) {
            // the other group's tile, or no keys for this warp: released once it has
            // landed (earlier, the release could fall into the stage's previous phase)
            if (lane == 0) mbar_arrive(w.kv_empty + 8 * stK);
            ok = mbar_wait(w.kv_full + 8 * stV, fV & 1, w.abort_flag);
            if (!(ok = __all_sync(0xffffffffu, ok))) break;
            if (lane == 0) mbar_arrive(w.kv_empty + 8 * stV);
            continue;
        }
        // ---- S = Q K^T over 2 x 16 keys (two 8-key halves each)
        float sc[2][2][4];
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[st][nt][i] = 0.f;
        {
            uint32_t f[2][4][4];  // a batch: two steps of the head dimension x two blocks of keys
            auto fetch = [&](int bt) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int ks = bt * 2 + i / 2, st = i % 2;
                    uint32_t(&x)[4] = f[bt & 1][i];
                    ldsm_x4(sK + (ks / 4) * C::kHalfBytes +
                                sw128_offset(k0 + st * 16 + (mi >> 1) * 8 + rr, (ks % 4) * 2 + (mi & 1)),
                            x[0], x[1], x[2], x[3]);
                }
            };
            fetch(0);
#pragma unroll
            for (int bt = 0; bt < KS / 2; ++bt) {
                if (bt + 1 < KS / 2) fetch(bt + 1);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int ks = bt * 2 + i / 2, st = i % 2;
                    const uint32_t(&x)[4] = f[bt & 1][i];
                    mma_bf16_16816(sc[st][0], qa[ks], x[0], x[1]);
                    mma_bf16_16816(sc[st][1], qa[ks], x[2], x[3]);
                }
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(w.kv_empty + 8 * stK);
        ok = mbar_wait(w.kv_full + 8 * stV, fV & 1, w.abort_flag);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
        if (it.own && end < k0 + 32) {
            // a cache row past the length may hold anything: zero its V, so that P = 0
            // keeps it out of the product
            for (int i = lane; i < 32 * (D / 8); i += 32) {
                const int row = k0 + i / (D / 8), ch = i % (D / 8);
                if (row >= end) st_shared_v4(sV + (ch >> 3) * C::kHalfBytes + sw128_offset(row, ch & 7), 0u, 0u, 0u, 0u);
            }
            fence_proxy_async_smem();  // ordered before the stage's next TMA write
            __syncwarp();
        }
        // the first of V's fragments, in flight during the softmax
        uint32_t f[2][4][4];  // a batch: two 16-column steps x two blocks of keys
        auto fetch = [&](int bt) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int col = (bt * 2 + i / 2) * 16 + (mi >> 1) * 8, st = i % 2;
                uint32_t(&x)[4] = f[bt & 1][i];
                ldsm_x4_trans(sV + (col / 64) * C::kHalfBytes +
                                  sw128_offset(k0 + st * 16 + (mi & 1) * 8 + rr, (col % 64) / 8),
                              x[0], x[1], x[2], x[3]);
            }
        };
        fetch(0);
        // a draft that some rows see and others do not: if its V is infinite or NaN, the
        // product would carry 0 * V into the rows that do not (82 sequences of 7 new
        // tokens, 192-token caches, D = 64: 22.8 us a call, 22.1 without the check)
        uint32_t odd_v = 0;
        const int all = vis_all - t * kPaTile;
        if (DRAFTS && it.own && all < min(end, k0 + 32)) {
            const int r0 = max(all, k0), n = (min(end, k0 + 32) - r0) * (D / 8);
#pragma unroll 1
            for (int i = lane; i < n; i += 32) {
                const uint4 v = ld_shared_v4(sV + (D > 64 ? (i % (D / 8) >> 3) * C::kHalfBytes : 0) +
                                             sw128_offset(r0 + i / (D / 8), i & 7));
                odd_v = add_zero_times_bf16x2(odd_v, v.x);
                odd_v = add_zero_times_bf16x2(odd_v, v.y);
                odd_v = add_zero_times_bf16x2(odd_v, v.z);
                odd_v = add_zero_times_bf16x2(odd_v, v.w);
            }
        }
        // ---- online softmax; keys at and past `vis` are not seen (their K may be
        //      anything, NaN included)
        const int key0 = t * kPaTile + k0 + 2 * tig;
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = sc[st][nt][i] * p.scale_log2;
                    sc[st][nt][i] = key0 + st * 16 + nt * 8 + (i & 1) < vis[i >> 1] ? x : -INFINITY;
                    mx[i >> 1] = fmaxf(mx[i >> 1], sc[st][nt][i]);
                }
        if (with_logits) {
            // (a pair of keys at a time; the second may be the first past the length)
            const int row = it.row0 + 16 * rg + gid;
            float* lg = p.logits + ((static_cast<int64_t>(it.b) * p.Hkv + it.kvh) * p.R + row) * p.Lp + key0;
            const bool r0 = 16 * rg + gid < it.nrows, r1 = 16 * rg + 8 + gid < it.nrows;
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
                    const int off = st * 16 + nt * 8;
                    if (key0 + off < it.len) {
                        if (r0) *reinterpret_cast<float2*>(lg + off) = make_float2(sc[st][nt][0], sc[st][nt][1]);
                        if (r1)
                            *reinterpret_cast<float2*>(lg + 8 * static_cast<int64_t>(p.Lp) + off) =
                                make_float2(sc[st][nt][2], sc[st][nt][3]);
                    }
                }
        }
        bool grow = false;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
            mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
            // O is rescaled only when the maximum has grown by more than 2^8: until
            // then l and O hold values up to 2^8 times larger, which fp32 takes without
            // loss (and bf16's P: its precision is relative)
            grow |= mx[i] > m_run[i] + 8.0f;
        }
        if (__any_sync(0xffffffffu, grow)) {
            float alpha[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                alpha[i] = 1.f;
                if (mx[i] > m_run[i] + 8.0f) {
                    alpha[i] = ex2_approx(m_run[i] - mx[i]);  // 0 while nothing was seen
                    m_run[i] = mx[i];
                    l_run[i] *= alpha[i];
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                oc[nt][0] *= alpha[0];
                oc[nt][1] *= alpha[0];
                oc[nt][2] *= alpha[1];
                oc[nt][3] *= alpha[1];
            }
        }
        uint32_t pa[2][4];
        const float m0 = m_run[0] == -INFINITY ? 0.f : m_run[0], m1 = m_run[1] == -INFINITY ? 0.f : m_run[1];
#pragma unroll
        for (int st = 0; st < 2; ++st) {
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sc[st][nt][i] = ex2_approx(sc[st][nt][i] - (i < 2 ? m0 : m1));
                    l_run[i >> 1] += sc[st][nt][i];  // this lane's keys; the quad's are added at the end
                }
            // P as the A fragment: rows = rows, k = the 16 keys; rounded to bf16, the
            // type that V has and the product takes (2^-8 of each weight at most; l is
            // summed before it)
            pa[st][0] = pack_bf16x2(sc[st][0][0], sc[st][0][1]);
            pa[st][1] = pack_bf16x2(sc[st][0][2], sc[st][0][3]);
            pa[st][2] = pack_bf16x2(sc[st][1][0], sc[st][1][1]);
            pa[st][3] = pack_bf16x2(sc[st][1][2], sc[st][1][3]);
        }
        // ---- O += P V
        if (DRAFTS && __any_sync(0xffffffffu, odd_v & 0x7fff7fffu)) {
            // key by key, over the keys that a row sees
#pragma unroll 1
            for (int j = 0; j < 32; ++j) {
                const int st = j >> 4, src = (lane & ~3) | (j >> 1 & 3), key = t * kPaTile + k0 + j;
                const uint32_t w0 = st ? (j & 8 ? pa[1][2] : pa[1][0]) : (j & 8 ? pa[0][2] : pa[0][0]);
                const uint32_t w1 = st ? (j & 8 ? pa[1][3] : pa[1][1]) : (j & 8 ? pa[0][3] : pa[0][1]);
                const uint32_t x0 = __shfl_sync(0xffffffffu, w0, src), x1 = __shfl_sync(0xffffffffu, w1, src);
                const float p0 = __uint_as_float(j & 1 ? x0 & 0xffff0000u : x0 << 16);
                const float p1 = __uint_as_float(j & 1 ? x1 & 0xffff0000u : x1 << 16);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint32_t v = ld_shared_u32(sV + (nt >> 3) * C::kHalfBytes + sw128_offset(k0 + j, nt & 7) + 4 * tig);
                    const float lo = __uint_as_float(v << 16), hi = __uint_as_float(v & 0xffff0000u);
                    if (key < vis[0]) oc[nt][0] += p0 * lo, oc[nt][1] += p0 * hi;
                    if (key < vis[1]) oc[nt][2] += p1 * lo, oc[nt][3] += p1 * hi;
                }
            }
        } else {
#pragma unroll
            for (int bt = 0; bt < NT / 4; ++bt) {
                if (bt + 1 < NT / 4) fetch(bt + 1);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int np = bt * 2 + i / 2, st = i % 2;
                    const uint32_t(&x)[4] = f[bt & 1][i];
                    mma_bf16_16816(oc[2 * np], pa[st], x[0], x[1]);
                    mma_bf16_16816(oc[2 * np + 1], pa[st], x[2], x[3]);
                }
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(w.kv_empty + 8 * stV);
    }

    // ---- the warps' (m, l, O) joined, 64 columns at a time, or all 128 where 8 rows
    //      leave room (columns 64 .. 127 lie where rows 8 .. 15 would)
    float l[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        l[i] = l_run[i] + __shfl_xor_sync(0xffffffffu, l_run[i], 1);
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    }
    // (all warps have left the tiles, and the last piece's join)
    if (!products_sync_and(ok)) return false;
    constexpr int kCols = 64, kStride = kCols + 8;  // rows 8 floats off a multiple of 32: no bank conflicts
    const bool few = D > kCols && it.nrows <= 8;
    const int64_t at = static_cast<int64_t>(it.slot) * (it.own ? p.w_own : p.w_pre);
    float* o_part = (it.own ? p.o_own : p.o_pre) + at * D;
    float2* ml_part = reinterpret_cast<float2*>(it.own ? p.ml_own : p.ml_pre) + at;
    float* mine = w.merge + w.warp * 16 * kStride + gid * kStride + 2 * tig;
    const int tid = w.warp * 32 + lane, shift = few ? 5 : 4;  // float4s of a row in a round: 1 << shift
#pragma unroll
    for (int c0 = 0; c0 < D; c0 += kCols) {
        if (c0 > 0) {
            if (few) break;
            products_sync();
        }
#pragma unroll
        for (int nt = 0; nt < kCols / 8; ++nt) {
            const float(&lo)[4] = oc[c0 / 8 + nt];
            const float(&hi)[4] = oc[(D > kCols && c0 == 0 ? kCols / 8 : c0 / 8) + nt];
            *reinterpret_cast<float2*>(mine + nt * 8) = make_float2(lo[0], lo[1]);
            *reinterpret_cast<float2*>(mine + 8 * kStride + nt * 8) =
                few ? make_float2(hi[0], hi[1]) : make_float2(lo[2], lo[3]);
        }
        if (c0 == 0 && tig == 0) {
            w.sh_ml[w.warp * 16 + gid] = make_float2(m_run[0], l[0]);
            w.sh_ml[w.warp * 16 + 8 + gid] = make_float2(m_run[1], l[1]);
        }
        products_sync();
        for (int i = tid; i < it.nrows << shift; i += kPaWarps * 32) {
            const int row = i >> shift, c = i & ((1 << shift) - 1);
            const int from = split_rows ? (row >> 4) * 4 : 0;  // the row's first warp
            const float2* ml = w.sh_ml + from * 16 + (row & 15);
            float f[kPaWarps], M = -INFINITY, L = 0.f;
            float2 part[kPaWarps];
#pragma unroll
            for (int k = 0; k < kPaWarps; ++k) {
                part[k] = k < group ? ml[k * 16] : make_float2(-INFINITY, 0.f);
                M = fmaxf(M, part[k].x);
            }
            const float Mu = M == -INFINITY ? 0.f : M;
            const float* src = w.merge + (from * 16 + (few ? row + 8 * (c >> 4) : row & 15)) * kStride + (c & 15) * 4;
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kPaWarps; ++k) {
                f[k] = ex2_approx(part[k].x - Mu);
                L += f[k] * part[k].y;
                if (k < group) {
                    const float4 v = *reinterpret_cast<const float4*>(src + k * 16 * kStride);
                    a.x += f[k] * v.x, a.y += f[k] * v.y, a.z += f[k] * v.z, a.w += f[k] * v.w;
                }
            }
            if (c0 == 0 && c == 0) ml_part[row] = make_float2(M, L);
            *reinterpret_cast<float4*>(o_part + static_cast<int64_t>(row) * D + c0 + c * 4) = a;
        }
    }
    return true;
}

// Rows, positions and tiles of the wide prefix, by one warp of every CTA beside
// the other roles.  The last CTA's picks the number of shares that each row
// tile's key range is cut into: the least time of the busiest SM, an item (row
// tile, share, KV head) counted with 6 key blocks for its start and its join.
// Items lie share by share, so that the SMs work on the same keys at the same
// time.
template <int D>
__device__ __forceinline__ void wide_prep(const PaParams& p, const PaSched& s, const OwnSeq* seqs, int lane)
{
    const int rows = s.wide ? s.N * p.G : 0, nRT = (rows + 127) / 128;
    // a row: [KV head][g][D] of q -> [KV head][D] for each g
    const int vecs = p.Hkv * (D / 8);
    for (int M = blockIdx.x; M < nRT * 128; M += gridDim.x) {
        uint4* dst = reinterpret_cast<uint4*>(p.wq + static_cast<int64_t>(M) * p.Hkv * D);
        if (M >= rows) {  // the last tile's idle rows: finite
            for (int v = lane; v < vecs; v += 32) dst[v] = make_uint4(0u, 0u, 0u, 0u);
            continue;
        }
        const int r = M / p.G, g = M % p.G, b = seq_of(p, seqs, r);
        const uint4* src =
            reinterpret_cast<const uint4*>(p.q + (static_cast<int64_t>(b) * p.n_new + token_of(p, r)) * p.Hq * D);
#pragma unroll 4
        for (int v = lane; v < vecs; v += 32) dst[v] = src[(v / (D / 8) * p.G + g) * (D / 8) + v % (D / 8)];
        if (lane == 0) p.wpos[M] = p.P - 1;
    }
    if (blockIdx.x != gridDim.x - 1) return;
    const int blocks = (p.P + 127) / 128;
    const int most = rows > 0 ? max(1, min(min(blocks, kPaWideUnits / (nRT * p.Hkv)), 255)) : 0;
    unsigned int best = ~0u;
    for (int n = lane + 1; n <= most; n += 32) {
        const long long items = static_cast<long long>(nRT) * p.Hkv * n;
        const long long cost = (items + p.n_sm - 1) / p.n_sm * ((blocks + n - 1) / n + 6);
        best = min(best, static_cast<unsigned int>(min(cost, 0xfffffell) << 8) | static_cast<unsigned int>(n));
    }
    best = __reduce_min_sync(0xffffffffu, best);
    const int ns = rows > 0 ? best & 255 : 0;
    for (int e = lane; e < nRT * ns; e += 32) {
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
    if (lane == 0) {
        p.wcount[0] = nRT * ns;
        p.wcount[1] = 0;
        p.wcount[2] = ns;
        p.wcount[3] = nRT;
    }
}

// DRAFTS: a sequence may bring several new tokens, which see different keys (without
// them the check of the unseen ones' V is left out: 128 sequences of 512 tokens 46.3
// us a call, 48.2 with it).
template <int D, bool DRAFTS>
__global__ void __launch_bounds__(kPaThreads, 1) pa_rows_kernel(const __grid_constant__ PaParams p)
{
    using C = PaCfg<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ __align__(8) uint64_t bar_q_full[2], bar_q_empty[2], bar_kv_full[C::kStages], bar_kv_empty[C::kStages];
    __shared__ __align__(8) uint64_t bar_go;  // the first piece's loads of Q are on their way
    __shared__ float2 sh_ml[kPaWarps * 16];
    __shared__ int sh_vis[2][kPaRows], sh_scan[kPaThreads / 32], sh_base, sh_b0;
    __shared__ PaPiece sh_piece[2];
    __shared__ OwnSeq sh_seq[kPaThreads];
    __shared__ volatile int abort_flag;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    const uint32_t sQ = smem_u32(smem), sRing = smem_u32(smem + C::kOffRing);
    if (tid == 0) {
        abort_flag = 0;
        sh_b0 = 0;
        mbar_init(smem_u32(&bar_go), 1);
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
    const OwnSeq* seqs = p.B <= kPaThreads ? sh_seq : nullptr;
    int mine = 0;
    for (int b = tb0; b < tb1; ++b) {
        const OwnSeq o = own_seq(p, b);
        mine += own_units(p, o);
        if (seqs) sh_seq[b] = o;
    }
    __syncwarp();
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) sh_scan[warp] = incl;
    __syncthreads();
    PaSched s;
    s.N = N;
    s.PT = (p.P + kPaTile - 1) / kPaTile;
    s.rt_pre = (N * p.G + kPaRows - 1) / kPaRows;
    s.wide = p.wq && s.rt_pre > p.rt_narrow;
    s.K = N > 0 && p.P > 0 && !s.wide ? s.rt_pre * p.Hkv * (kRunCost + s.PT) : 0;
    int excl = s.K + incl - mine;
    s.total = s.K;
    for (int k = 0; k < kPaThreads / 32; ++k) {
        if (k < warp) excl += sh_scan[k];
        s.total += sh_scan[k];
    }
    s.n = min(p.nCta, s.total);
    s.rate = s.total > 0 ? static_cast<float>(s.n) / static_cast<float>(s.total) : 0.f;
    PaIter iter;
    iter.c = cta;
    iter.u = cta < s.n ? share_start(s, cta) : 0;
    iter.u1 = cta < s.n ? share_start(s, cta + 1) : 0;
    if (tid == 0) sh_base = s.K;
    __syncthreads();
    // the sequence that the share starts in (a share that starts in the prefix
    // meets its sequences from the first one on)
    if (iter.u < iter.u1 && iter.u >= excl && iter.u < excl + mine) {
        int base = excl, b = tb0;
        for (; b < tb1; ++b) {
            const OwnSeq o = seq_at(p, seqs, b);
            const int units = own_units(p, o);
            if (iter.u < base + units) break;
            base += units;
        }
        sh_b0 = b;
        sh_base = base;
    }
    if (cta == s.n % p.nCta) {  // for the join and the weights (by a CTA without a share, if there is one)
        if (tid == 0) *p.sched = s;
        int base = excl;
        for (int b = tb0; b < tb1; ++b) {
            const OwnSeq o = seq_at(p, seqs, b);
            p.seqs[b] = PaSeq{o.row0, o.n, o.len, o.tiles, base};
            const PaRow row{o.row0, base, o.tiles, static_cast<uint32_t>(b) | static_cast<uint32_t>(o.rts - 1) << 24};
            for (int r = o.row0; r < o.row0 + o.n; ++r) p.rows[r] = row;
            base += own_units(p, o);
        }
    }
    __syncwarp();  // whole warps from here on (setmaxnreg wants them)
    __syncthreads();
    __syncwarp();
    iter.b = sh_b0;
    iter.base = sh_base;

    if (warp >= kPaWarps) {
        setmaxnreg_dec<kPaRegsLoad>();
        PaPiece it;
        if (warp == kPaWarps && lane == 0) {
            // -------------------------------------------------- K and V tiles
            const uint64_t pol = policy_evict_first();
            int n = 0;
            bool ok = true;
            while (ok && iter.next(p, s, seqs, &it)) {
                // when all SMs fill their rings, their first tiles are 24 MB, and a load
                // behind them takes 4 us
                if (n == 0 && it.t1 - it.t0 > 1 && !(ok = mbar_wait(smem_u32(&bar_go), 0, &abort_flag))) break;
                const CUtensorMap* tk = it.own ? &p.tm_kc : &p.tm_kp;
                const CUtensorMap* tv = it.own ? &p.tm_vc : &p.tm_vp;
                for (int t = it.t0; t < it.t1 && ok; ++t) {
                    for (int kv = 0; kv < 2; ++kv, ++n) {
                        const int st = n % C::kStages, f = n / C::kStages;
                        if (!(ok = mbar_wait(smem_u32(&bar_kv_empty[st]), (f & 1) ^ 1, &abort_flag))) break;
                        const uint32_t bar = smem_u32(&bar_kv_full[st]);
                        // of an own cache only the boxes that hold tokens (74 sequences of 139
                        // tokens in the mean, 16 KV heads: 64.4 us a call, 66.3 with whole tiles)
                        const int step = it.own ? kPaBox : kPaTile;
                        const int boxes = it.own ? min(kPaTile / kPaBox, (it.len - t * kPaTile + kPaBox - 1) / kPaBox) : 1;
                        mbar_arrive_expect_tx(bar, boxes * step * D * 2);
                        for (int h = 0; h < D / 64; ++h)
                            for (int i = 0; i < boxes; ++i)
                                tma_load_4d(sRing + st * C::kTileBytes + h * C::kHalfBytes + i * step * 128, kv ? tv : tk, bar,
                                            64 * h, it.kvh, t * kPaTile + i * step, it.b, pol);
                    }
                }
            }
            // all copies land before the CTA exits (the products may have given up on
            // one after the last was issued; else this finds them all there)
            for (int k = max(0, n - C::kStages); k < n; ++k)
                mbar_wait_drain(smem_u32(&bar_kv_full[k % C::kStages]), (k / C::kStages) & 1);
        } else if (warp > kPaWarps && warp <= kPaWarps + kPaPlanners) {
            // -------------------------------------------------- pieces and Q: the
            // planners take the pieces in turn, so that one's loads are in flight
            // (into registers) while the other waits for its Q buffer
            for (int piece = 0;; ++piece) {
                const bool more = iter.next(p, s, seqs, &it);
                const int qb = piece & 1;
                if (piece % kPaPlanners != warp - kPaWarps - 1) {
                    if (!more) break;
                    continue;
                }
                // lane = row: what it sees and where its q lies.  Rows past nrows see
                // nothing, and their Q is whatever is there (a row of S depends on its
                // own row of Q alone)
                if (!more) it.nrows = 0;  // the end
                int vis = 0;
                int64_t at = 0;
                if (lane < it.nrows) {
                    const int m = it.row0 + lane, r = it.seg_row0 + m / p.G, g = m % p.G;
                    const int b = it.own ? it.b : seq_of(p, seqs, r);
                    const int i = token_of(p, r);
                    vis = it.own ? own_visible(it.len, p.n_new, i) : it.len;
                    at = ((static_cast<int64_t>(b) * p.n_new + i) * p.Hq + it.kvh * p.G + g) * D;
                }
                __syncwarp();
                constexpr int kChunks = D / 8;       // 16-byte chunks of a row
                const uint32_t qbase = sQ + qb * C::kQBytes;
                uint4 v[kChunks];  // 32 rows: row k * 32 / kChunks + lane / kChunks
#pragma unroll
                for (int k = 0; k < kChunks; ++k) {
                    const int row = (k * 32 + lane) / kChunks;
                    const int64_t src = __shfl_sync(0xffffffffu, at, row);
                    v[k] = make_uint4(0u, 0u, 0u, 0u);
                    if (row < it.nrows) v[k] = __ldg(reinterpret_cast<const uint4*>(p.q + src) + lane % kChunks);
                }
                if (piece == 0 && lane == 0) mbar_arrive(smem_u32(&bar_go));
                bool ok = mbar_wait(smem_u32(&bar_q_empty[qb]), ((piece >> 1) & 1) ^ 1, &abort_flag);
                if (!(ok = __all_sync(0xffffffffu, ok))) break;
#pragma unroll
                for (int k = 0; k < kChunks; ++k) {
                    const int row = (k * 32 + lane) / kChunks, ch = lane % kChunks;
                    if (row < it.nrows)
                        st_shared_v4(qbase + (ch >> 3) * C::kQHalf + sw128_offset(row, ch & 7), v[k].x, v[k].y, v[k].z,
                                     v[k].w);
                }
                sh_vis[qb][lane] = vis;
                if (lane == 0) sh_piece[qb] = it;
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_q_full[qb]));
                if (!more) break;
            }
        } else if (warp == kPaWarps + 1 + kPaPlanners && p.wq) {
            wide_prep<D>(p, s, seqs, lane);
        }
        return;
    }
    // ---------------------------------------------------------- products
    setmaxnreg_inc<kPaRegsRows>();
    PaWarp w;
    w.sRing = sRing;
    w.kv_full = smem_u32(&bar_kv_full[0]);
    w.kv_empty = smem_u32(&bar_kv_empty[0]);
    w.abort_flag = &abort_flag;
    w.merge = reinterpret_cast<float*>(smem + C::kOffMerge);
    w.sh_ml = sh_ml;
    w.warp = warp;
    w.lane = lane;
    w.n = 0;
    for (int piece = 0;; ++piece) {
        const int qb = piece & 1;
        bool ok = mbar_wait(smem_u32(&bar_q_full[qb]), (piece >> 1) & 1, &abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        PaPiece it = sh_piece[qb];
        // the warps stay together whatever happens: each comes to the barrier in
        // pa_piece (or here, at the end of the work) with its own `ok`
        if (!ok || it.nrows == 0) it.t1 = it.t0 = 0;
        if (!ok) it.nrows = 1;
        w.sQ = sQ + qb * C::kQBytes;
        w.vis = sh_vis[qb];
        if (it.nrows == 0) {
            products_sync_and(true);
            break;
        }
        if (!pa_piece<D, DRAFTS>(p, it, w, ok)) break;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bar_q_empty[qb]));
    }
}

// --------------------------------------------------------------------- join
// The parts of one (row, head) from one segment: part e is m[e * s_ml], l[e *
// s_ml], o + e * s_o.
struct PaParts {
    const float *m, *l, *o;
    int64_t s_ml, s_o;
    int n;
};

// What the parts are found by that does not depend on the row.
struct PaPre {
    int ns, nrt;  // wide prefix: shares, row tiles
};

__device__ __forceinline__ PaPre pa_pre(const PaParams& p)
{
    return PaPre{p.wq ? p.wcount[2] : 0, p.wq ? p.wcount[3] : 0};
}

// Parts of packed row r, head g of KV head kvh: x[0] of the prefix, x[1] of the
// cache of sequence b, whose first packed row is row0 and whose runs are rts row
// tiles a KV head from unit `base` on (tiles 0: no own key is seen).
template <int D>
__device__ __forceinline__ void pa_parts(const PaParams& p, const PaSched& s, const PaPre& pre, int r, int b, int row0,
                                         int base, int tiles, int rts, int kvh, int g, PaParts (&x)[2])
{
    x[0] = x[1] = PaParts{nullptr, nullptr, nullptr, 0, 0, 0};
    if (tiles > 0) {
        const int m = (r - row0) * p.G + g, id = (b * p.Hkv + kvh) * p.rt_own_max + m / kPaRows;
        const PaRun run = run_of(s, base + (kvh * rts + m / kPaRows) * (kRunCost + tiles), tiles);
        const int64_t at = static_cast<int64_t>(id + run.c0) * p.w_own + m % kPaRows;
        x[1] = PaParts{p.ml_own + 2 * at, p.ml_own + 2 * at + 1, p.o_own + at * D, 2 * p.w_own,
                       static_cast<int64_t>(p.w_own) * D, run.n};
    }
    if (s.wide) {
        const int m = r * p.G + g;
        const int64_t step = static_cast<int64_t>(pre.nrt) * p.Hkv * 128;
        const int64_t at = (static_cast<int64_t>(m / 128) * p.Hkv + kvh) * 128 + m % 128;
        x[0] = PaParts{p.wm_part + at, p.wl_part + at, p.wo_part + at * D, step, step * D, pre.ns};
    } else if (s.K > 0) {
        const int m = r * p.G + g, id = kvh * s.rt_pre + m / kPaRows;
        const PaRun run = run_of(s, id * (kRunCost + s.PT), s.PT);
        const int64_t at = static_cast<int64_t>(id + run.c0) * p.w_pre + m % kPaRows;
        x[0] = PaParts{p.ml_pre + 2 * at, p.ml_pre + 2 * at + 1, p.o_pre + at * D, 2 * p.w_pre,
                       static_cast<int64_t>(p.w_pre) * D, run.n};
    }
}

// The maximum of a part with row sum l: -infinity where the row saw no key of it.
// Maxima skip NaN, sums do not: a part whose logits were all NaN has the maximum of
// an empty one, and must not pass for it.
__device__ __forceinline__ float part_max(float m, float l) { return m == -INFINITY && l != l ? 0.f : m; }

// lse of a row in log2 units for the weights exp2(x - lse2): x = -inf where the
// row sees nothing, and a row that sees no key at all gets weights 0.
__device__ __forceinline__ float weight_lse2(float M, float Ls) { return M == -INFINITY ? INFINITY : M + log2f(Ls); }

// WPR warps join the parts of one (row, head), CH parts at a time: their
// statistics and O are loaded together and added up with a running maximum,
// which saves a round trip to memory.
template <int D, int WPR, int CH>
__device__ __forceinline__ void pa_join(const PaParams& p, int block)
{
    constexpr int E = D / 32, kWarps = 8;
    __shared__ float sh_o[WPR > 1 ? kWarps : 1][D];
    __shared__ float2 sh_ml[kWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = warp % WPR;
    const int task = block * (kWarps / WPR) + warp / WPR;
    const int r = min(task / p.Hq, p.cap - 1), h = task % p.Hq, kvh = h / p.G, g = h % p.G;
    // loads that depend on nothing, together
    const PaSched s = *p.sched;
    const PaRow row = p.rows[r];
    const PaPre pre = pa_pre(p);
    const bool active = task / p.Hq < s.N;
    float acc[E], M = -INFINITY, Ls = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] = 0.f;
    if (active) {
        PaParts x[2];
        pa_parts<D>(p, s, pre, r, row.b(), row.row0, row.base, row.tiles, row.rts(), kvh, g, x);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            for (int e0 = sub * CH; e0 < x[k].n; e0 += WPR * CH) {
                float vm[CH], vl[CH], v[CH][E], top = M;
#pragma unroll
                for (int e = 0; e < CH; ++e) {
                    const int at = min(e0 + e, x[k].n - 1);
                    vm[e] = __ldg(x[k].m + at * x[k].s_ml);
                    vl[e] = __ldg(x[k].l + at * x[k].s_ml);
                    const float* src = x[k].o + at * x[k].s_o + lane * E;
                    if constexpr (E == 4) {
                        const float4 t = __ldg(reinterpret_cast<const float4*>(src));
                        v[e][0] = t.x, v[e][1] = t.y, v[e][2] = t.z, v[e][3] = t.w;
                    } else {
                        const float2 t = __ldg(reinterpret_cast<const float2*>(src));
                        v[e][0] = t.x, v[e][1] = t.y;
                    }
                }
#pragma unroll
                for (int e = 0; e < CH; ++e) {
                    vm[e] = e0 + e < x[k].n ? part_max(vm[e], vl[e]) : -INFINITY;
                    top = fmaxf(top, vm[e]);
                }
                if (top == -INFINITY) continue;
                const float a = ex2_approx(M - top);
                Ls *= a;
#pragma unroll
                for (int i = 0; i < E; ++i) acc[i] *= a;
#pragma unroll
                for (int e = 0; e < CH; ++e) {
                    // a part whose keys the row does not see has weight 0 and an O of zeros
                    const float w = ex2_approx(vm[e] - top);
                    Ls += w * vl[e];
#pragma unroll
                    for (int i = 0; i < E; ++i) acc[i] += w * v[e][i];
                }
                M = top;
            }
        }
    }
    if constexpr (WPR > 1) {
#pragma unroll
        for (int i = 0; i < E; ++i) sh_o[warp][lane * E + i] = acc[i];
        if (lane == 0) sh_ml[warp] = make_float2(M, Ls);
        __syncthreads();
        if (sub == 0) {
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < WPR; ++w) top = fmaxf(top, sh_ml[warp + w].x);
            Ls = 0.f;
#pragma unroll
            for (int i = 0; i < E; ++i) acc[i] = 0.f;
            if (top != -INFINITY) {
#pragma unroll
                for (int w = 0; w < WPR; ++w) {
                    const float f = ex2_approx(sh_ml[warp + w].x - top);
                    Ls += f * sh_ml[warp + w].y;
#pragma unroll
                    for (int i = 0; i < E; ++i) acc[i] += f * sh_o[warp + w][lane * E + i];
                }
            }
            M = top;
        }
    }
    if (active && sub == 0) {
        const float inv = Ls == 0.f ? 0.f : 1.0f / Ls;  // (0: no key is seen)
        uint32_t* dst = reinterpret_cast<uint32_t*>(p.o + (static_cast<int64_t>(r) * p.Hq + h) * D + lane * E);
#pragma unroll
        for (int i = 0; i < E; i += 2) dst[i / 2] = cvt_bf16x2(acc[i] * inv, acc[i + 1] * inv);
        if (lane == 0) {
            if (p.lse) p.lse[static_cast<int64_t>(h) * p.cap + r] = (M + log2f(Ls)) * kLn2;  // -inf without a key
            if (p.lse2) p.lse2[(static_cast<int64_t>(kvh) * p.cap + r) * p.G + g] = weight_lse2(M, Ls);
        }
    }
}

// ------------------------------------------------------------------ weights
// A block: one of the `chunks` equal shares of the cache rows of one (sequence,
// KV head), 1024 / rs of them at a time: four a thread (a row's logits of
// neighbouring keys lie together), by rs threads (a power of two), each of which
// takes every rs-th of the R rows.  The logits come mostly from L2 and their
// latency bounds the pass, so a thread has four 16-byte loads in flight, the
// first of them during the statistics.  FUSED: the block forms the rows' lse from
// their parts itself; else it reads what the join has left.
template <int D, bool FUSED>
__device__ __forceinline__ void pa_mass(const PaParams& p, int block, int chunks, int rs, float* sh_lse2)
{
    constexpr int U = 4;  // rows in flight
    __shared__ float4 sh_add[kPaMassThreads];
    const int at = kPaMassThreads / rs, keys = 4 * at;
    const int bh = block / chunks, ch = block % chunks;
    const int b = bh / p.Hkv, kvh = bh % p.Hkv, tid = threadIdx.x, sub = tid / at;
    const PaSeq q = p.seqs[b];
    PaSched s{};
    PaPre pre{};
    if constexpr (FUSED) {
        s = *p.sched;
        pre = pa_pre(p);
    }
    const int steps = (q.len + keys - 1) / keys;
    const int k0 = static_cast<int>(static_cast<int64_t>(steps) * ch / chunks) * keys;
    const int k1 = static_cast<int>(static_cast<int64_t>(steps) * (ch + 1) / chunks) * keys;
    if (k0 >= k1) return;
    const int nm = q.tiles > 0 ? q.n * p.G : 0;
    const int n_keys = min(q.len, q.tiles * kPaTile);  // cache rows with logits
    const int64_t base = static_cast<int64_t>(bh) * p.L;
    const float* lg = p.logits + static_cast<int64_t>(bh) * p.R * p.Lp;
    float4 x[U];
    auto load = [&](int key, int m0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int m = m0 + u * rs;
            x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (key < n_keys && m < nm)
                x[u] = __ldg(reinterpret_cast<const float4*>(lg + static_cast<int64_t>(m) * p.Lp + key));
        }
    };
    int key = k0 + tid % at * 4;
    load(key, sub);
    if constexpr (FUSED) {
        // eight lanes a row
        const int rts = (q.n * p.G + kPaRows - 1) / kPaRows;
        const int l8 = tid & 7;
        for (int m0 = 0; m0 < nm; m0 += kPaMassThreads / 8) {
            const int m = m0 + (tid >> 3);
            float M = -INFINITY, Ls = 0.f;
            if (m < nm) {
                PaParts part[2];
                pa_parts<D>(p, s, pre, q.row0 + m / p.G, b, q.row0, q.base, q.tiles, rts, kvh, m % p.G, part);
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    for (int e = l8; e < part[k].n; e += 8) {
                        const float vl = __ldg(part[k].l + e * part[k].s_ml);
                        const float vm = part_max(__ldg(part[k].m + e * part[k].s_ml), vl);
                        if (vm == -INFINITY) continue;
                        const float top = fmaxf(M, vm);
                        Ls = Ls * ex2_approx(M - top) + vl * ex2_approx(vm - top);
                        M = top;
                    }
            }
#pragma unroll
            for (int o = 4; o; o >>= 1) {
                const float m2 = __shfl_xor_sync(0xffffffffu, M, o), l2 = __shfl_xor_sync(0xffffffffu, Ls, o);
                const float top = fmaxf(M, m2);
                if (top != -INFINITY) Ls = Ls * ex2_approx(M - top) + l2 * ex2_approx(m2 - top);
                M = top;
            }
            if (m < nm && l8 == 0) sh_lse2[m] = weight_lse2(M, Ls);
        }
    } else {
        const float* l2 = p.lse2 + (static_cast<int64_t>(kvh) * p.cap + q.row0) * p.G;
        for (int m = tid; m < nm; m += kPaMassThreads) sh_lse2[m] = l2[m];
    }
    __syncthreads();
    for (int kb = k0;; key += keys) {
        float old[4], add[4] = {0.f, 0.f, 0.f, 0.f};
        if (sub == 0)
#pragma unroll
            for (int e = 0; e < 4; ++e) old[e] = key + e < q.len - p.n_new ? p.mass_in[base + key + e] : 0.f;
        for (int m0 = sub; m0 < nm; m0 += U * rs) {
            if (m0 > sub) load(key, m0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (m0 + u * rs >= nm) break;
                const float l = sh_lse2[m0 + u * rs];
                // exp2f: no weight is flushed to zero
                add[0] += exp2f(x[u].x - l);
                add[1] += exp2f(x[u].y - l);
                add[2] += exp2f(x[u].z - l);
                add[3] += exp2f(x[u].w - l);
            }
        }
        kb += keys;
        if (kb < k1) load(key + keys, sub);
        if (rs > 1) {
            sh_add[tid] = make_float4(add[0], add[1], add[2], add[3]);
            __syncthreads();
            if (sub == 0)
                for (int k = 1; k < rs; ++k) {
                    const float4 v = sh_add[k * at + tid];
                    add[0] += v.x, add[1] += v.y, add[2] += v.z, add[3] += v.w;
                }
        }
        if (sub == 0)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (key + e < q.len) p.mass_out[base + key + e] = old[e] + (key + e < n_keys ? add[e] : 0.f);
        if (kb >= k1) break;
        if (rs > 1) __syncthreads();
    }
}

// Up to kPaFusedR rows a (sequence, KV head), join and weights share a launch: a
// block of the weights then forms its rows' lse from their parts itself, eight
// lanes a row, which saves the launch between the two (call times, fused against
// not: 41.9 us against 46.0 at 40 rows, 4 sequences; 90.5 against 97.1 at 64 rows,
// 16 sequences of 4096; 110 against 115 at 256 rows, 16 sequences of 2048).  Every
// block does that work: at 512 rows it costs more (96.3 us against 94.1).
constexpr int kPaFusedR = 256;

template <int D, int WPR, int CH>
__global__ void __launch_bounds__(256, 4)
    pa_finish_kernel(const __grid_constant__ PaParams p, int join_blocks, int chunks, int rs)
{
    __shared__ float sh_lse2[kPaFusedR];
    const int mass = gridDim.x - join_blocks;  // first, as they take longer
    if (blockIdx.x >= mass) pa_join<D, WPR, CH>(p, blockIdx.x - mass);
    else pa_mass<D, true>(p, blockIdx.x, chunks, rs, sh_lse2);
}

template <int D, int WPR, int CH>
__global__ void __launch_bounds__(256) pa_join_kernel(const __grid_constant__ PaParams p)
{
    pa_join<D, WPR, CH>(p, blockIdx.x);
}

__global__ void __launch_bounds__(kPaMassThreads) pa_mass_kernel(const __grid_constant__ PaParams p, int chunks, int rs)
{
    extern __shared__ float sh_dyn[];
    pa_mass<128, false>(p, blockIdx.x, chunks, rs, sh_dyn);  // (D does not enter without the parts)
}

// Join and weights.
template <int D, int WPR, int CH>
int launch_finish(PaParams& p, cudaStream_t st)
{
    const long long pairs = static_cast<long long>(p.cap) * p.Hq;
    const int join = static_cast<int>((pairs + 8 / WPR - 1) / (8 / WPR));
    if (!p.mass_out) {
        p.lse2 = nullptr;
        pa_join_kernel<D, WPR, CH><<<join, 256, 0, st>>>(p);
        return LOGO_OK;
    }
    int rs = 1;  // four rows a thread, while four threads suffice for that
    while (rs < 4 && rs * 4 < p.R) rs *= 2;
    const int keys = 4 * kPaMassThreads / rs;
    const long long bh = static_cast<long long>(p.B) * p.Hkv;
    // one wave of blocks, as their start and the statistics cost as much as a few steps
    const int chunks = static_cast<int>(std::min<long long>((p.L + keys - 1) / keys, std::max(1ll, 4ll * p.n_sm / bh)));
    const long long mass = bh * chunks;
    if (join + mass > 0x7fffffffll) return LOGO_ERR_UNSUPPORTED;
    if (p.R <= kPaFusedR) {
        p.lse2 = nullptr;
        pa_finish_kernel<D, WPR, CH><<<static_cast<unsigned>(join + mass), 256, 0, st>>>(p, join, chunks, rs);
    } else {
        pa_join_kernel<D, WPR, CH><<<join, 256, 0, st>>>(p);
        pa_mass_kernel<<<static_cast<unsigned>(mass), kPaMassThreads, p.R * sizeof(float), st>>>(p, chunks, rs);
    }
    return LOGO_OK;
}

// ---------------------------------------------------------------------- host
int check_prefix(const logo_dims& d, int n_new, int P)
{
    int rc = check_dims(d);
    if (rc != LOGO_OK) return rc;
    if (n_new < 1 || P < 0) return LOGO_ERR_INVALID_ARG;
    const int64_t G = d.Hq / d.Hkv, cap = static_cast<int64_t>(d.B) * n_new;
    if (cap > (1ll << 24) || cap * G > (1ll << 28) || n_new * G > kPaMaxR) return LOGO_ERR_UNSUPPORTED;
    if (P > (1 << 30) || d.Hkv > (1 << 16)) return LOGO_ERR_UNSUPPORTED;
    // tiles, pieces and (row, head) pairs are counted in 32 bits
    const int64_t rt = (n_new * G + kPaRows - 1) / kPaRows;
    const int64_t tiles = d.Hkv * ((P + 127ll) / 128) + d.B * rt * d.Hkv * ((d.T + 127ll) / 128);
    if (tiles > (1ll << 28) || (cap * G / 128 + 1) * d.Hkv > (1ll << 23)) return LOGO_ERR_UNSUPPORTED;
    return LOGO_OK;
}

// Fills the sizes of a call and lays out its workspace; returns its bytes.
size_t prefix_layout(const logo_dims& d, int n_new, int P, bool with_mass, char* base, PaParams* p)
{
    const int64_t G = d.Hq / d.Hkv, cap = static_cast<int64_t>(d.B) * n_new, R = n_new * G;
    const int64_t rt_own = (R + kPaRows - 1) / kPaRows;
    // row tiles of the prefix up to which it is not wide
    const int64_t sms = device_sm_count(), PT = (P + kPaTile - 1ll) / kPaTile;
    const int64_t rt_pre = P > 0 ? (cap * G + kPaRows - 1) / kPaRows : 0;
    const int64_t run_units = PT + kRunCost;
    const int64_t rt_narrow =
        rt_pre * d.Hkv * run_units <= kPaNarrowCap * sms ? rt_pre : std::max<int64_t>(1, kPaNarrow * sms / (d.Hkv * run_units));
    const int64_t tiles = rt_narrow * d.Hkv * PT + d.B * d.Hkv * rt_own * ((d.T + kPaTile - 1) / kPaTile);
    const int64_t ctas = std::max<int64_t>(1, std::min(tiles, sms));
    const int64_t w_pre = std::min<int64_t>(kPaRows, cap * G), w_own = std::min<int64_t>(kPaRows, R);
    const int64_t runs_own = d.B * d.Hkv * rt_own, Lp = round_up(d.T, 4);
    const int64_t slots_pre = P > 0 ? rt_narrow * d.Hkv + ctas : 0, slots_own = runs_own + ctas;
    const bool wide = rt_pre > rt_narrow;
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
    char* row_info = take(cap * sizeof(PaRow));
    char* ml_pre = take(slots_pre * w_pre * 8);
    char* o_pre = take(slots_pre * w_pre * d.D * 4);
    char* ml_own = take(slots_own * w_own * 8);
    char* o_own = take(slots_own * w_own * d.D * 4);
    char* lse2 = take(with_mass ? d.Hkv * cap * G * 4 : 0);
    char* wq = take(wide ? (w_rt + 1) * 128 * d.Hkv * d.D * 2 : 0);
    char* wpos = take(w_rows * sizeof(int32_t));
    char* wtiles = take(w_units * sizeof(GlobalTile));
    char* wcount = take(4 * sizeof(int32_t));
    char* wo_part = take(w_units * 128 * d.D * 4);
    char* wm_part = take(w_units * 128 * 4);
    char* wl_part = take(w_units * 128 * 4);
    char* logits = take(with_mass ? static_cast<size_t>(d.B) * d.Hkv * R * Lp * 4 : 0);
    if (p) {
        p->sched = reinterpret_cast<PaSched*>(sched);
        p->seqs = reinterpret_cast<PaSeq*>(seqs);
        p->rows = reinterpret_cast<PaRow*>(row_info);
        p->ml_pre = reinterpret_cast<float*>(ml_pre);
        p->o_pre = reinterpret_cast<float*>(o_pre);
        p->ml_own = reinterpret_cast<float*>(ml_own);
        p->o_own = reinterpret_cast<float*>(o_own);
        p->lse2 = reinterpret_cast<float*>(lse2);
        p->wq = wide ? reinterpret_cast<logo_bf16*>(wq) : nullptr;
        p->wpos = reinterpret_cast<int32_t*>(wpos);
        p->wtiles = reinterpret_cast<GlobalTile*>(wtiles);
        p->wcount = reinterpret_cast<int32_t*>(wcount);
        p->wo_part = reinterpret_cast<float*>(wo_part);
        p->wm_part = reinterpret_cast<float*>(wm_part);
        p->wl_part = reinterpret_cast<float*>(wl_part);
        p->logits = reinterpret_cast<float*>(logits);
        p->B = d.B;
        p->L = d.T;
        p->Lp = static_cast<int>(Lp);
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
        p->rt_narrow = static_cast<int>(rt_narrow);
    }
    return off;
}

template <int D>
int launch_prefix(PaParams& p, cudaStream_t st)
{
    using C = PaCfg<D>;
    const auto rows_kernel = p.n_new > 1 ? pa_rows_kernel<D, true> : pa_rows_kernel<D, false>;
    static OncePerDevice limit[2];
    if (limit[p.n_new > 1]([&] { return set_smem_limit(rows_kernel, C::kSmemBytes); }) != cudaSuccess) return LOGO_ERR_CUDA;
    p.n_sm = device_sm_count();
    rows_kernel<<<p.nCta, kPaThreads, C::kSmemBytes, st>>>(p);
    if (p.wq) {
        const int64_t rts = (static_cast<int64_t>(p.cap) * p.G + 127) / 128;
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
        t.n_items = static_cast<int>(std::max<int64_t>(rts * p.Hkv, kPaWideUnits));
        t.scale_log2 = p.scale_log2;
        const int rc = launch_tile_shares(t, D, st);
        if (rc != LOGO_OK) return rc;
    }
    // few (row, head) pairs: their parts are many and four warps join a pair (1024
    // pairs, 22 parts: 52.9 us a call against 54.6 with one); more pairs keep the SMs
    // busy with one (4096 pairs: 70.8 us against 77.5; 2976: 41.1 against 45.2)
    const int rc = static_cast<long long>(p.cap) * p.Hq <= 1024 ? launch_finish<D, 4, 4>(p, st) : launch_finish<D, 1, 4>(p, st);
    if (rc != LOGO_OK) return rc;
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
    if (!encode_bf16_4d(&p.tm_kc, k_cache, dims.D, dims.Hkv, dims.T, dims.B, 64, kPaBox) ||
        !encode_bf16_4d(&p.tm_vc, v_cache, dims.D, dims.Hkv, dims.T, dims.B, 64, kPaBox))
        return LOGO_ERR_CUDA;
    if (prefix_len > 0 && (!encode_bf16_4d(&p.tm_kp, k_prefix, dims.D, dims.Hkv, prefix_len, 1, 64, kPaTile) ||
                           !encode_bf16_4d(&p.tm_vp, v_prefix, dims.D, dims.Hkv, prefix_len, 1, 64, kPaTile)))
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
