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
//     a row.  P is rounded to fp16, which keeps three bits more of it than bf16 would, relative
//     to well below the row's maximum (ca_base); it comes out of S^T's fragments by a
//     transposition in registers.
// The batch's (sequence, KV head, rows, 128 keys) units form a line, sequences without a
// selected row left out.  Each group of four warps takes an equal stretch of it, a cell,
// its warps 32 keys of a unit each through a ring of their own in shared memory (cp.async;
// no warp waits for another inside a run).  All groups of an SM are one CTA: as CTAs of
// their own the hardware favoured the first ones, and the last finished a quarter later.
// A run (sequence, KV head, rows) that spans several cells is joined from their parts, in
// order, by a second launch.  H 32/8, D = 128: 32 sequences of up to 16K rows, half of them
// selected, one token: 41.8 us for 183 MB (4.4 TB/s, 66% of the copy rate); one of 262139 rows:
// 61.1 us for 302 MB; 64 x 5 drafts over up to 8K rows: 140 us for 377 MB.
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

constexpr int kCaWarps = 4;                   // of a group
constexpr int kCaGroup = 32 * kCaWarps;
constexpr int kCaKeys = 32;                   // keys of a warp's step
constexpr int kCaUnit = kCaKeys * kCaWarps;   // keys of a unit
// What is subtracted from logits lies 2^10 below a maximum, which may grow by 2^5 before what is
// summed is rescaled: weights reach 2^15, near fp16's end, so that as little as can be falls
// below its beginning.  (16 x 4 drafts, H 16/1: 29.5 us; 29.0 with 2^9 and 2^6, 29.8 with 2^11 and
// 2^4, 31.6 with 2^13 and 2^2; 64 x 5 drafts 140, 140, 140, 146.)
constexpr float kCaHead = 10.f, kCaSlack = 5.f;
constexpr int kCaMaxTiles = 4;                // tiles of 8 rows that a warp holds
constexpr int kJoinThreads = 256;

// A run that several cells have parts of: its packed rows from r0 and KV head, of which its
// rows are row0 ..., and the first and last of the cells (last -1: there is no such run).
struct __align__(16) CaOpen {
    int r0, h, row0, nrow, first, last;
    int pad[2];
};

struct CaParams {
    const uint16_t* q;
    const uint8_t *k, *v, *ks, *vs;
    const int32_t *len, *pos, *cu_q, *n_sel;
    uint16_t* o;
    float* lse;
    float* parts;   // [2 * cells][rows * D, then rows of (max, sum)]
    CaOpen* table;  // [2][cells]: the run that a cell begins and does not end, the one that it comes into
    int B, n, Hq, Hkv, G, L;
    uint32_t magic;  // ceil(2^32 / G), 0 for G = 1
    float scale2;    // scale * log2(e)

    __device__ __forceinline__ int token_of(int row) const { return magic ? __umulhi(row, magic) : row; }  // row / G
};

// Sizes of the kernel for one tile of rows (NT = 1), whose warps have all channels of
// their keys, and of the one for more, whose warps have half of the channels of half of the keys.
template <int D, int NT>
struct CaShape {
    static constexpr bool kWide = NT > 1;
    static constexpr int kRows = 8 * NT;
    // groups an SM and steps of a warp's ring: as many warps as registers allow, but for one tile of
    // rows of D = 128, where three groups find all the bytes' latency to work in and leave fewer
    // parts to join (us, three and four groups: 32 sequences of up to 16K rows, one token 41.7 and
    // 42.0, one of 262139 rows 61.0 and 61.9, 100 of 300 rows 17.2 and 18.4, 64 x 2 drafts of 8K rows
    // 58.7 and 58.5; D = 64: 16 sequences of 32K rows 48.6 and 45.7, 128 of 4K rows 48.7 and 45.4, but
    // one of 100000 33.6 and 40.9).  Three tiles, 64 x 5 drafts: 140 with three, 192 with four, which
    // spill, 159 with two; four tiles of D = 128, 32 x 8 drafts over 8K rows: 138 with two, 151 with
    // three, which spill; of D = 64: 88 with two, 74 with three, which spill 8 bytes.
    static constexpr bool kLarge = NT == 4 && D == 128;
    static constexpr int kGroups = !kWide ? (D == 128 ? 3 : 4) : kLarge ? 2 : 3, kStages = NT == 2 || NT == 3 || kLarge ? 3 : 2;
    static constexpr int kThreads = kGroups * kCaGroup;
    static constexpr int kRunCost = 2;                         // units that beginning a run costs about as much as
    static constexpr int kCodes = kCaKeys * D / 2, kScales = kCaKeys * D / 16;  // bytes a step, K or V
    static constexpr int kStage = 2 * (kCodes + kScales);
    static constexpr int kSteps = D / 16;                      // k steps of S^T, m tiles of O^T
    static constexpr int kRing = kCaWarps * kStages * kStage;
    static constexpr int kQ = NT * kSteps * 32 * 8;            // fragments of Q
    // the warps' results: rows padded for the banks; or P's fragments of two units (and the queries as they come)
    static constexpr int kRowBytes = 4 * D + 16;
    static constexpr int kMerge = kWide ? 2 * NT * 2048 : kCaWarps * kRows * kRowBytes;
    static constexpr int kStats = (kCaWarps + 1) * kRows * 8 + 4 * kRows * 4;
    static constexpr int kGroupBytes = kRing + kQ + kMerge + kStats;
    static constexpr int kSmem = kGroups * kGroupBytes;
    static_assert(!kWide || kQ + kMerge >= kRows * D * 4, "half of the sums go where Q and P were");
    static constexpr int kPart = kRows * (D + 2);              // floats of a part
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// (the first `bytes`, then zeros)
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

template <int N>
__device__ __forceinline__ void cp_async_small(uint32_t dst, const void* src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(N) : "memory");
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

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
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

// Where byte `at` (a multiple of 4) of a step's key row lies: the 16-byte pieces of
// 128-byte lines exchanged so that both kinds of loads below meet every bank once.
// The exchange repeats every 8 keys.
template <int D>
__device__ __forceinline__ uint32_t piece(uint32_t key, uint32_t at)
{
    const uint32_t x = key * (D / 2) + at, line = x >> 7;
    const uint32_t f = D == 128 ? ((line & 1) << 1) | ((line & 2) << 1) : (line & 1) << 2;
    return x ^ (f << 4);
}

__device__ __forceinline__ void group_sync(int group)
{
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(kCaGroup) : "memory");
}

// Whether x holds in any thread of the group, which all arrive.
__device__ __forceinline__ bool group_any(int group, bool x)
{
    int r;
    asm volatile(
        "{\n\t.reg .pred P, Q;\n\t"
        "setp.ne.s32 P, %3, 0;\n\t"
        "bar.red.or.pred Q, %1, %2, P;\n\t"
        "selp.s32 %0, 1, 0, Q;\n\t}"
        : "=r"(r)
        : "r"(group + 1), "n"(kCaGroup), "r"(static_cast<int>(x))
        : "memory");
    return r != 0;
}

// A run: the units of one (sequence, KV head, row block), in the line's order.  On the line
// it has room for what beginning it costs, then its units.
struct CaRun {
    int b, h, rb;
    int nrb, units, len, r0, cnt;   // of the sequence
};

// Whether sequence b has selected rows; its part of the run's description.
__device__ __forceinline__ bool ca_sequence(const CaParams& p, int b, int rows, CaRun& r)
{
    r.b = b;
    r.r0 = p.cu_q[b];
    r.cnt = min(min(p.cu_q[b + 1], *p.n_sel) - r.r0, p.n);
    r.len = max(0, min(p.len[b], p.L));
    r.units = max(1, (r.len + kCaUnit - 1) / kCaUnit);
    r.nrb = (r.cnt * p.G + rows - 1) / rows;
    return r.cnt > 0;
}

__device__ __forceinline__ void ca_next(const CaParams& p, int rows, CaRun& r)
{
    if (++r.rb < r.nrb) return;
    r.rb = 0;
    if (++r.h < p.Hkv) return;
    r.h = 0;
    int b = r.b + 1;
#pragma unroll 1
    for (; b < p.B - 1; ++b)
        if (min(p.cu_q[b + 1], *p.n_sel) > p.cu_q[b]) break;
    ca_sequence(p, b, rows, r);  // (only called where another run follows)
}

__device__ __forceinline__ uint32_t ca_weight(const CaParams& p, int b, int rows, int cost)
{
    CaRun r;
    return b < p.B && ca_sequence(p, b, rows, r) ? static_cast<uint32_t>(r.units + cost) * r.nrb * p.Hkv : 0u;
}

// How the line is cut: SM i has `each` units, one more where i < extra, in `cells` equal
// cells, one for each group as long as there are units for all.
struct CaCut {
    uint32_t each, extra, cells;

    __device__ __forceinline__ CaCut(uint32_t total, uint32_t sms, uint32_t groups)
        : each(total / sms), extra(total % sms), cells(max(1u, min(each, groups)))
    {
    }
    __device__ __forceinline__ uint32_t units(uint32_t sm) const { return each + (sm < extra); }
    __device__ __forceinline__ uint32_t begin(uint32_t sm) const { return each * sm + min(sm, extra); }
    // first unit of cell k of an SM with u units, which are no fewer than its cells
    __device__ __forceinline__ uint32_t cell(uint32_t u, uint32_t k) const { return u * k / cells; }
    __device__ __forceinline__ uint32_t cell_of(uint32_t x) const
    {
        const uint32_t big = extra * (each + 1);
        const uint32_t sm = x < big ? x / (each + 1) : extra + (x - big) / each;  // (each = 0: x < big)
        const uint32_t in = x - begin(sm), u = units(sm);
        return sm * cells + ((in + 1) * cells - 1) / u;
    }
};

// The line's length; all threads of the CTA.
__device__ __forceinline__ uint32_t ca_length(const CaParams& p, int rows, int cost, uint32_t* sh)
{
    if (p.B <= 32) return __reduce_add_sync(0xffffffffu, ca_weight(p, threadIdx.x % 32, rows, cost));  // every warp for itself
    uint32_t w = 0;
#pragma unroll 1
    for (int b = threadIdx.x; b < p.B; b += blockDim.x) w += ca_weight(p, b, rows, cost);
    w = __reduce_add_sync(0xffffffffu, w);
    if (threadIdx.x % 32 == 0) sh[threadIdx.x / 32] = w;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return __reduce_add_sync(0xffffffffu, lane < blockDim.x / 32 ? sh[lane] : 0u);
}

// The sequence whose runs hold unit x of the line, and its first unit; every warp for itself.
__device__ __forceinline__ uint2 ca_find(const CaParams& p, int rows, int cost, uint32_t x)
{
    const int lane = threadIdx.x & 31;
    uint32_t base = 0;
#pragma unroll 1
    for (int b0 = 0;; b0 += 32) {
        const uint32_t mine = ca_weight(p, b0 + lane, rows, cost);
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += y;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, base + upto > x);
        if (past || b0 + 32 >= p.B) {
            const int k = past ? __ffs(past) - 1 : 31;
            return make_uint2(b0 + k, base + __shfl_sync(0xffffffffu, upto - mine, k));
        }
        base += __shfl_sync(0xffffffffu, upto, 31);
    }
}

// A group's stretch of the line and where it begins: run, unit of it, units left to the
// stretch's end.
struct CaCell {
    uint32_t cell, cells, x1, base;  // base: of the run, on the line
    CaCut cut;
    CaRun run;
    int unit;
    bool any;
};

// Writes down what joining needs to know of the run at c, which begins in cell `first` (-1: there is none).
template <typename S>
__device__ __forceinline__ void ca_open(const CaParams& p, const CaCell& c, CaOpen& to, int first)
{
    const int row0 = c.run.rb * S::kRows;
    to.r0 = c.run.r0, to.h = c.run.h, to.row0 = row0, to.nrow = min(S::kRows, c.run.cnt * p.G - row0), to.first = first;
    to.last = first < 0 ? -1 : static_cast<int>(c.cut.cell_of(c.base + S::kRunCost + c.run.units - 1));
}

template <typename S>
__device__ __forceinline__ CaCell ca_cell(const CaParams& p, int group, uint32_t* sh)
{
    const uint32_t total = ca_length(p, S::kRows, S::kRunCost, sh);
    const CaCut cut(total, gridDim.x, S::kGroups);
    CaCell c{0, cut.cells, 0, 0, cut, {}, 0, false};
    const uint32_t units = cut.units(blockIdx.x), begin = cut.begin(blockIdx.x);
    // the entries of the table that no cell writes
    const uint32_t spare = S::kGroups - cut.cells, mine = units ? 0 : cut.cells;
    CaOpen* const enters = p.table + gridDim.x * S::kGroups;
    if (threadIdx.x < spare) {
        const uint32_t k = gridDim.x * cut.cells + blockIdx.x * spare + threadIdx.x;
        p.table[k].last = enters[k].last = -1;
    }
    if (threadIdx.x < mine) {
        const uint32_t k = blockIdx.x * cut.cells + threadIdx.x;
        p.table[k].last = enters[k].last = -1;
    }
    if (units == 0 || group >= cut.cells) return c;
    c.any = true;
    c.cell = blockIdx.x * cut.cells + group;
    const uint32_t x0 = begin + cut.cell(units, group);
    c.x1 = begin + cut.cell(units, group + 1);
    const uint2 at = ca_find(p, S::kRows, S::kRunCost, x0);
    ca_sequence(p, at.x, S::kRows, c.run);
    const uint32_t weight = c.run.units + S::kRunCost, i = (x0 - at.y) / weight;
    c.run.h = i / c.run.nrb, c.run.rb = i % c.run.nrb;
    c.base = at.y + i * weight;
    c.unit = max(0, static_cast<int>(x0 - c.base) - S::kRunCost);
    if (threadIdx.x % kCaGroup == 0) {
        p.table[c.cell].last = -1;  // (as yet)
        if (S::kWide) ca_open<S>(p, c, enters[c.cell], c.unit ? static_cast<int>(cut.cell_of(c.base + S::kRunCost)) : -1);
    }
    return c;
}

// Units of the run that begins at `base` on the line which lie before x.
template <typename S>
__device__ __forceinline__ int ca_before(const CaRun& r, uint32_t base, uint32_t x)
{
    return max(0, min(r.units, static_cast<int>(min(x - base, 0x40000000u)) - S::kRunCost));
}

// The copies of a warp's steps into its ring, with a place on the line of their own.
template <int D, typename S>
struct CaCopies {
    const CaParams& p;
    uint32_t to_codes, to_scales;  // this lane's first pieces of a stage, in shared memory
    int warp, lane;
    CaRun run;
    int unit;
    uint32_t base, x1, fill = 0;
    const uint8_t *k, *v, *ks, *vs;

    __device__ __forceinline__ CaCopies(const CaParams& p_, uint32_t ring, int warp_, int lane_, const CaCell& c)
        : p(p_), to_codes(ring + piece<D>(lane_ * 16 / (D / 2), lane_ * 16 % (D / 2))),
          to_scales(ring + 2 * S::kCodes + lane_ * (D / 16)), warp(warp_), lane(lane_), run(c.run), unit(c.unit),
          base(c.base), x1(c.x1)
    {
        point();
    }
    __device__ __forceinline__ void point()
    {
        const int64_t row0 = (static_cast<int64_t>(run.b) * p.Hkv + run.h) * p.L + static_cast<int64_t>(unit) * kCaUnit + warp * kCaKeys;
        k = p.k + row0 * (D / 2) + lane * 16;
        v = p.v + row0 * (D / 2) + lane * 16;
        ks = p.ks + (row0 + lane) * (D / 16);
        vs = p.vs + (row0 + lane) * (D / 16);
    }
    // The next step's copies, one group (an empty one past the stretch's end).
    __device__ __forceinline__ void issue()
    {
        if (base + S::kRunCost + unit < x1) {
            const int rows = run.len - unit * kCaUnit - warp * kCaKeys;
            const uint32_t to = to_codes + fill * S::kStage, tos = to_scales + fill * S::kStage;
            if (rows >= kCaKeys) {
#pragma unroll
                for (int i = 0; i < S::kCodes / 512; ++i) {
                    cp_async16(to + i * 512, k + i * 512);
                    cp_async16(to + i * 512 + S::kCodes, v + i * 512);
                }
                cp_async_small<D / 16>(tos, ks);
                cp_async_small<D / 16>(tos + S::kScales, vs);
            } else if (rows > 0) {  // rows past the end are written as zeros
#pragma unroll 1
                for (int i = 0; i < S::kCodes / 512; ++i) {
                    const bool in = (i * 512 + lane * 16) / (D / 2) < rows;
                    cp_async16(to + i * 512, in ? k + i * 512 : p.k, in ? 16 : 0);
                    cp_async16(to + i * 512 + S::kCodes, in ? v + i * 512 : p.v, in ? 16 : 0);
                }
                const bool in = lane < rows;
                cp_async_small<D / 16>(tos, in ? ks : p.ks, in ? D / 16 : 0);
                cp_async_small<D / 16>(tos + S::kScales, in ? vs : p.vs, in ? D / 16 : 0);
            }
            k += kCaUnit * (D / 2), v += kCaUnit * (D / 2), ks += kCaUnit * (D / 16), vs += kCaUnit * (D / 16);
            if (++unit == run.units) {
                base += run.units + S::kRunCost;
                unit = 0;
                if (base + S::kRunCost < x1) {
                    ca_next(p, S::kRows, run);
                    point();
                }
            }
        }
        cp_async_commit();
        fill = fill + 1 == S::kStages ? 0 : fill + 1;
    }
};

// A run's queries: bf16 rows into `raw`, then fp16 fragments scaled by a power of two a row;
// what each row sees, and the factor from its products to logits (in powers of two).
// Begins and ends with a barrier of the group.
template <int D, typename S>
__device__ __forceinline__ void ca_queries(const CaParams& p, const CaRun& run, int row0, int nrow, int group, int tid,
                                           uint8_t* raw, uint2* q_frag, int* row_vis, float* row_mul)
{
    constexpr int NS = S::kSteps;
    const int lane = tid & 31, warp = tid >> 5;
    group_sync(group);  // the rows of the stretch before are no longer read
#pragma unroll 1
    for (int x = tid; x < S::kRows * (D / 8); x += kCaGroup) {
        const int r = x / (D / 8), token = p.token_of(row0 + r);
        uint4 w = make_uint4(0, 0, 0, 0);
        int vis = 0;
        if (r < nrow) {
            const int i = max(0, min(p.pos[run.r0 + token], p.n - 1));
            vis = min(run.len, max(0, run.len - p.n + i + 1));
            const int64_t at_q = (static_cast<int64_t>(run.b) * p.n + i) * p.Hq + run.h * p.G + row0 + r - token * p.G;
            w = __ldg(reinterpret_cast<const uint4*>(p.q + at_q * D) + x % (D / 8));
        }
        reinterpret_cast<uint4*>(raw)[x] = w;
        if (x % (D / 8) == 0) row_vis[r] = vis;
    }
    group_sync(group);
#pragma unroll 1
    for (int r = warp; r < S::kRows; r += kCaWarps) {
        // the row times 2^(140 - e), e the largest exponent: below 2^14
        uint2 w = make_uint2(0, 0);
        if (lane < D / 4) w = reinterpret_cast<const uint2*>(raw + r * D * 2)[lane];
        uint32_t top = 0;
        const uint32_t bits[4] = {w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t e = bits[c] >> 23 & 0xff;
            if (e != 0xff) top = max(top, e);
        }
        top = max(16u, __reduce_max_sync(0xffffffffu, top));
        const float up = __uint_as_float((267u - top) << 23);
        float f[4];
#pragma unroll
        for (int c = 0; c < 4; ++c)
            f[c] = (bits[c] >> 23 & 0xff) == 0xff ? __uint_as_float(0x7fc00000u) : __uint_as_float(bits[c]) * up;
        if (lane < D / 4)  // channels 4 lane ... 4 lane + 3: of thread lane / NS, step lane % NS
            q_frag[((r >> 3) * NS + lane % NS) * 32 + (r & 7) * 4 + lane / NS] = make_uint2(pack_f16(f[0], f[1]), pack_f16(f[2], f[3]));
        if (lane == 0) row_mul[r] = fmaxf(p.scale2 * __uint_as_float((top - 13) << 23), 1.2e-38f);  // 2^(top - 140)
    }
    group_sync(group);
}

// S^T of a warp's step, raw products: row g of a tile is key (g >> 1) + 4 (g & 1), row g + 8
// that plus 8; columns are rows of Q.  st: the stage; k_at, k_sc: this thread's pieces.
template <int D, int NT, typename F>
__device__ __forceinline__ void ca_scores(const uint8_t* st, uint32_t k_at, uint32_t k_sc, F frag, float (&s)[2][NT][4])
{
    constexpr int NS = D / 16;
    uint32_t kw[2][2][NS / 2], sc[2][2];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[mt][nt][j] = 0.f;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            // (8 keys are a whole number of the exchange's periods)
            const uint8_t* at_k = st + k_at + (16 * mt + 8 * e) * (D / 2);
            const uint8_t* at_s = st + k_sc + (16 * mt + 8 * e) * (D / 16);
            if (D == 128) {
                const uint4 x = *reinterpret_cast<const uint4*>(at_k);
                kw[mt][e][0] = x.x, kw[mt][e][1] = x.y, kw[mt][e][2 % (NS / 2)] = x.z;
                kw[mt][e][3 % (NS / 2)] = x.w;
                sc[mt][e] = *reinterpret_cast<const uint16_t*>(at_s);
            } else {
                const uint2 x = *reinterpret_cast<const uint2*>(at_k);
                kw[mt][e][0] = x.x, kw[mt][e][1] = x.y;
                sc[mt][e] = *at_s;
            }
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
                // the scale's f16 twice: code << 7 | code << 23
                const uint32_t f = (D == 128 && w >= NS / 4 ? sc[mt][e] >> 8 : sc[mt][e] & 0xff) * 0x800080u;
#pragma unroll
                for (int j = 0; j < 4; ++j) h[mt][e][j] = h2_mul(h[mt][e][j], f);
            }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint2 qf = frag(nt, 2 * w + half);
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    const uint32_t a[4] = {h[mt][0][2 * half], h[mt][1][2 * half], h[mt][0][2 * half + 1], h[mt][1][2 * half + 1]};
                    mma_f16(s[mt][nt], a, qf.x, qf.y);
                }
            }
    }
}

// A value that is not finite counts for the rows that see it alone: its product is left out,
// and the rows that see it are found by a product of their own.  scales: those of this
// thread's group of keys t, t + 4, t + 8, t + 12 of a tile, `step` bytes apart; room: how many
// of the keys from t on row g of a tile of rows sees.  Bits 0 and 1: whether rows 2t and
// 2t + 1 see a value that is not finite in this thread's group.
__device__ __forceinline__ uint32_t ca_seen_bad(const uint8_t* scales, int step, int room)
{
    uint32_t bad[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) bad[j] = scales[j * step] >= 0xf8 ? 0x3c00u : 0u;
    if (!__any_sync(0xffffffffu, (bad[0] | bad[1] | bad[2] | bad[3]) != 0)) return 0;
    const uint32_t a[4] = {bad[0] | bad[1] << 16, 0u, bad[2] | bad[3] << 16, 0u};
    float seen[4] = {0.f, 0.f, 0.f, 0.f};
    mma_f16(seen, a, (room > 0 ? 0x3c00u : 0u) | (room > 4 ? 0x3c000000u : 0u),
            (room > 8 ? 0x3c00u : 0u) | (room > 12 ? 0x3c000000u : 0u));
    return (seen[0] > 0.f ? 1u : 0u) | (seen[1] > 0.f ? 2u : 0u);
}

// Takes the scales that are not finite out of a warp's step.
__device__ __forceinline__ void ca_drop_bad(uint8_t* scales, int step)
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (scales[j * step] >= 0xf8) scales[j * step] = 0;
}

// What is subtracted from a row's logits q.k mul (powers of two) whose largest has q.k = top:
// kCaHead less than it, so that half of fp16's smallest number is 2^-35 of the row's largest weight
// and not 2^-25: one key often takes nearly all weight, and many others, or the V of others, the
// rest.  Rounded up, so no weight is above 2^kCaHead.
__device__ __forceinline__ float ca_base(float top, float mul) { return __fadd_ru(__fmul_ru(top, mul), -kCaHead); }

// The q.k above which that moves: no weight is above 2^(kCaHead + kCaSlack), whatever the
// quotient's error (a few units of the last place).
__device__ __forceinline__ float ca_limit(float base, float mul)
{
    const float x = __fdividef(__fadd_rd(base, kCaHead + kCaSlack), mul);
    return __fmaf_rd(fabsf(x), -0x1p-20f, x);
}

// (the sum is taken back to the maximum, near which its logarithm is exact to more places)
__device__ __forceinline__ float ca_lse(float base, float total)
{
    return (base + kCaHead + log2f(total * (1.f / (1 << static_cast<int>(kCaHead))))) * 0.693147181f;
}

template <int D>
__global__ void __launch_bounds__(CaShape<D, 1>::kThreads, 1) cache4_attn_kernel(CaParams p)
{
    using S = CaShape<D, 1>;
    constexpr int NS = S::kSteps;
    extern __shared__ __align__(128) uint8_t smem_all[];
    __shared__ uint32_t sh_line[32];
    const int group = threadIdx.x / kCaGroup, tid = threadIdx.x % kCaGroup;
    const int lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    uint8_t* const smem = smem_all + group * S::kGroupBytes;
    uint8_t* const my_ring = smem + warp * (S::kStages * S::kStage);
    uint2* const q_frag = reinterpret_cast<uint2*>(smem + S::kRing);
    uint8_t* const merge = smem + S::kRing + S::kQ;
    float2* const stats = reinterpret_cast<float2*>(merge + S::kMerge);  // [warp, all][row] (max, sum)
    int* const row_vis = reinterpret_cast<int*>(stats + (kCaWarps + 1) * S::kRows);
    float* const row_mul = reinterpret_cast<float*>(row_vis + S::kRows);
    // a thread's pieces: of K, keys (g >> 1) + 4 (g & 1) + 8 i; of V, keys t + 8 i and t + 4 + 8 i
    const int my_key = (g >> 1) + 4 * (g & 1);
    const uint32_t k_at = piece<D>(my_key, t * (D / 8)), k_sc = 2 * S::kCodes + my_key * (D / 16) + t * (D / 64);
    const uint32_t v_at[2] = {S::kCodes + piece<D>(t, g * (D / 16)), S::kCodes + piece<D>(t + 4, g * (D / 16))};
    const uint32_t v_sc = 2 * S::kCodes + S::kScales + t * (D / 16) + (D == 128 ? g : g >> 1);

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    CaCell c = ca_cell<S>(p, group, sh_line);
    if (!c.any) return;
    CaRun& run = c.run;
    CaCopies<D, S> copies(p, smem_u32(my_ring), warp, lane, c);
    uint32_t use = 0;  // stage
#pragma unroll 1
    for (int i = 0; i < S::kStages - 1; ++i) copies.issue();
#pragma unroll 1
    for (int unit = c.unit; c.base < c.x1; unit = 0) {
        // ---- a stretch of one run
        const int first = unit, last = ca_before<S>(run, c.base, c.x1), nrow = run.cnt * p.G;
        if (first < last) {
            ca_queries<D, S>(p, run, 0, nrow, group, tid, merge, q_frag, row_vis, row_mul);
            float mul[2], l[2], o[NS][4];
            float m[2], lim[2];  // what is subtracted (0 before there is a maximum) and q.k above which it moves
            int vis[2], vis_min = run.len;
            uint32_t poison = 0;  // bit j: row 2t + j sees a value that is not finite in this thread's group
            uint2 q1[NS];
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                q1[i] = q_frag[i * 32 + lane];
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                mul[j] = row_mul[2 * t + j], vis[j] = row_vis[2 * t + j];
                m[j] = 0.f, lim[j] = -INFINITY, l[j] = 0.f;
            }
            if (lane < nrow) vis_min = row_vis[lane];
            vis_min = __reduce_min_sync(0xffffffffu, vis_min);

#pragma unroll 1
            for (; unit < last; ++unit) {
                cp_async_wait<S::kStages - 2>();
                __syncwarp();
                copies.issue();
                uint8_t* const st = my_ring + use * S::kStage;
                use = use + 1 == S::kStages ? 0 : use + 1;
                const int key0 = unit * kCaUnit + warp * kCaKeys;
                if (key0 >= run.len) continue;
                float s[2][1][4];
                ca_scores<D, 1>(st, k_at, k_sc, [&](int, int i) { return q1[i]; }, s);
                // ---- what a row does not see; softmax
                const bool cut_here = key0 + kCaKeys > vis_min;
                const bool drafts = cut_here && vis_min < run.len;  // keys that some rows see and some do not
                if (cut_here) {
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (key0 + 16 * mt + my_key + 8 * (j >> 1) >= vis[j & 1]) s[mt][0][j] = -INFINITY;
                }
                float top[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) top[j] = fmaxf(max3f(s[0][0][j], s[0][0][j + 2], s[1][0][j]), s[1][0][j + 2]);
                if (__any_sync(0xffffffffu, top[0] > lim[0] || top[1] > lim[1])) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], d));
                        const bool none = lim[j] == -INFINITY;  // nothing seen so far: all sums are 0 (or NaN)
                        if (top[j] == -INFINITY) continue;
                        const float base = ca_base(top[j], mul[j]), now = none ? base : fmaxf(m[j], base);
                        const float keep = none ? 1.f : ex2_approx(m[j] - now);
                        l[j] *= keep;
#pragma unroll
                        for (int i = 0; i < NS; ++i) {
                            o[i][j] *= keep;
                            o[i][j + 2] *= keep;
                        }
                        m[j] = now;
                        lim[j] = ca_limit(now, mul[j]);
                    }
                }
                uint32_t pb[2][2];
                const uint64_t mu = f2_pack(-m[0], -m[1]), by = f2_pack(mul[0], mul[1]);
                uint64_t sum = f2_pack(l[0], l[1]);
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    float e[4];
#pragma unroll
                    for (int j = 0; j < 4; j += 2) {
                        f2_unpack(f2_fma(f2_pack(s[mt][0][j], s[mt][0][j + 1]), by, mu), e[j], e[j + 1]);
                        e[j] = ex2_approx(e[j]);
                        e[j + 1] = ex2_approx(e[j + 1]);
                        sum = f2_add(sum, f2_pack(e[j], e[j + 1]));
                    }
                    pb[mt][0] = transpose8(pack_f16(e[0], e[1]));
                    pb[mt][1] = transpose8(pack_f16(e[2], e[3]));
                }
                f2_unpack(sum, l[0], l[1]);
                if (__builtin_expect(drafts, 0)) {
#pragma unroll 1
                    for (int mt = 0; mt < 2; ++mt) {
                        const int room = row_vis[g] - key0 - 16 * mt - t;  // of keys t, t + 4 ...
                        poison |= ca_seen_bad(st + v_sc + 16 * mt * (D / 16), D / 4, room);
                    }
                    __syncwarp();
                    ca_drop_bad(st + v_sc, D / 4);
                    __syncwarp();
                }
                // ---- O^T: columns 2t, 2t + 1, 2t + 8, 2t + 9 of a tile are keys t, t + 4, t + 8, t + 12
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    uint32_t vw[4][NS / 4], code[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint8_t* at_v = st + v_at[j & 1] + (16 * mt + 8 * (j >> 1)) * (D / 2);
                        if (D == 128) {
                            const uint2 x = *reinterpret_cast<const uint2*>(at_v);
                            vw[j][0] = x.x, vw[j][1 % (NS / 4)] = x.y;
                        } else {
                            vw[j][0] = *reinterpret_cast<const uint32_t*>(at_v);
                        }
                        code[j] = st[v_sc + (16 * mt + 4 * j) * (D / 16)];
                    }
                    const uint32_t f[2] = {code[1] * 0x800000u + code[0] * 0x80u, code[3] * 0x800000u + code[2] * 0x80u};
#pragma unroll
                    for (int w = 0; w < NS / 4; ++w) {
                        uint32_t h[2][2][4];  // [keys 0 1 | 2 3][even | odd channel]
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t a = vw[2 * e][w], b = vw[2 * e + 1][w];
                            c4_decode((a & 0x0f0f0f0fu) | ((b * 16) & 0xf0f0f0f0u), h[e][0]);
                            c4_decode(((a >> 4) & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u), h[e][1]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                h[e][0][j] = h2_mul(h[e][0][j], f[e]);
                                h[e][1][j] = h2_mul(h[e][1][j], f[e]);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t a[4] = {h[0][0][i], h[0][1][i], h[1][0][i], h[1][1][i]};
                            mma_f16(o[4 * w + i], a, pb[mt][0], pb[mt][1]);
                        }
                    }
                }
            }

            // ---- the four warps' results of the stretch
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[j] += __shfl_xor_sync(0xffffffffu, l[j], d);
                if (lim[j] == -INFINITY) m[j] = -INFINITY;
                if (g == 0) stats[warp * S::kRows + 2 * t + j] = make_float2(m[j], l[j]);
            }
            group_sync(group);
            if (tid < nrow) {
                float top = -INFINITY, sum = 0.f;
#pragma unroll
                for (int w = 0; w < kCaWarps; ++w) top = fmaxf(top, stats[w * S::kRows + tid].x);
#pragma unroll
                for (int w = 0; w < kCaWarps; ++w) {
                    const float2 x = stats[w * S::kRows + tid];
                    sum += x.x == -INFINITY ? x.y : x.y * ex2_approx(x.x - top);
                }
                stats[kCaWarps * S::kRows + tid] = make_float2(top, sum);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = 2 * t + j;
                float top = -INFINITY;
#pragma unroll
                for (int w = 0; w < kCaWarps; ++w) top = fmaxf(top, stats[w * S::kRows + r].x);
                float keep = m[j] == -INFINITY ? 1.f : ex2_approx(m[j] - top);
                if (poison >> j & 1) keep = __uint_as_float(0x7fc00000u);
                if (r < nrow) {
                    float2* to = reinterpret_cast<float2*>(merge + (warp * S::kRows + r) * S::kRowBytes);
#pragma unroll
                    for (int i = 0; i < NS; ++i) to[i * 8 + g] = make_float2(o[i][j] * keep, o[i][j + 2] * keep);
                }
            }
            group_sync(group);
            const bool whole = first == 0 && last == run.units;
            float* part = p.parts + (2ll * c.cell + (first == 0)) * S::kPart;
#pragma unroll 1
            for (int x = tid; x < nrow * (D / 2); x += kCaGroup) {
                const int r = x / (D / 2), y = x % (D / 2);  // channels 2y, 2y + 1
                float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kCaWarps; ++w) {
                    const float2 v = reinterpret_cast<const float2*>(merge + (w * S::kRows + r) * S::kRowBytes)[y % NS * 8 + y / NS];
                    sum.x += v.x, sum.y += v.y;
                }
                const float2 all = stats[kCaWarps * S::kRows + r];
                if (!whole) {
                    reinterpret_cast<float2*>(part)[x] = sum;
                    if (y == 0) reinterpret_cast<float2*>(part + S::kRows * D)[r] = all;
                    continue;
                }
                const int token = p.token_of(r), hq = run.h * p.G + r - token * p.G, pr = run.r0 + token;
                const bool any = all.y != 0.f;  // (a NaN is not)
                const float inv = 1.f / all.y;
                reinterpret_cast<uint32_t*>(p.o + (static_cast<int64_t>(pr) * p.Hq + hq) * D)[y] =
                    any ? cvt_bf16x2(sum.x * inv, sum.y * inv) : 0u;
                if (y == 0 && p.lse) p.lse[static_cast<int64_t>(hq) * p.B * p.n + pr] = any ? ca_lse(all.x, all.y) : -INFINITY;
            }
            if (last < run.units && first == 0 && tid == 0) ca_open<S>(p, c, p.table[c.cell], c.cell);
        }
        c.base += run.units + S::kRunCost;
        if (c.base < c.x1) ca_next(p, S::kRows, run);
    }
    cp_async_wait<0>();
}

// The same for more rows, whose sums over all channels a warp cannot hold: a warp has all
// rows' sums over half of the group's keys (of V), of half of the channels.  So V's codes are
// still turned into operands once.  P goes through shared memory, and the running maxima are
// the group's.
template <int D, int NT>
__global__ void __launch_bounds__(CaShape<D, NT>::kThreads, 1) cache4_wide_kernel(CaParams p)
{
    using S = CaShape<D, NT>;
    constexpr int NS = S::kSteps, MT = D / 32;  // m tiles of a warp's channels
    extern __shared__ __align__(128) uint8_t smem_all[];
    __shared__ uint32_t sh_line[32];
    const int group = threadIdx.x / kCaGroup, tid = threadIdx.x % kCaGroup;
    const int lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    uint8_t* const smem = smem_all + group * S::kGroupBytes;
    uint8_t* const my_ring = smem + warp * (S::kStages * S::kStage);
    uint2* const q_frag = reinterpret_cast<uint2*>(smem + S::kRing);
    uint2* const p_both = reinterpret_cast<uint2*>(smem + S::kRing + S::kQ);  // of two units, [16 keys][tile of rows][lane]
    uint2* p_frag = p_both;
    float* const wtop = reinterpret_cast<float*>(smem + S::kRing + S::kQ + S::kMerge);  // [warp][row]: maxima, then sums
    int* const row_vis = reinterpret_cast<int*>(wtop + kCaWarps * S::kRows);
    float* const row_mul = reinterpret_cast<float*>(row_vis + S::kRows);
    float* const row_m = row_mul + S::kRows;    // what is subtracted (0 before there is a maximum)
    float* const row_lim = row_m + S::kRows;    // q.k above which it moves
    const int my_key = (g >> 1) + 4 * (g & 1);
    const uint32_t k_at = piece<D>(my_key, t * (D / 8)), k_sc = 2 * S::kCodes + my_key * (D / 16) + t * (D / 64);
    // of V: D / 16 channels, from half * D / 2 + g * D / 16, of keys t + 8 i and t + 4 + 8 i
    const int half = warp & 1, keys = warp >> 1;
    const uint32_t at = half * (D / 4) + g * (D / 32);
    const uint32_t v_at[2] = {S::kCodes + piece<D>(t, at), S::kCodes + piece<D>(t + 4, at)};
    const uint32_t v_sc = 2 * S::kCodes + S::kScales + t * (D / 16) + half * (D / 32) + (D == 128 ? g >> 1 : g >> 2);

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    CaCell c = ca_cell<S>(p, group, sh_line);
    if (!c.any) return;
    CaRun& run = c.run;
    CaCopies<D, S> copies(p, smem_u32(my_ring), warp, lane, c);
    uint32_t use = 0;  // stage
#pragma unroll 1
    for (int i = 0; i < S::kStages - 1; ++i) copies.issue();
#pragma unroll 1
    for (int unit = c.unit; c.base < c.x1; unit = 0) {
        // ---- a stretch of one run
        const int first = unit, last = ca_before<S>(run, c.base, c.x1);
        const int row0 = run.rb * S::kRows, nrow = min(S::kRows, run.cnt * p.G - row0);
        if (first < last) {
            ca_queries<D, S>(p, run, row0, nrow, group, tid, reinterpret_cast<uint8_t*>(p_both), q_frag, row_vis, row_mul);
            float l[NT][2], o[NT][MT][4];
            uint32_t poison = 0;  // bit 2 nt + j: row 8 nt + 2t + j sees a value that is not finite in this thread's channels
            if (tid < S::kRows) row_m[tid] = 0.f, row_lim[tid] = -INFINITY;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[nt][i][j] = 0.f;
            }
            int vis_min = lane < nrow ? row_vis[lane] : run.len;
            vis_min = __reduce_min_sync(0xffffffffu, vis_min);
            group_sync(group);

#pragma unroll 1
            for (; unit < last; ++unit) {
                cp_async_wait<S::kStages - 2>();
                __syncwarp();
                const uint32_t stage = use * S::kStage;
                use = use + 1 == S::kStages ? 0 : use + 1;
                p_frag = p_both + (unit & 1) * (S::kMerge / 16);  // (of the unit before some warps may still read theirs)
                const int key0 = unit * kCaUnit + warp * kCaKeys;
                const bool mine = key0 < run.len;
                const bool cut_here = unit * kCaUnit + kCaUnit > vis_min;  // (of any of the group's warps)
                float s[2][NT][4];
                bool moves = false;
                if (mine) {
                    ca_scores<D, NT>(my_ring + stage, k_at, k_sc, [&](int nt, int i) { return q_frag[(nt * NS + i) * 32 + lane]; }, s);
                    if (cut_here) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const int2 vis = reinterpret_cast<const int2*>(row_vis)[nt * 4 + t];
#pragma unroll
                            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    if (key0 + 16 * mt + my_key + 8 * (j >> 1) >= (j & 1 ? vis.y : vis.x)) s[mt][nt][j] = -INFINITY;
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const float2 lim = reinterpret_cast<const float2*>(row_lim)[nt * 4 + t];
                        moves |= fmaxf(max3f(s[0][nt][0], s[0][nt][2], s[1][nt][0]), s[1][nt][2]) > lim.x;
                        moves |= fmaxf(max3f(s[0][nt][1], s[0][nt][3], s[1][nt][1]), s[1][nt][3]) > lim.y;
                    }
                }
                // P by the maxima so far, and its sums
                float more[NT][2];
                const auto weights = [&] {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const float2 mm = reinterpret_cast<const float2*>(row_m)[nt * 4 + t];
                        const float2 mul = reinterpret_cast<const float2*>(row_mul)[nt * 4 + t];
                        const uint64_t mu = f2_pack(-mm.x, -mm.y), by = f2_pack(mul.x, mul.y);
                        uint64_t sum = f2_pack(0.f, 0.f);
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt) {
                            float e[4];
#pragma unroll
                            for (int j = 0; j < 4; j += 2) {
                                f2_unpack(f2_fma(f2_pack(s[mt][nt][j], s[mt][nt][j + 1]), by, mu), e[j], e[j + 1]);
                                e[j] = ex2_approx(e[j]);
                                e[j + 1] = ex2_approx(e[j + 1]);
                                sum = f2_add(sum, f2_pack(e[j], e[j + 1]));
                            }
                            p_frag[((warp * 2 + mt) * NT + nt) * 32 + lane] =
                                make_uint2(transpose8(pack_f16(e[0], e[1])), transpose8(pack_f16(e[2], e[3])));
                        }
                        f2_unpack(sum, more[nt][0], more[nt][1]);
                    }
                };
                if (mine) weights();
                // (past this all copies of the unit are there, and all have P and are done with the unit before)
                if (group_any(group, moves)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float top = -INFINITY;
                            if (mine) top = fmaxf(max3f(s[0][nt][j], s[0][nt][j + 2], s[1][nt][j]), s[1][nt][j + 2]);
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                            if (g == 0) wtop[warp * S::kRows + nt * 8 + 2 * t + j] = top;
                        }
                    group_sync(group);
                    float now[NT][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int r = nt * 8 + 2 * t + j;
                            float top = wtop[r];
#pragma unroll
                            for (int w = 1; w < kCaWarps; ++w) top = fmaxf(top, wtop[w * S::kRows + r]);
                            const float was = row_m[r];
                            const bool none = row_lim[r] == -INFINITY;  // nothing seen so far: all sums are 0 (or NaN)
                            const float base = ca_base(top, row_mul[r]);
                            now[nt][j] = top == -INFINITY ? was : none ? base : fmaxf(was, base);
                            const float keep = none ? 1.f : ex2_approx(was - now[nt][j]);
                            l[nt][j] *= keep;
#pragma unroll
                            for (int i = 0; i < MT; ++i) {
                                o[nt][i][j] *= keep;
                                o[nt][i][j + 2] *= keep;
                            }
                            if (none && top == -INFINITY) now[nt][j] = -INFINITY;
                        }
                    group_sync(group);
                    if (warp == 0 && g == 0) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                const int r = nt * 8 + 2 * t + j;
                                if (now[nt][j] == -INFINITY) continue;
                                row_m[r] = now[nt][j];
                                row_lim[r] = ca_limit(now[nt][j], row_mul[r]);
                            }
                    }
                    group_sync(group);
                    if (mine) weights();
                    group_sync(group);
                }
                if (mine) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) l[nt][0] += more[nt][0], l[nt][1] += more[nt][1];
                }
                copies.issue();  // into the stage that the unit before has left
                // ---- O^T: columns 2t, 2t + 1, 2t + 8, 2t + 9 of a tile are keys t, t + 4, t + 8, t + 12
                const bool drafts = cut_here && vis_min < run.len;  // keys that some rows see and some do not
#pragma unroll 1
                for (int w = 2 * keys; w < 2 * keys + 2 && unit * kCaUnit + w * kCaKeys < run.len; ++w) {
                    uint8_t* const st = smem + w * (S::kStages * S::kStage) + stage;
                    if (__builtin_expect(drafts, 0)) {
#pragma unroll 1
                        for (int mt = 0; mt < 2; ++mt)
#pragma unroll 1
                            for (int nt = 0; nt < NT; ++nt) {
                                const int room = row_vis[nt * 8 + g] - unit * kCaUnit - w * kCaKeys - 16 * mt - t;  // of keys t, t + 4 ...
                                poison |= ca_seen_bad(st + v_sc + 16 * mt * (D / 16), D / 4, room) << (2 * nt);
                            }
                        __syncwarp();
                        ca_drop_bad(st + v_sc, D / 4);
                        __syncwarp();
                    }
                    const uint2* const pf = p_frag + w * 2 * NT * 32 + lane;
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        uint32_t vw[4], code[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint8_t* at_v = st + v_at[j & 1] + (16 * mt + 8 * (j >> 1)) * (D / 2);
                            vw[j] = D == 128 ? *reinterpret_cast<const uint32_t*>(at_v) : *reinterpret_cast<const uint16_t*>(at_v);
                            code[j] = st[v_sc + (16 * mt + 4 * j) * (D / 16)];
                        }
                        const uint32_t f[2] = {code[1] * 0x800000u + code[0] * 0x80u, code[3] * 0x800000u + code[2] * 0x80u};
                        // even channels of two keys, odd ones of two keys (D = 64: of four, two words in one)
                        uint32_t ev[2 * MT], od[2 * MT];
#pragma unroll
                        for (int e = 0; e < MT / 2; ++e) {
                            const uint32_t a = MT == 4 ? vw[2 * e] : vw[0] + vw[2] * 0x10000u, b = MT == 4 ? vw[2 * e + 1] : vw[1] + vw[3] * 0x10000u;
                            uint32_t x[4], y[4];
                            c4_decode((a & 0x0f0f0f0fu) | ((b * 16) & 0xf0f0f0f0u), x);
                            c4_decode(((a >> 4) & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u), y);
#pragma unroll
                            for (int j = 0; j < 4; ++j) ev[4 * e + j] = x[j], od[4 * e + j] = y[j];
                        }
                        uint32_t ha[MT][4];
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            ha[i][0] = h2_mul(ev[i], f[0]), ha[i][1] = h2_mul(od[i], f[0]);
                            ha[i][2] = h2_mul(ev[MT + i], f[1]), ha[i][3] = h2_mul(od[MT + i], f[1]);
                        }
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint2 pp = pf[(mt * NT + nt) * 32];
#pragma unroll
                            for (int i = 0; i < MT; ++i) mma_f16(o[nt][i], ha[i], pp.x, pp.y);
                        }
                    }
                }
            }

            // ---- the stretch's results: sums over the warps' keys, then a thread's channels of its rows
            group_sync(group);
            float* const other = reinterpret_cast<float*>(q_frag);  // [row][channel]: the other half's (Q and P are done with)
            const int ch = half * (D / 2) + g * (D / 16);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int r = nt * 8 + 2 * t + j;
                    const float keep = poison >> (2 * nt + j) & 1 ? __uint_as_float(0x7fc00000u) : 1.f;
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) l[nt][j] += __shfl_xor_sync(0xffffffffu, l[nt][j], d);
                    if (g == 0) wtop[warp * S::kRows + r] = l[nt][j];
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        o[nt][i][j] *= keep, o[nt][i][j + 2] *= keep;
                        if (keys == 1) *reinterpret_cast<float2*>(other + r * D + ch + 2 * i) = make_float2(o[nt][i][j], o[nt][i][j + 2]);
                    }
                }
            group_sync(group);
            const bool whole = first == 0 && last == run.units;
            float* part = p.parts + (2ll * c.cell + (first == 0)) * S::kPart;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int r = nt * 8 + 2 * t + j;
                    if (keys == 1 || r >= nrow) continue;
                    const float total = wtop[r] + wtop[S::kRows + r] + wtop[2 * S::kRows + r] + wtop[3 * S::kRows + r];
                    const float top = row_lim[r] == -INFINITY ? -INFINITY : row_m[r];
                    const bool any = total != 0.f;  // (a NaN is not)
                    const float scale = whole ? 1.f / total : 1.f;
                    float2 x[MT];
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        const float2 y = *reinterpret_cast<const float2*>(other + r * D + ch + 2 * i);
                        x[i] = make_float2((o[nt][i][j] + y.x) * scale, (o[nt][i][j + 2] + y.y) * scale);
                    }
                    const bool one = half == 0 && g == 0;  // of a row's threads
                    if (!whole) {
#pragma unroll
                        for (int i = 0; i < MT; ++i) reinterpret_cast<float2*>(part + r * D + ch)[i] = x[i];
                        if (one) reinterpret_cast<float2*>(part + S::kRows * D)[r] = make_float2(top, total);
                        continue;
                    }
                    const int token = p.token_of(row0 + r), hq = run.h * p.G + row0 + r - token * p.G, pr = run.r0 + token;
                    uint32_t* out = reinterpret_cast<uint32_t*>(p.o + (static_cast<int64_t>(pr) * p.Hq + hq) * D + ch);
#pragma unroll
                    for (int i = 0; i < MT; ++i) out[i] = any ? cvt_bf16x2(x[i].x, x[i].y) : 0u;
                    if (one && p.lse) p.lse[static_cast<int64_t>(hq) * p.B * p.n + pr] = any ? ca_lse(top, total) : -INFINITY;
                }
            if (last < run.units && first == 0 && tid == 0) ca_open<S>(p, c, p.table[c.cell], c.cell);
        }
        c.base += run.units + S::kRunCost;
        if (c.base < c.x1) ca_next(p, S::kRows, run);
    }
    cp_async_wait<0>();
}

// Joins up to 8 rows' parts, of the n cells from `first` on: each row by as many warps as
// there are for it, which share the parts.
template <int D, int NT>
__device__ __forceinline__ void join_rows(const CaParams& p, const CaOpen& e, int first, int n, int r0, int rows,
                                          float (&sh)[kJoinThreads / 32][D + 1])
{
    using S = CaShape<D, NT>;
    constexpr int C = D / 32, W = kJoinThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ways = rows > 4 ? W / 8 : rows > 2 ? W / 4 : rows > 1 ? W / 2 : W;  // warps a row
    const int row = warp / ways, way = warp % ways, r = r0 + row;
    const auto part = [&](int i) { return p.parts + (2ll * (first + i) + (i == 0)) * S::kPart; };
    float top = -INFINITY, total = 0.f, sum[C];
#pragma unroll
    for (int c = 0; c < C; ++c) sum[c] = 0.f;
    if (row < rows) {
        for (int i = lane; i < n; i += 32) top = fmaxf(top, part(i)[S::kRows * D + 2 * r]);
        constexpr int AT = 4;  // parts in flight
#pragma unroll 1
        for (int i0 = way; i0 < n; i0 += AT * ways) {
            float2 st[AT];
            float v[AT][C];
#pragma unroll
            for (int k = 0; k < AT; ++k) {
                const int i = i0 + k * ways;
                st[k] = make_float2(-INFINITY, 0.f);
#pragma unroll
                for (int c = 0; c < C; ++c) v[k][c] = 0.f;
                if (i < n) {
                    st[k] = reinterpret_cast<const float2*>(part(i) + S::kRows * D)[r];
                    const float2* x = reinterpret_cast<const float2*>(part(i) + r * D) + lane * (C / 2);
#pragma unroll
                    for (int c = 0; c < C; c += 2) v[k][c] = x[c / 2].x, v[k][c + 1] = x[c / 2].y;
                }
            }
            if (i0 == way)
#pragma unroll
                for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
#pragma unroll
            for (int k = 0; k < AT; ++k) {
                const float keep = st[k].x == -INFINITY ? 1.f : ex2_approx(st[k].x - top);
                total += st[k].y * keep;
#pragma unroll
                for (int c = 0; c < C; ++c) sum[c] += v[k][c] * keep;
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) sh[warp][lane * C + c] = sum[c];
        if (lane == 0) sh[warp][D] = total;
    }
    __syncthreads();
    if (row >= rows || way > 0) return;
    for (int w = 1; w < min(ways, n); ++w) {
        total += sh[warp + w][D];
#pragma unroll
        for (int c = 0; c < C; ++c) sum[c] += sh[warp + w][lane * C + c];
    }
    const int token = p.token_of(e.row0 + r), hq = e.h * p.G + e.row0 + r - token * p.G, pr = e.r0 + token;
    const bool any = total != 0.f;
    const float inv = 1.f / total;
    uint32_t* out = reinterpret_cast<uint32_t*>(p.o + (static_cast<int64_t>(pr) * p.Hq + hq) * D + lane * C);
#pragma unroll
    for (int c = 0; c < C; c += 2) out[c / 2] = any ? cvt_bf16x2(sum[c] * inv, sum[c + 1] * inv) : 0u;
    if (lane == 0 && p.lse) p.lse[static_cast<int64_t>(hq) * p.B * p.n + pr] = any ? ca_lse(top, total) : -INFINITY;
}

// Joins the parts of runs, a CTA a cell.  The cells that have a part of a run share its
// rows: those that it comes into as well as the one that begins it (16 x 4 drafts, H 16/1, 64
// rows a KV head: 31.8 -> 29.3 us; with up to 8 rows the one that begins it has them all: 32 x 1
// 41.8 us, 43.8 when shared).
template <int D, int NT>
__global__ void __launch_bounds__(kJoinThreads) cache4_join_kernel(CaParams p)
{
    using S = CaShape<D, NT>;
    constexpr int W = kJoinThreads / 32;
    __shared__ float sh[W][D + 1];
    const int cell = blockIdx.x;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    CaOpen e = p.table[cell];
    if constexpr (!S::kWide) {
        if (e.last >= 0) join_rows<D, NT>(p, e, cell, e.last - cell + 1, 0, e.nrow, sh);
    } else {
        const CaOpen next = p.table[gridDim.x + cell];
#pragma unroll 1
        for (int k = 0; k < 2; ++k, e = next) {
            if (e.last < 0) continue;
            const int n = e.last - e.first + 1, share = (e.nrow + n - 1) / n, end = min(e.nrow, (cell - e.first + 1) * share);
#pragma unroll 1
            for (int r0 = (cell - e.first) * share; r0 < end; r0 += W) {
                join_rows<D, NT>(p, e, e.first, n, r0, min(W, end - r0), sh);
                __syncthreads();  // (sh is read)
            }
        }
    }
}

int check_cache4_attn(const logo_dims& d, int n_new)
{
    if (n_new < 1) return LOGO_ERR_INVALID_ARG;
    const int rc = check_dims(d);
    if (rc != LOGO_OK) return rc;
    if (static_cast<int64_t>(d.B) * n_new > (1 << 24) || d.Hkv > (1 << 16) ||
        static_cast<int64_t>(n_new) * (d.Hq / d.Hkv) > 8192 || static_cast<int64_t>(d.B) * n_new * d.Hq > (1 << 30))
        return LOGO_ERR_UNSUPPORTED;
    // the line's units are counted in 31 bits
    const int64_t units = (static_cast<int64_t>(d.T) + kCaUnit - 1) / kCaUnit + 4;  // (and a run's cost)
    const int64_t blocks = (static_cast<int64_t>(n_new) * (d.Hq / d.Hkv) + 8 * kCaMaxTiles - 1) / (8 * kCaMaxTiles);
    if (units * d.B * d.Hkv > (1ll << 31) / blocks - 1) return LOGO_ERR_UNSUPPORTED;
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
int ca_cells(CaShape<D, NT>)
{
    return device_sm_count() * CaShape<D, NT>::kGroups;
}

template <int D, int NT>
int ca_launch(CaShape<D, NT> s, CaParams& p, cudaStream_t st)
{
    using S = CaShape<D, NT>;
    void (*kernel)(CaParams);
    if constexpr (NT == 1) kernel = cache4_attn_kernel<D>;
    else kernel = cache4_wide_kernel<D, NT>;
    static OncePerDevice once;
    if (once([&] { return set_smem_limit(kernel, S::kSmem); }) != cudaSuccess) return LOGO_ERR_CUDA;
    // each launch is set up while the one before it on the stream runs (and waits for its end itself)
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(device_sm_count());
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) return LOGO_ERR_CUDA;
    cfg.gridDim = dim3(ca_cells(s));
    cfg.blockDim = dim3(kJoinThreads);
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, cache4_join_kernel<D, NT>, p) == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
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
        const size_t cells = ca_cells(s);
        bytes = round_up(2 * cells * sizeof(CaOpen), 256) + 2 * cells * S::kPart * sizeof(float);
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
    // (packed rows are written while queries of other tokens are still to be read)
    const size_t bytes = static_cast<size_t>(dims.B) * n_new * dims.Hq * dims.D * sizeof(logo_bf16);
    if (overlap(q, bytes, o_c, bytes)) return LOGO_ERR_INVALID_ARG;
    CaParams p{};
    p.q = q, p.k = cache.k, p.v = cache.v, p.ks = cache.k_scale, p.vs = cache.v_scale;
    p.len = seq_len, p.pos = pos, p.cu_q = cu_q, p.n_sel = n_sel_total, p.o = o_c, p.lse = lse_c;
    p.B = dims.B, p.n = n_new, p.Hq = dims.Hq, p.Hkv = dims.Hkv, p.G = dims.Hq / dims.Hkv, p.L = dims.T;
    p.magic = p.G > 1 ? 0xffffffffu / p.G + 1 : 0;
    p.scale2 = (scale > 0.f ? scale : 1.f / sqrtf(static_cast<float>(dims.D))) * 1.44269504f;
    return ca_dispatch(dims.D, ca_tiles(dims, n_new), [&](auto s) {
        p.table = static_cast<CaOpen*>(workspace);
        p.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + round_up(2 * ca_cells(s) * sizeof(CaOpen), 256));
        return ca_launch(s, p, static_cast<cudaStream_t>(stream));
    });
}
