// target_probs.cu -- logits to the target's probabilities: penalties for repeated
// tokens, biases, a grammar's mask, temperature, softmax:
// p_v = 2^((x_v - max x) log2(e) / T) / sum.
//
// HBM bounds it: 2 or 4 bytes read, 1/8 of one for the mask and 4 written per token.  Two
// streaming passes, a warp 1024 tokens, the second of which finds most logits in L2 (it goes
// through the rows backwards): the first leaves a maximum and a sum of exponentials a warp,
// the second joins a row's and writes.  (One pass that kept a row in the registers of a
// thread-block cluster between its read and its write took 122 us for 240 rows of 131072:
// clusters follow one another, wait for their slowest CTA and do the lists' work eight
// times.)  At the HBM rate an SM has little more than an instruction a token to spend, so
// both passes are laid out to save them: a warp's logits come to shared memory by
// asynchronous copies, and a thread of the first pass takes 32 in a row, whose masks are a
// word (eight at a time, with a byte of the masks: 94 us for 70).  Small CTAs end one by one,
// so an SM always has copies under way (a warp for several stretches, with a ring: 76 us).
// Short rows are one CTA's, which does both passes.
// The lists of tokens (history, drafts, biases) are counted ahead of that, a CTA a row, 11 us
// of the 70.  The first pass leaves listed tokens out of its stretches and then takes its
// part of the list, a thread a token, with their logits from shared memory; the second writes
// their probabilities over the zeros that it left.  (Adjusted where they are counted, from
// HBM, and left in p until the second pass: 94 us.)  Sums do not depend on the order of
// atomics.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "host_common.h"
#include "sm100.cuh"

namespace logo {
namespace {

constexpr int kTpThreads = 64, kTpWarps = kTpThreads / 32;
constexpr int kTpChunk = 1024;                             // tokens of a warp at a time
constexpr int kTpWords = 36;                               // room for the 33 words of a bit a token that they are in
constexpr int kTpRowWarps = 16;                            // chunks of a row up to which one CTA has them all
constexpr int kTpListThreads = 512;
constexpr int kTpAt = 4;                                   // list entries in flight per thread
constexpr int kTpMaxBiases = 4096;
constexpr int kTpNear = 8192;                              // listed tokens that are counted in shared memory
// a listed token's word: how often it was generated, its place among the biases (plus one), flags
constexpr uint32_t kTpSeen = 1u << 31, kTpBiased = 1u << 30, kTpTwice = 1u << 29, kTpCount = (1u << 15) - 1;
constexpr int kTpBiasAt = 15, kTpTake = 4;                 // listed tokens of a thread at a time
static_assert(LOGO_PROBS_MAX_COUNTED + 1024 <= kTpCount, "counts have room");

struct TpParams {
    const void* logits;
    const float *temperature, *penalty;
    const int32_t *history, *hist_len, *n_prompt, *draft, *bias_tok;
    const float* bias_val;
    const uint32_t* allowed;
    float* p;
    int B, m1, V, H, K;
    int chunks;         // of a row
    int words;          // of a bit a token: ceil(V / 32)
    int64_t listed;     // room for listed tokens a row (0: no lists)
    float2* stats;      // [rows][chunks] (maximum, sum)
    uint32_t* marks;    // [rows][words]: a bit a listed token
    uint32_t* bits;     // [rows * chunks][kTpChunk / 32]: a bit a token that counts in the passes
    uint2* part;        // [rows * chunks]: of the row's list the first that is in the chunk, and how many are
    uint2* list;        // [rows][listed]: listed tokens, ascending, with their words
    float* adjusted;    // [rows][listed]: their biases, then their adjusted logits
};

__device__ __forceinline__ float ex2(float x) { return ex2_approx(x); }

// A float's bits in an order that compares as unsigned numbers do (no NaN).
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);  // -0 as +0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

// Each launch is set up while the one before it on the stream runs, and waits here for its end.
__device__ __forceinline__ void wait_for_stream()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Which of eight tokens from v on are the vocabulary's.
__device__ __forceinline__ uint32_t inside(int V, int v)
{
    uint32_t ok = 0xffu;
    if (v < 0) ok = 0xffu << -v & 0xffu;
    if (v + 8 > V) ok &= v < V ? 0xffu >> (v + 8 - V) : 0;
    return ok;
}

// log2(e) / T, NaN for a T that is none.
__device__ __forceinline__ float steepness(float T) { return T > 0.f ? fminf(fmaxf(1.44269504f / T, 1.0e-30f), 3.0e38f) : NAN; }

// (largest x, sum of exponentials) of two parts; greedy (T = 0): the lowest token that has the
// largest x in the sum's place, or NaN where an x is.
__device__ __forceinline__ float2 join(float2 p, float2 q, float T, float c)
{
    const float top = fmaxf(p.x, q.x);
    if (T == 0.f) {
        if (p.y != p.y || q.y != q.y) return make_float2(top, NAN);
        if (p.x != q.x) return p.x > q.x ? p : q;
        return make_float2(top, __int_as_float(min(__float_as_int(p.y), __float_as_int(q.y))));
    }
    // (a part without a number: its sum is 0, or NaN)
    const float fp = p.x == -INFINITY ? 1.f : ex2((p.x - top) * c), fq = q.x == -INFINITY ? 1.f : ex2((q.x - top) * c);
    return make_float2(top, p.y * fp + q.y * fq);
}

// Over a warp, in every lane.
__device__ __forceinline__ float2 join_warp(float2 p, float T, float c)
{
    const float top = unordered(__reduce_max_sync(0xffffffffu, ordered(p.x)));
    if (T == 0.f) {
        const int token = __reduce_min_sync(0xffffffffu, p.y == p.y && p.x == top ? __float_as_int(p.y) : 0x7fffffff);
        return make_float2(top, __any_sync(0xffffffffu, p.y != p.y) ? NAN : __int_as_float(token));
    }
    float sum = p.x == -INFINITY ? p.y : p.y * ex2((p.x - top) * c);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    return make_float2(top, sum);
}

__device__ __forceinline__ float2 nothing(float T, int V) { return make_float2(-INFINITY, T == 0.f ? __int_as_float(V) : 0.f); }

// f(token, index) for the entries of a list that are tokens, kTpAt loads in flight.
template <typename F>
__device__ __forceinline__ void each_token(const int32_t* list, int len, int V, F f)
{
#pragma unroll 1
    for (int k0 = threadIdx.x; k0 < len; k0 += kTpAt * kTpListThreads) {
        uint32_t t[kTpAt];
#pragma unroll
        for (int k = 0; k < kTpAt; ++k) t[k] = k0 + k * kTpListThreads < len ? list[k0 + k * kTpListThreads] : 0xffffffffu;
#pragma unroll
        for (int k = 0; k < kTpAt; ++k)
            if (t[k] < static_cast<uint32_t>(V)) f(t[k], k0 + k * kTpListThreads);
    }
}

// A chunk of a row.  Chunks begin at multiples of eight of the whole tensor's elements, so
// that groups of eight tokens are aligned, and all but a row's first and last are whole.
struct TpPlace {
    int64_t item;  // among all rows' chunks
    int64_t g;     // its first group, of the tensor
    int v;         // its first token, of the row; less than 0 in a row's first chunk, if that begins in the row before

    __device__ __forceinline__ TpPlace(const TpParams& a, int row, int chunk)
    {
        const int64_t e0 = static_cast<int64_t>(row) * a.V;
        item = static_cast<int64_t>(row) * a.chunks + chunk;
        g = e0 / 8 + chunk * (kTpChunk / 8);
        v = chunk * kTpChunk - static_cast<int>(e0 & 7);
    }
    __device__ __forceinline__ bool whole(const TpParams& a) const { return v >= 0 && v + kTpChunk <= a.V; }
};

// Are the eight tokens from v on all the row's?
__device__ __forceinline__ bool whole8(const TpParams& a, int v) { return static_cast<uint32_t>(v) < static_cast<uint32_t>(max(a.V - 7, 0)); }

// Bits of eight tokens from a row of a bit a token.
__device__ __forceinline__ uint32_t bits_of(const uint32_t* row, int words, int v)
{
    const int w = max(v, 0) / 32;
    const uint32_t lo = row[w], hi = row[w + (w + 1 < words)];
    return (v < 0 ? lo << -v : __funnelshift_r(lo, hi, v & 31)) & 0xffu;
}

// A row's lists: the listed tokens in their order, with a word each, and what the passes take.
__global__ void __launch_bounds__(kTpListThreads) target_lists_kernel(TpParams a)
{
    extern __shared__ __align__(16) uint32_t smem[];
    __shared__ uint32_t sh_sum[kTpListThreads / 32];
    const int row = blockIdx.x, b = row / a.m1, i = row - b * a.m1, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int room = (a.words + 3) / 4 * 4;
    uint32_t *const bits = smem, *const before = smem + room;
    int32_t* const bias_tok = reinterpret_cast<int32_t*>(smem + 2 * room);
    float* const bias_val = reinterpret_cast<float*>(bias_tok) + a.K;
    for (int w = tid; w < room; w += kTpListThreads) bits[w] = 0;
    wait_for_stream();
    const int old = a.history ? max(0, min(a.hist_len[b], a.H)) : 0;
    const int prompt = max(a.n_prompt ? a.n_prompt[b] : 0, old - LOGO_PROBS_MAX_COUNTED);
    const int32_t* hist = a.history + static_cast<int64_t>(b) * a.H;
    const int32_t* draft = a.draft + static_cast<int64_t>(b) * (a.m1 - 1);
    const int n_draft = a.draft ? i : 0;
    for (int k = tid; k < a.K; k += kTpListThreads) {
        bias_tok[k] = a.bias_tok[static_cast<int64_t>(b) * a.K + k];
        bias_val[k] = a.bias_val[static_cast<int64_t>(b) * a.K + k];
    }
    __syncthreads();
    const auto mark = [&](uint32_t t, int) { atomicOr(bits + t / 32, 1u << (t & 31)); };
    each_token(hist, old, a.V, mark);
    each_token(draft, n_draft, a.V, mark);
    each_token(bias_tok, a.K, a.V, mark);
    __syncthreads();
    // listed tokens before each word's: a warp a stretch of words, a lane four at a time
    constexpr int W = kTpListThreads / 32;
    const int per = (a.words + W * 128 - 1) / (W * 128) * 128, w0 = warp * per;
    uint32_t mine = 0;
    for (int w = w0 + 4 * lane; w < min(w0 + per, room); w += 128) {
        const uint4 y = *reinterpret_cast<const uint4*>(bits + w);
        mine += __popc(y.x) + __popc(y.y) + __popc(y.z) + __popc(y.w);
    }
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0) sh_sum[warp] = mine;
    __syncthreads();
    uint32_t at = 0, n = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        if (w < warp) at += sh_sum[w];
        n += sh_sum[w];
    }
    for (int w = w0; w < min(w0 + per, room); w += 128) {
        const bool in = w + 4 * lane < room;
        const uint4 y = in ? *reinterpret_cast<const uint4*>(bits + w + 4 * lane) : make_uint4(0, 0, 0, 0);
        const uint32_t here = __popc(y.x) + __popc(y.y) + __popc(y.z) + __popc(y.w);
        uint32_t upto = here;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t z = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += z;
        }
        const uint32_t b0 = at + upto - here, b1 = b0 + __popc(y.x), b2 = b1 + __popc(y.y);
        if (in) *reinterpret_cast<uint4*>(before + w + 4 * lane) = make_uint4(b0, b1, b2, b2 + __popc(y.z));
        at += __shfl_sync(0xffffffffu, upto, 31);
    }
    // put together in shared memory where there is room, else in the workspace
    const bool near = a.listed <= kTpNear;
    uint2* const far_list = a.list + row * a.listed;
    uint2* const list = near ? reinterpret_cast<uint2*>(bias_val + a.K) : far_list;
    for (uint32_t k = tid; k < n; k += kTpListThreads) list[k] = make_uint2(0, 0);
    __syncthreads();
    for (int w = tid; w < a.words; w += kTpListThreads) a.marks[static_cast<int64_t>(row) * a.words + w] = bits[w];
    const auto ahead = [&](uint32_t t) { return before[t / 32] + __popc(bits[t / 32] & ((1u << (t & 31)) - 1)); };
    for (int k = tid; k < a.chunks; k += kTpListThreads) {
        const int v = TpPlace(a, row, k).v, end = v + kTpChunk;
        const uint32_t first = v <= 0 ? 0 : v < a.V ? ahead(v) : n;
        a.part[static_cast<int64_t>(row) * a.chunks + k] = make_uint2(first, (end < a.V ? ahead(end) : n) - first);
    }
    const auto place = [&](uint32_t t) {
        uint2* const to = list + ahead(t);
        to->x = t;  // (the same from all entries)
        return &to->y;
    };
    each_token(hist, old, a.V, [&](uint32_t t, int k) {
        if (k >= prompt) atomicAdd(place(t), 1u);
        else atomicOr(place(t), kTpSeen);
    });
    each_token(draft, n_draft, a.V, [&](uint32_t t, int) { atomicAdd(place(t), 1u); });
    each_token(bias_tok, a.K, a.V, [&](uint32_t t, int k) {
        uint32_t* const to = place(t);
        // (a second entry leaves the first's place and a mark that there are several)
        if (atomicOr(to, kTpBiased) & kTpBiased) atomicOr(to, kTpTwice);
        else atomicAdd(to, static_cast<uint32_t>(k + 1) << kTpBiasAt);
    });
    if (!near && !a.K) return;
    __syncthreads();
    for (uint32_t k = tid; k < n; k += kTpListThreads) {
        const uint2 e = list[k];
        if (near) far_list[k] = e;
        if (!(e.y & kTpBiased)) continue;
        float sum = bias_val[(e.y >> kTpBiasAt & 0x1fff) - 1];
        if (e.y & kTpTwice) {  // all that is listed for it, in the list's order
            sum = 0.f;
#pragma unroll 8
            for (int q = 0; q < a.K; ++q)
                if (bias_tok[q] == static_cast<int>(e.x)) sum = __fadd_rn(sum, bias_val[q]);
        }
        a.adjusted[row * a.listed + k] = sum;
    }
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

__device__ __forceinline__ void copy4(uint32_t dst, const void* src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// A warp's chunk in shared memory.  FIRST: the first pass, in which a thread has 32 tokens in
// a row, a word of the masks; the second: four times eight, a sector of what it writes.
template <bool HALF, bool FIRST>
struct TpStage {
    static constexpr int kResident = 20;                            // CTAs an SM
    static constexpr int kPieces = HALF ? 4 : 8;                    // of 16 bytes: a thread's 32 tokens
    static constexpr int kLogits = 32 * kPieces * 16;
    static constexpr int kMask = kTpWords * 4;
    static constexpr int kBytes = kLogits + 2 * kMask;              // (allowed, listed)
    static constexpr int kSmem = kTpWarps * kBytes;

    // Where a piece lies: in the first pass, which a thread reads in another order than it is
    // written, so that neither meets a bank twice.
    __device__ __forceinline__ static uint32_t slot(uint32_t piece) { return FIRST ? piece ^ ((piece >> 3) & (kPieces - 1)) : piece; }
    // The i-th piece that a thread copies: in the first pass they lie side by side, in the second
    // it is what the thread takes out itself.
    __device__ __forceinline__ static uint32_t mine(int lane, int i) { return HALF || FIRST ? lane + 32 * i : 2 * lane + (i & 1) + 32 * (i & ~1); }

    // A mask's words of the chunk.
    __device__ __forceinline__ static void copy_words(const TpParams& a, int lane, uint32_t to, const uint32_t* row, int v)
    {
        const int w = (v >> 5) + lane;
        if (static_cast<uint32_t>(w) < static_cast<uint32_t>(a.words)) copy4(to + lane * 4, row + w);
        if (lane == 0 && w + 32 < a.words) copy4(to + 128, row + w + 32);
    }
    __device__ __forceinline__ static void fill(const TpParams& a, uint8_t* stage, int row, const TpPlace& at)
    {
        const int lane = threadIdx.x & 31;
        const uint32_t to = smem_u32(stage);
        if (at.whole(a)) {
            const uint4* from = static_cast<const uint4*>(a.logits) + at.g * (HALF ? 1 : 2);
#pragma unroll
            for (int i = 0; i < kPieces; ++i) copy16(to + slot(mine(lane, i)) * 16, from + mine(lane, i));
        } else {
#pragma unroll 1
            for (int i = 0; i < kPieces; ++i) {
                const int piece = mine(lane, i), v = at.v + (HALF ? piece : piece / 2) * 8;
                const int64_t from = at.g * (HALF ? 1 : 2) + piece;
                if (whole8(a, v)) {
                    copy16(to + slot(piece) * 16, static_cast<const uint4*>(a.logits) + from);
                } else {  // a group that a row shares with its neighbour, or none of it
                    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < (HALF ? 8 : 4); ++j) {
                        const int t = v + (HALF ? j : (piece & 1) * 4 + j);
                        if (t < 0 || t >= a.V) continue;
                        if (HALF) w[j / 2] |= static_cast<uint32_t>(static_cast<const uint16_t*>(a.logits)[from * 8 + j]) << (j & 1) * 16;
                        else w[j % 4] = static_cast<const uint32_t*>(a.logits)[from * 4 + j];
                    }
                    *reinterpret_cast<uint4*>(stage + slot(piece) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        }
        const int64_t words = static_cast<int64_t>(row) * a.words;
        if (FIRST) {
            if (a.allowed) copy_words(a, lane, to + kLogits, a.allowed + words, at.v);
            if (a.listed) copy_words(a, lane, to + kLogits + kMask, a.marks + words, at.v);
        } else if (a.listed) {
            if (lane < kTpChunk / 128) copy16(to + kLogits + lane * 16, a.bits + at.item * (kTpChunk / 32) + lane * 4);
        } else if (a.allowed) {
            copy_words(a, lane, to + kLogits, a.allowed + words, at.v);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ static void wait()
    {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
    }
    // 32 bits from token `at` on of a mask's words, the first of which has token v >> 5 << 5.
    __device__ __forceinline__ static uint32_t bits_at(const uint8_t* stage, int mask, int v, int at)
    {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(stage + kLogits) + mask * kTpWords + (at >> 5) - (v >> 5);
        return __funnelshift_r(w[0], w[1], at);
    }
};

// x of eight tokens, -infinity for those without a bit.
template <bool HALF>
__device__ __forceinline__ void values8(const uint4& lo, const uint4& hi, uint32_t ok, float* x)
{
    const uint32_t h[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t u = HALF ? (j & 1 ? h[j / 2] & 0xffff0000u : h[j / 2] << 16) : h[j];
        x[j] = ok >> j & 1 ? __uint_as_float(u) : -INFINITY;
    }
}

// Takes further x of a row into a thread's pair.  token(k): x[k]'s.
template <int N, typename F>
__device__ __forceinline__ void add(float2& pair, const float (&x)[N], float T, float c, F token)
{
    float top = x[0];
#pragma unroll
    for (int k = 1; k < N; k += 2) top = max3f(top, x[k], x[k + 1 < N ? k + 1 : k]);
    if (T == 0.f) {
        int best = top > pair.x ? 0x7f7fffff : __float_as_int(pair.y);
        bool nan = pair.y != pair.y;
        pair.x = fmaxf(pair.x, top);
#pragma unroll
        for (int k = N - 1; k >= 0; --k) {
            if (x[k] == pair.x && top > -INFINITY) best = min(best, token(k));
            nan |= x[k] != x[k];
        }
        pair.y = nan ? NAN : __int_as_float(best);
        return;
    }
    if (top > pair.x) {
        pair.y *= ex2((pair.x - top) * c);  // (0 as yet for a first one)
        pair.x = top;
    }
    const float mid = pair.x == -INFINITY ? 0.f : pair.x;
    if constexpr (N == 1) {
        pair.y += ex2(__fmul_rn(__fadd_rn(x[0], -mid), c));
        return;
    }
    uint64_t part = f2_pack(0.f, 0.f);
    const uint64_t off = f2_pack(-mid, -mid), by = f2_pack(c, c);
    float lo, hi;
#pragma unroll
    for (int k = 0; k < N; k += 2) {
        f2_unpack(f2_mul(f2_add(f2_pack(x[k], x[(k + 1) % N]), off), by), lo, hi);
        part = f2_add(part, f2_pack(ex2(lo), ex2(hi)));
    }
    f2_unpack(part, lo, hi);
    pair.y += lo + hi;
}

// A listed token's logit, which is in the stage of the chunk at `at`, adjusted.
template <bool HALF>
__device__ __forceinline__ float adjust(const TpParams& a, const TpPlace& at, const uint8_t* stage, uint2 e, float bias, float rep, float freq, float pres)
{
    using Stage = TpStage<HALF, true>;
    const int off = static_cast<int>(e.x) - at.v;
    const uint8_t* const from = stage + Stage::slot(off / (HALF ? 8 : 4)) * 16;
    float y = HALF ? __uint_as_float(static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(from)[off % 8]) << 16)
                   : reinterpret_cast<const float*>(from)[off % 4];
    const uint32_t w = e.y, count = w & kTpCount;
    if (count || w & kTpSeen) y = y > 0.f ? __fdiv_rn(y, rep) : __fmul_rn(y, rep);
    if (count) y = __fsub_rn(y, __fadd_rn(__fmul_rn(static_cast<float>(count), freq), pres));
    if (w & kTpBiased) y = __fadd_rn(y, bias);
    if (a.allowed) {
        const uint32_t* words = reinterpret_cast<const uint32_t*>(stage + Stage::kLogits) - (at.v >> 5);
        if (!(words[e.x >> 5] >> (e.x & 31) & 1)) y = -INFINITY;
    }
    return y;
}

// What a chunk's sequence asks for.
struct TpAsked {
    float T, c, rep, freq, pres;

    __device__ __forceinline__ TpAsked(const TpParams& a, int row)
    {
        const int b = row / a.m1;
        T = a.temperature ? a.temperature[b] : 1.f, c = steepness(T);
        rep = a.penalty ? a.penalty[3 * b] : 1.f, freq = a.penalty ? a.penalty[3 * b + 1] : 0.f;
        pres = a.penalty ? a.penalty[3 * b + 2] : 0.f;
    }
};

// Of a row's listed tokens the first that is in a chunk, how many are, and this thread's first few.
struct TpListed {
    uint32_t first = 0, many = 0;
    uint2 e[kTpTake];

    __device__ __forceinline__ TpListed(const TpParams& a, int row, const TpPlace& at)
    {
        if (!a.listed) return;
        const uint2 part = a.part[at.item];
        first = part.x, many = part.y;
#pragma unroll
        for (int j = 0; j < kTpTake; ++j)
            if ((threadIdx.x & 31) + 32 * j < many) e[j] = a.list[row * a.listed + first + (threadIdx.x & 31) + 32 * j];
    }
};

// The first pass over a chunk: a thread's pair; ok: which of its 32 tokens count but for listed ones.
template <bool HALF>
__device__ __forceinline__ float2 first_pass(const TpParams& a, const uint8_t* stage, int row, const TpPlace& at,
                                             const TpAsked& q, TpListed& l, uint32_t& ok)
{
    using Stage = TpStage<HALF, true>;
    const int lane = threadIdx.x & 31, v = at.v + 32 * lane;  // this thread's first token
    ok = 0xffffffffu;
    if (!at.whole(a)) {
        if (v < 0) ok = 0xffffffffu << -v;
        if (v + 32 > a.V) ok &= v < a.V ? 0xffffffffu >> (v + 32 - a.V) : 0u;
    }
    uint32_t listed = ok;
    if (a.allowed) ok &= Stage::bits_at(stage, 0, at.v, v);
    if (a.listed) {
        listed &= Stage::bits_at(stage, 1, at.v, v);
        ok &= ~listed;
    }
    float2 pair = nothing(q.T, a.V);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        float x[16];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t piece = lane * Stage::kPieces + (2 * s + k) * (HALF ? 1 : 2);
            const uint4 lo = *reinterpret_cast<const uint4*>(stage + Stage::slot(piece) * 16);
            const uint4 hi = HALF ? lo : *reinterpret_cast<const uint4*>(stage + Stage::slot(piece + 1) * 16);
            values8<HALF>(lo, hi, ok >> (16 * s + 8 * k), x + 8 * k);
        }
        add(pair, x, q.T, q.c, [&](int k) { return v + 16 * s + k; });
    }
    // the listed tokens, in their order: a thread one of 32
    const uint2* const list = a.list + row * a.listed + l.first + lane;
    float* const adjusted = a.adjusted + row * a.listed + l.first + lane;
#pragma unroll 1
    for (uint32_t i0 = 0; i0 < l.many; i0 += 32 * kTpTake) {
        float bias[kTpTake];
#pragma unroll
        for (int j = 0; j < kTpTake; ++j) {
            bias[j] = 0.f;
            if (i0 + 32 * j + lane < l.many && l.e[j].y & kTpBiased) bias[j] = adjusted[i0 + 32 * j];
        }
#pragma unroll
        for (int j = 0; j < kTpTake; ++j) {
            if (i0 + 32 * j >= l.many) break;
            if (i0 + 32 * j + lane < l.many) {
                const float y[1] = {adjust<HALF>(a, at, stage, l.e[j], bias[j], q.rep, q.freq, q.pres)};
                adjusted[i0 + 32 * j] = y[0];
                add(pair, y, q.T, q.c, [&](int) { return static_cast<int>(l.e[j].x); });
            }
            if (i0 + 32 * (kTpTake + j) + lane < l.many) l.e[j] = list[i0 + 32 * (kTpTake + j)];
        }
    }
    return pair;
}

// The second: probabilities from a row's pair.  bits: the stage has, where the masks were, the
// tokens that count but for listed ones; else there are no lists.
template <bool HALF, bool FIRST>
__device__ __forceinline__ void second_pass(const TpParams& a, const uint8_t* stage, int row, const TpPlace& at, float T, float c,
                                            float2 total, bool bits, uint32_t first, uint32_t many, uint32_t token, float logit)
{
    using Stage = TpStage<HALF, FIRST>;
    const int lane = threadIdx.x & 31;
    const bool poor = total.y != total.y, special = poor || T == 0.f;  // (a NaN is all allowed tokens')
    const float scale = total.y == 0.f ? 1.f : 1.f / total.y;          // (where nothing is left all exponentials are 0)
    const float mid = total.x == -INFINITY ? 0.f : total.x;
    float* const out = a.p + at.g * 8;
    const bool all_whole = at.whole(a);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int v = at.v + 256 * k + 8 * lane;
        const bool whole = all_whole || whole8(a, v);
        uint32_t ok;
        if (bits) {
            ok = (stage + Stage::kLogits + k * 32)[lane];
        } else {
            ok = whole ? 0xffu : inside(a.V, v);
            if (a.allowed) ok &= Stage::bits_at(stage, 0, at.v, v);
        }
        const uint32_t piece = HALF ? 32 * k + lane : 64 * k + 2 * lane;
        const uint4 lo = *reinterpret_cast<const uint4*>(stage + Stage::slot(piece) * 16);
        const uint4 hi = HALF ? lo : *reinterpret_cast<const uint4*>(stage + Stage::slot(piece + 1) * 16);
        float x[8];
        values8<HALF>(lo, hi, ok, x);
        if (__builtin_expect(special, 0)) {
            const uint32_t all = !a.allowed || v >= a.V ? 0xffu : bits_of(a.allowed + static_cast<int64_t>(row) * a.words, a.words, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = poor ? (all >> j & 1 ? NAN : 0.f) : v + j == __float_as_int(total.y) ? 1.f : 0.f;
        } else {
            const uint64_t off = f2_pack(-mid, -mid), by = f2_pack(c, c), mul = f2_pack(scale, scale);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                float e0, e1;
                f2_unpack(f2_mul(f2_add(f2_pack(x[j], x[j + 1]), off), by), e0, e1);
                f2_unpack(f2_mul(f2_pack(ex2(e0), ex2(e1)), mul), x[j], x[j + 1]);
            }
        }
        float* const to = out + 256 * k + 8 * lane;
        if (whole) {
            reinterpret_cast<float4*>(to)[0] = make_float4(x[0], x[1], x[2], x[3]);
            reinterpret_cast<float4*>(to)[1] = make_float4(x[4], x[5], x[6], x[7]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (v + j >= 0 && v + j < a.V) to[j] = x[j];
        }
    }
    if (many && !special) {  // (a 0 is there now)
        __syncwarp();
        const uint2* const list = a.list + row * a.listed + first;
        const float* const adjusted = a.adjusted + row * a.listed + first;
        float* const to = a.p + static_cast<int64_t>(row) * a.V;
        const auto prob = [&](float y) { return __fmul_rn(ex2(__fmul_rn(__fadd_rn(y, -mid), c)), scale); };
        if (lane < many) to[token] = prob(logit);
#pragma unroll 1
        for (uint32_t i0 = 32 + lane; i0 < many + lane; i0 += 32 * kTpTake) {  // (where many neighbours are listed)
            uint32_t t[kTpTake];
            float y[kTpTake];
#pragma unroll
            for (int j = 0; j < kTpTake; ++j) {
                const uint32_t i = i0 + 32 * j;
                t[j] = i < many ? list[i].x : 0;
                y[j] = i < many ? adjusted[i] : 0.f;
            }
#pragma unroll
            for (int j = 0; j < kTpTake; ++j)
                if (i0 + 32 * j < many) to[t[j]] = prob(y[j]);
        }
    }
}

template <bool HALF>
__global__ void __launch_bounds__(kTpThreads, TpStage<HALF, true>::kResident) target_stats_kernel(TpParams a)
{
    using Stage = TpStage<HALF, true>;
    extern __shared__ __align__(16) uint8_t smem_stage[];
    wait_for_stream();
    // (rows first: the tokens that lists name are often neighbours, and their chunks take longest)
    const int lane = threadIdx.x & 31, row = blockIdx.x * kTpWarps + threadIdx.x / 32, chunk = blockIdx.y;
    if (row >= a.B * a.m1) return;
    const TpPlace at(a, row, chunk);
    uint8_t* const stage = smem_stage + threadIdx.x / 32 * Stage::kBytes;
    Stage::fill(a, stage, row, at);
    const TpAsked q(a, row);
    TpListed l(a, row, at);
    Stage::wait();
    uint32_t ok;
    const float2 pair = join_warp(first_pass<HALF>(a, stage, row, at, q, l, ok), q.T, q.c);
    if (a.listed) a.bits[at.item * (kTpChunk / 32) + lane] = ok;
    if (lane == 0) a.stats[at.item] = pair;
}

template <bool HALF>
__global__ void __launch_bounds__(kTpThreads, TpStage<HALF, false>::kResident) target_write_kernel(TpParams a)
{
    using Stage = TpStage<HALF, false>;
    extern __shared__ __align__(16) uint8_t smem_stage[];
    wait_for_stream();
    // what was read last comes first, but for the first chunks, as above
    const int lane = threadIdx.x & 31, row = a.B * a.m1 - 1 - static_cast<int>(blockIdx.x * kTpWarps + threadIdx.x / 32),
              chunk = blockIdx.y ? a.chunks - static_cast<int>(blockIdx.y) : 0;
    if (row < 0) return;
    const TpPlace at(a, row, chunk);
    uint8_t* const stage = smem_stage + threadIdx.x / 32 * Stage::kBytes;
    Stage::fill(a, stage, row, at);
    // listed tokens of the chunk, and their adjusted logits
    uint32_t first = 0, many = 0, token = 0;
    float logit = 0.f;
    if (a.listed) {
        const uint2 part = a.part[at.item];
        first = part.x, many = part.y;
        if (lane < many) token = a.list[row * a.listed + first + lane].x, logit = a.adjusted[row * a.listed + first + lane];
    }
    const float T = a.temperature ? a.temperature[row / a.m1] : 1.f, c = steepness(T);
    float2 total = nothing(T, a.V);
#pragma unroll 1
    for (int k0 = lane; k0 < a.chunks; k0 += 32 * kTpTake) {
        float2 q[kTpTake];
#pragma unroll
        for (int j = 0; j < kTpTake; ++j)
            if (k0 + 32 * j < a.chunks) q[j] = a.stats[static_cast<int64_t>(row) * a.chunks + k0 + 32 * j];
#pragma unroll
        for (int j = 0; j < kTpTake; ++j)
            if (k0 + 32 * j < a.chunks) total = join(total, q[j], T, c);
    }
    total = join_warp(total, T, c);
    Stage::wait();
    second_pass<HALF, false>(a, stage, row, at, T, c, total, a.listed != 0, first, many, token, logit);
}

// Both passes over a row of up to 16 chunks by one CTA, a warp a chunk, which stays in shared
// memory.  It saves a launch and the second read: 400 rows of 8100, float32, histories of 500
// 15.8 us (two kernels 22.0), one row of 2000 7.3 (9.3); at 16 chunks they are even (one row of
// 16300 9.6 and 9.6, 400 of them, bf16, histories of 1000 26.9 and 26.6), beyond that an SM is too slow for a row (32000: 13.1 and 9.6).
template <bool HALF>
__global__ void __launch_bounds__(kTpRowWarps * 32) target_row_kernel(TpParams a)
{
    using Stage = TpStage<HALF, true>;
    extern __shared__ __align__(16) uint8_t smem_stage[];
    __shared__ float2 sh[kTpRowWarps];
    wait_for_stream();
    const int lane = threadIdx.x & 31, row = blockIdx.x, chunk = threadIdx.x / 32;
    const TpPlace at(a, row, chunk);
    uint8_t* const stage = smem_stage + chunk * Stage::kBytes;
    Stage::fill(a, stage, row, at);
    const TpAsked q(a, row);
    TpListed l(a, row, at);
    Stage::wait();
    uint32_t ok;
    const float2 pair = join_warp(first_pass<HALF>(a, stage, row, at, q, l, ok), q.T, q.c);
    if (lane == 0) sh[chunk] = pair;
    __syncthreads();
    reinterpret_cast<uint32_t*>(stage + Stage::kLogits)[lane] = ok;
    const float2 total = join_warp(lane < a.chunks ? sh[lane] : nothing(q.T, a.V), q.T, q.c);
    __syncwarp();
    uint32_t token = 0;
    float logit = 0.f;
    if (lane < l.many) token = a.list[row * a.listed + l.first + lane].x, logit = a.adjusted[row * a.listed + l.first + lane];
    second_pass<HALF, true>(a, stage, row, at, q.T, q.c, total, true, l.first, l.many, token, logit);
}

int64_t tp_chunks(int V) { return (V + 7 + kTpChunk - 1) / kTpChunk; }  // (a row's first may begin 7 tokens early)

// Offsets of the workspace's parts; the last is its size.
struct TpRoom {
    size_t marks, bits, part, list, adjusted, bytes;
    int64_t listed;
};

TpRoom tp_room(int B, int m1, int V, int H, int K)
{
    const size_t rows = static_cast<size_t>(B) * m1;
    TpRoom r;
    r.listed = std::min<int64_t>(V, static_cast<int64_t>(H) + (m1 - 1) + K);
    r.marks = round_up(rows * tp_chunks(V) * sizeof(float2), 256);
    r.bits = r.marks + (r.listed ? round_up(rows * ((V + 31) / 32) * 4, 256) : 0);
    r.part = r.bits + (r.listed ? round_up(rows * tp_chunks(V) * (kTpChunk / 8), 256) : 0);
    r.list = r.part + (r.listed ? round_up(rows * tp_chunks(V) * sizeof(uint2), 256) : 0);
    r.adjusted = r.list + round_up(rows * r.listed * sizeof(uint2), 256);
    r.bytes = r.adjusted + round_up(rows * r.listed * sizeof(float), 256);
    return r;
}

int check_probs(int B, int m1, int V, int H, int K)
{
    if (B < 1 || m1 < 1 || V < 1 || H < 0 || K < 0) return LOGO_ERR_INVALID_ARG;
    if (V > LOGO_PROBS_MAX_VOCAB || m1 > 1024 || K > kTpMaxBiases || static_cast<int64_t>(B) * m1 > (1 << 24) ||
        static_cast<int64_t>(B) * H > (1ll << 40))
        return LOGO_ERR_UNSUPPORTED;
    return LOGO_OK;
}

template <bool HALF>
int tp_launch(TpParams& a, cudaStream_t st)
{
    const int lists_smem = (a.words + 3) / 4 * 32 + a.K * 8 + (a.listed <= kTpNear ? static_cast<int>(a.listed * sizeof(uint2)) : 0);
    static OncePerDevice once;
    if (once([] {
            // (the kernels overlap at their ends, and an SM splits its memory anew only when it is idle)
            const auto all_shared = [](auto kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared); };
            cudaError_t e = all_shared(target_lists_kernel);
            if (e == cudaSuccess) e = all_shared(target_stats_kernel<HALF>);
            if (e == cudaSuccess) e = all_shared(target_write_kernel<HALF>);
            if (e == cudaSuccess) e = set_smem_limit(target_lists_kernel, (LOGO_PROBS_MAX_VOCAB + 127) / 128 * 32 + kTpMaxBiases * 8 + kTpNear * static_cast<int>(sizeof(uint2)));
            if (e == cudaSuccess) e = all_shared(target_row_kernel<HALF>);
            if (e == cudaSuccess) e = set_smem_limit(target_row_kernel<HALF>, kTpRowWarps * TpStage<HALF, true>::kBytes);
            if (e == cudaSuccess) e = set_smem_limit(target_stats_kernel<HALF>, TpStage<HALF, true>::kSmem);
            return e == cudaSuccess ? set_smem_limit(target_write_kernel<HALF>, TpStage<HALF, false>::kSmem) : e;
        }) != cudaSuccess)
        return LOGO_ERR_CUDA;
    const unsigned rows = static_cast<unsigned>(a.B) * a.m1;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (a.listed) {
        cfg.gridDim = dim3(rows);
        cfg.blockDim = dim3(kTpListThreads);
        cfg.dynamicSmemBytes = lists_smem;
        if (cudaLaunchKernelEx(&cfg, target_lists_kernel, a) != cudaSuccess) return LOGO_ERR_CUDA;
    }
    if (a.chunks <= kTpRowWarps) {
        cfg.gridDim = dim3(rows);
        cfg.blockDim = dim3(32 * a.chunks);
        cfg.dynamicSmemBytes = a.chunks * TpStage<HALF, true>::kBytes;
        return cudaLaunchKernelEx(&cfg, target_row_kernel<HALF>, a) == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
    }
    cfg.gridDim = dim3((rows + kTpWarps - 1) / kTpWarps, static_cast<unsigned>(a.chunks));
    cfg.blockDim = dim3(kTpThreads);
    cfg.dynamicSmemBytes = TpStage<HALF, true>::kSmem;
    static_assert(TpStage<HALF, true>::kSmem == TpStage<HALF, false>::kSmem, "one size for both passes");
    if (cudaLaunchKernelEx(&cfg, target_stats_kernel<HALF>, a) != cudaSuccess) return LOGO_ERR_CUDA;
    return cudaLaunchKernelEx(&cfg, target_write_kernel<HALF>, a) == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}

}  // namespace
}  // namespace logo

using namespace logo;

extern "C" size_t logo_target_probs_workspace_size(int B, int m1, int V, int H, int K)
{
    return check_probs(B, m1, V, H, K) == LOGO_OK ? tp_room(B, m1, V, H, K).bytes : 0;
}

extern "C" int logo_target_probs(const void* logits, int logits_bf16, const float* temperature, const float* penalty,
                                 const int32_t* history, const int32_t* hist_len, const int32_t* n_prompt,
                                 const int32_t* draft, const int32_t* bias_tok, const float* bias_val,
                                 const int32_t* allowed, float* p, int B, int m1, int V, int H, int K, void* workspace,
                                 size_t workspace_bytes, void* stream)
{
    const int rc = check_probs(B, m1, V, H, K);
    if (rc != LOGO_OK) return rc;
    if (!logits || !p) return LOGO_ERR_INVALID_ARG;
    if ((history != nullptr) != (hist_len != nullptr) || (n_prompt && !history) || (!history && H > 0) ||
        (history && H < 1) || ((history || draft) && !penalty) || (draft && m1 < 2))
        return LOGO_ERR_INVALID_ARG;
    if ((bias_tok != nullptr) != (K > 0) || (bias_val != nullptr) != (K > 0)) return LOGO_ERR_INVALID_ARG;
    if (!aligned16(logits) || !aligned16(p) || (logits_bf16 && logits == p)) return LOGO_ERR_UNSUPPORTED;
    const TpRoom room = tp_room(B, m1, V, H, K);
    if (!workspace || workspace_bytes < room.bytes || !aligned16(workspace)) return LOGO_ERR_WORKSPACE;
    // (in place each stretch of a row is read before it is written; elsewhere over the logits it is another's)
    const size_t tokens = static_cast<size_t>(B) * m1 * V;
    if (logits != p && overlap(logits, tokens * (logits_bf16 ? 2 : 4), p, tokens * 4)) return LOGO_ERR_INVALID_ARG;
    uint8_t* const ws = static_cast<uint8_t*>(workspace);
    TpParams a{};
    a.logits = logits, a.temperature = temperature, a.penalty = penalty, a.history = history, a.hist_len = hist_len;
    a.n_prompt = n_prompt, a.draft = draft, a.bias_tok = bias_tok, a.bias_val = bias_val;
    a.allowed = reinterpret_cast<const uint32_t*>(allowed), a.p = p;
    a.B = B, a.m1 = m1, a.V = V, a.H = H, a.K = K;
    a.chunks = static_cast<int>(tp_chunks(V)), a.words = (V + 31) / 32;
    a.listed = history || draft || K > 0 ? room.listed : 0;
    a.stats = reinterpret_cast<float2*>(ws);
    a.marks = reinterpret_cast<uint32_t*>(ws + room.marks);
    a.bits = reinterpret_cast<uint32_t*>(ws + room.bits), a.part = reinterpret_cast<uint2*>(ws + room.part);
    a.list = reinterpret_cast<uint2*>(ws + room.list), a.adjusted = reinterpret_cast<float*>(ws + room.adjusted);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return logits_bf16 ? tp_launch<true>(a, st) : tp_launch<false>(a, st);
}
