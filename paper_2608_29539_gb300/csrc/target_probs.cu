// target_probs.cu -- logits to the target's probabilities: penalties for repeated
// tokens, biases, a grammar's mask, temperature, softmax:
// p_v = 2^((x_v - max x) log2(e) / T) / sum.
//
// HBM bounds it: 2 or 4 bytes read, 1/8 of one for the mask and 4 written per token.  Two
// streaming passes, the second of which finds most logits in L2 (it goes through the rows
// backwards): the first leaves a maximum and a sum of exponentials per 4096 tokens, the
// second takes all of a row's and writes.  (One pass that kept a row in the registers of a
// thread-block cluster between its read and its write took 122 us for 240 rows of 131072:
// clusters follow one another, wait for their slowest CTA and do the lists' work eight
// times.)
// The lists of tokens (history, drafts, biases) are counted ahead of that, a CTA a row.  The
// listed tokens are left out of the first pass; between the passes, when their logits are in
// L2, they are adjusted, in the tokens' order, so that sums do not depend on the order of
// atomics, and lie in p until the second pass takes them from there.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "host_common.h"
#include "sm100.cuh"

namespace logo {
namespace {

constexpr int kTpThreads = 256;
constexpr int kTpGroups = 2;                               // groups of eight tokens a thread
constexpr int kTpChunk = kTpThreads * kTpGroups;           // groups a CTA
constexpr int kTpListThreads = 512;
constexpr int kTpAt = 4;                                   // list entries in flight per thread
constexpr int kTpNear = 8192;                              // listed tokens that are counted in shared memory
// a listed token's word: how often it was generated, its place among the biases (plus one), flags
constexpr uint32_t kTpSeen = 1u << 31, kTpBiased = 1u << 30, kTpTwice = 1u << 29, kTpCount = (1u << 15) - 1;
constexpr int kTpBiasAt = 15, kTpTake = 8;                 // listed tokens of a thread at a time
static_assert(LOGO_PROBS_MAX_COUNTED + 1024 <= kTpCount, "counts have room");

struct TpParams {
    const void* logits;
    const float *temperature, *penalty;
    const int32_t *history, *hist_len, *n_prompt, *draft, *bias_tok;
    const float* bias_val;
    const uint32_t* allowed;
    float* p;
    int B, m1, V, H, K;
    int chunks;         // CTAs a row
    int words;          // of a bit a token: ceil(V / 32)
    int64_t listed;     // room for listed tokens a row (0: no lists)
    int pairs;          // of a row: one a chunk, then its listed tokens'
    float2* stats;      // [rows][pairs] (maximum, sum)
    uint32_t* marks;    // [rows][words]: a bit a listed token
    uint16_t* bits;     // [rows][chunks * groups]: of eight tokens, those allowed and not listed; in the upper byte those listed
    uint2* far;         // [rows][listed], where that is more than shared memory is used for
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

// Over a CTA's warps, in its first one; sh: a pair per warp.
template <int WARPS>
__device__ __forceinline__ float2 join_block(float2 p, float T, float c, float2* sh)
{
    if (threadIdx.x % 32 == 0) sh[threadIdx.x / 32] = p;
    __syncthreads();
    if (threadIdx.x >= 32) return p;
    return join_warp(threadIdx.x < WARPS ? sh[threadIdx.x] : make_float2(-INFINITY, T == 0.f ? __int_as_float(0x7f7fffff) : 0.f), T, c);
}

// A warp's pair: its largest x, then the sum.  tokens(k): the token of x[k], ascending.
template <int N, typename F>
__device__ __forceinline__ float2 pair_of(const float (&x)[N], float T, float c, int V, F tokens)
{
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < N; k += 2) top = max3f(top, x[k], x[k + 1]);
    top = unordered(__reduce_max_sync(0xffffffffu, ordered(top)));
    if (T == 0.f) {
        int chosen = V;
        bool nan = false;
#pragma unroll
        for (int k = N - 1; k >= 0; --k) {
            if (x[k] == top && top > -INFINITY) chosen = tokens(k);
            nan |= x[k] != x[k];
        }
        chosen = __reduce_min_sync(0xffffffffu, chosen);
        return make_float2(top, __any_sync(0xffffffffu, nan) ? NAN : __int_as_float(chosen));
    }
    const float mid = top == -INFINITY ? 0.f : top;
    uint64_t part = f2_pack(0.f, 0.f);
    const uint64_t off = f2_pack(-mid, -mid), by = f2_pack(c, c);
    float lo, hi;
#pragma unroll
    for (int k = 0; k < N; k += 2) {
        f2_unpack(f2_mul(f2_add(f2_pack(x[k], x[k + 1]), off), by), lo, hi);
        part = f2_add(part, f2_pack(ex2(lo), ex2(hi)));
    }
    f2_unpack(part, lo, hi);
    float sum = lo + hi;
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    return make_float2(top, sum);
}

template <bool HALF>
__device__ __forceinline__ float logit(const TpParams& a, int64_t e)
{
    return HALF ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(a.logits)[e]) << 16)
                : static_cast<const float*>(a.logits)[e];
}

// f(token, index) for the entries of a list that are tokens, kTpAt loads in flight.
template <typename F>
__device__ __forceinline__ void each_token(const int32_t* list, int len, int V, F f)
{
#pragma unroll 1
    for (int k0 = threadIdx.x; k0 < len; k0 += kTpAt * kTpListThreads) {
        uint32_t t[kTpAt];
#pragma unroll
        for (int k = 0; k < kTpAt; ++k) t[k] = k0 + k * kTpListThreads < len ? __ldg(list + k0 + k * kTpListThreads) : 0xffffffffu;
#pragma unroll
        for (int k = 0; k < kTpAt; ++k)
            if (t[k] < static_cast<uint32_t>(V)) f(t[k], k0 + k * kTpListThreads);
    }
}

// Eight tokens of a row.  Groups begin at multiples of eight of the whole tensor's
// elements, so all but a row's first and last are whole and aligned.
struct TpGroup {
    int64_t g;     // of the tensor
    int v;         // its first token; less than 0 in a row's first group
    bool in;       // a group of the row
};

__device__ __forceinline__ TpGroup group_of(const TpParams& a, int row, int chunk, int k)
{
    const int64_t e0 = static_cast<int64_t>(row) * a.V;
    const uint32_t at = chunk * kTpChunk + k * kTpThreads + threadIdx.x;
    const int v = static_cast<int>(at * 8) - static_cast<int>(e0 & 7);
    return TpGroup{e0 / 8 + at, v, v < a.V};
}

// Bits of eight tokens from a row of a bit a token.
__device__ __forceinline__ uint32_t bits_of(const uint32_t* row, int words, int v)
{
    const int w = max(v, 0) / 32;
    const uint32_t lo = row[w], hi = row[w + (w + 1 < words)];
    return (v < 0 ? lo << -v : __funnelshift_r(lo, hi, v & 31)) & 0xffu;
}

// A row's lists: the listed tokens counted, then adjusted, into p; their pair, and what is
// left to the passes.
template <bool HALF>
__global__ void __launch_bounds__(kTpListThreads) target_lists_kernel(TpParams a)
{
    extern __shared__ __align__(16) uint32_t smem[];
    __shared__ uint32_t sh_sum[kTpListThreads / 32];
    __shared__ float2 sh_pair[kTpListThreads / 32];
    const int row = blockIdx.x, b = row / a.m1, i = row - b * a.m1, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int room = (a.words + 3) / 4 * 4;
    uint32_t *const bits = smem, *const before = smem + room;
    for (int w = tid; w < room; w += kTpListThreads) bits[w] = 0;
    wait_for_stream();
    const int old = a.history ? max(0, min(a.hist_len[b], a.H)) : 0;
    const int prompt = max(a.n_prompt ? a.n_prompt[b] : 0, old - LOGO_PROBS_MAX_COUNTED);
    const int32_t* hist = a.history + static_cast<int64_t>(b) * a.H;
    const int32_t* draft = a.draft + static_cast<int64_t>(b) * (a.m1 - 1);
    const int n_draft = a.draft ? i : 0;
    const int32_t* tok = a.bias_tok + static_cast<int64_t>(b) * a.K;
    const float* val = a.bias_val + static_cast<int64_t>(b) * a.K;
    const float T = a.temperature ? a.temperature[b] : 1.f, c = steepness(T);
    const float rep = a.penalty ? a.penalty[3 * b] : 1.f, freq = a.penalty ? a.penalty[3 * b + 1] : 0.f,
                pres = a.penalty ? a.penalty[3 * b + 2] : 0.f;
    __syncthreads();
    const int64_t row0 = static_cast<int64_t>(row) * a.V;
    const auto mark = [&](uint32_t t, int) { atomicOr(bits + t / 32, 1u << (t & 31)); };
    each_token(hist, old, a.V, mark);
    each_token(draft, n_draft, a.V, mark);
    each_token(tok, a.K, a.V, mark);
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
    // the tokens and their words in shared memory where there is room, else in the workspace
    uint2* const list = a.listed <= kTpNear ? reinterpret_cast<uint2*>(smem + 2 * room) : a.far + row * a.listed;
    for (uint32_t k = tid; k < n; k += kTpListThreads) list[k] = make_uint2(0, 0);
    __syncthreads();
    for (int w = tid; w < a.words; w += kTpListThreads) a.marks[static_cast<int64_t>(row) * a.words + w] = bits[w];
    const auto place = [&](uint32_t t) {
        uint2* const to = list + before[t / 32] + __popc(bits[t / 32] & ((1u << (t & 31)) - 1));
        to->x = t;  // (the same from all entries)
        return &to->y;
    };
    each_token(hist, old, a.V, [&](uint32_t t, int k) {
        if (k >= prompt) atomicAdd(place(t), 1u);
        else atomicOr(place(t), kTpSeen);
    });
    each_token(draft, n_draft, a.V, [&](uint32_t t, int) { atomicAdd(place(t), 1u); });
    each_token(tok, a.K, a.V, [&](uint32_t t, int k) {
        uint32_t* const to = place(t);
        // (a second entry leaves the first's place and a mark that there are several)
        if (atomicOr(to, kTpBiased) & kTpBiased) atomicOr(to, kTpTwice);
        else atomicAdd(to, static_cast<uint32_t>(k + 1) << kTpBiasAt);
    });
    __syncthreads();
    // adjusted in the tokens' order
    const uint32_t* allowed = a.allowed ? a.allowed + static_cast<int64_t>(row) * a.words : nullptr;
    float2 pair = nothing(T, a.V);
#pragma unroll 1
    for (uint32_t k0 = tid; k0 < n + tid; k0 += kTpTake * kTpListThreads) {
        uint2 e[kTpTake];
        uint32_t in[kTpTake];
        float x[kTpTake];
#pragma unroll
        for (int j = 0; j < kTpTake; ++j) {
            const uint32_t k = k0 + j * kTpListThreads;
            e[j] = k < n ? list[k] : make_uint2(a.V, 0);
            x[j] = k < n ? logit<HALF>(a, row0 + e[j].x) : -INFINITY;
            in[j] = allowed && k < n ? __ldg(allowed + e[j].x / 32) >> (e[j].x & 31) & 1 : 1;
        }
#pragma unroll
        for (int j = 0; j < kTpTake; ++j) {
            const uint32_t t = e[j].x, w = e[j].y, count = w & kTpCount;
            if (t == a.V) continue;
            float y = x[j];
            if (count || w & kTpSeen) y = y > 0.f ? __fdiv_rn(y, rep) : __fmul_rn(y, rep);
            if (count) y = __fsub_rn(y, __fadd_rn(__fmul_rn(static_cast<float>(count), freq), pres));
            if (w & kTpBiased) {
                float sum = 0.f;
                if (w & kTpTwice) {  // all that is listed for it, in the list's order
#pragma unroll 8
                    for (int q = 0; q < a.K; ++q)
                        if (__ldg(tok + q) == t) sum = __fadd_rn(sum, val[q]);
                } else {
                    sum = val[(w >> kTpBiasAt & 0x1fff) - 1];
                }
                y = __fadd_rn(y, sum);
            }
            if (!in[j]) y = -INFINITY;
            a.p[row0 + t] = y;
            x[j] = y;
        }
        pair = join(pair, pair_of(x, T, c, a.V, [&](int j) { return static_cast<int>(e[j].x); }), T, c);
    }
    pair = join_block<W>(pair, T, c, sh_pair);
    if (tid == 0) a.stats[static_cast<int64_t>(row) * a.pairs + a.chunks] = pair;
}

// A thread's tokens as they come; of each group, the bits of those that count here and, in the
// upper byte, of those that are listed.
template <bool HALF>
struct TpTokens {
    uint4 raw[kTpGroups][2];
    uint32_t ok[kTpGroups];

    // FIRST: the bits are put together, and written for the second pass, else read.
    template <bool FIRST>
    __device__ __forceinline__ TpTokens(const TpParams& a, int row, int chunk, std::bool_constant<FIRST>)
    {
#pragma unroll
        for (int k = 0; k < kTpGroups; ++k) {
            const TpGroup t = group_of(a, row, chunk, k);
            ok[k] = 0;
            raw[k][0] = raw[k][1] = make_uint4(0, 0, 0, 0);
            if (!t.in) continue;
            uint16_t* const bits = a.bits + static_cast<int64_t>(row) * a.chunks * kTpChunk + chunk * kTpChunk + k * kTpThreads + threadIdx.x;
            if (!FIRST && a.listed) {
                ok[k] = *bits;
            } else {
                const int64_t words = static_cast<int64_t>(row) * a.words;
                ok[k] = inside(a.V, t.v) & (a.allowed ? bits_of(a.allowed + words, a.words, t.v) : 0xffu);
                if (a.listed) {
                    const uint32_t listed = inside(a.V, t.v) & bits_of(a.marks + words, a.words, t.v);
                    ok[k] &= ~listed;
                    *bits = static_cast<uint16_t>(listed << 8 | ok[k]);
                }
            }
            if (t.v >= 0 && t.v + 8 <= a.V) {
                raw[k][0] = static_cast<const uint4*>(a.logits)[t.g * (HALF ? 1 : 2)];
                if (!HALF) raw[k][1] = static_cast<const uint4*>(a.logits)[t.g * 2 + 1];
            } else {
                uint32_t word[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool in = t.v + j >= 0 && t.v + j < a.V;
                    word[j] = !in ? 0 : HALF ? static_cast<const uint16_t*>(a.logits)[t.g * 8 + j] : static_cast<const uint32_t*>(a.logits)[t.g * 8 + j];
                }
                if (HALF) {
                    raw[k][0] = make_uint4(word[0] | word[1] << 16, word[2] | word[3] << 16, word[4] | word[5] << 16, word[6] | word[7] << 16);
                } else {
                    raw[k][0] = make_uint4(word[0], word[1], word[2], word[3]);
                    raw[k][1] = make_uint4(word[4], word[5], word[6], word[7]);
                }
            }
        }
    }
    // -infinity for those that are left out
    __device__ __forceinline__ void logits(float (&x)[kTpGroups * 8]) const
    {
#pragma unroll
        for (int k = 0; k < kTpGroups; ++k) {
            const uint32_t h[8] = {raw[k][0].x, raw[k][0].y, raw[k][0].z, raw[k][0].w, raw[k][1].x, raw[k][1].y, raw[k][1].z, raw[k][1].w};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t u = HALF ? (j & 1 ? h[j / 2] & 0xffff0000u : h[j / 2] << 16) : h[j];
                x[8 * k + j] = ok[k] >> j & 1 ? __uint_as_float(u) : -INFINITY;
            }
        }
    }
};

template <bool HALF>
__global__ void __launch_bounds__(kTpThreads) target_stats_kernel(TpParams a)
{
    __shared__ float2 sh[kTpThreads / 32];
    wait_for_stream();
    const int row = blockIdx.x, chunk = blockIdx.y;  // (rows first: the tokens that lists name are often neighbours)
    const float T = a.temperature ? a.temperature[row / a.m1] : 1.f, c = steepness(T);
    float x[kTpGroups * 8];
    TpTokens<HALF>(a, row, chunk, std::true_type()).logits(x);
    float2 pair = pair_of(x, T, c, a.V, [&](int k) { return group_of(a, row, chunk, k / 8).v + k % 8; });
    pair = join_block<kTpThreads / 32>(pair, T, c, sh);
    if (threadIdx.x == 0) a.stats[static_cast<int64_t>(row) * a.pairs + chunk] = pair;
}

template <bool HALF>
__global__ void __launch_bounds__(kTpThreads) target_write_kernel(TpParams a)
{
    __shared__ float2 sh_total;
    wait_for_stream();
    const int row = a.B * a.m1 - 1 - blockIdx.x, chunk = a.chunks - 1 - blockIdx.y;  // what was read last comes first
    const float T = a.temperature ? a.temperature[row / a.m1] : 1.f, c = steepness(T);
    const TpTokens<HALF> tokens(a, row, chunk, std::false_type());
    if (threadIdx.x < 32) {
        float2 pair = nothing(T, a.V);
        for (int k = threadIdx.x; k < a.pairs; k += 32) pair = join(pair, a.stats[static_cast<int64_t>(row) * a.pairs + k], T, c);
        pair = join_warp(pair, T, c);
        if (threadIdx.x == 0) sh_total = pair;
    }
    __syncthreads();
    const float2 total = sh_total;
    float x[kTpGroups * 8];
    tokens.logits(x);
#pragma unroll
    for (int k = 0; k < kTpGroups; ++k) {  // listed tokens, whose adjusted logits lie in p
        const uint32_t take = tokens.ok[k] >> 8;
        if (!take) continue;
        const TpGroup t = group_of(a, row, chunk, k);
        const float* from = a.p + t.g * 8;
        if (t.v >= 0 && t.v + 8 <= a.V) {
            const float4 lo = reinterpret_cast<const float4*>(from)[0], hi = reinterpret_cast<const float4*>(from)[1];
            const float y[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (take >> j & 1) x[8 * k + j] = y[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (take >> j & 1) x[8 * k + j] = from[j];
        }
    }
    const float mid = total.x == -INFINITY ? 0.f : total.x, sum = total.y;
    const bool greedy = T == 0.f, poor = sum != sum;  // a NaN is all allowed tokens'
    const int chosen = __float_as_int(sum);
    const float scale = sum == 0.f ? 1.f : 1.f / sum;  // (where nothing is left all exponentials are 0)
    if (greedy) {
#pragma unroll
        for (int k = 0; k < kTpGroups * 8; ++k) x[k] = group_of(a, row, chunk, k / 8).v + k % 8 == chosen ? 1.f : 0.f;
    } else {
        const uint64_t off = f2_pack(-mid, -mid), by = f2_pack(c, c), to = f2_pack(scale, scale);
#pragma unroll
        for (int k = 0; k < kTpGroups * 8; k += 2) {
            float lo, hi;
            f2_unpack(f2_mul(f2_add(f2_pack(x[k], x[k + 1]), off), by), lo, hi);
            f2_unpack(f2_mul(f2_pack(ex2(lo), ex2(hi)), to), x[k], x[k + 1]);
        }
    }
#pragma unroll
    for (int k = 0; k < kTpGroups; ++k) {
        const TpGroup t = group_of(a, row, chunk, k);
        if (!t.in) continue;
        if (poor) {
            const uint32_t ok = a.allowed ? bits_of(a.allowed + static_cast<int64_t>(row) * a.words, a.words, t.v) : 0xffu;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[8 * k + j] = ok >> j & 1 ? NAN : 0.f;
        }
        float* to = a.p + t.g * 8;
        if (t.v >= 0 && t.v + 8 <= a.V) {
            __stcs(reinterpret_cast<float4*>(to), make_float4(x[8 * k], x[8 * k + 1], x[8 * k + 2], x[8 * k + 3]));
            __stcs(reinterpret_cast<float4*>(to) + 1, make_float4(x[8 * k + 4], x[8 * k + 5], x[8 * k + 6], x[8 * k + 7]));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (t.v + j >= 0 && t.v + j < a.V) to[j] = x[8 * k + j];
        }
    }
}

int64_t tp_chunks(int V) { return (V / 8 + 2 + kTpChunk - 1) / kTpChunk; }

// Offsets of the workspace's parts; the last is its size.
struct TpRoom {
    size_t marks, bits, far, bytes;
    int64_t listed;
};

TpRoom tp_room(int B, int m1, int V, int H, int K)
{
    const size_t rows = static_cast<size_t>(B) * m1;
    TpRoom r;
    r.listed = std::min<int64_t>(V, static_cast<int64_t>(H) + (m1 - 1) + K);
    r.marks = round_up(rows * (tp_chunks(V) + 1) * sizeof(float2), 256);
    r.bits = r.marks + (r.listed ? round_up(rows * ((V + 31) / 32) * 4, 256) : 0);
    r.far = r.bits + (r.listed ? round_up(rows * tp_chunks(V) * kTpChunk * 2, 256) : 0);
    r.bytes = r.far + (r.listed > kTpNear ? round_up(rows * r.listed * sizeof(uint2), 256) : 0);
    return r;
}

int check_probs(int B, int m1, int V, int H, int K)
{
    if (B < 1 || m1 < 1 || V < 1 || H < 0 || K < 0) return LOGO_ERR_INVALID_ARG;
    if (V > LOGO_PROBS_MAX_VOCAB || m1 > 1024 || K > 4096 || static_cast<int64_t>(B) * m1 > (1 << 24) ||
        static_cast<int64_t>(B) * H > (1ll << 40))
        return LOGO_ERR_UNSUPPORTED;
    return LOGO_OK;
}

template <bool HALF>
int tp_launch(const TpParams& a, cudaStream_t st)
{
    const int lists_smem = (a.words + 3) / 4 * 32 + (a.listed <= kTpNear ? static_cast<int>(a.listed * sizeof(uint2)) : 0);
    static OncePerDevice once;
    if (once([] { return set_smem_limit(target_lists_kernel<HALF>, (LOGO_PROBS_MAX_VOCAB + 127) / 128 * 32 + kTpNear * static_cast<int>(sizeof(uint2))); }) != cudaSuccess)
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
        if (cudaLaunchKernelEx(&cfg, target_lists_kernel<HALF>, a) != cudaSuccess) return LOGO_ERR_CUDA;
        cfg.dynamicSmemBytes = 0;
    }
    cfg.gridDim = dim3(rows, a.chunks);
    cfg.blockDim = dim3(kTpThreads);
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
    uint8_t* const ws = static_cast<uint8_t*>(workspace);
    TpParams a{};
    a.logits = logits, a.temperature = temperature, a.penalty = penalty, a.history = history, a.hist_len = hist_len;
    a.n_prompt = n_prompt, a.draft = draft, a.bias_tok = bias_tok, a.bias_val = bias_val;
    a.allowed = reinterpret_cast<const uint32_t*>(allowed), a.p = p;
    a.B = B, a.m1 = m1, a.V = V, a.H = H, a.K = K;
    a.chunks = static_cast<int>(tp_chunks(V)), a.words = (V + 31) / 32;
    a.listed = history || draft || K > 0 ? room.listed : 0;
    a.pairs = a.chunks + (a.listed > 0);
    a.stats = reinterpret_cast<float2*>(ws), a.marks = reinterpret_cast<uint32_t*>(ws + room.marks);
    a.bits = reinterpret_cast<uint16_t*>(ws + room.bits), a.far = reinterpret_cast<uint2*>(ws + room.far);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return logits_bf16 ? tp_launch<true>(a, st) : tp_launch<false>(a, st);
}
