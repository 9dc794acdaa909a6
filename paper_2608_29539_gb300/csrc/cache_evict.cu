// cache_evict.cu -- cuts a sequence's cache back to its budget by accumulated
// attention weight.
//
// Every cache row of a (sequence, KV head) has a rank key: rows inside the
// recent window above all others, then the order-preserving image of the fp32
// weight; equal keys go to the lower row.  A radix select (11, 11 and 10 bits a
// pass; it ends as soon as all rows of a digit stay, which is after two passes
// unless weights are equal or nearly so) finds the key of the last row that
// stays and how many of the rows with that key do; one ordered pass lists the
// holes (rows below `end` that go) and the movers (rows at or above `end` that
// stay) in rising order, and mover i is copied into hole i.  No mover's row is any
// mover's destination, so the copies need no order, and no fewer rows could be
// moved.
//
// A CTA or a thread-block cluster takes a (sequence, KV head), each CTA an equal
// stretch of its rows: keys are formed once and stay in shared memory, the passes'
// histograms meet in distributed shared memory, and the same CTAs then move the
// rows (4 D bytes a moved row of K and V, read and written), so that the cut of a
// whole batch is one launch.  The plan is bound by latency (barriers and round
// trips): 64 pairs of 16384 rows cut to 2048 take 37 us, the plan 20 of them, in
// which HBM idles, and the moves 17 for 102 MB, 6.2 TB/s; 256 pairs of 2056 rows cut
// to 2048 take 12 us and hardly move: that time is the plan's own passes and
// barriers, four or five walks over the rows.
#include <cuda_bf16.h>

#include <algorithm>
#include <cstdint>

#include "cluster.cuh"
#include "host_common.h"
#include "logo_status.cuh"

namespace logo {
namespace {

constexpr int kEvThreads = 512;
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvMaxCluster = 8;          // portable cluster size
constexpr int kEvSmemKeys = 48 * 1024;    // keys of a CTA's stretch in shared memory; longer ones are formed anew each pass
constexpr int kEvMovesAt = 3;             // moves in flight per warp
constexpr int kEvBins = 2048;
static_assert(kEvBins == 4 * kEvThreads, "a thread scans four digits");

struct EvParams {
    logo_bf16 *k, *v;
    const float* mass;
    const int32_t *slot_pos, *seq_len, *n_seen;
    float* mass_out;
    int32_t *pos_out, *new_len;
    int32_t* lists;  // [B * Hkv][L]: holes from the front, movers from the back
    int B, L, Hkv, D, budget, recent, smem_keys;
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

template <bool CLUSTER>
__device__ __forceinline__ void evict_sync()
{
    if constexpr (CLUSTER) cluster_sync();
    else __syncthreads();
}

template <bool IN_SMEM, bool CLUSTER>
__global__ void __launch_bounds__(kEvThreads, 2) evict_kernel(EvParams p)
{
    extern __shared__ __align__(16) uint32_t sh_keys[];
    __shared__ __align__(16) int hist[2][kEvBins];  // this CTA's, two passes' worth (read by the cluster)
    __shared__ int sh_count[3];                     // ties, holes, movers of this CTA (read by the cluster)
    __shared__ int sh_warp[3][kEvWarps];            // ... of each warp
    __shared__ uint32_t sh_prefix;
    __shared__ int sh_need, sh_ties;
    const uint32_t cs = CLUSTER ? cluster_size() : 1, rank = CLUSTER ? cluster_rank() : 0;
    const int bh = blockIdx.x / cs, b = bh / p.Hkv, h = bh % p.Hkv;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int first_recent = p.n_seen[b] - p.recent;  // (in flight beside the length)
    const int len = max(0, min(p.seq_len[b], p.L)), end = min(len, p.budget);
    const int64_t base = static_cast<int64_t>(bh) * p.L;
    const float* mass = p.mass + base;
    const int32_t* pos = p.slot_pos + base;
    if (h == 0 && rank == 0 && tid == 0) p.new_len[b] = end;
    // this CTA's rows [s0, s0 + cnt)
    const int per = static_cast<int>((len + cs - 1) / cs + 3) & ~3;  // (a multiple of 4, for the loads below)
    const int s0 = min(len, per * static_cast<int>(rank)), cnt = min(len - s0, per);
    if (len <= p.budget) {  // (all CTAs of the cluster)
        for (int i = tid; i < cnt; i += kEvThreads) {
            const float m = mass[s0 + i];
            const int q = pos[s0 + i];
            p.mass_out[base + s0 + i] = m;
            p.pos_out[base + s0 + i] = q;
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) reinterpret_cast<int4*>(hist[k])[tid] = make_int4(0, 0, 0, 0);
    if constexpr (IN_SMEM) {
        int i0 = 0;
        if (((reinterpret_cast<uintptr_t>(mass + s0) | reinterpret_cast<uintptr_t>(pos + s0)) & 15) == 0) {
            // four at a time (1024 pairs of 2000 rows: 72 us a call, 84 one at a time;
            // 256 pairs of 2056: 11.9, 13.3); what is left over, or not aligned, below
            i0 = cnt & ~3;
#pragma unroll 4
            for (int i = tid * 4; i < i0; i += 4 * kEvThreads) {
                const float4 m = *reinterpret_cast<const float4*>(mass + s0 + i);
                const int4 q = *reinterpret_cast<const int4*>(pos + s0 + i);
                *reinterpret_cast<uint4*>(sh_keys + i) =
                    make_uint4(evict_key(m.x, q.x, first_recent), evict_key(m.y, q.y, first_recent),
                               evict_key(m.z, q.z, first_recent), evict_key(m.w, q.w, first_recent));
            }
        }
#pragma unroll 8
        for (int i = i0 + tid; i < cnt; i += kEvThreads) sh_keys[i] = evict_key(mass[s0 + i], pos[s0 + i], first_recent);
    }
    __syncthreads();
    auto key_at = [&](int i) { return IN_SMEM ? sh_keys[i] : evict_key(mass[s0 + i], pos[s0 + i], first_recent); };

    // ---- the key of the end-th largest, and how many rows with it stay
    uint32_t prefix = 0;
    int need = end, ties = 0;
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, buf = pass & 1;
        const uint32_t mask = pass < 2 ? 2047u : 1023u;
        const int above = pass == 0 ? 31 : pass == 1 ? 21 : 10;  // bits decided before (pass 0: none, and no key differs)
#pragma unroll 4
        for (int i0 = warp * 32; i0 < cnt; i0 += kEvThreads) {
            const int i = i0 + lane;
            const uint32_t k = i < cnt ? key_at(i) : 0u;
            const bool in = i < cnt && (pass == 0 || (k ^ prefix) >> above == 0);
            const int digit = (k >> shift) & mask;
            int same;
            const uint32_t who = __match_all_sync(0xffffffffu, in ? digit : -1, &same);
            if (same) {  // equal weights: count once
                if (in && lane == 0) atomicAdd(&hist[buf][digit], __popc(who));
            } else if (in) {
                atomicAdd(&hist[buf][digit], 1);
            }
        }
        evict_sync<CLUSTER>();  // every CTA's histogram of this pass is complete
        // thread t: digits 2047 - 4 t down to 2044 - 4 t
        int own[4] = {0, 0, 0, 0};
        const int at = kEvThreads - 1 - tid;
        if constexpr (CLUSTER) {
            int4 v[kEvMaxCluster];  // all reads in flight
#pragma unroll
            for (uint32_t r = 0; r < kEvMaxCluster; ++r)
                v[r] = r < cs ? cluster_read4(&hist[buf][4 * at], r) : make_int4(0, 0, 0, 0);
#pragma unroll
            for (uint32_t r = 0; r < kEvMaxCluster; ++r)
                own[0] += v[r].w, own[1] += v[r].z, own[2] += v[r].y, own[3] += v[r].x;
        } else {
            const int4 v = reinterpret_cast<const int4*>(hist[buf])[at];
            own[0] = v.w, own[1] = v.z, own[2] = v.y, own[3] = v.x;
        }
        reinterpret_cast<int4*>(hist[buf ^ 1])[tid] = make_int4(0, 0, 0, 0);  // the last pass's, read by all by now
        const int sum = own[0] + own[1] + own[2] + own[3];
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        if (lane == 31) sh_warp[0][warp] = incl;
        __syncthreads();
        int before = incl - sum;  // rows with a larger digit
#pragma unroll
        for (int k = 0; k < kEvWarps; ++k) before += k < warp ? sh_warp[0][k] : 0;
        if (before < need && need <= before + sum) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (before < need && need <= before + own[i]) {
                    sh_prefix = prefix | static_cast<uint32_t>(4 * at + 3 - i) << shift;
                    sh_need = need - before;
                    sh_ties = own[i];
                }
                before += own[i];
            }
        }
        __syncthreads();
        prefix = sh_prefix;
        need = sh_need;
        ties = sh_ties;
        if (need == ties) break;  // all rows with this digit stay
    }

    // ---- ordered: a warp takes a stretch of 32-row groups
    const int seg = (cnt + 32 * kEvWarps - 1) / (32 * kEvWarps) * 32;
    const int w0 = min(cnt, warp * seg), w1 = min(cnt, w0 + seg);
    const uint32_t below = (1u << lane) - 1;
    // (this CTA's count i of every warp, in sh_warp) -> first number of this warp
    // over the cluster; all threads
    auto first_of = [&](int i) {
        int mine = 0, total = 0;
#pragma unroll
        for (int k = 0; k < kEvWarps; ++k) {
            mine += k < warp ? sh_warp[i][k] : 0;
            total += sh_warp[i][k];
        }
        if (tid == 0) sh_count[i] = total;
        return mine;
    };
    auto over_cluster = [&](int i, int* all) {  // counts of the CTAs before this one; of all
        if constexpr (!CLUSTER) {
            *all = sh_count[i];
            return 0;
        }
        int c[kEvMaxCluster], mine = 0, sum = 0;
#pragma unroll
        for (uint32_t r = 0; r < kEvMaxCluster; ++r) c[r] = r < cs ? cluster_read(&sh_count[i], r) : 0;
#pragma unroll
        for (uint32_t r = 0; r < kEvMaxCluster; ++r) {
            mine += r < rank ? c[r] : 0;
            sum += c[r];
        }
        *all = sum;
        return mine;
    };
    int all, tie0 = 0;
    const bool all_ties = need == ties;  // the usual case: no equal keys to tell apart
    if (!all_ties) {
        int n = 0;
        for (int i0 = w0; i0 < w1; i0 += 32)
            n += __popc(__ballot_sync(0xffffffffu, i0 + lane < w1 && key_at(i0 + lane) == prefix));
        if (lane == 0) sh_warp[0][warp] = n;
        __syncthreads();
        tie0 = first_of(0);
        evict_sync<CLUSTER>();
        tie0 += over_cluster(0, &all);
    }
    // does row i stay?  `t`: ties before this group, moved on
    auto keeps = [&](int i, int& t) {
        const uint32_t k = i < w1 ? key_at(i) : 0u;
        if (all_ties) return i < w1 && k >= prefix;  // (prefix: the least key that stays, or a bound below it)
        const uint32_t eq = __ballot_sync(0xffffffffu, i < w1 && k == prefix);
        const bool keep = i < w1 && (k > prefix || (k == prefix && t + __popc(eq & below) < need));
        t += __popc(eq);
        return keep;
    };
    int n_hole = 0, n_move = 0, t = tie0;
#pragma unroll 4
    for (int i0 = w0; i0 < w1; i0 += 32) {
        const int i = i0 + lane;
        const bool keep = keeps(i, t);
        n_hole += __popc(__ballot_sync(0xffffffffu, i < w1 && s0 + i < end && !keep));
        n_move += __popc(__ballot_sync(0xffffffffu, keep && s0 + i >= end));
    }
    if (lane == 0) {
        sh_warp[1][warp] = n_hole;
        sh_warp[2][warp] = n_move;
    }
    __syncthreads();
    int hole = first_of(1), move = first_of(2);
    evict_sync<CLUSTER>();
    int holes;
    hole += over_cluster(1, &holes);
    move += over_cluster(2, &all);
    int32_t* lists = p.lists + base;
    const bool copies = p.mass_out != p.mass || p.pos_out != p.slot_pos;
    t = tie0;
#pragma unroll 4
    for (int i0 = w0; i0 < w1; i0 += 32) {
        const int i = i0 + lane, s = s0 + i;
        const bool keep = keeps(i, t);
        const bool is_hole = i < w1 && s < end && !keep, is_move = keep && s >= end;
        const uint32_t bh_ = __ballot_sync(0xffffffffu, is_hole), bm = __ballot_sync(0xffffffffu, is_move);
        if (is_hole) lists[hole + __popc(bh_ & below)] = s;
        if (is_move) lists[p.L - 1 - (move + __popc(bm & below))] = s;
        if (copies && keep && s < end) {
            p.mass_out[base + s] = mass[s];
            p.pos_out[base + s] = pos[s];
        }
        hole += __popc(bh_);
        move += __popc(bm);
    }
    evict_sync<CLUSTER>();  // the lists are written (and no CTA leaves while another reads its counts)

    // ---- the moves: half a warp takes K, half V, a 16-byte chunk a lane (D = 64:
    //      two moves at once)
    const int chunks = p.D / 8, per_warp = 16 / chunks;  // moves side by side
    const int half = lane / 16, sub = lane % 16 / chunks, ch = lane % chunks;
    uint4* rows = reinterpret_cast<uint4*>(half ? p.v : p.k);
    const int64_t row0 = (static_cast<int64_t>(b) * p.L * p.Hkv + h) * chunks + ch;
    const int64_t step = static_cast<int64_t>(p.Hkv) * chunks;
    // an equal stretch of the lists a warp, 32 moves at a time: a lane looks one up
    // and moves its weight and position, then all lanes move the rows
    const int n_warps = static_cast<int>(cs) * kEvWarps, w_all = static_cast<int>(rank) * kEvWarps + warp;
    const int m0 = static_cast<int>(static_cast<int64_t>(holes) * w_all / n_warps);
    const int m1 = static_cast<int>(static_cast<int64_t>(holes) * (w_all + 1) / n_warps);
    for (int c0 = m0; c0 < m1; c0 += 32) {
        const int n = min(32, m1 - c0);
        const int to = lane < n ? lists[c0 + lane] : 0, from = lane < n ? lists[p.L - 1 - (c0 + lane)] : 0;
        float m = 0.f;
        int q = 0;
        if (lane < n) {
            m = mass[from];
            q = pos[from];
        }
        for (int r = 0; r < n; r += kEvMovesAt * per_warp) {
            uint4 v[kEvMovesAt];
#pragma unroll
            for (int j = 0; j < kEvMovesAt; ++j) {
                const int i = r + j * per_warp + sub, src = __shfl_sync(0xffffffffu, from, i & 31);
                if (i < n) v[j] = rows[row0 + src * step];
            }
#pragma unroll
            for (int j = 0; j < kEvMovesAt; ++j) {
                const int i = r + j * per_warp + sub, dst = __shfl_sync(0xffffffffu, to, i & 31);
                if (i < n) rows[row0 + dst * step] = v[j];
            }
        }
        if (lane < n) {
            p.mass_out[base + to] = m;
            p.pos_out[base + to] = q;
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

// CTAs per (sequence, KV head): the least of what the barriers and exchanges of a
// cluster cost, more where SMs hold two CTAs, plus a CTA's share of the rows to
// rank and to move, in units of a row to rank (1.2 ns; moving one of D = 128 takes
// as long as ranking four).  All CTAs are to be resident at once, and clusters do
// not fill the last places of a group of SMs: 76 of four take 33.5 us where 72
// take 24.1, 48 of six 57 where 48 of five take 40.  Both tables were set by hand to
// come near the best of 1 to 8 CTAs a pair.  Measured (us) with each: 24 pairs of 6000
// rows, 5800 stay 11.9 13.5 11.6 11.7 12.2 15.5 18.2 19.9; 8 of 15822, 8781 stay 73 44
// 32 28 25 24 23 22; 40 of 6000, 5800 stay 11.8 13.5 12.0 15.4 16.0 17.1 29 32; 88 of
// 15822 (D = 64), 8781 stay 93 69 55 73 72 72 94 94.  Over 60 shapes the choice is
// within 8% of the best but for one: 16 of 15822 (D = 64) 27.2 us, 22.2 with six.
int evict_ctas(int64_t pairs, const logo_dims& d, int budget)
{
    constexpr int64_t kCost[] = {0, 3500, 2600, 2600, 3000, 3300, 3800, 4200};
    constexpr int64_t kCrowd[] = {0, 3000, 4000, 4000, 4100, 4900, 5100, 5300};
    static_assert(sizeof kCost / sizeof *kCost == kEvMaxCluster, "a cost for each cluster size");
    const int64_t sms = device_sm_count();
    const int64_t work = d.T + d.D / 32ll * std::max(0, std::min(budget, d.T - budget));
    int best = 1;
    int64_t least = work;
    for (int cs = 2; cs <= kEvMaxCluster && pairs * cs <= 2 * sms * (cs <= 4 ? 95 : 83) / 100; ++cs) {
        const int64_t crowd = pairs * cs > sms * 9 / 10 ? kCrowd[cs - 1] : 0;
        const int64_t cost = kCost[cs - 1] + crowd + work / cs;
        if (cost < least) {
            least = cost;
            best = cs;
        }
    }
    return best;
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
    if (new_len == seq_len || new_len == n_seen) return LOGO_ERR_INVALID_ARG;  // CTAs that start later read both
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
    const int64_t pairs = static_cast<int64_t>(dims.B) * dims.Hkv;
    const int cs = evict_ctas(pairs, dims, budget);
    const int per = ((dims.T + cs - 1) / cs + 3) & ~3;
    p.smem_keys = per <= kEvSmemKeys ? per : 0;
    auto kernel = p.smem_keys == 0 ? evict_kernel<false, true> : cs > 1 ? evict_kernel<true, true> : evict_kernel<true, false>;
    if (p.smem_keys > 8000) {  // more than the default limit of dynamic shared memory allows
        if (set_smem_limit(kernel, kEvSmemKeys * 4) != cudaSuccess) return LOGO_ERR_CUDA;
    }
    cudaLaunchAttribute attr{};
    const cudaLaunchConfig_t cfg = cluster_config(static_cast<unsigned>(pairs) * cs, kEvThreads, cs, p.smem_keys * 4,
                                                  static_cast<cudaStream_t>(stream), &attr);
    return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? LOGO_OK : LOGO_ERR_CUDA;
}
