// prefix_sched.h -- how the prefix attention's key tiles are shared out among
// CTAs.  Plain arithmetic, the same on host and device.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define LOGO_SCHED_FN __host__ __device__ __forceinline__
#else
#define LOGO_SCHED_FN inline
#endif

namespace logo {

// A run's start and end (its Q, the join of the warps) are counted as this many
// tiles when the shares are cut (with 1, 2 and 3: 16 sequences of 8192 tokens, 32
// rows 51.6, 49.8 and 50.0 us a call; 256 rows, 2048 tokens 120, 110 and 115; 128
// sequences of 512 tokens, four rows 70.2, 70.8 and 71.9).
constexpr int kRunCost = 2;

// All runs of a call (the tiles of one segment, KV head and row tile) lie on one
// line: the prefix's KV heads, then the own caches' (sequence, KV head, row
// tile).  A run takes kRunCost + tiles units, its tiles the last ones.  CTA c of
// n takes the units [total c / n, total (c + 1) / n).
struct PaSched {
    int K;      // length of the prefix part; 0 if there is none, or if it is wide
    int total;  // length of the line
    int N, PT, n, wide, rt_pre;  // rt_pre: row tiles of a prefix that is not wide
    float rate;                  // n / total
};

// A row tile's keys of one segment and KV head: the first share that holds some
// of them, and the number of shares.
struct PaRun {
    int c0, n;
};

LOGO_SCHED_FN int share_start(const PaSched& s, int c)
{
    return static_cast<int>(static_cast<long long>(s.total) * c / s.n);
}

// The CTA whose share holds unit u: the last c with floor(total c / n) <= u, that
// is total c < (u + 1) n (n <= total: no share is empty).  The quotient in fp32 is
// off by less than one as long as n < 2^20 (four roundings), so the share that it
// names is right or a neighbour of the right one.
LOGO_SCHED_FN int share_owner(const PaSched& s, int u)
{
    const long long total = s.total, at = (u + 1ll) * s.n;
    int c = static_cast<int>(static_cast<float>(u + 1) * s.rate);
    if (total * c >= at) --c;
    else if (total * (c + 1) < at) ++c;
    return c;
}

// The shares of the run whose first unit is `first`.  It follows from the line
// alone, whether or not the CTAs that work on the run got to its end.
LOGO_SCHED_FN PaRun run_of(const PaSched& s, int first, int tiles)
{
    const int c0 = share_owner(s, first + kRunCost);
    return PaRun{c0, share_owner(s, first + kRunCost + tiles - 1) - c0 + 1};
}

}  // namespace logo
