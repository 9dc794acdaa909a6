"""The shares of the prefix attention's line of key tiles (csrc/prefix_sched.h), on
the CPU: which CTAs hold parts of a run follows from the line alone, so the join
reads nothing that a CTA writes only when it gets to the run's end (a wait that
gave up would leave it undefined).  Compared with a walk over every CTA's share,
tile by tile, and with the definition of a unit's owner in exact arithmetic."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_29539_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <random>
#include <vector>
#include "prefix_sched.h"
using namespace logo;

static int bad = 0;
#define CHECK(x) do { if (!(x) && bad++ < 5) std::printf("line %d: %s\n", __LINE__, #x); } while (0)

static PaSched line(int total, int n)
{
    PaSched s{};
    s.total = total;
    s.n = n;
    s.rate = static_cast<float>(n) / static_cast<float>(total);
    return s;
}

static int owner(const PaSched& s, long long u)  // the last c with floor(total c / n) <= u
{
    int c = 0;
    while (c + 1 < s.n && static_cast<long long>(s.total) * (c + 1) / s.n <= u) ++c;
    return c;
}

int main()
{
    std::mt19937 rng(1);
    auto pick = [&](int lo, int hi) { return lo + static_cast<int>(rng() % static_cast<unsigned>(hi - lo + 1)); };
    // runs of random lengths, their tiles given out share by share
    for (int rep = 0; rep < 400; ++rep) {
        std::vector<int> tiles(pick(1, 60)), first;
        int total = 0;
        const int longest = rep % 3 == 0 ? 1 : rep % 3 == 1 ? 6 : 300;
        for (int& t : tiles) {
            t = pick(1, longest);
            first.push_back(total);
            total += kRunCost + t;
        }
        const int ctas[] = {1, 2, 7, 148, 152, 160};
        const int n = std::min(ctas[rep % 6], total);
        const PaSched s = line(total, n);
        std::vector<int> c0(tiles.size(), -1), c1(tiles.size(), -1);
        std::size_t run = 0;
        for (int c = 0; c < n; ++c) {
            CHECK(share_start(s, c) < share_start(s, c + 1));
            for (int u = share_start(s, c); u < share_start(s, c + 1); ++u) {
                while (u >= first[run] + kRunCost + tiles[run]) ++run;
                if (u < first[run] + kRunCost) continue;
                if (c0[run] < 0) c0[run] = c;
                c1[run] = c;
            }
        }
        CHECK(share_start(s, n) == total);
        for (std::size_t k = 0; k < tiles.size(); ++k) {
            const PaRun r = run_of(s, first[k], tiles[k]);
            CHECK(r.c0 == c0[k] && r.n == c1[k] - c0[k] + 1);
        }
    }
    // long lines: units around every share's ends, and random ones
    for (int total : {1, 2, 151, 152, 153, 16777215, 16777217, 123456789, 805306368, 1073741823, 2147483646})
        for (int n : {1, 3, 148, 152, 160, 1000}) {
            if (n > total) continue;
            const PaSched s = line(total, n);
            for (int c = 0; c <= n; ++c)
                for (long long u = share_start(s, c) - 3ll; u <= share_start(s, c) + 3ll; ++u)
                    if (u >= 0 && u < total) CHECK(share_owner(s, static_cast<int>(u)) == owner(s, u));
            for (int i = 0; i < 200; ++i) {
                const int u = static_cast<int>(rng() % static_cast<unsigned>(total));
                CHECK(share_owner(s, u) == owner(s, u));
            }
        }
    std::printf("%d wrong\n", bad);
    return bad != 0;
}
"""


def test_owners_and_runs(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "sched.cpp", tmp_path / "sched"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


@pytest.mark.gpu
@pytest.mark.parametrize("P,n", [(0, 1), (700, 3)])
def test_nothing_in_the_workspace_is_taken_over(P, n):
    """The same bits whatever an earlier call has left in the workspace."""
    import torch

    import test_gpu_prefix_attn as T
    from paper_2608_29539_gb300 import logo as Lg
    B, Hq, Hkv, D, L = 7, 8, 2, 128, 400
    q, kp, vp, kc, vc = (t.cuda() for t in T._inputs(B, n, Hq, Hkv, D, P, L, 2))
    pos, cu, ns, rows = T._pack(T._z(B, n, 0.8, P))
    lens = torch.tensor([400, 3, 0, 129, 256, 17, 300], dtype=torch.int32, device="cuda")
    mass = torch.rand(B, Hkv, L, device="cuda")
    ws = Lg.logo_decode_prefix_workspace(q, kp if P else None, kc, True)
    outs = []
    for fill in (0x00, 0xff, 0x7f):
        ws.fill_(fill)
        o, lse, m = torch.zeros(B * n, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(Hq, B * n, device="cuda"), \
            torch.zeros_like(mass)
        Lg.logo_decode_prefix_attn(q, kp if P else None, vp if P else None, kc, vc, lens, pos.cuda(), cu.cuda(), ns.cuda(),
                                   mass_in=mass, mass_out=m, o_c=o, lse_c=lse, workspace=ws)
        outs.append((o, lse, m))
    torch.cuda.synchronize()
    assert Lg.logo_get_device_status() == 0
    assert bool((outs[0][0][:len(rows)] != 0).any())
    for other in outs[1:]:
        for a, b in zip(outs[0], other):
            assert torch.equal(a, b)
