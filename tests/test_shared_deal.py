"""Host-side walk (no GPU) of how decode_shared deals its work out: every unit of shared keys is taken once, and neither kind of keys is left to
a few workgroups where the other has many."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

from paper_2509_16495_amd import build as BLD

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++ to compile the functions for the host")

SOURCE = r"""
#include "shared_deal.h"
#include <algorithm>
#include <vector>
using namespace shiftattn::shared_deal;
// The plan of a batch: group i has steps[i] steps of keys in common and cols[i] columns of each of hkv KV heads; `own` is the other keys' weight.
// Returns in out: units, units that are not taken exactly once, workgroups that take shared keys; and in times: the longest of the workgroups' loads of
// either kind, the longest unit, all units' weight.
extern "C" void walk(const int* steps, const int* cols, int groups, int hkv, float own, int range_min, int* out, double* times) {
    float shared = 0;
    for (int g = 0; g < groups; ++g) shared += static_cast<float>(steps[g]) * hkv * tiles_of(cols[g]) * cost_of(cols[g]);
    const int range = range_of(shared, own);
    std::vector<int> units(groups + 1, 0);
    std::vector<uint32_t> line(groups + 1, 0), each(groups, 0);
    uint32_t longest = 0;
    for (int g = 0; g < groups; ++g) {
        const int ranges = steps[g] > 0 ? ranges_of(steps[g], cols[g], range, range_min) : 0, n = ranges * hkv * tiles_of(cols[g]);
        if (n) each[g] = among(range_steps(steps[g], ranges), cols[g]);
        longest = std::max(longest, each[g]);
        units[g + 1] = units[g] + n, line[g + 1] = line[g] + n * each[g];
    }
    const int all = units[groups];
    int n_p = all;
    if (!one_each(all, shared, own)) n_p = workgroups_of(all, static_cast<float>(line[groups]), static_cast<float>(longest), own);
    std::vector<int> taken(all, 0);
    double most = 0;
    auto unit_at = [&](uint32_t x) {
        for (int g = 0; g < groups; ++g)
            if (line[g] < x && line[g + 1] >= x) return units[g] + units_before(x, line[g], each[g], units[g + 1] - units[g]);
        return 0;
    };
    for (int wg = 0; wg < n_p; ++wg) {
        const int first = n_p < all ? unit_at(first_of(line[groups], n_p, wg)) : wg, end = n_p < all ? unit_at(first_of(line[groups], n_p, wg + 1)) : wg + 1;
        double load = 0;
        for (int u = first; u < end; ++u) {
            if (u >= 0 && u < all) ++taken[u];
            load += each[std::upper_bound(units.begin(), units.end(), u) - units.begin() - 1];
        }
        most = std::max(most, load);
    }
    out[0] = all, out[1] = 0, out[2] = n_p;
    for (const int n : taken) out[1] += n != 1;
    times[0] = most, times[1] = own / (kWorkgroups - n_p), times[2] = longest, times[3] = line[groups];
}
extern "C" int does_pay(int blocks, int members, int cols) { return pays(blocks, members, cols); }
"""


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("deal"))
    src, lib = os.path.join(d, "deal.cpp"), os.path.join(d, "deal.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.check_call(["g++", "-std=c++20", "-O1", "-shared", "-fPIC", "-I", BLD.CSRC, src, "-o", lib])
    return ctypes.CDLL(lib)


@pytest.fixture(scope="module")
def walk(built):
    f = built.walk

    def call(groups, hkv, G, range_min=2, alone=0):
        """groups: (tokens in common, tokens of each member's own) of every group; alone: tokens of sequences of no group."""
        steps = (ctypes.c_int * len(groups))(*[pre // 16 // 4 + (pre // 16 % 4 > 0) for pre, _ in groups])
        cols = (ctypes.c_int * len(groups))(*[len(tails) * G for _, tails in groups])
        own = float(sum(-(-(t + pre % 16) // 32) for pre, tails in groups for t in tails) + -(-alone // 32)) * hkv
        out, times = (ctypes.c_int * 3)(), (ctypes.c_double * 4)()
        f(steps, cols, len(groups), hkv, ctypes.c_float(own), range_min, out, times)
        units, missed, n_p = out
        shared, mine, longest, line = times
        assert missed == 0 and (units == 0 or 1 <= n_p <= min(units, 508))
        return max(shared, mine), (line + own) / 512, longest, n_p
    return call


# 512 workgroups, one for every unit, left four to the sequences' own keys of the first, the fourth and the fifth batch
@pytest.mark.parametrize("groups,size,pre,suf,hkv,G", [(64, 2, 1000, 1000, 8, 4), (60, 2, 1000, 1000, 8, 4), (32, 4, 1000, 1000, 8, 4), (64, 2, 64, 4000, 8, 8), (512, 2, 64, 4000, 1, 8),
                                                       (256, 2, 1000, 1000, 1, 8), (20, 4, 512, 1000, 8, 8), (128, 2, 200, 1500, 1, 8)])
def test_many_small_groups(walk, groups, size, pre, suf, hkv, G):
    time, even, longest, _ = walk([(pre, [suf] * size)] * groups, hkv, G)
    assert time <= 1.25 * even + longest


def test_any_batch(walk):
    """With m workgroups for shared keys, where shared / m + longest meets own / (512 - m), both are (all work + m longest) / 512; m is rounded down,
    from 1 on by less than half."""
    rng = random.Random(4)
    log = lambda lo, hi: min(hi, max(lo, int(lo * (hi / lo) ** rng.random())))
    for _ in range(3000):
        hkv, G = rng.choice([(1, 8), (1, 16), (2, 8), (8, 4), (8, 8), (4, 1)])
        n, members, pre, suf = log(1, min(512, 1024 // hkv)), log(2, 256), log(16, 100000), log(1, 5000)
        members = max(2, min(members, 1024 // hkv // n))
        groups = [(log(16, pre) if rng.random() < 0.8 else 0, [log(1, suf) for _ in range(rng.randint(2, members))]) for _ in range(n)]
        time, even, longest, n_p = walk(groups, hkv, G, alone=rng.choice([0, log(1, 100000)]))
        assert time <= 2 * (even + longest) + 1, (groups, hkv, G, n_p)


def test_few_units_have_a_workgroup_each(walk):
    """One prompt, as many ranges as its part of the workgroups: what follows of the rule for more units does not change it."""
    time, even, longest, n_p = walk([(16384, [700] * 61)], 1, 8)
    assert time <= even + longest and n_p > 250
    time, even, longest, n_p = walk([(32768, [1100] * 256)], 1, 8)
    assert time <= even + longest and n_p > 300


def test_what_pays(built):
    """A group shares where that saves more than its tiles take: long prompts, or many members; never no keys."""
    pays = lambda tokens, members, G: bool(built.does_pay(tokens // 16, members, members * G))
    assert pays(1000, 2, 4) and pays(30000, 2, 16) and pays(64, 20, 1) and pays(2000, 64, 8)
    assert not pays(64, 2, 8) and not pays(16, 4, 4) and not pays(15, 256, 8) and not pays(0, 1024, 1)
    for members in (2, 3, 17, 256):
        for G in (1, 8, 16):
            at = [pays(16 * b, members, G) for b in range(2000)]
            assert at == sorted(at) and at[-1], (members, G)      # once it pays, more tokens do too
