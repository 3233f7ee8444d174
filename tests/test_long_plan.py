"""The launch plans of the operators for long caches, compiled from their header without CUDA."""
import subprocess

import pytest

import paper_2406_09297_gb300.build as build

DRIVER = r"""
#include <cstdio>
#include <vector>
#include "mlkv_plan.h"

int main()
{
    int n, sms, d, chunks;
    double bytes;
    while (std::scanf("%d %d %d %d %lf", &n, &sms, &d, &chunks, &bytes) == 5) {
        std::vector<int> n_kt(n), pairs(n);
        for (int &x : n_kt)
            if (std::scanf("%d", &x) != 1)
                return 1;
        for (int &x : pairs)
            if (std::scanf("%d", &x) != 1)
                return 1;
        const mlkv::PrefixPlan p = mlkv::plan_prefix(n_kt.data(), pairs.data(), n, sms, d, bytes, chunks);
        std::printf("%d %d %d %.9g\n", p.kc, p.sms, p.beside ? 1 : 0, p.us);
    }
    return 0;
}
"""

SMS, CHUNKS = 152, 256


def compiled(tmp, name, source):
    src, exe = str(tmp / f"{name}.cpp"), str(tmp / name)
    with open(src, "w") as f:
        f.write(source)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", build.CSRC, "-I", build.INCLUDE, "-o", exe, src], check=True)
    return exe


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = compiled(tmp_path_factory.mktemp("plan"), "plans", DRIVER)

    def run(cases):
        """[(n_kt, pairs, d, bytes)] -> [(kc, sms, beside, us)]"""
        text = "".join(f"{len(k)} {SMS} {d} {CHUNKS} {b} {' '.join(map(str, k))} {' '.join(map(str, p))}\n"
                       for k, p, d, b in cases)
        out = subprocess.run([exe], input=text, check=True, capture_output=True, text=True).stdout.split("\n")
        return [(int(a), int(s), bool(int(c)), float(u)) for a, s, c, u in (x.split() for x in out if x)]
    return run


def _case(prefixes, per, tokens, g, G, d, own=256):
    """`prefixes` of `tokens` positions, `per` sequences each with `own` positions."""
    pairs = -(-per // (2 * (128 // G))) * g
    return [-(-tokens // 128)] * prefixes, [pairs] * prefixes, d, 4.0 * g * d * own * per * prefixes


def test_every_shape_has_a_plan(plans):
    """Whatever the number of units: a shape that 1024 sequences allow is planned, within what a unit's word holds."""
    cases = [_case(n, per, tokens, g, G, d)
             for n in (1, 2, 7, 40, 76, 80, 200, 512, 1024) for per in (1, 2, 12, 64, 1024) if n * per <= 1024
             for tokens in (1, 129, 8192, 1000000) for g, G in ((1, 12), (8, 4), (12, 1), (64, 16), (255, 1))
             for d in (64, 128)]
    assert len(cases) > 800
    for (n_kt, pairs, d, _), (kc, sms, beside, us) in zip(cases, plans(cases)):
        assert us < 1e20, (n_kt[0], len(n_kt), pairs[0], d)
        assert 1 <= kc <= n_kt[0] and -(-n_kt[0] // kc) <= CHUNKS
        assert 1 <= sms <= SMS and (not beside or sms <= SMS - 8)
        # no less than the tiles take on all the SMs (0.95 us each of 64 channels, 1.5 of 128)
        assert us >= sum(n_kt) * pairs[0] / SMS * (0.95 if d == 64 else 1.5)


def test_uneven_prefixes(plans):
    cases = [([x % 70 * 9 for x in range(n)], [(x % 3) * 8 for x in range(n)], 128, 1e6) for n in (5, 50, 500, 1000)]
    for (n_kt, _, _, _), (kc, _, _, us) in zip(cases, plans(cases)):
        assert us < 1e20 and 1 <= kc <= max(n_kt)


@pytest.mark.parametrize("g,G,d,tokens,per", [(8, 4, 128, 8192, 12), (12, 1, 64, 4000, 10), (4, 3, 64, 16384, 12)])
def test_one_prefix_more_takes_little_more(plans, g, G, d, tokens, per):
    """Twelve sequences a prefix, 8 KV heads of 128: 76 prefixes 649 us, 80 once were 2449, end to end."""
    us = [p[3] for p in plans([_case(n, per, tokens, g, G, d) for n in range(20, 1024 // per + 1)])]
    work = range(20, 1024 // per + 1)
    for a, b, n in zip(us, us[1:], work):
        # at most the new prefix's part, and a wave of units more
        assert b <= a * (n + 1) / n + 1.2 * us[0], (n, a, b)


BLOCKS = r"""
#include <chrono>
#include <cstdio>
#include <cstring>
#include <random>
#include <vector>
#include "mlkv_plan.h"

using Order = std::vector<long long>;

static Order blocks_of(const std::vector<int> &n, const std::vector<int> &pre, bool none)
{
    Order o;
    mlkv::for_query_blocks(static_cast<int>(n.size()), n.data(), none ? nullptr : pre.data(), [&](int beta, int qb) {
        o.push_back(beta * 1000000LL + qb);
        return true;
    });
    return o;
}

// as the order is defined
static Order plain(const std::vector<int> &n, const std::vector<int> &pre)
{
    Order o;
    int most = 0;
    for (size_t i = 0; i < n.size(); ++i)
        most = std::max(most, n[i] + pre[i]);
    for (int seen = most - 1; seen >= 0; --seen)
        for (size_t i = 0; i < n.size(); ++i)
            if (seen >= pre[i] && seen - pre[i] < n[i])
                o.push_back(static_cast<long long>(i) * 1000000LL + seen - pre[i]);
    return o;
}

int main()
{
    std::mt19937 rng(3);
    for (int k = 0; k < 3000; ++k) {
        const int b = 1 + rng() % (k % 50 == 0 ? 1024 : 12), most = 1 + rng() % 9, far = 1 + rng() % (k % 3 ? 5 : 400);
        std::vector<int> n(b), pre(b);
        for (int i = 0; i < b; ++i) {
            n[i] = 1 + rng() % most;
            pre[i] = rng() % 4 ? rng() % far : 0;
        }
        if (blocks_of(n, pre, false) != plain(n, pre))
            return std::printf("order %d\n", k), 1;
        if (blocks_of(n, std::vector<int>(), true) != plain(n, std::vector<int>(b, 0)))
            return std::printf("order without prefixes %d\n", k), 1;
    }
    int visits = 0;   // a visit that says no is the last
    const int n2[2] = {3, 2}, pre2[2] = {1, 7};
    const bool all = mlkv::for_query_blocks(2, n2, pre2, [&](int, int) { return ++visits < 3; });
    if (all || visits != 3)
        return std::printf("stop\n"), 1;
    // 1024 prompts of two blocks behind prefixes of one block, and of 7813 (a million positions)
    double us[2];
    for (int far = 0; far < 2; ++far) {
        std::vector<int> n(1024, 2), pre(1024, far ? 7813 : 1);
        pre[5] = 0;
        us[far] = 1e30;
        for (int r = 0; r < 9; ++r) {
            const auto t0 = std::chrono::steady_clock::now();
            long long sum = 0;
            mlkv::for_query_blocks(1024, n.data(), pre.data(), [&](int beta, int qb) { sum += beta ^ qb; return true; });
            const double t = std::chrono::duration<double, std::micro>(std::chrono::steady_clock::now() - t0).count();
            us[far] = std::min(us[far], t + (sum == 42 ? 1e-9 : 0));
        }
    }
    std::printf("%g %g\n", us[0], us[1]);
    return 0;
}
"""


def test_query_blocks_of_prompts(tmp_path):
    """Their order, and that a far prefix costs the host nothing: the work is the prompts' own."""
    out = subprocess.run([compiled(tmp_path, "blocks", BLOCKS)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
    near, far = (float(x) for x in out.stdout.split())
    assert far <= 5 * near + 50, (near, far)
