"""The launch plans of the operators for long caches, compiled from their header without CUDA."""
import os
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
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", build.CSRC, "-o", exe, src], check=True)
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
