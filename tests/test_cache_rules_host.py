"""How attention over the paged cache cuts chunks of prompts (csrc/launch_rules.h), compiled for the host."""
import ctypes
import random
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HARNESS = r"""
#include "launch_rules.h"
using namespace ifv2::rules;
extern "C" int pps(int d, int small, long long tiles, int pages, long long sum) { return tile_splits(tile_size(d, small), tiles, pages, sum).pps; }
extern "C" double us(int d, int small, long long tiles, int pages, long long sum) { return tile_splits(tile_size(d, small), tiles, pages, sum).us; }
extern "C" double unit(int d, int pages, long long sum) { return unit_us(d, pages, sum); }
static PageWork work(int n, const long long *units, const int *pages) {
    PageWork w;
    for (int i = 0; i < n; ++i) w.add(units[i], pages[i], units[i] * pages[i]);
    return w;
}
extern "C" int unit_pages(int n, const long long *units, const int *pages, int d, int fp32, int bytes, long long least) {
    return unit_pps(work(n, units, pages), d, fp32, bytes, least);
}
extern "C" long long unit_groups(int n, const long long *units, const int *pages, int pps, int two) {
    PageWork w = work(two ? n / 2 : n, units, pages);
    if (two) w.add(work(n - n / 2, units + n / 2, pages + n / 2));
    return w.groups(pps);
}
extern "C" int groups(int d, int small) { return tile_size(d, small).groups; }
extern "C" int most_groups() { return kMostTileGroups; }
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    src, lib = d / "rules.cpp", d / "rules.so"
    src.write_text(HARNESS)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2509_24663_amd", "csrc"), str(src), "-o", str(lib)])
    L = ctypes.CDLL(str(lib))
    for f in (L.pps, L.us):
        f.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong]
    L.unit.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_longlong]
    L.unit_pages.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_longlong), ctypes.POINTER(ctypes.c_int), *[ctypes.c_int] * 3, ctypes.c_longlong]
    L.unit_groups.restype = ctypes.c_longlong
    L.us.restype = L.unit.restype = ctypes.c_double
    return L


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("small", [0, 1])
def test_splits_cover_all_pages_within_their_bounds(rules, d, small):
    for tiles in (1, 2, 3, 18, 64, 172, 255, 256, 257, 1000, 1025, 10 ** 6):
        for pages in (1, 2, 7, 64, 544, 2048, 4097):
            for sum_ in (tiles * pages, tiles * (pages + 1) // 2):
                pps = rules.pps(d, small, tiles, pages, sum_)
                splits = -(-pages // pps)
                assert 1 <= pps <= pages and splits <= 64
                assert splits == 1 or tiles * splits * rules.groups(d, small) <= rules.most_groups()       # what the scratch query counts on


def _work(units, pages):
    return len(units), (ctypes.c_longlong * len(units))(*units), (ctypes.c_int * len(pages))(*pages)


def test_pages_of_a_workgroup(rules):
    def pps(units, pages, d=128, fp32=0, bytes_=1, least=0):
        return rules.unit_pages(*_work(units, pages), d, fp32, bytes_, least)

    rng = random.Random(1)
    for _ in range(300):
        units = [rng.choice([1, 2, 8, 400]) for _ in range(rng.choice([1, 5, 40]))]
        pages = [int(30000 ** rng.random()) for _ in units]
        if rng.random() < 0.3:
            pages = [pages[0]] * len(pages)
        total = sum(u * p for u, p in zip(units, pages))
        least = -(-total // 2048)
        x = pps(units, pages, rng.choice([64, 128]), rng.randrange(2), rng.choice([1, 2]), least)
        assert x >= least and x >= 4 and x % 4 == 0
        exact = sum(u * -(-p // x) for u, p in zip(units, pages))
        for two in (0, 1):
            n = rules.unit_groups(*_work(units, pages), x, two)
            assert n == exact if len(set(pages)) <= 16 else abs(n - exact) <= sum(units)
        assert sum(u * -(-p // x) for u, p in zip(units, pages) if p > x) <= 4096       # what the scratch query counts on
    assert pps([2], [516]) == 8 and pps([2], [8000]) >= 32                          # long contexts: fewer, longer splits
    assert pps([4], [12]) == 12 and pps([4], [24]) < 24                             # short ones: one launch
    assert pps([4], [8], 128, 1, 4) == 4 and pps([4], [24], 64) == 24


def test_tiles_of_one_round_are_not_split_and_few_are(rules):
    assert rules.pps(128, 0, 256, 544, 256 * 544) == 544              # 2048 tokens of 16 heads on 2: a workgroup on each CU
    assert rules.pps(128, 0, 2, 516, 2 * 516) <= 16 and rules.pps(128, 1, 4, 516, 4 * 516) <= 16      # 16 tokens: the keys are what is shared out
    assert rules.pps(128, 0, 10 ** 5, 500, 10 ** 5 * 500) == 500


def test_which_kernel_and_which_tiles(rules):
    def best(d, large, small, pages, unit):
        us = [rules.us(d, 0, large, pages, large * pages), rules.us(d, 1, small, pages, small * pages), rules.unit(d, pages, unit)]
        return us.index(min(us))

    assert best(128, 256, 512, 544, 4096 * 544) == 0          # 2048 tokens of 16 heads on 2 over 34816
    assert best(128, 38, 76, 21, 600 * 21) == 1               # 300 over 1300
    assert best(64, 2, 6, 107, 36 * 107) in (1, 2)            # 72 of 4 heads on 1, 2 KV heads, over 6800: as good
    assert best(128, 2, 2, 516, 8 * 516) == 1                 # 4 tokens over 33000
    assert best(128, 4, 4, 11, 32 * 11) == 2                  # a few tokens over a short context: launches are what it costs
