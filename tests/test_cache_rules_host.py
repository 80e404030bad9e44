"""How attention over the paged cache cuts chunks of prompts (csrc/launch_rules.h), compiled for the host."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HARNESS = r"""
#include "launch_rules.h"
using namespace ifv2::rules;
extern "C" int pps(long long tiles, int pages) { return tile_splits(tiles, pages).pps; }
extern "C" int pays(long long tiles, int pages, long long group_pages) { return tile_pays(tiles, pages, group_pages); }
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    src, lib = d / "rules.cpp", d / "rules.so"
    src.write_text(HARNESS)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2509_24663_amd", "csrc"), str(src), "-o", str(lib)])
    L = ctypes.CDLL(str(lib))
    L.pps.argtypes = [ctypes.c_longlong, ctypes.c_int]
    L.pays.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong]
    return L


def test_splits_cover_all_pages_within_their_bounds(rules):
    for tiles in (1, 2, 3, 18, 64, 172, 255, 256, 257, 1000, 1025, 10 ** 6):
        for pages in (1, 2, 7, 64, 544, 2048, 4097):
            pps = rules.pps(tiles, pages)
            splits = -(-pages // pps)
            assert 1 <= pps <= pages and splits <= 64
            assert splits == 1 or tiles * splits <= 1024       # what the scratch query counts on


def test_tiles_of_one_round_are_not_split_and_few_are(rules):
    assert rules.pps(256, 544) == 544              # 2048 tokens of 16 heads on 2: a workgroup on each CU
    assert rules.pps(2, 516) <= 16                 # 16 tokens: the keys are what is shared out
    assert rules.pps(10 ** 5, 500) == 500


def test_where_the_tile_kernel_pays(rules):
    assert not rules.pays(0, 0, 0)
    assert rules.pays(256, 544, 2048 * 2 * 544) and rules.pays(2, 516, 16 * 2 * 516)
    assert not rules.pays(2, 11, 16 * 2 * 11)      # a short context: launches are what it costs
