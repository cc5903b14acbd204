"""Which tokens of a cache in pages a tile of rows walks (csrc/bsa_paged_plan.h), compiled for the
host: every token that a query sees once, nothing outside the tables and pages."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_16429_amd", "csrc")

SOURCE = """
#include "bsa_paged_plan.h"
using namespace bsa::paged;
template <int KT>
static int walk(int prefix, int ql, int kl, int left, int sinks, int first, int last, int32_t* out)
{
    Shape s = {};
    s.left = left;
    s.sinks = sinks;
    const Tiles<KT> tiles(s, Sequence{ql, kl, prefix}, first, last);
    for (int t = 0; t < tiles.count; ++t) {
        const Tile x = tiles[t];
        out[4 * t] = x.at;
        out[4 * t + 1] = x.count;
        out[4 * t + 2] = x.token;
        out[4 * t + 3] = x.shared;
    }
    return tiles.count;
}
extern "C" int walk_of(int kt, int prefix, int ql, int kl, int left, int sinks, int first, int last,
                       int32_t* out)
{
    return kt == 32 ? walk<32>(prefix, ql, kl, left, sinks, first, last, out)
                    : walk<64>(prefix, ql, kl, left, sinks, first, last, out);
}
extern "C" int page(int pages, int shift, const int32_t* table, int at, int count)
{
    Shape s = {};
    s.pages = pages;
    s.page_shift = shift;
    return page_of(s, table, at, count);
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, lib = d / "plan.hip", d / "plan.so"
    src.write_text(SOURCE)
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950",
                    "--offload-host-only", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC,
                    "-I", os.path.join(ROOT, "include"), str(src), "-o", str(lib)], check=True)
    return ctypes.CDLL(str(lib))


UNBOUNDED = 1 << 30


@pytest.mark.parametrize("seed", range(8))
@pytest.mark.parametrize("kt", [32, 64])
def test_every_visible_token_once(plan, kt, seed):
    rng = random.Random(seed)
    out = np.empty((4096, 4), dtype=np.int32)
    for _ in range(300):
        P = rng.choice([0, 0, 1, 31, 32, 33, 64, 100, rng.randint(0, 400)])
        kl = rng.choice([0, 1, 31, 32, 33, 64, rng.randint(0, 400)])
        ql = rng.choice([1, 1, 2, rng.randint(1, 70)])
        left = rng.choice([UNBOUNDED, UNBOUNDED, 0, 1, 31, 32, 63, rng.randint(0, 500)])
        sinks = rng.choice([0, 0, 1, 4, 32, 33, 100, 1000, 2**31 - 1])
        i0 = rng.randint(0, ql - 1)
        i1 = rng.randint(i0, ql - 1)
        p0 = P + kl - ql
        n = plan.walk_of(kt, P, ql, kl, left, sinks, p0 + i0, p0 + i1, out.ctypes.data_as(ctypes.c_void_p))
        walked = []
        for at, count, token, shared in out[:n].tolist():
            assert at % kt == 0 and 0 <= at < count
            assert count == (P if shared else kl) and token == (at if shared else P + at)
            walked += range(token, token + min(kt, count - at))
        assert len(set(walked)) == len(walked) and set(walked) <= set(range(P + kl))
        for i in {i0, i1, rng.randint(i0, i1)}:
            p = p0 + i
            seen = {j for j in range(max(0, p + 1)) if j >= p - left or j < sinks}
            assert seen <= set(walked)
        # nothing far away either: at most two ends of each part's two runs are partly unseen
        any_seen = {j for i in range(i0, i1 + 1) for j in range(max(0, p0 + i + 1))
                    if j >= p0 + i - left or j < sinks}
        assert len(walked) <= len(any_seen) + 8 * kt


def test_extreme_lengths(plan):
    """The largest sizes: nothing overflows."""
    most = (1 << 29) - 1
    out = np.empty((64, 4), dtype=np.int32)
    ptr = out.ctypes.data_as(ctypes.c_void_p)
    p = 2 * most - 1
    assert plan.walk_of(32, most, 1, most, 100, 4, p, p, ptr) == 1 + 4
    assert plan.walk_of(32, most, most, 0, UNBOUNDED, 2**31 - 1, 0, 0, ptr) == 1
    assert plan.walk_of(32, 0, most, 0, UNBOUNDED, 0, -most, -1, ptr) == 0


def test_pages_that_are_none(plan):
    table = np.array([3, -1, 7, 8, 2**31 - 1, -2**31, 0], dtype=np.int32)
    ptr = table.ctypes.data_as(ctypes.c_void_p)
    got = [plan.page(8, 3, ptr, at, 50) for at in range(56)]
    want = [3] * 8 + [-1] * 8 + [7] * 8 + [-1] * 24 + [0] * 2 + [-1] * 6
    assert got == want
