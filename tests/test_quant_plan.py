"""How the dense layer in 8 bits cuts a product and the workspace it asks for, by the host code itself (built here, no GPU)."""
import ctypes
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2002_02645_amd", "csrc")
SOURCE = """
#include "quant_plan.h"
extern "C" long long room(long long b, long long m, long long d_pad) { return (long long)fz::quant_room(b, m, d_pad, 256); }
extern "C" long long rows(long long b) { return fz::quant_workspace_rows(b); }
extern "C" void plan(long long b, long long m, long long d_pad, long long *out)
{
    const fz::QuantPlan p = fz::plan_quant_product(b, m, d_pad, 256);
    const long long v[] = {p.bm, p.bn, p.x_tiles, p.w_tiles, p.nk, p.splits, p.wgs, (long long)p.part};
    for (int i = 0; i < 8; ++i) out[i] = v[i];
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(at / "plan.cpp"), "-o", str(at / "plan.so")])
    lib = ctypes.CDLL(str(at / "plan.so"))
    i64 = ctypes.c_longlong
    lib.room.restype = lib.rows.restype = i64
    lib.room.argtypes, lib.rows.argtypes, lib.plan.argtypes = [i64] * 3, [i64], [i64] * 3 + [ctypes.c_void_p]

    class Plans:
        room, rows = staticmethod(lib.room), staticmethod(lib.rows)

        @staticmethod
        def plan(b, m, d_pad):
            out = (i64 * 8)()
            lib.plan(b, m, d_pad, ctypes.addressof(out))
            return dict(zip(("bm", "bn", "x_tiles", "w_tiles", "nk", "splits", "wgs", "part"), out))
    return Plans


LAYERS = [(32768, 4096), (8192, 8192), (1024, 8192), (1, 128), (70, 5120), (16, 65536), (131072, 8192), (258, 1152), (300, 30080), (50021, 4096), (129, 4194304),
          (1 << 24, 128)]


@pytest.mark.parametrize("m,d_pad", LAYERS)
def test_a_workspace_serves_every_smaller_batch(plans, m, d_pad):
    rng = random.Random(m + d_pad)
    batches = sorted(set(list(range(1, 700)) + [2 ** i + o for i in range(4, 21) for o in (-1, 0, 1)] + [int(2 ** rng.uniform(9, 20)) for _ in range(200)]))
    most_rows = most_part = 0
    for b in batches:
        p, rows, room = plans.plan(b, m, d_pad), plans.rows(b), plans.room(b, m, d_pad)
        if p["wgs"] == 0:     # refused: more tiles than a launch has workgroups
            assert b * m > 1 << 38
            continue
        assert p["x_tiles"] * p["bm"] >= b and p["w_tiles"] * p["bn"] >= m and p["nk"] * 128 == d_pad
        assert 1 <= p["splits"] <= min(p["nk"], 64) and p["wgs"] == p["x_tiles"] * p["w_tiles"] * p["splits"]
        # what any smaller batch takes fits what this one asks for
        most_rows, most_part = max(most_rows, p["x_tiles"] * p["bm"]), max(most_part, 4 * p["part"])
        assert most_rows <= rows and most_part <= room, (b, p)
        assert p["part"] == (p["wgs"] * p["bm"] * p["bn"] if p["splits"] > 1 else 0)
    sizes = [(plans.rows(b), plans.room(b, m, d_pad)) for b in batches]
    assert all(a[0] <= c[0] and a[1] <= c[1] for a, c in zip(sizes, sizes[1:]))


def test_every_accepted_layer_has_a_launch(plans):
    # a grid dimension has less than 2^32 threads, a workgroup 512 of them
    rng = random.Random(5)
    sizes = [(1, m, d) for m in (2147483647 - 513, 1100000000, 1 << 30, 1073741824 + 1, 1 << 23) for d in (128, 256, 1024)]
    sizes += [(int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 31)) - 600, 128 * int(2 ** rng.uniform(0, 8))) for _ in range(3000)]
    for b, m, d in sizes:
        if m < 1 or b * m > 1 << 38:     # (beyond the memory of any device)
            continue
        p = plans.plan(b, m, d)
        assert 0 < p["wgs"] * 512 < 1 << 32, (b, m, d, p)
        assert p["splits"] == 1 or p["x_tiles"] * p["w_tiles"] * p["bm"] * p["bn"] // 4 < 1 << 32
    assert plans.plan(1 << 30, 1 << 30, 128)["wgs"] == 0
