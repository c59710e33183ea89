"""The paged cache's calls without a GPU: refusals, workspace queries, and the plan that cuts sequences into units."""
from __future__ import annotations

import os

import pytest

from tests.test_ops_host import INVALID, P, SIZE, run

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2606_10440_amd import ops, sim
    if not os.path.exists(sim.LIB_PATH):
        from paper_2606_10440_amd import build
        build.build()
    return ops.lib()


APPEND = [("type", 2), ("k", P), ("k_stride", 256), ("k_head", 128), ("v", P), ("v_stride", 256), ("v_head", 128), ("T", 3),
          ("heads", 2), ("D", 128), ("slots", P), ("kc", P), ("kc_stride", 4096), ("vc", P), ("vc_stride", 4096), ("pages", 4),
          ("page_size", 16)]
CACHE_BAD = [(dict(type=0), INVALID), (dict(type=3), INVALID), (dict(D=0), INVALID), (dict(D=12), INVALID),
             (dict(D=264), INVALID), (dict(D=-8), INVALID), (dict(pages=-1), INVALID), (dict(page_size=0), INVALID),
             (dict(kc=None), INVALID), (dict(vc=None), INVALID), (dict(kc=P + 8), INVALID), (dict(vc=P + 2), INVALID),
             (dict(kc_stride=4100), INVALID), (dict(vc_stride=4088), INVALID), (dict(kc_stride=-4096), INVALID)]


@pytest.mark.parametrize("change,want", CACHE_BAD + [
    (dict(heads=0), INVALID), (dict(T=-1), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(slots=None), INVALID),
    (dict(k=P + 1), INVALID), (dict(slots=P + 4), INVALID), (dict(k_stride=-1), INVALID), (dict(v_head=-128), INVALID),
    (dict(T=1 << 31), SIZE), (dict(pages=1 << 31), SIZE), (dict(T=0), 0), (dict(pages=0, kc=None, vc=None), 0)])
def test_append_refusals(lib, change, want):
    assert run(lib, "sim_cache_append", APPEND, **change) == want


ATTEND = [("type", 2), ("q", P), ("q_stride", 1024), ("q_head", 128), ("B", 3), ("q_heads", 8), ("heads", 2), ("D", 128),
          ("kc", P), ("kc_stride", 4096), ("vc", P), ("vc_stride", 4096), ("pages", 4), ("page_size", 16), ("table", P),
          ("table_stride", 64), ("table_pages", 64), ("lengths", P), ("scale", 0.1), ("window", 0), ("out", P),
          ("out_stride", 1024), ("lse", None), ("ws", P), ("ws_bytes", 1 << 30)]


@pytest.mark.parametrize("change,want", CACHE_BAD + [
    (dict(heads=0), INVALID), (dict(heads=3), INVALID), (dict(q_heads=0), INVALID), (dict(B=-1), INVALID),
    (dict(table_pages=-1), INVALID), (dict(window=-1), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=3e38), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(lengths=None), INVALID),
    (dict(table=None), INVALID), (dict(q=P + 1), INVALID), (dict(out=P + 1), INVALID), (dict(table=P + 2), INVALID),
    (dict(lengths=P + 2), INVALID), (dict(lse=P + 2), INVALID), (dict(out_stride=1023), INVALID), (dict(q_stride=-1), INVALID),
    (dict(table_stride=-1), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 4), INVALID), (dict(ws_bytes=64), INVALID),
    (dict(table_pages=1 << 30), SIZE), (dict(B=1 << 31), SIZE), (dict(B=1 << 26), SIZE), (dict(B=0), 0)])
def test_attention_refusals(lib, change, want):
    assert run(lib, "sim_cache_attention", ATTEND, **change) == want


def test_workspace_queries(lib):
    ask = lib.sim_cache_attention_workspace
    for bad in [(-1, 8, 2, 128, 64, 16, 0), (0, 8, 2, 128, 64, 16, 0), (3, 8, 3, 128, 64, 16, 0), (3, 8, 0, 128, 64, 16, 0),
                (3, 8, 2, 12, 64, 16, 0), (3, 8, 2, 512, 64, 16, 0), (3, 8, 2, 128, -1, 16, 0), (3, 8, 2, 128, 64, 0, 0),
                (3, 8, 2, 128, 64, 16, -1), (3, 8, 2, 128, 1 << 30, 16, 0), (1 << 40, 8, 2, 128, 64, 16, 0)]:
        assert ask(*bad) == 0, bad
    assert ask(3, 8, 2, 128, 8, 16, 0) == 0  # one unit a sequence
    assert ask(3, 8, 2, 128, 64, 16, 0) > 0 and ask(3, 8, 2, 128, 64, 16, 64) == 0


def test_units_fit_the_workspace(lib, tmp_path):
    """However the lengths are, the units that the plan cuts are no more than the workspace has places for."""
    import subprocess
    src = tmp_path / "plan.cpp"
    src.write_text("""
#include "ops_forms.h"
#include <cstdio>
#include <random>
using namespace simops;
int main() {
    // however many steps there are together, a unit is a number of them, and one is enough for any sequence
    if (attend_unit((int64_t)1 << 50, 1) != kAttendMostSteps || attend_steps((int64_t)1 << 30, 0) > kAttendMostSteps) return 4;
    std::mt19937_64 rng(1);
    const auto upto = [&](int64_t n) { return (int64_t)(rng() % (uint64_t)n); };
    for (int i = 0; i < 20000; i++) {
        const int64_t B = 1 + upto(i % 3 ? 8 : 300), cap = 1 + upto((int64_t)1 << (4 + upto(16)));
        const int32_t window = i % 4 ? 0 : 1 + (int32_t)upto(4000);
        const int64_t units = attend_units(1 + upto(i % 5 ? 16 : 2000), 1 + (int)upto(3)), most = attend_max_units(B, units, cap, window);
        int64_t total = 0, n = 0;
        std::vector<int64_t> steps(B);
        for (auto &s : steps) {
            const int64_t end = upto(4) ? upto(cap + 1) : cap, start = window ? std::max<int64_t>(0, end - window) : 0;
            s = (end + kAttendKeys - 1) / kAttendKeys - start / kAttendKeys;
            if (s > attend_steps(cap, window)) return 1;
            total += s;
        }
        const int unit = attend_unit(total, units);
        for (int64_t s : steps) {
            n += attend_splits(cap, window) ? std::max<int64_t>(1, (s + unit - 1) / unit) : 1;
            if (s > kAttendWhole && !attend_splits(cap, window)) return 2;
        }
        if (n > most) { printf("%ld %ld %d %ld\\n", (long)B, (long)cap, window, (long)units); return 3; }
    }
    return 0;
}
""".replace("#include <random>", "#include <random>\n#include <vector>"))
    exe = str(tmp_path / "plan")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2606_10440_amd", "csrc"),
                    str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stdout)
