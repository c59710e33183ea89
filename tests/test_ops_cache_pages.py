"""Which keys' and values' pages share memory, without a GPU: the rule against every page of each, and its refusals."""
from __future__ import annotations

import os
import subprocess

import pytest

from tests.test_ops_cache_host import APPEND, lib  # noqa: F401
from tests.test_ops_host import INVALID, P, run

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_rule_against_every_page(tmp_path):
    src = tmp_path / "pages.cpp"
    src.write_text("""
#include "ops_forms.h"
#include <cstdio>
#include <random>
using namespace simops;
int main() {
    std::mt19937_64 rng(1);
    const auto upto = [&](uint64_t n) { return rng() % n; };
    int met = 0, apart = 0;
    for (int i = 0; i < 200000; i++) {
        const uint64_t page = 1 + upto(6), pages = upto(7), stride = page + upto(12), a = 100 + upto(120), b = 100 + upto(120);
        bool want = false;
        for (uint64_t x = 0; x < pages; x++)
            for (uint64_t y = 0; y < pages; y++) {
                const uint64_t p = a + x * stride, q = b + y * stride;
                want |= p < q + page && q < p + page;
            }
        (want ? met : apart)++;
        if (pages_meet(a, stride, b, stride, pages, page) != want) return printf("%lu %lu %lu %lu %lu\\n", a, b, stride, pages, page), 1;
        // of different strides: whenever they do, and never where one array lies behind the other
        const uint64_t other = page + upto(12);
        bool shared = false;
        for (uint64_t x = 0; x < pages; x++)
            for (uint64_t y = 0; y < pages; y++) {
                const uint64_t p = a + x * stride, q = b + y * other;
                shared |= p < q + page && q < p + page;
            }
        if (shared && !pages_meet(a, stride, b, other, pages, page)) return 2;
        if (pages && (a + (pages - 1) * stride + page <= b || b + (pages - 1) * other + page <= a) && pages_meet(a, stride, b, other, pages, page)) return 3;
    }
    // sizes past 64 bits
    if (pages_meet(1 << 20, 1ull << 62, (1ull << 63) + 7, 1ull << 62, 1ull << 31, 1 << 20) != true) return 4;
    return met > 1000 && apart > 1000 ? 0 : 5;
}
""")
    exe = str(tmp_path / "pages")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2606_10440_amd", "csrc"),
                    str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stdout)


# pages of 4096 elements, 8192 bytes
@pytest.mark.parametrize("change", [
    dict(), dict(vc=P + 16), dict(vc=P + 8176), dict(vc=P + 4 * 8192 - 16), dict(kc=P + 8192), dict(kc_stride=8192, vc_stride=8192, vc=P + 8176),
    dict(kc_stride=8192, vc_stride=8192, vc=P + 8192 + 16), dict(kc_stride=8192, vc=P + 8192), dict(pages=1, vc=P + 8176)])
def test_parts_that_share_memory_are_refused(lib, change):  # noqa: F811
    assert run(lib, "sim_cache_append", APPEND, **change) == INVALID
