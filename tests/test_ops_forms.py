"""Which form of the operators' kernels a size runs, asked of the rules that
the launchers use (``csrc/ops_forms.h``, compiled here): every form is run by
the GPU tests that are meant for it."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

from tests import test_gpu_ops_forms as forms
from tests import test_gpu_ops_layer_tiles as layer_tiles

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")

DRIVER = r"""
#include <cstdio>
#include <cstring>
#include "ops_forms.h"
using namespace simops;
int main() {
    char what[8];
    long long a, b, c, d, e, f;
    const char *product[] = {"skinny_small", "skinny_large", "256x256", "128x128", "64x128", "64x64", "simple"};
    while (scanf("%7s %lld %lld %lld %lld %lld %lld", what, &a, &b, &c, &d, &e, &f) == 7) {
        if (!strcmp(what, "product")) puts(product[product_form(a, b, c)]);
        else if (!strcmp(what, "one")) puts(linear_in_one(a, c) ? "one" : "two");
        else if (!strcmp(what, "layer")) printf("%d\n", (int[]){0, 1, 2, 4}[layer_form(a, b, c, d, e, f)]);
        else if (!strcmp(what, "inputs")) puts(a * few_input_pitch(b, c) <= kFewInputs ? "lds" : "past");
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    at = tmp_path_factory.mktemp("forms")
    (at / "driver.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2606_10440_amd", "csrc"), str(at / "driver.cpp"),
                    "-o", str(at / "driver")], check=True)

    def run(what, cases):
        lines = "".join(" ".join([what, *(str(int(v)) for v in c), *["0"] * (6 - len(c))]) + "\n" for c in cases)
        out = subprocess.run([str(at / "driver")], input=lines, capture_output=True, text=True, check=True).stdout.split()
        assert len(out) == len(cases)
        return out

    return run


def test_products_run_the_form_they_are_for(ask):
    assert ask("product", [c[1:] for c in forms.CASES]) == [c[0] for c in forms.CASES]
    assert set(forms.PRODUCTS) == {"skinny_small", "skinny_large", "256x256", "128x128", "64x128", "64x64", "simple"}


def test_linear_layers_of_one_launch(ask):
    assert set(ask("one", forms.IN_ONE)) == {"one"}
    assert ask("one", [(2, 70, 8193), (33, 70, 64), (1, 33, 16385)]) == ["two"] * 3


@pytest.mark.parametrize("weights", ["same", "mx4"])
def test_few_tokens_inputs_in_lds_and_past_it(ask, weights):
    cols = forms.COLS[weights]
    both = 0
    for T, E, k, D, F in forms.PAST_LDS:
        assert ask("layer", [(T, E, k, D, F, weights == "mx4")]) == ["0"]
        n = [c for c in forms.tokens_of_experts(forms.spread(T, E, k, False), k) if c]
        kinds = ask("inputs", [(c, D, cols) for c in n])
        assert "past" in kinds
        both += "lds" in kinds
    assert both


def test_layer_tilings(ask):
    want = [2] * 4 + [4] * 4 + [1] * 3
    assert [int(v) for v in ask("layer", [(*c, False) for c in layer_tiles.CASES])] == want
    assert [int(v) for v in ask("layer", [(*c, True) for c in layer_tiles.CASES])] == [min(v, 2) for v in want]
