"""Which form of the products by group a call takes (csrc/grouped_forms.h, compiled for the host): every form is one that GPU tests of
the products reach, and what is chosen is near the fastest of the forms that profiles/operators_forms.md has the times of."""
import os
import shutil
import subprocess

import pytest

from tests import test_gpu_feature_forms as more
from tests import test_gpu_features as features

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ELEMENT = {"f32": 0, "bf16": 1, "f16": 2}

MAIN = r"""
#include <stdio.h>
#include "grouped_forms.h"
static void rows(const ds_mm_sizes& p, int t, bool transposed) {
  const int depth = transposed ? p.outer : p.inner, width = transposed ? p.inner : p.outer;
  if (ds_rows_in_tiles(p, t, depth, width)) {
    const bool large = t == DS_ELEM_F32 ? ds_wide_tiles(p.rows, width) : ds_narrow_tiles(p.rows, p.groups, width) > kNarrowTiles;
    printf("tiles-%s ", large ? "large" : "small");
  } else {
    const ds_few_form f = ds_choose_few(p, t, transposed, false);
    printf("few-%d%s%s ", 1 << f.shift, f.half ? "-half" : "", f.eight_waves ? "-eight" : "");
  }
}
int main() {
  int t, r, i, o, g;
  while (scanf("%d %d %d %d %d", &t, &r, &i, &o, &g) == 5) {
    const ds_mm_sizes p = {r, i, o, g};
    rows(p, t, false);
    rows(p, t, true);
    const int side = t == DS_ELEM_F32 ? 128 : 256, unit = t == DS_ELEM_F32 ? 32 : 64;
    if (ds_weights_in_tiles(p, t)) printf("tiles-%s\n", ds_weight_chunks(r, (int64_t)((i + side - 1) / side) * ((o + side - 1) / side), unit) > 1 ? "cut" : "whole");
    else printf("%s\n", ds_weights_shared(p) ? "shared" : "alone");
  }
}
"""


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    """(forward, dx, dW) of every (type, rows, inner, outer, groups)."""
    cxx = shutil.which("g++")
    assert cxx, "g++ is needed"
    at = tmp_path_factory.mktemp("forms")
    (at / "main.cpp").write_text(MAIN)
    subprocess.run([cxx, "-std=c++17", "-I", os.path.join(ROOT, "paper_2506_22668_amd", "csrc"), str(at / "main.cpp"), "-o", str(at / "main")], check=True)

    def choose(shapes):
        text = "\n".join(f"{ELEMENT[s[0]]} {s[1]} {s[2]} {s[3]} {s[4]}" for s in shapes)
        out = subprocess.run([str(at / "main")], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(shapes)
        return [tuple(line.split()) for line in out]
    return choose


def shapes_of(test):
    return next(m.args[1] for m in test.pytestmark if m.args[0] == "rows, inner, outer, groups")


FEW = {f"few-{n}{eight}" for n in (16, 32) for eight in ("", "-eight")} | {"few-64"}
HALF = {f"few-{n}-half{eight}" for n in (16, 32) for eight in ("", "-eight")} | {"few-64-half"}
TILES = {f"tiles-{size}-{rows}" for size in ("small", "large") for rows in ("whole", "odd")}


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_every_form_is_one_that_gpu_tests_compare_with_the_formula(forms, t):
    """Of the tiles both kinds of rows: of whole pieces of 16 bytes, which come to LDS by themselves, and odd ones, which come through registers."""
    shapes = [(t, *s) for test in (features.test_grouped_mm, features.test_grouped_mm_many_tiles, features.test_grouped_mm_few_rows,
                                   features.test_grouped_mm_narrow, more.test_gradients_of_aligned_rows, more.test_products_of_further_forms,
                                   more.test_products_of_many_groups) for s in shapes_of(test)]
    seen, piece = [set(), set(), set()], 4 if t == "f32" else 8
    for (_, _, inner, outer, _), form in zip(shapes, forms(shapes)):
        for kind, name, widths in zip(seen, form, ((inner,), (outer,), (inner, outer))):
            tiles = name.startswith("tiles")
            assert not tiles or min(inner, outer) >= 8   # (their loads need rows of 16 bytes)
            kind.add(name + ("" if not tiles else "-odd" if any(w % piece for w in widths) else "-whole"))
    assert FEW | TILES <= seen[0], (FEW | TILES) - seen[0]
    assert FEW - {"few-16-eight", "few-32-eight"} | HALF | TILES <= seen[1], (FEW | HALF | TILES) - seen[1]
    assert {"alone", "shared", "tiles-cut-whole", "tiles-cut-odd"} <= seen[2], seen[2]
    # the aligned rows are there for the tiles of the weights
    assert [f[2] for f in forms([(t, *s) for s in shapes_of(more.test_gradients_of_aligned_rows)])].count("tiles-cut") >= 5


def table():
    with open(os.path.join(ROOT, "profiles", "operators_forms.md")) as f:
        for line in f:
            cells = [c.strip() for c in line.strip().strip("|").split("|")]
            if len(cells) == 10 and cells[0] in ELEMENT:
                yield (cells[0], *map(int, cells[1:5])), tuple(map(float, cells[5:]))


def test_the_choice_is_near_the_fastest_form_measured(forms):
    rows = list(table())
    assert len(rows) == 323
    forward, backward = [], []
    for (few, tiles, both, dx_tiles, dw_tiles), form in zip((r[1] for r in rows), forms([r[0] for r in rows])):
        forward.append((tiles if form[0].startswith("tiles") else few) / min(few, tiles) - 1)
        dx, dw = dx_tiles - both, dw_tiles - both   # (what tiles change of either gradient)
        took = both + dx * form[1].startswith("tiles") + dw * form[2].startswith("tiles")
        backward.append(took / (both + min(dx, 0) + min(dw, 0)) - 1)
    print(f"forward {sum(forward) / 323:.4f} {max(forward):.3f}, both gradients {sum(backward) / 323:.4f} {max(backward):.3f}")
    assert sum(forward) / 323 < 0.01 and sum(f > 0.12 for f in forward) <= 3 and max(forward) < 0.35
    assert sum(backward) / 323 < 0.03 and sum(b > 0.12 for b in backward) <= 19 and max(backward) < 0.55
