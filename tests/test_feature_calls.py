"""Operators on rows of features without a GPU: what the C entries and the binding refuse, sizes of workspaces, and the rows
of a group from offsets that hold anything (csrc/group_range.h, compiled for the host)."""
import ctypes as C
import os
import shutil
import subprocess
import types

import pytest

from paper_2506_22668_amd import binding
from paper_2506_22668_amd.binding import DS_ECAPACITY, DS_EINVAL, DistShapError

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def ctx():
    """The entries look at their arguments before they touch the GPU; all that they need for it is a context to leave the message in."""
    return C.create_string_buffer(1 << 16)


P = 1 << 20   # stands for a device address: aligned, never followed
LAYER_NORM = dict(dtype=0, rows=5, cols=8, x=P, xs=8, weight=None, bias=None, eps=1e-5, y=P, ys=8, mean=None, rstd=None)
NORM_BACKWARD = dict(dtype=1, rows=5, cols=8, dy=P, dys=8, x=P, xs=8, mean=P, rstd=P, weight=None, dx=P, dxs=8, dweight=P, dbias=P,
                     ws=P, wsn=1 << 20)
DROPOUT = dict(dtype=2, rows=5, cols=8, x=P, xs=8, residual=None, rs=0, p=0.5, seed=1, tag=0, y=P, ys=8)
GROUP_ROWS = dict(ids=P, rows=5, groups=3, offsets=P, order=P, ws=None, wsn=0)
GROUPED_MM = dict(dtype=0, rows=5, inner=8, outer=8, groups=3, x=P, xs=8, w=P, offsets=P, order=None, bias=None, relu=0, y=P, ys=8)
MM_BACKWARD = dict(dtype=0, rows=5, inner=8, outer=8, groups=3, dy=P, dys=8, x=P, xs=8, w=P, offsets=P, order=None, gate=None, gs=0,
                   dx=P, dxs=8, dw=P, db=P, ws=P, wsn=1 << 40)


@pytest.mark.parametrize("name, good, bad", [
    ("ds_layer_norm", LAYER_NORM, [dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(cols=0), dict(cols=4097), dict(eps=-1.0),
                                   dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(y=None), dict(x=P + 2),
                                   dict(xs=-1), dict(ys=7), dict(ys=0), dict(xs=1 << 50)]),
    ("ds_layer_norm_backward", NORM_BACKWARD, [dict(dtype=9), dict(rows=-1), dict(cols=5000), dict(dy=None), dict(x=None), dict(dx=None),
                                               dict(mean=None), dict(rstd=None), dict(dweight=None), dict(dbias=None), dict(dxs=3),
                                               dict(ws=P + 4), dict(dy=P + 1)]),
    ("ds_dropout", DROPOUT, [dict(dtype=7), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(rows=-1), dict(cols=0),
                             dict(cols=(1 << 20) + 1), dict(x=None), dict(y=None), dict(residual=P + 1), dict(ys=7), dict(rs=-8, residual=P)]),
    ("ds_group_rows", GROUP_ROWS, [dict(rows=-1), dict(rows=(1 << 30) + 1), dict(groups=0), dict(groups=1025), dict(ids=None),
                                   dict(order=None), dict(offsets=None)]),
    ("ds_grouped_mm", GROUPED_MM, [dict(dtype=3), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(inner=0), dict(outer=0), dict(groups=0),
                                   dict(groups=1025), dict(x=None), dict(w=None), dict(offsets=None), dict(y=None), dict(ys=7),
                                   dict(w=P + 2), dict(inner=(1 << 20) + 1)]),
    ("ds_grouped_mm_backward", MM_BACKWARD, [dict(dtype=3), dict(rows=-1), dict(inner=0), dict(outer=0), dict(groups=0), dict(dy=None),
                                             dict(x=None), dict(w=None), dict(offsets=None), dict(dx=None), dict(dw=None), dict(db=None),
                                             dict(dxs=7), dict(gate=P + 1, gs=8), dict(gate=P, gs=-8)]),
])
def test_bad_arguments_are_refused_before_any_work(ctx, name, good, bad):
    lib = binding.load_library()
    fn = getattr(lib, name)
    assert fn(None, *good.values()) == DS_EINVAL
    for change in bad:
        assert set(change) <= set(good)
        assert fn(ctx, *{**good, **change}.values()) == DS_EINVAL, change
        assert lib.ds_last_error(ctx), change


def test_a_workspace_that_is_too_small_is_refused(ctx):
    lib = binding.load_library()
    need = C.c_int64()
    assert lib.ds_layer_norm_backward_workspace(5, 8, C.byref(need)) == 0 and need.value > 0
    for change in (dict(wsn=need.value - 1), dict(ws=None)):
        assert lib.ds_layer_norm_backward(ctx, *{**NORM_BACKWARD, **change}.values()) == DS_ECAPACITY
    assert lib.ds_group_rows_workspace(5, 3, C.byref(need)) == 0 and need.value == 0
    assert lib.ds_group_rows_workspace(1_000_003, 3, C.byref(need)) == 0 and need.value > 0
    assert lib.ds_group_rows(ctx, *{**GROUP_ROWS, "rows": 1_000_003, "ws": P, "wsn": need.value - 4}.values()) == DS_ECAPACITY


def test_sizes_out_of_range_have_no_workspace():
    lib = binding.load_library()
    need = C.c_int64()
    for rows, cols in [(-1, 8), (8, 0), (8, 4097)]:
        assert lib.ds_layer_norm_backward_workspace(rows, cols, C.byref(need)) == DS_EINVAL
    for rows, groups in [(-1, 8), (8, 0), (8, 1025), ((1 << 30) + 1, 8)]:
        assert lib.ds_group_rows_workspace(rows, groups, C.byref(need)) == DS_EINVAL
    for args in [(5, 1, 1, 1, 1), (0, -1, 1, 1, 1), (0, 1, 0, 1, 1), (0, 1, 1, 0, 1), (0, 1, 1, 1, 0)]:
        assert lib.ds_grouped_mm_backward_workspace(*args, C.byref(need)) == DS_EINVAL
    assert lib.ds_layer_norm_backward_workspace(8, 8, None) == DS_EINVAL


def _context():
    """A Context over a library that must not be reached."""
    c = object.__new__(binding.Context)
    c.torch, c.lib, c.h = torch, None, None
    c.device, c._index = torch.device("cpu"), -1
    c._elements = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    return c


F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("call", [
    lambda c: c.layer_norm(torch.zeros(4)),                                                 # not rows
    lambda c: c.layer_norm(torch.zeros(4, 4, dtype=torch.float64)),                         # a type it does not have
    lambda c: c.layer_norm(torch.zeros(4, 4), weight=torch.zeros(5)),
    lambda c: c.layer_norm(torch.zeros(4, 4, dtype=BF16), weight=torch.zeros(4, dtype=BF16)),   # parameters are fp32
    lambda c: c.layer_norm_backward(torch.zeros(4, 3), torch.zeros(4, 4), torch.zeros(4), torch.zeros(4)),
    lambda c: c.layer_norm_backward(torch.zeros(4, 4, dtype=BF16), torch.zeros(4, 4), torch.zeros(4), torch.zeros(4)),
    lambda c: c.layer_norm_backward(torch.zeros(4, 4), torch.zeros(4, 4), torch.zeros(3), torch.zeros(4)),
    lambda c: c.layer_norm_backward(torch.zeros(4, 4), torch.zeros(4, 4), None, torch.zeros(4)),
    lambda c: c.dropout(torch.zeros(4, 4), 0.5, 1, residual=torch.zeros(4, 4, dtype=BF16)),
    lambda c: c.dropout(torch.zeros(4, 4), 0.5, 1, residual=torch.zeros(3, 4)),
    lambda c: c.group_rows(torch.zeros(4, dtype=torch.int64), 3),
    lambda c: c.group_rows(torch.zeros(2, 2, dtype=torch.int32), 3),
    lambda c: c.grouped_mm(torch.zeros(4, 4), torch.zeros(2, 5, 4), torch.zeros(3, dtype=torch.int64)),
    lambda c: c.grouped_mm(torch.zeros(4, 4), torch.zeros(2, 4, 4, dtype=BF16), torch.zeros(3, dtype=torch.int64)),
    lambda c: c.grouped_mm(torch.zeros(4, 4), torch.zeros(2, 4, 4), torch.zeros(2, dtype=torch.int64)),
    lambda c: c.grouped_mm(torch.zeros(4, 4), torch.zeros(2, 4, 4), torch.zeros(3, dtype=torch.int32)),
    lambda c: c.grouped_mm(torch.zeros(4, 4), torch.zeros(2, 4, 4), None),
    lambda c: c.grouped_mm(torch.zeros(4, 4), torch.zeros(2, 4, 4), torch.zeros(3, dtype=torch.int64), order=torch.zeros(4, dtype=torch.int64)),
    lambda c: c.grouped_mm(torch.zeros(4, 4), torch.zeros(2, 4, 4), torch.zeros(3, dtype=torch.int64), bias=torch.zeros(4)),
    lambda c: c.grouped_mm_backward(torch.zeros(4, 5), torch.zeros(4, 4), torch.zeros(2, 4, 4), torch.zeros(3, dtype=torch.int64)),
    lambda c: c.grouped_mm_backward(torch.zeros(4, 4), torch.zeros(4, 4), torch.zeros(2, 4, 4), torch.zeros(3, dtype=torch.int64),
                                    gate=torch.zeros(4, 3)),
])
def test_the_binding_refuses_shapes_and_types(call):
    with pytest.raises(DistShapError) as e:
        call(_context())
    assert e.value.code == DS_EINVAL


def test_a_tensor_of_another_device_is_refused():
    c = _context()
    c._index, c.device = 0, torch.device("cuda:0")
    with pytest.raises(DistShapError):
        c.layer_norm(torch.zeros(4, 4))


def test_a_capture_of_a_stream_that_is_not_the_contexts_is_refused():
    c = _context()
    c._raw_stream, c._current_stream = 0, lambda i: 7
    c.torch = types.SimpleNamespace(cuda=types.SimpleNamespace(current_stream=lambda i: types.SimpleNamespace(cuda_stream=7),
                                                               is_current_stream_capturing=lambda: True))
    with pytest.raises(DistShapError):
        c._queue(None)


MAIN = r"""
#include <stdio.h>
#include "group_range.h"
int main() {
  const int64_t big = (int64_t)1 << 62;
  const int64_t values[] = {-big, -1, 0, 1, 3, 7, 8, 9, (int64_t)1 << 32, big};
  const int n = sizeof(values) / sizeof(*values), rows = 8;
  long bad = 0;
  for (int a = 0; a < n; ++a)
    for (int b = 0; b < n; ++b) {
      const int64_t offsets[2] = {values[a], values[b]};
      for (int g = 0; g <= 1; ++g) {
        int begin = -1, end = -1;
        ds_group_range(offsets, 1, rows, g, &begin, &end);
        bad += !(0 <= begin && begin <= end && end <= rows);
        if (values[a] >= 0 && values[a] <= values[b] && values[b] <= rows)
          bad += g == 0 ? begin != values[a] || end != values[b] : begin != values[b] || end != rows;
      }
    }
  const int32_t order[] = {5, -1, 8, 7, 0, 2147483647, -2147483647 - 1, 3};
  const int want[] = {5, -1, -1, 7, 0, -1, -1, 3};
  for (int i = 0; i < rows; ++i) bad += ds_ordered_row(order, rows, i) != want[i] || ds_ordered_row(nullptr, rows, i) != i;
  printf("%ld\n", bad);
}
"""


def test_rows_of_a_group_stay_inside_whatever_the_offsets_hold(tmp_path):
    cxx = shutil.which("g++")
    assert cxx, "g++ is needed"
    src, exe = tmp_path / "main.cpp", tmp_path / "main"
    src.write_text(MAIN)
    subprocess.run([cxx, "-std=c++17", "-I", os.path.join(ROOT, "paper_2506_22668_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout == "0\n"


TILES = r"""
#include <stdio.h>
#include <stdlib.h>
#include <vector>
#include "group_range.h"
#include "mm_split.h"
static unsigned long long state = 88172645463325252ull;
static unsigned long long draw() { state ^= state << 13; state ^= state >> 7; state ^= state << 17; return state; }
int main() {
  long bad = 0, capped = 0;
  const int sizes[] = {16, 32, 64, 128, 256};
  const int all_rows[] = {1, 5, 1000, 70001, 1 << 22, 1 << 28, 1 << 29, 1 << 30};
  const int all_groups[] = {1, 2, 64, 65, 1000, 1024};
  for (int rows : all_rows) for (int groups : all_groups) for (int size : sizes) for (int shape = 0; shape < 4; ++shape) {
    std::vector<int64_t> offsets(groups + 1);
    for (int g = 0; g <= groups; ++g)
      offsets[g] = shape == 0 ? (int64_t)rows * g / groups                               // ascending: the tiles are exact
                 : shape == 1 ? (g % 2 ? rows : 0)                                        // every other group has all rows
                 : shape == 2 ? (int64_t)(draw() % (2ull * rows)) - rows / 2 : (g % 2 ? (int64_t)1 << 62 : -((int64_t)1 << 62));
    for (int none = 0; none < 2; ++none) {   // with the tiles of the rows of no group (row products), or without (gradients of the weights)
      const int most = ds_most_parts(rows, size, groups + none);
      std::vector<int> upto(groups + none), begin(groups + none), end(groups + none);
      long long exact = 0;
      int sum = 0;
      for (int g = 0; g < groups + none; ++g) {
        ds_group_range(offsets.data(), groups, rows, g, &begin[g], &end[g]);
        exact += ds_parts_of(begin[g], end[g], size);
        upto[g] = sum = ds_add_parts(sum, ds_parts_of(begin[g], end[g], size), most);
      }
      bad += sum < 0 || sum > most || (shape == 0 && sum != exact);
      capped += sum != exact;
      for (int g = 0; g < groups + none; ++g) {
        const int before = g ? upto[g - 1] : 0, own = ds_parts_of(begin[g], end[g], size);
        if (upto[g] <= before) continue;
        const int ends[] = {before, upto[g] - 1};
        for (int tile : ends) {
          // counted from the sum in front of the group, or from its own sum back
          const int64_t one = begin[g] + (int64_t)(tile - before) * size, other = begin[g] + (int64_t)(tile - (upto[g] - own)) * size;
          bad += one < begin[g] || one >= end[g] || other < begin[g] || other >= end[g] || (shape == 0 && one != other);
        }
      }
      if (none) continue;
      for (int wgs : {1, 3, 256, 512}) {
        const int chunks = sum < wgs ? sum : wgs;
        for (int g = 0; g < groups; ++g) {
          const int before = g ? upto[g - 1] : 0, own = ds_parts_of(begin[g], end[g], size);
          if (own == 0) continue;
          int first = -1, last = -1;
          ds_group_owners(before, own, sum, [&](int x) { return (int)ds_mm_even_owner(x, chunks, sum); }, &first, &last);
          bad += first < 0 || last < first || last >= chunks;
          if (shape == 0) bad += first != ds_mm_even_owner(before, chunks, sum) || last != ds_mm_even_owner(before + own - 1, chunks, sum);
        }
      }
    }
  }
  printf("%ld %d\n", bad, capped > 0);
}
"""


def test_tiles_of_offsets_that_do_not_ascend_are_counted_without_an_overflow(tmp_path):
    """1,024 groups that all have up to 2^30 rows: tiles, steps and workgroups stay in range, and are exact where offsets ascend."""
    cxx = shutil.which("g++")
    assert cxx, "g++ is needed"
    src, exe = tmp_path / "tiles.cpp", tmp_path / "tiles"
    src.write_text(TILES)
    subprocess.run([cxx, "-std=c++17", "-O1", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2506_22668_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout == "0 1\n"


LINES = r"""
#include <stdio.h>
#include <initializer_list>
#include "group_range.h"
int main() {
  long bad = 0;
  const int64_t counts[] = {1, 2, 255, 65536, 16777215, 16777216, 16777217, 33554433, 1000000007, 0x7fff0000};
  for (int64_t n : counts) for (int threads : {256, 512}) {
    const ds_lines l = ds_launch_lines(n, threads);
    const int64_t all = (int64_t)l.x * l.y;
    bad += all < n || all - n >= l.y || all > 0x7fffffff || (int64_t)l.x * threads > 0xffffffffll || l.y > 65535 || (n * threads < 4294967296ll && l.y != 1);
  }
  printf("%ld\n", bad);
}
"""


def test_a_launch_has_no_more_threads_in_a_line_than_are_counted(tmp_path):
    cxx = shutil.which("g++")
    assert cxx, "g++ is needed"
    src, exe = tmp_path / "lines.cpp", tmp_path / "lines"
    src.write_text(LINES)
    subprocess.run([cxx, "-std=c++17", "-I", os.path.join(ROOT, "paper_2506_22668_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout == "0\n"


def _idle():
    """A context whose calls do nothing: what the binding makes of arguments and outputs is left."""
    c = _context()
    c.lib, c._queue, c._workspace = types.SimpleNamespace(**{name: None for name in binding.EXPORTED_SYMBOLS}), lambda *a: None, lambda *a: (None, None, 0)
    return c


OFFSETS = torch.tensor([0, 2, 4])


@pytest.mark.parametrize("call", [
    lambda c, x, w: c.layer_norm(x, w[0, 0]),
    lambda c, x, w: c.layer_norm(x, want_stats=True)[0],
    lambda c, x, w: c.layer_norm(x.detach(), None, w[0, 0]),
    lambda c, x, w: c.layer_norm_backward(x, x.detach(), torch.zeros(4), torch.zeros(4))[0],
    lambda c, x, w: c.layer_norm_backward(x.detach(), x.detach(), torch.zeros(4), torch.zeros(4), w[0, 0])[2],
    lambda c, x, w: c.dropout(x, 0.5, 1),
    lambda c, x, w: c.dropout(x.detach(), 0.5, 1, residual=x),
    lambda c, x, w: c.grouped_mm(x, w.detach(), OFFSETS),
    lambda c, x, w: c.grouped_mm(x.detach(), w, OFFSETS),
    lambda c, x, w: c.grouped_mm(x.detach(), w.detach(), OFFSETS, bias=w[:, 0]),
    lambda c, x, w: c.grouped_mm_backward(x, x.detach(), w.detach(), OFFSETS)[1],
    lambda c, x, w: c.grouped_mm_backward(x.detach(), x, w, OFFSETS)[2],
])
def test_a_gradient_is_not_lost_silently(call):
    """The calls have gradients of their own and none for autograd: a backward pass through them says so, and does not leave them out."""
    x, w = torch.zeros(4, 4, requires_grad=True), torch.zeros(2, 4, 4, requires_grad=True)
    out = call(_idle(), x, w)
    with pytest.raises(DistShapError, match="backward"):
        (out.nan_to_num().sum() + x.sum() + w.sum()).backward()
    with torch.no_grad():
        assert not call(_idle(), x, w).requires_grad
    assert not call(_idle(), x.detach(), w.detach()).requires_grad
