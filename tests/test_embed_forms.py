"""Which form the gradient of a table takes: one launch, which needs no workspace, or rows sorted first. From the sizes alone, so it needs no GPU."""
import ctypes as C

import pytest

from paper_2506_22668_amd import binding


def in_one_launch(rows, cols, vocab):
    need = C.c_int64()
    assert binding.load_library().ds_embed_backward_workspace(rows, cols, vocab, C.byref(need)) == 0
    return need.value == 0


# Both forms were timed at these sizes (128 columns of bf16, ids evenly spread): where one takes 1.3 times the other it is not chosen
@pytest.mark.parametrize("rows, vocab, one", [
    (1000, 4096, True), (2000, 4096, True), (4000, 4096, True), (8000, 4096, True), (4000, 1024, True), (4000, 128, True), (1000, 128, True), (2000, 32, True),
    (1000, 32, True), (1000, 8, True), (4000, 8, False), (3000, 8, False), (4000, 1, False), (8000, 8, False), (8000, 1, False), (8000, 32, False)])
def test_the_faster_form_is_chosen(rows, vocab, one):
    assert in_one_launch(rows, 128, vocab) == one


@pytest.mark.parametrize("cols", [8, 64, 128])
def test_borders(cols):
    """1,024 rows to a workgroup, 4,096 rows of fewer than 512 ids, 8,192 of more."""
    assert in_one_launch(1024, cols, 8) and not in_one_launch(1025, cols, 8)
    assert in_one_launch(1024, cols, 1) and not in_one_launch(1025, cols, 1)
    assert in_one_launch(2048, cols, 16) and not in_one_launch(2049, cols, 16)
    assert in_one_launch(4096, cols, 511) and not in_one_launch(4097, cols, 511)
    assert in_one_launch(8192, cols, 512) and not in_one_launch(8193, cols, 512)
