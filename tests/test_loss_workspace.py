"""Scratch memory of the losses: what is enough for many rows of many columns is enough for fewer, so that a program keeps one for its largest batch."""
import os

import pytest

from paper_2605_26444_amd import binding as B


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2605_26444_amd import build
        build.build()
    return B.lib()


@pytest.mark.parametrize("V", [1, 33, 4096, 4097, 9001, 32000, 128256, 152064, 2 ** 24, 2 ** 30])
def test_fewer_rows_take_no_more(V):
    sizes = [B.nanospec_loss_workspace(rows, V) for rows in list(range(1, 5000)) + [2 ** 15, 2 ** 22]]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("rows", [1, 2, 7, 37, 127, 128, 509, 1021, 2047, 2048, 2049, 4096, 2 ** 22])
def test_fewer_columns_take_no_more(rows):
    sizes = [B.nanospec_loss_workspace(rows, V) for V in list(range(1, 300000, 61)) + [2 ** 20 + 1, 2 ** 30]]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_the_parts_fit():
    """a pair of 8 bytes a piece of a row -- at most 2048 pieces beside a row's first, of 4096 columns each -- and 32 bytes a row"""
    for rows in (1, 5, 100, 1999, 2048, 70000):
        for V in (1, 4096, 4097, 128256, 2 ** 30):
            pieces = min(-(-2048 // rows), -(-V // 4096))
            assert B.nanospec_loss_workspace(rows, V) >= 8 * rows * pieces + 32 * rows
