"""Attention of chunks with heads above 128, whose tiles are 32 tokens, over sequences that a workgroup walks for more than 16 of them (blocks that are not cut, and parts of more), against
the formula in double, within test_gpu_paged_chunk's bounds."""
import pytest

from tests.test_gpu_paged_chunk import KINDS, Case, label

pytestmark = pytest.mark.gpu

LONG = [
    # as many blocks as the card has places, so that none is cut: past 512 and past 1024 positions (64 parts of 16 tokens, the window of page numbers, once and twice)
    (256, 256, 256, 16, [(1150, 3)], None), (256, 256, 144, 16, [(610, 1)], 0.7), (128, 128, 240, 64, [(1300, 140)], None), (256, 128, 208, 32, [(2100, 64), (520, 64)], 0.6),
    # cut into parts of 19 to 21 tiles
    (64, 64, 240, 16, [(2300, 2)], None), (64, 64, 256, 32, [(2250, 20)], 0.5), (120, 60, 144, 256, [(2200, 9)], None),
]


def keep_off_page_0(case):
    """The pool's first page swapped with one that no sequence has, whose rows are NaN."""
    t, free = case.table, int(case.table[0, -1])
    if free == 0:
        return
    at_0, at_free = t == 0, t == free
    t[at_0], t[at_free] = free, 0
    for pool in (*case.k, *case.v) if case.q8 else (case.k, case.v):
        pool[0], pool[free] = pool[free].clone(), pool[0].clone()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("args", LONG, ids=label)
def test_long_walks(args, kind):
    case = Case(kind, *args[:5], keep=args[5], seed=21)
    keep_off_page_0(case)
    case.check(case.run())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("args", [LONG[0], LONG[4]], ids=label)
def test_long_walks_over_pages_that_are_none(args, kind):
    case = Case(kind, *args[:5], seed=22)
    keep_off_page_0(case)
    (past, new), = case.runs
    for pos, none in zip((530, 555, 800, 1100, past + new - 1), (-1, case.shape.n_pages, -(1 << 31), -1, -1)):
        case.table[0, pos // case.shape.page_size] = none
    case.check(case.run())
