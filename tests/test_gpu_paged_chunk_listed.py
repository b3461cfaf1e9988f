"""Attention of chunks where surviving rows are listed and sequences are more than a wave's lanes, and batches whose starts name rows that do not exist, against the formula in double,
within test_gpu_paged_chunk's bounds."""
import pytest
import torch

from tests.test_gpu_paged_chunk import KINDS, Case, label

pytestmark = pytest.mark.gpu

# at least 2e8 scores of the longest sequence; the kernels in the order of their blocks: 32, 128 and 256 rows, cut; 128 rows, whole
LISTED = [(64, 4, 16, 16, [(i % 37, 1 + i % 2) for i in range(99)] + [(21500, 1)], 0.5), (64, 1, 64, 16, [((7 * i) % 50, i % 3) for i in range(66)] + [(0, 0)] * 8 + [(22000, 80)], 0.4),
          (16, 1, 16, 32, [((5 * i) % 70, 12 + i % 5) for i in range(70)] + [(12500, 33)], 0.7), (256, 64, 16, 64, [(i % 9, 11) for i in range(80)] + [(1500, 40)], 0.3)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("args", LISTED, ids=label)
def test_listed_rows_of_many_sequences(kind, args):
    case = Case(kind, *args[:5], keep=args[5], seed=23)
    assert case.N * case.shape.n_heads * case.max_len >= 200000000 and len(case.runs) > 64
    got = case.run()
    case.check(got)
    assert torch.all(got[case.mask == 0] == 0)


@pytest.mark.parametrize("kind", KINDS)
def test_rows_that_do_not_exist_are_not_counted(kind):
    # starts from before the first row to behind the last: what exists are the sequences' last tokens
    case = Case(kind, 4, 2, 64, 16, [(60, 30), (0, 5), (200, 40)], keep=0.8, seed=24)
    want, off = case.want()
    case.starts[0], case.starts[-1] = -7, case.N + 11
    got = case.run().double()
    assert torch.all((got - want).abs() <= off)
