"""The paged operators where a definition decides a single bit: codes of exact ties."""
import pytest
import torch

from tests.test_gpu_paged_q8 import Append

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,coarse", [("bf16", True), ("f32", True), ("f32", False)])
def test_ties_of_ordinary_rows_go_to_even(dtype, coarse):
    # rint(127 x / max|x|): 127 x is exact in double, the quotient is rounded once, and no quotient of such numbers that is no tie lies within 2^-35 of one (max has at most 24 bits,
    # |x| no less than max / 508 where a border is near), so its rounding to 2^-47 decides nothing.  Rows of bf16 numbers have ties by themselves, also as floats (coarse).
    case = Append(dtype, 8, 8, 128, 16, [(0, 300)], 0, False, seed=31)
    if coarse:
        case.rows = case.rows.to(torch.bfloat16).to(case.rows.dtype)
    _, k, v = case.heads(case.rows)
    _, pools = case.run(True, norm=False)
    page, row, _ = case.there()
    ties = 0
    for x, (codes, _) in zip((k.double(), v.double()), pools):
        quotient = 127.0 * x / x.abs().amax(-1, keepdim=True)
        ties += int((quotient - torch.floor(quotient) == 0.5).sum())
        assert torch.equal(codes.cpu()[page, :, row].double(), torch.round(quotient))
    assert not coarse or ties > 500                                   # of 614400
