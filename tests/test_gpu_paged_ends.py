"""The paged operators where a definition decides a single bit: codes of exact ties, float queries that round past the largest bf16 number, infinite values whose probability is 0."""
import math

import pytest
import torch

import paper_2601_11676_amd as H
from tests.test_gpu_paged_chunk import Case
from tests.test_gpu_paged_q8 import DEV, Append

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


def test_float_queries_past_the_largest_bf16_number_over_codes():
    # Rounded to one bf16 number such a query would be an infinity, and with a code of 0 NaN.  Head 0: the largest float, codes of 0 there, the rest as it is; head 1: 255.7 * 2^120 (of
    # more the first two parts may add up to 2^128), codes of 0 and 1 and scales of some 2^-126, which leave scores of up to 2.
    D, n = 64, 50
    g = torch.Generator().manual_seed(32)
    shape = H.PagedShape(2, 2, D, 16, 4, 4, "f32")
    k, v = (torch.randint(-127, 128, shape.pool, generator=g, dtype=torch.int8) for _ in range(2))
    ks, vs = (0.005 + 0.02 * torch.rand(shape.pool[:3], generator=g) for _ in range(2))
    q = torch.randn(1, 2, D, generator=g)
    q[0, 0, 20], q[0, 1, 20] = torch.finfo(torch.float32).max, 255.7 * 2.0 ** 120
    k[:, 0, :, 20] = 0
    k[:, 1, :, 20] = torch.randint(0, 2, (4, 16), generator=g, dtype=torch.int8)
    ks[:, 1] = (1 + 3 * torch.rand(4, 16, generator=g)) * 2.0 ** -126
    out = torch.empty(1, 2, D, device=DEV)
    ws = torch.empty(H.halo_paged_workspace_bytes(shape, 1), dtype=torch.uint8, device=DEV)
    H.halo_paged_attention_q8(shape, q.to(DEV), (k.to(DEV), ks.to(DEV)), (v.to(DEV), vs.to(DEV)), torch.arange(4, dtype=torch.int32, device=DEV)[None],
                              torch.tensor([n], dtype=torch.int32, device=DEV), n, out, ws, scale=0.125)
    out = out.cpu().double()
    assert torch.isfinite(out).all()
    kk, vv = ((c.double() * s.double()[..., None]).transpose(0, 1).reshape(2, 64, D)[:, :n] for c, s in ((k, ks), (v, vs)))
    for h in range(2):
        x, F = q[0, h].double(), 2.0 ** -24
        p = torch.softmax(kk[h] @ x * 0.125, 0)
        # scores off by three passes of D roundings of sum |q k|, scale and exponent by a few, sums of n: as where all queries are ordinary
        S = 0.125 * float((kk[h].abs() @ x.abs()).max())
        off = 2 * F * (6 * D * S + 12 * S + 3 * n + 80) * (p @ vv[h].abs())
        assert torch.all((out[0, h] - p @ vv[h]).abs() <= off + F * (p @ vv[h]).abs())


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hk,D,past,new", [(2, 2, 64, 300, 40), (4, 1, 128, 200, 100), (1, 1, 256, 150, 90), (64, 32, 64, 0, 700)])
@pytest.mark.parametrize("low", [-math.inf, -400.0])
def test_infinite_values_whose_probability_is_0(kind, Hq, Hk, D, past, new, low):
    # Elements of 0 * infinity are NaN, whatever the tile: positions that all rows of a block see, and positions among the block's own.  Infinities that count stay infinities, and
    # rows before such positions keep their bits.  low: the score of those positions (exp of -400 and less is 0 in float); -infinity only of bf16 (infinite float keys give NaN).
    if low == -math.inf and kind == "f32":
        low = -3.0e38
    case = Case(kind, Hq, Hk, D, 16, [(past, new)], seed=33, sigma=0.2)
    case.q = case.q.clone()
    case.q[..., 0] = 1.0                                              # scores: what key element 0 has, and little else
    n, s = past + new, case.shape
    for j in range(n):
        case.k[int(case.table[0, j // 16]), :, j % 16, 0] = 0.0
    clean = case.run()
    none = sorted({7, past + 9, past + new // 2, n - 5})              # probability 0, of all rows that see them
    full = [past + 21, n - 3]                                         # ordinary ones
    for j, (value, dim) in [(j, (math.inf, 3)) for j in none] + [(j, (-math.inf, 5)) for j in full]:
        page, row = int(case.table[0, j // 16]), j % 16
        case.v[page, :, row, dim] = value
        if dim == 3:
            case.k[page, :, row, 0] = low if math.isinf(low) or low < -1e30 else low / case.scale
    got = case.run()
    for i in range(new):
        pos = past + i
        seen = [j for j in none if j <= pos]
        assert torch.isnan(got[i, :, 3]).all() if seen else torch.isfinite(got[i, :, 3]).all(), (i, got[i, :, 3])
        if any(j <= pos for j in full):
            assert torch.all(got[i, :, 5] == -math.inf), i
        else:
            assert torch.isfinite(got[i, :, 5]).all(), i
        other = [d for d in range(D) if d not in (3, 5)]
        assert torch.isfinite(got[i][:, other]).all()
    first = min(none + full)
    if first >= past:
        assert torch.equal(got[:first - past], clean[:first - past])
