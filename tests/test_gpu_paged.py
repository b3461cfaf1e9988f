"""Appending to a paged cache, attention over its pages and the norms around a block, on the GPU against the oracle in double.

Tolerances are bounds, derived from the roundings that a result goes through: u = finfo(type).eps / 2 for the one that stores it, and for
attention in bf16 two of each probability, the second of what the first left; float operations count 2^-24 each, worst case."""
import numpy as np
import pytest
import torch

import paper_2601_11676_amd as H
from oracle import ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
F = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def normal(g, shape, dtype, sigma=1.0):
    return (torch.randn(shape, generator=g) * sigma).to(DT[dtype])


def np64(t):
    return t.detach().cpu().double().numpy()


# ---------------------------------------------------------------- append
def append_case(dtype, Hq, Hk, D, page, lens, rotary, pairs, seed=0, fused=True, shuffle=False):
    """Sequences with (past, new) tokens each; everything of the pools that no sequence has yet is NaN."""
    g = gen(seed)
    need = [(p + n + page - 1) // page for p, n in lens]
    n_pages, width = sum(need) + 2, max(need) + 1
    ids = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), width), -7, dtype=torch.int32)
    at = 0
    for i, c in enumerate(need):
        table[i, :c] = ids[at:at + c]
        at += c
    seq = torch.tensor([i for i, (_, n) in enumerate(lens) for _ in range(n)], dtype=torch.int32)
    pos = torch.tensor([p + j for p, n in lens for j in range(n)], dtype=torch.int32)
    if shuffle:
        order = torch.randperm(len(seq), generator=g)
        seq, pos = seq[order], pos[order]
    N = len(seq)
    if fused:
        rows = normal(g, (N, Hq + 2 * Hk + 1, D), dtype)             # one head more than is used between tokens
        q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:Hq + 2 * Hk]
    else:
        q, k, v = (normal(g, (N, h, D), dtype) for h in (Hq, Hk, Hk))
    shape = H.PagedShape(Hq, Hk, D, page, n_pages, width, dtype)
    rope = H.halo_rope_table(max(p + n for p, n in lens), rotary) if rotary else None
    pool = torch.full(shape.pool, float("nan"), dtype=DT[dtype])
    return shape, q, k, v, pos, seq, table, rope, pairs, pool


def on_device(view):
    """The same view of the same strides on the GPU."""
    base = view if view._base is None else view._base
    return torch.as_strided(base.to(DEV), view.shape, view.stride(), view.storage_offset())


def run_append(case, with_q=True, stream=None):
    shape, q, k, v, pos, seq, table, rope, pairs, pool = case
    kp, vp = pool.to(DEV), pool.to(DEV)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device=DEV) if with_q else None
    H.halo_paged_append(shape, on_device(q) if with_q else None, on_device(k), on_device(v), pos.to(DEV), table.to(DEV), kp, vp, q_out=out,
                        rope=None if rope is None else torch.from_numpy(rope).to(DEV), rope_pairs=pairs,
                        seq=None if seq is None else seq.to(DEV), stream=stream)
    torch.cuda.synchronize()
    return out, kp, vp


def check_append(case, got):
    shape, q, k, v, pos, seq, table, rope, pairs, pool = case
    args = (np64(q), np64(k), np64(v), pos.numpy(), None if seq is None else seq.numpy(), table.numpy(), rope, pairs, np64(pool), np64(pool))
    want = ref.paged_append(*args)
    # |a cos| + |b sin| of each element: the same turn with nothing but additions
    size = ref.paged_append(np.abs(args[0]), np.abs(args[1]), np.abs(args[2]), *args[3:6],
                            None if rope is None else np.abs(rope) * [[[1.0], [-1.0]]], pairs, np64(pool), np64(pool))
    size2 = ref.paged_append(np.abs(args[0]), np.abs(args[1]), np.abs(args[2]), *args[3:6], None if rope is None else np.abs(rope), pairs,
                             np64(pool), np64(pool))
    for name, g, w, s, s2 in zip(("q", "k", "v"), got, want, size, size2):
        if g is None:
            continue
        g = np64(g)
        assert np.array_equal(np.isnan(g), np.isnan(w)), name          # the rest of the pool is untouched
        bound = U[shape.dtype] * np.abs(w) + 3 * F * np.maximum(np.abs(s), np.abs(s2)) * (1 + U[shape.dtype])
        bad = np.abs(g - w) > bound
        assert not np.any(bad & ~np.isnan(w)), (name, np.argwhere(bad & ~np.isnan(w))[:3])
    assert np.array_equal(np.nan_to_num(np64(got[2])), np.nan_to_num(want[2]))       # values are moved, not computed


APPENDS = [("bf16", 8, 2, 128, 16, [(0, 1)], 128, False), ("bf16", 32, 32, 128, 16, [(15, 1), (16, 1), (300, 1)], 128, False),
           ("bf16", 6, 2, 64, 32, [(0, 70), (31, 2), (5, 0), (100, 33)], 32, True), ("f32", 4, 4, 16, 16, [(3, 20)], 16, False),
           ("f32", 5, 1, 80, 64, [(60, 9), (0, 1)], 48, True), ("f32", 3, 3, 256, 256, [(255, 2)], 256, False),
           ("bf16", 7, 7, 96, 16, [(0, 40)], 96, True), ("bf16", 16, 1, 256, 16, [(9, 600)], 128, False),
           ("bf16", 2, 1, 112, 4096, [(4090, 10)], 0, False), ("bf16", 64, 8, 128, 16, [(7, 530), (0, 61)], 128, False)]


@pytest.mark.parametrize("args", APPENDS, ids=lambda a: "-".join(map(str, a[:5])))
def test_append(args):
    case = append_case(*args)
    check_append(case, run_append(case))


def test_append_tokens_in_any_order_and_dense():
    case = append_case("bf16", 4, 2, 64, 16, [(0, 37), (12, 5), (40, 1)], 64, False, fused=False, shuffle=True)
    check_append(case, run_append(case))


def test_append_one_token_of_each_sequence_without_a_list():
    case = list(append_case("f32", 4, 2, 32, 16, [(4, 1), (16, 1), (31, 1)], 32, False))
    case[5] = None
    check_append(case, run_append(case))


def test_append_without_queries():
    case = append_case("bf16", 4, 2, 64, 16, [(0, 20)], 64, False)
    check_append(case, run_append(case, with_q=False))


def test_append_padding_writes_nothing():
    # sequences, positions and pages that are none, one of each kind between good tokens
    case = list(append_case("bf16", 4, 2, 64, 16, [(0, 12), (10, 4)], 64, False))
    pos, seq, table = case[4].clone(), case[5].clone(), case[6].clone()
    pos[1], pos[3], pos[5] = -1, 1 << 30, 14                          # the last: past the table of angles
    seq[7], seq[9] = -1, 2
    table[1, 0] = case[0].n_pages                                     # sequence 1's first page is none: its tokens 12 .. 15
    case[4], case[5], case[6] = pos, seq, table
    out, kp, vp = run_append(case)
    check_append(case, (out, kp, vp))
    gone = [1, 3, 5, 7, 9, 12, 13, 14, 15]
    assert torch.all(out[gone] == 0) and not torch.any(out[[0, 2, 4, 6, 8, 10, 11]] == 0)
    assert int((~torch.isnan(vp[:, 0, :, 0])).sum()) == 7


# ---------------------------------------------------------------- attention
def attend_case(dtype, Hq, Hk, D, page, lens, keep=None, seed=0, garbage=True, sigma=2.0, extra=1):
    g = gen(seed)
    need = [max(0, (n + page - 1) // page) for n in lens]
    n_pages, width = sum(need) + 2, max(need) + extra
    ids = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), width), -3, dtype=torch.int32)
    if garbage:
        table[:] = int(ids[-1])                                       # a page that exists, of NaN
    shape = H.PagedShape(Hq, Hk, D, page, n_pages, width, dtype)
    kp, vp = (torch.full(shape.pool, float("nan") if garbage else 0.0, dtype=DT[dtype]) for _ in range(2))
    at = 0
    for i, (n, c) in enumerate(zip(lens, need)):
        table[i, :c] = ids[at:at + c]
        at += c
        for p in (kp, vp):
            rows = normal(g, (c * page, Hk, D), dtype)
            if garbage:
                rows[n:] = float("nan")
            p[table[i, :c].long()] = rows.view(c, page, Hk, D).transpose(1, 2)
    q = normal(g, (len(lens), Hq, D), dtype, sigma)
    mask = None
    if keep is not None:
        mask = (torch.rand((len(lens), Hq), generator=g) < keep).to(torch.uint8)
    return shape, q, kp, vp, table, torch.tensor(lens, dtype=torch.int32), mask


def run_attend(case, max_len=None, scale=None, stream=None):
    shape, q, kp, vp, table, lens, mask = case
    T = q.shape[0]
    ws = torch.full((H.halo_paged_workspace_bytes(shape, T),), 0xff, dtype=torch.uint8, device=DEV)      # all NaN
    out = torch.full((T, shape.n_heads, shape.head_dim), float("nan"), dtype=q.dtype, device=DEV)
    dev = [x.to(DEV) for x in (kp, vp, table, lens)]
    H.halo_paged_attention(shape, on_device(q), *dev, max(1, int(lens.max())) if max_len is None else max_len, out, ws,
                           mask=None if mask is None else mask.to(DEV), scale=scale, stream=stream)
    torch.cuda.synchronize()
    return out


def attend_bound(case, want, lens, scale=None):
    """|error| <= u |o| (storing) + [bf16: u^2 (W + |o|), each weight off by two roundings in numerator and sum] + the float sums': scores off by D roundings
    of sum |q k|, then as an exponent; exponentials and the sums over the positions in float.  W = sum_j p_j |v_j|."""
    shape, q, kp, vp, table, _, mask = case
    scale = abs(shape.head_dim ** -0.5 if scale is None else scale)
    W = ref.paged_attention(np64(q), np64(kp), np.abs(np64(vp)), table.numpy(), lens, None if mask is None else mask.numpy(),
                            shape.head_dim ** -0.5 if scale is None else scale)
    u = U[shape.dtype]
    k = np.nan_to_num(np64(kp))
    S = scale * float(np.sqrt((np64(q) ** 2).sum(-1).max() * (k ** 2).sum(-1).max()))      # no sum |q k| is larger
    gamma = F * (2 * shape.head_dim * S + 8 * S + float(max(1, np.max(lens))) + 64)
    rounded = 0.0 if shape.dtype == "f32" else u * u * (W + np.abs(want)) * (1 + 2 * u)
    return u * np.abs(want) + (rounded + 2 * gamma * W) * (1 + u)


def check_attend(case, got, max_len=None, scale=None):
    shape, q, kp, vp, table, lens, mask = case
    lens = lens.numpy() if max_len is None else np.minimum(lens.numpy(), max_len)
    want = ref.paged_attention(np64(q), np64(kp), np64(vp), table.numpy(), lens, None if mask is None else mask.numpy(), scale)
    got = np64(got)
    assert np.all(np.isfinite(got))
    off = np.abs(got - want) - attend_bound(case, want, lens, scale)
    assert np.all(off <= 0), (np.argwhere(off > 0)[:4], off.max())
    assert np.all(got[want == 0] == 0)


SHORT = [1, 15, 16, 17, 31, 32, 33, 47, 48, 64, 255, 256, 257]
ATTENDS = [
    ("bf16", 4, 4, 128, 16, SHORT, None), ("bf16", 8, 2, 64, 16, SHORT, None), ("f32", 4, 2, 64, 32, SHORT, None),
    ("f32", 3, 3, 128, 16, [1, 40, 100], None), ("bf16", 8, 1, 256, 16, [5, 70, 300], None), ("f32", 4, 1, 256, 64, [3, 70], None),
    ("bf16", 5, 5, 16, 16, [1, 33, 200], None), ("bf16", 6, 2, 80, 64, [1, 33, 200], None), ("f32", 6, 2, 96, 16, [17, 200], None),
    ("f32", 4, 4, 48, 256, [17, 200], None), ("bf16", 4, 2, 144, 16, [9, 90], None), ("f32", 4, 2, 208, 16, [9, 90], None),
    ("bf16", 16, 1, 128, 16, [50, 3], None), ("bf16", 20, 1, 128, 16, [50, 3], None), ("bf16", 66, 2, 64, 32, [100], None),
    ("f32", 40, 2, 64, 16, [100, 20], None), ("bf16", 256, 256, 16, 16, [20, 40], 0.5), ("bf16", 8, 2, 128, 16, [0, 30, 0, 99], None),
    ("bf16", 32, 32, 128, 16, [301], 0.5), ("bf16", 12, 4, 96, 32, SHORT, 0.4), ("f32", 16, 8, 64, 16, [0, 77, 5, 300], 0.3),
    # longer ones: cut over the grid and joined
    ("bf16", 8, 8, 128, 16, [2000, 1, 0, 1025, 3000], 0.6), ("bf16", 64, 8, 128, 64, [5003], None), ("f32", 4, 2, 64, 32, [3000, 40], None),
    ("bf16", 40, 2, 64, 16, [1500, 700, 33], 0.5), ("bf16", 20, 1, 256, 256, [1100, 64], 0.7), ("f32", 2, 1, 240, 16, [1100, 900], None),
    ("bf16", 2, 2, 80, 16, [1600] * 3, None), ("bf16", 1, 1, 128, 4096, [9000], None), ("f32", 6, 6, 112, 16, [1030, 2, 1500], 0.5),
    ("bf16", 16, 2, 64, 16, [50 + 37 * i for i in range(70)], 0.5), ("f32", 1, 1, 16, 16, [6000], None),
    ("bf16", 130, 130, 32, 16, [1100, 40], 0.3), ("bf16", 130, 130, 32, 16, [2100, 40], 0.3), ("bf16", 2, 2, 80, 16, [2600] * 3, None),
    ("bf16", 40, 2, 64, 16, [2500, 700, 33], 0.5), ("bf16", 8, 2, 128, 128, [2048, 2047], None), ("bf16", 8, 2, 128, 128, [2049, 1], None),
    # more than 16 queries a cache head, of caches large enough to be read once: 32 at a time
    ("bf16", 40, 2, 128, 16, [2000, 33, 0, 1500] * 17, 0.6), ("bf16", 34, 2, 64, 32, [2500] + [7 * i for i in range(130)], 0.5),
    ("bf16", 96, 2, 96, 16, [5000, 700] * 9, 0.3), ("bf16", 17, 1, 48, 16, [3000 + i for i in range(140)], None),
    ("f32", 24, 8, 96, 16, [600] * 10, 0.6), ("f32", 16, 4, 64, 16, SHORT + [1100], 0.7), ("f32", 5, 1, 64, 16, SHORT, None),
    ("f32", 10, 2, 128, 16, [2000, 45, 700], None), ("f32", 8, 2, 128, 32, [1700, 45, 700], 0.6), ("f32", 30, 6, 240, 16, [40, 900], None),
    ("f32", 4, 1, 32, 16, [7000, 2], None), ("f32", 6, 6, 256, 16, [700, 33], None), ("bf16", 64, 64, 48, 16, [300 * i for i in range(9)], 0.5),
    # short caches of many sequences, and many a little longer: fewer waves a workgroup
    ("bf16", 16, 8, 128, 16, [1 + i % 16 for i in range(70)], 0.7), ("bf16", 8, 8, 64, 32, [3 * i for i in range(80)], 0.6),
    ("f32", 32, 8, 64, 16, [2 * i for i in range(64)], None), ("f32", 48, 4, 128, 16, [(5 * i) % 321 for i in range(130)], 0.6),
    ("bf16", 40, 8, 80, 16, [257 + 5 * i for i in range(65)], 0.6), ("bf16", 4, 4, 256, 16, [(7 * i) % 129 for i in range(129)], 0.5),
    ("bf16", 64, 32, 128, 16, [(11 * i) % 257 for i in range(70)], 0.5), ("f32", 4, 4, 256, 64, [20, 32, 0, 1], None),
    ("bf16", 32, 8, 128, 16, [64, 63, 0, 1, 33], 0.5), ("bf16", 32, 8, 128, 16, [600 - i for i in range(64)], None),
    ("bf16", 16, 16, 128, 16, [500 + i % 100 for i in range(64)], 0.8),
    # float with more than 16 queries a cache head, of large caches; and such queries over many short caches
    ("f32", 40, 2, 128, 16, [2000, 33, 0, 1500] * 9, 0.6), ("f32", 34, 2, 64, 32, [2500] + [7 * i for i in range(70)], 0.5),
    ("f32", 96, 2, 96, 16, [5000, 700] * 5, 0.3), ("f32", 17, 1, 48, 16, [1500 + i for i in range(140)], None),
    ("f32", 160, 8, 128, 16, [(11 * i) % 129 for i in range(80)], 0.5), ("f32", 64, 2, 128, 16, [(7 * i) % 257 for i in range(260)], None),
    ("f32", 40, 2, 96, 64, [1020 - i for i in range(50)], 0.4), ("bf16", 160, 8, 128, 16, [(11 * i) % 257 for i in range(80)], 0.5),
    ("bf16", 66, 2, 64, 16, [(13 * i) % 513 for i in range(260)], 0.7), ("bf16", 34, 2, 80, 16, [300 + i % 200 for i in range(260)], None),
    ("f32", 20, 1, 16, 16, [40000, 30000, 5], None),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seqs,longest", [(3, 30), (140, 60), (140, 200)])
def test_rows_of_short_caches_that_the_mask_leaves_empty(dtype, seqs, longest):
    case = attend_case(dtype, 8, 4, 64, 16, [(longest - 7 * i) % (longest + 1) for i in range(seqs)], keep=0.5, seed=9)
    mask, lens = case[6], case[5]
    mask[0] = 0
    mask[1, :2], mask[1, 2:] = 0, 255
    got = run_attend(case)
    check_attend(case, got)
    assert torch.all(got[0] == 0) and torch.all(got[1, :2] == 0) and torch.all(got[1, 2:] != 0) and torch.all(got.cpu()[lens.cpu() == 0] == 0)


@pytest.mark.parametrize("args", ATTENDS, ids=lambda a: "-".join(map(str, a[:5])) + f"-{max(a[5])}x{len(a[5])}")
def test_attention(args):
    case = attend_case(*args[:6], keep=args[6])
    check_attend(case, run_attend(case))


@pytest.mark.parametrize("longest", [900, 3000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_the_mask_leaves_empty(dtype, longest):
    case = attend_case(dtype, 8, 2, 64, 16, [longest, 40, 300, 0, 17], keep=0.5, seed=4)
    mask = case[6]
    mask[0] = 0
    mask[1] = 1
    mask[2, :4] = 0                                                   # a head of the cache without a survivor
    mask[2, 5] = 255                                                  # any byte but 0
    got = run_attend(case)
    check_attend(case, got)
    assert torch.all(got[0] == 0) and torch.all(got[3] == 0) and torch.all(got[2, :4] == 0) and torch.all(got[2, 5] != 0)
    mask[:] = 0
    assert torch.all(run_attend(case) == 0)


@pytest.mark.parametrize("longest", [900, 2500])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_out_of_bounds_and_pages_that_are_none(dtype, longest):
    case = list(attend_case(dtype, 4, 2, 64, 16, [longest, 100, 64, 200, 48], seed=5))
    shape, q, kp, vp, table, lens, mask = case
    table[1, 2], table[1, 3], table[2, :4] = -1, shape.n_pages, -(1 << 31)        # holes; a sequence without any page
    table[3, 12] = (1 << 31) - 1
    lens[4] = -5
    got = run_attend(case)
    check_attend(case, got)
    assert torch.all(got[2] == 0) and torch.all(got[4] == 0) and torch.all(got[[0, 1, 3]] != 0)
    # lengths past max_len count as max_len
    lens[0] = 1 << 30
    check_attend(case, run_attend(case, max_len=longest - 3), max_len=longest - 3)


@pytest.mark.parametrize("longest", [700, 1900, 2500])
def test_nan_stays_in_its_query(longest):
    # queries of NaN beside good ones of the same cache head, masked or not: the others' results keep their bits
    case = list(attend_case("bf16", 8, 2, 128, 16, [longest, 50], seed=6))
    clean = run_attend(case)
    case[1] = case[1].clone()
    case[1][0, 1] = float("nan")
    case[1][1, 6] = float("inf")
    got = run_attend(case)
    keep = torch.ones(2, 8, dtype=torch.bool)
    keep[0, 1] = keep[1, 6] = False
    assert torch.equal(got.cpu()[keep], clean.cpu()[keep]) and torch.all(torch.isnan(got.cpu()[0, 1]))
    case[6] = keep.to(torch.uint8)
    got = run_attend(case)
    assert torch.equal(got.cpu()[keep], clean.cpu()[keep]) and torch.all(got.cpu()[~keep] == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("longest", [300, 2000, 4100])
def test_far_apart_scores(dtype, longest):
    # one key far above, then far below the rest, scores of several hundred: the maximum moves in any step
    case = attend_case(dtype, 4, 4, 64, 16, [longest, longest - 20, 100], seed=7, garbage=False)
    shape, q, kp, vp, table, lens, _ = case
    for t, n in enumerate([longest, longest - 20, 100]):
        for h, j in enumerate([0, n // 2, n - 1, 70]):
            kp[table[t, j // 16], h, j % 16] = (q[t, h].float() * (30.0 if h < 3 else -30.0)).to(kp.dtype)
    got = run_attend(case)
    check_attend(case, got)
    # a row with one dominant token is that token's values, bit for bit: its probability is the same in the product and in the sum
    for h, j in enumerate([0, 50, 99] if dtype == "bf16" else []):
        assert torch.equal(got[2, h].cpu(), vp[table[2, j // 16], h, j % 16])


def test_scales():
    case = attend_case("f32", 4, 2, 64, 16, [100, 40], seed=8)
    for scale in (0.0, 1.0, -0.125):
        check_attend(case, run_attend(case, scale=scale), scale=scale)


def test_tokens_apart_and_pages_shared():
    # queries as a view of a fused projection's rows; two sequences with the same first pages, one page twice in a row
    case = list(attend_case("bf16", 8, 4, 64, 16, [200, 150, 100], seed=9))
    rows = normal(gen(1), (3, 8 + 2 * 4, 64), "bf16", 2.0)
    case[1] = rows[:, :8]
    table = case[4]
    table[1, :5] = table[0, :5]
    table[2, 3] = table[2, 2]
    check_attend(case, run_attend(case))


@pytest.mark.parametrize("longest", [600, 4000])
def test_attention_repeats_its_bits_on_any_stream(longest):
    case = attend_case("bf16", 8, 2, 128, 16, [longest, 77, 400], keep=0.7, seed=10)
    first = run_attend(case)
    other = torch.cuda.Stream()
    for s in (None, other, None):
        assert torch.equal(run_attend(case, stream=s), first)


def test_a_larger_bound_or_workspace_changes_no_length():
    # max_len only bounds: both ways of cutting agree with the oracle for the same short sequences
    case = attend_case("bf16", 8, 2, 64, 16, [60, 300, 7], seed=11, extra=200)
    for m in (300, 1000, 1025, 2048, 2049, 3000):
        check_attend(case, run_attend(case, max_len=m))


def test_many_sequences():
    case = attend_case("bf16", 2, 1, 16, 16, [(i * 7) % 40 for i in range(4096)], keep=0.8, seed=12)
    check_attend(case, run_attend(case))
    for last in (1500, 9000):
        case = attend_case("bf16", 2, 1, 16, 16, [(i * 7) % 40 for i in range(4095)] + [last], keep=0.8, seed=12)
        check_attend(case, run_attend(case))


@pytest.mark.parametrize("dtype,D,longest", [("bf16", 128, 1500), ("bf16", 128, 2300), ("f32", 64, 1700), ("f32", 64, 500)])
def test_pools_past_32_bits(dtype, D, longest):
    # the sequences' pages lie beyond 2^32 bytes and 2^31 elements of the pools, of which only they are ever written
    page, Hk = 256, 8
    n_pages = (1 << 31) // (page * Hk * D) + 40
    small = list(attend_case(dtype, 16, Hk, D, page, [longest, 300], seed=13, garbage=False))
    shape, q, kp, vp, table, lens, _ = small
    big = H.PagedShape(16, Hk, D, page, n_pages, shape.max_pages, dtype)
    far = torch.where(table >= 0, table + n_pages - shape.n_pages, table)
    pools = [torch.empty(big.pool, dtype=DT[dtype], device=DEV) for _ in range(2)]
    for p, s in zip(pools, (kp, vp)):
        p[n_pages - shape.n_pages:] = s.to(DEV)
    ws = torch.empty(H.halo_paged_workspace_bytes(big, 2), dtype=torch.uint8, device=DEV)
    rope = torch.from_numpy(H.halo_rope_table(3000, D)).to(DEV)
    k, v = (normal(gen(i), (2, Hk, D), dtype) for i in (1, 2))
    for pool, sh, tab in ((pools, big, far), ([kp.to(DEV), vp.to(DEV)], shape, table)):
        out = torch.empty(q.shape, dtype=q.dtype, device=DEV)
        q_rot = torch.empty_like(out)
        H.halo_paged_append(sh, q.to(DEV), k.to(DEV), v.to(DEV), (lens - 1).to(DEV), tab.to(DEV), *pool, q_out=q_rot, rope=rope)
        H.halo_paged_attention(sh, q_rot, *pool, tab.to(DEV), lens.to(DEV), longest, out, ws)
        torch.cuda.synchronize()
        if sh is big:
            first = out, q_rot, pool[0][n_pages - shape.n_pages:].clone(), pool[1][n_pages - shape.n_pages:].clone()
    for a, b in zip(first, (out, q_rot, *pool)):
        assert torch.equal(a, b)


# ---------------------------------------------------------------- norm
def norm_case(dtype, stream, T, d, post, gate, weights=True, seed=0):
    g = gen(seed)
    h, y = normal(g, (T, d), stream, 3.0), normal(g, (T, d), dtype)
    w = [normal(g, (d,), dtype) if weights else None for _ in range(2)]
    gt = {"none": None, "channel": normal(g, (d,), dtype), "token": normal(g, (T, d), dtype)}[gate]
    return h, y, w[0] if post else None, gt, w[1]


def check_norm(case, stream, dtype, post, s, eps, h2, x):
    h, y, w_post, gate, w_pre = (None if t is None else np64(t) for t in case)
    hw, xw = ref.block_norm(h, y, w_post, gate, w_pre, post, s, eps)
    d = h.shape[1]
    gu = np.abs(hw - np.float32(s).astype(np.float64) * h)
    # the sum of d squares is off by d roundings and its root by half of that; five more in the products; two in the residual
    ez = F * ((d / 2 + 8) * gu + 3 * (np.abs(s * h) + gu))
    assert np.all(np.abs(np64(h2) - hw) <= U[stream] * np.abs(hw) + ez * (1 + U[stream]))
    size = np.sqrt((hw ** 2).mean(1, keepdims=True) + eps)
    rel = F * (d / 2 + 8) + np.sqrt((ez ** 2).mean(1, keepdims=True)) / size
    ex = np.abs(xw) * rel + ez / size * (1.0 if w_pre is None else np.abs(w_pre))
    assert np.all(np.abs(np64(x) - xw) <= U[dtype] * np.abs(xw) + ex * (1 + U[dtype]) * 1.01 + 2.0 ** -126)


def run_norm(case, post, s, eps, in_place=False):
    h, y, w_post, gate, w_pre = (None if t is None else t.to(DEV) for t in case)
    x = torch.full(y.shape, float("nan"), dtype=y.dtype, device=DEV)
    h2 = None if in_place else torch.full(h.shape, float("nan"), dtype=h.dtype, device=DEV)
    H.halo_block_norm(h, y, x, h_out=h2, post_norm=post, w_post=w_post, gate=gate, res_scale=s, w_pre=w_pre, eps=eps)
    torch.cuda.synchronize()
    return h if in_place else h2, x


@pytest.mark.parametrize("dtype,stream", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("T,d", [(1, 8), (3, 64), (5, 512), (1, 520), (9, 1000), (2, 4096), (1, 8192), (3, 8200), (2, 16384), (2, 16392), (1, 32768)])
def test_norm(dtype, stream, T, d):
    for i, (post, gate, weights) in enumerate([(True, "channel", True), (False, "none", True), (True, "token", False), (False, "token", True)]):
        case = norm_case(dtype, stream, T, d, post, gate, weights, seed=i)
        check_norm(case, stream, dtype, post, 0.75, 1e-5, *run_norm(case, post, 0.75, 1e-5))


def test_norm_in_place_many_rows_and_zeros():
    case = norm_case("bf16", "f32", 2049, 264, True, "channel")
    case[0][7], case[1][7] = 0, 0                                    # a row of zeros: eps keeps it finite
    case[1][8] = 0
    got = run_norm(case, True, 1.0, 1e-5, in_place=True)
    check_norm(case, "f32", "bf16", True, 1.0, 1e-5, *got)
    assert torch.all(got[1][7] == 0)


def test_norm_with_output_over_y():
    case = norm_case("bf16", "bf16", 5, 4096, True, "none")
    want = run_norm(case, True, 1.0, 1e-5)
    h, y, w_post, _, w_pre = (None if t is None else t.to(DEV) for t in case)
    H.halo_block_norm(h, y, y, post_norm=True, w_post=w_post, w_pre=w_pre)
    torch.cuda.synchronize()
    assert torch.equal(h, want[0]) and torch.equal(y, want[1])


# ---------------------------------------------------------------- together
def test_step_in_a_graph():
    """append -> attention -> norm of a batch, captured once: every replay, with lengths and positions moved on between them, has the bits of
    the same calls made directly."""
    T, Hq, Hk, D, page, d = 5, 8, 2, 64, 16, 512
    case = attend_case("bf16", Hq, Hk, D, page, [1000, 40, 15, 1, 300], seed=20, garbage=False, extra=70)
    shape, q, kp, vp, table, lens, _ = [None if t is None else t.to(DEV) if isinstance(t, torch.Tensor) else t for t in case]
    k, v = (normal(gen(i), (T, Hk, D), "bf16").to(DEV) for i in (1, 2))
    rope = torch.from_numpy(H.halo_rope_table(2000, D)).to(DEV)
    pos = lens - 1
    ws = torch.empty(H.halo_paged_workspace_bytes(shape, T), dtype=torch.uint8, device=DEV)
    h0 = torch.randn((T, d), device=DEV)
    w = torch.randn(d, device=DEV).to(torch.bfloat16)
    q_rot, out = torch.empty_like(q), torch.empty_like(q)
    h, x = torch.empty_like(h0), torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
    for max_len in (1024, 2060):                                      # one launch, two
        def step():
            H.halo_paged_append(shape, q, k, v, pos, table, kp, vp, q_out=q_rot, rope=rope)
            H.halo_paged_attention(shape, q_rot, kp, vp, table, lens, max_len, out, ws)
            H.halo_block_norm(h0, out.view(T, -1), x, h_out=h, post_norm=True, w_post=w, w_pre=w)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for i in range(4):
            lens += 1
            pos += 1
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (q_rot, out, h, x, kp, vp)]
            for t in (q_rot, out, h, x):
                t.fill_(float("nan"))
            step()
            torch.cuda.synchronize()
            for a, b in zip(got, (q_rot, out, h, x, kp, vp)):
                assert torch.equal(a, b)
