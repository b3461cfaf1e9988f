"""Attention over a paged cache where single terms of its sums show: queries and keys that make the scores exact, values that cancel.  Against the
oracle in double, as tests/test_gpu_paged.py."""
import numpy as np
import pytest
import torch

import paper_2601_11676_amd as H
from oracle import ref

DEV = "cuda"
F = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def paged(dtype, Hq, Hk, D, page, lens, max_len, seed=0):
    """A call's shape, page table (scattered pages; entries past a length name a page of NaN), lengths and pools of NaN."""
    g = torch.Generator().manual_seed(seed)
    need = [(n + page - 1) // page for n in lens]
    width, n_pages = (max_len + page - 1) // page, sum(need) + 1
    ids = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), width), int(ids[-1]), dtype=torch.int32)
    at = 0
    for t, c in enumerate(need):
        table[t, :c] = ids[at:at + c]
        at += c
    shape = H.PagedShape(Hq, Hk, D, page, n_pages, width, dtype)
    pools = [torch.full(shape.pool, float("nan"), dtype=DT[dtype]) for _ in range(2)]
    return shape, table, torch.tensor(lens, dtype=torch.int32), pools


def put(pool, table, t, rows):
    """rows [tokens][heads][D] to the pages of sequence t."""
    page = pool.shape[2]
    for i in range(0, len(rows), page):
        part = rows[i:i + page]
        pool[int(table[t, i // page]), :, :len(part)] = part.transpose(0, 1).to(pool.dtype)


def attend(shape, table, lens, pools, q, max_len, scale=1.0, mask=None):
    ws = torch.full((H.halo_paged_workspace_bytes(shape, len(lens)),), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device=DEV)
    H.halo_paged_attention(shape, q.to(DEV), pools[0].to(DEV), pools[1].to(DEV), table.to(DEV), lens.to(DEV), max_len, out, ws, scale=scale,
                           mask=None if mask is None else mask.to(DEV))
    torch.cuda.synchronize()
    return out.cpu().double().numpy()


def wanted(table, lens, pools, q, scale=1.0, mask=None):
    return ref.paged_attention(*(x.double().numpy() for x in (q, *pools)), table.numpy(), lens.numpy(), None if mask is None else mask.numpy(), scale)


# ---------------------------------------------------------------- probabilities
def left_over():
    """Scores s (bf16) of whose exp(s) two bf16 parts leave the most, with the parts and what they leave in units of the power of two below exp(s)."""
    s = -torch.arange(1, 257, dtype=torch.float64) / 256
    s = s.to(torch.bfloat16).double().unique()
    r = torch.exp(s)
    a = r.to(torch.bfloat16).double()
    b = (r - a).to(torch.bfloat16).double()
    left = (r - a - b) / 2.0 ** torch.floor(torch.log2(r))
    best = left.abs().argsort(descending=True)[:8]
    assert left[best].abs().min() >= 2.0 ** -18
    return s[best], a[best], b[best], left[best]


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hk,D,length,max_len", [
    (8, 8, 128, 300, 300), (8, 8, 64, 50, 50), (16, 8, 96, 700, 700), (8, 8, 256, 90, 90), (8, 8, 128, 4000, 4000), (32, 8, 64, 5000, 5000),
    (8, 8, 256, 1500, 1500), (160, 8, 128, 300, 20000), (160, 8, 64, 3000, 40000)])
def test_probabilities_are_as_fine_as_floats(Hq, Hk, D, length, max_len):
    # Cache head i: two tokens of score 0 with values a, b and one of score s_i with value -1, where a + b is exp(s_i) but for its last eight bits; the rest at -200
    # counts for nothing.  The result is those bits: (a + b - r) / (2 + r).  Off by: r's exponent of s log2(e), two roundings, and its own, 2 (|s| + 1) F;
    # six terms of the sum, each at most r, to 2 F of it (a truncating sum's); the result's rounding.
    s, a, b, left = left_over()
    shape, table, lens, pools = paged("bf16", Hq, Hk, D, 16, [length], max_len)
    k, v = torch.zeros(length, Hk, D), torch.zeros(length, Hk, D)
    k[:, :, 0] = -200.0
    at = length // 2 // 16 * 16 + 4                                   # three tokens of one page
    k[at:at + 2, :, 0], k[at + 2, :, 0] = 0.0, s.float()
    v[at], v[at + 1], v[at + 2] = a.float()[:, None], b.float()[:, None], -1.0
    put(pools[0], table, 0, k)
    put(pools[1], table, 0, v)
    q = torch.zeros(1, Hq, D, dtype=torch.bfloat16)
    q[:, :, 0] = 1.0
    got, want = attend(shape, table, lens, pools, q, max_len), wanted(table, lens, pools, q)
    r = torch.exp(s).numpy().repeat(Hq // Hk)[None, :, None]
    bound = r * F * (2 * (np.abs(s.numpy()).repeat(Hq // Hk)[None, :, None] + 1) + 12) / (2 + r) + 2.0 ** -8 * np.abs(want)
    assert np.all(np.abs(want) > 1.5 * bound)                         # two parts alone would give 0
    assert np.all(np.abs(got - want) <= bound), np.abs(got - want).max((0, 2)) / bound.max((0, 2))


# ---------------------------------------------------------------- scores of -infinity
@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hk,D,length,max_len", [
    (4, 2, 64, 40, 40), (4, 2, 64, 200, 200), (6, 2, 128, 900, 900), (2, 2, 256, 700, 700), (32, 2, 96, 300, 300), (2, 2, 64, 6000, 6000),
    (32, 2, 128, 3000, 3000), (4, 2, 256, 2500, 2500), (80, 2, 128, 400, 200000), (80, 2, 64, 9000, 200000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_minus_infinity(dtype, Hq, Hk, D, length, max_len):
    # keys of -infinity in the dimension that a query asks for: such a token counts for nothing beside others (weight 0), and where all are like that the
    # formula has no value (0 / 0).  Sequences, of the first cache head: all; all but the last five; all but the first seven; all but some in the middle; all, some of the
    # pages being none; no page at all; none.  The other cache head has none of them but in the last sequence, which has all.
    lens = [length] * 6 + [length - 3]
    shape, table, lens, pools = paged(dtype, Hq, Hk, D, 16, lens, max_len, seed=1)
    g = torch.Generator().manual_seed(2)
    values = []
    for t, n in enumerate(lens.tolist()):
        k, v = torch.zeros(n, Hk, D), torch.randint(-4, 5, (n, Hk, D), generator=g).float()
        k[:, :, 0] = -torch.randint(0, 6, (n, Hk), generator=g).float()
        none = torch.ones(n, dtype=torch.bool)
        if 1 <= t <= 3:
            none[[slice(n - 5, n), slice(0, 7), slice(n // 2, n // 2 + 20)][t - 1]] = False
        k[none & (t < 6), 0, 0] = -torch.inf
        if t == 6:
            k[:, 1, 0] = -torch.inf
        put(pools[0], table, t, k)
        put(pools[1], table, t, v)
    table[4, 1::2] = -1
    table[5] = shape.n_pages
    q = torch.zeros(7, Hq, D, dtype=DT[dtype])
    q[:, :, 0] = 1.0
    got, want = attend(shape, table, lens, pools, q, max_len), wanted(table, lens, pools, q)
    half = Hq // 2
    empty = np.zeros((7, Hq), dtype=bool)
    empty[[0, 4], :half] = empty[6, half:] = True
    assert np.array_equal(np.isnan(want).all(-1), empty) and np.array_equal(np.isnan(want).any(-1), empty)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.all(got[5] == 0)
    # probabilities off by 2 (|s| + 1) F, at most 14 F, sums in any order by F a term, in the numerator and in the sum; values up to 4
    bound = 2.0 ** -8 * (dtype == "bf16") * np.abs(want) + 4 * 2 * (14 + length) * F
    assert np.all((np.abs(got - want) <= bound) | empty[..., None])


# ---------------------------------------------------------------- every position once
def marked(n, Hk, D, seed):
    """Values of n tokens: dimension 0 is 1; of the others each sums to exactly 0 over the tokens, +1 and -1 in random order (with an odd n one of them 0)."""
    g = torch.Generator().manual_seed(seed)
    signs = torch.cat([torch.ones(n // 2), -torch.ones(n // 2), torch.zeros(n % 2)])
    v = signs[torch.rand(Hk * (D - 1), n, generator=g).argsort(1)].view(Hk, D - 1, n).permute(2, 0, 1)
    return torch.cat([torch.ones(n, Hk, 1), v], dim=2)


LONG = [("bf16", 8, 8, 128, 16, [2000, 1, 0, 1025, 3001]), ("bf16", 64, 8, 128, 64, [5003]), ("f32", 4, 2, 64, 32, [3000, 40]), ("bf16", 20, 1, 256, 256, [1100, 64]),
        ("f32", 2, 1, 240, 16, [1100, 900]), ("bf16", 1, 1, 128, 4096, [9000]), ("f32", 6, 6, 112, 16, [1030, 2, 1500]), ("f32", 1, 1, 16, 16, [6000]),
        ("bf16", 16, 2, 64, 16, [50 + 37 * i for i in range(70)]), ("bf16", 34, 2, 80, 64, [9000, 4001]), ("f32", 10, 2, 128, 16, [2000, 45, 700]),
        ("f32", 4, 1, 32, 16, [7000, 2]), ("f32", 20, 1, 16, 16, [40000, 30000, 5]), ("bf16", 8, 2, 48, 16, [33333, 16, 20001]),
        ("bf16", 40, 2, 96, 32, [60000]), ("f32", 40, 2, 128, 16, [30011, 333]), ("bf16", 4, 4, 256, 16, [7777, 700, 2]), ("f32", 3, 1, 256, 16, [5555, 16]),
        ("bf16", 32, 32, 128, 16, [301]), ("bf16", 8, 8, 64, 32, [3 * i for i in range(80)]), ("f32", 16, 16, 128, 16, [500 + i % 100 for i in range(64)])]


@pytest.mark.parametrize("args", LONG, ids=lambda a: "-".join(map(str, a[:5])) + f"-{max(a[5])}x{len(a[5])}")
def test_marks_show_what_is_lost_or_doubled(args):
    # what the next test could not see does not happen: any token alone, and any run of 16, 32, 64 or 256 that a share may end in, has a sum other than 0
    # in some dimension
    _, _, Hk, D, _, lens = args
    for t, n in enumerate(lens):
        v = marked(n, Hk, D, t)[:, :, 1:]
        assert bool((v.sum(0) == 0).all())
        for run in (1, 16, 32, 64, 256):
            if run < n:
                sums = torch.stack([v[i:i + run].sum(0) for i in range(0, n, run)])
                assert bool((sums != 0).any(-1).all()), (n, run)


@pytest.mark.gpu
@pytest.mark.parametrize("bound", ["exact", "larger"])
@pytest.mark.parametrize("args", LONG, ids=lambda a: "-".join(map(str, a[:5])) + f"-{max(a[5])}x{len(a[5])}")
def test_every_position_counts_once(args, bound):
    # Scores of 0: every probability is 1, the sums are of whole numbers below 2^24 and exact in any order.  The results are 0, but 1 in the first dimension: the
    # number of positions times its reciprocal, off by two roundings and the result's.
    dtype, Hq, Hk, D, page, lens = args
    max_len = max(lens) if bound == "exact" else 3 * max(lens) + 2100
    shape, table, lens, pools = paged(dtype, Hq, Hk, D, page, lens, max_len, seed=3)
    g = torch.Generator().manual_seed(4)
    for t, n in enumerate(lens.tolist()):
        put(pools[0], table, t, torch.randn(n, Hk, D, generator=g))
        put(pools[1], table, t, marked(n, Hk, D, t))
    got = attend(shape, table, lens, pools, torch.zeros(len(lens), Hq, D, dtype=DT[dtype]), max_len)
    some = lens.numpy() > 0
    assert np.all(got[:, :, 1:] == 0) and np.all(got[~some] == 0)
    assert np.all(np.abs(got[some][:, :, 0] - 1) <= 3 * F + 2.0 ** -8 * (dtype == "bf16"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,Hq,Hk,D", [("bf16", 1, 1, 256), ("f32", 8, 1, 240), ("bf16", 32, 1, 128), ("f32", 32, 1, 128), ("f32", 4, 2, 64), ("bf16", 2, 1, 64)])
def test_as_many_sequences_as_there_can_be(dtype, Hq, Hk, D):
    # 4096 short caches under a bound that takes the kernel of even shares: it has the line of all tiles in LDS beside its own part, at its longest here
    lens, max_len = [(i * 7) % 40 for i in range(4095)] + [3000], 20000
    shape, table, lens, pools = paged(dtype, Hq, Hk, D, 16, lens, max_len, seed=5)
    for t, n in enumerate(lens.tolist()):
        put(pools[0], table, t, torch.zeros(n, Hk, D))
        put(pools[1], table, t, marked(n, Hk, D, t % 40))
    got = attend(shape, table, lens, pools, torch.zeros(len(lens), Hq, D, dtype=DT[dtype]), max_len)
    some = lens.numpy() > 0
    assert np.all(got[:, :, 1:] == 0) and np.all(got[~some] == 0)
    assert np.all(np.abs(got[some][:, :, 0] - 1) <= 3 * F + 2.0 ** -8 * (dtype == "bf16"))
