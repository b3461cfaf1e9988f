"""Attention of chunks of new tokens over a paged cache, of rows and of eight-bit codes, on the GPU against the formula in double.

Tolerances are bounds: u = finfo(type).eps / 2 for the rounding that stores a result, u once more of each probability that a bf16 row rounds; float operations count
2^-24 each, worst case; products of parts (three bf16 values a float) leave out 2 * 2^-24 of theirs and are summed in six passes."""
import math

import pytest
import torch

import paper_2601_11676_amd as H

pytestmark = pytest.mark.gpu
DEV = "cuda"
F = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


class Case:
    """Sequences of (past, new) tokens over scattered pages.  What no sequence has yet is NaN, entries of the page table behind a sequence name a page of NaN.
    kind: bf16, f32, or with q8 a cache of codes under such queries."""

    def __init__(self, kind, Hq, Hk, D, page, runs, keep=None, seed=0, sigma=1.5, before=0, behind=0, wide=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.q8 = kind.replace("q8", "").strip("-") or "bf16", "q8" in kind
        dt = DT[self.dtype]
        lens = [p + n for p, n in runs]
        need = [-(-n // page) for n in lens]
        width, n_pages = max(need) + 1, sum(need) + 2
        ids = torch.randperm(n_pages, generator=g).to(torch.int32)
        self.shape = H.PagedShape(Hq, Hk, D, page, n_pages, width, self.dtype)
        self.table = torch.full((len(runs), width), int(ids[-1]), dtype=torch.int32)
        at = 0
        for i, c in enumerate(need):
            self.table[i, :c] = ids[at:at + c]
            at += c
        self.lens = torch.tensor(lens, dtype=torch.int32)
        self.runs, self.max_len = list(runs), max(1, max(lens))
        starts = [before]
        for _, n in runs:
            starts.append(starts[-1] + n)
        self.starts = torch.tensor(starts, dtype=torch.int32)
        self.N = starts[-1] + behind
        rows = (torch.randn((self.N, Hq + wide, D), generator=g) * sigma).to(dt)
        self.q = rows[:, :Hq]
        self.mask = None if keep is None else (torch.rand((self.N, Hq), generator=g) < keep).to(torch.uint8)
        if self.q8:
            self.k, self.v = (self.codes(g) for _ in range(2))
        else:
            self.k, self.v = (self.rows(g, dt) for _ in range(2))
        self.scale = D ** -0.5

    def unused(self, pool):
        """Marks of the pool's rows that no sequence has."""
        free = torch.ones(self.shape.pool[0], self.shape.page_size, dtype=torch.bool)
        for i, n in enumerate(self.lens.tolist()):
            for j in range(0, n, self.shape.page_size):
                free[int(self.table[i, j // self.shape.page_size]), :min(n - j, self.shape.page_size)] = False
        return free

    def rows(self, g, dt):
        pool = torch.randn(self.shape.pool, generator=g).to(dt)
        return pool.masked_fill_(self.unused(pool)[:, None, :, None], math.nan)

    def codes(self, g):
        codes = torch.randint(-127, 128, self.shape.pool, generator=g, dtype=torch.int8)
        scales = (0.005 + 0.02 * torch.rand(self.shape.pool[:3], generator=g))
        return codes, scales.masked_fill_(self.unused(codes)[:, None, :], math.nan)

    def run(self, max_len=None, stream=None, ws=None, out=None):
        s = self.shape
        if ws is None:
            ws = torch.full((H.halo_paged_chunk_workspace_bytes(s, self.N, len(self.runs)),), 0xff, dtype=torch.uint8, device=DEV)
        if out is None:
            out = torch.full((self.N, s.n_heads, s.head_dim), 77.0, dtype=DT[self.dtype], device=DEV)
        base = self.q if self.q._base is None else self.q._base
        q = torch.as_strided(base.to(DEV), self.q.shape, self.q.stride(), self.q.storage_offset())
        call = H.halo_paged_chunk_attention_q8 if self.q8 else H.halo_paged_chunk_attention
        k, v = (tuple(x.to(DEV) for x in p) if self.q8 else p.to(DEV) for p in (self.k, self.v))
        call(s, q, k, v, self.table.to(DEV), self.starts.to(DEV), self.lens.to(DEV), self.max_len if max_len is None else max_len, out, ws,
             mask=None if self.mask is None else self.mask.to(DEV), scale=self.scale, stream=stream)
        torch.cuda.synchronize()
        return out.cpu()

    def row_values(self, pool, i, n):
        """[n][kv heads][D] in double of sequence i's first n positions, and which of them are in pages."""
        s = self.shape
        page = self.table[i, :-(-n // s.page_size)].long()
        there = ((page >= 0) & (page < s.n_pages)).repeat_interleave(s.page_size)[:n]
        ids = torch.where((page >= 0) & (page < s.n_pages), page, 0)
        x = pool[0][ids].double() * pool[1][ids].double()[..., None] if self.q8 else pool[ids].double()
        return x.permute(0, 2, 1, 3).reshape(-1, s.n_kv_heads, s.head_dim)[:n], there

    def want(self, max_len=None):
        """The formula, row by row of the batch, and what its error may be; rows of no sequence are the outputs' fill, off by nothing."""
        s, group = self.shape, self.shape.n_heads // self.shape.n_kv_heads
        out, off = torch.full((self.N, s.n_heads, s.head_dim), 77.0, dtype=torch.float64), torch.zeros(self.N, s.n_heads, s.head_dim, dtype=torch.float64)
        split = self.dtype == "f32"
        for i in range(len(self.runs)):
            a, b = int(self.starts[i]), int(self.starts[i + 1])
            n = max(0, min(int(self.lens[i]), self.max_len if max_len is None else max_len))
            if a == b:
                continue
            k, there = self.row_values(self.k, i, n)
            v, _ = self.row_values(self.v, i, n)
            pos = n - (b - a) + torch.arange(b - a)
            sees = (torch.arange(n) <= pos[:, None]) & there
            for h in range(s.n_heads):
                q, kh, vh = self.q[a:b, h].double(), k[:, h // group], v[:, h // group]
                kh, vh = (torch.where(there[:, None], x, 0.0) for x in (kh, vh))
                score = (q @ kh.T * self.scale).masked_fill(~sees, -math.inf)
                top = score.amax(-1, keepdim=True) if n else torch.zeros(b - a, 1, dtype=torch.float64)
                e = torch.where(sees, torch.exp(score - torch.where(top == -math.inf, 0.0, top)), 0.0)
                p = e / e.sum(-1, keepdim=True).clamp(min=1e-300)
                o, W = p @ vh, p @ vh.abs()
                S = abs(self.scale) * float(q.norm(dim=-1).max() * kh.norm(dim=-1).max()) if n else 0.0      # no sum |q k| is larger
                u, D = U[self.dtype], s.head_dim
                gamma = F * ((7 if split else 2) * D * S + 12 * S + (6 if split else 1) * max(1, n) + 80)
                out[a:b, h] = o
                off[a:b, h] = u * o.abs() + ((0.0 if split else u * W) + 2 * gamma * W) * (1 + u)
        if self.mask is not None:
            a, b = int(self.starts[0]), int(self.starts[-1])
            out[a:b] = torch.where(self.mask[a:b, :, None] != 0, out[a:b], 0.0)
            off[a:b] = torch.where(self.mask[a:b, :, None] != 0, off[a:b], 0.0)
        return out, off

    def check(self, got, max_len=None):
        want, off = self.want(max_len)
        assert torch.isfinite(got).all()
        bad = (got.double() - want).abs() > off
        assert not bad.any(), (bad.nonzero()[:4], ((got.double() - want).abs() - off).max())
        assert torch.all(got.double()[off == 0] == want[off == 0])


KINDS = ["bf16", "f32", "q8", "q8-f32"]
CHUNKS = [
    # few rows of a sequence: narrow blocks, whole and cut
    (8, 8, 128, 16, [(0, 1)], None), (8, 2, 64, 16, [(0, 1), (15, 1), (16, 1), (300, 2)], None), (6, 2, 128, 32, [(31, 1), (500, 5), (0, 3)], 0.6),
    (16, 2, 64, 16, [(2000, 3), (17, 1), (0, 4)], None), (5, 5, 80, 64, [(700, 7), (64, 0), (1, 9)], 0.5), (4, 1, 256, 16, [(900, 3), (30, 8)], None),
    (20, 1, 128, 16, [(3000, 1)], None), (7, 7, 16, 16, [(100, 31)], None), (3, 1, 240, 256, [(300, 10)], None), (1, 1, 48, 4096, [(5000, 2)], None),
    # more rows: blocks of 128, whole and cut
    (4, 4, 128, 16, [(0, 33), (0, 200), (5, 127)], None), (8, 2, 64, 16, [(0, 64), (63, 65), (64, 64), (1, 129)], 0.5), (16, 1, 96, 16, [(40, 60)], None),
    (40, 2, 128, 16, [(1500, 40), (0, 7)], 0.7), (2, 2, 112, 32, [(0, 300)], None), (3, 3, 256, 64, [(100, 150), (0, 33)], None),
    (6, 2, 144, 16, [(9, 90)], 0.4), (5, 1, 208, 16, [(0, 70)], None), (64, 8, 128, 64, [(900, 64)], None), (2, 1, 64, 128, [(0, 1025)], None),
    # many scores under a mask: the surviving rows are listed first, of blocks whole and cut
    (64, 64, 16, 16, [(2300, 700), (0, 400)], 0.5), (64, 4, 64, 16, [(2300, 700), (5, 0), (0, 410)], 0.3), (256, 2, 16, 16, [(7900, 100)], 0.4),
    # as many blocks as the card has places: nothing is cut
    (64, 64, 64, 16, [(0, 600), (13, 510)], 0.5), (80, 40, 32, 16, [(0, 300), (0, 500), (100, 90)], None), (128, 128, 16, 32, [(3, 20)] * 20, 0.3),
]


def label(a):
    return "-".join(map(str, a[:4])) + "-" + "x".join(f"{p}+{n}" for p, n in a[4][:4])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("args", CHUNKS, ids=label)
def test_chunks(kind, args):
    case = Case(kind, *args[:5], keep=args[5])
    case.check(case.run())


@pytest.mark.parametrize("kind", KINDS)
def test_many_sequences(kind):
    # more than a wave's lanes of them, among them empty ones, of blocks whole and cut
    for Hq, Hk, past, new in [(4, 2, 37, 5), (8, 8, 11, 40)]:
        runs = [((past * i) % 301, (new * i * i) % (new + 3)) for i in range(150)]
        case = Case(kind, Hq, Hk, 64, 16, runs, keep=0.7, seed=3)
        case.check(case.run())


@pytest.mark.parametrize("kind", KINDS)
def test_rows_of_no_sequence_stay(kind):
    case = Case(kind, 4, 2, 64, 16, [(5, 3), (0, 0), (40, 40)], before=2, behind=5, wide=1)
    got = case.run()
    case.check(got)
    assert torch.all(got[:2] == 77) and torch.all(got[-5:] == 77)
    case = Case(kind, 4, 2, 64, 16, [(5, 0), (0, 0)], behind=3)       # no row of any sequence
    assert torch.all(case.run() == 77)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("past", [0, 1500])
def test_masks_that_leave_nothing(kind, past):
    case = Case(kind, 8, 2, 64, 16, [(past, 40), (past, 1), (0, 5)], keep=0.5, seed=4)
    m, s = case.mask, case.starts
    m[:16] = 0                                                        # some rows, a sequence, a cache head, single heads; any byte but 0 keeps
    m[s[1]:s[2]] = 0
    m[s[2]:, :4] = 0
    m[20:30, 1] = 0
    m[31] = 255
    got = case.run()
    case.check(got)
    assert torch.all(got[:16] == 0) and torch.all(got[s[1]:s[2]] == 0) and torch.all((got[31] != 0).any(-1))
    m[:] = 0
    assert torch.all(case.run() == 0)


@pytest.mark.parametrize("kind", ["bf16", "q8-f32"])
def test_listed_rows_that_leave_nothing(kind):
    # the same where survivors are listed: no row of a cache head, of a sequence, of a block; runs of one
    case = Case(kind, 64, 4, 32, 16, [(2300, 700), (0, 3), (0, 400)], keep=0.4, seed=16, before=1, behind=2)
    m, s = case.mask, case.starts.tolist()
    m[:, :16] = 0
    m[s[0]:s[0] + 600, 16:32] = 0
    m[s[0] + 10, 20] = 3
    m[s[1]:s[2]] = 0
    got = case.run()
    case.check(got)
    assert torch.all(got[s[0]:s[-1], :16] == 0) and torch.all((got[s[0] + 10, 20] != 0).any()) and torch.all(got[:1] == 77) and torch.all(got[-2:] == 77)
    m[:] = 0
    assert torch.all(case.run()[1:-2] == 0)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("past", [40, 1200])
def test_pages_that_are_none_and_odd_lengths(kind, past):
    case = Case(kind, 4, 2, 64, 16, [(past, 70), (90, 30), (64, 64), (past, 5), (10, 6), (7, 20)], seed=5)
    t, s = case.table, case.shape
    t[0, 1], t[0, (past + 70) // 16] = -1, s.n_pages                  # holes, one at the end; a sequence without any page; the first pages
    t[1, :] = -(1 << 31)
    t[2, :5] = (1 << 31) - 1
    case.lens[4] = -5
    case.lens[5] = 12                                                 # fewer positions than rows: the first 8 see none
    got = case.run()
    case.check(got)
    st = case.starts.tolist()
    assert torch.all(got[st[1]:st[2]] == 0) and torch.all(got[st[4]:st[5]] == 0) and torch.all(got[st[5]:st[5] + 8] == 0)
    assert torch.all((got[st[5] + 8:] != 0).any(-1))
    # lengths past max_len count as max_len
    case.lens[0] = 1 << 30
    case.check(case.run(max_len=past + 70 - 3), max_len=past + 70 - 3)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq,Hk,D,past,new", [(4, 2, 64, 0, 100), (4, 4, 128, 700, 40), (2, 1, 96, 30, 7), (64, 64, 64, 0, 1100)])
def test_what_later_positions_hold(kind, Hq, Hk, D, past, new):
    # NaN and infinities in keys and values of single positions: rows before them keep their bits, rows from them on have what the formula has
    case = Case(kind, Hq, Hk, D, 16, [(past, new)], seed=6)
    clean = case.run()
    at = [new // 3, new // 3 + 1, new - 2]                            # new tokens, of different tiles and neighbours
    for j, bad in zip(at, (math.inf, -math.inf, math.nan)):
        page, row = int(case.table[0, (past + j) // 16]), (past + j) % 16
        if case.q8:
            case.k[1][page, 0, row] = math.nan
            case.v[1][page, :, row] = math.nan
        else:
            case.v[page, :, row, 3] = bad
            case.k[page, 0, row, 5] = math.nan if j == at[2] else 1.0
    case_k = case.k
    got = case.run()
    first = at[0]
    assert torch.equal(got[:first], clean[:first])
    if not case.q8:
        other = [d for d in range(D) if d != 3]
        seen = got[first:at[2]]
        assert not torch.isfinite(seen[:, :, 3]).any() and torch.isfinite(seen[:, :, other]).all()
        assert torch.isnan(got[at[2]:, :Hq // Hk]).all()              # the key's NaN: all of its cache head's rows
        assert torch.equal(got[:at[1], :, 3][first:] == math.inf, torch.ones(at[1] - first, Hq, dtype=torch.bool))
    else:
        assert torch.isnan(got[first:]).all()
    assert case_k is case.k


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_scores_of_infinity(kind):
    # a row whose scores are all -infinity has no value; beside others such a score counts for nothing.  Float keys are finite, their products are not.
    case = Case(kind, 2, 2, 64, 16, [(0, 40)], seed=7)
    case.q = (case.q.abs() + 0.5) * 100
    page = case.table[0].long()
    case.k[page[0], 0, 0] = -math.inf if kind == "bf16" else -3.0e37
    got = case.run()
    assert torch.isnan(got[0, 0]).all() and torch.isfinite(got[1:]).all() and torch.isfinite(got[:, 1]).all()
    one = U[kind] * case.v[page[0], 0, 1].double().abs()              # one position is left: its probability is 1
    assert torch.all((got[1, 0].double() - case.v[page[0], 0, 1].double()).abs() <= one)


def test_large_and_small_floats_are_numbers():
    # A value that a row sees alone is its result, to the bit: probability 1, three parts that add up; up to 2^120, from where sums may overflow on their way (the largest float is
    # (2^8 - 1) 2^120 + 2^120 - 2^104 in parts, whose first two are 2^128), and from 2^-110 on, below which last parts are below 2^-126 and count as 0.  A key past the largest bf16 number against a query of 2^-126: the product is a number like any other.
    largest = torch.finfo(torch.float32).max
    case = Case("f32", 4, 2, 64, 16, [(0, 1)] * 6 + [(0, 2)], seed=17)
    for i, v in enumerate([largest * 2.0 ** -8, -largest * 2.0 ** -8, 1.3e36, -1.2345678e36, 3.3895e35, 1.2345678e-32]):
        case.v[int(case.table[i, 0]), :, 0, i::7] = v
    case.q = case.q.clone()
    case.q[6:, :, 9] = 2.0 ** -126
    page = int(case.table[6, 0])
    case.k[page, :, 1, 9], case.k[page, :, 0, 9] = largest, 0.0
    got = case.run()
    for i in range(6):
        assert torch.equal(got[i], case.v[int(case.table[i, 0]), :, 0].repeat_interleave(2, 0))
    # scores of at most 8 * 8 / 8 + 4 / 8 with 65 terms, each product and sum of six passes off by 2^-24 of it: 6 * 65 * 9 * 2^-24 = 2.1e-4, twice in a probability, of values up to 5
    want, _ = case.want()
    assert torch.all((got[6:].double() - want[6:]).abs() <= 2 * 2.1e-4 * 2 * 5)


@pytest.mark.parametrize("kind", KINDS)
def test_nan_stays_in_its_row(kind):
    case = Case(kind, 4, 2, 128, 16, [(50, 60)], seed=8)
    clean = case.run()
    case.q = case.q.clone()
    case.q[17, 1], case.q[33, 2, 5] = math.nan, math.inf
    got = case.run()
    keep = torch.ones(60, 4, dtype=torch.bool)
    keep[17, 1] = keep[33, 2] = False
    assert torch.equal(got[keep], clean[keep]) and torch.isnan(got[17, 1]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales(kind, scale):
    case = Case(kind, 4, 2, 64, 16, [(70, 50), (0, 3)], seed=9, sigma=0.5)
    case.scale = scale
    case.check(case.run())


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("past,new", [(0, 150), (2500, 20)])
def test_far_apart_scores(kind, past, new):
    # single keys far above and below the rest, scores of several hundred: the maximum moves in any step
    case = Case(kind, 4, 4, 64, 16, [(past, new)], seed=10, sigma=2.0)
    n = past + new
    for h, j in enumerate([0, n // 2, n - 3, 70]):
        case.k[int(case.table[0, j // 16]), h, j % 16] = (case.q[new // 2, h].float() * (30.0 if h < 3 else -30.0)).to(case.k.dtype)
    case.check(case.run())


def test_single_tokens_agree_with_the_attention_of_one_token():
    # as many sequences of one new token each: the same formula, each within its own bound
    case = Case("bf16", 16, 4, 128, 16, [(37 * i % 900, 1) for i in range(40)], keep=0.6, seed=11)
    got = case.run()
    case.check(got)
    s, out = case.shape, torch.empty(40, 16, 128, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(H.halo_paged_workspace_bytes(s, 40), dtype=torch.uint8, device=DEV)
    H.halo_paged_attention(s, case.q.contiguous().to(DEV), case.k.to(DEV), case.v.to(DEV), case.table.to(DEV), case.lens.to(DEV), case.max_len, out, ws,
                           mask=case.mask.to(DEV))
    want, off = case.want()
    assert torch.all((out.cpu().double() - got.double()).abs() <= 2 * off)


@pytest.mark.parametrize("kind", KINDS)
def test_graphs_that_share_a_workspace(kind):
    # two captured calls, one cut into parts, replayed in turn with eager work between: each equals its eager result
    cases = [Case(kind, 8, 2, 64, 16, [(1200, 20), (3, 9)], keep=0.7, seed=12), Case(kind, 4, 4, 64, 32, [(600, 90)], seed=13)]
    eager = [c.run() for c in cases]
    ws = torch.full((max(H.halo_paged_chunk_workspace_bytes(c.shape, c.N, 2) for c in cases),), 0xff, dtype=torch.uint8, device=DEV)
    graphs = []
    for c in cases:
        dev = [tuple(x.to(DEV) for x in p) if c.q8 else p.to(DEV) for p in (c.k, c.v)] + [x.to(DEV) for x in (c.table, c.starts, c.lens)]
        q, mask = c.q.contiguous().to(DEV), None if c.mask is None else c.mask.to(DEV)
        out = torch.zeros(q.shape, dtype=q.dtype, device=DEV)
        call = H.halo_paged_chunk_attention_q8 if c.q8 else H.halo_paged_chunk_attention
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(c.shape, q, *dev, c.max_len, out, ws, mask=mask)
        graphs.append((graph, out, q, dev, mask))
    for _ in range(3):
        for (graph, out, *_), want in zip(graphs, eager):
            out.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.cpu(), want)


def test_another_stream():
    case = Case("bf16", 4, 2, 64, 16, [(900, 30)], seed=14)
    want = case.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    assert torch.equal(case.run(stream=s), want)
    with torch.cuda.stream(s):
        assert torch.equal(case.run(), want)


@pytest.mark.parametrize("kind", ["bf16", "q8"])
def test_offsets_past_32_bits(kind):
    # pools whose last pages lie past 2^32 bytes (rows of 16: the codes' scales too)
    D, page, Hk = 16, 4096, 2
    n_pages = (1 << 30) // (Hk * page) + 3 if kind == "q8" else (1 << 32) // (Hk * page * D * 2) + 3
    shape = H.PagedShape(4, Hk, D, page, n_pages, 2)
    g = torch.Generator().manual_seed(15)
    small = Case(kind, 4, Hk, D, page, [(4000, 120)], seed=15)
    pools = []
    for p in (small.k, small.v):
        big = tuple(torch.empty((n_pages,) + x.shape[1:], dtype=x.dtype, device=DEV) for x in (p if small.q8 else (p,)))
        for b, x in zip(big, p if small.q8 else (p,)):
            for j in range(2):
                b[n_pages - 1 - j] = x[int(small.table[0, j])].to(DEV)
        pools.append(big if small.q8 else big[0])
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device=DEV)
    out = torch.zeros(120, 4, D, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(H.halo_paged_chunk_workspace_bytes(shape, 120, 1), dtype=torch.uint8, device=DEV)
    call = H.halo_paged_chunk_attention_q8 if small.q8 else H.halo_paged_chunk_attention
    call(shape, small.q.contiguous().to(DEV), *pools, table, small.starts.to(DEV), small.lens.to(DEV), 4120, out, ws)
    small.check(out.cpu())
    del pools
    torch.cuda.empty_cache()
