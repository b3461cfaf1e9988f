"""Appends that norm heads, a cache of eight-bit codes written, read back and attended over by single tokens, on the GPU against the formulas in double.

Tolerances are bounds: u = finfo(type).eps / 2 for a rounding, float operations 2^-24 each, worst case.  Codes are whole numbers and have to be equal; a quotient within 1e-9 of
the border of two (where double's own roundings decide) may be either, and counts."""
import math

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
EPS = 1e-3


def np64(t):
    return t.detach().cpu().double().numpy()


class Append:
    def __init__(self, dtype, Hq, Hk, D, page, lens, rotary, pairs, weights=True, fused=True, seed=0):
        g = torch.Generator().manual_seed(seed)
        dt = DT[dtype]
        need = [-(-(p + n) // page) for p, n in lens]
        n_pages, width = sum(need) + 2, max(need) + 1
        ids = torch.randperm(n_pages, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), width), -7, dtype=torch.int32)
        at = 0
        for i, c in enumerate(need):
            self.table[i, :c] = ids[at:at + c]
            at += c
        self.seq = torch.tensor([i for i, (_, n) in enumerate(lens) for _ in range(n)], dtype=torch.int32)
        self.pos = torch.tensor([p + j for p, n in lens for j in range(n)], dtype=torch.int32)
        N = len(self.seq)
        if fused:
            self.rows = (torch.randn((N, Hq + 2 * Hk + 1, D), generator=g) * 1.7).to(dt)
        else:
            self.rows = torch.randn((N, Hq + 2 * Hk, D), generator=g).to(dt)
        self.shape = H.PagedShape(Hq, Hk, D, page, n_pages, width, dtype)
        self.rope = torch.from_numpy(H.halo_rope_table(max(p + n for p, n in lens), rotary)) if rotary else None
        self.pairs, self.dtype = pairs, dtype
        self.w = [(1.0 + 0.3 * torch.randn(D, generator=g)).to(dt) if weights else None for _ in range(2)]

    def heads(self, rows):
        Hq, Hk = self.shape.n_heads, self.shape.n_kv_heads
        return rows[:, :Hq], rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:Hq + 2 * Hk]

    def pools(self, codes):
        s = self.shape
        if codes:
            return [(torch.full(s.pool, 99, dtype=torch.int8, device=DEV), torch.full(s.pool[:3], -5.0, device=DEV)) for _ in range(2)]
        return [torch.full(s.pool, math.nan, dtype=DT[self.dtype], device=DEV) for _ in range(2)]

    def run(self, codes, norm=True, with_q=True, pools=None, stream=None):
        pools = pools or self.pools(codes)
        q, k, v = self.heads(self.rows.to(DEV))
        out = torch.full((len(self.pos), self.shape.n_heads, self.shape.head_dim), math.nan, dtype=DT[self.dtype], device=DEV) if with_q else None
        args = dict(q_out=out, rope=None if self.rope is None else self.rope.to(DEV), rope_pairs=self.pairs,
                    seq=None if self.seq is None else self.seq.to(DEV), stream=stream)
        if norm:
            args.update(eps=EPS, w_q=None if self.w[0] is None else self.w[0].to(DEV), w_k=None if self.w[1] is None else self.w[1].to(DEV))
        if codes:
            H.halo_paged_append_q8(self.shape, q if with_q else None, k, v, self.pos.to(DEV), self.table.to(DEV), *pools, qk_norm=norm, **args)
        else:
            H.halo_paged_append_norm(self.shape, q if with_q else None, k, v, self.pos.to(DEV), self.table.to(DEV), *pools, **args)
        torch.cuda.synchronize()
        return out, pools

    def there(self):
        """Page and row of each token, and which tokens have one."""
        s, pos, seq = self.shape, self.pos.long(), (torch.arange(len(self.pos)) if self.seq is None else self.seq.long())
        most = s.max_pages * s.page_size if self.rope is None else min(s.max_pages * s.page_size, self.rope.shape[0])
        ok = (seq >= 0) & (seq < self.table.shape[0]) & (pos >= 0) & (pos < most)
        page = self.table.long()[torch.where(ok, seq, 0), torch.where(ok, pos, 0) // s.page_size]
        ok &= (page >= 0) & (page < s.n_pages)
        return torch.where(ok, page, 0), torch.where(ok, pos, 0) % s.page_size, ok

    def want(self, norm=True):
        """q, k, v in double, and for q and k the size of what their float operations round."""
        q, k, v = (x.double() for x in self.heads(self.rows))
        size = []
        _, _, ok = self.there()
        pos = torch.where(ok, self.pos.long(), 0)
        for i, x in enumerate((q, k)):
            if norm:
                x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
                x = x if self.w[i] is None else x * self.w[i].double()
            a = x.abs()
            if self.rope is not None:
                half = self.rope.shape[2]
                cs = self.rope[pos].double()[:, :, None]
                turned, bound = x.clone(), a.clone()
                lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if self.pairs else (slice(0, half), slice(half, 2 * half))
                turned[..., lo] = x[..., lo] * cs[:, 0] - x[..., hi] * cs[:, 1]
                turned[..., hi] = x[..., hi] * cs[:, 0] + x[..., lo] * cs[:, 1]
                bound[..., lo] = a[..., lo] * cs[:, 0].abs() + a[..., hi] * cs[:, 1].abs()
                bound[..., hi] = a[..., hi] * cs[:, 0].abs() + a[..., lo] * cs[:, 1].abs()
                x, a = turned, bound
            size.append(a)
            if i == 0:
                q = torch.where(ok[:, None, None], x, 0.0)
            else:
                k = x
        return q, k, v, size

    def near(self, got, want, size):
        # the mean of D squares, its root and quotient: (D / 2 + 4) roundings; weight and rotation 4; and the one that stores
        F_ops = (self.shape.head_dim / 2 + 8) * F
        u = U[self.dtype]
        assert torch.all((got.cpu().double() - want).abs() <= u * want.abs() + F_ops * size * (1 + u))


APPENDS = [("bf16", 8, 2, 128, 16, [(0, 1)], 128, False), ("bf16", 32, 32, 128, 16, [(15, 1), (16, 1), (300, 1)], 128, False),
           ("bf16", 6, 2, 64, 32, [(0, 70), (31, 2), (5, 0), (100, 33)], 32, True), ("f32", 4, 4, 16, 16, [(3, 20)], 16, False),
           ("f32", 5, 1, 80, 64, [(60, 9), (0, 1)], 48, True), ("f32", 3, 3, 256, 256, [(255, 2)], 256, False),
           ("bf16", 7, 7, 96, 16, [(0, 40)], 96, True), ("bf16", 16, 1, 256, 16, [(9, 600)], 128, False), ("f32", 2, 1, 240, 16, [(0, 19)], 240, False),
           ("bf16", 2, 1, 112, 4096, [(4090, 10)], 0, False), ("bf16", 64, 8, 128, 16, [(7, 530), (0, 61)], 128, False),
           ("bf16", 3, 1, 16, 16, [(0, 33)], 16, True), ("bf16", 5, 5, 80, 16, [(2, 50)], 64, False), ("f32", 40, 40, 128, 16, [(0, 130)], 128, True)]


@pytest.mark.parametrize("args", APPENDS, ids=lambda a: "-".join(map(str, a[:5])))
@pytest.mark.parametrize("weights", [True, False])
def test_append_norm(args, weights):
    case = Append(*args, weights=weights)
    out, (kp, vp) = case.run(False)
    q, k, v, size = case.want()
    page, row, ok = case.there()
    assert ok.all()
    case.near(out, q, size[0])
    case.near(kp.cpu()[page, :, row], k, size[1])
    assert torch.equal(vp.cpu()[page, :, row].double(), v)            # moved, not computed
    for pool in (kp.cpu(), vp.cpu()):                                 # the rest of the pools is untouched
        pool[page, :, row] = math.nan
        assert torch.isnan(pool).all()


def quotients(x):
    """Steps max|x| / 127 and quotients x / step of rows, in double."""
    step = x.abs().amax(-1, keepdim=True) / 127.0
    return step[..., 0], torch.where(step > 0, x / torch.where(step > 0, step, 1.0), 0.0)


def check_codes(pool, x, page, row):
    codes, scales = (t.cpu() for t in pool)
    step, quotient = quotients(x)
    got, want = codes[page, :, row].double(), torch.round(quotient)
    border = (quotient - torch.floor(quotient) - 0.5).abs() < 1e-9
    assert torch.all((got == want) | (border & ((got - quotient).abs() < 0.5 + 1e-9))), ((got != want) & ~border).nonzero()[:3]
    assert border.double().mean() < 0.2                               # exact ties of rows whose largest is 127 steps of its own spacing
    s = scales[page, :, row].double()
    # rounded once; of rows that end at the largest float down, where 127 of it would pass that
    down = torch.where(step * (1 + F) * 127 >= 2.0 ** 128 * (1 - F), 2.0, 1.0)
    assert torch.all((s - step).abs() <= down * step * F * (1 + 1e-6) + 2.0 ** -150)


@pytest.mark.parametrize("args", APPENDS, ids=lambda a: "-".join(map(str, a[:5])))
@pytest.mark.parametrize("norm", [True, False])
def test_append_and_read_codes(args, norm):
    case = Append(*args)
    out, (kp, vp) = case.run(True, norm)
    q, k, v, size = case.want(norm)
    page, row, ok = case.there()
    case.near(out, q, size[0])
    check_codes(kp, k, page, row)
    check_codes(vp, v, page, row)
    read = [torch.full((len(case.pos), case.shape.n_kv_heads, case.shape.head_dim), math.nan, dtype=DT[case.dtype], device=DEV) for _ in range(2)]
    H.halo_paged_read_q8(case.shape, case.pos.to(DEV), case.table.to(DEV), kp, vp, *read, seq=case.seq.to(DEV))
    for got, pool, x in zip(read, (kp, vp), (k, v)):
        stands = pool[0].cpu()[page, :, row].double() * pool[1].cpu()[page, :, row].double()[..., None]
        u = U[case.dtype]
        assert torch.all((got.cpu().double() - stands).abs() <= stands.abs() * ((1 + u) * (1 + F) - 1) + 2.0 ** -149)
        # half a step, and 127 times a scale's rounding of 2^-24: 254 * 2^-24 half steps
        assert torch.all((stands - x).abs() <= x.abs().amax(-1, keepdim=True) / 254 * (1 + 254 * F + 1e-6))
    for codes, scales in (kp, vp):                                    # the rest of the pools is untouched
        codes, scales = codes.cpu(), scales.cpu()
        codes[page, :, row], scales[page, :, row] = 99, -5.0
        assert torch.all(codes == 99) and torch.all(scales == -5.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_at_the_ends_of_the_numbers(dtype):
    # rows of zeros, exact ties, the smallest and largest numbers, infinities and NaN: codes and scales as the definition says
    case = Append(dtype, 1, 1, 64, 16, [(0, 10)], 0, False)
    v = case.rows[:, 2]
    v[0] = 0
    v[1] = torch.arange(64) - 31.5                                    # largest magnitude 31.5 -> see below: quotients of 127 x / 31.5
    v[1, 0] = -127.0                                                  # steps of 1: ties at every x.5, to even
    v[2] = -0.0
    v[3], v[3, 5] = 0, 2.0 ** -126
    v[4] = torch.finfo(DT[dtype]).max * (torch.arange(64) % 2 * 2 - 1)
    v[5, 7] = math.inf
    v[6, 63] = math.nan
    v[7], v[7, 3] = -1.0, 1.0
    v[8, 0] = -math.inf
    _, (kp, vp) = case.run(True, norm=False)
    page, row, _ = case.there()
    codes, scales = vp[0].cpu()[page, 0, row], vp[1].cpu()[page, 0, row]
    assert torch.all(codes[[0, 2, 5, 6, 8]] == 0) and torch.all(scales[[0, 2]] == 0) and torch.isnan(scales[[5, 6, 8]]).all()
    assert scales[1] == 1 and torch.equal(codes[1].double(), torch.round(v[1].double()))
    assert codes[3, 5] == 127 and codes[3].abs().sum() == 127 and scales[3] == torch.tensor(2.0 ** -126, dtype=torch.float64).div(127).float()
    assert torch.equal(codes[4].double(), 127.0 * torch.sign(v[4].double())) and torch.isfinite(scales[4])
    assert codes[7, 3] == 127 and torch.all(codes[7, 4:] == -127)
    good = [0, 1, 2, 3, 4, 7, 9]
    check_codes(vp, case.heads(case.rows)[2].double()[good], page[good], row[good])
    read = [torch.empty(10, 1, 64, dtype=DT[dtype], device=DEV) for _ in range(2)]
    H.halo_paged_read_q8(case.shape, case.pos.to(DEV), case.table.to(DEV), kp, vp, *read, seq=case.seq.to(DEV))
    assert torch.isnan(read[1][[5, 6, 8]]).all() and torch.isfinite(read[1][good]).all()


def test_ties_of_float_rows():
    # largest 127 m with odd m of 16 bits: steps of m, and rows of (c + 1/2) m, 24 bits: quotients that no product with a rounded 127 / largest gives
    case = Append("f32", 8, 8, 64, 16, [(0, 200)], 0, False)
    g = torch.Generator().manual_seed(5)
    m = torch.randint(1 << 14, 1 << 15, (200, 8, 1), generator=g).double() * 2 + 1
    x = (torch.randint(-126, 126, (200, 8, 64), generator=g).double() + 0.5) * m
    x[..., 9] = 127 * m[..., 0]
    case.rows[:, 16:24] = x.float()
    assert torch.equal(case.rows[:, 16:24].double(), x)
    _, (_, vp) = case.run(True, norm=False)
    page, row, _ = case.there()
    assert torch.equal(vp[0].cpu()[page, :, row].double(), torch.round(x / m)) and torch.equal(vp[1].cpu()[page, :, row].double(), m[..., 0])


@pytest.mark.parametrize("codes", [False, True])
def test_padding_writes_nothing(codes):
    # sequences, positions and pages that are none, one of each kind between good tokens
    case = Append("bf16", 4, 2, 64, 16, [(0, 12), (10, 4)], 64, False)
    case.pos[1], case.pos[3], case.pos[5] = -1, 1 << 30, 14           # the last: past the table of angles
    case.seq[7], case.seq[9] = -1, 2
    case.table[1, 0] = case.shape.n_pages
    out, pools = case.run(codes)
    q, k, v, size = case.want()
    page, row, ok = case.there()
    assert ok.sum() == 7 and torch.all(out.cpu()[~ok] == 0)
    case.near(out, q, size[0])
    if codes:
        check_codes(pools[0], k[ok], page[ok], row[ok])
        assert int((pools[1][1] != -5.0).sum()) == 7 * 2
        read = [torch.full((16, 2, 64), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        H.halo_paged_read_q8(case.shape, case.pos.to(DEV), case.table.to(DEV), *pools, *read, seq=case.seq.to(DEV))
        none = [1, 3, 7, 9, 12, 13, 14, 15]                           # no table of angles here: position 14 is one, of a row that nobody wrote
        assert all(torch.all(r[none] == 0) for r in read) and torch.all(read[0][5] == -5.0 * 99)
    else:
        assert int((~torch.isnan(pools[1][:, 0, :, 0])).sum()) == 7


@pytest.mark.parametrize("codes", [False, True])
def test_without_queries_without_a_list_and_dense(codes):
    case = Append("f32", 4, 2, 32, 16, [(4, 1), (16, 1), (31, 1)], 32, False, fused=False)
    case.seq = None
    _, with_q = case.run(codes)
    _, pools = case.run(codes, with_q=False)
    for a, b in zip(with_q, pools):
        assert all(torch.equal(torch.nan_to_num(x.float()), torch.nan_to_num(y.float())) for x, y in zip(a if codes else (a,), b if codes else (b,)))
    q, k, v, size = case.want()
    page, row, ok = case.there()
    if codes:
        check_codes(pools[0], k, page, row)
    else:
        case.near(pools[0].cpu()[page, :, row], k, size[1])


def test_norms_of_zeros_and_of_nan():
    # a head of zeros has a norm of 0 (eps > 0); NaN stays in its head, and in its cache row
    case = Append("bf16", 4, 2, 64, 16, [(0, 6)], 64, False)
    clean, cleaned = case.run(False)
    case.rows[2, 1], case.rows[3, 4] = 0, 0
    case.rows[4, 0, 3], case.rows[5, 5, 9] = math.nan, math.inf
    out, pools = case.run(False)
    page, row, _ = case.there()
    assert torch.all(out[2, 1] == 0) and torch.all(pools[0].cpu()[page[3], 0, row[3]] == 0)
    assert torch.isnan(out[4, 0]).all() and torch.isnan(pools[0].cpu()[page[5], 1, row[5]]).any()
    keep = torch.ones(6, 4, dtype=torch.bool)
    keep[2, 1] = keep[4, 0] = False
    assert torch.equal(out.cpu()[keep], clean.cpu()[keep]) and torch.equal(pools[0].cpu()[page[5], 0, row[5]], cleaned[0].cpu()[page[5], 0, row[5]])


# ---------------------------------------------------------------- attention of single tokens over codes
def attend_case(dtype, Hq, Hk, D, page, lens, keep=None, seed=0, extra=1):
    g = torch.Generator().manual_seed(seed)
    need = [max(0, -(-n // page)) for n in lens]
    n_pages, width = sum(need) + 2, max(need) + extra
    ids = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), width), int(ids[-1]), dtype=torch.int32)
    shape = H.PagedShape(Hq, Hk, D, page, n_pages, width, dtype)
    pools = [(torch.randint(-127, 128, shape.pool, generator=g, dtype=torch.int8), torch.full(shape.pool[:3], math.nan)) for _ in range(2)]
    at = 0
    for i, (n, c) in enumerate(zip(lens, need)):
        table[i, :c] = ids[at:at + c]
        at += c
        for _, scales in pools:                                       # behind the length: NaN
            rows = 0.005 + 0.02 * torch.rand((c * page, Hk), generator=g)
            rows[n:] = math.nan
            scales[table[i, :c].long()] = rows.view(c, page, Hk).transpose(1, 2)
    q = (torch.randn((len(lens), Hq, D), generator=g) * 2).to(DT[dtype])
    mask = None if keep is None else (torch.rand((len(lens), Hq), generator=g) < keep).to(torch.uint8)
    return shape, q, pools, table, torch.tensor(lens, dtype=torch.int32), mask


def run_attend(case, max_len=None, scale=None, stream=None):
    shape, q, pools, table, lens, mask = case
    T = q.shape[0]
    ws = torch.full((H.halo_paged_workspace_bytes(shape, T),), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full(q.shape, math.nan, dtype=q.dtype, device=DEV)
    H.halo_paged_attention_q8(shape, q.to(DEV), *(tuple(x.to(DEV) for x in p) for p in pools), table.to(DEV), lens.to(DEV),
                              max(1, int(lens.max())) if max_len is None else max_len, out, ws, mask=None if mask is None else mask.to(DEV), scale=scale,
                              stream=stream)
    torch.cuda.synchronize()
    return out


def check_attend(case, got, max_len=None, scale=None):
    """|error| <= u |o| + 2 gamma W: scores off by D roundings of sum |q k| (three passes of float queries) and one of the key's scale, then as an exponent; exponentials,
    the value's scale, three parts of a probability and the sums over the positions in float.  W = sum_j p_j |v_j|."""
    shape, q, pools, table, lens, mask = case
    lens = lens.numpy() if max_len is None else np.minimum(lens.numpy(), max_len)
    sc = shape.head_dim ** -0.5 if scale is None else scale
    # what the rows stand for has at most 31 bits: the oracle takes floats, so off by one rounding each, which the bound has
    k, v = (c.float() * s[..., None] for c, s in pools)
    args = np64(q), np64(k), table.numpy(), lens, None if mask is None else mask.numpy(), sc
    want = ref.paged_attention(args[0], args[1], np64(v), *args[2:])
    W = ref.paged_attention(args[0], args[1], np.abs(np64(v)), *args[2:])
    S = abs(sc) * float(np.sqrt((np64(q) ** 2).sum(-1).max() * (np.nan_to_num(np64(k)) ** 2).sum(-1).max()))
    gamma = F * (6 * shape.head_dim * S + 12 * S + 3.0 * max(1, int(np.max(lens))) + 80)
    u = U[shape.dtype]
    got = np64(got)
    assert np.all(np.isfinite(got))
    off = np.abs(got - want) - (u * np.abs(want) + 2 * gamma * W * (1 + u))
    assert np.all(off <= 0), (np.argwhere(off > 0)[:4], off.max())
    assert np.all(got[want == 0] == 0)


SHORT = [1, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 255, 256, 257]
ATTENDS = [
    (4, 4, 128, 16, SHORT, None), (8, 2, 64, 16, SHORT, None), (8, 1, 256, 16, [5, 70, 300], None), (5, 5, 16, 16, [1, 33, 200], None),
    (6, 2, 80, 64, [1, 33, 200], None), (4, 2, 144, 16, [9, 90], None), (20, 1, 128, 16, [50, 3], None), (66, 2, 64, 32, [100], None),
    (256, 256, 16, 16, [20, 40], 0.5), (8, 2, 128, 16, [0, 30, 0, 99], None), (32, 32, 128, 16, [301], 0.5), (12, 4, 96, 32, SHORT, 0.4),
    (8, 8, 128, 16, [2000, 1, 0, 1025, 9000], 0.6), (64, 8, 128, 64, [9003], None), (40, 2, 64, 16, [5500, 700, 33], 0.5),
    (20, 1, 256, 256, [3100, 64], 0.7), (2, 2, 80, 16, [6600] * 3, None), (1, 1, 128, 4096, [9000], None), (2, 1, 240, 16, [2100, 900], 0.8),
    (16, 2, 64, 16, [50 + 77 * i for i in range(70)], 0.5), (40, 2, 128, 16, [2000, 33, 0, 1500] * 34, 0.6), (96, 2, 96, 16, [9000, 700] * 12, 0.3),
    (16, 8, 128, 16, [1 + i % 16 for i in range(70)], 0.7), (8, 8, 64, 32, [6 * i for i in range(80)], 0.6),
    (32, 8, 128, 16, [(11 * i) % 1025 for i in range(70)], None), (20, 1, 16, 16, [40000, 30000, 5], None),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("args", ATTENDS, ids=lambda a: "-".join(map(str, a[:4])) + f"-{max(a[4])}x{len(a[4])}")
def test_attention_over_codes(dtype, args):
    case = attend_case(dtype, *args[:5], keep=args[5])
    check_attend(case, run_attend(case))


@pytest.mark.parametrize("longest", [900, 9000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_and_pages_that_are_none(dtype, longest):
    case = list(attend_case(dtype, 8, 2, 64, 16, [longest, 100, 64, 200, 48, 40], keep=0.6, seed=5))
    shape, q, pools, table, lens, mask = case
    table[1, 2], table[1, 3], table[2, :4] = -1, shape.n_pages, -(1 << 31)
    table[3, 12] = (1 << 31) - 1
    lens[4] = -5
    mask[5], mask[0, :4] = 0, 0
    got = run_attend(case)
    check_attend(case, got)
    assert torch.all(got[[2, 4, 5]] == 0) and torch.all(got[0, :4] == 0)
    lens[0] = 1 << 30
    check_attend(case, run_attend(case, max_len=longest - 3), max_len=longest - 3)
    mask[:] = 0
    assert torch.all(run_attend(case, max_len=longest) == 0)


@pytest.mark.parametrize("longest", [300, 9000])
def test_a_row_of_nan_reaches_its_cache_head_only(longest):
    case = attend_case("bf16", 4, 2, 64, 16, [longest, 40], seed=6)
    clean = run_attend(case)
    page = int(case[3][0, 5])
    case[2][1][1][page, 1, 3] = math.nan
    got = run_attend(case)
    assert torch.isnan(got[0, 2:]).all() and torch.equal(got[0, :2], clean[0, :2]) and torch.equal(got[1], clean[1])


@pytest.mark.parametrize("scale", [0.0, -0.5, 2.0])
def test_scales(scale):
    case = attend_case("bf16", 4, 2, 64, 16, [300, 20], seed=7)
    check_attend(case, run_attend(case, scale=scale), scale=scale)


def test_a_run_of_them_as_they_are_used():
    """Prompts appended as codes, normed and rotated, and attended over as a chunk; then single tokens over the same cache, captured once and replayed: each result is
    that of the formula over what the cache stands for."""
    Hq, Hk, D, page, counts, steps = 8, 2, 64, 16, [37, 5, 60], 4
    g = torch.Generator().manual_seed(8)
    per = -(-(max(counts) + steps) // page)
    shape = H.PagedShape(Hq, Hk, D, page, 3 * per, per)
    table = torch.randperm(3 * per, generator=g).to(torch.int32).view(3, per).to(DEV)
    k, v = ((torch.zeros(shape.pool, dtype=torch.int8, device=DEV), torch.zeros(shape.pool[:3], device=DEV)) for _ in range(2))
    rope = torch.from_numpy(H.halo_rope_table(per * page, D)).to(DEV)
    w = [(1 + 0.1 * torch.randn(D, generator=g)).to(torch.bfloat16).to(DEV) for _ in range(2)]
    N = sum(counts)
    qkv = torch.randn(N, Hq + 2 * Hk, D, generator=g).to(torch.bfloat16).to(DEV)
    seq = torch.repeat_interleave(torch.arange(3), torch.tensor(counts)).to(torch.int32).to(DEV)
    pos = torch.cat([torch.arange(n) for n in counts]).to(torch.int32).to(DEV)
    starts = torch.tensor([0, 37, 42, 102], dtype=torch.int32, device=DEV)
    lens = torch.tensor(counts, dtype=torch.int32, device=DEV)
    q, out = torch.empty(N, Hq, D, dtype=torch.bfloat16, device=DEV), torch.empty(N, Hq, D, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(max(H.halo_paged_chunk_workspace_bytes(shape, N, 3), H.halo_paged_workspace_bytes(shape, 3)), dtype=torch.uint8, device=DEV)
    H.halo_paged_append_q8(shape, qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:], pos, table, k, v, q_out=q, qk_norm=True, w_q=w[0], w_k=w[1], rope=rope,
                           seq=seq)
    H.halo_paged_chunk_attention_q8(shape, q, k, v, table, starts, lens, per * page, out, ws)

    def attended(q, s, n):
        ids = table[s].long()
        kk, vv = ((p[0][ids].double() * p[1][ids].double()[..., None]).permute(0, 2, 1, 3).reshape(-1, Hk, D)[:n] for p in (k, v))
        score = torch.einsum("hd,jhd->hj", q.double(), kk.repeat_interleave(Hq // Hk, 1)) * D ** -0.5
        p = torch.softmax(score, -1)
        values = vv.repeat_interleave(Hq // Hk, 1)
        return torch.einsum("hj,jhd->hd", p, values), torch.einsum("hj,jhd->hd", p, values.abs())

    def close(got, q, s, n):
        o, W = attended(q, s, n)
        # a rounding that stores, one of each probability; scores of up to about 8, 64 products each, and the sums over the positions, in float
        assert torch.all((got.double() - o).abs() <= U["bf16"] * o.abs() + (U["bf16"] + 2 * F * (2 * 64 * 64 + 100)) * W)

    for t in range(N):
        close(out[t], q[t], int(seq[t]), int(pos[t]) + 1)
    new, q1, o1 = torch.zeros(3, Hq + 2 * Hk, D, dtype=torch.bfloat16, device=DEV), torch.empty(3, Hq, D, dtype=torch.bfloat16, device=DEV), torch.empty(
        3, Hq, D, dtype=torch.bfloat16, device=DEV)
    at, after = lens.clone(), lens.clone()

    def token():
        H.halo_paged_append_q8(shape, new[:, :Hq], new[:, Hq:Hq + Hk], new[:, Hq + Hk:], at, table, k, v, q_out=q1, qk_norm=True, w_q=w[0], w_k=w[1], rope=rope)
        torch.add(at, 1, out=after)
        H.halo_paged_attention_q8(shape, q1, k, v, table, after, per * page, o1, ws)
        at.add_(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token()
    at.copy_(lens)
    for i in range(steps):
        new.copy_(torch.randn(new.shape, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        for s in range(3):
            close(o1[s], q1[s], s, counts[s] + i + 1)


def test_offsets_past_32_bits():
    # rows whose codes lie past 2^32 bytes, and their scales too
    D, page, Hk = 16, 4096, 2
    n_pages = (1 << 30) // (Hk * page) + 3
    shape = H.PagedShape(4, Hk, D, page, n_pages, 2)
    pools = [(torch.empty(shape.pool, dtype=torch.int8, device=DEV), torch.empty(shape.pool[:3], device=DEV)) for _ in range(2)]
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device=DEV)
    g = torch.Generator().manual_seed(9)
    n = 4096 + 30
    rows = torch.randn(n, 4 + 2 * Hk, D, generator=g).to(torch.bfloat16).to(DEV)
    pos, seq = torch.arange(n, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    H.halo_paged_append_q8(shape, None, rows[:, 4:6], rows[:, 6:], pos, table, *pools, seq=seq)
    read = [torch.empty(n, Hk, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    H.halo_paged_read_q8(shape, pos, table, *pools, *read, seq=seq)
    for x, r in zip((rows[:, 4:6], rows[:, 6:]), read):
        assert torch.all((r.double() - x.double()).abs() <= x.double().abs().amax(-1, keepdim=True) * (1 / 254 + 2.0 ** -8) * (1 + 1e-5))
    lens, q = torch.tensor([n], dtype=torch.int32, device=DEV), rows[:1, :4].contiguous()
    out = torch.empty(1, 4, D, dtype=torch.bfloat16, device=DEV)
    H.halo_paged_attention_q8(shape, q, *pools, table, lens, n, out, torch.empty(H.halo_paged_workspace_bytes(shape, 1), dtype=torch.uint8, device=DEV))
    kk, vv = (torch.cat([p[0][t].double() * p[1][t].double()[..., None] for t in (n_pages - 1, n_pages - 2)], 1)[:, :n] for p in pools)
    score = torch.stack([kk[h // 2] @ q[0, h].double() for h in range(4)]) / 4
    p = torch.softmax(score, -1)
    o, W = (torch.stack([p[h] @ x[h // 2] for h in range(4)]) for x in (vv, vv.abs()))
    assert torch.all((out[0].double() - o).abs() <= 2.0 ** -8 * o.abs() + 2 * F * (6 * 16 * 16 + 3 * n + 80) * W)
    del pools
    torch.cuda.empty_cache()
