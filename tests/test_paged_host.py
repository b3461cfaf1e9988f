"""Serving a batch over a paged cache, without a GPU: where tokens lie and how the work is cut (the kernels' own integer arithmetic, built
for the host), what the entry points refuse, the rotation table, and the oracle's definitions against plain numpy."""
import ctypes as C
import json
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2601_11676_amd as H
from oracle import ref

HERE = os.path.dirname(os.path.abspath(__file__))


# ---------------------------------------------------------------- index arithmetic
@pytest.fixture(scope="module")
def index(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("paged") / "check")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-o", exe,
                    os.path.join(HERE, "paged_index_check.cpp")], check=True)

    def ask(lines):
        p = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=60)
        assert p.returncode == 0, p.stderr
        return p.stdout.split()
    return ask


def test_rows_and_pages_that_are_none(index):
    # a page outside the pool is no row; the last row of a pool past 2^31 rows is in it
    asked, want = [], []
    for n, kv, shift in [(1, 1, 4), (7, 3, 4), (100, 8, 8), (1 << 20, 256, 12)]:
        for page in (0, n - 1, n, -1, -(1 << 31), (1 << 31) - 1):
            for head, pos in [(0, 0), (kv - 1, (1 << shift) - 1), (kv - 1, 5 * (1 << shift) + 3), (0, (1 << 30) - 1)]:
                asked.append(f"row {n} {kv} {shift} {page} {head} {pos}")
                want.append(((page * kv + head) << shift) + pos % (1 << shift) if 0 <= page < n else -1)
    got = [int(v) for v in index(asked)]
    assert got == want
    assert max(got) == (1 << 40) - 1
    assert [int(v) for v in index(["len -5 10", "len 0 10", "len 7 10", "len 10 10", "len 2000000000 10"])] == [0, 0, 7, 10, 10]


def test_every_tile_has_one_worker_and_both_launches_agree(index):
    rng = np.random.default_rng(3)
    asked = ["cut 2048 4 1 1", "cut 4 1 3 0 0 0", "cut 2 1 2 1 1", "cut 8 4 0", "cut 3 2 4 5 0 1 6"]
    for _ in range(400):
        n = int(rng.integers(1, 40))
        tiles = rng.integers(0, int(rng.choice([2, 5, 40, 300])), n)
        asked.append(f"cut {rng.choice([1, 4, 36, 2048])} {rng.choice([1, 2, 4, 16])} {n} " + " ".join(map(str, tiles)))
    assert set(index(asked)) == {"ok"}


# ---------------------------------------------------------------- refusals
ONE, ODD, NULL, ST = C.c_void_p(0x1000), C.c_void_p(0x1004), None, C.c_void_p(0)     # never dereferenced


def _refused(fn, args, cases):
    for at, value, code in cases:
        a = list(args)
        for i, v in zip(at, value) if isinstance(at, tuple) else [(at, value)]:
            a[i] = v
        assert fn(*a) == code, (at, value, code)


def _shape(**kw):
    return H.PagedShape(**{**dict(n_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=10, max_pages=4), **kw})


BAD_SHAPES = [(dict(dtype="fp8"), -3), (dict(n_kv_heads=3), -2), (dict(n_kv_heads=0), -2), (dict(n_heads=0), -2), (dict(n_heads=258), -2),
              (dict(head_dim=72), -2), (dict(head_dim=0), -2), (dict(head_dim=272), -2), (dict(page_size=8), -2), (dict(page_size=48), -2),
              (dict(page_size=8192), -2), (dict(n_pages=0), -2), (dict(max_pages=0), -2), (dict(max_pages=(1 << 26) + 1), -2)]


def test_append_refuses():
    fn, s = H.load_library().halo_paged_append, _shape()
    args = [C.byref(s.c), 3, ONE, 512, ONE, 128, ONE, 128, ONE, ONE, 2, ONE, ONE, 64, 64, 0, C.c_void_p(0x9000), ONE, ONE, ST]
    _refused(fn, args, [(0, None, -1), (4, NULL, -1), (6, NULL, -1), (8, NULL, -1), (11, NULL, -1), (17, NULL, -1), (18, NULL, -1),
                        (2, NULL, -1), (16, NULL, -1),                              # q and q_out go together
                        (1, -1, -4), (10, 0, -4), (3, 511, -4), (3, 516, -4), (5, 127, -4), (7, 0, -4), (7, -128, -4), (16, ONE, -4),
                        (2, ODD, -4), (4, ODD, -4), (6, ODD, -4), (16, ODD, -4), (17, ODD, -4), (18, ODD, -4), (12, ODD, -4),
                        (8, C.c_void_p(0x1002), -4), (9, C.c_void_p(0x1001), -4), (11, C.c_void_p(0x1003), -4),
                        (13, 0, -4), (14, 8, -4), (14, 72, -4), (14, 80, -4),
                        (1, 0, 0)])                                                 # nothing to do
    for kw, code in BAD_SHAPES:
        b = _shape(**kw)
        assert fn(C.byref(b.c), *args[1:]) == code, kw


def test_attention_refuses():
    fn, s = H.load_library().halo_paged_attention, _shape()
    need = H.halo_paged_workspace_bytes(s, 3)
    args = [C.byref(s.c), 3, ONE, 512, ONE, ONE, ONE, ONE, 64, ONE, 0.125, ONE, ONE, need, ST]
    _refused(fn, args, [(0, None, -1), (2, NULL, -1), (4, NULL, -1), (5, NULL, -1), (6, NULL, -1), (7, NULL, -1), (11, NULL, -1),
                        (1, -1, -4), (1, 4097, -4), (8, 0, -4), (8, 65, -4), (10, float("nan"), -4), (10, float("inf"), -4),
                        (3, 511, -4), (3, 504, -4), (3, 516, -4), (2, ODD, -4), (4, ODD, -4), (5, ODD, -4), (11, ODD, -4),
                        (6, C.c_void_p(0x1002), -4), (7, C.c_void_p(0x1001), -4), (12, ODD, -4),
                        (12, NULL, -5), (13, need - 1, -5),
                        (1, 0, 0)])
    for kw, code in BAD_SHAPES:
        b = _shape(**kw)
        assert fn(C.byref(b.c), *args[1:]) == code, kw
        assert H.halo_paged_workspace_bytes(b, 3) == 0
    # tiles that 32 bits do not number
    big = _shape(n_heads=256, n_kv_heads=256, max_pages=1 << 20)
    assert fn(C.byref(big.c), 4096, ONE, 256 * 64, ONE, ONE, ONE, ONE, 1 << 24, NULL, 1.0, ONE, ONE, 1 << 40, ST) == -4


def test_norm_refuses():
    fn = H.load_library().halo_block_norm
    args = [ONE, ONE, ONE, ONE, ONE, ONE, ONE, 2, 64, 1, 1, 1, 0, 1.0, 1e-5, ST]
    _refused(fn, args, [(0, NULL, -1), (1, NULL, -1), (5, NULL, -1), (6, NULL, -1), (9, 2, -3), ((9, 10), (0, 1), -3), (10, -1, -3),
                        (7, -1, -4), (8, 0, -4), (8, 60, -4), (8, 32776, -4), (14, -1.0, -4), (14, float("nan"), -4),
                        (13, float("inf"), -4), (13, float("nan"), -4), *[(i, ODD, -4) for i in range(7)], (7, 0, 0)])


def test_workspace_grows_with_the_sequences_only():
    s = _shape()
    sizes = [H.halo_paged_workspace_bytes(s, T) for T in (0, 1, 2, 63, 64, 1000, 4096)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert H.halo_paged_workspace_bytes(s, 4097) == 0 and H.halo_paged_workspace_bytes(s, -1) == 0


def test_binding_refuses_what_the_library_cannot_see():
    s = _shape()
    x, i = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        H.halo_paged_append(s, None, x, x, i, i, x, x)
    with pytest.raises(ValueError, match="device tensor"):
        H.halo_paged_attention(s, x, x, x, i, i, 16, x, x)
    with pytest.raises(ValueError):
        H.halo_block_norm(torch.zeros(2, 64), torch.zeros(2, 64), torch.zeros(2, 64))


# ---------------------------------------------------------------- what is launched
LAUNCHES = """
import ctypes as C, json, sys
recorder = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
recorder.recorder_take.restype = C.c_char_p
lib = C.CDLL(sys.argv[2])
lib.halo_paged_workspace_bytes.restype = C.c_size_t
p, out = C.c_void_p(1 << 30), []
for heads, kv, dim, dtype, T, max_len, mask in json.load(sys.stdin):
    shape = C.byref((C.c_int32 * 7)(heads, kv, dim, 16, 1000, max(1, (max_len + 15) // 16), dtype))
    ws = lib.halo_paged_workspace_bytes(shape, T)
    rc = lib.halo_paged_attention(shape, T, p, C.c_int64(heads * dim), p, p, p, p, max_len, p if mask else None, C.c_float(1.0), p, p,
                                  C.c_size_t(ws), None)
    out.append((rc, [l.split() for l in recorder.recorder_take().decode().split("\\n")[:-1]]))
json.dump(out, sys.stdout)
"""


def _launches(calls, tmp_path):
    shim = str(tmp_path / "recorder.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", shim, os.path.join(HERE, "launch_recorder.c")], check=True)
    p = subprocess.run([sys.executable, "-c", LAUNCHES, shim, H.library_path()], input=json.dumps(calls), capture_output=True, text=True,
                       timeout=120)
    assert p.returncode == 0, p.stderr
    return json.loads(p.stdout)


def test_attention_launches(tmp_path):
    # (heads, cache heads, dim, dtype, sequences, longest, mask) -> kernels and workgroups
    cases = [((32, 8, 128, 1, 1, 2048, 0), [("attend_item", 8, 512)]), ((32, 8, 128, 1, 1, 2049, 0), [("attend_stream", 65, 256), ("attend_join", 8, 256)]),
             ((32, 8, 64, 1, 64, 4096, 1), [("attend_item", 512, 512)]), ((32, 8, 64, 1, 63, 4096, 1), [("attend_stream", 512, 256), ("attend_join", 504, 256)]),
             ((32, 8, 256, 1, 64, 2049, 1), [("attend_stream", 256, 256), ("attend_join", 512, 256)]),
             ((20, 1, 64, 1, 3, 2048, 0), [("attend_item", 6, 512)]), ((40, 4, 64, 1, 64, 2048, 0), [("attend_item", 256, 512)]),
             ((160, 8, 128, 1, 16, 8000, 0), [("attend_stream", 256, 256), ("attend_join", 128, 256)]), ((71, 1, 64, 1, 200, 5000, 0), [("attend_stream", 512, 256), ("attend_join", 600, 256)]), ((12, 4, 64, 0, 5, 1536, 0), [("attend_item", 20, 512)]),
             ((12, 4, 64, 0, 5, 1537, 0), [("attend_stream", 123, 256), ("attend_join", 20, 256)]), ((20, 4, 64, 0, 5, 1024, 0), [("attend_item", 20, 512)]),
             ((20, 4, 64, 0, 5, 1025, 0), [("attend_stream", 83, 256), ("attend_join", 20, 256)]), ((8, 8, 256, 1, 1, 1024, 0), [("attend_item", 8, 256)]),
             ((8, 8, 256, 0, 1, 513, 0), [("attend_stream", 17, 256), ("attend_join", 8, 256)]), ((256, 256, 16, 1, 4096, 4096, 1), [("attend_item", 1 << 20, 512)]),
             ((256, 256, 16, 1, 4096, 9000, 1), [("attend_stream", 512, 256), ("attend_join", 1 << 20, 256)]), ((8, 8, 64, 1, 0, 64, 0), []),
             # fewer waves: up to two tiles, and of 512 pairs up to 8 and 16
             ((32, 8, 64, 1, 1, 64, 0), [("attend_item", 8, 128)]), ((32, 8, 128, 1, 1, 65, 0), [("attend_item", 8, 512)]),
             ((32, 8, 128, 1, 64, 256, 0), [("attend_item", 512, 128)]), ((32, 8, 128, 1, 64, 257, 0), [("attend_item", 512, 256)]),
             ((32, 8, 128, 1, 64, 512, 0), [("attend_item", 512, 256)]), ((32, 8, 128, 1, 64, 513, 0), [("attend_item", 512, 512)]),
             ((32, 8, 128, 1, 63, 256, 0), [("attend_item", 504, 512)]), ((16, 16, 128, 0, 32, 128, 0), [("attend_item", 512, 128)]),
             ((16, 16, 128, 0, 32, 129, 0), [("attend_item", 512, 256)]),
             # more than 16 queries a cache head: 32 at a time of caches past 64 MiB
             ((20, 1, 128, 0, 64, 1024, 0), [("attend_stream", 512, 256), ("attend_join", 128, 256)]),
             ((20, 1, 128, 0, 64, 1025, 0), [("attend_stream", 256, 256), ("attend_join", 64, 256)]),
             ((20, 1, 144, 0, 64, 1025, 0), [("attend_stream", 256, 256), ("attend_join", 128, 256)]),
             ((160, 8, 128, 0, 64, 129, 0), [("attend_item", 512, 256)]), ((160, 8, 128, 1, 64, 257, 0), [("attend_item", 512, 256)])]
    for (call, want), (rc, got) in zip(cases, _launches([c for c, _ in cases], tmp_path)):
        assert rc == 0, call
        assert len(got) == len(want), (call, got)
        for (name, x, y, z, threads), (n, grid, block) in zip(got, want):
            cut = int(y) if n == "attend_join" else 1                 # of a pair over workgroups
            assert n in name and int(x) * int(y) * int(z) == grid * cut and int(threads) == block, (call, got)


# ---------------------------------------------------------------- rotation table
@pytest.mark.parametrize("n,dim,theta", [(1, 2, 10000.0), (70, 64, 10000.0), (9000, 16, 500000.0), (300, 128, 1.0)])
def test_rope_table(n, dim, theta):
    got = H.halo_rope_table(n, dim, theta)
    angle = np.arange(n)[:, None] * np.float64(theta) ** (-2.0 * np.arange(dim // 2) / dim)
    want = np.stack([np.cos(angle), np.sin(angle)], axis=1)
    # one rounding to float (2^-24 of the value), and the double angle's own: up to a few units of 2^-53 of the largest angle
    assert got.dtype == np.float32 and got.shape == want.shape
    assert np.all(np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + 8 * 2.0 ** -53 * n)


def test_rope_table_refuses():
    lib = H.load_library()
    buf = np.zeros(64, dtype=np.float32).ctypes.data_as(C.c_void_p)
    for n, dim, theta, code in [(-1, 4, 1e4, -4), (1, 0, 1e4, -4), (1, 3, 1e4, -4), (1, 4, 0.0, -4), (1, 4, float("nan"), -4),
                                (1, 4, float("inf"), -4), (0, 4, 1e4, 0)]:
        assert lib.halo_rope_table(n, dim, theta, buf) == code
    assert lib.halo_rope_table(1, 4, 1e4, None) == -1


# ---------------------------------------------------------------- the oracle against numpy
def test_oracle_append_is_a_complex_product():
    rng = np.random.default_rng(1)
    N, Hq, Hk, D, page = 6, 3, 1, 32, 16
    q, k, v = (rng.standard_normal((N, h, D)).astype(np.float32) for h in (Hq, Hk, Hk))
    table = np.array([[3, 1], [0, 9]], dtype=np.int32)
    pos, seq = np.array([0, 15, 16, 31, 20, 2]), np.array([0, 0, 0, 0, 1, 1])     # token 4: page 9 does not exist
    kp = np.zeros((4, Hk, page, D))
    for pairs in (False, True):
        rope = H.halo_rope_table(32, 16)
        out, k2, v2 = ref.paged_append(q, k, v, pos, seq, table, rope, pairs, kp, kp)
        turn = rope[pos, 0] + 1j * rope[pos, 1].astype(np.float64)
        a, b = (slice(0, 16, 2), slice(1, 16, 2)) if pairs else (slice(0, 8), slice(8, 16))
        for x, y in ((q, out), (k, np.stack([k2[table[s, p // page], :, p % page] if (s, p) != (1, 20) else k[0] * np.nan
                                             for s, p in zip(seq, pos)]))):
            z = (x[..., a] + 1j * x[..., b].astype(np.float64)) * turn[:, None]
            for i in (0, 1, 2, 3, 5):
                assert np.allclose(y[i][:, a], z[i].real, atol=1e-12) and np.allclose(y[i][:, b], z[i].imag, atol=1e-12)
                assert np.array_equal(y[i][:, 16:], x[i][:, 16:])
        assert np.all(out[4] == 0) and np.count_nonzero(np.abs(v2).sum((1, 3))) == 5
        assert np.array_equal(v2[1, :, 15], v[3])


def test_oracle_attention_is_softmax():
    rng = np.random.default_rng(2)
    T, Hq, Hk, D, page = 3, 4, 2, 16, 16
    q = rng.standard_normal((T, Hq, D)).astype(np.float32)
    kp, vp = (rng.standard_normal((8, Hk, page, D)).astype(np.float32) for _ in range(2))
    table = np.array([[5, 2, 7], [0, -1, 3], [1, 1, 1]], dtype=np.int32)
    lens, mask = np.array([37, 40, 0]), np.array([[1, 0, 1, 1], [1, 1, 1, 1], [1, 1, 1, 1]])
    out = ref.paged_attention(q, kp, vp, table, lens, mask)
    for t in range(2):
        there = [j for j in range(lens[t]) if table[t, j // page] >= 0]
        assert len(there) == (37 if t == 0 else 24)
        for h in range(Hq):
            K, V = (np.stack([p[table[t, j // page], h // 2, j % page] for j in there]).astype(np.float64) for p in (kp, vp))
            e = np.exp(K @ q[t, h] / 4.0)
            assert np.allclose(out[t, h], mask[t, h] * (e @ V) / e.sum(), atol=1e-12)
    assert np.all(out[2] == 0)


def test_oracle_norm():
    rng = np.random.default_rng(3)
    h, y, g, a, b = (rng.standard_normal(s).astype(np.float32) for s in ((2, 24), (2, 24), (24,), (24,), (24,)))
    h2, x = ref.block_norm(h, y, a, g, b, True, 0.5, 1e-3)
    u = y / np.sqrt((y.astype(np.float64) ** 2).mean(1, keepdims=True) + 1e-3) * a * g
    assert np.allclose(h2, 0.5 * h + u, atol=1e-12)
    assert np.allclose(x, h2 / np.sqrt((h2 ** 2).mean(1, keepdims=True) + 1e-3) * b, atol=1e-12)
    h2, x = ref.block_norm(h, y, a, None, None, False)               # w_post has no meaning without the norm it scales
    assert np.allclose(h2, h.astype(np.float64) + y, atol=1e-12)
