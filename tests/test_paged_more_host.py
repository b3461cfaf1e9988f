"""Chunks over a paged cache, a cache of codes and appends that norm, without a GPU: what the entry points refuse, calls that do nothing, the workspace, what is launched."""
import ctypes as C
import json
import os
import subprocess
import sys

import pytest
import torch

import paper_2601_11676_amd as H
from paper_2601_11676_amd.binding import _pool_q8

HERE = os.path.dirname(os.path.abspath(__file__))
ONE, ODD, OFF, NULL, ST = C.c_void_p(0x1000), C.c_void_p(0x1004), C.c_void_p(0x1002), None, C.c_void_p(0)     # never dereferenced


def _refused(fn, args, cases):
    for at, value, code in cases:
        a = list(args)
        for i, v in zip(at, value) if isinstance(at, tuple) else [(at, value)]:
            a[i] = v
        assert fn(*a) == code, (at, value, code)


def _shape(**kw):
    return H.PagedShape(**{**dict(n_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=10, max_pages=4), **kw})


BAD_SHAPES = [(dict(dtype="fp8"), -3), (dict(n_kv_heads=3), -2), (dict(n_kv_heads=0), -2), (dict(n_heads=258), -2), (dict(head_dim=72), -2),
              (dict(head_dim=272), -2), (dict(page_size=8), -2), (dict(page_size=48), -2), (dict(n_pages=0), -2), (dict(max_pages=0), -2)]
TOKENS = [(2, NULL, -1), (4, NULL, -1), (6, NULL, -1), (8, NULL, -1), (11, NULL, -1), (1, -1, -4), (10, 0, -4), (3, 511, -4), (3, 516, -4), (5, 127, -4),
          (7, 0, -4), (7, -128, -4), (2, ODD, -4), (4, ODD, -4), (6, ODD, -4), (8, OFF, -4), (9, OFF, -4), (11, OFF, -4), (1, 0, 0)]


def test_append_norm_refuses():
    fn, s = H.load_library().halo_paged_append_norm, _shape()
    args = [C.byref(s.c), 3, ONE, 512, ONE, 128, ONE, 128, ONE, ONE, 2, ONE, ONE, ONE, 1e-5, ONE, 64, 64, 0, C.c_void_p(0x9000), ONE, ONE, ST]
    _refused(fn, args, TOKENS + [(0, None, -1), (19, NULL, -1), (20, NULL, -1), (21, NULL, -1), (19, ONE, -4), (12, ODD, -4), (13, ODD, -4), (14, -1.0, -4),
                                 (14, float("nan"), -4), (14, float("inf"), -4), (15, ODD, -4), (16, 0, -4), (17, 8, -4), (17, 72, -4), (17, 80, -4),
                                 (19, ODD, -4), (20, ODD, -4), (21, ODD, -4)])
    for kw, code in BAD_SHAPES:
        b = _shape(**kw)
        assert fn(C.byref(b.c), *args[1:]) == code, kw


def test_append_q8_refuses():
    fn, s = H.load_library().halo_paged_append_q8, _shape()
    args = [C.byref(s.c), 3, ONE, 512, ONE, 128, ONE, 128, ONE, ONE, 2, ONE, 1, ONE, ONE, 1e-5, ONE, 64, 64, 0, C.c_void_p(0x9000), ONE, ONE, ONE, ONE, ST]
    _refused(fn, args, TOKENS + [(0, None, -1), (20, NULL, -1), *[(i, NULL, -1) for i in range(21, 25)], (20, ONE, -4), (13, ODD, -4), (14, ODD, -4),
                                 (15, -1.0, -4), (15, float("nan"), -4), (16, ODD, -4), (17, 0, -4), (18, 8, -4), (21, ODD, -4), (23, ODD, -4), (22, OFF, -4),
                                 (24, OFF, -4)])
    for kw, code in BAD_SHAPES:
        b = _shape(**kw)
        assert fn(C.byref(b.c), *args[1:]) == code, kw


def test_read_q8_refuses():
    fn, s = H.load_library().halo_paged_read_q8, _shape()
    args = [C.byref(s.c), 3, ONE, ONE, 2, ONE, ONE, ONE, ONE, ONE, ONE, ONE, ST]
    _refused(fn, args, [(0, None, -1), (2, NULL, -1), *[(i, NULL, -1) for i in range(5, 12)], (1, -1, -4), (4, 0, -4), (2, OFF, -4), (3, OFF, -4), (5, OFF, -4),
                        (6, ODD, -4), (8, ODD, -4), (7, OFF, -4), (9, OFF, -4), (10, ODD, -4), (11, ODD, -4), (1, 0, 0)])
    for kw, code in BAD_SHAPES:
        b = _shape(**kw)
        assert fn(C.byref(b.c), *args[1:]) == code, kw


def test_attention_q8_refuses():
    fn, s = H.load_library().halo_paged_attention_q8, _shape()
    need = H.halo_paged_workspace_bytes(s, 3)
    args = [C.byref(s.c), 3, ONE, 512, ONE, ONE, ONE, ONE, ONE, ONE, 64, ONE, 0.125, ONE, ONE, need, ST]
    _refused(fn, args, [(0, None, -1), (2, NULL, -1), *[(i, NULL, -1) for i in range(4, 10)], (13, NULL, -1), (1, -1, -4), (1, 4097, -4), (10, 0, -4), (10, 65, -4),
                        (12, float("nan"), -4), (3, 511, -4), (3, 516, -4), (2, ODD, -4), (4, ODD, -4), (6, ODD, -4), (13, ODD, -4), (5, OFF, -4), (7, OFF, -4),
                        (8, OFF, -4), (9, OFF, -4), (14, ODD, -4), (14, NULL, -5), (15, need - 1, -5), (1, 0, 0)])
    for kw, code in BAD_SHAPES:
        b = _shape(**kw)
        assert fn(C.byref(b.c), *args[1:]) == code, kw


@pytest.mark.parametrize("codes", [False, True])
def test_chunks_refuse(codes):
    lib, s = H.load_library(), _shape()
    fn = lib.halo_paged_chunk_attention_q8 if codes else lib.halo_paged_chunk_attention
    need = H.halo_paged_chunk_workspace_bytes(s, 3, 2)
    pools = [ONE] * (4 if codes else 2)
    args = [C.byref(s.c), 3, ONE, 512, *pools, 2, ONE, ONE, ONE, 64, ONE, 0.125, ONE, ONE, need, ST]
    at = 4 + len(pools)                                               # n_seq, starts, page_table, lens, max_len, mask, scale, out, workspace, bytes
    _refused(fn, args, [(0, None, -1), (2, NULL, -1), *[(i, NULL, -1) for i in range(4, at)], (at + 1, NULL, -1), (at + 2, NULL, -1), (at + 3, NULL, -1),
                        (at + 7, NULL, -1), (1, -1, -4), (1, (1 << 21) + 1, -4), (at, -1, -4), (at, 4097, -4), (at + 4, 0, -4), (at + 4, 65, -4),
                        (at + 6, float("nan"), -4), (at + 6, float("inf"), -4), (3, 511, -4), (3, 516, -4), (2, ODD, -4), (4, ODD, -4), (at - 2, ODD if not codes else OFF, -4),
                        (at - 1, ODD if not codes else OFF, -4), (at + 7, ODD, -4), (at + 1, OFF, -4), (at + 2, OFF, -4), (at + 3, OFF, -4), (at + 8, ODD, -4),
                        (at + 8, NULL, -5), (at + 9, need - 1, -5), (1, 0, 0), (at, 0, 0)])
    for kw, code in BAD_SHAPES:
        b = _shape(**kw)
        assert fn(C.byref(b.c), *args[1:]) == code, kw
        assert H.halo_paged_chunk_workspace_bytes(b, 3, 2) == 0


def test_calls_without_tokens_do_nothing_whatever_their_pointers():
    lib, s = H.load_library(), _shape()
    b = C.byref(s.c)
    assert lib.halo_paged_append_norm(b, 0, *[None] * 1, 0, None, 0, None, 0, None, None, 0, None, None, None, 0.0, None, 0, 0, 0, None, None, None, None) == 0
    assert lib.halo_paged_append_q8(b, 0, None, 0, None, 0, None, 0, None, None, 0, None, 0, None, None, 0.0, None, 0, 0, 0, *[None] * 6) == 0
    assert lib.halo_paged_read_q8(b, 0, None, None, 0, *[None] * 8) == 0
    assert lib.halo_paged_attention_q8(b, 0, None, 0, *[None] * 6, 0, None, 0.0, None, None, 0, None) == 0
    assert lib.halo_paged_chunk_attention(b, 0, None, 0, None, None, 3, None, None, None, 0, None, 0.0, None, None, 0, None) == 0
    assert lib.halo_paged_chunk_attention_q8(b, 5, None, 0, *[None] * 4, 0, None, None, None, 0, None, 0.0, None, None, 0, None) == 0


def test_chunk_workspace_serves_smaller_calls():
    s = _shape()
    sizes = [H.halo_paged_chunk_workspace_bytes(s, N, n) for N, n in ((0, 0), (1, 1), (40, 8), (5000, 8), (5000, 4096), (1 << 21, 4096))]
    assert sizes == sorted(sizes) and sizes[0] > 0
    for N, n in ((-1, 1), (1, -1), ((1 << 21) + 1, 1), (1, 4097)):
        assert H.halo_paged_chunk_workspace_bytes(s, N, n) == 0


def test_binding_refuses_what_the_library_cannot_see():
    s = _shape()
    x, i, c = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), torch.zeros(s.pool, dtype=torch.int8)
    pool = (c, torch.zeros(s.pool[:3]))
    for call in (lambda: H.halo_paged_append_norm(s, None, x, x, i, i, x, x), lambda: H.halo_paged_append_q8(s, None, x, x, i, i, pool, pool),
                 lambda: H.halo_paged_read_q8(s, i, torch.zeros(3, 4, dtype=torch.int32), pool, pool, x, x),
                 lambda: H.halo_paged_chunk_attention(s, x, c.bfloat16(), c.bfloat16(), i, i, i, 16, x, x),
                 lambda: H.halo_paged_attention_q8(s, x, pool, pool, i, i, 16, x, x)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(ValueError, match="scales are"):
        _pool_q8((c, torch.zeros(3)), s)
    with pytest.raises(ValueError, match="pages are"):
        _pool_q8((c[1:], pool[1]), s)
    with pytest.raises(ValueError, match="int8"):
        _pool_q8((c.float(), pool[1]), s)
    with pytest.raises(ValueError, match="row of the page table"):
        H.halo_paged_read_q8(s, i, torch.zeros(2, 4, dtype=torch.int32), pool, pool, x, x)


# ---------------------------------------------------------------- what is launched
CALLS = """
import ctypes as C, json, sys
recorder = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
recorder.recorder_take.restype = C.c_char_p
lib = C.CDLL(sys.argv[2])
lib.halo_paged_chunk_workspace_bytes.restype = C.c_size_t
p, i64, out = C.c_void_p(1 << 30), C.c_int64, []
for what, heads, kv, dim, dtype, N, n_seq, max_len, mask in json.load(sys.stdin):
    shape = C.byref((C.c_int32 * 7)(heads, kv, dim, 16, 1000, max(1, (max_len + 15) // 16), dtype))
    if what == "read":
        rc = lib.halo_paged_read_q8(shape, N, p, p, n_seq, p, p, p, p, p, p, p, None)
    elif what == "codes":
        rc = lib.halo_paged_append_q8(shape, N, p, i64(heads * dim), p, i64(kv * dim), p, i64(kv * dim), p, p, n_seq, p, 1, p, p, C.c_float(1e-5), None, 0, 0, 0,
                                      C.c_void_p(1 << 31), p, p, p, p, None)
    else:
        ws = i64(lib.halo_paged_chunk_workspace_bytes(shape, N, n_seq))
        pools = [p] * (4 if what == "q8" else 2)
        fn = lib.halo_paged_chunk_attention_q8 if what == "q8" else lib.halo_paged_chunk_attention
        rc = fn(shape, N, p, i64(heads * dim), *pools, n_seq, p, p, p, max_len, p if mask else None, C.c_float(1.0), p, p, ws, None)
    out.append((rc, [l.split() for l in recorder.recorder_take().decode().split("\\n")[:-1]]))
json.dump(out, sys.stdout)
"""


def _launches(calls, tmp_path):
    shim = str(tmp_path / "recorder.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", shim, os.path.join(HERE, "launch_recorder.c")], check=True)
    p = subprocess.run([sys.executable, "-c", CALLS, shim, H.library_path()], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
    assert p.returncode == 0, p.stderr
    return json.loads(p.stdout)


def test_chunk_launches(tmp_path):
    # (cache, heads, cache heads, dim, dtype, tokens, sequences, longest, mask) -> kernels, rows of a block, workgroups of the first that attends
    up = lambda n: -(-n // 8) * 8
    cases = [(("rows", 64, 8, 128, 1, 512, 1, 16512, 0), ["chunk_attend", "chunk_join"], up(17 * 8 + 256)),              # few blocks: cut
             (("rows", 40, 40, 128, 1, 4099, 7, 937, 1), ["chunk_attend"], 920),                                         # many: whole
             (("rows", 32, 32, 128, 1, 8192, 1, 8192, 1), ["chunk_rows", "chunk_attend"], up(33 * 32)),                  # many scores under a mask
             (("rows", 64, 8, 128, 1, 640, 16, 3040, 0), ["chunk_attend"], up((640 * 8 // 128 + 16) * 8)),               # blocks of 128 rows
             (("q8", 64, 8, 128, 1, 4, 4, 3000, 0), ["chunk_attend", "chunk_join"], up(5 * 8 + 512)),                    # of 32
             (("q8", 64, 8, 128, 1, 4, 4, 256, 0), ["chunk_attend"], up(5 * 8)),                                         # a part has two tiles at least
             (("rows", 12, 4, 64, 0, 777, 3, 545, 0), ["chunk_attend", "chunk_join"], up((777 * 3 // 128 + 3) * 4 + 512)),
             (("q8", 8, 8, 64, 0, 0, 3, 64, 0), [], 0)]
    for (call, names, groups), (rc, got) in zip(cases, _launches([c for c, _, _ in cases], tmp_path)):
        assert rc == 0 and len(got) == len(names), (call, got)
        assert all(n in g[0] for n, g in zip(names, got)), (call, got)
        attend = [g for g in got if "chunk_attend" in g[0]]
        assert not attend or int(attend[0][1]) == groups, (call, got)


def test_grids_of_any_call_stay_within_a_launch(tmp_path):
    calls = [(what, heads, kv, dim, dtype, N, n_seq, max_len, mask)
             for heads, kv in ((256, 1), (256, 256), (1, 1), (64, 8)) for dim, dtype in ((128, 1), (64, 0), (256, 0), (16, 1))
             for N, n_seq, max_len in ((1, 1, 1 << 30), (1 << 21, 1, 1 << 30), (1 << 21, 4096, 1 << 20), (4096, 4096, 5), (5, 4096, 1 << 20))
             for what, mask in (("rows", 0), ("rows", 1), ("q8", 1))]
    calls += [(what, 8, 8, dim, 1, N, 9, 64, 0) for what in ("read", "codes") for dim in (16, 256) for N in (1, 1 << 24, (1 << 31) - 1)]
    for call, (rc, launches) in zip(calls, _launches(calls, tmp_path)):
        assert rc == 0 and launches, call
        for _, x, y, z, threads in launches:
            assert 0 < int(x) * int(threads) < 1 << 32 and 0 < int(y) <= 65535 and 0 < int(z) <= 65535, (call, launches)
        if call[0] in ("read", "codes"):
            assert sum(int(g[1]) for g in launches) == call[5]
