"""Calls of the serving operators without tokens, and tensors without elements, without a GPU."""
import ctypes as C

import pytest
import torch

import paper_2601_11676_amd as H

ONE, ST = C.c_void_p(0x1000), C.c_void_p(0)          # never dereferenced


def test_no_tokens_no_pointers():
    # tensors without elements have no address: with no tokens nothing is looked at, as in the library's other calls
    lib, s = H.load_library(), H.PagedShape(8, 2, 64, 16, 10, 4)
    shape, none = C.byref(s.c), None
    assert lib.halo_paged_append(shape, 0, none, 0, none, 0, none, 0, none, none, 2, ONE, none, 0, 0, 0, none, ONE, ONE, ST) == 0
    assert lib.halo_paged_append(shape, 0, none, 0, none, 0, none, 0, none, none, 0, none, ONE, 5, 7, 0, none, ONE, ONE, ST) == 0
    assert lib.halo_paged_attention(shape, 0, none, 0, ONE, ONE, none, none, 0, none, 1.0, none, none, 0, ST) == 0
    assert lib.halo_block_norm(none, none, ONE, none, ONE, none, none, 0, 64, 1, 1, 1, 0, 1.0, 1e-5, ST) == 0
    bad = C.byref(H.PagedShape(8, 3, 64, 16, 10, 4).c)
    assert lib.halo_paged_append(bad, 0, none, 0, none, 0, none, 0, none, none, 2, ONE, none, 0, 0, 0, none, ONE, ONE, ST) == -2
    assert lib.halo_paged_attention(bad, 0, none, 0, ONE, ONE, none, none, 0, none, 1.0, none, none, 0, ST) == -2
    assert lib.halo_block_norm(none, none, ONE, none, ONE, none, none, 0, 60, 1, 1, 1, 0, 1.0, 1e-5, ST) == -4


class OnDevice:
    """A host tensor that says it is on the device; an address is all that the binding takes of it."""

    def __init__(self, *size, dtype=torch.bfloat16):
        self._t = torch.zeros(size, dtype=dtype)
        self.is_cuda = True

    def __getattr__(self, name):
        return getattr(self._t, name)


@pytest.fixture
def binding(monkeypatch):
    monkeypatch.setattr("paper_2601_11676_amd.binding._stream", lambda stream: 0)
    s = H.PagedShape(8, 2, 64, 16, 10, 4)
    return s, OnDevice(*s.pool), OnDevice(*s.pool)


def test_tensors_of_no_tokens(binding):
    s, kp, vp = binding
    q, k, i = OnDevice(0, 8, 64), OnDevice(0, 2, 64), OnDevice(0, dtype=torch.int32)
    table, ws = OnDevice(0, 4, dtype=torch.int32), OnDevice(H.halo_paged_workspace_bytes(s, 0), dtype=torch.uint8)
    rope = OnDevice(5, 2, 32, dtype=torch.float32)
    for t, seq in ((table, None), (OnDevice(3, 4, dtype=torch.int32), i)):
        H.halo_paged_append(s, q, k, k, i, t, kp, vp, q_out=OnDevice(0, 8, 64), rope=rope, seq=seq)
    H.halo_paged_append(s, None, k, k, i, table, kp, vp)
    H.halo_paged_attention(s, q, kp, vp, table, i, 64, OnDevice(0, 8, 64), ws, mask=OnDevice(0, 8, dtype=torch.uint8))
    H.halo_block_norm(OnDevice(0, 64, dtype=torch.float32), OnDevice(0, 64), OnDevice(0, 64), post_norm=True, w_post=OnDevice(64), w_pre=OnDevice(64))
    with pytest.raises(H.HaloError):                 # the shape still is
        H.halo_block_norm(OnDevice(0, 60), OnDevice(0, 60), OnDevice(0, 60))


def test_a_table_of_no_angles_is_refused(binding):
    # its address is 0, which to the library means no rotation
    s, kp, vp = binding
    k, pos, table = OnDevice(1, 2, 64), OnDevice(1, dtype=torch.int32), OnDevice(1, 4, dtype=torch.int32)
    rope = OnDevice(0, 2, 32, dtype=torch.float32)
    rope.data_ptr = lambda: 0                        # as of a device tensor without elements
    for empty in (rope, OnDevice(4, 2, 0, dtype=torch.float32)):
        with pytest.raises(ValueError, match="angles"):
            H.prepared(H.halo_paged_append, s, None, k, k, pos, table, kp, vp, rope=empty)
    H.prepared(H.halo_paged_append, s, None, k, k, pos, table, kp, vp, rope=OnDevice(1, 2, 32, dtype=torch.float32))
