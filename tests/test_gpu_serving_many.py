"""More tokens than one launch holds (2^32 threads along x): the rows around a launch's end against a call of those rows alone."""
import pytest
import torch

import paper_2601_11676_amd as H

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_norm_of_more_rows_than_a_launch():
    T, d = (1 << 26) + 5, 8                          # four rows a workgroup of 256 threads: the first launch ends at 2^26 - 4
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    h, y = (torch.empty(T, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    w = torch.randn(d, device=DEV).to(torch.bfloat16)
    out, x = (torch.full((T, d), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    H.halo_block_norm(h, y, x, h_out=out, post_norm=True, w_post=w, w_pre=w)
    torch.cuda.synchronize()
    assert not bool(torch.isnan(x[:, 0]).any()) and not bool(torch.isnan(out[:, 0]).any())
    for rows in (slice(0, 9), slice((1 << 26) - 11, (1 << 26) + 5)):
        o2, x2 = (torch.empty_like(h[rows]) for _ in range(2))
        H.halo_block_norm(h[rows].contiguous(), y[rows].contiguous(), x2, h_out=o2, post_norm=True, w_post=w, w_pre=w)
        torch.cuda.synchronize()
        assert torch.equal(o2, out[rows]) and torch.equal(x2, x[rows])


def test_append_of_more_tokens_than_a_launch():
    N, D = (1 << 24) + 3, 16                         # a workgroup of 256 threads a token: the first launch ends at 2^24 - 1
    shape = H.PagedShape(1, 1, D, 16, 4, 4, "bf16")
    qkv = torch.empty(N, 3, D, dtype=torch.bfloat16, device=DEV).normal_()
    pos, seq = torch.full((N,), -1, dtype=torch.int32, device=DEV), torch.zeros(N, dtype=torch.int32, device=DEV)
    some = torch.tensor([0, 5, (1 << 24) - 2, (1 << 24) - 1, 1 << 24, N - 1], device=DEV)
    pos[some] = torch.arange(10, 10 + 9 * len(some), 9, dtype=torch.int32, device=DEV)
    table = torch.tensor([[2, 0, 3, 1]], dtype=torch.int32, device=DEV)
    rope = torch.from_numpy(H.halo_rope_table(64, D)).to(DEV)
    got = [torch.zeros(shape.pool, dtype=torch.bfloat16, device=DEV) for _ in range(2)] + [torch.full((N, 1, D), float("nan"), dtype=torch.bfloat16, device=DEV)]
    H.halo_paged_append(shape, qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], pos, table, got[0], got[1], q_out=got[2], rope=rope, seq=seq)
    few = qkv[some]
    want = [torch.zeros_like(got[0]), torch.zeros_like(got[1]), torch.empty(len(some), 1, D, dtype=torch.bfloat16, device=DEV)]
    H.halo_paged_append(shape, few[:, :1], few[:, 1:2], few[:, 2:], pos[some], table, want[0], want[1], q_out=want[2], rope=rope, seq=seq[some])
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2][some], want[2])
    rest = torch.ones(N, dtype=torch.bool, device=DEV)
    rest[some] = False
    assert bool((got[2][rest] == 0).all())           # padding
