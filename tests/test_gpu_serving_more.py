"""examples/serve_batch.py on the GPU as a program uses it, beside other work."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def close(got, want, tolerance):
    assert bool(torch.isfinite(got).all())
    assert float((got.double() - want.double()).norm()) <= tolerance * float(want.double().norm())


@pytest.mark.parametrize("dtype,tolerance", [("f32", 2e-3), ("bf16", 0.15)])      # of a step of two such blocks: tests/test_gpu_serving.py
def test_replays_beside_tensors_made_after_the_capture(dtype, tolerance):
    # the same weights twice, one server decoding call by call, one by replays; whatever a program allocates in between stays as it is
    from serve_batch import Config, Server
    c = Config(d=256, heads=8, kv_heads=2, head_dim=32, ffn_groups=6, rank=32, blocks=2, dtype=dtype)
    eager, graph = Server(c, 3, 60), Server(c, 3, 60)
    token_in = torch.zeros(3, c.d, dtype=eager.shape.torch_dtype, device="cuda")
    step, replay = eager.decoder(token_in, True), graph.decoder(token_in)
    g = torch.Generator().manual_seed(5)
    mine = []
    for i in range(12):
        token_in.copy_(torch.randn(3, c.d, generator=g))
        for n in (3 * 8, 3 * 6, 3, 3 * 8 * 32, 3 * 256, 3 * 12 * 32, 300000, 1 << 20, 4 << 20):
            for dt in (torch.uint8, eager.shape.torch_dtype, torch.float32):
                mine.append(torch.full((n,), 7 + i, dtype=dt, device="cuda"))
        got, want = replay(), step()
        torch.cuda.synchronize()
        close(got, want, tolerance)
    for j, t in enumerate(mine):
        assert bool((t == 7 + j // 27).all()), (j, t.dtype, t.numel())


@pytest.mark.parametrize("dtype,tolerance", [("f32", 2e-3), ("bf16", 0.15)])
def test_prompts_of_more_tokens_than_a_call_takes(dtype, tolerance):
    # at once, in two parts of the server's own making, against calls of fewer tokens; heads and groups all kept, so that no choice between
    # nearly equal scores tells the two apart
    from serve_batch import Config, Server
    c = Config(d=256, heads=8, kv_heads=2, head_dim=32, ffn_groups=6, rank=32, blocks=2, keep_heads=1.0, keep_groups=1.0, dtype=dtype)
    once, parts = Server(c, 3, 5000), Server(c, 3, 5000)
    counts = [4500, 1, 700]
    g = torch.Generator().manual_seed(6)
    embedded = [torch.randn(n, c.d, generator=g).to(once.shape.torch_dtype).cuda() for n in counts]
    got = once.prompt(torch.cat(embedded), counts)
    first = parts.prompt(torch.cat([embedded[0][:2000], embedded[2]]), [2000, 0, 700])
    second = parts.prompt(torch.cat([embedded[0][2000:], embedded[1]]), [2500, 1, 0])
    torch.cuda.synchronize()
    want = torch.cat([first[:2000], second, first[2000:]])
    assert once.lens.tolist() == parts.lens.tolist() == counts
    for rows in (slice(0, 4096), slice(4096, None), slice(4499, 4501), slice(-1, None)):
        close(got[rows], want[rows], tolerance)
    token_in = torch.randn(3, c.d, generator=g).to(once.shape.torch_dtype).cuda()
    close(once.decoder(token_in)(), parts.decoder(token_in, True)(), tolerance)
    torch.cuda.synchronize()
