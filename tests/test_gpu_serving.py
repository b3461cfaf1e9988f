"""examples/serve_batch.py: prompts and decoding of a batch through the library's calls, against the same blocks in double."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def np64(t):
    return t.detach().cpu().double().numpy()


class Reference:
    """The example's blocks in double, one sequence after the other; which heads and groups survive is taken from the run."""

    def __init__(self, server):
        self.c, self.rope = server.c, server.rope.cpu().double().numpy()
        self.w = [{n: np64(getattr(b, n)) for n in ("Wqkv", "Wo", "Wg", "Wu", "Wd", "w_attn", "w_ffn", "w_next", "gate")} for b in server.blocks]
        self.k = [[[] for _ in server.blocks] for _ in range(len(server.lens))]
        self.v = [[[] for _ in server.blocks] for _ in range(len(server.lens))]

    def token(self, s, embedded, head_masks, group_masks):
        c = self.c
        norm = lambda z: z / np.sqrt((z * z).mean() + 1e-5)
        h = embedded.copy()
        x = norm(h) * self.w[0]["w_attn"]
        for i, w in enumerate(self.w):
            heads = (w["Wqkv"] @ x).reshape(-1, c.head_dim)
            pos, half = len(self.k[s][i]), c.head_dim // 2
            z = (heads[:, :half] + 1j * heads[:, half:]) * (self.rope[pos, 0] + 1j * self.rope[pos, 1])
            turned = np.concatenate([z.real, z.imag], axis=1)
            self.k[s][i].append(turned[c.heads:c.heads + c.kv_heads])
            self.v[s][i].append(heads[c.heads + c.kv_heads:])
            K, V = np.stack(self.k[s][i]), np.stack(self.v[s][i])
            o = np.zeros((c.heads, c.head_dim))
            for j in range(c.heads):
                if head_masks[i][j]:
                    score = K[:, j * c.kv_heads // c.heads] @ turned[j] / np.sqrt(c.head_dim)
                    e = np.exp(score - score.max())
                    o[j] = e @ V[:, j * c.kv_heads // c.heads] / e.sum()
            h = h + w["gate"] * norm(w["Wo"] @ o.reshape(-1))
            x = norm(h) * w["w_ffn"]
            gate, up = w["Wg"] @ x, w["Wu"] @ x
            act = (gate / (1.0 + np.exp(-gate)) * up).reshape(c.ffn_groups, 128) * group_masks[i][:, None]
            h = 0.9 * h + np.einsum("gjm,gm->j", w["Wd"], act)
            x = norm(h) * (self.w[i + 1]["w_attn"] if i + 1 < len(self.w) else w["w_next"])
        return x


@pytest.mark.parametrize("dtype,tolerance", [("f32", 2e-3), ("bf16", 0.15)])
@pytest.mark.parametrize("eager", [True, False])
def test_prompts_and_decoding(dtype, tolerance, eager):
    # float: some 14 stages a block of sums of up to 768 terms, each off by at most 768 * 2^-24 of its size, two blocks, the norms' and the
    # products' factors below 2: 2 * 14 * 768 * 2^-24 * 2 = 2.6e-3 of a row's largest, 2e-3 in the mean.  bf16: as many roundings
    # to 2^-8 at most, 2 * 14 * 2^-8 = 0.11 if all of one sign, and the probabilities' and activations' own beside them.
    from serve_batch import Config, Server
    c = Config(d=256, heads=8, kv_heads=2, head_dim=32, ffn_groups=6, rank=32, blocks=2, dtype=dtype)
    s = Server(c, 3, 60)
    ref = Reference(s)
    counts = [5, 1, 21]
    g = torch.Generator().manual_seed(3)
    embedded = torch.randn(sum(counts), c.d, generator=g).to(s.shape.torch_dtype)
    seen = {}
    step = s.step

    def spied(b, *args):
        seen["b"] = b
        return step(b, *args)
    s.step = spied

    def masks(t):
        return ([m[t].cpu().numpy() for m in seen["b"]["head_mask"]], [m[t].cpu().numpy() for m in seen["b"]["group_mask"]])

    def close(got, want):
        assert np.linalg.norm(got - want) <= tolerance * np.linalg.norm(want)

    x = s.prompt(embedded.cuda(), counts)
    torch.cuda.synchronize()
    t = 0
    for i, n in enumerate(counts):
        for _ in range(n):
            heads, groups = masks(t)
            assert all(m.sum() == c.keep_heads for m in heads) and all(m.sum() == c.keep_groups for m in groups)
            close(np64(x[t]), ref.token(i, np64(embedded[t]), heads, groups))
            t += 1
    token_in = torch.zeros(3, c.d, dtype=s.shape.torch_dtype, device="cuda")
    token = s.decoder(token_in, eager)
    for _ in range(30):
        token_in.copy_(torch.randn(3, c.d, generator=g))
        x = token()
        torch.cuda.synchronize()
        for i in range(3):
            close(np64(x[i]), ref.token(i, np64(token_in[i]), *masks(i)))
    assert s.lens.tolist() == [35, 31, 51]
    del s.step                                       # or the server refers to itself, and its tensors stay until some later collection
