"""examples/serve_codes.py: prompts as chunks and decoding over a cache of eight-bit codes, against the same blocks in double."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def np64(t):
    return t.detach().cpu().double().numpy()


def kept(rows):
    """What rows of a head stand for as codes."""
    step = np.abs(rows).max(-1, keepdims=True) / 127.0
    return np.rint(rows / np.where(step > 0, step, 1.0)) * step


class Reference:
    """The example's blocks in double, one sequence after the other; which heads and groups survive is taken from the run."""

    def __init__(self, server):
        self.c, self.rope = server.c, server.rope.cpu().double().numpy()
        self.w = [{n: np64(getattr(b, n)) for n in ("Wqkv", "Wo", "Wg", "Wu", "Wd", "w_attn", "w_ffn", "w_next", "gate", "w_q", "w_k")} for b in server.blocks]
        self.k, self.v = ([[[] for _ in server.blocks] for _ in range(len(server.lens))] for _ in range(2))

    def token(self, s, embedded, head_masks, group_masks):
        c = self.c
        norm = lambda z: z / np.sqrt((z * z).mean(-1, keepdims=True) + 1e-5)
        h = embedded.copy()
        x = norm(h) * self.w[0]["w_attn"]
        for i, w in enumerate(self.w):
            heads = (w["Wqkv"] @ x).reshape(-1, c.head_dim)
            pos, half, n = len(self.k[s][i]), c.head_dim // 2, c.heads + c.kv_heads
            normed = norm(heads[:n]) * np.where(np.arange(n)[:, None] < c.heads, w["w_q"], w["w_k"])
            z = (normed[:, :half] + 1j * normed[:, half:]) * (self.rope[pos, 0] + 1j * self.rope[pos, 1])
            turned = np.concatenate([z.real, z.imag], axis=1)
            self.k[s][i].append(kept(turned[c.heads:]))
            self.v[s][i].append(kept(heads[n:]))
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


@pytest.mark.parametrize("dtype,tolerance", [("f32", 1.2e-2), ("bf16", 0.15)])
@pytest.mark.parametrize("eager", [True, False])
def test_prompts_and_decoding(dtype, tolerance, eager):
    # The stages' roundings: 2e-3 in float and 0.11 in bf16 (two blocks, 14 stages each), and codes that fall the other way where a quotient lies next to a border, a step of 1 / 127 of a
    # row's largest: for the token's own row at most in every element, 2 blocks * 1 / 127 / sqrt(3) of what attention gives there = 1e-2 with the probability of 1 that a
    # first token has.
    from serve_codes import Config, CodesServer
    c = Config(d=256, heads=8, kv_heads=2, head_dim=32, ffn_groups=6, rank=32, blocks=2, dtype=dtype)
    s = CodesServer(c, 3, 60)
    ref = Reference(s)
    counts = [5, 0, 21]
    g = torch.Generator().manual_seed(3)
    seen, step = {}, s.step

    def spied(b, *args):
        seen["b"] = b
        return step(b, *args)
    s.step = spied

    def masks(t):
        return ([m[t].cpu().numpy() for m in seen["b"]["head_mask"]], [m[t].cpu().numpy() for m in seen["b"]["group_mask"]])

    def close(got, want):
        assert np.linalg.norm(got - want) <= tolerance * np.linalg.norm(want)

    for part in (counts, [3, 2, 4]):                                  # the second over what the first left
        embedded = torch.randn(sum(part), c.d, generator=g).to(s.shape.torch_dtype)
        x = s.prompt(embedded.cuda(), part)
        torch.cuda.synchronize()
        t = 0
        for i, n in enumerate(part):
            for _ in range(n):
                close(np64(x[t]), ref.token(i, np64(embedded[t]), *masks(t)))
                t += 1
    assert len(s.prompt(embedded[:0].cuda(), [0, 0, 0])) == 0
    token_in = torch.zeros(3, c.d, dtype=s.shape.torch_dtype, device="cuda")
    token = s.decoder(token_in, eager)
    for _ in range(20):
        token_in.copy_(torch.randn(3, c.d, generator=g))
        x = token()
        torch.cuda.synchronize()
        for i in range(3):
            close(np64(x[i]), ref.token(i, np64(token_in[i]), *masks(i)))
    assert s.lens.tolist() == s.cached == [28, 22, 45]
    with pytest.raises(ValueError, match="no room"):
        s.prompt(torch.zeros(40, c.d, dtype=s.shape.torch_dtype, device="cuda"), [0, 40, 0])
    del s.step


def test_the_command_runs(capsys, monkeypatch):
    import serve_codes
    monkeypatch.setattr(sys, "argv", ["serve_codes.py", "--sequences", "3", "--prompt", "40", "--new", "4", "--blocks", "2"])
    serve_codes.main()
    assert "finite: True" in capsys.readouterr().out
