"""A batch of sequences through a small stack of transformer blocks over a paged cache: prompts at once, then token by token.

Every block is  attention (projections, append, head mask, attention over the pages)  and  FFN (predictor, group mask, FFN of the
surviving groups), with halo_block_norm between them.  The projections are plain matrix products; all else is the library's.
Weights are random; what is shown is how the calls go together.

    python examples/serve_batch.py [--sequences 8] [--prompt 100] [--new 32] [--blocks 4] [--dtype bf16] [--eager]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2601_11676_amd as H  # noqa: E402

GROUP = 128                                          # neurons per FFN group
ROWS = 4096                                          # queries that one call of halo_paged_attention takes at most


class Config:
    def __init__(self, d=1024, heads=16, kv_heads=4, head_dim=64, ffn_groups=24, rank=64, blocks=4, keep_heads=0.75,
                 keep_groups=0.5, plr=(0.0, 0.05, 0.1), dtype="bf16"):
        self.d, self.heads, self.kv_heads, self.head_dim = d, heads, kv_heads, head_dim
        self.ffn_groups, self.rank, self.blocks, self.dtype, self.plr = ffn_groups, rank, blocks, dtype, plr
        self.keep_heads, self.keep_groups = round(keep_heads * heads), round(keep_groups * ffn_groups)


class Block:
    """One block's weights and its cache."""

    def __init__(self, c: Config, shape: H.PagedShape, g: torch.Generator):
        def normal(*size, sigma):
            return torch.empty(size, device="cuda", dtype=shape.torch_dtype).normal_(0.0, sigma, generator=g)

        wide, ffn = (c.heads + 2 * c.kv_heads) * c.head_dim, c.ffn_groups * GROUP
        self.Wqkv, self.Wo = normal(wide, c.d, sigma=c.d ** -0.5), normal(c.d, c.heads * c.head_dim, sigma=c.d ** -0.5)
        self.Wg, self.Wu = normal(ffn, c.d, sigma=c.d ** -0.5), normal(ffn, c.d, sigma=c.d ** -0.5)
        self.Wd = H.pack_down_proj(normal(ffn, c.d, sigma=ffn ** -0.5), GROUP)
        # the predictors of the heads and of the FFN's groups
        self.At_heads, self.Bt_heads = normal(c.rank, c.d, sigma=c.d ** -0.5), normal(c.heads, c.rank, sigma=0.1)
        self.At, self.Bt = normal(c.rank, c.d, sigma=c.d ** -0.5), normal(c.ffn_groups, c.rank, sigma=0.1)
        self.w_attn, self.w_ffn, self.w_next = (1.0 + normal(c.d, sigma=0.1) for _ in range(3))
        self.gate = normal(c.d, sigma=0.5)
        self.k_pages, self.v_pages = (torch.zeros(shape.pool, device="cuda", dtype=shape.torch_dtype) for _ in range(2))


class Server:
    """Sequences, their pages and the step that takes some tokens of them through all blocks."""

    def __init__(self, c: Config, sequences: int, longest: int, page_size: int = 16, seed: int = 0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.c, per_seq = c, -(-longest // page_size)
        self.shape = H.PagedShape(c.heads, c.kv_heads, c.head_dim, page_size, sequences * per_seq, per_seq, c.dtype)
        # pages are handed out as sequences grow: here all at once, in scattered order
        self.table = torch.randperm(sequences * per_seq, device="cuda", generator=g).to(torch.int32).view(sequences, per_seq)
        self.lens = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.cached = [0] * sequences                # the same as the host counts it
        self.rope = torch.from_numpy(H.halo_rope_table(longest, c.head_dim)).cuda()
        self.longest = longest
        self.blocks = [Block(c, self.shape, g) for _ in range(c.blocks)]
        self.heads_as_groups = H.Shape(c.d, c.heads * GROUP, GROUP, c.rank, c.dtype)
        self.ffn = H.Shape(c.d, c.ffn_groups * GROUP, GROUP, c.rank, c.dtype)
        self.head_dev, self.group_dev = (torch.from_numpy(H.halo_build_schedule(k, c.plr)).cuda()
                                         for k in (c.keep_heads, c.keep_groups))

    def buffers(self, tokens: int):
        c, dt = self.c, self.shape.torch_dtype

        def empty(*size, dtype=dt):
            return torch.empty(size, dtype=dtype, device="cuda")

        return {"qkv": empty(tokens, (c.heads + 2 * c.kv_heads) * c.head_dim), "q": empty(tokens, c.heads, c.head_dim),
                "o": empty(tokens, c.heads, c.head_dim), "y": empty(tokens, c.d), "x": empty(tokens, c.d),
                "h": empty(tokens, c.d, dtype=torch.float32), "scores": empty(tokens, c.heads, dtype=torch.float32),
                "head_mask": [empty(tokens, c.heads, dtype=torch.uint8) for _ in self.blocks],
                "group_mask": [empty(tokens, c.ffn_groups, dtype=torch.uint8) for _ in self.blocks],
                "ws": empty(max(H.halo_paged_workspace_bytes(self.shape, tokens), H.halo_workspace_bytes(self.ffn, tokens, c.keep_groups),
                                H.halo_workspace_bytes(self.heads_as_groups, tokens, c.keep_heads)), dtype=torch.uint8)}

    def step(self, b, embedded, pos, seq, rows, lens, max_len: int):
        """Tokens at positions pos of sequences seq (None: one of each) through all blocks.  rows [tokens][max_pages]: the page table's row of
        each token's sequence; lens: what each may see, itself included.  The result is b["x"]."""
        c, n_dev = self.c, len(self.c.plr)
        b["h"].zero_()
        H.halo_block_norm(b["h"], embedded, b["x"], w_pre=self.blocks[0].w_attn)
        for i, k in enumerate(self.blocks):
            # attention: heads predicted to matter, keys and values of all of them
            H.halo_predict_scores(self.heads_as_groups, b["x"], k.At_heads, k.Bt_heads, b["scores"], b["ws"])
            H.halo_build_group_mask(b["scores"], c.keep_heads, self.head_dev, n_dev, None, b["head_mask"][i])
            torch.matmul(b["x"], k.Wqkv.t(), out=b["qkv"])
            heads = b["qkv"].view(-1, c.heads + 2 * c.kv_heads, c.head_dim)
            q, kn, vn = heads[:, :c.heads], heads[:, c.heads:c.heads + c.kv_heads], heads[:, c.heads + c.kv_heads:]
            H.halo_paged_append(self.shape, q, kn, vn, pos, self.table, k.k_pages, k.v_pages, q_out=b["q"], rope=self.rope, seq=seq)
            H.halo_paged_attention(self.shape, b["q"], k.k_pages, k.v_pages, rows, lens, max_len, b["o"], b["ws"], mask=b["head_mask"][i])
            torch.matmul(b["o"].view(-1, c.heads * c.head_dim), k.Wo.t(), out=b["y"])
            H.halo_block_norm(b["h"], b["y"], b["x"], post_norm=True, gate=k.gate, w_pre=k.w_ffn)
            # FFN of the surviving groups
            H.halo_ffn_forward(self.ffn, b["x"], k.At, k.Bt, k.Wg, k.Wu, k.Wd, c.keep_groups, self.group_dev, n_dev, None, b["y"],
                               b["ws"], mask=b["group_mask"][i])
            after = self.blocks[i + 1].w_attn if i + 1 < len(self.blocks) else k.w_next
            H.halo_block_norm(b["h"], b["y"], b["x"], res_scale=0.9, w_pre=after)
        return b["x"]

    def room(self, counts):
        """Refuses counts[i] new tokens of sequence i where there is no room for them."""
        if len(counts) != len(self.cached) or min(counts) < 0:
            raise ValueError(f"new tokens of {len(self.cached)} sequences expected")
        for i, (have, new) in enumerate(zip(self.cached, counts)):
            if have + new > self.longest:
                raise ValueError(f"sequence {i} holds {have} tokens: no room for {new} more, {self.longest} is the longest")

    def prompt(self, embedded, counts):
        """New tokens of all sequences at once, counts[i] of sequence i, one after the other in `embedded`: every token attends over what is
        cached up to itself.  Of more than ROWS tokens, a part of them after the other: each finds its sequence's earlier ones in the cache."""
        self.room(counts)
        if len(embedded) != sum(counts):
            raise ValueError(f"{sum(counts)} tokens expected")
        new = torch.tensor(counts, dtype=torch.int32)
        seq = torch.repeat_interleave(torch.arange(len(counts), dtype=torch.int32), new).to(self.lens.device)
        at = torch.cat([torch.arange(n, dtype=torch.int32) for n in counts]).to(self.lens.device)
        pos = (at + self.lens[seq.long()]).to(torch.int32)
        parts = []
        for i in range(0, len(seq), ROWS):
            e, p, s = embedded[i:i + ROWS], pos[i:i + ROWS], seq[i:i + ROWS]
            parts.append(self.step(self.buffers(len(s)), e, p, s, self.table[s.long()].contiguous(), p + 1, self.longest))
        self.lens += new.to(self.lens.device)
        self.cached = [have + n for have, n in zip(self.cached, counts)]
        return parts[0] if len(parts) == 1 else torch.cat(parts) if parts else torch.empty_like(embedded)

    def decoder(self, embedded, eager=False):
        """One token of each sequence, in `embedded`, per call; captured into a graph once.  max_len bounds every replay's lengths."""
        b, lens = self.buffers(len(self.lens)), torch.empty_like(self.lens)

        def one():
            torch.add(self.lens, 1, out=lens)        # with the new token
            x = self.step(b, embedded, self.lens, None, self.table, lens, self.longest)
            self.lens.add_(1)
            return x

        def counted(run):
            def token():
                self.room([1] * len(self.cached))
                x = run()
                self.cached = [have + 1 for have in self.cached]
                return x
            return token

        if eager:
            return counted(one)
        before = self.lens.clone()
        side = torch.cuda.Stream()                   # once outside the capture, as a program warms up
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            one()
        torch.cuda.current_stream().wait_stream(side)
        self.lens.copy_(before)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = one()

        def replay():
            graph.replay()
            return out
        replay.keeps = self, b, lens, embedded       # replays read and write all of it, whoever else still knows it
        return counted(replay)


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("sequences", 8), ("prompt", 100), ("new", 32), ("blocks", 4)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    p.add_argument("--eager", action="store_true")
    a = p.parse_args()
    c = Config(blocks=a.blocks, dtype=a.dtype)
    s = Server(c, a.sequences, a.prompt + a.new + 1)
    counts = [max(1, a.prompt * (i + 1) // a.sequences) for i in range(a.sequences)]
    x = s.prompt(torch.randn(sum(counts), c.d, device="cuda").to(s.shape.torch_dtype), counts)
    last = torch.tensor(counts).cumsum(0).cuda() - 1
    embedded = x[last].clone()                       # stands for the next token's embedding
    token = s.decoder(embedded, a.eager)
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(a.new):
        embedded.copy_(token())
    torch.cuda.synchronize()
    ms = (time.perf_counter() - start) * 1e3 / a.new
    print(f"{a.sequences} sequences, {a.blocks} blocks: {sum(counts)} prompt tokens, then {a.new} steps of {ms:.3f} ms; "
          f"lengths {s.lens.tolist()}; finite: {bool(torch.isfinite(embedded).all())}")


if __name__ == "__main__":
    main()
