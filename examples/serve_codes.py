"""The server of serve_batch.py over a cache of eight-bit codes, with the heads of queries and keys normed: half the memory for the same tokens, and a prompt's tokens attend as a
chunk of their sequence, which reads the cache once for many of them.

    python examples/serve_codes.py [--sequences 8] [--prompt 100] [--new 32] [--blocks 4] [--dtype bf16] [--eager]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from serve_batch import Config, Server  # noqa: E402  (also finds the package)
import paper_2601_11676_amd as H  # noqa: E402


class CodesServer(Server):
    def __init__(self, c: Config, sequences: int, longest: int, page_size: int = 16, seed: int = 0):
        super().__init__(c, sequences, longest, page_size, seed)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 1)
        for k in self.blocks:
            k.k_pages, k.v_pages = ((torch.zeros(self.shape.pool, dtype=torch.int8, device="cuda"), torch.zeros(self.shape.pool[:3], device="cuda"))
                                    for _ in range(2))
            k.w_q, k.w_k = ((1.0 + torch.empty(c.head_dim, device="cuda").normal_(0.0, 0.1, generator=g)).to(self.shape.torch_dtype) for _ in range(2))

    def buffers(self, tokens: int):
        b = super().buffers(tokens)
        need = H.halo_paged_chunk_workspace_bytes(self.shape, tokens, len(self.lens))
        if b["ws"].nbytes < need:
            b["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        return b

    def attend(self, b, k, new, pos, seq, rows, lens, max_len: int, mask):
        """rows: the page table (one new token of each sequence), or with seq where each sequence's new tokens begin."""
        q, kn, vn = new
        H.halo_paged_append_q8(self.shape, q, kn, vn, pos, self.table, k.k_pages, k.v_pages, q_out=b["q"], qk_norm=True, w_q=k.w_q, w_k=k.w_k, rope=self.rope,
                               seq=seq)
        if seq is None:
            H.halo_paged_attention_q8(self.shape, b["q"], k.k_pages, k.v_pages, rows, lens, max_len, b["o"], b["ws"], mask=mask)
        else:
            H.halo_paged_chunk_attention_q8(self.shape, b["q"], k.k_pages, k.v_pages, self.table, rows, lens, max_len, b["o"], b["ws"], mask=mask)

    def prompt(self, embedded, counts):
        """New tokens of all sequences at once, counts[i] of sequence i, one after the other in `embedded`: a chunk of each sequence."""
        self.room(counts)
        if len(embedded) != sum(counts):
            raise ValueError(f"{sum(counts)} tokens expected")
        if not len(embedded):
            return torch.empty_like(embedded)
        new = torch.tensor(counts, dtype=torch.int32)
        starts = torch.cat([torch.zeros(1, dtype=torch.int32), new.cumsum(0, dtype=torch.int32)])
        seq = torch.repeat_interleave(torch.arange(len(counts), dtype=torch.int32), new).to(self.lens.device)
        at = torch.cat([torch.arange(n, dtype=torch.int32) for n in counts]).to(self.lens.device)
        pos = (at + self.lens[seq.long()]).to(torch.int32)
        lens = self.lens + new.to(self.lens.device)
        longest = max(have + n for have, n in zip(self.cached, counts))
        x = self.step(self.buffers(len(embedded)), embedded, pos, seq, starts.to(self.lens.device), lens, longest)
        self.lens.copy_(lens)
        self.cached = [have + n for have, n in zip(self.cached, counts)]
        return x


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("sequences", 8), ("prompt", 100), ("new", 32), ("blocks", 4)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    p.add_argument("--eager", action="store_true")
    a = p.parse_args()
    c = Config(blocks=a.blocks, dtype=a.dtype)
    s = CodesServer(c, a.sequences, a.prompt + a.new + 1)
    counts = [max(1, a.prompt * (i + 1) // a.sequences) for i in range(a.sequences)]
    x = s.prompt(torch.randn(sum(counts), c.d, device="cuda").to(s.shape.torch_dtype), counts)
    embedded = x[torch.tensor(counts).cumsum(0).cuda() - 1].clone()      # stands for the next token's embedding
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
