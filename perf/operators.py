"""Serving a batch of sequences: the operators around the projections of an attention block, as measurable cases.

  append   new tokens' queries and keys are rotated by their positions, keys and values go to the pages of their sequences'
           cache (halo_paged_append)
  attend   one new token of each sequence attends over its pages, surviving heads only (halo_paged_attention)
  norm     the norm after a block, its gate and the scaled residual, and the norm before the next block (halo_block_norm)

Where `own` is false, `run` computes the same with elementary torch operations.  Head layouts are those of the 7B, 13B and
70B shapes that this repository's workloads use, and small or odd ones beside them.
"""
import math

import torch

own = False                                          # True: `run` calls the library
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _append(name, heads, kv, dim, page, seqs, new, past, dtype, rotary=1.0, pairs=False):
    return {"name": name, "kind": "append", "heads": heads, "kv": kv, "dim": dim, "page": page, "seqs": seqs, "new": new,
            "past": past, "dtype": dtype, "rotary": rotary, "pairs": pairs}


def _attend(name, heads, kv, dim, page, seqs, lo, hi, keep, dtype):
    return {"name": name, "kind": "attend", "heads": heads, "kv": kv, "dim": dim, "page": page, "seqs": seqs, "lo": lo,
            "hi": hi, "keep": keep, "dtype": dtype}


def _norm(name, d, tokens, dtype, stream, post, gate):
    return {"name": name, "kind": "norm", "d": d, "tokens": tokens, "dtype": dtype, "stream": stream, "post": post,
            "gate": gate}


def listed():
    return [
        # one sequence being generated on the 70B shape: its token goes to the cache
        _append("append_1", 64, 8, 128, 16, 1, 1, 5000, "bf16"),
        # a batch of 48 sequences being generated on the 7B shape
        _append("append_48", 32, 32, 128, 16, 48, 1, 300, "bf16"),
        # prompts of a few sequences, 5003 tokens in all, on the 70B shape; far positions
        _append("append_prompts", 64, 8, 128, 64, 4, 5003, 60000, "bf16"),
        # a float32 model of small heads, a part of each rotated, neighbouring elements as pairs
        _append("append_f32", 12, 4, 64, 32, 7, 333, 50, "f32", 0.5, True),
        # one short sequence on the 7B shape, half of the heads kept: latency
        _attend("attend_short", 32, 32, 128, 16, 1, 301, 301, 0.5, "bf16"),
        # one long sequence on the 70B shape: few heads, so the length is what can be split
        _attend("attend_long", 64, 8, 128, 64, 1, 32771, 32771, 1.0, "bf16"),
        # a batch in full service on the 13B shape: lengths all over, an idle slot among them, three quarters of the heads kept
        _attend("attend_batch", 40, 40, 128, 16, 24, 0, 4000, 0.75, "bf16"),
        # a float32 model of small heads
        _attend("attend_f32", 12, 4, 64, 32, 5, 40, 777, 1.0, "f32"),
        # the largest: many long sequences on the 70B shape
        _attend("attend_many", 64, 8, 128, 16, 96, 500, 8192, 1.0, "bf16"),
        # between two blocks of the 70B shape: one token
        _norm("norm_1", 8192, 1, "bf16", "f32", True, "channel"),
        # a float32 model of an odd width, no norm after the block
        _norm("norm_f32", 1000, 77, "f32", "f32", False, "none"),
        # a prompt between two blocks of the 13B shape, residual stream in bf16, a gate for each token
        _norm("norm_prompt", 5120, 4099, "bf16", "bf16", True, "token"),
    ]


def draw(rng):
    def spread(lo, hi):                              # over the logarithm
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))

    kind = rng.choice(["append", "attend", "attend", "attend", "norm"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "norm":
        d = 8 * spread(8, 2048)
        case = _norm("", d, spread(1, min(8192, (40 << 20) // d)), dtype, rng.choice(["f32", dtype]), rng.random() < 0.6,
                     rng.choice(["none", "channel", "token"]))
    else:
        kv = rng.choice([1, 2, 4, 5, 8, 8, 32, 40])
        heads = kv * (rng.choice([1, 1, 2]) if kv >= 32 else rng.choice([1, 2, 3, 4, 7, 8, 16, 20]))
        dim, page = rng.choice([64, 80, 96, 128, 128, 128, 256]), rng.choice([16, 16, 32, 64, 256])
        if kind == "append":
            seqs = spread(1, 64)
            new = 1 if rng.random() < 0.4 else spread(2, 12000)
            new = max(seqs if new > 1 else 1, min(new, 20000000 // ((heads + 2 * kv) * dim)))
            case = _append("", heads, kv, dim, page, seqs, new, spread(1, 100000 if seqs * new < 100 else 3000), dtype,
                           rng.choice([1.0, 1.0, 0.5]), rng.random() < 0.3)
        else:
            seqs = spread(1, 192)
            top = 100000000 // (seqs * kv * dim) if dtype == "f32" else 200000000 // (seqs * kv * dim)
            hi = spread(1, max(2, min(60000, top)))
            case = _attend("", heads, kv, dim, page, seqs, hi if rng.random() < 0.3 else rng.randint(0, hi), hi,
                           rng.choice([1.0, 1.0, 0.5, 0.25, round(rng.uniform(0.1, 0.9), 2)]), dtype)
    return {k: v for k, v in case.items() if k != "name"}


# --------------------------------------------------------------------------
# sizes that follow from a case
# --------------------------------------------------------------------------
def _lengths(case):
    """Cached tokens of each sequence, its new one among them: spread evenly over lo..hi, in scattered order."""
    n, lo, hi = case["seqs"], case["lo"], case["hi"]
    if n == 1:
        return [hi]
    rank = sorted(range(n), key=lambda i: (i * 0.6180339887498949) % 1.0)
    out = [0] * n
    for r, i in enumerate(rank):
        out[i] = lo + (hi - lo) * r // (n - 1)
    return out


def _new_tokens(case):
    """(first position, new tokens) of each sequence: one each in decoding, else `new` cut into uneven parts."""
    n, new = case["seqs"], case["new"]
    past = [case["past"] * (i + 1) // n for i in range(n)]
    if new == 1:
        return [(p, 1) for p in past]
    cuts = [new * (i * (i + 3)) // (n * (n + 3)) for i in range(n + 1)]
    return [(past[i], cuts[i + 1] - cuts[i]) for i in range(n)]


def _rotary(case):
    return 16 * max(1, int(case["dim"] * case["rotary"]) // 16)


def _kept(case):
    return max(1, min(case["heads"], round(case["keep"] * case["heads"])))


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _normal(g, shape, sigma, dtype):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, sigma, generator=g)


def _pages(g, counts):
    """A page table whose sequences own `counts` pages scattered over the pool (a few of which are free), 0 in the rows' rest."""
    pool = sum(counts) + 3
    ids = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros((len(counts), max(1, max(counts))), dtype=torch.int32, device=DEV)
    at = 0
    for i, c in enumerate(counts):
        table[i, :c] = ids[at:at + c]
        at += c
    return table, pool


def _append_inputs(case, g):
    dt, D, Hq, Hk, page = DTYPES[case["dtype"]], case["dim"], case["heads"], case["kv"], case["page"]
    runs = _new_tokens(case)
    # the cache is as far as this call reads and writes it: a sequence's page table begins where its new tokens' pages do,
    # positions before them lie in one page that all sequences share
    counts = [(p + n + page - 1) // page - p // page for p, n in runs]
    own_pages, pool = _pages(g, counts)
    width = max((p + n + page - 1) // page for p, n in runs)
    table = torch.full((len(runs), width), pool, dtype=torch.int32, device=DEV)
    for i, (p, n) in enumerate(runs):
        table[i, p // page:p // page + counts[i]] = own_pages[i, :counts[i]]
    pool += 1
    N = sum(n for _, n in runs)
    seq = torch.tensor([i for i, (_, n) in enumerate(runs) for _ in range(n)], dtype=torch.int32, device=DEV)
    pos = torch.tensor([p + j for p, n in runs for j in range(n)], dtype=torch.int32, device=DEV)
    qkv = _normal(g, (N, (Hq + 2 * Hk) * D), 1.0, dt)
    rot = _rotary(case)
    angle = torch.arange(width * page, dtype=torch.float64, device=DEV)[:, None] \
        * 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device=DEV) / rot)
    rope = torch.stack([angle.cos(), angle.sin()], dim=1).float().contiguous()       # [positions][cos, sin][rotary / 2]
    cache = (pool, Hk, page, D)
    return {"qkv": qkv, "seq": seq, "pos": pos, "table": table, "rope": rope, "k_pages": _normal(g, cache, 1.0, dt),
            "v_pages": _normal(g, cache, 1.0, dt)}


def _attend_inputs(case, g):
    dt, D, Hq, Hk, page = DTYPES[case["dtype"]], case["dim"], case["heads"], case["kv"], case["page"]
    lens = _lengths(case)
    table, pool = _pages(g, [(n + page - 1) // page for n in lens])
    mask = torch.zeros((len(lens), Hq), dtype=torch.uint8, device=DEV)
    mask.scatter_(1, torch.rand((len(lens), Hq), generator=g, device=DEV).argsort(1)[:, :_kept(case)], 1)
    cache = (pool, Hk, page, D)
    return {"q": _normal(g, (len(lens), Hq, D), 2.0, dt), "table": table, "mask": mask if case["keep"] < 1.0 else None,
            "lens": torch.tensor(lens, dtype=torch.int32, device=DEV), "longest": max(1, max(lens)),
            "k_pages": _normal(g, cache, 1.0, dt), "v_pages": _normal(g, cache, 1.0, dt)}


def _norm_inputs(case, g):
    dt, d, T = DTYPES[case["dtype"]], case["d"], case["tokens"]
    gate = {"none": None, "channel": (d,), "token": (T, d)}[case["gate"]]
    return {"h": _normal(g, (T, d), 3.0, DTYPES[case["stream"]]), "y": _normal(g, (T, d), 0.7, dt),
            "w_post": (1.0 + _normal(g, (d,), 0.2, torch.float32)).to(dt) if case["post"] else None,
            "gate": None if gate is None else _normal(g, gate, 0.5, dt),
            "w_pre": (1.0 + _normal(g, (d,), 0.2, torch.float32)).to(dt)}


RES_SCALE, EPS = 0.875, 1e-5


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return {"append": _append_inputs, "attend": _attend_inputs, "norm": _norm_inputs}[case["kind"]](case, g)


def prepare(case, seed):
    """A program's buffers, and (own) the shape and the workspace that it keeps."""
    s = {"case": case, **_inputs(case, seed)}
    if case["kind"] == "norm":
        s["h_out"], s["x"] = torch.zeros_like(s["h"]), torch.zeros_like(s["y"])
    else:
        n = s["qkv"].shape[0] if case["kind"] == "append" else case["seqs"]
        s["out"] = torch.zeros((n, case["heads"], case["dim"]), dtype=DTYPES[case["dtype"]], device=DEV)
    if own and case["kind"] != "norm":
        import paper_2601_11676_amd as H
        s["shape"] = H.PagedShape(case["heads"], case["kv"], case["dim"], case["page"], s["k_pages"].shape[0],
                                  s["table"].shape[1], case["dtype"])
        if case["kind"] == "attend":
            s["workspace"] = torch.empty(H.halo_paged_workspace_bytes(s["shape"], case["seqs"]), dtype=torch.uint8, device=DEV)
    return s


# --------------------------------------------------------------------------
# the passes
# --------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "norm": _own_norm}[case["kind"]](case, s)
    return {"append": _plain_append, "attend": _plain_attend, "norm": _plain_norm}[case["kind"]](case, s)


def _split(case, qkv):
    """Queries, keys and values of a fused projection's rows: views."""
    Hq, Hk, D = case["heads"], case["kv"], case["dim"]
    rows = qkv.view(qkv.shape[0], Hq + 2 * Hk, D)
    return rows[:, :Hq], rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:]


def _own_append(case, s):
    import paper_2601_11676_amd as H
    q, k, v = _split(case, s["qkv"])
    H.halo_paged_append(s["shape"], q, k, v, s["pos"], s["table"], s["k_pages"], s["v_pages"], q_out=s["out"],
                        rope=s["rope"], rope_pairs=case["pairs"], seq=s["seq"])
    return {"q": s["out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _own_attend(case, s):
    import paper_2601_11676_amd as H
    H.halo_paged_attention(s["shape"], s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["longest"], s["out"],
                           s["workspace"], mask=s["mask"])
    return s["out"]


def _own_norm(case, s):
    import paper_2601_11676_amd as H
    H.halo_block_norm(s["h"], s["y"], s["x"], h_out=s["h_out"], post_norm=case["post"], w_post=s["w_post"], gate=s["gate"],
                      res_scale=RES_SCALE, w_pre=s["w_pre"], eps=EPS)
    return {"h": s["h_out"], "x": s["x"]}


def _rotate(x, cos, sin, pairs):
    """x [tokens][heads][dim], the first 2 * cos.shape[1] elements of each head rotated."""
    half = cos.shape[1]
    c, n = cos[:, None], sin[:, None]
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if pairs else (x[..., :half], x[..., half:2 * half])
    first, second = a * c - b * n, b * c + a * n
    turned = torch.stack([first, second], dim=-1).flatten(-2) if pairs else torch.cat([first, second], dim=-1)
    return torch.cat([turned, x[..., 2 * half:]], dim=-1)


def _plain_append(case, s):
    q, k, v = _split(case, s["qkv"])
    pos, page = s["pos"].long(), case["page"]
    cs = s["rope"][pos]
    s["out"].copy_(_rotate(q.float(), cs[:, 0], cs[:, 1], case["pairs"]))
    ids = s["table"].long()[s["seq"].long(), pos // page]
    s["k_pages"][ids, :, pos % page] = _rotate(k.float(), cs[:, 0], cs[:, 1], case["pairs"]).to(k.dtype)
    s["v_pages"][ids, :, pos % page] = v
    return {"q": s["out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_attend(case, s):
    T, Hq, Hk, D, page = case["seqs"], case["heads"], case["kv"], case["dim"], case["page"]
    n = (s["longest"] + page - 1) // page
    ids = s["table"][:, :n].long()
    there = torch.arange(n * page, device=DEV) < s["lens"][:, None]
    for t in range(0, T, 8):                         # eight sequences at a time: the gathered rows in 32 bits
        at = slice(t, min(T, t + 8))
        k, v = (p[ids[at]].float().permute(0, 2, 1, 3, 4).reshape(-1, Hk, n * page, D) for p in (s["k_pages"], s["v_pages"]))
        q = s["q"][at].float().view(-1, Hk, Hq // Hk, D) * D ** -0.5
        score = torch.matmul(q, k.transpose(2, 3).contiguous())
        score = torch.where(there[at, None, None], score, -math.inf)
        top = score.amax(-1, keepdim=True)
        e = torch.exp(score - torch.where(top > -math.inf, top, 0.0))
        o = torch.matmul(e, v) / e.sum(-1, keepdim=True).clamp(min=1e-30)
        o = o.view(-1, Hq, D)
        s["out"][at] = (o if s["mask"] is None else o * s["mask"][at, :, None]).to(s["out"].dtype)
    return s["out"]


def _plain_norm(case, s):
    def unit(x):
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)

    u = s["y"].float()
    if case["post"]:
        u = unit(u) * s["w_post"].float()
    if s["gate"] is not None:
        u = u * s["gate"].float()
    h = RES_SCALE * s["h"].float() + u
    s["h_out"].copy_(h)
    s["x"].copy_(unit(h) * s["w_pre"].float())
    return {"h": s["h_out"], "x": s["x"]}


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "norm":
        n, stream = case["tokens"] * case["d"], 4 if case["stream"] == "f32" else 2
        by = n * (2 * stream + 2 * size) + size * case["d"] * (1 + case["post"])
        by += size * {"none": 0, "channel": case["d"], "token": n}[case["gate"]]
        return {"bytes": by, "flops": n * (5 + 4 * case["post"] + (case["gate"] != "none"))}
    Hq, Hk, D = case["heads"], case["kv"], case["dim"]
    if case["kind"] == "append":
        runs = _new_tokens(case)
        N, rot = sum(n for _, n in runs), _rotary(case)
        rows = len({p + j for p, n in runs for j in range(n)})
        return {"bytes": 2 * size * N * (Hq + 2 * Hk) * D + 4 * rot * rows + 12 * N, "flops": 3 * N * (Hq + Hk) * rot}
    lens = _lengths(case)
    share = _kept(case) / Hq
    read = 1.0 if share == 1.0 else 1.0 - (1.0 - share) ** (Hq // Hk)     # a head of the cache is read if one of its queries is kept
    by = size * (2 * sum(lens) * read * Hk * D + len(lens) * (1 + share) * Hq * D) + 4 * sum(-(-n // case["page"]) for n in lens)
    return {"bytes": by + len(lens) * Hq, "flops": 4 * sum(lens) * share * Hq * D}


# --------------------------------------------------------------------------
# the same in 64 bits
# --------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "norm": _exact_norm}[case["kind"]](case, s)


def _exact_append(case, s):
    """A rotated pair is a complex number times the unit number of its angle."""
    D, Hq, Hk, page = case["dim"], case["heads"], case["kv"], case["page"]
    x = s["qkv"].double().view(-1, Hq + 2 * Hk, D)
    rot, half = _rotary(case), _rotary(case) // 2
    i = torch.arange(half, device=DEV)
    re, im = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + half)
    assert rot == 2 * half
    turn = torch.complex(s["rope"][s["pos"].long(), 0].double(), s["rope"][s["pos"].long(), 1].double())[:, None]
    z = torch.complex(x[:, :Hq + Hk][..., re], x[:, :Hq + Hk][..., im]) * turn
    y = x.clone()
    y[:, :Hq + Hk, re], y[:, :Hq + Hk, im] = z.real, z.imag
    k, v = s["k_pages"].double(), s["v_pages"].double()
    page_of = torch.gather(s["table"][s["seq"].long()].long(), 1, (s["pos"].long() // page)[:, None])[:, 0]
    row = (page_of * Hk * page + s["pos"].long() % page)[:, None] + page * torch.arange(Hk, device=DEV)
    k.view(-1, D)[row.reshape(-1)] = y[:, Hq:Hq + Hk].reshape(-1, D)
    v.view(-1, D)[row.reshape(-1)] = x[:, Hq + Hk:].reshape(-1, D)
    return {"q": y[:, :Hq], "k_pages": k, "v_pages": v}


def _exact_attend(case, s):
    """Sequence by sequence, one head of the cache after the other."""
    Hq, Hk, D, page = case["heads"], case["kv"], case["dim"], case["page"]
    out = torch.zeros((case["seqs"], Hq, D), dtype=torch.float64, device=DEV)
    for t, n in enumerate(_lengths(case)):
        if n == 0:
            continue
        ids = s["table"][t, :(n + page - 1) // page].long()
        k = s["k_pages"][ids].double().transpose(1, 2).reshape(-1, Hk, D)[:n]
        v = s["v_pages"][ids].double().transpose(1, 2).reshape(-1, Hk, D)[:n]
        for j in range(Hk):
            heads = range(j * (Hq // Hk), (j + 1) * (Hq // Hk))
            score = k[:, j].contiguous() @ s["q"][t, heads.start:heads.stop].double().T.contiguous() / math.sqrt(D)
            weight = torch.exp(score - torch.logsumexp(score, 0))
            out[t, heads.start:heads.stop] = weight.T.contiguous() @ v[:, j].contiguous()
    return out if s["mask"] is None else out * s["mask"][:, :, None].double()


def _exact_norm(case, s):
    u, d = s["y"].double(), case["d"]
    if case["post"]:
        u = u / torch.sqrt((u ** 2).sum(1, keepdim=True) / d + EPS) * s["w_post"].double()
    if s["gate"] is not None:
        u = s["gate"].double() * u
    h = s["h"].double() * RES_SCALE + u
    return {"h": h, "x": h / torch.sqrt((h ** 2).sum(1, keepdim=True) / d + EPS) * s["w_pre"].double()}
