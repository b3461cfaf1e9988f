"""Serving over a paged cache, prompts and an 8-bit cache: the operators as measurable cases.

  append   queries' and keys' heads are normed and rotated, keys and values go to the pages (halo_paged_append_norm)
  store    the same into a cache of 8-bit codes (halo_paged_append_q8), and what the cache then stands for (halo_paged_read_q8)
  attend   one new token of each sequence attends over a cache of 8-bit codes (halo_paged_attention_q8)
  chunk    chunks of new tokens attend over their sequences' pages, each token up to itself: packed prompts, parts of prompts,
           drafted tokens (halo_paged_chunk_attention, halo_paged_chunk_attention_q8)

Where `own` is false, `run` computes the same with elementary torch operations.  Head layouts are those of the 7B, 13B and
70B shapes that this repository's workloads use, and small or odd ones beside them.
"""
import math

import torch

own = False                                          # True: `run` calls the library
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def _append(name, heads, kv, dim, page, seqs, new, past, dtype, rotary=1.0, pairs=False):
    return {"name": name, "kind": "append", "heads": heads, "kv": kv, "dim": dim, "page": page, "seqs": seqs, "new": new,
            "past": past, "dtype": dtype, "rotary": rotary, "pairs": pairs}


def _store(name, heads, kv, dim, page, seqs, new, past, norm, rotary=1.0, pairs=False):
    return {"name": name, "kind": "store", "heads": heads, "kv": kv, "dim": dim, "page": page, "seqs": seqs, "new": new,
            "past": past, "dtype": "bf16", "norm": norm, "rotary": rotary, "pairs": pairs}


def _attend(name, heads, kv, dim, page, seqs, lo, hi, keep):
    return {"name": name, "kind": "attend", "heads": heads, "kv": kv, "dim": dim, "page": page, "seqs": seqs, "lo": lo,
            "hi": hi, "keep": keep, "dtype": "bf16", "q8": True}


def _chunk(name, heads, kv, dim, page, seqs, new, past, keep, dtype, q8=False):
    return {"name": name, "kind": "chunk", "heads": heads, "kv": kv, "dim": dim, "page": page, "seqs": seqs, "new": new,
            "past": past, "keep": keep, "dtype": dtype, "q8": q8}


def listed():
    return [
        # one sequence being generated on the 70B shape, by a model that norms its heads: latency
        _append("append_norm_1", 64, 8, 128, 16, 1, 1, 5000, "bf16"),
        # prompts of a few sequences on the 70B shape, heads normed
        _append("append_norm_prompts", 64, 8, 128, 64, 4, 4099, 3000, "bf16"),
        # a batch of 48 sequences being generated on the 7B shape, into an 8-bit cache
        _store("store_48", 32, 32, 128, 16, 48, 1, 300, False),
        # prompts on the 13B shape into an 8-bit cache, heads normed
        _store("store_prompts", 40, 40, 128, 16, 5, 3001, 50, True),
        # one short sequence on the 7B shape over an 8-bit cache, half of the heads kept: latency
        _attend("attend_q8_short", 32, 32, 128, 16, 1, 301, 301, 0.5),
        # one long sequence on the 70B shape: few heads, so the length is what can be split
        _attend("attend_q8_long", 64, 8, 128, 64, 1, 32771, 32771, 1.0),
        # a batch in full service on the 70B shape: lengths all over, an idle slot among them
        _attend("attend_q8_many", 64, 8, 128, 16, 96, 0, 8192, 1.0),
        # drafted tokens of 8 sequences looked over at once on the 70B shape: few rows over longer caches
        _chunk("chunk_drafts", 64, 8, 128, 16, 8, 40, 1500, 1.0, "bf16"),
        # a part of a long prompt on the 70B shape: its tokens over all that came before
        _chunk("chunk_part", 64, 8, 128, 64, 1, 512, 16000, 1.0, "bf16"),
        # packed prompts of uneven lengths on the 13B shape, three quarters of the heads kept
        _chunk("chunk_prompts", 40, 40, 128, 16, 7, 4099, 0, 0.75, "bf16"),
        # a float32 model of small heads, prompts with something cached
        _chunk("chunk_f32", 12, 4, 64, 32, 3, 777, 200, 1.0, "f32"),
        # the largest: long prompts on the 70B shape, their second halves, over an 8-bit cache
        _chunk("chunk_q8", 64, 8, 128, 16, 2, 8192, 8192, 1.0, "bf16", True),
    ]


def draw(rng):
    def spread(lo, hi):                              # over the logarithm
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))

    kind = rng.choice(["append", "store", "attend", "attend", "chunk", "chunk", "chunk", "chunk"])
    kv = rng.choice([1, 2, 4, 5, 8, 8, 32, 40])
    heads = kv * (rng.choice([1, 1, 2]) if kv >= 32 else rng.choice([1, 2, 3, 4, 7, 8, 16, 20]))
    dim, page = rng.choice([64, 80, 96, 128, 128, 128, 256]), rng.choice([16, 16, 32, 64, 256])
    keep = rng.choice([1.0, 1.0, 0.5, round(rng.uniform(0.1, 0.9), 2)])
    if kind == "attend":
        seqs = spread(1, 192)
        hi = spread(1, max(2, min(60000, 400000000 // (seqs * kv * dim))))
        case = _attend("", heads, kv, dim, page, seqs, hi if rng.random() < 0.3 else rng.randint(0, hi), hi, keep)
    elif kind == "chunk":
        dtype = rng.choice(["bf16", "bf16", "f32", "q8", "q8"])
        seqs = spread(1, 24)
        new = max(seqs, spread(1, 6000))
        past = 0 if rng.random() < 0.3 else spread(1, 20000)
        # at most a quarter of the largest listed case's products, and float32 a quarter of that
        most = (1 << 38) // (8 if dtype == "f32" else 2)
        while new * heads * dim * (past + new // seqs) > most:
            new, past = max(seqs, new // 2), past // 2
            seqs = max(1, seqs // 2) if new == seqs else seqs
        case = _chunk("", heads, kv, dim, page, seqs, new, past, keep, "f32" if dtype == "f32" else "bf16", dtype == "q8")
    else:
        seqs = spread(1, 64)
        new = 1 if rng.random() < 0.4 else spread(2, 8000)
        new = max(seqs if new > 1 else 1, min(new, 20000000 // ((heads + 2 * kv) * dim)))
        past = spread(1, 100000 if seqs * new < 100 else 2000)
        rotary, pairs = rng.choice([1.0, 1.0, 0.5]), rng.random() < 0.3
        if kind == "append":
            case = _append("", heads, kv, dim, page, seqs, new, past, rng.choice(["bf16", "bf16", "f32"]), rotary, pairs)
        else:
            case = _store("", heads, kv, dim, page, seqs, new, past, rng.random() < 0.5, rotary, pairs)
    return {k: v for k, v in case.items() if k != "name"}


# --------------------------------------------------------------------------
# sizes that follow from a case
# --------------------------------------------------------------------------
def _runs(case):
    """(tokens before, new tokens) of each sequence: one new one each in decoding (attend: its length is lo..hi, in scattered order; 0 is an idle
    slot), else `new` cut into uneven parts."""
    n = case["seqs"]
    if case["kind"] == "attend":
        if n == 1:
            return [(case["hi"] - 1, 1)]
        rank = sorted(range(n), key=lambda i: (i * 0.6180339887498949) % 1.0)
        out = [None] * n
        for r, i in enumerate(rank):
            out[i] = (case["lo"] + (case["hi"] - case["lo"]) * r // (n - 1) - 1, 1)
        return out
    new = case["new"]
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


def _codes(g, shape):
    """A pool of 8-bit rows: codes as rows of normal numbers have them, and their scales."""
    codes = torch.empty(shape, dtype=torch.int8, device=DEV)
    for i in range(0, shape[0], 1024):               # in parts: a large pool's numbers in 32 bits would be four times its size
        part = codes[i:i + 1024]
        part.copy_(_normal(g, part.shape, 45.0, torch.float32).round_().clamp_(-127.0, 127.0))
    return codes, torch.empty(shape[:3], device=DEV).uniform_(0.01, 0.03, generator=g)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _append_inputs(case, g):
    dt, D, Hq, Hk, page = DTYPES[case["dtype"]], case["dim"], case["heads"], case["kv"], case["page"]
    runs = _runs(case)
    # the cache is as far as this call reads and writes it: a sequence's page table begins where its new tokens' pages do,
    # positions before them lie in one page that all sequences share
    counts = [(p + n + page - 1) // page - p // page for p, n in runs]
    own_pages, pool = _pages(g, counts)
    width = max((p + n + page - 1) // page for p, n in runs)
    table = torch.full((len(runs), width), pool, dtype=torch.int32, device=DEV)
    for i, (p, n) in enumerate(runs):
        table[i, p // page:p // page + counts[i]] = own_pages[i, :counts[i]]
    cache = (pool + 1, Hk, page, D)
    N = sum(n for _, n in runs)
    s = {"seq": _int32([i for i, (_, n) in enumerate(runs) for _ in range(n)]),
         "pos": _int32([p + j for p, n in runs for j in range(n)]), "table": table, "qkv": _normal(g, (N, (Hq + 2 * Hk) * D), 1.0, dt),
         "w_q": (1.0 + _normal(g, (D,), 0.2, torch.float32)).to(dt), "w_k": (1.0 + _normal(g, (D,), 0.2, torch.float32)).to(dt)}
    rot = _rotary(case)
    angle = torch.arange(width * page, dtype=torch.float64, device=DEV)[:, None] \
        * 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device=DEV) / rot)
    s["rope"] = torch.stack([angle.cos(), angle.sin()], dim=1).float().contiguous()       # [positions][cos, sin][rotary / 2]
    if case["kind"] == "append":
        s["k"], s["v"] = _normal(g, cache, 1.0, dt), _normal(g, cache, 1.0, dt)
    else:
        s["k"], s["v"] = _codes(g, cache), _codes(g, cache)
    return s


def _attend_inputs(case, g):
    dt, D, Hq, Hk, page = DTYPES[case["dtype"]], case["dim"], case["heads"], case["kv"], case["page"]
    runs = _runs(case)
    lens = [p + n for p, n in runs]
    table, pool = _pages(g, [(n + page - 1) // page for n in lens])
    cache = (pool, Hk, page, D)
    starts = [0]
    for _, n in runs:
        starts.append(starts[-1] + n)
    N = starts[-1]
    mask = torch.zeros((N, Hq), dtype=torch.uint8, device=DEV)
    mask.scatter_(1, torch.rand((N, Hq), generator=g, device=DEV).argsort(1)[:, :_kept(case)], 1)
    s = {"q": _normal(g, (N, Hq, D), 2.0, dt), "table": table, "mask": mask if case["keep"] < 1.0 else None, "lens": _int32(lens),
         "longest": max(1, max(lens)), "starts": _int32(starts)}
    if case["q8"]:
        s["k"], s["v"] = _codes(g, cache), _codes(g, cache)
    else:
        s["k"], s["v"] = _normal(g, cache, 1.0, dt), _normal(g, cache, 1.0, dt)
    return s


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (_append_inputs if case["kind"] in ("append", "store") else _attend_inputs)(case, g)


def prepare(case, seed):
    """A program's buffers, and (own) the shape and the workspace that it keeps."""
    s = {"case": case, **_inputs(case, seed)}
    dt, Hq, Hk, D = DTYPES[case["dtype"]], case["heads"], case["kv"], case["dim"]
    N = (s["qkv"] if "qkv" in s else s["q"]).shape[0]
    s["out"] = torch.zeros((N, Hq, D), dtype=dt, device=DEV)
    if case["kind"] == "store":
        s["k_read"], s["v_read"] = (torch.zeros((N, Hk, D), dtype=dt, device=DEV) for _ in range(2))
    if own:
        import paper_2601_11676_amd as H
        pool = (s["k"] if torch.is_tensor(s["k"]) else s["k"][0]).shape[0]
        s["shape"] = H.PagedShape(Hq, Hk, D, case["page"], pool, s["table"].shape[1], case["dtype"])
        need = {"attend": lambda: H.halo_paged_workspace_bytes(s["shape"], N),
                "chunk": lambda: H.halo_paged_chunk_workspace_bytes(s["shape"], N, case["seqs"])}.get(case["kind"])
        if need:
            s["workspace"] = torch.empty(need(), dtype=torch.uint8, device=DEV)
    return s


# --------------------------------------------------------------------------
# the passes
# --------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        return {"append": _own_append, "store": _own_store, "attend": _own_attend, "chunk": _own_chunk}[case["kind"]](case, s)
    return {"append": _plain_append, "store": _plain_store, "attend": _plain_attention, "chunk": _plain_attention}[case["kind"]](case, s)


def _split(case, qkv):
    """Queries, keys and values of a fused projection's rows: views."""
    Hq, Hk, D = case["heads"], case["kv"], case["dim"]
    rows = qkv.view(qkv.shape[0], Hq + 2 * Hk, D)
    return rows[:, :Hq], rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:]


def _own_append(case, s):
    import paper_2601_11676_amd as H
    q, k, v = _split(case, s["qkv"])
    H.halo_paged_append_norm(s["shape"], q, k, v, s["pos"], s["table"], s["k"], s["v"], q_out=s["out"], w_q=s["w_q"], w_k=s["w_k"],
                             eps=EPS, rope=s["rope"], rope_pairs=case["pairs"], seq=s["seq"])
    return {"q": s["out"], "k_pages": s["k"], "v_pages": s["v"]}


def _own_store(case, s):
    import paper_2601_11676_amd as H
    q, k, v = _split(case, s["qkv"])
    H.halo_paged_append_q8(s["shape"], q, k, v, s["pos"], s["table"], s["k"], s["v"], q_out=s["out"], qk_norm=case["norm"],
                           w_q=s["w_q"] if case["norm"] else None, w_k=s["w_k"] if case["norm"] else None, eps=EPS, rope=s["rope"],
                           rope_pairs=case["pairs"], seq=s["seq"])
    H.halo_paged_read_q8(s["shape"], s["pos"], s["table"], s["k"], s["v"], s["k_read"], s["v_read"], seq=s["seq"])
    return {"q": s["out"], "k": s["k_read"], "v": s["v_read"]}


def _own_attend(case, s):
    import paper_2601_11676_amd as H
    H.halo_paged_attention_q8(s["shape"], s["q"], s["k"], s["v"], s["table"], s["lens"], s["longest"], s["out"], s["workspace"],
                              mask=s["mask"])
    return s["out"]


def _own_chunk(case, s):
    import paper_2601_11676_amd as H
    call = H.halo_paged_chunk_attention_q8 if case["q8"] else H.halo_paged_chunk_attention
    call(s["shape"], s["q"], s["k"], s["v"], s["table"], s["starts"], s["lens"], s["longest"], s["out"], s["workspace"], mask=s["mask"])
    return s["out"]


def _unit(x, w):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.to(x.dtype)


def _rotate(x, cos, sin, pairs):
    """x [tokens][heads][dim], the first 2 * cos.shape[1] elements of each head rotated."""
    half = cos.shape[1]
    c, n = cos[:, None], sin[:, None]
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if pairs else (x[..., :half], x[..., half:2 * half])
    first, second = a * c - b * n, b * c + a * n
    turned = torch.stack([first, second], dim=-1).flatten(-2) if pairs else torch.cat([first, second], dim=-1)
    return torch.cat([turned, x[..., 2 * half:]], dim=-1)


def _place(case, s):
    """Page and row of each new token."""
    pos = s["pos"].long()
    return s["table"].long()[s["seq"].long(), pos // case["page"]], pos % case["page"]


def _plain_append(case, s):
    q, k, v = _split(case, s["qkv"])
    cs = s["rope"][s["pos"].long()]
    s["out"].copy_(_rotate(_unit(q.float(), s["w_q"]), cs[:, 0], cs[:, 1], case["pairs"]))
    ids, row = _place(case, s)
    s["k"][ids, :, row] = _rotate(_unit(k.float(), s["w_k"]), cs[:, 0], cs[:, 1], case["pairs"]).to(k.dtype)
    s["v"][ids, :, row] = v
    return {"q": s["out"], "k_pages": s["k"], "v_pages": s["v"]}


def _plain_store(case, s):
    """Keys and values in 64 bits up to their codes: a value may lie next to the border of two."""
    q, k, v = _split(case, s["qkv"])
    cs = s["rope"][s["pos"].long()]
    q, k = q.float(), k.double()
    if case["norm"]:
        q, k = _unit(q, s["w_q"]), _unit(k, s["w_k"])
    s["out"].copy_(_rotate(q, cs[:, 0], cs[:, 1], case["pairs"]))
    ids, row = _place(case, s)
    k = _rotate(k, cs[:, 0].double(), cs[:, 1].double(), case["pairs"])
    for x, (codes, scales), read in ((k, s["k"], s["k_read"]), (v.double(), s["v"], s["v_read"])):
        step = x.abs().amax(-1) / 127.0
        codes[ids, :, row] = (x / step.clamp(min=1e-300)[..., None]).round().to(torch.int8)
        scales[ids, :, row] = step.float()
        read.copy_(codes[ids, :, row].float() * scales[ids, :, row][..., None])
    return {"q": s["out"], "k": s["k_read"], "v": s["v_read"]}


def _plain_attention(case, s):
    """Sequence by sequence: its rows of the cache in 32 bits, some of its new tokens at a time."""
    Hq, Hk, D, page = case["heads"], case["kv"], case["dim"], case["page"]
    at = 0
    for i, (past, new) in enumerate(_runs(case)):
        n = past + new
        if n == 0:
            s["out"][at:at + new] = 0.0
        else:
            ids = s["table"][i, :(n + page - 1) // page].long()
            k, v = ((p[ids].float() if torch.is_tensor(p) else p[0][ids].float() * p[1][ids][..., None]).permute(1, 0, 2, 3)
                    .reshape(Hk, -1, D)[:, :n] for p in (s["k"], s["v"]))
            kt, v = k.transpose(1, 2).contiguous(), v.contiguous()
            some = max(1, (1 << 28) // (Hq * n))
            for t in range(0, new, some):
                q = s["q"][at + t:at + min(new, t + some)].float() * D ** -0.5
                r = q.shape[0]
                q = q.view(r, Hk, Hq // Hk, D).permute(1, 0, 2, 3).reshape(Hk, -1, D)
                score = torch.matmul(q, kt).view(Hk, r, Hq // Hk, n)
                sees = torch.arange(n, device=DEV) <= past + t + torch.arange(r, device=DEV)[:, None]
                score = torch.where(sees[:, None], score, -math.inf)
                e = torch.exp(score - score.amax(-1, keepdim=True))
                o = torch.matmul(e.view(Hk, -1, n), v).view(Hk, r, Hq // Hk, D) / e.sum(-1, keepdim=True)
                o = o.permute(1, 0, 2, 3).reshape(r, Hq, D)
                rows = slice(at + t, at + t + r)
                s["out"][rows] = (o if s["mask"] is None else o * s["mask"][rows, :, None]).to(s["out"].dtype)
        at += new
    return s["out"]


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    Hq, Hk, D = case["heads"], case["kv"], case["dim"]
    runs = _runs(case)
    N = sum(n for _, n in runs)
    if case["kind"] in ("append", "store"):
        rot = _rotary(case)
        by = 4 * rot * len({p + j for p, n in runs for j in range(n)}) + 12 * N
        if case["kind"] == "append":
            return {"bytes": by + 2 * size * N * (Hq + 2 * Hk) * D, "flops": N * (Hq + Hk) * (4 * D + 3 * rot)}
        # in and out, the codes and scales written, and read again, and what they stand for
        by += size * N * (2 * Hq + 2 * Hk) * D + 2 * 2 * N * Hk * (D + 4) + 2 * size * N * Hk * D
        return {"bytes": by, "flops": N * (3 * (Hq + Hk) * rot + 4 * case["norm"] * (Hq + Hk) * D + 6 * Hk * D)}
    share = _kept(case) / Hq
    cached = sum(p + n for p, n in runs)
    seen = sum(n * p + n * (n + 1) // 2 for p, n in runs)
    # a head of the cache is read if one of its queries is kept: with many rows that is every one
    read = 1.0 if share == 1.0 or case["kind"] == "chunk" else 1.0 - (1.0 - share) ** (Hq // Hk)
    row = D + 4 if case["q8"] else size * D
    by = 2 * cached * read * Hk * row + size * N * (1 + share) * Hq * D + N * Hq * (share < 1.0)
    return {"bytes": by + 4 * sum(-(-(p + n) // case["page"]) for p, n in runs), "flops": 4 * seen * share * Hq * D}


# --------------------------------------------------------------------------
# the same in 64 bits
# --------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    return (_exact_append if case["kind"] in ("append", "store") else _exact_attention)(case, s)


def _exact_append(case, s):
    """A rotated pair is a complex number times the unit number of its angle."""
    D, Hq, Hk, page = case["dim"], case["heads"], case["kv"], case["page"]
    x = s["qkv"].double().view(-1, Hq + 2 * Hk, D).clone()
    half = _rotary(case) // 2
    if case.get("norm", True):
        length = torch.sqrt((x[:, :Hq + Hk] ** 2).sum(-1, keepdim=True) / D + EPS)
        x[:, :Hq + Hk] /= length
        x[:, :Hq] *= s["w_q"].double()
        x[:, Hq:Hq + Hk] *= s["w_k"].double()
    i = torch.arange(half, device=DEV)
    re, im = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + half)
    turn = torch.complex(s["rope"][s["pos"].long(), 0].double(), s["rope"][s["pos"].long(), 1].double())[:, None]
    z = torch.complex(x[:, :Hq + Hk][..., re], x[:, :Hq + Hk][..., im]) * turn
    x[:, :Hq + Hk, re], x[:, :Hq + Hk, im] = z.real, z.imag
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    if case["kind"] == "store":
        steps = [torch.linalg.vector_norm(r, math.inf, dim=-1, keepdim=True) / 127 for r in (k, v)]
        k, v = (torch.round(r / torch.where(t > 0, t, 1.0)) * t for r, t in zip((k, v), steps))
        return {"q": q, "k": k, "v": v}
    out = [s["k"].double(), s["v"].double()]
    page_of = torch.gather(s["table"][s["seq"].long()].long(), 1, (s["pos"].long() // page)[:, None])[:, 0]
    row = (page_of * Hk * page + s["pos"].long() % page)[:, None] + page * torch.arange(Hk, device=DEV)
    for pages, r in zip(out, (k, v)):
        pages.view(-1, D)[row.reshape(-1)] = r.reshape(-1, D)
    return {"q": q, "k_pages": out[0], "v_pages": out[1]}


def _exact_attention(case, s):
    """Sequence by sequence, one head of the cache after the other."""
    Hq, Hk, D, page = case["heads"], case["kv"], case["dim"], case["page"]
    group, starts = Hq // Hk, s["starts"].tolist()
    out = torch.zeros((starts[-1], Hq, D), dtype=torch.float64, device=DEV)
    for i, n in enumerate(s["lens"].tolist()):
        first, new = starts[i], starts[i + 1] - starts[i]
        if n == 0 or new == 0:
            continue
        ids = s["table"][i, :(n + page - 1) // page].long()
        for j in range(Hk):
            if case["q8"]:
                k, v = ((c[ids, j].double() * t[ids, j].double()[..., None]).reshape(-1, D)[:n] for c, t in (s["k"], s["v"]))
            else:
                k, v = (p[ids, j].double().reshape(-1, D)[:n] for p in (s["k"], s["v"]))
            kt = k.T.contiguous()
            for t in range(0, new, 1024):
                rows = slice(first + t, first + min(new, t + 1024))
                q = s["q"][rows, j * group:(j + 1) * group].double()
                score = (q.reshape(-1, D) @ kt / math.sqrt(D)).view(q.shape[0], group, n)
                last = n - new + t + torch.arange(q.shape[0], device=DEV)
                score.masked_fill_(torch.arange(n, device=DEV) > last[:, None, None], -math.inf)
                weight = torch.exp(score - torch.logsumexp(score, -1, keepdim=True))
                out[rows, j * group:(j + 1) * group] = (weight.view(-1, n) @ v).view(-1, group, D)
    return out if s["mask"] is None else out * s["mask"][:, :, None].double()
