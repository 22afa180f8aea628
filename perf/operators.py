"""Serving operators over a paged key/value cache, and the choice of a token: what they compute, in elementary torch
operations and in 64 bits, and the calls that a program makes of them.

Kinds of case, and what each stands for in use:

  attention  new rows of a batch of sequences (one each when decoding, chunks of prompts, both mixed) against the keys
             and values that the sequences hold in pages
  append     the step before it: queries and keys rotated to their positions, keys and values stored into the pages
  copy       pages copied in every layer: the last page of forked sequences, or pages moved together
  sample     one token per row of logits by temperature, top-k, top-p and min-p, from given uniform numbers

Heads and widths are those of the repository's configurations with the heads of all tracks side by side: tiny 8 x 32,
mid 64 x 64, large 128 x 128 on 16 KV heads, dense 64 x 128 on 8 KV heads.  The cache is [layers, pages, KV heads, page size,
head width]; sequences own shuffled pages of it.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
HEADS = {"tiny": (8, 8, 32), "mid": (64, 64, 64), "large": (128, 16, 128), "dense": (64, 8, 128)}   # query heads, KV heads, width


def listed():
    return [
        # interactive use: one sequence, one new token; latency
        {"name": "attn_decode_1x777", "kind": "attention", "heads": "mid", "dtype": "bf16", "page": 16, "decodes": 1, "shortest": 777, "longest": 777, "chunks": 0, "chunk": 0, "mix": 1},
        # a serving batch of grouped heads, contexts of any length: every key and value read once from memory
        {"name": "attn_decode_64_grouped", "kind": "attention", "heads": "large", "dtype": "bf16", "page": 64, "decodes": 64, "shortest": 128, "longest": 8192, "chunks": 0, "chunk": 0, "mix": 2},
        # continuous batching: decode steps of running sequences beside chunks of new prompts
        {"name": "attn_mixed_36_and_4", "kind": "attention", "heads": "mid", "dtype": "bf16", "page": 16, "decodes": 36, "shortest": 64, "longest": 2048, "chunks": 4, "chunk": 400, "mix": 3},
        # a long prompt's last chunk: 2048 tokens over 16384 positions, bound by the matrix cores
        {"name": "attn_chunk_2048_of_16384", "kind": "attention", "heads": "dense", "dtype": "bf16", "page": 32, "decodes": 0, "shortest": 16384, "longest": 16384, "chunks": 1, "chunk": 2048, "mix": 4},
        # the fp32 configuration: a few short sequences and one small prompt
        {"name": "attn_fp32_tiny", "kind": "attention", "heads": "tiny", "dtype": "fp32", "page": 16, "decodes": 3, "shortest": 5, "longest": 64, "chunks": 1, "chunk": 33, "mix": 5},
        # one decode step's rows
        {"name": "append_decode_64", "kind": "append", "heads": "large", "dtype": "bf16", "page": 64, "sequences": 64, "rows": 1, "past": 2000, "layout": "half", "part": 128, "scaling": "none"},
        # prompts of 1024 tokens behind long contexts: interleaved pairs in half of the head, frequencies scaled by parts
        {"name": "append_prefill_8x1024", "kind": "append", "heads": "dense", "dtype": "bf16", "page": 32, "sequences": 8, "rows": 1024, "past": 100003, "layout": "interleaved", "part": 64, "scaling": "by_parts"},
        # sequences forked in the middle of a page: 8 pages in 32 layers
        {"name": "copy_fork_8", "kind": "copy", "heads": "dense", "dtype": "bf16", "page": 16, "layers": 32, "pages": 512, "pairs": 8},
        # compaction: 480 pages moved in 8 layers
        {"name": "copy_compact_480", "kind": "copy", "heads": "large", "dtype": "bf16", "page": 32, "layers": 8, "pages": 1000, "pairs": 480},
        # one sequence's next token
        {"name": "sample_1x32000", "kind": "sample", "rows": 1, "vocab": 32000, "filters": "all"},
        # a serving batch whose requests ask for different filters
        {"name": "sample_256x32000", "kind": "sample", "rows": 256, "vocab": 32000, "filters": "mixed"},
        # a large vocabulary of odd length, temperature alone: every weight counts
        {"name": "sample_64x130001", "kind": "sample", "rows": 64, "vocab": 130001, "filters": "none"},
    ]


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, odd ones among them."""
    def spread(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(("decode", "decode", "chunk", "mixed", "fp32", "append", "append", "copy", "sample", "sample"))
    page = rng.choice((16, 32, 64, 128))
    if kind == "decode":
        heads = rng.choice(("mid", "large", "dense"))
        batch = spread(1, 96)
        longest = spread(40, min(16384, 131072 // batch))
        return {"kind": "attention", "heads": heads, "dtype": "bf16", "page": page, "decodes": batch, "shortest": rng.randint(1, longest), "longest": longest,
                "chunks": 0, "chunk": 0, "mix": rng.randint(1, 10**6)}
    if kind == "chunk":
        chunk = spread(2, 1500)
        longest = chunk + spread(1, 8192)
        return {"kind": "attention", "heads": rng.choice(("mid", "dense")), "dtype": "bf16", "page": page, "decodes": 0, "shortest": chunk, "longest": longest,
                "chunks": rng.randint(1, 2), "chunk": chunk, "mix": rng.randint(1, 10**6)}
    if kind == "mixed":
        chunk = spread(16, 512)
        return {"kind": "attention", "heads": rng.choice(("mid", "large", "dense")), "dtype": "bf16", "page": page, "decodes": spread(2, 48), "shortest": chunk, "longest": chunk + spread(64, 1500),
                "chunks": rng.randint(1, 4), "chunk": chunk, "mix": rng.randint(1, 10**6)}
    if kind == "fp32":
        chunk = spread(1, 300)
        return {"kind": "attention", "heads": rng.choice(("tiny", "mid")), "dtype": "fp32", "page": page, "decodes": rng.randint(0, 8), "shortest": chunk, "longest": chunk + spread(1, 500),
                "chunks": rng.randint(1, 3), "chunk": chunk, "mix": rng.randint(1, 10**6)}
    if kind == "append":
        heads = rng.choice(("tiny", "mid", "large", "dense"))
        width = HEADS[heads][2]
        sequences = spread(1, 64)
        return {"kind": "append", "heads": heads, "dtype": "fp32" if heads == "tiny" else "bf16", "page": page, "sequences": sequences, "rows": spread(1, 4096 // sequences),
                "past": spread(1, 200000), "layout": rng.choice(("half", "interleaved")), "part": rng.choice((width, width // 2, width // 4)),
                "scaling": rng.choice(("none", "linear", "by_parts"))}
    if kind == "copy":
        pairs = spread(1, 400)
        return {"kind": "copy", "heads": rng.choice(("mid", "large", "dense")), "dtype": "bf16", "page": rng.choice((16, 32)), "layers": spread(1, 8),
                "pages": 2 * pairs + rng.randint(0, 200), "pairs": pairs}
    vocab = spread(700, 130001)
    return {"kind": "sample", "rows": spread(1, min(256, 8000000 // vocab)), "vocab": vocab, "filters": rng.choice(("none", "all", "mixed", "mixed"))}


def normal(gen, dtype, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def lengths(case):
    """(new rows, keys with the new ones) of every sequence: a property of the case.  Decoding sequences first, and among
    them any length from the shortest to the longest; a chunk is the end of what its sequence holds so far."""
    rng = random.Random(case["mix"])
    out = [(1, rng.randint(case["shortest"], case["longest"])) for _ in range(case["decodes"])]
    for _ in range(case["chunks"]):
        out.append((case["chunk"], rng.randint(max(case["shortest"], case["chunk"]), case["longest"])))
    return out


def page_table(gen, keys, page, spare):
    """Shuffled pages of a pool for sequences of `keys` positions each: (table [n, width], pages in the pool)."""
    need = [(k + page - 1) // page for k in keys]
    total = sum(need) + spare
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros((len(need), max(need)), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total


def frequencies(case):
    """Angles per position of the pairs, in 64 bits, and the magnitude of the rotated vectors."""
    part = case["part"]
    freq = 10000.0 ** (-2.0 * np.arange(part // 2, dtype=np.float64) / part)
    if case["scaling"] == "linear":
        return freq / 8.0, 1.0
    if case["scaling"] == "by_parts":
        turns = 4096.0 * freq / (2.0 * np.pi)
        keep = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        return freq * (keep + (1.0 - keep) / 16.0), 0.1 * math.log(16.0) + 1.0
    return freq, 1.0


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = case["kind"]
    state = {"case": case}
    if kind == "sample":
        return prepare_sample(case, gen, state)
    n_heads, n_kv, width = HEADS[case["heads"]]
    dtype = DTYPES[case["dtype"]]
    page = case["page"]
    if kind == "copy":
        shape = (case["layers"], case["pages"], n_kv, page, width)
        order = torch.randperm(case["pages"], generator=gen, device="cuda").cpu().tolist()
        state["pairs"] = np.array([order[:case["pairs"]], order[case["pairs"]:2 * case["pairs"]]], dtype=np.int32).T.copy()   # (from, to)
    else:
        if kind == "attention":
            lens = lengths(case)
        else:
            # every page of the new rows, and a past whose pages are elsewhere: the table's first entries
            lens = [(case["rows"], case["past"] + 7 * b + case["rows"]) for b in range(case["sequences"])]
        rows = [q for q, _ in lens]
        state["lens"] = lens
        state["row_start"] = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32, device="cuda")
        state["kv_len"] = torch.tensor([k for _, k in lens], dtype=torch.int32, device="cuda")
        if kind == "attention":
            table, total = page_table(gen, [k for _, k in lens], page, 5)
        else:
            first = [(k - q) // page for q, k in lens]
            new, total = page_table(gen, [k - f * page for (q, k), f in zip(lens, first)], page, 5)
            table = torch.zeros((len(lens), max(f + new.shape[1] for f in first)), dtype=torch.int32, device="cuda")
            for b, f in enumerate(first):
                table[b, f:f + new.shape[1]] = new[b]
        state["table"] = table
        shape = (1, total, n_kv, page, width)
        # one product's output: a row holds its queries, keys and values side by side
        state["qkv"] = normal(gen, dtype, sum(rows), n_heads + 2 * n_kv, width)
        state["out"] = torch.empty((sum(rows), n_heads, width), dtype=dtype, device="cuda")
    state["k"] = normal(gen, dtype, *shape)
    state["v"] = normal(gen, dtype, *shape)
    if kind == "append":
        state["freq"] = torch.tensor(frequencies(case)[0], device="cuda")
    if own:
        from paper_2602_07306_amd import binding as PB
        state["cache"] = PB.PTPagedCache(state["k"], state["v"])
        if kind != "copy":
            state["batch"] = PB.PTPagedBatch(state["row_start"], state["kv_len"], state["table"], total_rows=sum(rows),
                                             max_q_len=max(rows), max_kv_len=max(k for _, k in lens))
        if kind == "attention":
            state["workspace"] = torch.empty(PB.pt_paged_attention_bytes(state["cache"], state["batch"], n_heads), dtype=torch.uint8, device="cuda")
        if kind == "append":
            layout = PB.PT_ROPE_HALF if case["layout"] == "half" else PB.PT_ROPE_INTERLEAVED
            how = {"none": dict(), "linear": dict(scaling=PB.PT_ROPE_LINEAR, factor=8.0),
                   "by_parts": dict(scaling=PB.PT_ROPE_BY_PARTS, factor=16.0, low=1.0, high=32.0, original_len=4096, magnitude=frequencies(case)[1])}
            state["rope"] = PB.PTRope(layout, case["part"], 10000.0, **how[case["scaling"]])
    return state


def prepare_sample(case, gen, state):
    """Logits as of a language model: a broad normal, and a few tokens that stand out of it."""
    rows, vocab = case["rows"], case["vocab"]
    logits = 2.2 * torch.randn((rows, vocab), generator=gen, device="cuda", dtype=torch.float32)
    best = torch.randint(0, vocab, (rows, 24), generator=gen, device="cuda")
    logits.scatter_(1, best, 5.0 + 6.0 * torch.rand((rows, 24), generator=gen, device="cuda"))
    state["logits"] = logits
    state["uniform"] = torch.rand((rows,), generator=gen, device="cuda", dtype=torch.float32)

    def choice(values, dtype):
        pick = torch.randint(0, len(values), (rows,), generator=gen, device="cuda")
        return torch.tensor(values, dtype=dtype, device="cuda")[pick]

    state["temperature"] = 0.6 + 0.7 * torch.rand((rows,), generator=gen, device="cuda")
    some = {"all": ([40], [0.95], [0.02]), "mixed": ([0, 0, 1, 20, 50, 400], [1.0, 1.0, 0.8, 0.9, 0.95, 0.99], [0.0, 0.0, 0.02, 0.1])}.get(case["filters"])
    state["top_k"] = choice(some[0], torch.int32) if some else None
    state["top_p"] = choice(some[1], torch.float32) if some else None
    state["min_p"] = choice(some[2], torch.float32) if some else None
    state["out"] = torch.empty((rows,), dtype=torch.int32, device="cuda")
    if own:
        from paper_2602_07306_amd import binding as PB
        state["workspace"] = torch.empty(PB.pt_sample_bytes(rows, vocab), dtype=torch.uint8, device="cuda")
    return state


def run(state):
    case = state["case"]
    kind = case["kind"]
    if kind == "sample":
        return run_own_sample(state) if own else plain_sample(state)
    if kind == "copy":
        if own:
            from paper_2602_07306_amd import binding as PB
            PB.pt_page_copy(state["cache"], state["pairs"])
        else:
            src, dst = torch.tensor(state["pairs"].T.astype(np.int64), device="cuda")
            state["k"][:, dst] = state["k"][:, src]
            state["v"][:, dst] = state["v"][:, src]
        return [state["k"], state["v"]]
    n_heads, n_kv, _ = HEADS[case["heads"]]
    q, k, v = state["qkv"].split((n_heads, n_kv, n_kv), dim=1)
    if kind == "attention":
        if own:
            from paper_2602_07306_amd import binding as PB
            return PB.pt_paged_attention(state["cache"], 0, state["batch"], q, out=state["out"], workspace=state["workspace"])
        return plain_attention(state, q)
    if own:
        from paper_2602_07306_amd import binding as PB
        PB.pt_paged_append(state["cache"], 0, state["batch"], k, v, q=q, q_out=state["out"], rope=state["rope"])
        return [state["out"], state["k"], state["v"]]
    return plain_append(state, q, k, v)


def run_own_sample(state):
    from paper_2602_07306_amd import binding as PB
    return PB.pt_sample(state["logits"], state["uniform"], temperature=state["temperature"], top_k=state["top_k"], top_p=state["top_p"],
                        min_p=state["min_p"], out=state["out"], workspace=state["workspace"])


# -- the operators in elementary torch operations ------------------------------------------------------------------

def held(pages, table, keys):
    """The first `keys` positions of a sequence, [KV heads, keys, width] in 32 bits."""
    size = pages.shape[2]
    rows = pages[table[:(keys + size - 1) // size].long()]                     # [n, KV heads, size, width]
    return rows.permute(1, 0, 2, 3).reshape(pages.shape[1], -1, pages.shape[3])[:, :keys].float().contiguous()


def plain_attention(state, q):
    case = state["case"]
    n_heads, n_kv, width = HEADS[case["heads"]]
    group = n_heads // n_kv
    at = 0
    for b, (n, keys) in enumerate(state["lens"]):
        k = held(state["k"][0], state["table"][b], keys).transpose(1, 2).contiguous()
        v = held(state["v"][0], state["table"][b], keys)
        step = max(1, (1 << 28) // (n_heads * keys))     # rows at once: a gigabyte of scores
        for lo in range(0, n, step):
            hi = min(n, lo + step)
            x = q[at + lo:at + hi].float().reshape(hi - lo, n_kv, group, width).permute(1, 2, 0, 3).reshape(n_kv, group * (hi - lo), width)
            s = torch.bmm(x, k) / math.sqrt(width)
            position = keys - n + torch.arange(lo, hi, device="cuda")
            ahead = torch.arange(keys, device="cuda")[None, :] > position[:, None]
            s = s.view(n_kv, group, hi - lo, keys).masked_fill_(ahead, float("-inf")).view(n_kv, -1, keys)
            s = torch.exp(s - s.amax(-1, keepdim=True))
            o = torch.bmm(s, v) / s.sum(-1, keepdim=True)
            state["out"][at + lo:at + hi] = o.view(n_kv, group, hi - lo, width).permute(2, 0, 1, 3).reshape(hi - lo, n_heads, width).to(q.dtype)
        at += n
    return state["out"]


def plain_rotated(x, cos, sin, layout, part):
    y = x.float()
    if layout == "half":
        a, b = y[..., :part // 2], y[..., part // 2:part]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    else:
        a, b = y[..., 0:part:2], y[..., 1:part:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    return torch.cat((turned, y[..., part:]), dim=-1).to(x.dtype)


def plain_append(state, q, k, v):
    case = state["case"]
    new = torch.diff(state["row_start"]).long()
    owner = torch.repeat_interleave(torch.arange(new.numel(), device="cuda"), new, output_size=q.shape[0])
    position = (state["kv_len"].long() - new)[owner] + torch.arange(q.shape[0], device="cuda") - state["row_start"].long()[owner]
    angle = position[:, None].double() * state["freq"]                            # far positions: in 64 bits
    magnitude = frequencies(case)[1]
    cos, sin = (magnitude * torch.cos(angle)).float()[:, None], (magnitude * torch.sin(angle)).float()[:, None]
    state["out"].copy_(plain_rotated(q, cos, sin, case["layout"], case["part"]))
    page = state["table"].long()[owner, position // case["page"]]
    slot = position % case["page"]
    state["k"][0, page, :, slot] = plain_rotated(k, cos, sin, case["layout"], case["part"])
    state["v"][0, page, :, slot] = v
    return [state["out"], state["k"], state["v"]]


def plain_sample(state):
    logits = state["logits"].double()
    rows, vocab = logits.shape
    best = logits.amax(-1, keepdim=True)
    w = torch.exp((logits - best) / state["temperature"].double()[:, None])
    if state["top_k"] is not None:
        order = torch.sort(logits, dim=-1, descending=True, stable=True).indices
        ws = w.gather(1, order)
        k = state["top_k"].long()
        k = torch.where(k > 0, k, vocab)
        ws = ws * (torch.arange(vocab, device="cuda")[None, :] < k[:, None])
        before = torch.cumsum(ws, -1) - ws
        p = state["top_p"].double()[:, None]
        ws = ws * ((before < p * ws.sum(-1, keepdim=True)) | (p >= 1.0))
        ws = ws * (ws >= state["min_p"].double()[:, None])
        w = torch.zeros_like(w).scatter_(1, order, ws)
    c = torch.cumsum(w, -1)
    over = (c > state["uniform"].double()[:, None] * c[:, -1:]) & (w > 0)
    state["out"].copy_(over.to(torch.int8).argmax(-1))
    return state["out"]


# -- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": 4.0 * n + case["rows"] * (24.0 if case["filters"] != "none" else 12.0), "flops": 2.0 * n}
    n_heads, n_kv, width = HEADS[case["heads"]]
    size = 2 if case["dtype"] == "bf16" else 4
    if kind == "copy":
        n = float(case["pairs"] * case["layers"] * n_kv * case["page"] * width)
        return {"bytes": 4.0 * n * size, "flops": 0.0}
    if kind == "append":
        rows = float(case["sequences"] * case["rows"])
        return {"bytes": 2.0 * rows * (n_heads + 2 * n_kv) * width * size, "flops": 3.0 * rows * (n_heads + n_kv) * case["part"]}
    lens = lengths(case)
    seen = sum(n * (keys - n) + n * (n + 1) // 2 for n, keys in lens)
    return {"bytes": float(size * width * (2 * n_heads * sum(n for n, _ in lens) + 2 * n_kv * sum(keys for _, keys in lens))),
            "flops": 4.0 * n_heads * width * seen}


# -- the definitions in 64 bits ------------------------------------------------------------------------------------------

def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "sample":
        return exact_sample(state)
    if kind == "copy":
        outs = []
        for name in ("k", "v"):
            pages = list(range(case["pages"]))
            for src, dst in state["pairs"]:
                pages[dst] = src
            outs.append(state[name][:, torch.tensor(pages, device="cuda")])
        return outs
    n_heads, n_kv, width = HEADS[case["heads"]]
    x = state["qkv"].double()
    if kind == "attention":
        out = torch.zeros((x.shape[0], n_heads, width), dtype=torch.float64, device="cuda")
        at = 0
        for b, (n, keys) in enumerate(state["lens"]):
            where = torch.arange(keys, device="cuda")
            page = state["table"][b].long()[where // case["page"]]
            seen = where[None, :] <= (torch.arange(n, device="cuda") + keys - n)[:, None]
            for h in range(n_kv):
                k = state["k"][0, page, h, where % case["page"]].double().t().contiguous()
                v = state["v"][0, page, h, where % case["page"]].double()
                for c in range(h * (n_heads // n_kv), (h + 1) * (n_heads // n_kv)):
                    s = (x[at:at + n, c] @ k) * width ** -0.5
                    p = torch.softmax(torch.where(seen, s, -math.inf), dim=-1)
                    out[at:at + n, c] = p @ v
            at += n
        return out
    # a pair of elements as a complex number, turned by its angle
    freq, magnitude = frequencies(case)
    part = case["part"]
    k_cache, v_cache = state["k"].double(), state["v"].double()
    first = torch.arange(part // 2, device="cuda") if case["layout"] == "half" else 2 * torch.arange(part // 2, device="cuda")
    second = first + (part // 2 if case["layout"] == "half" else 1)
    at = 0
    for b, (n, keys) in enumerate(state["lens"]):
        where = torch.arange(keys - n, keys, device="cuda")
        angle = where.double()[:, None] * torch.tensor(freq, device="cuda")[None, :]
        turn = torch.polar(torch.full_like(angle, magnitude), angle)[:, None, :]
        rows = x[at:at + n]
        z = torch.complex(rows[:, :n_heads + n_kv, first], rows[:, :n_heads + n_kv, second]) * turn
        rows[:, :n_heads + n_kv, first] = z.real
        rows[:, :n_heads + n_kv, second] = z.imag
        page = state["table"][b].long()[where // case["page"]]
        k_cache[0, page, :, where % case["page"]] = rows[:, n_heads:n_heads + n_kv]
        v_cache[0, page, :, where % case["page"]] = rows[:, n_heads + n_kv:]
        at += n
    return [x[:, :n_heads].contiguous(), k_cache, v_cache]


def exact_sample(state):
    """Row by row on the host: the tokens sorted, cut by each filter in turn, and the rest walked in index order."""
    logits = state["logits"].cpu().numpy().astype(np.float64)
    get = lambda name, off: state[name].cpu().numpy().astype(np.float64) if state[name] is not None else np.full(len(logits), off)
    temperature, top_k, top_p, min_p = get("temperature", 1.0), get("top_k", 0), get("top_p", 1.0), get("min_p", 0.0)
    uniform = get("uniform", 0.0)
    out = np.empty(len(logits), dtype=np.int32)
    for r, row in enumerate(logits):
        weight = np.exp((row - row.max()) / temperature[r])
        if top_k[r] > 0 or top_p[r] < 1.0 or min_p[r] > 0.0:
            order = np.argsort(-row, kind="stable")
            if top_k[r] > 0:
                order = order[:int(top_k[r])]
            if top_p[r] < 1.0:
                mass = np.cumsum(weight[order])
                order = order[:1 + int(np.count_nonzero(mass[:-1] < top_p[r] * mass[-1]))]
            order = np.sort(order[weight[order] >= min_p[r]])
        else:
            order = np.arange(len(row))
        mass = np.cumsum(weight[order])
        out[r] = order[min(int(np.searchsorted(mass, uniform[r] * mass[-1], side="right")), len(order) - 1)]
    return torch.from_numpy(out)
