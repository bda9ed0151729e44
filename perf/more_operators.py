"""The operators of decoding several continuations of one prompt, as cases that can
be timed and checked: keys and values appended to the paged cache with the rotation
of their positions, attention for sequences that share a long prefix, the choice of
the next beams from their logits, and the reordering of the beams' cached tokens.

Each case is a dict of plain values; "op" says which operator it is.

  "append"   `seqs` sequences, the last rows_min to rows of whose own_min to own
             tokens are new: queries of q_heads heads and keys and values of
             kv_heads heads of head_dim, in `type`, for a cache of type `cache`;
             with `tree` the rows are nodes of draft trees, at positions of their own
  "prefix"   `groups` groups of `per` sequences; a group's sequences share their
             first `shared` pages (shared_min in the first group), and each has own_min
             to own tokens behind them, the last rows_min to rows of which are queries
  "beams"    `groups` groups of `beams` beams, logits of `vocab` tokens in `type`
             (rows `pad` elements further apart), `n` candidates a group; `ended` of
             a hundred beams have ended, with `first` only a group's first beam is alive
  "reorder"  `layers` layers of a pool, `groups` groups of `beams` beams of own_min to
             own tokens behind `shared` shared pages; `kept` of a group's beams go on

With `own` false, run() computes them in elementary torch operations in 32 bits (the
angles of the rotation and the beams' scores in 64); with `own` true, through the
framework's calls.

The cache's layout is the framework's: pages [layer][page][K, V][head] of 16
tokens, K as [16][head_dim], V as [4][head_dim][4] (token t at [t / 4][:][t % 4]).
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
PAGE = 16
END = 2
BASE = 10000.0
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def append(name, seqs, rows, length, q_heads, kv_heads, head_dim, kind, cache, rows_min=0, len_min=0, tree=False):
    c = {"op": "append", "seqs": seqs, "rows": rows, "rows_min": rows_min or rows, "own": length,
         "own_min": len_min or length, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "type": kind,
         "cache": cache, "tree": tree}
    return dict(c, name=name) if name else c


def prefix(name, groups, per, shared, length, rows, q_heads, kv_heads, head_dim, cache, shared_min=0, len_min=0,
           rows_min=0):
    c = {"op": "prefix", "groups": groups, "per": per, "shared": shared, "shared_min": shared_min or shared,
         "own": length, "own_min": len_min or length, "rows": rows, "rows_min": rows_min or rows, "q_heads": q_heads,
         "kv_heads": kv_heads, "head_dim": head_dim, "cache": cache}
    return dict(c, name=name) if name else c


def beams(name, groups, n_beams, vocab, kind, n, ended=0, first=False, pad=0):
    c = {"op": "beams", "groups": groups, "beams": n_beams, "vocab": vocab, "type": kind, "n": n, "ended": ended,
         "first": first, "pad": pad}
    return dict(c, name=name) if name else c


def reorder(name, layers, groups, n_beams, kept, shared, length, kv_heads, head_dim, cache, len_min=0):
    c = {"op": "reorder", "layers": layers, "groups": groups, "beams": n_beams, "kept": kept, "shared": shared,
         "own": length, "own_min": len_min or length, "kv_heads": kv_heads, "head_dim": head_dim, "cache": cache}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoded token of one sequence: launches and latency
        append("ak_root", 1, 1, 1025, 32, 32, 128, "f16", "f16"),
        # trees of draft nodes of 61 requests served together, grouped heads, bf16 projections
        append("ak_trees61", 61, 9, 16000, 32, 8, 128, "bf16", "f16", rows_min=1, len_min=500, tree=True),
        # prompts' passes that go on in the middle of a page, fp32 projections of 40 heads
        append("ak_prompts", 2, 2001, 4003, 40, 40, 128, "f32", "f16", rows_min=1500, len_min=1777),
        # four beams of one prompt of 1008 tokens, twelve tokens on
        prefix("pa_beams4", 1, 4, 63, 12, 1, 32, 32, 128, "f16"),
        # the fp32 decoder's heads: seven beams with drafts, odd everything
        prefix("pa_f32", 1, 7, 19, 37, 3, 4, 4, 64, "f32", len_min=5, rows_min=1),
        # two prompts, eight answers each being written: grouped heads, short and long answers, drafts
        prefix("pa_answers16", 2, 8, 500, 700, 5, 32, 8, 128, "f16", shared_min=130, len_min=9, rows_min=1),
        # sixty-four samples of one long document
        prefix("pa_samples64", 1, 64, 2000, 600, 1, 32, 8, 128, "f16", len_min=100),
        # a step of four beams of one prompt: launches and latency
        beams("bs_four", 1, 4, 32000, "f32", 8, ended=0),
        # thirteen prompts of five beams in half precision: an odd vocabulary, rows that are not aligned, ended beams
        beams("bs_prompts13", 13, 5, 50021, "f16", 10, ended=15),
        # a large batch over a large vocabulary
        beams("bs_batch32", 32, 16, 131072, "bf16", 32, ended=5),
        # four beams of the fp32 decoder, nine tokens behind the prompt: one page each
        reorder("rp_page", 4, 1, 4, 2, 3, 9, 4, 64, "f32"),
        # eight prompts of eight beams with up to 500 tokens of their own, a few of the layers
        reorder("rp_batch64", 4, 8, 8, 3, 20, 500, 8, 128, "f16", len_min=250),
    ]


def draw(rng):
    """One more case: the same operators over their whole ranges."""
    def span(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    op = rng.choice(["append", "prefix", "prefix", "beams", "beams", "reorder"])
    if op == "beams":
        vocab, n_beams, kind = span(1000, 200000), rng.randint(1, 16), rng.choice(["f32", "f16", "bf16"])
        groups = span(1, max(1, min(64, (120 << 20) // (vocab * n_beams * SIZE[kind]))))
        return beams("", groups, n_beams, vocab, kind, rng.randint(1, 2 * n_beams),
                     rng.choice([0, 0, rng.randint(1, 60)]), rng.random() < 0.2, rng.choice([0, 0, 1, 24]))
    cache = rng.choice(["f32", "f16", "f16", "f16"])
    kv_heads = rng.choice([4, 8, 32, 40])
    group = rng.choice([1, 1, 2, 4, 8] if kv_heads < 32 else [1])
    hd = rng.choice([64, 128])
    if op == "reorder":
        n_beams, layers = rng.randint(2, 16), rng.randint(1, 5)
        most = (300 << 20) // (2 * kv_heads * PAGE * hd * SIZE[cache] * n_beams * layers)   # pages of a beam, all groups
        groups = span(1, max(1, min(16, most)))
        length = span(1, max(1, min(2000, PAGE * (most // groups))))
        return reorder("", layers, groups, n_beams, rng.randint(1, n_beams - 1), rng.randint(0, 20), length, kv_heads, hd,
                       cache, len_min=rng.randint(1, length))
    if op == "append":
        seqs = span(1, 64)
        length = span(1, min(30000, (60 << 20) // (seqs * kv_heads * hd)))
        rows = span(1, max(1, min(length, 4000 // seqs)))
        len_min = rng.randint(max(1, length // 8), length)
        rows_min, tree = rng.randint(1, min(rows, len_min)), rows <= 64 and rng.random() < 0.3
        return append("", seqs, rows, length, kv_heads * group, kv_heads, hd, rng.choice(["f32", "f16", "bf16"]), cache,
                      rows_min=rows_min, len_min=len_min, tree=tree)
    groups, per = rng.choice([1, 1, 2, 3, 5]), span(1, 64)
    per = max(1, per // groups)
    seqs = groups * per
    shared = span(1, max(1, min(3000, (60 << 20) // (PAGE * kv_heads * max(groups * hd * SIZE[cache], seqs * group)))))
    length = span(1, max(1, min(1500, (30 << 20) // (seqs * kv_heads * hd * SIZE[cache]))))
    most = (60 << 20) // (seqs * kv_heads * group * (PAGE * shared + length))
    rows = span(1, max(1, min(length, 40, most)))
    if cache == "f32":
        rows = min(rows, 4)
    len_min = rng.randint(1, length)
    return prefix("", groups, per, shared, length, rows, kv_heads * group, kv_heads, hd, cache,
                  shared_min=rng.randint(1, shared), len_min=len_min, rows_min=rng.randint(1, min(rows, len_min)))


# --- inputs -----------------------------------------------------------------

def spread(most, least, n):
    """n numbers from most down to least."""
    return [most - (most - least) * i // max(1, n - 1) for i in range(n)]


def ragged(case):
    """New rows and own tokens of each sequence, and the pages that each shares with its group."""
    if case["op"] == "append":
        n, shared = case["seqs"], [0] * case["seqs"]
    else:
        groups = case["groups"]
        per = case["beams"] if case["op"] == "reorder" else case["per"]
        n = groups * per
        shared = [s for s in spread(case["shared"], case.get("shared_min", case["shared"]), groups) for _ in range(per)]
    rows = spread(case.get("rows", 1), case.get("rows_min", 1), n)
    lens = [max(r, o) for r, o in zip(rows, reversed(spread(case["own"], case["own_min"], n)))]
    return rows, lens, shared


def tables(case, g):
    """Page table, where a group's sequences share their first pages, and the pool's pages."""
    rows, lens, shared = ragged(case)
    n = len(lens)
    per = n // case.get("groups", n)
    mine = -(-max(lens) // PAGE)
    if case["op"] == "append":           # only the last pages are written: the table repeats a pool of that many
        few = min(mine, max(rows) // PAGE + 2)
        ids = torch.randperm(n * few, generator=g, device=DEV).to(torch.int32).reshape(n, few)
        return ids[:, torch.arange(mine, device=DEV) % few].contiguous(), n * few
    width = max(shared) + mine
    total = n * mine + (n // per) * max(shared)
    ids = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    own_ids, shared_ids = ids[: n * mine].reshape(n, mine), ids[n * mine:].reshape(n // per, max(shared))
    table = torch.cat([shared_ids.repeat_interleave(per, 0), own_ids], 1)
    if min(shared) < max(shared):        # a group that shares fewer pages has its own ones right behind them
        at = torch.arange(width, device=DEV)[None]
        s = torch.tensor(shared, device=DEV)[:, None]
        table = table.gather(1, torch.where(at < s, at, (max(shared) + at - s).clamp_max(width - 1)))
    return table.contiguous(), total


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = random.Random(seed)
    op = case["op"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    if op == "beams":
        rows, vocab = case["groups"] * case["beams"], case["vocab"]
        x = torch.empty(rows, vocab + case["pad"], dtype=TYPES[case["type"]], device=DEV)
        for i in range(0, rows, 64):      # a head's logits: mostly flat, a few tokens far ahead
            y = normal(min(64, rows - i), vocab + case["pad"])
            x[i:i + 64] = 2 * y + 1.5 * y.clamp_min(2.5)
        scores = -3 * torch.rand(case["groups"], case["beams"], generator=g, device=DEV).cumsum(1) - 5
        if case["first"]:
            scores[:, 0], scores[:, 1:] = 0.0, -math.inf
        ended = ints([[r.randrange(100) < case["ended"] for _ in range(case["beams"])] for _ in range(case["groups"])])
        return {"op": op, "x": x[:, :vocab], "scores": scores, "n": case["n"], "ended": ended if case["ended"] else None}

    rows, lens, shared = ragged(case)
    table, total = tables(case, g)
    t, hd, heads = TYPES[case["cache"]], case["head_dim"], case["kv_heads"]
    pages = normal(case.get("layers", 1), total, 2, heads, PAGE * hd).to(t)
    per = case["beams"] if op == "reorder" else case.get("per", 1)
    s = {"op": op, "pages": pages, "table": table, "lengths": ints([PAGE * b + n for b, n in zip(shared, lens)]),
         "shared": ints(shared[::per]), "max_shared": max(shared), "max_own": max(lens), "per": per}
    if op == "reorder":
        parents = []
        for _ in range(case["groups"]):   # the beams that go on stay where they are, the others become one of them
            kept = r.sample(range(case["beams"]), case["kept"])
            parents.append([i if i in kept else r.choice(kept) for i in range(case["beams"])])
        return dict(s, parents=ints(parents))
    s["offsets"] = ints([0] + list(np.cumsum(rows)))
    s["max_rows"], s["group_offsets"] = max(rows), ints(list(range(0, len(rows) + 1, per)))
    s["max_length"] = max(PAGE * b + n for b, n in zip(shared, lens))
    if op == "prefix":
        s["q"] = (1.5 * normal(sum(rows), case["q_heads"], hd)).to(t)
        return s
    kind = TYPES[case["type"]]            # one projection's output: queries, keys and values of a row side by side
    qkv = normal(sum(rows), case["q_heads"] + 2 * heads, hd).to(kind)
    s["q"], s["k"], s["v"] = qkv.split([case["q_heads"], heads, heads], 1)
    s["positions"] = None
    if case["tree"]:                      # a node stands behind its parent: its position is at most its slot
        s["positions"] = ints([n - k + r.randint(i // 3, i) for k, n in zip(rows, lens) for i in range(k)])
    return s


# --- one pass ---------------------------------------------------------------

def row_maps(s):
    """Sequence and cache slot of each row, on the device."""
    off, lengths = s["offsets"].long(), s["lengths"].long()
    i = torch.arange(s["q"].shape[0], device=DEV)
    seq = (i[:, None] >= off[None, 1:]).sum(1)
    return seq, lengths[seq] - off[seq + 1] + i


def plain_append(s):
    q, k, v, pages, table = s["q"], s["k"], s["v"], s["pages"], s["table"]
    hd, heads = q.shape[2], k.shape[1]
    seq, slot = row_maps(s)
    pos = slot if s["positions"] is None else s["positions"].long()
    j = torch.arange(hd // 2, dtype=torch.float64, device=DEV)
    angle = pos.double()[:, None] * torch.exp(j * (-2.0 / hd * math.log(BASE)))
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def rotated(x):
        a, b = x.float().split(hd // 2, 2)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], 2).to(pages.dtype)

    page = table[seq, slot // PAGE].long()
    at = slot % PAGE
    n = pages.shape[1]
    pages[0, :, 0].view(n, heads, PAGE, hd)[page, :, at] = rotated(k)
    pages[0, :, 1].view(n, heads, 4, hd, 4)[page, :, at // 4, :, at % 4] = v.to(pages.dtype)
    return {"q": rotated(q), "pages": pages}


def plain_prefix(s):
    pages, table, lengths, per = s["pages"], s["table"].long(), s["lengths"].long(), s["per"]
    n, width = table.shape
    heads, hd = pages.shape[3], s["q"].shape[2]
    group = s["q"].shape[1] // heads

    def keys_values(ids):                                               # of [some][pages] ids
        got = pages[0, ids].float()                                     # [some][pages][2][heads][16 hd]
        some, count = ids.shape
        k = got[:, :, 0].reshape(some, count, heads, PAGE, hd).permute(0, 2, 4, 1, 3).reshape(some, heads, hd, -1)
        v = got[:, :, 1].reshape(some, count, heads, 4, hd, 4).permute(0, 2, 1, 3, 5, 4).reshape(some, heads, -1, hd)
        return k, v

    # the queries of each sequence, side by side in rows of the longest
    off = s["offsets"].long()
    rows = off[1:] - off[:-1]
    i = torch.arange(s["max_rows"], device=DEV)
    on = i < rows[:, None]
    at = (off[:-1, None] + i).clamp_max(s["q"].shape[0] - 1)
    q = s["q"].float()[at].reshape(n, -1, heads, group, hd).permute(0, 2, 3, 1, 4).reshape(n, heads, -1, hd)
    together = q.reshape(n // per, per, heads, -1, hd).transpose(1, 2).reshape(n // per, heads, -1, hd)
    shared = s["shared"].long()
    k1, v1 = keys_values(table[::per, : s["max_shared"]])
    p1 = torch.matmul(together, k1) / math.sqrt(hd)
    t = torch.arange(p1.shape[-1], device=DEV)
    p1 = p1.masked_fill_((t >= PAGE * shared[:, None])[:, None, None], -math.inf)
    p1 = p1.reshape(n // per, heads, per, -1, t.numel()).transpose(1, 2).reshape(n, heads, -1, t.numel())
    first = shared.repeat_interleave(per)
    own_pages = torch.arange(-(-s["max_own"] // PAGE), device=DEV)
    k2, v2 = keys_values(table.gather(1, (first[:, None] + own_pages).clamp_max(width - 1)))
    p2 = torch.matmul(q, k2) / math.sqrt(hd)
    t = PAGE * first[:, None] + torch.arange(p2.shape[-1], device=DEV)
    pos = (lengths - rows)[:, None] + i
    see = (t[:, None] <= pos[:, :, None]) | ~on[:, :, None]
    p2 = p2.reshape(n, heads, group, -1, t.shape[1]).masked_fill_(~see[:, None, None], -math.inf).reshape(p2.shape)
    top = torch.maximum(p1.max(-1, keepdim=True).values, p2.max(-1, keepdim=True).values)
    p1, p2 = p1.sub_(top).exp_(), p2.sub_(top).exp_()
    total = p1.sum(-1, keepdim=True) + p2.sum(-1, keepdim=True)
    p1 = p1.reshape(n // per, per, heads, -1, p1.shape[-1]).transpose(1, 2).reshape(n // per, heads, -1, p1.shape[-1])
    o = torch.matmul(p1, v1).reshape(n // per, heads, per, -1, hd).transpose(1, 2).reshape(n, heads, -1, hd)
    o = (o + torch.matmul(p2, v2)) / total
    o = o.reshape(n, heads, group, -1, hd).permute(0, 3, 1, 2, 4).reshape(n, -1, heads * group, hd)
    return o[on].to(s["q"].dtype)


def plain_beams(s):
    groups, count = s["scores"].shape
    vocab = s["x"].shape[1]
    x = s["x"].double().reshape(groups, count, vocab)
    m = x.max(2, keepdim=True).values
    score = s["scores"].double()[..., None]
    value = score + (x - m - (x - m).exp().sum(2, keepdim=True).log())
    if s["ended"] is not None:
        token = torch.arange(vocab, device=DEV)
        kept = torch.where(token == END, score, torch.full_like(score, -math.inf))
        value = torch.where(s["ended"][..., None] != 0, kept, value)
    v, at = value.reshape(groups, -1).sort(dim=1, descending=True, stable=True)
    at = at[:, : s["n"]]
    parent, token = at // vocab, at % vocab
    return {"score": v[:, : s["n"]].float(), "parent": parent.to(torch.int32), "token": token.to(torch.int32)}


def plain_reorder(s):
    table, pages = s["table"].long(), s["pages"]
    n, per = table.shape[0], s["per"]
    first = s["shared"].long().repeat_interleave(per)
    parent = (s["parents"].long() + per * torch.arange(n // per, device=DEV)[:, None]).reshape(-1)
    i = torch.arange(-(-s["max_own"] // PAGE), device=DEV)
    at = (first[:, None] + i).clamp_max(table.shape[1] - 1)
    mine = table.gather(1, at)
    theirs = table[parent].gather(1, at)
    moved = PAGE * at < s["lengths"].long()[parent][:, None]
    pages[:, mine.reshape(-1)] = pages[:, torch.where(moved, theirs, mine).reshape(-1)]
    return pages


def run(state):
    s = state
    if own:
        from paper_2609_26100_amd import ops

        if s["op"] == "append":
            q = ops.append_kv(s["q"], s["k"], s["v"], s["pages"], s["table"], s["offsets"], s["lengths"],
                              positions=s["positions"], rope=BASE, max_rows=s["max_rows"])
            return {"q": q, "pages": s["pages"]}
        if s["op"] == "prefix":
            return ops.prefix_attention(s["q"], s["pages"], s["table"], s["offsets"], s["lengths"], s["shared"],
                                        s["group_offsets"], max_rows=s["max_rows"], max_length=s["max_length"],
                                        max_shared=s["max_shared"], max_group_rows=s["max_rows"] * s["per"])
        if s["op"] == "beams":
            r = ops.beam_select(s["x"], s["scores"], s["n"], ended=s["ended"], end_token=END)
            return {"score": r.score, "parent": r.parent, "token": r.token}
        ops.reorder_pages(s["pages"], s["table"], s["parents"], s["lengths"], s["shared"], max_own=s["max_own"])
        return s["pages"]
    return {"append": plain_append, "prefix": plain_prefix, "beams": plain_beams, "reorder": plain_reorder}[s["op"]](s)


# --- what a pass cannot do without -------------------------------------------

def work(case):
    if case["op"] == "beams":
        n = case["groups"] * case["beams"] * case["vocab"]
        return {"bytes": n * SIZE[case["type"]] + case["groups"] * (8 * case["beams"] + 12 * case["n"]), "flops": 5.0 * n}
    rows, lens, shared = ragged(case)
    es, hd, heads = SIZE[case["cache"]], case["head_dim"], case["kv_heads"]
    if case["op"] == "reorder":
        moved = case["beams"] - case["kept"]          # pages written, and those of the beams that go on read once
        read = min(moved, case["kept"])
        pages = -(-(case["own"] + case["own_min"]) // 2 // PAGE)
        return {"bytes": case["layers"] * case["groups"] * (moved + read) * pages * 2 * heads * PAGE * hd * es,
                "flops": 0.0}
    if case["op"] == "append":
        n = sum(rows) * hd
        return {"bytes": n * (case["q_heads"] + 2 * heads) * (SIZE[case["type"]] + es) + 4 * sum(rows),
                "flops": 3.0 * n * (case["q_heads"] + heads)}
    per = case["per"]
    kv = sum(lens) + PAGE * sum(shared[::per])
    pairs = sum(k * (PAGE * b + n) - k * (k - 1) // 2 for k, n, b in zip(rows, lens, shared))
    return {"bytes": es * hd * (2 * kv * heads + 2 * sum(rows) * case["q_heads"]),
            "flops": 4.0 * hd * pairs * case["q_heads"]}


# --- the same in 64 bits ------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "beams":
        scores, tokens, parents = [], [], []
        for g in range(case["groups"]):
            at = slice(g * case["beams"], (g + 1) * case["beams"])
            value = s["scores"][g].double()[:, None] + torch.log_softmax(s["x"][at].double(), 1)
            for b in range(case["beams"] if s["ended"] is not None else 0):
                if int(s["ended"][g, b]):
                    value[b] = -math.inf
                    value[b, END] = s["scores"][g, b].double()
            value = value.reshape(-1)
            order = torch.argsort(value, descending=True, stable=True)[: case["n"]]
            scores.append(value[order])
            parents.append(torch.div(order, case["vocab"], rounding_mode="floor").to(torch.int32))
            tokens.append((order % case["vocab"]).to(torch.int32))
        return {"score": torch.stack(scores), "parent": torch.stack(parents), "token": torch.stack(tokens)}
    rows, lens, shared = ragged(case)
    hd, heads = case["head_dim"], case["kv_heads"]
    table = s["table"].long().cpu()
    if case["op"] == "reorder":
        out, old = s["pages"].double(), s["pages"].double()
        for i, p in enumerate(s["parents"].reshape(-1).tolist()):
            p += i // case["beams"] * case["beams"]
            pg = range(shared[i], shared[i] + -(-lens[p] // PAGE))
            out[:, table[i, pg]] = old[:, table[p, pg]]
        return out
    if case["op"] == "append":
        seq = [i for i, k in enumerate(rows) for _ in range(k)]
        slot = torch.tensor([n - k + i for k, n in zip(rows, lens) for i in range(k)], device=DEV)
        pos = slot if s["positions"] is None else s["positions"]
        turn = pos.double()[:, None] / BASE ** (torch.arange(0, hd, 2, device=DEV).double() / hd)
        z = torch.polar(torch.ones_like(turn), turn)[:, None]
        page = table[seq, (slot // PAGE).cpu()].to(DEV)
        pages = s["pages"].double()

        def turned(x):
            y = torch.complex(x[..., : hd // 2].double(), x[..., hd // 2:].double()) * z
            return torch.cat([y.real, y.imag], -1)

        k, v, d = turned(s["k"]), s["v"].double(), torch.arange(hd, device=DEV)[None]
        t = (slot % PAGE)[:, None]
        for h in range(heads):
            pages[0, page[:, None], 0, h, t * hd + d] = k[:, h]
            pages[0, page[:, None], 1, h, (t // 4 * hd + d) * 4 + t % 4] = v[:, h]
        return {"q": turned(s["q"]), "pages": pages}
    group = case["q_heads"] // heads
    out = torch.empty(sum(rows), case["q_heads"], hd, dtype=torch.float64, device=DEV)
    r0 = 0
    for i, (n, length) in enumerate(zip(rows, lens)):
        length += PAGE * shared[i]
        ids = table[i, : -(-length // PAGE)].to(DEV)
        hidden = torch.arange(length, device=DEV) > torch.arange(length - n, length, device=DEV)[:, None, None]
        k = s["pages"][0, ids, 0].transpose(0, 1).reshape(heads, -1, hd)[:, :length].double()
        v = s["pages"][0, ids, 1].reshape(-1, heads, 4, hd, 4).permute(1, 0, 2, 4, 3).reshape(heads, -1, hd)[:, :length]
        for h in range(heads):
            q = s["q"][r0:r0 + n, h * group:(h + 1) * group].double()
            a = (q @ k[h].T * hd ** -0.5).masked_fill(hidden, -math.inf)
            out[r0:r0 + n, h * group:(h + 1) * group] = torch.softmax(a, 2) @ v[h].double()
        r0 += n
    return out
