"""The operators next to the verification step, as cases that can be timed and
checked: log probabilities of given tokens, attention with a sliding window and
sinks over the paged KV cache, and copies of cache pages.

Each case is a dict of plain values; "op" says which operator it is.

  "logprobs"  rows x vocab logits of `type` (rows `pad` elements further apart
              than vocab), `tokens` given tokens a row, `top` alternatives
  "window"    attention of one layer: `seqs` sequences of len_min to len cached
              tokens, the last rows_min to rows of each being the queries;
              q_heads query heads over kv_heads heads of head_dim in the cache,
              `sinks` first tokens and the last `window` (0: all) are seen
  "copy"      `layers` layers of a pool of pages of kv_heads heads: `sources`
              pages, each copied to `fan` others

With `own` false, run() computes them in elementary torch operations in 32 bits;
with `own` true, through the framework's calls.

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
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def logprobs(name, rows, vocab, kind, tokens, top, pad=0):
    c = {"op": "logprobs", "rows": rows, "vocab": vocab, "type": kind, "tokens": tokens, "top": top, "pad": pad}
    return dict(c, name=name) if name else c


def window(name, seqs, rows, length, q_heads, kv_heads, head_dim, kind, sinks, win, len_min=0, rows_min=0):
    c = {"op": "window", "seqs": seqs, "rows": rows, "rows_min": rows_min or rows, "len": length,
         "len_min": len_min or length, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "type": kind,
         "sinks": sinks, "window": win}
    return dict(c, name=name) if name else c


def copy(name, layers, sources, fan, kv_heads, head_dim, kind):
    c = {"op": "copy", "layers": layers, "sources": sources, "fan": fan, "kv_heads": kv_heads, "head_dim": head_dim,
         "type": kind}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoded token's log probability and its five alternatives: launches and latency
        logprobs("lp_root", 1, 32000, "f32", 1, 5),
        # every node of a draft tree, twenty alternatives each
        logprobs("lp_tree61", 61, 32000, "f32", 1, 20),
        # answers of four choices scored in half precision: an odd vocabulary, rows that are not aligned
        logprobs("lp_choices777", 777, 50021, "f16", 4, 8),
        # a long text scored token by token over a large vocabulary
        logprobs("lp_text2048", 2048, 131072, "bf16", 1, 3),
        # one decoded token of a long context under a window
        window("wa_root", 1, 1, 4000, 32, 32, 128, "f16", 4, 1024),
        # the fp32 decoder's heads, odd everything
        window("wa_f32", 2, 33, 301, 4, 4, 64, "f32", 1, 100, len_min=77, rows_min=5),
        # eight requests served together: grouped heads, short and long contexts, drafts of one to nine nodes
        window("wa_batch8", 8, 9, 16000, 32, 8, 128, "f16", 16, 2048, len_min=500, rows_min=1),
        # a draft chain behind a very long context, all of it seen
        window("wa_long", 1, 5, 100003, 32, 8, 128, "f16", 0, 0),
        # a prompt's pass behind as many tokens, under a window
        window("wa_prompt2048", 1, 2048, 4096, 32, 32, 128, "f16", 4, 1024),
        # the page that two sequences share when one of them goes on, in the fp32 decoder
        copy("cp_one", 4, 1, 1, 4, 64, "f32"),
        # 700 pages moved one by one
        copy("cp_moves700", 2, 700, 1, 40, 128, "f16"),
        # a prompt of 1040 tokens forked to seven other sequences
        copy("cp_fork7", 4, 65, 7, 32, 128, "f16"),
    ]


def draw(rng):
    """One more case: the same operators over their whole ranges."""
    def span(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["logprobs", "logprobs", "window", "window", "window", "copy"])
    if op == "logprobs":
        vocab = span(1000, 200000)
        rows = span(1, max(1, min(2048, (200 << 20) // vocab)))
        top = rng.choice([0, 1, rng.randint(2, 32)])
        return logprobs("", rows, vocab, rng.choice(["f32", "f16", "bf16"]), rng.randint(0 if top else 1, 8), top,
                        rng.choice([0, 0, 1, 24]))
    if op == "copy":
        kind = rng.choice(["f32", "f16", "f16"])
        heads, hd = rng.choice([(4, 64), (8, 128), (32, 128), (40, 128), (52, 128)])
        size = 2 * heads * PAGE * hd * (4 if kind == "f32" else 2)
        fan, layers = rng.choice([1, 1, rng.randint(2, 7)]), rng.randint(1, 6)
        most = max(1, min(700, (400 << 20) // (size * fan * layers)))
        return copy("", layers, span(1, most), fan, heads, hd, kind)
    kind = rng.choice(["f32", "f16", "f16", "f16"])
    kv_heads = rng.choice([4, 8, 32, 40])
    group = rng.choice([1, 1, 2, 4, 8] if kv_heads < 32 else [1])
    hd = rng.choice([64, 128])
    seqs = rng.randint(1, 8)
    length = span(1, min(100000, (100 << 20) // (seqs * kv_heads * hd)))
    rows = span(1, min(length, 2048, max(1, (250 << 20) // (seqs * kv_heads * group * length))))
    if kind == "f32":
        rows = min(rows, 64)
    sinks = rng.choice([0, 1, 4, rng.randint(5, 70)])
    win = rng.choice([0, span(1, 4096), span(64, 4096)])
    len_min = rng.randint(max(1, length // 8), length)
    return window("", seqs, rows, length, kv_heads * group, kv_heads, hd, kind, sinks, win, len_min=len_min,
                  rows_min=rng.randint(1, min(rows, len_min)))


# --- inputs -----------------------------------------------------------------

def ragged(case):
    """Rows and cached tokens of each sequence, spread evenly between the least and the most."""
    n = case["seqs"]
    rows, lens = [], []
    for i in range(n):
        rows.append(case["rows"] - (case["rows"] - case["rows_min"]) * i // max(1, n - 1))
        lens.append(max(rows[-1], case["len_min"] + (case["len"] - case["len_min"]) * (i + 1) // n))
    return rows, lens


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = random.Random(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    t = TYPES[case["type"]]
    if case["op"] == "logprobs":
        rows, vocab = case["rows"], case["vocab"]
        x = torch.empty(rows, vocab + case["pad"], dtype=t, device=DEV)
        for i in range(0, rows, 256):     # a head's logits: mostly flat, a few tokens far ahead
            y = normal(min(256, rows - i), vocab + case["pad"])
            x[i:i + 256] = 2 * y + 1.5 * y.clamp_min(2.5)
        tok = torch.randint(0, vocab, (rows, case["tokens"]), generator=g, device=DEV, dtype=torch.int32)
        if case["tokens"]:                # the first given token is a likely one, as in a decoded text
            tok[:, 0] = x[:, :vocab][:, : min(vocab, 4096)].max(1).indices
        return {"op": "logprobs", "x": x[:, :vocab], "tokens": tok, "top": case["top"]}
    hd, heads = case["head_dim"], case["kv_heads"]
    if case["op"] == "copy":
        n = case["sources"]
        total = n * (1 + case["fan"])
        pages = normal(case["layers"], total, 2, heads, PAGE * hd).to(t)
        order = list(range(total))
        r.shuffle(order)
        src = [p for p in order[:n] for _ in range(case["fan"])]
        return {"op": "copy", "pages": pages, "src": src, "dst": order[n:]}
    rows, lens = ragged(case)
    per_seq = -(-max(lens) // PAGE)
    total = case["seqs"] * per_seq
    pages = normal(1, total, 2, heads, PAGE * hd).to(t)
    table = torch.randperm(total, generator=g, device=DEV).to(torch.int32).reshape(case["seqs"], per_seq)
    q = (1.5 * normal(sum(rows), case["q_heads"], hd)).to(t)
    off = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32, device=DEV)
    return {"op": "window", "pages": pages, "table": table, "q": q, "offsets": off,
            "lengths": torch.tensor(lens, dtype=torch.int32, device=DEV), "max_rows": max(rows),
            "max_length": max(lens), "sinks": case["sinks"], "window": case["window"]}


# --- one pass ---------------------------------------------------------------

def plain_logprobs(x, tokens, top):
    x = x.float()
    m = x.max(1, keepdim=True).values
    e = (x - m).exp()
    s = e.sum(1, keepdim=True)
    out = {"entropy": (s.log() - ((x - m) * e).sum(1, keepdim=True) / s)[:, 0]}
    if tokens.shape[1]:
        got = x.gather(1, tokens.long())
        out["logprob"] = got - m - s.log()
        at = torch.arange(x.shape[1], device=x.device)
        ahead = [((x > got[:, i:i + 1]) | ((x == got[:, i:i + 1]) & (at < tokens[:, i:i + 1]))).sum(1)
                 for i in range(tokens.shape[1])]
        out["rank"] = torch.stack(ahead, 1).to(torch.int32)
    if top:
        v, at = x.sort(dim=1, descending=True, stable=True)
        out["top_logprob"] = v[:, :top] - m - s.log()
        out["top_token"] = at[:, :top].to(torch.int32)
    return out


def plain_window(s):
    pages, table, lengths = s["pages"], s["table"], s["lengths"].long()
    n, per_seq = table.shape
    heads, hd = pages.shape[3], s["q"].shape[2]
    group = s["q"].shape[1] // heads
    got = pages[0, table.long()].float()                                 # [n][pages][2][heads][16 hd]
    k = got[:, :, 0].reshape(n, per_seq, heads, PAGE, hd).permute(0, 2, 1, 3, 4).reshape(n, heads, -1, hd)
    v = got[:, :, 1].reshape(n, per_seq, heads, 4, hd, 4).permute(0, 2, 1, 3, 5, 4).reshape(n, heads, -1, hd)
    # the queries of each sequence, side by side in rows of the longest
    off = s["offsets"].long()
    rows = off[1:] - off[:-1]
    i = torch.arange(s["max_rows"], device=off.device)
    on = i < rows[:, None]
    at = (off[:-1, None] + i).clamp_max(s["q"].shape[0] - 1)
    q = s["q"].float()[at].reshape(n, -1, heads, group, hd).permute(0, 2, 3, 1, 4).reshape(n, heads, -1, hd)
    pos = (lengths - rows)[:, None] + i
    t = torch.arange(per_seq * PAGE, device=off.device)
    see = t <= pos[:, :, None]
    if s["window"]:
        see = see & ((t < s["sinks"]) | (t > pos[:, :, None] - s["window"]))
    see = see & on[:, :, None] | (~on[:, :, None] & (t == 0))
    p = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(hd)
    p = p.reshape(n, heads, group, -1, t.numel()).masked_fill_(~see[:, None, None], -math.inf)
    p = p.sub_(p.max(-1, keepdim=True).values).exp_()
    p = p.div_(p.sum(-1, keepdim=True))
    o = torch.matmul(p.reshape(n, heads, -1, t.numel()), v)
    o = o.reshape(n, heads, group, -1, hd).permute(0, 3, 1, 2, 4).reshape(n, -1, heads * group, hd)
    return o[on].to(s["q"].dtype)


def run(state):
    if own:
        from paper_2609_26100_amd import ops

        if state["op"] == "logprobs":
            r = ops.token_logprobs(state["x"], state["tokens"], state["top"])
            out = {"entropy": r.entropy}
            if state["tokens"].shape[1]:
                out.update(logprob=r.logprob, rank=r.rank)
            if state["top"]:
                out.update(top_logprob=r.top_logprob, top_token=r.top_token)
            return out
        if state["op"] == "copy":
            ops.copy_pages(state["pages"], state["src"], state["dst"])
            return state["pages"]
        return ops.window_attention(state["q"], state["pages"], state["table"], state["offsets"], state["lengths"],
                                    sinks=state["sinks"], window=state["window"], max_rows=state["max_rows"],
                                    max_length=state["max_length"])
    if state["op"] == "logprobs":
        return plain_logprobs(state["x"], state["tokens"], state["top"])
    if state["op"] == "copy":
        src = torch.tensor(state["src"], device=DEV)
        dst = torch.tensor(state["dst"], device=DEV)
        state["pages"][:, dst] = state["pages"][:, src]
        return state["pages"]
    return plain_window(state)


# --- what a pass cannot do without -------------------------------------------

def work(case):
    es = 4 if case["type"] == "f32" else 2
    if case["op"] == "logprobs":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * es + 4 * case["rows"] * (1 + 3 * case["tokens"] + 2 * case["top"]), "flops": 6.0 * n}
    if case["op"] == "copy":
        size = 2 * case["kv_heads"] * PAGE * case["head_dim"] * es
        return {"bytes": case["layers"] * case["sources"] * (1 + case["fan"]) * size, "flops": 0.0}
    kv, pairs = 0, 0
    for n, length in zip(*ragged(case)):
        first, win, sinks = length - n, case["window"], case["sinks"]
        if win:
            kv += min(length, sinks + min(length, win + n - 1))
            for p in range(first, length):
                low = max(0, p + 1 - win)                                # first token of the row's window
                pairs += p + 1 - low + min(low, sinks)
        else:
            kv += length
            pairs += n * first + n * (n + 1) // 2
    hd, rows = case["head_dim"], sum(ragged(case)[0])
    return {"bytes": es * hd * (2 * kv * case["kv_heads"] + 2 * rows * case["q_heads"]),
            "flops": 4.0 * hd * pairs * case["q_heads"]}


# --- the same in 64 bits ------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "copy":
        out = s["pages"].double()
        for a, b in zip(s["src"], s["dst"]):
            out[:, b] = s["pages"][:, a].double()
        return out
    if case["op"] == "logprobs":
        parts = []
        for i in range(0, case["rows"], 128):
            x = s["x"][i:i + 128].double()
            lp = x - torch.logsumexp(x, 1, keepdim=True)
            tok = s["tokens"][i:i + 128].long()
            part = {"entropy": -(lp.exp() * lp).sum(1)}
            order = torch.argsort(x, dim=1, descending=True, stable=True)
            if case["tokens"]:
                place = torch.empty_like(order)
                place.scatter_(1, order, torch.arange(x.shape[1], device=DEV).expand_as(order).contiguous())
                part["logprob"] = lp.gather(1, tok)
                part["rank"] = place.gather(1, tok).to(torch.int32)
            if case["top"]:
                part["top_token"] = order[:, : case["top"]].to(torch.int32)
                part["top_logprob"] = lp.gather(1, order[:, : case["top"]])
            parts.append(part)
        return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    rows, lens = ragged(case)
    hd, group = case["head_dim"], case["q_heads"] // case["kv_heads"]
    out = torch.empty(sum(rows), case["q_heads"], hd, dtype=torch.float64, device=DEV)
    r0 = 0
    for i, (n, length) in enumerate(zip(rows, lens)):
        ids = s["table"][i, : -(-length // PAGE)].long()
        for h in range(case["kv_heads"]):
            k = s["pages"][0, ids, 0, h].reshape(-1, hd)[:length].double()
            v = s["pages"][0, ids, 1, h].reshape(-1, 4, hd, 4).transpose(2, 3).reshape(-1, hd)[:length].double()
            key = torch.arange(length, device=DEV)[None]
            query = torch.arange(length - n, length, device=DEV)[:, None]
            hidden = key > query
            if case["window"]:
                hidden |= (key >= case["sinks"]) & (query - key >= case["window"])
            for j in range(h * group, (h + 1) * group):
                a = s["q"][r0:r0 + n, j].double() @ k.T * hd ** -0.5
                out[r0:r0 + n, j] = torch.softmax(a.masked_fill(hidden, -math.inf), 1) @ v
        r0 += n
    return out
