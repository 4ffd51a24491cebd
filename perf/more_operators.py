"""What is measured of the serving operators: attention of a batch that shares a prefix, the weights
that cached rows gather, eviction of rows by those weights, and the verification of drafted tokens.

Each case is one pass through one operator.  The plain forms are elementary torch operations in 32
bits (64 where a choice between tokens hangs on them), rounded once at the end; `exact` computes the
same results from their definitions in 64 bits.
"""

import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
         "i8": torch.int8, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1, "e4m3": 1}
SCALED = ("i8", "e4m3")


def _gar():
    from paper_2004_09362_gb300 import gar
    return gar


# ------------------------------------------------------------------------------- the cases

def _prefix(name, groups, share, q_heads, kv_heads, dim, prefix, rest, page, cache, dtype, drafts=False):
    c = {"op": "prefix", "groups": groups, "share": share, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
         "prefix": prefix, "rest": rest, "page": page, "cache": cache, "dtype": dtype, "drafts": drafts}
    return dict(c, name=name) if name else c


def _weigh(name, batch, q_heads, kv_heads, dim, length, page, cache, dtype, window=0):
    c = {"op": "weigh", "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "length": length,
         "page": page, "cache": cache, "dtype": dtype, "window": window}
    return dict(c, name=name) if name else c


def _evict(name, batch, kv_heads, dim, length, keep, first, recent, page, cache, even=False):
    c = {"op": "evict", "batch": batch, "kv_heads": kv_heads, "dim": dim, "length": length, "keep": keep,
         "first": first, "recent": recent, "page": page, "cache": cache, "even": even}
    return dict(c, name=name) if name else c


def _verify(name, batch, drafts, vocab, dtype):
    c = {"op": "verify", "batch": batch, "drafts": drafts, "vocab": vocab, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # four drafted tokens and the one before them at a chat's start: the smallest call
        _prefix("prefix_drafts_short", 1, 5, 32, 8, 128, 425, 5, 16, "bf16", "bf16", drafts=True),
        # drafted tokens of a serving batch over an 8-bit cache, lengths of all kinds, an odd page size
        _prefix("prefix_drafts_i8", 24, 5, 20, 4, 64, 4096, 5, 24, "i8", "f16", drafts=True),
        # a batch of chats after one system prompt
        _prefix("prefix_chats", 1, 64, 32, 8, 128, 8192, 1024, 16, "bf16", "bf16"),
        # questions to one very long document
        _prefix("prefix_document", 1, 32, 32, 8, 128, 131072, 200, 64, "bf16", "bf16"),
        # many samples of one long prompt: as much arithmetic as memory
        _prefix("prefix_samples", 1, 250, 32, 8, 128, 16384, 300, 32, "f16", "f16"),
        # the weights of one sequence's rows, an odd head size
        _weigh("weigh_one", 1, 10, 5, 80, 1021, 16, "f16", "f16"),
        # a serving batch of different lengths
        _weigh("weigh_batch", 24, 32, 8, 128, 8192, 16, "bf16", "bf16"),
        # a full cache in its steady state: one row too many in each sequence
        _evict("evict_step", 48, 8, 128, 1025, 1024, 4, 64, 16, "bf16", even=True),
        # prompts cut down to a quarter, lengths of all kinds
        _evict("evict_prompt_i8", 8, 4, 96, 16001, 4000, 5, 129, 24, "i8"),
        # one sequence's four drafts
        _verify("verify_one", 1, 4, 32768, "f32"),
        # an odd vocabulary in 16 bits
        _verify("verify_odd", 57, 3, 50021, "bf16"),
        # a large batch over a large vocabulary
        _verify("verify_batch", 256, 5, 131072, "f32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = 3 * 10 ** 8
    while True:
        op = rng.choice(["prefix", "prefix", "weigh", "evict", "verify"])
        page = rng.choice([1, 5, 16, 24, 32, 64, 128])
        dim = rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        kv = rng.choice([1, 2, 3, 4, 8, 8])
        if op == "prefix":
            drafts = rng.random() < 0.4
            groups = _log(rng, 1, 32) if drafts else rng.choice([1, 1, 1, 2, 5])
            share = _log(rng, 1, 16) if drafts else _log(rng, 1, 256)
            c = _prefix(None, groups, share, kv * rng.choice([1, 2, 4, 5, 8]), kv, dim, _log(rng, 1, 131072),
                        share if drafts else _log(rng, 1, 2048), page, rng.choice([dtype, dtype, dtype, "i8", "e4m3"]),
                        dtype, drafts)
        elif op == "weigh":
            length = _log(rng, 1, 131072)
            c = _weigh(None, _log(rng, 1, 128), kv * rng.choice([1, 2, 4, 5, 8, 16]), kv, dim, length, page,
                       rng.choice([dtype, dtype, "i8", "e4m3"]), dtype, rng.choice([0, 0, 0, 1 + length // 3]))
        elif op == "evict":
            length = _log(rng, 2, 65536)
            keep = max(1, int(length * rng.choice([0.1, 0.25, 0.5, 0.9, 1.0]))) - rng.choice([0, 0, 1])
            keep = max(1, keep)
            first = rng.choice([0, min(4, keep), keep // 5])
            c = _evict(None, _log(rng, 1, 64), kv, dim, length, keep, first, min(keep - first, rng.choice([0, 1, 32, keep // 4])),
                       page, rng.choice(["bf16", "f16", "f32", "i8"]), rng.random() < 0.3)
        else:
            c = _verify(None, _log(rng, 1, 256), rng.choice([0, 1, 2, 4, 5, 8, 15]), _log(rng, 2, 200000),
                        rng.choice(["f32", "f32", "bf16", "f16"]))
        if _cost(c) < most and work(c)["flops"] < 7 * 10 ** 10:
            return c


def _cost(c):
    """Elements that the plain form holds at once."""
    if c["op"] == "prefix":
        rows = c["groups"] * (c["prefix"] + c["page"]) + c["groups"] * c["share"] * (c["rest"] + c["page"])
        scores = c["groups"] * c["share"] * c["q_heads"] * (c["prefix"] + c["rest"])
        return max(rows * c["kv_heads"] * c["dim"], scores)
    if c["op"] == "weigh":
        return c["batch"] * (c["length"] + c["page"]) * max(c["kv_heads"] * c["dim"], c["q_heads"])
    if c["op"] == "evict":
        return 2 * c["batch"] * (c["length"] + c["page"]) * c["kv_heads"] * c["dim"]
    return c["batch"] * (2 * c["drafts"] + 1) * c["vocab"]


def _lengths(count, most):
    """A batch's lengths: the first is the longest, one sequence is empty, one holds one token."""
    n = [max(0, int(most * ((b * 0.6180339887498949) % 1.0))) for b in range(count)]
    n[0] = most
    if count > 5:
        n[1], n[2] = 0, 1
    return n


def _rest(c):
    """Each sequence's own rows: a draft sees those before it, a chat has what it has."""
    batch = c["groups"] * c["share"]
    return [1 + b % c["share"] for b in range(batch)] if c["drafts"] else _lengths(batch, c["rest"])


def _evict_lengths(c):
    return [c["length"]] * c["batch"] if c["even"] else _lengths(c["batch"], c["length"])


def work(c):
    size = BYTES[c.get("cache", c.get("dtype"))]
    scale = 4 if c.get("cache") in SCALED else 0
    if c["op"] == "prefix":
        batch = c["groups"] * c["share"]
        n, own_n = _lengths(c["groups"], c["prefix"]), _rest(c)
        rows = sum(n) + (c["groups"] * c["share"] if c["drafts"] else sum(own_n))
        seen = sum(n) * c["share"] + sum(own_n)
        return {"bytes": rows * c["kv_heads"] * 2 * (c["dim"] * size + scale) + 4 * (rows // c["page"])
                + batch * c["q_heads"] * (2 * c["dim"] * BYTES[c["dtype"]] + 4),
                "flops": 4 * seen * c["q_heads"] * c["dim"]}
    if c["op"] == "weigh":
        n = _lengths(c["batch"], c["length"])
        seen = sum(min(v, c["window"]) if c["window"] else v for v in n)
        rows = c["batch"] * -(-c["length"] // c["page"]) * c["page"]
        return {"bytes": seen * c["kv_heads"] * (c["dim"] * size + scale) + 4 * (seen // c["page"])
                + 8 * rows * c["kv_heads"] + c["batch"] * c["q_heads"] * (c["dim"] * BYTES[c["dtype"]] + 4),
                "flops": 2 * seen * c["q_heads"] * c["dim"]}
    if c["op"] == "evict":
        n = _evict_lengths(c)
        # rows past `keep` that stay: their share of `keep`, if weights do not depend on the place
        moved = sum(round((v - c["keep"]) * (c["keep"] - c["first"]) / (v - c["first"])) for v in n if v > c["keep"])
        rows = c["batch"] * -(-c["length"] // c["page"]) * c["page"]
        return {"bytes": c["kv_heads"] * (16 * rows + moved * 4 * (c["dim"] * size + scale)),
                "flops": sum(n) * c["kv_heads"]}
    # the first draft that is refused decides which one row of each is read whole
    rows = 2 if c["drafts"] else 1
    return {"bytes": c["batch"] * (rows * c["vocab"] * size + c["drafts"] * (2 * size + 20) + 8),
            "flops": 2 * c["batch"] * rows * c["vocab"]}


# ------------------------------------------------------------------------------- the inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _pool(tables, lens, heads, page, dim, cache, g, clean=False):
    """A paged cache for tables of [rows][width] pages whose rows have `lens` tokens, pages in a scattered order.
    What pages hold past a row's end was never written (NaN in float caches) unless `clean`."""
    need = [[-(-v // page) for v in n] for n in lens]
    total = sum(sum(v) for v in need)
    count = total + 1 + total // 16
    ids = torch.randperm(count, generator=g, device="cuda")[:total].to(torch.int32)
    shape = (count, heads, page, dim)
    s = {}
    for w in ("k", "v"):
        if cache in SCALED:
            if cache == "i8":
                x = torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8)
            else:
                x = (torch.randn(shape, generator=g, device="cuda", dtype=torch.float16) * 100).clamp_(-448, 448).to(TORCH["e4m3"])
            s[w + "_scale"] = torch.rand(shape[:3], generator=g, device="cuda") * 0.01 + (0.01 if cache == "i8" else 0.004)
        else:
            x = torch.randn(shape, generator=g, device="cuda", dtype=TORCH[cache])
        s[w] = x
    out, at = [], 0
    for width, n, pages in zip(tables, lens, need):
        table = torch.full((len(n), width), -1, dtype=torch.int32, device="cuda")
        taken = torch.arange(width, device="cuda")[None] < torch.tensor(pages, device="cuda")[:, None]
        table[taken] = ids[at:at + sum(pages)]
        at += sum(pages)
        length = torch.tensor(n, dtype=torch.int32, device="cuda")
        if cache not in SCALED and not clean:
            row = torch.arange(width * page, device="cuda").view(1, width, page)
            past = (row >= length[:, None, None]) & taken[:, :, None]
            b, p, o = past.nonzero(as_tuple=True)
            for w in ("k", "v"):
                s[w][table[b, p].long(), :, o] = float("nan")
        out.append((table, length))
    return s, out


def _width(most, page):
    return max(1, -(-most // page))


def _prefix_inputs(c, seed):
    g = _gen(seed)
    page, batch = c["page"], c["groups"] * c["share"]
    n = _lengths(c["groups"], c["prefix"])
    rest = [c["share"]] * c["groups"] if c["drafts"] else _rest(c)
    s, tables = _pool([_width(c["prefix"], page), _width(c["rest"], page)], [n, rest], c["kv_heads"], page, c["dim"], c["cache"], g)
    (s["prefix_table"], s["prefix_lens"]), (s["table"], s["lens"]) = tables
    if c["drafts"]:
        s["table"] = s["table"].repeat_interleave(c["share"], 0)
        s["lens"] = torch.tensor(_rest(c), dtype=torch.int32, device="cuda")
    s["q"] = torch.randn((batch, c["q_heads"], c["dim"]), generator=g, device="cuda").to(TORCH[c["dtype"]]) * 2
    return s


def _weigh_inputs(c, seed):
    g = _gen(seed)
    n = _lengths(c["batch"], c["length"])
    width = _width(c["length"], c["page"])
    s, tables = _pool([width], [n], c["kv_heads"], c["page"], c["dim"], c["cache"], g)
    s["table"], s["lens"] = tables[0]
    s["q"] = torch.randn((c["batch"], c["q_heads"], c["dim"]), generator=g, device="cuda").to(TORCH[c["dtype"]]) * 2
    # what earlier tokens left, and the log of the sum of this one's weights
    rows = width * c["page"]
    s["weights"] = torch.rand((c["batch"], c["kv_heads"], rows), generator=g, device="cuda").square_()
    x, seen = _scores(s, c, s["table"], s["lens"])
    s["lse"] = torch.logsumexp(torch.where(seen[:, None, None], x, -math.inf), -1).reshape(c["batch"], -1)
    return s


def _evict_inputs(c, seed):
    g = _gen(seed)
    n = _evict_lengths(c)
    width = _width(c["length"], c["page"])
    s, tables = _pool([width], [n], c["kv_heads"], c["page"], c["dim"], c["cache"], g, clean=True)
    s["table"], s["lens"] = tables[0]
    shape = (c["batch"], c["kv_heads"], width * c["page"])
    # a few rows gather most of the weight, some none at all, some the same; earlier evictions have mixed the positions
    w = torch.randn(shape, generator=g, device="cuda").mul_(2).exp_()
    u = torch.rand(shape, generator=g, device="cuda")
    s["weights"] = torch.where(u < 0.05, 0.0, torch.where(u < 0.15, 0.5, w))
    at = torch.arange(shape[2], device="cuda") + torch.rand(shape, generator=g, device="cuda") * 16
    at[..., :c["first"]] -= 1000
    s["positions"] = at.argsort(-1).argsort(-1).to(torch.int32) * 2
    return s


def _verify_inputs(c, seed):
    g = _gen(seed)
    shape = (c["batch"], c["drafts"] + 1, c["vocab"])
    x = torch.randn(shape, generator=g, device="cuda") * 2.5
    s = {"target": torch.softmax(x, -1).to(TORCH[c["dtype"]])}
    x = x[:, :-1] + torch.randn((c["batch"], c["drafts"], c["vocab"]), generator=g, device="cuda") * 0.8
    s["draft"] = torch.softmax(x, -1).to(TORCH[c["dtype"]])
    if c["drafts"]:
        # drafted from the draft's probabilities; some sequences have fewer drafts
        total = s["draft"].float().cumsum(-1)
        u = torch.rand((c["batch"], c["drafts"], 1), generator=g, device="cuda") * total[..., -1:]
        s["tokens"] = torch.searchsorted(total, u).squeeze(-1).clamp_(max=c["vocab"] - 1)
        few = torch.arange(c["batch"], device="cuda") % 8 == 5
        s["tokens"][few, c["drafts"] - 1] = -1
    else:
        s["tokens"] = torch.empty((c["batch"], 0), dtype=torch.int64, device="cuda")
    s["uniform"] = torch.rand(shape[:2], generator=g, device="cuda")
    return s


INPUTS = {"prefix": _prefix_inputs, "weigh": _weigh_inputs, "evict": _evict_inputs, "verify": _verify_inputs}


def prepare(case, seed):
    c = case
    s = INPUTS[c["op"]](c, seed)
    if own and c["op"] != "verify":
        s["cache"] = _gar().KVCache(s["k"], s["v"], s.get("k_scale"), s.get("v_scale"))
        if c["op"] == "prefix":
            s["plan"] = _gar().gar_attn_plan_create(c["q_heads"], c["kv_heads"], c["dim"])
    s["case"] = c
    return s


# ------------------------------------------------------------------------------- the passes

def _whole(s, w, table, cache):
    """Rows [sequences, heads, width * page, dim] of a table's pages, in 32 bits."""
    ids = table.long().clamp(min=0)
    if cache in SCALED:
        x = s[w].view(torch.uint8)[ids].view(s[w].dtype).float() * s[w + "_scale"][ids][..., None]
    else:
        x = s[w][ids].float()
    return x.transpose(1, 2).flatten(2, 3)


def _seen(table, lens, page, window=0):
    at = torch.arange(table.shape[1] * page, device="cuda")[None]
    n = lens.long()[:, None]
    return (at < n) & ((at >= n - window) if window else (at >= 0))


def _scores(s, c, table, lens):
    """[sequences, cached heads, queries of each, rows] in 32 bits, and which rows count."""
    seen = _seen(table, lens, c["page"], c.get("window", 0))
    k = torch.where(seen[:, None, :, None], _whole(s, "k", table, c["cache"]), 0.0)
    q = s["q"].float()
    batch, heads, dim = q.shape
    q = q.view(batch, c["kv_heads"], heads // c["kv_heads"], dim)
    if table.shape[0] != batch:  # a prefix's queries are all of its sequences'
        q = q.view(table.shape[0], -1, *q.shape[1:]).transpose(1, 2).flatten(2, 3)
    return torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(dim)), seen


def _plain_prefix(s):
    c = s["case"]
    batch, heads, dim = s["q"].shape
    kv, group = c["kv_heads"], heads // c["kv_heads"]
    parts = []
    for table, lens in ((s["prefix_table"], s["prefix_lens"]), (s["table"], s["lens"])):
        y, seen = _scores(s, c, table, lens)
        y = torch.where(seen[:, None, None], y, -math.inf)
        m = y.amax(-1, keepdim=True)
        p = torch.exp(y - torch.where(m == -math.inf, 0.0, m))
        v = torch.where(seen[:, None, :, None], _whole(s, "v", table, c["cache"]), 0.0)
        o, l = torch.matmul(p, v), p.sum(-1, keepdim=True)
        if table.shape[0] != batch:
            m, l, o = (x.unflatten(2, (-1, group)).transpose(1, 2).flatten(0, 1) for x in (m, l, o))
        parts.append((m, l, o))
    top = torch.maximum(parts[0][0], parts[1][0])
    off = torch.where(top == -math.inf, 0.0, top)
    total = sum(torch.exp(m - off) * l for m, l, _ in parts)
    out = sum(torch.exp(m - off) * o for m, _, o in parts) / torch.where(total == 0, 1.0, total)
    return {"out": out.reshape(batch, heads, dim).to(s["q"].dtype), "lse": (torch.log(total) + top).reshape(batch, heads)}


def _plain_weigh(s):
    c = s["case"]
    y, seen = _scores(s, c, s["table"], s["lens"])
    p = torch.exp(y - s["lse"].view(*y.shape[:3], 1)).sum(2)
    return {"weights": s["weights"] + torch.where(seen[:, None], p, 0.0)}


def _plain_evict(s):
    c, page = s["case"], s["case"]["page"]
    batch, heads, rows = s["weights"].shape
    at = torch.arange(rows, device="cuda")
    n = s["lens"].long()[:, None, None]
    there = at < n
    newest = torch.where(there, s["positions"], -1).amax(-1, keepdim=True)
    kept_for_sure = (at < c["first"]) | (s["positions"] > newest - c["recent"])
    key = torch.where(kept_for_sure, math.inf, s["weights"])
    key = torch.where(there, key, -math.inf)
    # the largest first, equal ones by their row
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    stays = torch.zeros_like(there.expand_as(key)).scatter_(-1, order[..., :c["keep"]], True) & there
    stays = torch.where(n > c["keep"], stays, there)
    target = (at < c["keep"]) & there & ~stays
    source = (at >= c["keep"]) & stays
    b, h, to = target.nonzero(as_tuple=True)     # in the order of the rows, as many of one as of the other
    _, _, frm = source.nonzero(as_tuple=True)
    to_page, from_page = s["table"][b, to // page].long(), s["table"][b, frm // page].long()
    for x in ("k", "v", "k_scale", "v_scale"):
        if x in s:
            s[x][to_page, h, to % page] = s[x][from_page, h, frm % page]
    left = n.clamp(max=c["keep"])
    weights, positions = s["weights"].clone(), s["positions"].clone()
    weights[b, h, to], positions[b, h, to] = s["weights"][b, h, frm], s["positions"][b, h, frm]
    return dict(_cache_of(s), weights=torch.where(at < left, weights, 0.0), positions=torch.where(at < left, positions, -1),
                lengths=left.flatten().to(torch.int32))


def _cache_of(s):
    return {x: s[x] for x in ("k", "v", "k_scale", "v_scale") if x in s}


def _clamped(x):
    return torch.where(x > 0, x, 0.0).clamp(max=1.0)


def _plain_verify(s):
    drafts, tokens = s["tokens"].shape[1], s["tokens"]
    batch, _, vocab = s["target"].shape
    each = torch.arange(batch, device="cuda")
    if drafts:
        at = tokens.clamp(0, vocab - 1)[..., None]
        inside = (tokens >= 0) & (tokens < vocab)
        p = torch.where(inside, _clamped(s["target"][:, :-1].gather(-1, at).squeeze(-1).double()), 0.0)
        q = torch.where(inside, _clamped(s["draft"].gather(-1, at).squeeze(-1).double()), 0.0)
        good = s["uniform"][:, :-1].double() * q < p
        accepted = good.long().cumprod(-1).sum(-1)
        stop = accepted.clamp(max=drafts - 1)
        # the rest of the target where a draft was refused, the target itself where there is no more of them
        refused = (accepted < drafts) & (tokens[each, stop] >= 0)
        rest = _clamped(s["target"][each, accepted].double())
        left = (rest - _clamped(s["draft"][each, stop].double())).clamp(min=0.0)
        rest = torch.where((refused & (left > 0).any(-1))[:, None], left, rest)
    else:
        accepted = torch.zeros(batch, dtype=torch.int64, device="cuda")
        rest = _clamped(s["target"][:, 0].double())
    total = rest.cumsum(-1)
    u = s["uniform"][:, -1].double()[:, None]    # a number of its own: those before it decided on the drafts
    past = total > u * total[:, -1:]
    last = torch.where(rest > 0, torch.arange(vocab, device="cuda"), -1).amax(-1)
    token = torch.where(past.any(-1), past.long().argmax(-1), last)
    at = torch.arange(drafts + 1, device="cuda")[None]
    given = torch.cat([tokens, torch.full((batch, 1), -1, dtype=torch.int64, device="cuda")], -1)
    out = torch.where(at < accepted[:, None], given, torch.where(at == accepted[:, None], token[:, None], -1))
    return {"tokens": out, "accepted": accepted.to(torch.int32)}


PLAIN = {"prefix": _plain_prefix, "weigh": _plain_weigh, "evict": _plain_evict, "verify": _plain_verify}


def run(state):
    s, c = state, state["case"]
    if not own:
        return PLAIN[c["op"]](s)
    gar = _gar()
    if c["op"] == "prefix":
        out, lse = gar.gar_prefix_attention(s["plan"], s["q"], s["cache"], s["prefix_table"], s["prefix_lens"],
                                            s["table"], s["lens"], lse=True)
        return {"out": out, "lse": lse}
    if c["op"] == "weigh":
        return {"weights": gar.gar_kv_weigh(s["q"], s["cache"], s["table"], s["lens"], s["lse"], s["weights"],
                                            window=c["window"])}
    if c["op"] == "evict":
        weights, positions, lengths = gar.gar_kv_evict(s["cache"], s["weights"], s["positions"], s["table"], s["lens"],
                                                       c["keep"], first=c["first"], recent=c["recent"])
        return dict(_cache_of(s), weights=weights, positions=positions, lengths=lengths)
    tokens, accepted = gar.gar_verify_drafts(s["target"], s["draft"], s["tokens"], s["uniform"])
    return {"tokens": tokens, "accepted": accepted}


# ------------------------------------------------------------------------------- 64 bits

def _rows(s, c, w, table, b, n, first=0):
    """Rows [first, n) of one sequence, [heads, rows, dim] in 64 bits."""
    page = c["page"]
    ids = table[b, first // page:-(-n // page)].long()
    x = s[w].view(torch.uint8)[ids].view(s[w].dtype).double() if c["cache"] in SCALED else s[w][ids].double()
    if c["cache"] in SCALED:
        x = x * s[w + "_scale"][ids].double()[..., None]
    return x.permute(1, 0, 2, 3).flatten(1, 2)[:, first % page:first % page + n - first]


def _exact_prefix(c, seed):
    s = _prefix_inputs(c, seed)
    kv, dim, share = c["kv_heads"], c["dim"], c["share"]
    group, batch = c["q_heads"] // kv, c["groups"] * share
    n, rest = _lengths(c["groups"], c["prefix"]), _rest(c)
    q = s["q"].double().view(c["groups"], share, kv, group, dim)
    out = torch.zeros((c["groups"], share, kv, group, dim), dtype=torch.float64, device="cuda")
    lse = torch.full(out.shape[:-1], -math.inf, dtype=torch.float64, device="cuda")
    for g in range(c["groups"]):
        for h in range(kv):
            k, v = (_rows(s, c, w, s["prefix_table"], g, n[g])[h] for w in ("k", "v"))
            y = torch.einsum("sgd,nd->sgn", q[g, :, h], k) / math.sqrt(dim)
            for i in range(share):
                b = g * share + i
                if n[g] + rest[b] == 0:
                    continue
                k2, v2 = (_rows(s, c, w, s["table"], b, rest[b])[h] for w in ("k", "v"))
                z = torch.cat([y[i], q[g, i, h] @ k2.T / math.sqrt(dim)], -1)
                lse[g, i, h] = torch.logsumexp(z, -1)
                p = torch.softmax(z, -1)
                out[g, i, h] = p[:, :n[g]] @ v + p[:, n[g]:] @ v2
    return {"out": out.view(batch, c["q_heads"], dim), "lse": lse.view(batch, c["q_heads"])}


def _exact_weigh(c, seed):
    s = _weigh_inputs(c, seed)
    kv, dim = c["kv_heads"], c["dim"]
    got = s["weights"].double()
    for b, n in enumerate(_lengths(c["batch"], c["length"])):
        first = max(0, n - c["window"]) if c["window"] else 0
        if n == first:
            continue
        q = s["q"][b].double().view(kv, -1, dim)
        y = torch.einsum("hgd,hnd->hgn", q, _rows(s, c, "k", s["table"], b, n, first)) / math.sqrt(dim)
        got[b, :, first:n] += (y - s["lse"][b].double().view(kv, -1, 1)).exp().sum(1)
    return {"weights": got}


def _exact_evict(c, seed):
    s = _evict_inputs(c, seed)
    keep, page, rows = c["keep"], c["page"], s["weights"].shape[2]
    old = {x: v.clone() for x, v in _cache_of(s).items()}
    weights, positions = torch.zeros_like(s["weights"]), torch.full_like(s["positions"], -1)
    place = torch.arange(rows, device="cuda")
    for b, n in enumerate(_evict_lengths(c)):
        for h in range(c["kv_heads"]):
            w, p = s["weights"][b, h, :n].double(), s["positions"][b, h, :n].double()
            to = frm = place[:0]
            if n > keep:
                sure = (place[:n] < c["first"]) | (p > p.max() - c["recent"])
                free = (~sure).nonzero().flatten()
                free = free[torch.sort(-w[free], dim=-1, stable=True).indices][:max(0, keep - int(sure.sum()))]
                kept = torch.cat([sure.nonzero().flatten(), free]).sort().values[:keep]
                is_kept = torch.zeros(n, dtype=torch.bool, device="cuda")
                is_kept[kept] = True
                to, frm = (~is_kept[:keep]).nonzero().flatten(), kept[kept >= keep]
            m = min(n, keep)
            weights[b, h, :m], positions[b, h, :m] = s["weights"][b, h, :m], s["positions"][b, h, :m]
            weights[b, h, to], positions[b, h, to] = s["weights"][b, h, frm], s["positions"][b, h, frm]
            at = s["table"][b].long()
            for x, v in old.items():
                s[x][at[to // page], h, to % page] = v[at[frm // page], h, frm % page]
    lengths = torch.tensor([min(n, keep) for n in _evict_lengths(c)], dtype=torch.int32, device="cuda")
    return dict({x: v.double() if v.is_floating_point() else v for x, v in _cache_of(s).items()}, weights=weights.double(),
                positions=positions, lengths=lengths)


def _exact_verify(c, seed):
    s = _verify_inputs(c, seed)
    tokens = torch.full((c["batch"], c["drafts"] + 1), -1, dtype=torch.int64)
    accepted = torch.zeros(c["batch"], dtype=torch.int32)
    given, uniform = s["tokens"].tolist(), s["uniform"].double().tolist()
    for b in range(c["batch"]):
        i, r = 0, None
        while i < c["drafts"] and given[b][i] >= 0:
            t = given[b][i]
            if not uniform[b][i] * float(s["draft"][b, i, t]) < float(s["target"][b, i, t]):
                r = (s["target"][b, i].double() - s["draft"][b, i].double()).relu()
                break
            tokens[b, i] = t
            i += 1
        if r is None or not bool(r.any()):
            r = s["target"][b, i].double()
        total = r.cumsum(0)
        k = int(torch.searchsorted(total, uniform[b][-1] * total[-1:], right=True)[0])
        tokens[b, i] = k if k < c["vocab"] else int(r.nonzero().max())
        accepted[b] = i
    return {"tokens": tokens.cuda(), "accepted": accepted.cuda()}


EXACT = {"prefix": _exact_prefix, "weigh": _exact_weigh, "evict": _exact_evict, "verify": _exact_verify}


def exact(case, seed):
    return EXACT[case["op"]](case, seed)
