"""What is measured of the decoding operators: rotary positions, the quantised paged cache, and
attention of one new token over that cache.

Each case is one pass through one operator.  The plain forms are elementary torch operations
in 32 bits, rounded once at the end; `exact` computes the same results from their definitions
in 64 bits.
"""

import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
         "i8": torch.int8, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1, "e4m3": 1}
QMAX = {"i8": 127.0, "e4m3": 448.0}
PAIRS = ["half", "interleaved"]


def _gar():
    from paper_2004_09362_gb300 import gar
    return gar


# ------------------------------------------------------------------------------- the cases

def _rope(name, tokens, heads, dim, rot, dtype, layout="half", inverse=False, scaling="none",
          factor=1.0, start=0):
    c = {"op": "rope", "tokens": tokens, "heads": heads, "dim": dim, "rot": rot, "dtype": dtype,
         "layout": layout, "inverse": inverse, "scaling": scaling, "factor": factor, "start": start}
    return dict(c, name=name) if name else c


def _cache(name, tokens, heads, dim, page, cache, dtype, rot=0, layout="half", skip=0):
    c = {"op": "cache", "tokens": tokens, "heads": heads, "dim": dim, "page": page, "cache": cache,
         "dtype": dtype, "rot": rot, "layout": layout, "skip": skip}
    return dict(c, name=name) if name else c


def _attn(name, batch, q_heads, kv_heads, dim, length, page, cache, dtype, window=0):
    c = {"op": "attn", "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
         "length": length, "page": page, "cache": cache, "dtype": dtype, "window": window}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the query of one new token: the smallest call there is
        _rope("rope_token", 1, 8, 128, 128, "bf16", start=424),
        # a prompt far into a context stretched eightfold, a third of an odd head rotated
        _rope("rope_part_long", 1021, 5, 80, 32, "f32", "interleaved", scaling="parts", factor=8.0,
              start=100000),
        # gradients of queries and keys of a training batch, turned back
        _rope("rope_train_grad", 16384, 40, 128, 128, "bf16", inverse=True),
        # one decoding step of 24 sequences: keys rotated as they are written, in 8-bit floats
        _cache("cache_step_e4m3", 24, 8, 128, 16, "e4m3", "bf16", rot=128),
        # a prompt with padding tokens that are not kept
        _cache("cache_padded_i8", 1531, 3, 96, 24, "i8", "f16", skip=7),
        # a batch of long prompts
        _cache("cache_prompt_i8", 32768, 8, 128, 64, "i8", "bf16", rot=64, layout="interleaved"),
        # one sequence at a chat's start
        _attn("attn_one_short", 1, 32, 8, 128, 425, 16, "bf16", "bf16"),
        # one very long document
        _attn("attn_one_long", 1, 64, 8, 128, 262143, 64, "bf16", "bf16"),
        # a serving batch of very different lengths, one of them empty
        _attn("attn_batch_e4m3", 127, 32, 8, 128, 8192, 16, "e4m3", "bf16"),
        # a sliding window over an odd page size
        _attn("attn_window_i8", 24, 20, 4, 64, 4096, 24, "i8", "f16", window=1000),
        # 32-bit checks of a model with a head for each query, an odd head size
        _attn("attn_f32", 7, 6, 6, 80, 2000, 5, "f32", "f32"),
        # all queries share one wide head
        _attn("attn_shared_f16", 8, 16, 1, 256, 12345, 32, "f16", "f16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = 4 * 10 ** 8
    while True:
        op = rng.choice(["rope", "cache", "attn", "attn"])
        if op == "rope":
            dim = rng.choice([64, 80, 96, 128, 192, 256])
            scaling = rng.choice(["none", "none", "linear", "parts"])
            c = _rope(None, _log(rng, 1, 16384), _log(rng, 1, 64), dim,
                      rng.choice([dim, dim, dim // 2, 32]), rng.choice(["f32", "bf16", "f16"]),
                      rng.choice(PAIRS), rng.random() < 0.4, scaling,
                      1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]), _log(rng, 1, 100000) - 1)
        elif op == "cache":
            dim = rng.choice([64, 80, 96, 128, 192, 256])
            c = _cache(None, _log(rng, 1, 32768), _log(rng, 1, 16), dim, rng.choice([1, 5, 16, 24, 32, 64, 128]),
                       rng.choice(["i8", "e4m3"]), rng.choice(["bf16", "f16", "f32"]),
                       rng.choice([0, 0, dim, dim // 2]), rng.choice(PAIRS), rng.choice([0, 3, 7]))
        else:
            dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
            kv = rng.choice([1, 2, 3, 4, 8, 8])
            length = _log(rng, 1, 131072)
            c = _attn(None, _log(rng, 1, 256), kv * rng.choice([1, 2, 4, 5, 8, 16]), kv,
                      rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256]), length, rng.choice([1, 5, 16, 24, 32, 64, 128]),
                      rng.choice([dtype, dtype, "i8", "e4m3"]), dtype,
                      rng.choice([0, 0, 0, 1 + length // 3]))
        if _cost(c) < most and work(c)["bytes"] < most:
            return c


def _cost(c):
    """Elements that the plain form holds at once."""
    if c["op"] == "attn":
        return c["batch"] * (c["length"] + c["page"]) * c["kv_heads"] * c["dim"]
    return c["tokens"] * c["heads"] * c["dim"]


def _lengths(c):
    """The batch's lengths: the first is the longest, one sequence is empty, one holds one token."""
    n = [max(0, int(c["length"] * ((b * 0.6180339887498949) % 1.0))) for b in range(c["batch"])]
    n[0] = c["length"]
    if len(n) > 5:
        n[1], n[2] = 0, 1
    return n


def work(c):
    if c["op"] == "rope":
        x = c["tokens"] * c["heads"] * c["dim"]
        t = c["tokens"] * (8 + 4 * c["rot"])
        return {"bytes": 2 * x * BYTES[c["dtype"]] + t, "flops": 3 * c["tokens"] * c["heads"] * c["rot"]}
    if c["op"] == "cache":
        kept = len(_kept(c["tokens"], c["skip"]))
        rows = 2 * kept * c["heads"]
        both = 2 * rows * c["dim"] * BYTES[c["dtype"]]
        table = kept * (8 + 4 * c["rot"]) if c["rot"] else 0
        zeros = 2 * (c["tokens"] - kept) * c["heads"] * (c["dim"] * BYTES[c["dtype"]] + 4)
        return {"bytes": both + rows * (c["dim"] + 8) + 8 * c["tokens"] + table + zeros, "flops": 6 * rows * c["dim"]}
    n = _lengths(c)
    seen = sum(min(v, c["window"]) if c["window"] else v for v in n)
    scales = 8 if c["cache"] in QMAX else 0
    q = c["batch"] * c["q_heads"]
    return {"bytes": seen * c["kv_heads"] * (2 * c["dim"] * BYTES[c["cache"]] + scales)
            + q * (2 * c["dim"] * BYTES[c["dtype"]] + 4) + c["batch"] * 4 + 4 * (seen // c["page"]),
            "flops": 4 * seen * c["q_heads"] * c["dim"]}


# ------------------------------------------------------------------------------- the inputs

def _kept(tokens, skip):
    """The tokens that have a place in the cache: all but each `skip`-th."""
    return [t for t in range(tokens) if not (skip and t % skip == skip - 1)]


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(shape, dtype, g, spread=True):
    """Normal values; with `spread`, a few channels are much larger than the rest, as activations are."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if spread:
        x *= 1.0 + 7.0 * (torch.rand(shape[-1], generator=g, device="cuda") < 0.03)
    return x.to(TORCH[dtype])


def _frequencies(rot, scaling, factor, original=8192.0, base=10000.0):
    """Angle per position of each pair (64 bits), and the factor on the rotation: `parts` divides the
    frequencies of few turns over the original context by `factor` and leaves those of many."""
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "parts":
        keep = ((original * f / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _table(count, rot, scaling="none", factor=1.0):
    f, m = _frequencies(rot, scaling, factor)
    a = torch.arange(count, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack([a.cos() * m, a.sin() * m], -1).float().contiguous()


def _pages(kept, count, g):
    return torch.randperm(count, generator=g, device="cuda")[:kept]


def _slots(c, g):
    """A slot of the cache for each token, in pages of a scattered order; -1 for a token not kept."""
    kept = torch.tensor(_kept(c["tokens"], c["skip"]), device="cuda")
    need = -(-len(kept) // c["page"])
    count = need + 1 + need // 8
    page = _pages(need, count, g)
    at = torch.arange(len(kept), device="cuda")
    slots = torch.full((c["tokens"],), -1, dtype=torch.int64, device="cuda")
    slots[kept] = page[at // c["page"]] * c["page"] + at % c["page"]
    return slots, count


def _attn_inputs(c, seed):
    g = _gen(seed)
    n, ps = _lengths(c), c["page"]
    width = max(1, -(-c["length"] // ps))
    need = [-(-v // ps) for v in n]
    count = sum(need) + 1 + sum(need) // 16
    ids = _pages(sum(need), count, g)
    table = torch.full((c["batch"], width), -1, dtype=torch.int32, device="cuda")
    lens = torch.tensor(n, dtype=torch.int32, device="cuda")
    taken = torch.arange(width, device="cuda")[None] < torch.tensor(need, device="cuda")[:, None]
    table[taken] = ids.to(torch.int32)
    shape = (count, c["kv_heads"], ps, c["dim"])
    s = {"q": _randn((c["batch"], c["q_heads"], c["dim"]), c["dtype"], g, spread=False) * 2, "table": table, "lens": lens}
    for w in ("k", "v"):
        if c["cache"] in QMAX:
            if c["cache"] == "i8":
                x = torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8)
            else:
                x = (torch.randn(shape, generator=g, device="cuda", dtype=torch.float16) * 100).clamp_(-448, 448).to(TORCH["e4m3"])
            s[w + "_scale"] = torch.rand(shape[:3], generator=g, device="cuda") * 0.01 + (0.01 if c["cache"] == "i8" else 0.004)
        else:
            x = torch.randn(shape, generator=g, device="cuda", dtype=TORCH[c["cache"]])
            # what the last pages hold past a sequence's end was never written
            at = torch.arange(width * ps, device="cuda").view(1, width, ps)
            past = (at >= lens[:, None, None]) & taken[:, :, None]
            b, p, o = past.nonzero(as_tuple=True)
            x[table[b, p].long(), :, o] = float("nan")
        s[w] = x
    return s


def _rope_inputs(c, seed):
    g = _gen(seed)
    pos = torch.arange(c["tokens"], device="cuda") + c["start"]
    pos = pos[torch.randperm(c["tokens"], generator=g, device="cuda")] if seed % 2 else pos
    return {"x": _randn((c["tokens"], c["heads"], c["dim"]), c["dtype"], g), "pos": pos}


def _cache_inputs(c, seed):
    g = _gen(seed)
    shape = (c["tokens"], c["heads"], c["dim"])
    slots, count = _slots(c, g)
    start = int(seed) % 1000
    return {"k": _randn(shape, c["dtype"], g), "v": _randn(shape, c["dtype"], g), "slots": slots, "pages": count,
            "pos": torch.arange(c["tokens"], device="cuda") + start}


def prepare(case, seed):
    c = case
    if c["op"] == "rope":
        s = _rope_inputs(c, seed)
        s["cos_sin"] = _table(c["start"] + c["tokens"], c["rot"], c["scaling"], c["factor"])
    elif c["op"] == "cache":
        s = _cache_inputs(c, seed)
        shape = (s["pages"], c["heads"], c["page"], c["dim"])
        s["cos_sin"] = _table(c["tokens"] + 1000, c["rot"]) if c["rot"] else None
        for w in ("k", "v"):
            s["cache_" + w] = torch.zeros(shape, dtype=torch.int8, device="cuda").view(TORCH[c["cache"]])
            s["cache_" + w + "_scale"] = torch.zeros(shape[:3], device="cuda")
        if own:
            s["cache"] = _gar().KVCache(s["cache_k"], s["cache_v"], s["cache_k_scale"], s["cache_v_scale"])
    else:
        s = _attn_inputs(c, seed)
        if own:
            s["cache"] = _gar().KVCache(s["k"], s["v"], s.get("k_scale"), s.get("v_scale"))
            s["plan"] = _gar().gar_attn_plan_create(c["q_heads"], c["kv_heads"], c["dim"])
    s["case"] = c
    return s


# ------------------------------------------------------------------------------- the passes

def _turn(x, cos_sin, rot, layout, inverse):
    """The rotation of x's first `rot` channels, in 32 bits."""
    c, n = cos_sin[:, None, :, 0], cos_sin[:, None, :, 1]
    n = -n if inverse else n
    x = x.float()
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if layout == "half" else (x[..., 0:rot:2], x[..., 1:rot:2])
    y, z = a * c - b * n, b * c + a * n
    turned = torch.cat([y, z], -1) if layout == "half" else torch.stack([y, z], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _codes(x, cache):
    """8-bit codes of x (as 32-bit numbers) and the scale of each row."""
    scale = x.abs().amax(-1) / QMAX[cache]
    y = x / torch.where(scale > 0, scale, 1.0)[..., None]
    y = y.clamp(-QMAX[cache], QMAX[cache])
    return (y.round() if cache == "i8" else y).to(TORCH[cache]), scale


def _plain_cache(s):
    c, ps = s["case"], s["case"]["page"]
    slots = s["slots"]
    kept = slots >= 0
    page, at = slots[kept] // ps, slots[kept] % ps
    back = []
    for w in ("k", "v"):
        x = s[w][kept].float()
        if w == "k" and c["rot"]:
            x = _turn(x, s["cos_sin"][s["pos"][kept]], c["rot"], c["layout"], False)
        code, scale = _codes(x, c["cache"])
        s["cache_" + w].view(torch.uint8)[page, :, at] = code.view(torch.uint8)
        s["cache_" + w + "_scale"][page, :, at] = scale
    for w in ("k", "v"):
        there = slots.clamp(min=0)
        x = s["cache_" + w].view(torch.uint8)[there // ps, :, there % ps].view(TORCH[c["cache"]]).float()
        scale = torch.where(kept[:, None], s["cache_" + w + "_scale"][there // ps, :, there % ps], 0.0)
        back.append((x * scale[..., None]).to(TORCH[c["dtype"]]))
    return {"k": back[0], "v": back[1], "k_scale": s["cache_k_scale"], "v_scale": s["cache_v_scale"]}


def _plain_attn(s):
    c = s["case"]
    b, hq, d = s["q"].shape
    hk, ps = c["kv_heads"], c["page"]
    ids = s["table"].long().clamp(min=0)
    lens = s["lens"].long()[:, None]
    at = torch.arange(ids.shape[1] * ps, device="cuda")[None]
    seen = (at < lens) & ((at >= lens - c["window"]) if c["window"] else (at >= 0))

    def whole(w):
        x = s[w].view(torch.uint8)[ids].view(s[w].dtype).float() if c["cache"] in QMAX else s[w][ids].float()
        if c["cache"] in QMAX:
            x = x * s[w + "_scale"][ids][..., None]
        x = x.transpose(1, 2).reshape(b, hk, -1, d)
        return torch.where(seen[:, None, :, None], x, 0.0)

    q = s["q"].float().view(b, hk, hq // hk, d)
    y = torch.matmul(q, whole("k").transpose(-1, -2)) * (1.0 / math.sqrt(d))
    y = torch.where(seen[:, None, None], y, -math.inf)
    m = y.amax(-1, keepdim=True)
    p = torch.exp(y - torch.where(m == -math.inf, 0.0, m))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, whole("v")) / torch.where(total == 0, 1.0, total)
    lse = torch.log(total) + m
    return {"out": out.reshape(b, hq, d).to(s["q"].dtype), "lse": lse.reshape(b, hq)}


def run(state):
    s, c = state, state["case"]
    if c["op"] == "rope":
        if own:
            return _gar().gar_rope(s["x"], s["pos"], s["cos_sin"], c["layout"], c["inverse"])
        return _turn(s["x"], s["cos_sin"][s["pos"]], c["rot"], c["layout"], c["inverse"]).to(s["x"].dtype)
    if c["op"] == "cache":
        if own:
            gar = _gar()
            rotate = (s["pos"], s["cos_sin"], c["layout"]) if c["rot"] else ()
            gar.gar_kv_write(s["cache"], s["k"], s["v"], s["slots"], *rotate)
            k, v = gar.gar_kv_read(s["cache"], s["slots"], c["dtype"])
            return {"k": k, "v": v, "k_scale": s["cache_k_scale"], "v_scale": s["cache_v_scale"]}
        return _plain_cache(s)
    if own:
        out, lse = _gar().gar_decode_attention(s["plan"], s["q"], s["cache"], s["table"], s["lens"],
                                               window=c["window"], lse=True)
        return {"out": out, "lse": lse}
    return _plain_attn(s)


# ------------------------------------------------------------------------------- 64 bits

def _exact_turn(x, pos, rot, layout, inverse, scaling="none", factor=1.0):
    """The rotation as a product of complex numbers."""
    f, m = _frequencies(rot, scaling, factor)
    a = pos.double()[:, None, None] * f
    r = torch.polar(torch.full_like(a, m), -a if inverse else a)
    x = x.double()
    if layout == "half":
        z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * r
        return torch.cat([z.real, z.imag, x[..., rot:]], -1)
    z = torch.view_as_complex(x[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * r
    return torch.cat([torch.view_as_real(z).flatten(-2), x[..., rot:]], -1)


def _exact_cache(c, seed):
    s = _cache_inputs(c, seed)
    kept = s["slots"] >= 0
    where = s["slots"][kept]
    got = {}
    for w in ("k", "v"):
        x = s[w].double()
        if w == "k" and c["rot"]:
            x = _exact_turn(x, s["pos"], c["rot"], c["layout"], False)
        scale = (x.abs().amax(-1) / QMAX[c["cache"]]).float().double()  # the format holds it in 32 bits
        y = x / scale.clamp(min=1e-300)[..., None]
        if c["cache"] == "i8":
            y = y.round()
        else:  # 3 bits after the leading one, no exponent under -6
            step = torch.exp2(torch.frexp(y)[1].clamp(min=-5).double() - 4)
            y = ((y / step).round() * step).clamp(-448, 448)
        got[w] = torch.where(kept[:, None, None], y * scale[..., None], 0.0)
        full = torch.zeros((s["pages"] * c["page"], c["heads"]), dtype=torch.float64, device="cuda")
        full[where] = scale[kept]
        got[w + "_scale"] = full.view(s["pages"], c["page"], c["heads"]).transpose(1, 2).contiguous()
    return {n: got[n] for n in ("k", "v", "k_scale", "v_scale")}


def _exact_attn(c, seed):
    s = _attn_inputs(c, seed)
    hk, d, ps = c["kv_heads"], c["dim"], c["page"]
    group = c["q_heads"] // hk
    out = torch.zeros((c["batch"], c["q_heads"], d), dtype=torch.float64, device="cuda")
    lse = torch.full((c["batch"], c["q_heads"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(c)):
        first = max(0, n - c["window"]) if c["window"] else 0
        if n == first:
            continue
        ids = s["table"][b, first // ps:-(-n // ps)].long()
        cut = slice(first % ps, first % ps + n - first)
        kv = []
        for w in ("k", "v"):
            x = s[w].view(torch.uint8)[ids].view(s[w].dtype).double() if c["cache"] in QMAX else s[w][ids].double()
            if c["cache"] in QMAX:
                x = x * s[w + "_scale"][ids].double()[..., None]
            kv.append(x.permute(1, 0, 2, 3).flatten(1, 2)[:, cut])
        y = torch.einsum("hgd,hnd->hgn", s["q"][b].double().view(hk, group, d), kv[0]) / math.sqrt(d)
        lse[b] = torch.logsumexp(y, -1).flatten()
        out[b] = torch.einsum("hgn,hnd->hgd", torch.softmax(y, -1), kv[1]).reshape(-1, d)
    return {"out": out, "lse": lse}


def exact(case, seed):
    c = case
    if c["op"] == "rope":
        s = _rope_inputs(c, seed)
        return _exact_turn(s["x"], s["pos"], c["rot"], c["layout"], c["inverse"], c["scaling"], c["factor"])
    return _exact_cache(c, seed) if c["op"] == "cache" else _exact_attn(c, seed)
