"""The operators of a latent-attention layer around its paged cache, as measurable cases.

Five operators that a serving step of a model with one shared latent row a token
runs around splash_mla_attend, or, for a prompt, in its place:
  append   norm of the new tokens' latents, rotary turn of their shared keys, and
           the write into the paged cache in the cache's format (splash_mla_append)
  gather   the histories of a few requests read back from the cache into dense
           bf16 rows (splash_mla_gather)
  absorb   query heads taken through the key up-projection, rotary part turned:
           the attention's packed query rows (splash_mla_absorb_q)
  expand   the attention's latent outputs taken through the value up-projection
           (splash_mla_expand_out)
  prefill  causal attention of ragged prompts over expanded keys and values
           (splash_mla_prefill)

`run` computes the operators in elementary torch operations, or, where `own` is
true, calls the library; `exact` follows the definitions in float64.  Lengths are
drawn from the case's own `lengths_seed` (a case has one amount of work) and
dealt to the requests in an order made from the seed of `prepare`.
"""
import math
import random

import torch

own = False

PAGE = 64
LATENT, ROPE, NOPE, VALUE = 512, 64, 128, 128
ROW_BYTES = {"bf16": 1152, "e4m3": 580, "latent": 656}   # a cached row and its scale
TOP = 448.0
EPS = 1e-6
SCALE = 1.0 / math.sqrt(NOPE + ROPE)


def _append(batch, new_lo, new_hi, fmt, norm, interleaved, before, far, seed):
    return {"kind": "append", "batch": batch, "new_lo": new_lo, "new_hi": new_hi, "format": fmt, "norm": norm,
            "interleaved": interleaved, "before": before, "far": far, "lengths_seed": seed}


def _gather(batch, lo, hi, fmt, seed):
    return {"kind": "gather", "batch": batch, "lo": lo, "hi": hi, "format": fmt, "lengths_seed": seed}


def _absorb(tokens, heads, interleaved, far):
    return {"kind": "absorb", "tokens": tokens, "heads": heads, "interleaved": interleaved, "far": far}


def _expand(tokens, heads):
    return {"kind": "expand", "tokens": tokens, "heads": heads}


def _prefill(batch, heads, new_lo, new_hi, old_lo, old_hi, lengths, seed):
    return {"kind": "prefill", "batch": batch, "heads": heads, "new_lo": new_lo, "new_hi": new_hi, "old_lo": old_lo,
            "old_hi": old_hi, "lengths": lengths, "lengths_seed": seed}


def listed():
    return [
        # one new token for every request of a decode batch
        dict(_append(256, 1, 1, "latent", True, True, 1536, 131072, 1), name="append_decode"),
        # the prompts of a few new requests and the next pieces of others
        dict(_append(16, 256, 1024, "e4m3", True, False, 1536, 32768, 2), name="append_prompts"),
        # one short history, read back before a prompt's next piece
        dict(_gather(1, 1000, 1000, "bf16", 0), name="gather_short"),
        # a few long histories of 8-bit rows, for the pieces that follow them
        dict(_gather(6, 4096, 16384, "latent", 3), name="gather_long"),
        # a few decoding requests on a rank that holds some of the heads
        dict(_absorb(4, 20, True, 4096), name="absorb_few"),
        # a large decode batch with all heads on its owner
        dict(_absorb(256, 128, True, 131072), name="absorb_decode"),
        dict(_expand(4, 20), name="expand_few"),
        dict(_expand(256, 128), name="expand_decode"),
        # short prompts on a rank with few heads: launches and latency
        dict(_prefill(4, 8, 16, 200, 0, 0, "uniform", 4), name="prefill_tiny"),
        # one long prompt with all heads
        dict(_prefill(1, 128, 4096, 4096, 0, 0, "uniform", 0), name="prefill_prompt"),
        # prompts of very different lengths on a rank with a quarter of the heads
        dict(_prefill(8, 32, 1, 4096, 0, 1, "lognormal", 9), name="prefill_ragged"),
        # the next pieces of two long prompts, over their histories
        dict(_prefill(2, 20, 300, 512, 8192, 20000, "uniform", 6), name="prefill_pieces"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above, sizes over their logarithm."""
    kind = rng.choices(["append", "gather", "absorb", "expand", "prefill"], [18, 16, 18, 13, 35])[0]
    seed = rng.randrange(1 << 30)
    fmt = rng.choice(["bf16", "e4m3", "latent"])
    if kind == "append":
        new_hi = rng.choice([1, rng.randrange(2, 9), _log_int(rng, 16, 2048)])
        batch = _log_int(rng, 1, 1024 if new_hi <= 8 else max(1, 10000 // new_hi))
        return _append(batch, rng.choice([0, 1, new_hi]), new_hi, fmt, rng.random() < 0.75, rng.random() < 0.5,
                       rng.choice([0, 512, 1536]), _log_int(rng, 64, 1 << 20), seed)
    if kind == "gather":
        batch, hi = _log_int(rng, 1, 64), _log_int(rng, 1, 32768)
        while batch * hi > 6 * 16384:
            batch, hi = max(1, batch // 2), max(1, hi // 2)
        return _gather(batch, rng.choice([0, 1, hi]), hi, fmt, seed)
    if kind in ("absorb", "expand"):
        heads = rng.choice([1, 4, 8, 20, 32, 64, 128, rng.randrange(1, 129)])
        tokens = _log_int(rng, 1, max(2, min(4096, 40000 // heads)))
        if kind == "expand":
            return _expand(tokens, heads)
        return _absorb(tokens, heads, rng.random() < 0.5, _log_int(rng, 64, 1 << 20))
    heads = rng.choice([1, 4, 8, 20, 32, 64, 128, rng.randrange(1, 129)])
    lengths = rng.choice(["uniform", "lognormal"])
    new_hi = rng.choice([_log_int(rng, 1, 64), _log_int(rng, 16, 4096), _log_int(rng, 256, 8192)])
    new_lo = rng.choice([0, 1, new_hi])
    old_hi = rng.choice([0, 0, _log_int(rng, 1, 32768)])
    old_lo = old_hi // rng.randrange(1, 9)
    batch = _log_int(rng, 1, 64)
    while True:
        case = _prefill(batch, heads, min(new_lo, new_hi), new_hi, old_lo, old_hi, lengths, seed)
        # no dearer than the listed ones, the plain form's padded rows among them
        if work(case)["flops"] <= 5.0e11 and batch * heads * new_hi * (new_hi + old_hi) <= 1.8e9:
            return case
        if batch > 1:
            batch //= 2
        else:
            old_lo, old_hi, new_hi = old_lo // 2, old_hi // 2, max(1, new_hi * 3 // 4)


# ---------------------------------------------------------------- sizes --

def _new_lengths(case):
    """The step's new tokens of each request, the longest of them as long as the case says."""
    rng = random.Random(case["lengths_seed"] + 1)
    lo, hi = case["new_lo"], case["new_hi"]
    if case.get("lengths") == "lognormal":
        mid = max(lo, hi / 6, 1)
        n = [min(max(round(mid * rng.lognormvariate(0.0, 1.0)), lo), hi) for _ in range(case["batch"])]
    else:
        n = [rng.randint(lo, hi) for _ in range(case["batch"])]
    n[-1] = hi
    return n


def _old_lengths(case):
    """Tokens before the new ones (a cached history) of each request."""
    rng = random.Random(case["lengths_seed"])
    lo, hi = (case["old_lo"], case["old_hi"]) if case["kind"] == "prefill" else (0, case.get("far", PAGE))
    return [rng.randint(lo, hi) for _ in range(case["batch"])]


def _lengths(case):
    """Rows of each history that is read back, the longest as long as the case says."""
    rng = random.Random(case["lengths_seed"])
    n = [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]
    n[-1] = case["hi"]
    return n


def _pages(n):
    return -(-n // PAGE)


def work(case):
    if case["kind"] == "append":
        n = sum(_new_lengths(case))
        # bf16 rows in, cached rows out, slot and position; the norm's weight
        return {"bytes": n * (1152 + ROW_BYTES[case["format"]] + 8) + (1024 if case["norm"] else 0),
                "flops": n * (4 * LATENT + 3 * ROPE)}
    if case["kind"] == "gather":
        n = sum(_lengths(case))
        return {"bytes": n * (ROW_BYTES[case["format"]] + 1152) + 4 * sum(_pages(s) for s in _lengths(case)),
                "flops": 0 if case["format"] == "bf16" else n * LATENT}
    if case["kind"] == "absorb":
        rows = case["tokens"] * case["heads"]
        return {"bytes": rows * 2 * (NOPE + ROPE + LATENT + ROPE) + case["heads"] * 2 * NOPE * LATENT + 4 * case["tokens"],
                "flops": rows * (2 * NOPE * LATENT + 3 * ROPE)}
    if case["kind"] == "expand":
        rows = case["tokens"] * case["heads"]
        return {"bytes": rows * 2 * (LATENT + VALUE) + case["heads"] * 2 * VALUE * LATENT, "flops": rows * 2 * VALUE * LATENT}
    h, new, old = case["heads"], _new_lengths(case), _old_lengths(case)
    rows, keys = sum(new), sum(new) + sum(old)
    visible = sum(n * o + n * (n + 1) // 2 for n, o in zip(new, old))
    return {"bytes": rows * h * (2 * (NOPE + ROPE) + 2 * VALUE + 4) + keys * (2 * h * (NOPE + VALUE) + 2 * ROPE),
            "flops": 2 * h * (NOPE + ROPE + VALUE) * visible}


# --------------------------------------------------------------- inputs --

def _encode(rows, fmt):
    """Rows [..., 576] in fp32 to the pool's bytes and per-row scales: the cache's formats, each value rounded once."""
    if fmt == "bf16":
        return rows.bfloat16(), None
    if fmt == "e4m3":
        amax = rows.abs().amax(-1)
        scale = torch.where(amax > 0, (amax / TOP).clamp(min=2.0 ** -126), 1.0)
        return (rows / scale[..., None]).clamp(-TOP, TOP).to(torch.float8_e4m3fn).view(torch.uint8), scale
    tiles = rows[..., :LATENT].unflatten(-1, (4, 128))
    # the least power of two that holds the tile's largest magnitude in the codes' range
    m, e = torch.frexp(tiles.abs().amax(-1) / TOP)
    e = torch.where(m == 0, 0, torch.where(m > 0.5, e, e - 1).clamp(-126, 63))
    scale = torch.ldexp(torch.ones_like(m), e)
    out = torch.empty((*rows.shape[:-1], 656), dtype=torch.uint8, device=rows.device)
    out[..., :LATENT] = torch.ldexp(tiles, -e[..., None]).clamp(-TOP, TOP).to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2)
    out[..., LATENT:528] = scale.view(torch.uint8).reshape(*rows.shape[:-1], 16)
    out[..., 528:] = rows[..., LATENT:].bfloat16().view(torch.uint8)
    return out, None


def _decode(pool, scales, fmt):
    """The pool's rows in fp32."""
    if fmt == "bf16":
        return pool.float()
    if fmt == "e4m3":
        return pool.view(torch.float8_e4m3fn).float() * scales[..., None]
    codes = pool[..., :LATENT].view(torch.float8_e4m3fn).float().unflatten(-1, (4, 128))
    return torch.cat([(codes * pool.view(torch.float32)[..., 128:132][..., None]).flatten(-2),
                      pool.view(torch.bfloat16)[..., 264:].float()], -1)


def _pool(gen, pages, fmt):
    """Pages of N(0, 1) rows, their latent's quarters times powers of two of their own."""
    pool = torch.empty((pages, PAGE, 656 if fmt == "latent" else 576), device="cuda",
                       dtype=torch.bfloat16 if fmt == "bf16" else torch.uint8)
    scales = torch.empty((pages, PAGE), device="cuda") if fmt == "e4m3" else None
    for p in range(0, pages, 512):
        n = min(512, pages - p)
        x = torch.randn((n, PAGE, 576), generator=gen, device="cuda")
        x[..., :LATENT].unflatten(-1, (4, 128)).mul_(
            torch.exp2(torch.randint(-3, 1, (n, PAGE, 4, 1), generator=gen, device="cuda").float()))
        rows, s = _encode(x, fmt)
        pool[p:p + n] = rows
        if s is not None:
            scales[p:p + n] = s
    return pool, scales


def _ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def _indptr(n):
    at = [0]
    for k in n:
        at.append(at[-1] + k)
    return _ints(at)


def _frequencies():
    return [10000.0 ** (-2.0 * j / ROPE) for j in range(ROPE // 2)]


def _shuffled(seed, *lists):
    both = list(zip(*lists))
    random.Random(seed).shuffle(both)
    return [list(x) for x in zip(*both)]


def _table(gen, held, pages):
    """A block table whose request b holds held[b] pages of the pool."""
    perm = torch.randperm(pages, generator=gen, device="cuda").int().cpu()
    table, off = torch.full((len(held), max(1, max(held))), -1, dtype=torch.int32), 0
    for b, n in enumerate(held):
        table[b, :n] = perm[off:off + n]
        off += n
    return table


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def turned(st):
        st["inv_freq"] = torch.tensor(_frequencies(), dtype=torch.float64).cuda()
        if own:
            from paper_2609_37626_amd import binding as B
            st["rope"] = B.make_rope(ROPE, _frequencies(), interleaved=case["interleaved"])

    st = {"case": case}
    if case["kind"] == "append":
        old, new = _shuffled(seed, _old_lengths(case), _new_lengths(case))
        first = [o // PAGE for o in old]
        held = [_pages(o + n) - f if n else 0 for o, n, f in zip(old, new, first)]
        pages = sum(held) + 5
        table = _table(gen, held, pages)
        st["slots"] = _ints([int(table[b, p // PAGE - f]) * PAGE + p % PAGE
                             for b, (o, n, f) in enumerate(zip(old, new, first)) for p in range(o, o + n)])
        st["positions"] = _ints([p for o, n in zip(old, new) for p in range(o, o + n)])
        st["pool"], st["scales"] = _pool(gen, pages, case["format"])
        # the fused down-projection's rows: the query's latent, the token's latent, its shared rotary key
        rows = randn(sum(new), case["before"] + 576).mul_(torch.exp2(randn(sum(new), 1))).bfloat16()
        st["latent"], st["key"] = rows[:, case["before"]:case["before"] + LATENT], rows[:, case["before"] + LATENT:]
        st["weight"] = (1.0 + 0.1 * randn(LATENT)).bfloat16() if case["norm"] else None
        turned(st)
        if own:
            from paper_2609_37626_amd import binding as B
            st["desc"] = B.make_desc(len(new), 128, max(1, max(held)), pages, _code(case), st["scales"])
        return st
    if case["kind"] == "gather":
        lens, = _shuffled(seed, _lengths(case))
        pages = max(1, sum(_pages(s) for s in lens))
        st["table"] = _table(gen, [_pages(s) for s in lens], pages).cuda()
        st["indptr"] = _indptr(lens)
        st["pool"], st["scales"] = _pool(gen, pages, case["format"])
        st["latent"] = torch.empty((sum(lens), LATENT), dtype=torch.bfloat16, device="cuda")
        st["key"] = torch.empty((sum(lens), ROPE), dtype=torch.bfloat16, device="cuda")
        if own:
            from paper_2609_37626_amd import binding as B
            st["desc"] = B.make_desc(len(lens), 128, int(st["table"].shape[1]), pages, _code(case), st["scales"])
        return st
    if case["kind"] in ("absorb", "expand"):
        n, h = case["tokens"], case["heads"]
        # the up-projection as it stands in a model: each head's key rows, then its value rows
        w = (randn(h, NOPE + VALUE, LATENT) / math.sqrt(LATENT)).bfloat16()
        if case["kind"] == "absorb":
            st["weight"] = w[:, :NOPE]
            st["q"] = randn(n, h, NOPE + ROPE).bfloat16()
            st["positions"] = torch.randint(0, case["far"], (n,), generator=gen, device="cuda", dtype=torch.int32)
            st["out"] = torch.empty((n, h, LATENT + ROPE), dtype=torch.bfloat16, device="cuda")
            turned(st)
        else:
            st["weight"] = w[:, NOPE:]
            st["o"] = randn(n, h, LATENT).bfloat16()
            st["out"] = torch.empty((n, h, VALUE), dtype=torch.bfloat16, device="cuda")
        return st
    h = case["heads"]
    old, new = _shuffled(seed, _old_lengths(case), _new_lengths(case))
    rows, keys = sum(new), sum(new) + sum(old)
    st["q_indptr"], st["kv_indptr"] = _indptr(new), _indptr([o + n for o, n in zip(old, new)])
    st["longest"] = max(new), max(o + n for o, n in zip(old, new))
    st["q"] = randn(rows, h, NOPE + ROPE).bfloat16()
    # the up-projection's rows: each head's keys and values side by side
    kv = torch.empty((keys, h, NOPE + VALUE), dtype=torch.bfloat16, device="cuda")
    for at in range(0, keys, 4096):
        kv[at:at + 4096] = randn(min(4096, keys - at), h, NOPE + VALUE)
    st["k"], st["v"] = kv[..., :NOPE], kv[..., NOPE:]
    st["key"] = randn(keys, ROPE).bfloat16()
    st["out"] = torch.empty((rows, h, VALUE), dtype=torch.bfloat16, device="cuda")
    st["lse"] = torch.empty((rows, h), dtype=torch.float32, device="cuda")
    if own:
        from paper_2609_37626_amd import binding as B
        st["ws"] = torch.empty(B.mla_prefill_workspace_size(case["batch"], rows, h), dtype=torch.uint8, device="cuda")
    return st


def _code(case):
    from paper_2609_37626_amd import binding as B
    return {"bf16": B.KV_BF16, "e4m3": B.KV_FP8_E4M3, "latent": B.KV_FP8_LATENT}[case["format"]]


# ----------------------------------------------------------- plain forms --

def _turn(x, positions, inv_freq, interleaved):
    """x [tokens, ..., 64] in fp32, turned; far positions' angles need 64 bits."""
    angle = positions.double()[:, None] * inv_freq
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if x.dim() == 3:
        cos, sin = cos[:, None], sin[:, None]
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    a, b = x[..., :ROPE // 2], x[..., ROPE // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _plain_append(st):
    case, x = st["case"], st["latent"].double()
    if st["weight"] is not None:      # 64 bits: a value next to a scale's border decides the scale
        x = x * st["weight"].double() / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + EPS)
    rows = torch.cat([x.float(), _turn(st["key"].float(), st["positions"], st["inv_freq"], case["interleaved"])], -1)
    rows, scales = _encode(rows, case["format"])
    at = st["slots"].long()
    st["pool"].flatten(0, 1)[at] = rows
    if scales is not None:
        st["scales"].flatten()[at] = scales


def _plain_gather(st):
    n = st["latent"].shape[0]
    row = torch.arange(n, device="cuda")
    b = torch.searchsorted(st["indptr"][1:].long(), row, right=True)
    at = row - st["indptr"].long()[b]
    page = st["table"].long()[b, at // PAGE]
    scales = None if st["scales"] is None else st["scales"].flatten()[page * PAGE + at % PAGE]
    x = _decode(st["pool"].flatten(0, 1)[page * PAGE + at % PAGE], scales, st["case"]["format"])
    st["latent"].copy_(x[:, :LATENT])
    st["key"].copy_(x[:, LATENT:])


def _plain_absorb(st):
    q = st["q"].float()
    x = torch.bmm(q[..., :NOPE].transpose(0, 1).contiguous(), st["weight"].float())
    st["out"][..., :LATENT].copy_(x.transpose(0, 1))
    st["out"][..., LATENT:].copy_(_turn(q[..., NOPE:], st["positions"], st["inv_freq"], st["case"]["interleaved"]))


def _plain_expand(st):
    x = torch.bmm(st["o"].float().transpose(0, 1).contiguous(), st["weight"].float().transpose(1, 2).contiguous())
    st["out"].copy_(x.transpose(0, 1))


def _plain_prefill(st):
    """Every request padded to the longest."""
    qi, ki = st["q_indptr"].long(), st["kv_indptr"].long()
    rows, keys = st["longest"]
    nq, nk = qi[1:] - qi[:-1], ki[1:] - ki[:-1]
    i, j = torch.arange(rows, device="cuda"), torch.arange(keys, device="cuda")
    b, h = nq.numel(), st["case"]["heads"]
    from_q = (qi[:-1, None] + i).clamp(max=st["q"].shape[0] - 1)
    from_k = (ki[:-1, None] + j).clamp(max=st["k"].shape[0] - 1)
    q = st["q"][from_q].float().transpose(1, 2).flatten(0, 1)                       # [b * h, rows, 192]
    k = torch.cat([st["k"][from_k], st["key"][from_k][:, :, None].expand(-1, -1, h, -1)], -1)
    k = k.permute(0, 2, 3, 1).flatten(0, 1).float().contiguous()                    # [b * h, 192, keys]
    z = torch.bmm(q, k).mul_(SCALE).unflatten(0, (b, h))
    del q, k
    hidden = (j > (nk - nq)[:, None, None] + i[:, None]) | (j >= nk[:, None, None])
    z.masked_fill_(hidden[:, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    w = z.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    v = st["v"][from_k].float().transpose(1, 2).flatten(0, 1)
    o = torch.bmm(w.flatten(0, 1), v).unflatten(0, (b, h)) / total.clamp(min=1e-37)
    lse = (top + torch.log(total)).squeeze(-1)
    real = (i < nq[:, None])
    st["out"].copy_(o.transpose(1, 2)[real])
    st["lse"].copy_(lse.transpose(1, 2)[real])


def run(st):
    case = st["case"]
    if own:
        from paper_2609_37626_amd import binding as B
        if case["kind"] == "append":
            B.splash_mla_append(st["latent"], st["key"], st["slots"], st["pool"], st["scales"], st["desc"],
                                norm_weight=st["weight"], norm_eps=EPS, positions=st["positions"], rope=st["rope"])
        elif case["kind"] == "gather":
            B.splash_mla_gather(st["pool"], st["table"], st["indptr"], st["latent"], st["key"], st["desc"])
        elif case["kind"] == "absorb":
            B.splash_mla_absorb_q(st["q"], st["weight"], st["out"], positions=st["positions"], rope=st["rope"])
        elif case["kind"] == "expand":
            B.splash_mla_expand_out(st["o"], st["weight"], st["out"])
        else:
            B.splash_mla_prefill(st["q"], st["k"], st["key"], st["v"], st["q_indptr"], st["kv_indptr"], st["out"], st["lse"],
                                 st["ws"], softmax_scale=SCALE)
    elif case["kind"] == "append":
        _plain_append(st)
    elif case["kind"] == "gather":
        _plain_gather(st)
    elif case["kind"] == "absorb":
        _plain_absorb(st)
    elif case["kind"] == "expand":
        _plain_expand(st)
    else:
        _plain_prefill(st)
    return _outputs(st)


def _outputs(st):
    case = st["case"]
    if case["kind"] == "append":
        if case["format"] == "bf16":
            return {"rows": st["pool"]}
        if case["format"] == "e4m3":
            return {"codes": st["pool"].view(torch.float8_e4m3fn), "scales": st["scales"]}
        return {"codes": st["pool"][..., :LATENT].view(torch.float8_e4m3fn),
                "scales": st["pool"].view(torch.float32)[..., 128:132], "key": st["pool"].view(torch.bfloat16)[..., 264:]}
    if case["kind"] == "gather":
        return {"latent": st["latent"], "key": st["key"]}
    if case["kind"] == "prefill":
        return {"out": st["out"], "lse": st["lse"]}
    return {"out": st["out"]}


# ------------------------------------------------------------ the result --

def _exact_turn(x, positions, interleaved):
    """Each pair as a complex number, turned by its position times its frequency."""
    y = x.double()
    pairs = y.unflatten(-1, (ROPE // 2, 2)) if interleaved else y.unflatten(-1, (2, ROPE // 2)).transpose(-1, -2)
    turn = torch.stack([positions.double() * f for f in _frequencies()], -1)
    turn = turn.reshape(turn.shape[0], *[1] * (x.dim() - 2), ROPE // 2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(turn), turn))
    return z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2)


def _exact_append(st):
    """The rows before their last rounding (codes: the values over the scale that they are rounded from)."""
    case, x = st["case"], st["latent"].double()
    if case["norm"]:
        x = x * torch.rsqrt((x * x).sum(-1, keepdim=True) / LATENT + EPS) * st["weight"].double()
    y = torch.cat([x, _exact_turn(st["key"], st["positions"], case["interleaved"])], -1)
    page, place = st["slots"].long() // PAGE, st["slots"].long() % PAGE
    if case["format"] == "bf16":
        rows = st["pool"].double()
        rows[page, place] = y
        return {"rows": rows}
    if case["format"] == "e4m3":
        codes, scales = st["pool"].view(torch.float8_e4m3fn).double(), st["scales"].double()
        scales[page, place] = y.abs().max(-1).values / TOP
        codes[page, place] = y / scales[page, place][:, None]
        return {"codes": codes, "scales": scales}
    codes = st["pool"][..., :LATENT].view(torch.float8_e4m3fn).double()
    scales, key = st["pool"].view(torch.float32)[..., 128:132].double(), st["pool"].view(torch.bfloat16)[..., 264:].double()
    tiles = y[:, :LATENT].reshape(-1, 4, 128)
    new = torch.exp2(torch.ceil(torch.log2(tiles.abs().amax(-1) / TOP)))
    scales[page, place] = new
    codes[page, place] = (tiles / new[..., None]).reshape(-1, LATENT)
    key[page, place] = y[:, LATENT:]
    return {"codes": codes, "scales": scales, "key": key}


def _exact_gather(st):
    latent, key = [], []
    at = st["indptr"].tolist()
    for b in range(len(at) - 1):
        n = at[b + 1] - at[b]
        pages = st["table"][b, :_pages(n)].long()
        x = st["pool"][pages]
        if st["case"]["format"] == "bf16":
            rows = x.double()
        elif st["case"]["format"] == "e4m3":
            rows = x.view(torch.float8_e4m3fn).double() * st["scales"][pages].double()[..., None]
        else:
            rows = torch.cat([x[..., 128 * t:128 * t + 128].view(torch.float8_e4m3fn).double()
                              * x.view(torch.float32)[..., 128 + t:129 + t].double() for t in range(4)]
                             + [x.view(torch.bfloat16)[..., 264:].double()], -1)
        rows = rows.reshape(-1, 576)[:n]
        latent.append(rows[:, :LATENT])
        key.append(rows[:, LATENT:])
    return {"latent": torch.cat(latent), "key": torch.cat(key)}


def _exact_prefill(st):
    out, lse = st["out"].double(), st["lse"].double()
    qi, ki = st["q_indptr"].tolist(), st["kv_indptr"].tolist()
    for b in range(len(qi) - 1):
        nq, nk = qi[b + 1] - qi[b], ki[b + 1] - ki[b]
        if nq == 0:
            continue
        hide = torch.ones((nq, nk), dtype=torch.bool, device="cuda").tril(nk - nq).logical_not()
        for h in range(st["case"]["heads"]):
            q, k = st["q"][qi[b]:qi[b + 1], h].double(), st["k"][ki[b]:ki[b + 1], h].double()
            z = q[:, :NOPE] @ k.T.contiguous() + q[:, NOPE:] @ st["key"][ki[b]:ki[b + 1]].double().T.contiguous()
            z = (z / math.sqrt(NOPE + ROPE)).masked_fill_(hide, -math.inf)
            lse[qi[b]:qi[b + 1], h] = torch.logsumexp(z, -1)
            out[qi[b]:qi[b + 1], h] = torch.softmax(z, -1) @ st["v"][ki[b]:ki[b + 1], h].double()
    return {"out": out, "lse": lse}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(st)
    if case["kind"] == "gather":
        return _exact_gather(st)
    if case["kind"] == "prefill":
        return _exact_prefill(st)
    x = (st["q"][..., :NOPE] if case["kind"] == "absorb" else st["o"]).double()
    w = st["weight"].double() if case["kind"] == "absorb" else st["weight"].double().transpose(1, 2)
    y = torch.empty((*x.shape[:2], w.shape[2]), dtype=torch.float64, device="cuda")
    for h in range(case["heads"]):
        y[:, h] = x[:, h] @ w[h].contiguous()
    if case["kind"] == "absorb":
        y = torch.cat([y, _exact_turn(st["q"][..., NOPE:], st["positions"], case["interleaved"])], -1)
    return {"out": y}
