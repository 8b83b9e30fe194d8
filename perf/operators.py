"""The operators of a serving step over an 8-bit paged K/V cache, as measurable cases.

Four operators that one decode or prefill step runs one after the other:
  tables  block table, slot map and positions of the step's new tokens, built on
          the GPU from the requests' lengths (splash_step_tables)
  rope    rotary positions with up to four axes, queries and keys in one call
          (splash_rope)
  append  the new K and V rows into a cache of 8-bit codes, with one power-of-two
          scale for each 64-token block and KV head (splash_gqa_append)
  attend  attention of the step's query rows over that cache (splash_gqa_attend)

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
TOP = {"e4m3": 448.0, "int8": 127.0}      # the largest magnitude of a code


def _attend(batch, heads, kv_heads, dim, q_chunk, code, lengths, lo, hi, seed):
    return {"kind": "attend", "batch": batch, "heads": heads, "kv_heads": kv_heads, "dim": dim, "q_chunk": q_chunk,
            "code": code, "lengths": lengths, "lo": lo, "hi": hi, "lengths_seed": seed}


def _append(batch, new_lo, new_hi, heads, kv_heads, dim, code, lo, hi, seed):
    return {"kind": "append", "batch": batch, "new_lo": new_lo, "new_hi": new_hi, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "code": code, "lo": lo, "hi": hi, "lengths_seed": seed}


def _rope(tokens, heads, kv_heads, rot, packed, sections, interleaved, far):
    return {"kind": "rope", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "rot": rot, "packed": packed,
            "sections": sections, "interleaved": interleaved, "far": far}


def _tables(batch, new_lo, new_hi, lo, hi, padding, seed):
    return {"kind": "tables", "batch": batch, "new_lo": new_lo, "new_hi": new_hi, "lo": lo, "hi": hi,
            "padding": padding, "lengths_seed": seed}


def listed():
    return [
        # a few short requests on a small model's rank: launches and latency
        dict(_attend(4, 16, 2, 64, 1, "e4m3", "uniform", 128, 512, 0), name="attend_tiny"),
        # a large decode batch of short requests, eight KV heads
        dict(_attend(256, 64, 8, 128, 1, "e4m3", "uniform", 1024, 4096, 1), name="attend_many_short"),
        # a few very long histories, split over the chip
        dict(_attend(4, 64, 8, 128, 1, "int8", "uniform", 65536, 131072, 2), name="attend_few_long"),
        # speculative decoding over a ragged batch, some of its places empty
        dict(_attend(64, 32, 4, 128, 4, "e4m3", "lognormal", 0, 32768, 3), name="attend_ragged_spec4"),
        # eight causal query tokens over wide heads: 64 query rows per KV head
        dict(_attend(16, 16, 2, 256, 8, "int8", "uniform", 8192, 32768, 4), name="attend_chunk8_wide"),
        # one new token for every request of a decode batch
        dict(_append(256, 1, 1, 64, 8, 128, "e4m3", 1024, 4096, 1), name="append_decode"),
        # the prompts of a few new requests and the next pieces of others
        dict(_append(16, 512, 2048, 32, 8, 128, "int8", 512, 4096, 5), name="append_prefill"),
        # the rotary part of packed latent-attention query rows and keys in a decode step
        dict(_rope(256, 128, 1, 64, 576, "32", True, 131072), name="rope_decode_packed"),
        # time, height and width positions of a prompt with images
        dict(_rope(16384, 32, 8, 128, 128, "16,24,24", False, 16384), name="rope_prefill_3axes"),
        # a decode step's tables
        dict(_tables(256, 1, 1, 1024, 4096, 0, 1), name="tables_decode"),
        # a prefill step's tables: prompts beside decoding requests, padded to the captured size
        dict(_tables(128, 0, 2048, 2048, 32768, 4096, 6), name="tables_prefill"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above, sizes over their logarithm."""
    kind = rng.choices(["attend", "append", "rope", "tables"], [50, 20, 18, 12])[0]
    seed = rng.randrange(1 << 30)
    if kind == "tables":
        hi = _log_int(rng, 64, 32768)
        new_hi = rng.choice([1, rng.randrange(2, 9), min(hi, _log_int(rng, 16, 2048))])
        batch = _log_int(rng, 1, 2048 if new_hi <= 8 else 128)
        return _tables(batch, rng.choice([0, 1]), new_hi, max(new_hi, hi // rng.randrange(1, 17)), max(hi, new_hi),
                       rng.choice([0, rng.randrange(1, 4096)]), seed)
    if kind == "rope":
        rot = rng.choice([32, 64, 80, 96, 128, 128])
        pairs = rot // 2
        axes = rng.choice([1, 1, 2, 3])
        cuts = sorted(rng.sample(range(1, pairs), axes - 1))
        sections = ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [pairs]))
        heads = rng.choice([1, 8, 12, 16, 32, 64, 128])
        most = int(16384 * 40 * 128 / (rot * (heads + 8)))
        return _rope(_log_int(rng, 1, max(2, most)), heads, rng.choice([1, 2, 4, 8]), rot, rot + rng.choice([0, 64, 512]),
                     sections, rng.random() < 0.5, _log_int(rng, 64, 1 << 20))
    kv_heads = rng.choice([1, 2, 4, 8])
    code = rng.choice(["e4m3", "int8"])
    dim = rng.choice([64, 128, 128, 256])
    heads = kv_heads * rng.choice([1, 2, 4, 8, 8, 16, rng.randrange(3, 16)])
    if kind == "append":
        new_hi = rng.choice([1, rng.randrange(2, 9), _log_int(rng, 16, 2048)])
        batch = _log_int(rng, 1, 1024 if new_hi <= 8 else 16)
        while batch * new_hi * kv_heads * dim > 16 * 1280 * 8 * 128:
            batch = max(1, batch // 2)
            new_hi = max(1, new_hi if batch > 1 else new_hi // 2)
        return _append(batch, rng.choice([0, 1, new_hi]), new_hi, heads, kv_heads, dim, code, new_hi,
                       new_hi + _log_int(rng, 1, 4096), seed)
    lengths = rng.choice(["uniform", "lognormal"])
    hi = _log_int(rng, 64, 131072)
    lo = rng.choice([0, 1, hi // rng.randrange(1, 17)])
    q = rng.choices([1, 2, rng.randrange(3, 9)], [55, 20, 25])[0]
    batch = _log_int(rng, 1, 256)
    while True:
        case = _attend(batch, heads, kv_heads, dim, q, code, lengths, lo, hi, seed)
        w = work(case)
        # no dearer than the listed ones, the plain form's padded rows among them
        if w["bytes"] <= 1.2e9 and w["flops"] <= 1.5e11 and batch * hi * kv_heads * dim <= 1.0e9:
            return case
        batch, hi = max(1, batch // 2), hi if batch > 1 else hi // 2
        lo = min(lo, hi)


# ---------------------------------------------------------------- sizes --

def _lengths(case):
    rng = random.Random(case["lengths_seed"])
    if case.get("lengths") == "lognormal":
        return [0 if case["lo"] == 0 and rng.random() < 0.05 else
                min(max(round(rng.lognormvariate(8.0, 1.5)), case["lo"]), case["hi"]) for _ in range(case["batch"])]
    return [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]


def _new_lengths(case):
    """The step's new tokens of each request, in the order of _lengths(), at most its length."""
    rng = random.Random(case["lengths_seed"] + 1)
    return [min(rng.randint(case["new_lo"], case["new_hi"]), s) for s in _lengths(case)]


def _sections(case):
    """Pairs of each position axis."""
    return [int(n) for n in case["sections"].split(",")]


def _pages(n):
    return -(-n // PAGE)


def work(case):
    if case["kind"] == "tables":
        lens, new = _lengths(case), _new_lengths(case)
        taken = sum(_pages(s) - _pages(s - n) for s, n in zip(lens, new))
        rows = sum(new) + case["padding"]
        # lengths in, offsets out; slot, position and request of each row; free
        # pages read and table entries written, the entries read of the pages
        # that were there
        return {"bytes": 4 * (3 * len(lens) + 3 * rows + 2 * taken + sum(n > 0 and (s - n) % PAGE > 0 for s, n in zip(lens, new))),
                "flops": 0}
    if case["kind"] == "rope":
        n = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["rot"]
        return {"bytes": 4 * n + 4 * case["tokens"] * len(_sections(case)), "flops": 3 * n}
    if case["kind"] == "append":
        tokens, hk, d = sum(_new_lengths(case)), case["kv_heads"], case["dim"]
        blocks = sum(_pages(s) - (s - n) // PAGE for s, n in zip(_lengths(case), _new_lengths(case)) if n)
        # bf16 rows in, codes out, one scale each way per block, head and side
        return {"bytes": 2 * tokens * hk * d * 3 + 2 * blocks * hk * 8 + 4 * tokens, "flops": 4 * tokens * hk * d}
    lens, q, h, hk, d = _lengths(case), case["q_chunk"], case["heads"], case["kv_heads"], case["dim"]
    visible = sum(max(0, s - q + i + 1) for s in lens for i in range(q))
    pages = sum(_pages(s) for s in lens)
    return {"bytes": sum(lens) * 2 * hk * d + pages * (8 * hk + 4) + len(lens) * q * h * (4 * d + 4) + 4 * len(lens),
            "flops": 4 * h * d * visible}


# --------------------------------------------------------------- inputs --

def _codes(gen, pages, kv_heads, dim, code):
    """Blocks of N(0, 1) values times a power of two of their own, in 8 bits: codes and scales."""
    codes = torch.empty((pages, kv_heads, PAGE, dim), dtype=torch.uint8 if code == "e4m3" else torch.int8, device="cuda")
    scales = torch.empty((pages, kv_heads), dtype=torch.float32, device="cuda")
    step = max(1, (1 << 28) // (kv_heads * PAGE * dim))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        x = torch.randn((n, kv_heads, PAGE, dim), generator=gen, device="cuda")
        x *= torch.exp2(torch.randint(-2, 2, (n, kv_heads, 1, 1), generator=gen, device="cuda").float())
        s = torch.exp2(torch.ceil(torch.log2(x.abs().amax((2, 3)) / TOP[code])))
        x /= s[:, :, None, None]
        codes[p:p + n] = x.to(torch.float8_e4m3fn).view(torch.uint8) if code == "e4m3" else x.round().to(torch.int8)
        scales[p:p + n] = s
    return codes, scales


def _deal(case, seed):
    """Lengths and new lengths in the order of this seed."""
    both = list(zip(_lengths(case), _new_lengths(case) if "new_lo" in case else [0] * case["batch"]))
    random.Random(seed).shuffle(both)
    return [s for s, _ in both], [n for _, n in both]


def _table(gen, held, width, pages):
    """A block table whose request b holds held[b] pages of the pool, and the pages that no request holds."""
    perm = torch.randperm(pages, generator=gen, device="cuda").int().cpu()
    table = torch.full((len(held), width), -1, dtype=torch.int32)
    off = 0
    for b, n in enumerate(held):
        table[b, :n] = perm[off:off + n]
        off += n
    return table, perm[off:].clone()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32).cuda()

    st = {"case": case}
    if case["kind"] == "rope":
        n, h, hk, rot, axes = case["tokens"], case["heads"], case["kv_heads"], case["rot"], len(_sections(case))
        st["q"] = torch.randn((n, h, rot), generator=gen, device="cuda").bfloat16()
        st["k"] = torch.randn((n, hk, rot), generator=gen, device="cuda").bfloat16()
        # rows as the attention takes them: the rotary part last
        st["q_rows"] = torch.zeros((n, h, case["packed"]), dtype=torch.bfloat16, device="cuda")
        st["k_rows"] = torch.zeros((n, hk, case["packed"]), dtype=torch.bfloat16, device="cuda")
        st["positions"] = torch.randint(0, case["far"], (axes, n), generator=gen, device="cuda", dtype=torch.int32)
        st["inv_freq"] = torch.tensor([10000.0 ** (-2.0 * j / rot) for j in range(rot // 2)], dtype=torch.float64).cuda()
        axis = [a for a, n_pairs in enumerate(_sections(case)) for _ in range(n_pairs)]
        st["pair_axis"] = torch.tensor(axis).cuda()
        if own:
            from paper_2609_37626_amd import binding as B
            st["rope"] = B.make_rope(rot, [10000.0 ** (-2.0 * j / rot) for j in range(rot // 2)], pair_axis=axis,
                                     interleaved=case["interleaved"])
        return st

    lens, new = _deal(case, seed)
    st["seq"] = ints(lens)
    if case["kind"] == "tables":
        width = max(1, max(_pages(s) for s in lens))
        pages = sum(_pages(s) for s in lens) + 7
        table, free = _table(gen, [_pages(s - n) for s, n in zip(lens, new)], width, pages)
        rows = sum(new) + case["padding"]
        st.update(new=ints(new), table=table.cuda(), free=free.cuda(), pages=pages, rows=rows,
                  taken=ints([3, 0]), taken_out=ints([0, 0]), indptr=ints([0] * (len(lens) + 1)),
                  slots=torch.empty(rows, dtype=torch.int32, device="cuda"),
                  positions=torch.empty(rows, dtype=torch.int32, device="cuda"),
                  requests=torch.empty(rows, dtype=torch.int32, device="cuda"))
        return st

    hk, d, code = case["kv_heads"], case["dim"], case["code"]
    if case["kind"] == "append":
        # the pages that the step writes to, and a few that others hold
        first = [(s - n) // PAGE if n else 0 for s, n in zip(lens, new)]
        held = [_pages(s) - f if n else 0 for s, n, f in zip(lens, new, first)]
        pages = sum(held) + 5
        table, _ = _table(gen, held, max(1, max(held)), pages)
        slots = [int(table[b, p // PAGE - f]) * PAGE + p % PAGE
                 for b, (s, n, f) in enumerate(zip(lens, new, first)) for p in range(s - n, s)]
        st["slots"] = ints(slots)
        st["k_pages"], st["k_scales"] = _codes(gen, pages, hk, d, code)
        st["v_pages"], st["v_scales"] = _codes(gen, pages, hk, d, code)
        # the fused projection's rows: queries, keys and values side by side
        qkv = torch.randn((len(slots), case["heads"] + 2 * hk, d), generator=gen, device="cuda").bfloat16()
        st["k"], st["v"] = qkv[:, case["heads"]:case["heads"] + hk], qkv[:, case["heads"] + hk:]
        if own:
            from paper_2609_37626_amd import binding as B
            st["desc"] = B.make_gqa_desc(len(lens), case["heads"], hk, d, max(1, max(held)), pages,
                                         B.GQA_E4M3 if code == "e4m3" else B.GQA_INT8)
        return st

    pages = max(1, sum(_pages(s) for s in lens))
    table, _ = _table(gen, [_pages(s) for s in lens], max(1, max(_pages(s) for s in lens)), pages)
    n = len(lens) * case["q_chunk"]
    st["table"] = table.cuda()
    st["k_pages"], st["k_scales"] = _codes(gen, pages, hk, d, code)
    st["v_pages"], st["v_scales"] = _codes(gen, pages, hk, d, code)
    st["q"] = torch.randn((n, case["heads"], d), generator=gen, device="cuda").bfloat16()
    st["out"] = torch.empty((n, case["heads"], d), dtype=torch.bfloat16, device="cuda")
    st["lse"] = torch.empty((n, case["heads"]), dtype=torch.float32, device="cuda")
    if own:
        from paper_2609_37626_amd import binding as B
        st["desc"] = B.make_gqa_desc(len(lens), case["heads"], hk, d, int(table.shape[1]), pages,
                                     B.GQA_E4M3 if code == "e4m3" else B.GQA_INT8)
        st["ws"] = torch.empty(B.gqa_workspace_size(st["desc"], case["q_chunk"]), dtype=torch.uint8, device="cuda")
    return st


# ----------------------------------------------------------- plain forms --

def _values(codes, code):
    return codes.view(torch.float8_e4m3fn).float() if code == "e4m3" else codes.float()


def _plain_tables(st):
    seq, new, table, free = st["seq"].long(), st["new"].long(), st["table"], st["free"]
    old_pages, pages = (seq - new + PAGE - 1) // PAGE, (seq + PAGE - 1) // PAGE
    need = pages - old_pages
    upto = torch.cumsum(new, 0)
    before = torch.cumsum(need, 0) - need
    k = torch.arange(table.shape[1], device="cuda")
    index = st["taken"][0] + before[:, None] + k - old_pages[:, None]
    fresh = torch.where(index < free.numel(), free[index.clamp(0, free.numel() - 1)], -1)
    table.copy_(torch.where((k >= old_pages[:, None]) & (k < pages[:, None]), fresh, table))
    row = torch.arange(st["rows"], device="cuda")
    b = torch.searchsorted(upto, row, right=True)
    real = b < seq.numel()
    b = b.clamp(max=seq.numel() - 1)
    pos = (seq - upto)[b] + row
    page = table[b, (pos // PAGE).clamp(0, table.shape[1] - 1)].long()
    total = need.sum() + st["taken"][0]
    st["indptr"].copy_(torch.cat([upto.new_zeros(1), upto]))
    st["slots"].copy_(torch.where(real & (page >= 0), page * PAGE + pos % PAGE, -1))
    st["positions"].copy_(torch.where(real, pos, 0))
    st["requests"].copy_(torch.where(real, b, -1))
    st["taken_out"].copy_(torch.stack([total.clamp(max=free.numel()), (total - free.numel()).clamp(min=0)]))


def _plain_rope(x, out, st):
    angle = st["positions"].double()[st["pair_axis"]].T * st["inv_freq"]      # [tokens, pairs]: far positions need 64 bits
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    x, rot = x.float(), x.shape[-1]
    to = out[..., out.shape[-1] - rot:]
    if st["case"]["interleaved"]:
        a, b = x[..., 0::2], x[..., 1::2]
        to.copy_(torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2))
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:]
        to.copy_(torch.cat([a * cos - b * sin, b * cos + a * sin], -1))


def _plain_append(x, slots, codes, scales, code):
    x, page, offset = x.float(), slots.long() // PAGE, slots.long() % PAGE
    pages = codes.shape[0]
    # the step's largest magnitude of each block, and its first and last new row
    amax = torch.zeros_like(scales).scatter_reduce(0, page[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
    first = torch.full((pages,), PAGE, device="cuda").scatter_reduce(0, page, offset, "amin")
    last = torch.full((pages,), -1, device="cuda").scatter_reduce(0, page, offset, "amax")
    # the least power of two that holds it, never below the block's own
    m, e = torch.frexp(amax / TOP[code])
    e = torch.where(amax > 0, torch.where(m > 0.5, e, e - 1).clamp(min=-126), -126)
    mine = torch.where((first == 0)[:, None], -126, torch.frexp(scales)[1] - 1)
    e = torch.maximum(e, mine)
    touched = (last >= 0)[:, None]
    scale = torch.where(touched, torch.ldexp(torch.ones_like(scales), e), scales)
    # rows that were there take the new scale
    value = _values(codes, code) * (scales / scale)[:, :, None, None]
    row = torch.arange(PAGE, device="cuda")
    kept = (touched & (mine < e))[:, :, None] & ((row < last[:, None]) & (first > 0)[:, None])[:, None, :]
    value = torch.where(kept[..., None], value, 0)
    again = value.to(torch.float8_e4m3fn).view(torch.uint8) if code == "e4m3" else value.round().to(torch.int8)
    codes.copy_(torch.where(kept[..., None], again, codes))
    x = x / scale[page][:, :, None]
    codes[page, :, offset] = x.to(torch.float8_e4m3fn).view(torch.uint8) if code == "e4m3" else x.round().to(torch.int8)
    scales.copy_(scale)


def _plain_attend(st):
    case, seq, table = st["case"], st["seq"].long(), st["table"]
    b, q, h, hk, d = seq.numel(), case["q_chunk"], case["heads"], case["kv_heads"], case["dim"]
    g, keys = h // hk, table.shape[1] * PAGE
    pages = table.clamp(min=0).long()
    # [b * kv head, keys, d]
    k = (_values(st["k_pages"][pages], case["code"]) * st["k_scales"][pages][..., None, None]).transpose(1, 2).reshape(b * hk, keys, d)
    rows = st["q"].float().reshape(b, q, hk, g, d).permute(0, 2, 1, 3, 4).reshape(b * hk, q * g, d)
    z = torch.bmm(rows, k.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(d)).reshape(b, hk, q, g, keys)
    del k
    sees = torch.arange(keys, device="cuda") <= seq[:, None, None] - q + torch.arange(q, device="cuda")[:, None]
    z = z.masked_fill_(~sees[:, None, :, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    w = torch.exp(z.sub_(top))
    total = w.sum(-1, keepdim=True)
    v = (_values(st["v_pages"][pages], case["code"]) * st["v_scales"][pages][..., None, None]).transpose(1, 2).reshape(b * hk, keys, d)
    out = torch.bmm(w.reshape(b * hk, q * g, keys), v).reshape(b, hk, q, g, d) / total.clamp(min=1e-37)
    st["out"].copy_(out.permute(0, 2, 1, 3, 4).reshape(b * q, h, d))
    st["lse"].copy_((top + torch.log(total)).permute(0, 2, 1, 3, 4).reshape(b * q, h))


def run(st):
    case = st["case"]
    if own:
        from paper_2609_37626_amd import binding as B
        if case["kind"] == "tables":
            B.splash_step_tables(st["seq"], 1, st["free"], st["taken"], st["taken_out"], st["table"], st["pages"],
                                 st["indptr"], st["slots"], st["positions"], st["requests"], new_lens=st["new"])
        elif case["kind"] == "rope":
            B.splash_rope(st["q"], st["positions"], st["rope"], out=st["q_rows"][..., case["packed"] - case["rot"]:],
                          x2=st["k"], out2=st["k_rows"][..., case["packed"] - case["rot"]:])
        elif case["kind"] == "append":
            B.splash_gqa_append(st["k"], st["v"], st["slots"], st["k_pages"], st["v_pages"], st["k_scales"],
                                st["v_scales"], st["desc"])
        else:
            B.splash_gqa_attend(st["q"], st["k_pages"], st["v_pages"], st["k_scales"], st["v_scales"], st["table"],
                                st["seq"], case["q_chunk"], st["out"], st["lse"], st["desc"], st["ws"])
    elif case["kind"] == "tables":
        _plain_tables(st)
    elif case["kind"] == "rope":
        _plain_rope(st["q"], st["q_rows"], st)
        _plain_rope(st["k"], st["k_rows"], st)
    elif case["kind"] == "append":
        _plain_append(st["k"], st["slots"], st["k_pages"], st["k_scales"], case["code"])
        _plain_append(st["v"], st["slots"], st["v_pages"], st["v_scales"], case["code"])
    else:
        _plain_attend(st)
    return _outputs(st)


def _outputs(st):
    case = st["case"]
    if case["kind"] == "tables":
        return {k: st[k] for k in ("table", "indptr", "slots", "positions", "requests", "taken_out")}
    if case["kind"] == "rope":
        return {"q": st["q_rows"], "k": st["k_rows"]}
    if case["kind"] == "append":
        as_values = (lambda c: c.view(torch.float8_e4m3fn)) if case["code"] == "e4m3" else (lambda c: c)
        return {"k_pages": as_values(st["k_pages"]), "k_scales": st["k_scales"],
                "v_pages": as_values(st["v_pages"]), "v_scales": st["v_scales"]}
    return {"out": st["out"], "lse": st["lse"]}


# ------------------------------------------------------------ the result --

def _exact_tables(st):
    seq, new, free = st["seq"].tolist(), st["new"].tolist(), st["free"].tolist()
    table, at, short = st["table"].cpu().clone(), st["taken"].tolist()[0], 0
    indptr, slots, positions, requests = [0], [], [], []
    for b, (s, n) in enumerate(zip(seq, new)):
        for k in range(_pages(s - n), _pages(s)):
            table[b, k] = free[at] if at < len(free) else -1
            short += at >= len(free)
            at = min(len(free), at + 1)
        for p in range(s - n, s):
            page = int(table[b, p // PAGE])
            slots.append(page * PAGE + p % PAGE if page >= 0 else -1)
            positions.append(p)
            requests.append(b)
        indptr.append(len(slots))
    rest = st["rows"] - len(slots)
    full = {"table": table, "indptr": indptr, "slots": slots + [-1] * rest, "positions": positions + [0] * rest,
            "requests": requests + [-1] * rest, "taken_out": [at, short]}
    return {k: torch.as_tensor(v, dtype=torch.int32).cuda() for k, v in full.items()}


def _exact_rope(st, x, rows):
    """Each pair as a complex number, turned by its axis' position times its frequency."""
    case = st["case"]
    rot = case["rot"]
    y = x.double()
    pairs = y.reshape(*y.shape[:-1], rot // 2, 2) if case["interleaved"] else y.reshape(*y.shape[:-1], 2, rot // 2).transpose(-1, -2)
    turn = torch.empty((x.shape[0], rot // 2), dtype=torch.float64, device="cuda")
    for j in range(rot // 2):
        turn[:, j] = st["positions"][int(st["pair_axis"][j])].double() * 10000.0 ** (-2.0 * j / rot)
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(turn), turn)[:, None]
    z = torch.view_as_real(z)
    full = rows.double().clone()
    full[..., rows.shape[-1] - rot:] = z.reshape(*y.shape) if case["interleaved"] else z.transpose(-1, -2).reshape(*y.shape)
    return full


def _exact_append(st, side):
    """Every block's scale, and the values over it that its codes are rounded from (None: the codes are whole numbers)."""
    code = st["case"]["code"]
    x, codes, scales = st[side].double(), st[side + "_pages"], st[side + "_scales"].double().clone()
    value = _values(codes, code).double()
    slots = st["slots"].tolist()
    blocks = {}
    for i, s in enumerate(slots):
        blocks.setdefault(s // PAGE, []).append(i)
    for page, rows in blocks.items():
        offsets = [slots[i] % PAGE for i in rows]
        need = x[rows].abs().amax((0, 2)) / TOP[code]
        for h in range(x.shape[1]):
            top = float(need[h])
            e = -126 if top == 0 else max(-126, math.ceil(math.log2(top)))
            old = float(scales[page, h])
            new = max(2.0 ** e, old if min(offsets) else 0.0)
            if min(offsets):
                value[page, h, :max(offsets)] *= old / new
            scales[page, h] = new
        value[page][:, offsets] = (x[rows] / scales[page][None, :, None]).transpose(0, 1)
    return (value if code == "e4m3" else None), scales


def _exact_attend(st):
    case = st["case"]
    q, h, hk, d = case["q_chunk"], case["heads"], case["kv_heads"], case["dim"]
    g = h // hk
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    for b, s in enumerate(st["seq"].tolist()):
        pages = st["table"][b, :_pages(s)].long()
        for j in range(hk):
            def history(side):
                v = _values(st[side + "_pages"][pages, j], case["code"]).double()
                return (v * st[side + "_scales"][pages, j].double()[:, None, None]).reshape(-1, d)[:s]
            if s == 0:
                continue
            k, v = history("k"), history("v")
            for i in range(q):
                n = s - q + i + 1
                if n <= 0:
                    continue
                z = st["q"][b * q + i, j * g:(j + 1) * g].double() @ k[:n].T.contiguous() / math.sqrt(d)
                out[b * q + i, j * g:(j + 1) * g] = torch.softmax(z, -1) @ v[:n]
                lse[b * q + i, j * g:(j + 1) * g] = torch.logsumexp(z, -1)
    return {"out": out, "lse": lse}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "tables":
        return _exact_tables(st)
    if case["kind"] == "rope":
        return {"q": _exact_rope(st, st["q"], st["q_rows"]), "k": _exact_rope(st, st["k"], st["k_rows"])}
    if case["kind"] == "append":
        (k, ks), (v, vs) = _exact_append(st, "k"), _exact_append(st, "v")
        return {"k_pages": k, "k_scales": ks, "v_pages": v, "v_scales": vs}
    return _exact_attend(st)
