"""Generation on a paged key/value cache held in 8 bits, as measurable cases.

Five operators, through `paper_2105_04779_amd.el_attn`:

  plan     the block table of the next step from the sequences' lengths, on the device: who goes on from whom, pages for the new
           positions, copies for shared pages that are written, the slot of every new token (`plan_pages`)
  append   the new tokens' keys and values into pages of 8-bit codes with a scale for each block of positions and head
           (`PagedCache8.append`)
  copy     codes and scales of the partly filled last pages of sequences that fork (`PagedCache8.copy_pages`)
  attend   one new token of every sequence over its pages (`PagedCache8.attend`), or the same as a segment with its
           log-sum-exp (`PagedCache8.attend_segment`)
  sample   the next token of every row of logits from a given random number, after temperature, top-k, top-p and min-p
           (`sample_tokens`)

`run` computes them in plain torch, or with `own` set through the library.  Inputs are drawn on the device from the seed alone.
Lengths are an even spread over [len_lo, n] in random order, so that a case has the same amount of work for every seed; pages
are handed out in random order.  Codes are returned as the numbers they are, next to their scales: code times scale is the value.
"""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_LARGEST = {"e4m3": 448.0, "int8": 127.0}                                      # of the codes
_SMALLEST_SCALE = 2.0 ** -126


def _attend(fmt, dtype, B, beam, heads, kv_heads, d, n, len_lo, page, block, out="storage", segment=False, softcap=0.0, window=0,
            slopes=False, heads_first=False):
    return {"kind": "attend", "fmt": fmt, "dtype": dtype, "B": B, "beam": beam, "heads": heads, "kv_heads": kv_heads, "d": d, "n": n,
            "len_lo": len_lo, "page": page, "block": block, "out": "f32" if segment else dtype if out == "storage" else out,
            "segment": segment, "softcap": softcap, "window": window, "slopes": slopes, "heads_first": heads_first}


def _append(fmt, dtype, B, T, kv_heads, d, n, page, block, ragged=False):
    return {"kind": "append", "fmt": fmt, "dtype": dtype, "B": B, "T": T, "kv_heads": kv_heads, "d": d, "n": n, "len_lo": max(T, n // 2),
            "page": page, "block": block, "ragged": ragged, "heads_first": False}


def _copy(fmt, pairs, kv_heads, d, page, block):
    return {"kind": "copy", "fmt": fmt, "pairs": pairs, "kv_heads": kv_heads, "d": d, "page": page, "block": block, "heads_first": False}


def _plan(B, T, n, len_lo, page, forks=0.0, new=0.0, room=1.0):
    return {"kind": "plan", "B": B, "T": T, "n": n, "len_lo": len_lo, "page": page, "forks": forks, "new": new, "room": room}


def _sample(dtype, rows, vocab, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, pad=0, banned=0.0):
    return {"kind": "sample", "dtype": dtype, "rows": rows, "vocab": vocab, "temperature": temperature, "top_k": top_k, "top_p": top_p,
            "min_p": min_p, "mixed": mixed, "pad": pad, "banned": banned}


def listed():
    cases = {
        # a step of 8 sentences with beam 4, continuations of some tokens: the beams go on from their parents
        "plan_beams": _plan(32, 1, 160, 100, 16, forks=0.5),
        # batch serving: 512 requests of up to 8192 positions, an eighth of them new with a prompt of up to 512
        "plan_batch": _plan(512, 512, 8192, 1024, 16, forks=0.1, new=0.125, room=1.5),
        # one token of 64 sequences
        "append8_one_e4m3": _append("e4m3", "bf16", 64, 1, 8, 128, 2000, 16, 16),
        # prompts of mixed length, padded to the longest, larger pages
        "append8_prompts_int8": _append("int8", "f16", 16, 2048, 8, 128, 2048, 64, 32, ragged=True),
        # the forks of one step: 128 sentences, beam 4
        "copy8_forks_e4m3": _copy("e4m3", 512, 16, 64, 16, 16),
        # the forks of several layers kept in one pool, larger pages
        "copy8_layers_int8": _copy("int8", 2048, 16, 64, 64, 16),
        # one sentence, interactive use, 16 heads of 64, an odd length: launches and latency alone
        "attend8_one_e4m3": _attend("e4m3", "bf16", 1, 1, 16, 16, 64, 613, 613, 16, 16),
        # batch serving with shared key heads, mixed lengths
        "attend8_batch_e4m3": _attend("e4m3", "bf16", 64, 1, 32, 8, 128, 4096, 1024, 16, 16),
        # two long contexts: the work is split over the cache's length
        "attend8_long_int8": _attend("int8", "f16", 2, 1, 32, 8, 128, 131072, 100000, 64, 64, segment=True),
        # one sentence, beam 4, all filters; an odd vocabulary, so rows start anywhere
        "sample_beams_bf16": _sample("bf16", 4, 50265, temperature=0.8, top_k=50, top_p=0.95, min_p=0.02),
        # a serving batch: every request with settings of its own
        "sample_batch_bf16": _sample("bf16", 256, 128003, temperature=0.9, top_k=40, top_p=0.9, min_p=0.05, mixed=True),
        # full precision, the whole distribution at temperature 1 for half of the rows, a large nucleus for the others
        "sample_all_f32": _sample("f32", 512, 128003, top_p=0.98, mixed=True, banned=0.1),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "copy", "plan", "sample", "sample"])
    dtype, fmt = rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice(["e4m3", "e4m3", "int8"])
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    block = rng.choice([page, page, page // 2, 8, 1])
    kv_heads, d = rng.choice([1, 2, 4, 8, 12, 16]), rng.choice([64, 64, 80, 96, 128, 128, 256])
    row = kv_heads * d                                                         # bytes of a position's keys
    if kind == "attend":
        n = _log_int(rng, 1, 131072)
        group, beam = rng.choice([1, 1, 2, 4, 7, 8]), rng.choice([1, 1, 1, 2, 4, 5])
        most = (1 << 28) // (row * max(1, group * beam // 4))                  # positions: never beyond the largest listed case
        n = min(n, most)
        B = min(_log_int(rng, 1, 512), most // n)
        return _attend(fmt, dtype, B, beam, kv_heads * group, kv_heads, d, n, rng.randint(max(1, n // 4), n), page, block,
                       out=rng.choice(["storage", "f32"]), segment=rng.random() < 0.3,
                       softcap=rng.choice([0.0, 0.0, 0.0, 20.0, 50.0]), window=rng.choice([0, 0, 0, _log_int(rng, 1, n)]),
                       slopes=rng.random() < 0.25, heads_first=rng.random() < 0.3)
    if kind == "append":
        T = rng.choice([1, 1, _log_int(rng, 1, 2048)])
        B = min(_log_int(rng, 1, 512), max(1, (1 << 25) // (T * row)))
        n = max(T, _log_int(rng, 1, 2048))
        return _append(fmt, dtype, B, T, kv_heads, d, n, page, block, ragged=T > 1 and rng.random() < 0.5)
    if kind == "copy":
        return _copy(fmt, min(_log_int(rng, 1, 4096), max(1, (1 << 27) // (page * row))), kv_heads, d, page, block)
    if kind == "plan":
        n = _log_int(rng, 1, 8192)
        B = _log_int(rng, 1, 512)
        return _plan(B, rng.choice([1, 1, 1, _log_int(rng, 1, 512)]), n, rng.randint(max(1, n // 4), n), page, forks=rng.choice([0.0, 0.1, 0.5]),
                     new=rng.choice([0.0, 0.0, 0.125, 0.5]), room=rng.choice([0.5, 1.0, 1.5]))
    vocab = _log_int(rng, 1000, 200000)
    rows = min(_log_int(rng, 1, 512), max(1, (1 << 26) // vocab))
    return _sample(dtype, rows, vocab, temperature=rng.choice([0.0, 0.5, 0.8, 1.0, 1.0, 1.7]), top_k=rng.choice([0, 0, 1, 20, 50, 400]),
                   top_p=rng.choice([1.0, 1.0, 0.5, 0.9, 0.99]), min_p=rng.choice([0.0, 0.0, 0.02, 0.1]), mixed=rng.random() < 0.5,
                   pad=rng.choice([0, 0, 7, 64]), banned=rng.choice([0.0, 0.0, 0.1, 0.999]))


def _lengths_sorted(case):
    """Evenly spread over [len_lo, n], both ends included (a single sequence has the full length)."""
    B, lo, n = case["B"], case["len_lo"], case["n"]
    return [n - (n - lo) * k // max(1, B - 1) for k in range(B)]


def _round_to_codes(y, fmt):
    """The nearest code, ties to even; beyond the largest, the largest."""
    y = y.clamp(-_LARGEST[fmt], _LARGEST[fmt])
    return y.round().to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)


def _pool(g, case, pages):
    """Codes and scales of values of about 1, every head with a size of its own: [codes, scales]."""
    fmt, page, kvh, d, block = (case[k] for k in ("fmt", "page", "kv_heads", "d", "block"))
    shape = (pages, kvh, page // block, block, d)
    x = torch.randn(shape, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn((kvh, 1, 1, 1), generator=g, device="cuda"))
    scale = (torch.maximum(x.amax((3, 4)), -x.amin((3, 4))) / _LARGEST[fmt]).clamp(min=_SMALLEST_SCALE)
    x /= scale[..., None, None]
    codes = _round_to_codes(x, fmt).view(torch.uint8).reshape(pages, kvh, page, d).transpose(1, 2)
    if not case["heads_first"]:
        codes = codes.contiguous()
    return codes.view(_TORCH[fmt]), scale


def _table(gc, lengths, page):
    """Pages in random order, every sequence its own; entries behind a sequence's last page are -1."""
    held = [-(-int(n) // page) for n in lengths]
    pages = sum(held) + 3
    order = torch.randperm(pages, generator=gc).to(torch.int32)
    table = torch.full((len(held), max(held)), -1, dtype=torch.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    return table, pages


def _prepare_sample(s, g):
    case = s["case"]
    rows, V = case["rows"], case["vocab"]
    rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")
    # a language model's logits: a broad bulk, a few tokens far above it
    x = torch.randn((rows, V + case["pad"]), generator=g, device="cuda") * 2.0
    hot = torch.randint(V, (rows, 12), generator=g, device="cuda")
    x.scatter_add_(1, hot, rand(rows, 12) * 12.0)
    if case["banned"]:
        x[rand(rows, V + case["pad"]) < case["banned"]] = float("-inf")
    s["logits"] = x.to(_TORCH[case["dtype"]])[:, :V]
    s["uniform"] = rand(rows)
    s["rule"] = {k: case[k] for k in ("temperature", "top_k", "top_p", "min_p")}
    if case["mixed"]:                                                          # half of the rows with the filter, at a strength of its own
        for k, off in (("top_k", 0), ("top_p", 1.0), ("min_p", 0.0)):
            if case[k] != off:
                value = off + (case[k] - off) * (0.5 + rand(rows))
                value = torch.where(rand(rows) < 0.5, value, torch.full_like(value, off))
                s["rule"][k] = value.to(torch.int32) if k == "top_k" else value
        s["rule"]["temperature"] = case["temperature"] * (0.75 + 0.5 * rand(rows))


def _prepare_plan(s, g, gc):
    case = s["case"]
    B, T, n, page = (case[k] for k in ("B", "T", "n", "page"))
    lengths = torch.tensor(_lengths_sorted(case))[torch.randperm(B, generator=gc)]
    table, used = _table(gc, lengths.tolist(), page)
    s["pages"] = used + int(case["room"] * B * (1 + T // page))
    # room in the table for what is to come
    columns = -(-(n + T) // page)
    full = torch.full((B, columns), -1, dtype=torch.int32)
    full[:, :table.shape[1]] = table
    # pages beyond those in use are as good as any: spread over the whole pool
    spread = torch.randperm(s["pages"], generator=gc).to(torch.int32)
    s["table"] = torch.where(full >= 0, spread[full.clamp(min=0).long()], full).cuda()
    s["lengths"] = lengths.to(torch.int32).cuda()
    parents = torch.arange(B)
    parents = torch.where(torch.rand(B, generator=gc) < case["forks"], torch.randint(B, (B,), generator=gc), parents)
    fresh = torch.rand(B, generator=gc) < case["new"]
    s["parents"] = torch.where(fresh, torch.full_like(parents, -1), parents).to(torch.int32).cuda()
    prompt = torch.randint(1, T + 1, (B,), generator=gc)
    s["counts"] = torch.where(fresh, prompt, torch.ones_like(prompt)).to(torch.int32).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    gc = torch.Generator().manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind == "sample":
        _prepare_sample(s, g)
        return s
    if kind == "plan":
        _prepare_plan(s, g, gc)
        return s
    if kind == "copy":
        pages = 2 * case["pairs"] + 5
        order = torch.randperm(pages, generator=gc).to(torch.int32)
        s["src"], s["dst"] = order[:case["pairs"]].cuda(), order[case["pairs"]:2 * case["pairs"]].cuda()
        s["counts"] = torch.randint(1, case["page"] + 1, (case["pairs"],), generator=gc).to(torch.int32).cuda()
    else:
        lengths = torch.tensor(_lengths_sorted(case))[torch.randperm(case["B"], generator=gc)]
        table, pages = _table(gc, lengths.tolist(), case["page"])
        s["table"], s["lengths"] = table.cuda(), lengths.to(torch.int32).cuda()
    s["K"], s["K_scale"] = _pool(g, case, pages)
    s["V"], s["V_scale"] = _pool(g, case, pages)
    if kind == "append":
        shape, dt = (case["B"], case["T"], case["kv_heads"], case["d"]), _TORCH[case["dtype"]]
        s["k"] = torch.randn(shape, generator=g, device="cuda", dtype=dt)
        s["v"] = torch.randn(shape, generator=g, device="cuda", dtype=dt)
        # a prompt's own length where prompts are padded: all that the sequence holds, up to what was passed
        s["counts"] = s["lengths"].clamp(max=case["T"]) if case["ragged"] else None
    if kind == "attend":
        shape, h = (case["B"], case["beam"], case["heads"], case["d"]), case["heads"]
        s["q"] = torch.randn(shape, generator=g, device="cuda", dtype=_TORCH[case["dtype"]]) * 2.0
        s["slopes"] = torch.pow(2.0, -8.0 * (torch.arange(h, device="cuda") + 1) / h) if case["slopes"] else None
    if own:
        from paper_2105_04779_amd import el_attn
        s["cache"] = el_attn.PagedCache8(s["K"], s["V"], s["K_scale"], s["V_scale"])
    return s


# ---- through the library -------------------------------------------------------------------------------------------------
def _run_own(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "sample":
        from paper_2105_04779_amd import el_attn
        tokens, logprob = el_attn.sample_tokens(s["logits"], s["uniform"], **s["rule"])
        return {"tokens": tokens, "logprob": logprob}
    if kind == "plan":
        from paper_2105_04779_amd import el_attn
        plan = el_attn.plan_pages(s["table"], s["lengths"], s["counts"], pages=s["pages"], page_size=case["page"], tokens=case["T"],
                                  parents=s["parents"])
        return {"table": plan.table, "lengths": plan.lengths, "granted": plan.granted, "slots": plan.slots, "copies": plan.copies, "free": plan.free}
    cache = s["cache"]
    if kind == "append":
        cache.append(s["k"], s["v"], s["table"], s["lengths"], counts=s["counts"])
    if kind == "copy":
        cache.copy_pages(s["src"], s["dst"], counts=s["counts"])
    if kind != "attend":
        return {"K": s["K"], "V": s["V"], "K_scale": s["K_scale"], "V_scale": s["V_scale"]}
    rule = {"n": case["n"], "softcap": case["softcap"], "window": case["window"], "slopes": s["slopes"]}
    if case["segment"]:
        A, lse = cache.attend_segment(s["q"], s["table"], s["lengths"], **rule)
        return {"out": A, "lse": lse}
    return {"out": cache.attend(s["q"], s["table"], s["lengths"], out_dtype=case["out"], **rule)}


# ---- in plain torch ------------------------------------------------------------------------------------------------------
def _values_of(codes, scale, table, block, n):
    """[B, kv_heads, n, d] in fp32: a sequence's pages one behind the other (absent pages: any values, masked later)."""
    B, cols = table.shape
    at = table.clamp(min=0).long().reshape(-1)
    x = codes.view(torch.uint8)[at].view(codes.dtype).float()                  # [B * cols, page, kv_heads, d]
    x = x * scale[at].repeat_interleave(block, 2).transpose(1, 2)[..., None]
    x = x.reshape(B, cols * codes.shape[1], codes.shape[2], codes.shape[3])[:, :n]
    return x.transpose(1, 2).contiguous()


def _plain_attend(s):
    case = s["case"]
    B, x, h, kvh, d, n = (case[k] for k in ("B", "beam", "heads", "kv_heads", "d", "n"))
    g = h // kvh
    K = _values_of(s["K"], s["K_scale"], s["table"], case["block"], n)
    V = _values_of(s["V"], s["V_scale"], s["table"], case["block"], n)
    q = s["q"].float().reshape(B, x, kvh, g, d).permute(0, 2, 1, 3, 4).reshape(B, kvh, x * g, d)
    scores = torch.matmul(q, K.transpose(2, 3).contiguous()) * d ** -0.5
    if case["softcap"]:
        scores = case["softcap"] * torch.tanh(scores / case["softcap"])
    t = torch.arange(n, device="cuda")
    behind = s["lengths"].long()[:, None] - 1 - t                              # [B, n]: how far a position lies back
    if s["slopes"] is not None:
        slope = s["slopes"].float().reshape(kvh, 1, g).expand(kvh, x, g).reshape(1, kvh, x * g, 1)
        scores = scores - slope * behind[:, None, None].float()
    keep = behind >= 0
    if case["window"]:
        keep &= behind < case["window"]
    scores = scores.masked_fill(~keep[:, None, None], float("-inf"))
    m = scores.amax(3, keepdim=True)
    p = torch.exp(scores - m)
    total = p.sum(3, keepdim=True)
    out = torch.matmul(p, V) / total
    out = out.reshape(B, kvh, x, g, d).permute(0, 2, 1, 3, 4).reshape(B, x, h, d).to(_TORCH[case["out"]])
    if not case["segment"]:
        return {"out": out}
    lse = (m + torch.log(total)).reshape(B, kvh, x, g).permute(0, 2, 1, 3).reshape(B * x, h)
    return {"out": out.reshape(B * x, h * d), "lse": lse}


def _append_into(codes, scale, new, s, at, there, block, fmt):
    """Positions `at` [B, T] (where `there`) of every sequence.  A block that holds earlier positions keeps its scale as long as that
    suffices, and is rounded again to the larger one where it does not."""
    page, kvh, d = codes.shape[1:]
    per = page // block
    row = torch.arange(at.shape[0], device="cuda")[:, None].expand_as(at)
    where = torch.where(there, s["table"].long()[row, (at // page).clamp(0, s["table"].shape[1] - 1)], 0)
    place = where * per + at % page // block                                   # block of the pool
    blocks = codes.shape[0] * per
    size = new.float().abs().amax(3)                                           # [B, T, kv_heads]
    largest = torch.full((blocks + 1, kvh), -1.0, device="cuda")               # (behind the last: tokens that are not there)
    to = torch.where(there, place, blocks)
    largest.scatter_reduce_(0, to.reshape(-1, 1).expand(-1, kvh), size.reshape(-1, kvh), "amax")
    largest = largest[:blocks]
    touched = largest >= 0
    needed = (largest * (1.0 / _LARGEST[fmt])).clamp(min=_SMALLEST_SCALE)
    # positions of the block that the sequence had before
    first = s["lengths"].long() - (there.sum(1) if s["counts"] is None else s["counts"].long())
    had = torch.zeros(blocks + 1, dtype=torch.int64, device="cuda")
    had[to.reshape(-1)] = (first[:, None] - at // block * block).clamp(0, block).reshape(-1)
    had = had[:blocks, None].expand_as(touched)
    old = scale.transpose(1, 2).reshape(blocks, kvh)
    grows = touched & (had > 0) & (needed > old)
    now = torch.where(touched, torch.where((had > 0) & ~grows, old, needed), old)
    inverse = 1.0 / now
    # what was there, where the scale grew
    value = codes.reshape(blocks, block, kvh, d).float()
    again = _round_to_codes(value * old[:, None, :, None] * inverse[:, None, :, None], fmt)
    redo = grows[:, None] & (torch.arange(block, device="cuda")[None, :, None] < had[:, None])
    raw = codes.view(torch.uint8)
    raw.copy_(torch.where(redo[..., None], again.view(torch.uint8), raw.reshape(blocks, block, kvh, d)).reshape(raw.shape))
    # the new ones; a token that is not there is written over by what its place holds
    fresh = _round_to_codes(new.float() * inverse[place][..., None], fmt).view(torch.uint8)
    flat = raw.reshape(codes.shape[0] * page, kvh, d)
    slot = torch.where(there, where * page + at % page, codes.shape[0] * page)
    flat = torch.cat([flat, flat[:1]])
    flat[slot.reshape(-1)] = fresh.reshape(-1, kvh, d)
    raw.copy_(flat[:-1].reshape(raw.shape))
    scale.copy_(now.reshape(codes.shape[0], per, kvh).transpose(1, 2))


def _plain_append(s):
    case = s["case"]
    T, lengths = case["T"], s["lengths"].long()
    counts = torch.full_like(lengths, T) if s["counts"] is None else s["counts"].long()
    i = torch.arange(T, device="cuda")
    at = (lengths - counts)[:, None] + i
    there = i < counts[:, None]
    for name, new in (("K", s["k"]), ("V", s["v"])):
        _append_into(s[name], s[name + "_scale"], new, s, at, there, case["block"], case["fmt"])
    return {k: s[k] for k in ("K", "V", "K_scale", "V_scale")}


def _plain_copy(s):
    block = s["case"]["block"]
    src, dst = s["src"].long(), s["dst"].long()
    t = torch.arange(s["case"]["page"], device="cuda") < s["counts"][:, None]
    for name in ("K", "V"):
        raw, scale = s[name].view(torch.uint8), s[name + "_scale"]
        raw[dst] = torch.where(t[:, :, None, None], raw[src], raw[dst])
        scale[dst] = torch.where(t[:, ::block][:, None], scale[src], scale[dst])
    return {k: s[k] for k in ("K", "V", "K_scale", "V_scale")}


def _plain_plan(s):
    page, T, pages = s["case"]["page"], s["case"]["T"], s["pages"]
    cols = s["table"].shape[1]
    p = s["parents"].long()
    there = (p >= 0) & (p < s["table"].shape[0])
    had = torch.where(there, s["lengths"].long()[p.clamp(min=0)].clamp(0, cols * page), 0)
    row = torch.where(there[:, None], s["table"].long()[p.clamp(min=0)], -1)
    counts = s["counts"].long().clamp(0, T)
    counts = torch.where(had + counts <= cols * page, counts, 0)
    held = (had + page - 1) // page
    b, j = torch.arange(p.shape[0], device="cuda"), torch.arange(cols, device="cuda")
    row = torch.where((j < held[:, None]) & (row >= 0) & (row < pages), row, -1)
    # who may write into a page that several name: who has most of it, the first of those that write
    extent = (had[:, None] - j * page).clamp(max=page)
    writes = ((counts > 0) & (had % page != 0))[:, None] & (j == held[:, None] - 1)
    key = (extent << 32) + torch.where(writes, (1 << 31) + (1 << 30) - b[:, None], 0)
    mark = torch.zeros(pages + 1, dtype=torch.int64, device="cuda")
    mark.scatter_reduce_(0, torch.where(row >= 0, row, pages).reshape(-1), torch.where(row >= 0, key, 0).reshape(-1), "amax")
    fresh = writes & ((row < 0) | (mark[row.clamp(min=0)] != key))             # the page is absent, or another's: a new one
    fresh_any = fresh.any(1)
    held_then = (had + counts + page - 1) // page
    need = torch.where(counts > 0, held_then - held + fresh_any, 0)
    before = torch.cumsum(need, 0) - need
    free = mark[:pages] == 0
    available = free.sum()
    granted = torch.where((need == 0) | (before + need <= available), counts, 0)
    taken = torch.where(granted > 0, need, 0)
    order = torch.argsort((~free).to(torch.uint8), stable=True)                # free pages first, the lowest in front
    nth = before[:, None] + torch.where(fresh, 0, fresh_any[:, None] + j - held[:, None])
    takes = (fresh | ((j >= held[:, None]) & (j < held_then[:, None]))) & (granted > 0)[:, None]
    table = torch.where(takes, order[nth.clamp(0, pages - 1)], row)
    lengths = had + granted
    copied = (fresh & (row >= 0) & (granted > 0)[:, None])
    some = copied.any(1)
    pick = lambda x: torch.where(copied, x, 0).sum(1)
    copies = torch.stack([torch.where(some, pick(row), -1), torch.where(some, pick(table), -1), torch.where(some, had % page, 0)])
    i = torch.arange(T, device="cuda")
    at = had[:, None] + i
    of = torch.gather(table, 1, (at // page).clamp(max=cols - 1))
    slots = torch.where(i < granted[:, None], of * page + at % page, -1)
    whole = lambda x: x.to(torch.int32)
    return {"table": whole(table), "lengths": whole(lengths), "granted": whole(granted), "slots": slots, "copies": whole(copies),
            "free": whole(available - taken.sum()).reshape(1)}


def _per_row(value, rows):
    """A filter's setting of every row, [rows, 1]: fp32 numbers in 64 bits."""
    return (value if torch.is_tensor(value) else torch.full((rows,), float(value), device="cuda"))[:, None].double()


def _plain_sample(s):
    # in 64 bits: which token it is hangs on sums of a whole vocabulary next to a border
    rows, V = s["logits"].shape
    t, k, top_p, min_p = (_per_row(s["rule"][name], rows) for name in ("temperature", "top_k", "top_p", "min_p"))
    x, order = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
    away = x.double() - x[:, :1].double()
    w = torch.where(t > 0, torch.exp(away / torch.where(t > 0, t, 1.0)), (away == 0).double())
    nth = torch.arange(V, device="cuda")
    keep = ((nth < k) | (k <= 0)) & ((t > 0) | (nth < 1)) & (x > float("-inf"))
    w = torch.where(keep, w, 0.0)
    before = torch.cumsum(w, 1) - w
    keep &= ((before < top_p * w.sum(1, keepdim=True)) | (top_p >= 1.0)) & ((w >= min_p) | (min_p <= 0)) | (nth == 0)
    w = torch.where(keep, w, 0.0)
    at = torch.zeros_like(w).scatter_(1, order, w)                             # back in the order of the vocabulary
    upto = torch.cumsum(at, 1)
    total = upto[:, -1:]
    chosen = (upto > s["uniform"].double()[:, None] * total) & (at > 0)
    token = chosen.to(torch.uint8).argmax(1)
    logprob = torch.log(torch.gather(at, 1, token[:, None]) / total)[:, 0]
    none = x[:, 0] == float("-inf")                                            # no token may follow
    token, logprob = torch.where(none, -1, token), torch.where(none, float("-inf"), logprob)
    return {"tokens": token.to(torch.int32), "logprob": logprob.float()}


def run(state):
    if own:
        return _run_own(state)
    return {"attend": _plain_attend, "append": _plain_append, "copy": _plain_copy, "plan": _plain_plan, "sample": _plain_sample}[state["case"]["kind"]](state)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------
def _exact_attend(s):
    case = s["case"]
    B, x, h, d, page, block = (case[k] for k in ("B", "beam", "heads", "d", "page", "block"))
    g = h // case["kv_heads"]
    out = torch.zeros((B, x, h, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, x, h), float("-inf"), dtype=torch.float64, device="cuda")
    raw = {name: s[name].view(torch.uint8) for name in ("K", "V")}
    for b, length in enumerate(s["lengths"].tolist()):
        first = max(0, length - case["window"]) if case["window"] else 0
        t = torch.arange(first, length, device="cuda")
        where = s["table"][b].long()[torch.div(t, page, rounding_mode="floor")]
        for i in range(h // g):
            kv = []
            for name in ("K", "V"):
                codes = raw[name][where, t % page, i].view(s[name].dtype).float().double()
                kv.append(codes * s[name + "_scale"][where, i, t % page // block].double()[:, None])
            of = slice(i * g, (i + 1) * g)                                     # the query heads that share this one
            z = (s["q"][b, :, of].double().reshape(x * g, d) @ kv[0].T / math.sqrt(d)).reshape(x, g, length - first)
            if case["softcap"]:
                z = torch.tanh(z / case["softcap"]) * case["softcap"]
            if s["slopes"] is not None:
                z = z + s["slopes"][of].double()[:, None] * (t - (length - 1)).double()
            lse[b, :, of] = torch.logsumexp(z, 2)
            out[b, :, of] = (torch.softmax(z, 2).reshape(x * g, -1) @ kv[1]).reshape(x, g, d)
    if not case["segment"]:
        return {"out": out}
    return {"out": out.reshape(B * x, h * d), "lse": lse.reshape(B * x, h)}


def _exact_append(s):
    """Scales as quotients in 64 bits, codes unrounded: what a rounding may be half a step away from."""
    case = s["case"]
    page, block, most = case["page"], case["block"], _LARGEST[case["fmt"]]
    table, lengths = s["table"].tolist(), s["lengths"].tolist()
    counts = [case["T"]] * case["B"] if s["counts"] is None else s["counts"].tolist()
    made = {}
    for name, new in (("K", s["k"]), ("V", s["v"])):
        codes, scale, new = s[name].float().double(), s[name + "_scale"].double(), new.double()
        for b, (length, count) in enumerate(zip(lengths, counts)):
            first = length - count
            for start in range(first // block * block, length, block):
                lo, hi = max(start, first), min(start + block, length)
                here, j, o = table[b][start // page], start % page // block, start % page
                got = new[b, lo - first:hi - first]
                need = got.abs().amax((0, 2)) / most
                if start < first:
                    old = scale[here, :, j].clone()
                    grown = torch.maximum(old, need)
                    codes[here, o:o + first - start] *= (old / grown)[None, :, None]
                    need = grown
                scale[here, :, j] = need
                codes[here, o + lo - start:o + hi - start] = got / need[None, :, None]
        made[name], made[name + "_scale"] = codes, scale
    return made


def _exact_sample(s):
    made = {"tokens": [], "logprob": []}
    rows = s["logits"].shape[0]
    settings = {name: _per_row(value, rows)[:, 0].tolist() for name, value in s["rule"].items()}
    for r in range(rows):
        row = s["logits"][r].double()
        if bool((row == float("-inf")).all()):
            made["tokens"].append(-1)
            made["logprob"].append(float("-inf"))
            continue
        best = int(torch.nonzero(row == row.max())[0])
        t, k, top_p, min_p = (settings[name][r] for name in ("temperature", "top_k", "top_p", "min_p"))
        if t <= 0:
            made["tokens"].append(best)
            made["logprob"].append(0.0)
            continue
        rank = torch.argsort(row, descending=True, stable=True)
        rank = rank[row[rank] > float("-inf")]
        if k > 0:
            rank = rank[:int(k)]
        p = torch.softmax(row[rank] / t, 0)
        n = len(rank)
        if top_p < 1.0:
            n = 1 + int((torch.cumsum(p, 0)[:-1] < top_p).sum())
        if min_p > 0:
            n = max(1, min(n, int((p >= min_p * p[0]).sum())))
        kept, index = torch.sort(rank[:n])
        p = p[:n][index] / p[:n].sum()
        at = min(int((torch.cumsum(p, 0) <= s["uniform"][r].double()).sum()), n - 1)
        made["tokens"].append(int(kept[at]))
        made["logprob"].append(float(torch.log(p[at])))
    return {"tokens": torch.tensor(made["tokens"], dtype=torch.int32), "logprob": torch.tensor(made["logprob"], dtype=torch.float64)}


def exact(case, seed):
    if case["kind"] in ("copy", "plan"):
        return None                                                            # moved or counted, not computed
    s = prepare(case, seed)
    if case["kind"] == "append" and case["B"] * (1 + case["T"] / case["block"]) > 20000:
        return None
    return {"attend": _exact_attend, "append": _exact_append, "sample": _exact_sample}[case["kind"]](s)


def work(case):
    kind = case["kind"]
    if kind == "sample":
        rows, V = case["rows"], case["vocab"]
        # an exponential, a sum and the comparisons of every logit
        return {"bytes": float(rows) * (V * _BYTES[case["dtype"]] + 12 + 16 * case["mixed"]), "flops": 8.0 * rows * V}
    if kind == "plan":
        # the entries in use are read, every entry of the new table and every slot is written; 28 bytes a sequence beside them
        read = sum(-(-n // case["page"]) for n in _lengths_sorted(case))
        columns = -(-(case["n"] + case["T"]) // case["page"])
        return {"bytes": 4.0 * read + case["B"] * (4.0 * columns + 8.0 * case["T"] + 32.0), "flops": 0.0}
    row = 2.0 * case["kv_heads"] * case["d"]                                   # bytes of a position's keys and values
    scales = 8.0 * case["kv_heads"] / case["block"]                            # of its share of their scales
    if kind == "copy":
        # counts are uniform over [1, page]
        return {"bytes": case["pairs"] * (2.0 * (row + scales) * (case["page"] + 1) / 2 + 12), "flops": 0.0}
    if kind == "append":
        moved = sum(min(n, case["T"]) for n in _lengths_sorted(case)) if case["ragged"] else case["B"] * case["T"]
        # the largest of a block, a product and a rounding of every element
        return {"bytes": moved * (row * (1 + _BYTES[case["dtype"]]) + 4) + case["B"] * 8, "flops": 3.0 * moved * row}
    rows = float(case["B"] * case["beam"] * case["heads"])
    read = sum(min(n, case["window"] or n) for n in _lengths_sorted(case))
    return {"bytes": read * (row + scales + 4.0 / case["page"]) + rows * (case["d"] * (_BYTES[case["dtype"]] + _BYTES[case["out"]]) + 4.0 * case["segment"]),
            "flops": 4.0 * case["heads"] * case["beam"] * case["d"] * read}
