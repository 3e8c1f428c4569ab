"""Beam search on a paged key/value cache, as measurable cases.

Four operators, through `paper_2105_04779_amd.el_attn`:

  attend   one new token of every sequence over its pages of projected keys and values (`PagedCache.attend`), or the same as a
           segment with its log-sum-exp (`PagedCache.attend_segment`)
  append   the new tokens' keys and values into the pages (`PagedCache.append`)
  copy     the partly filled last page of every beam that forks (`PagedCache.copy_pages`)
  score    log-probabilities of given tokens, entropy and the best alternatives of every row of logits (`score_tokens`)

`run` computes them in plain torch, or with `own` set through the library.  Inputs are drawn on the device from the seed alone.
Lengths are an even spread over [len_lo, n] in random order, so that a case has the same amount of work for every seed; pages
are handed out in random order.
"""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _attend(dtype, B, beam, heads, kv_heads, d, n, len_lo, page, out="storage", segment=False, softcap=0.0, window=0,
            slopes=False, heads_first=False):
    return {"kind": "attend", "dtype": dtype, "B": B, "beam": beam, "heads": heads, "kv_heads": kv_heads, "d": d, "n": n,
            "len_lo": len_lo, "page": page, "out": "f32" if segment else dtype if out == "storage" else out, "segment": segment, "softcap": softcap,
            "window": window, "slopes": slopes, "heads_first": heads_first}


def _append(dtype, B, T, kv_heads, d, n, page, ragged=False):
    return {"kind": "append", "dtype": dtype, "B": B, "T": T, "kv_heads": kv_heads, "d": d, "n": n, "len_lo": max(T, n // 2),
            "page": page, "ragged": ragged, "heads_first": False}


def _copy(dtype, pairs, kv_heads, d, page):
    return {"kind": "copy", "dtype": dtype, "pairs": pairs, "kv_heads": kv_heads, "d": d, "page": page, "heads_first": False}


def _score(dtype, rows, vocab, k, pad=0, banned=0.0):
    return {"kind": "score", "dtype": dtype, "rows": rows, "vocab": vocab, "k": k, "pad": pad, "banned": banned}


def listed():
    cases = {
        # one sentence, interactive use, 16 heads of 64, an odd length: launches and latency alone
        "attend_one_bf16": _attend("bf16", 1, 1, 16, 16, 64, 613, 613, 16),
        # decoder-only generation: each beam's own continuation, to be joined with the shared prompt's segment
        "attend_suffix_bf16": _attend("bf16", 512, 1, 16, 16, 64, 256, 1, 16, segment=True),
        # full precision, four beams on their sentence's cache, a bias by distance, pages that fit no tile
        "attend_slopes_f32": _attend("f32", 8, 4, 8, 8, 64, 777, 301, 24, slopes=True),
        # batch serving with shared key heads, mixed lengths
        "attend_batch_bf16": _attend("bf16", 64, 1, 32, 8, 128, 4096, 1024, 16),
        # capped scores and a window, wide heads, every head's positions together in a page
        "attend_window_f16": _attend("f16", 24, 1, 16, 8, 256, 8192, 2048, 32, softcap=50.0, window=1024, heads_first=True),
        # two long contexts: the work is split over the cache's length
        "attend_long_bf16": _attend("bf16", 2, 1, 32, 8, 128, 131072, 100000, 64),
        # one token of 64 sequences
        "append_one_bf16": _append("bf16", 64, 1, 8, 128, 2000, 16),
        # prompts of mixed length, padded to the longest
        "append_prompts_f16": _append("f16", 16, 2048, 8, 128, 2048, 16, ragged=True),
        # the forks of one step: 128 sentences, beam 4
        "copy_forks_bf16": _copy("bf16", 512, 16, 64, 16),
        # the forks of several layers kept in one pool, larger pages
        "copy_layers_bf16": _copy("bf16", 2048, 16, 64, 64),
        # one sentence, beam 4, twice as many alternatives as beams; an odd vocabulary, so rows start anywhere
        "score_beams_bf16": _score("bf16", 4, 50265, 8),
        # a large batch over a large vocabulary, fp32 logits with a tenth of the tokens banned
        "score_batch_f32": _score("f32", 1024, 128003, 20, banned=0.1),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "copy", "score", "score"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    kv_heads, d = rng.choice([1, 2, 4, 8, 12, 16]), rng.choice([64, 64, 80, 96, 128, 128, 256])
    row = kv_heads * d * _BYTES[dtype]                                 # bytes of a position's keys
    if kind == "attend":
        n = _log_int(rng, 1, 131072)
        group, beam = rng.choice([1, 1, 2, 4, 7, 8]), rng.choice([1, 1, 1, 2, 4, 5])
        most = (1 << 29) // (row * max(1, group * beam // 4))          # positions: never beyond the largest listed case
        n = min(n, most)
        B = min(_log_int(rng, 1, 512), most // n)
        return _attend(dtype, B, beam, kv_heads * group, kv_heads, d, n, rng.randint(max(1, n // 4), n), page,
                       out=rng.choice(["storage", "f32"]), segment=rng.random() < 0.3,
                       softcap=rng.choice([0.0, 0.0, 0.0, 20.0, 50.0]), window=rng.choice([0, 0, 0, _log_int(rng, 1, n)]),
                       slopes=rng.random() < 0.25, heads_first=rng.random() < 0.3)
    if kind == "append":
        T = rng.choice([1, 1, _log_int(rng, 1, 2048)])
        B = min(_log_int(rng, 1, 512), max(1, (1 << 26) // (T * row)))
        n = max(T, _log_int(rng, 1, 2048))
        return _append(dtype, B, T, kv_heads, d, n, page, ragged=T > 1 and rng.random() < 0.5)
    if kind == "copy":
        return _copy(dtype, min(_log_int(rng, 1, 4096), max(1, (1 << 28) // (page * row))), kv_heads, d, page)
    vocab = _log_int(rng, 1000, 200000)
    rows = min(_log_int(rng, 1, 1024), max(1, (1 << 28) // (vocab * _BYTES[dtype])))
    return _score(dtype, rows, vocab, rng.choice([0, 1, 4, 8, 10, 20, 50]), pad=rng.choice([0, 0, 7, 64]),
                  banned=rng.choice([0.0, 0.0, 0.1, 0.999]))


def _lengths_sorted(case):
    """Evenly spread over [len_lo, n], both ends included (a single sequence has the full length)."""
    B, lo, n = case["B"], case["len_lo"], case["n"]
    return [n - (n - lo) * k // max(1, B - 1) for k in range(B)]


def _pool(g, case, pages):
    shape = (pages, case["kv_heads"], case["page"], case["d"]) if case["heads_first"] else \
            (pages, case["page"], case["kv_heads"], case["d"])
    pool = [torch.randn(shape, generator=g, device="cuda", dtype=_TORCH[case["dtype"]]) for _ in range(2)]
    return [p.transpose(1, 2) for p in pool] if case["heads_first"] else pool


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


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    gc = torch.Generator().manual_seed(seed)
    kind, dt = case["kind"], _TORCH[case["dtype"]]
    s = {"case": case}
    if kind == "score":
        rows, V = case["rows"], case["vocab"]
        # a language model's logits: a broad bulk, a few tokens far above it
        x = torch.randn((rows, V + case["pad"]), generator=g, device="cuda") * 2.0
        hot = torch.randint(V, (rows, 12), generator=g, device="cuda")
        x.scatter_add_(1, hot, torch.rand((rows, 12), generator=g, device="cuda") * 12.0)
        if case["banned"]:
            x[torch.rand(x.shape, generator=g, device="cuda") < case["banned"]] = float("-inf")
        s["logits"] = x.to(dt)[:, :V]
        s["tokens"] = hot[:, 0].to(torch.int32)
        return s
    if kind == "copy":
        pages = 2 * case["pairs"] + 5
        s["K"], s["V"] = _pool(g, case, pages)
        order = torch.randperm(pages, generator=gc).to(torch.int32)
        s["src"], s["dst"] = order[:case["pairs"]].cuda(), order[case["pairs"]:2 * case["pairs"]].cuda()
        s["counts"] = torch.randint(1, case["page"] + 1, (case["pairs"],), generator=gc).to(torch.int32).cuda()
    else:
        lengths = torch.tensor(_lengths_sorted(case))[torch.randperm(case["B"], generator=gc)]
        table, pages = _table(gc, lengths.tolist(), case["page"])
        s["table"], s["lengths"] = table.cuda(), lengths.to(torch.int32).cuda()
        s["K"], s["V"] = _pool(g, case, pages)
    if kind == "append":
        shape = (case["B"], case["T"], case["kv_heads"], case["d"])
        s["k"] = torch.randn(shape, generator=g, device="cuda", dtype=dt)
        s["v"] = torch.randn(shape, generator=g, device="cuda", dtype=dt)
        # a prompt's own length where prompts are padded: all that the sequence holds, up to what was passed
        s["counts"] = s["lengths"].clamp(max=case["T"]) if case["ragged"] else None
    if kind == "attend":
        s["q"] = torch.randn((case["B"], case["beam"], case["heads"], case["d"]), generator=g, device="cuda", dtype=dt) * 2.0
        h = case["heads"]
        s["slopes"] = torch.pow(2.0, -8.0 * (torch.arange(h, device="cuda") + 1) / h) if case["slopes"] else None
    if own:
        from paper_2105_04779_amd import el_attn
        s["cache"] = el_attn.PagedCache(s["K"], s["V"])
    return s


# ---- through the library -------------------------------------------------------------------------------------------------
def _run_own(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "score":
        from paper_2105_04779_amd import el_attn
        logprob, entropy, top_logprob, top_index = el_attn.score_tokens(s["logits"], s["tokens"], k=case["k"])
        return {"logprob": logprob, "entropy": entropy, "top_logprob": top_logprob, "top_index": top_index}
    cache = s["cache"]
    if kind == "append":
        cache.append(s["k"], s["v"], s["table"], s["lengths"], counts=s["counts"])
        return {"K": cache.K, "V": cache.V}
    if kind == "copy":
        cache.copy_pages(s["src"], s["dst"], counts=s["counts"])
        return {"K": cache.K, "V": cache.V}
    rule = {"n": case["n"], "softcap": case["softcap"], "window": case["window"], "slopes": s["slopes"]}
    if case["segment"]:
        A, lse = cache.attend_segment(s["q"], s["table"], s["lengths"], **rule)
        return {"out": A, "lse": lse}
    return {"out": cache.attend(s["q"], s["table"], s["lengths"], out_dtype=case["out"], **rule)}


# ---- in plain torch ------------------------------------------------------------------------------------------------------
def _rows_of(pool, table, n):
    """[B, kv_heads, n, d] in fp32: a sequence's pages one behind the other (absent pages: any values, masked later)."""
    B, cols = table.shape
    x = pool[table.clamp(min=0).long().reshape(-1)].float()
    x = x.reshape(B, cols * pool.shape[1], pool.shape[2], pool.shape[3])[:, :n]
    return x.transpose(1, 2).contiguous()


def _plain_attend(s):
    case = s["case"]
    B, x, h, kvh, d, n = (case[k] for k in ("B", "beam", "heads", "kv_heads", "d", "n"))
    g = h // kvh
    K, V = _rows_of(s["K"], s["table"], n), _rows_of(s["V"], s["table"], n)
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


def _plain_append(s):
    case, page = s["case"], s["case"]["page"]
    T, lengths = case["T"], s["lengths"].long()
    counts = torch.full_like(lengths, T) if s["counts"] is None else s["counts"].long()
    i = torch.arange(T, device="cuda")
    at = (lengths - counts)[:, None] + i
    b, i = torch.nonzero(i < counts[:, None], as_tuple=True)
    at = at[b, i]
    where = s["table"][b, at // page].long()
    s["K"][where, at % page] = s["k"][b, i]
    s["V"][where, at % page] = s["v"][b, i]
    return {"K": s["K"], "V": s["V"]}


def _plain_copy(s):
    pair, t = torch.nonzero(torch.arange(s["case"]["page"], device="cuda") < s["counts"][:, None], as_tuple=True)
    src, dst = s["src"].long()[pair], s["dst"].long()[pair]
    s["K"][dst, t] = s["K"][src, t]
    s["V"][dst, t] = s["V"][src, t]
    return {"K": s["K"], "V": s["V"]}


def _best(x, k):
    """The k largest of every row, the lowest index first among equals: (values, indices); banned tokens are none of them."""
    V = x.shape[1]
    bits = x.contiguous().view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7fffffff), bits)                  # ordered like the values, -0 like 0
    key = order * (1 << 32) + (V - 1 - torch.arange(V, device=x.device))
    index = V - 1 - (torch.topk(key, k, dim=1).values & 0xffffffff)
    return torch.gather(x, 1, index), index


def _plain_score(s):
    k, x = s["case"]["k"], s["logits"].float()
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    weighted = torch.where(e > 0, e * (x - m), torch.zeros_like(e)).sum(1, keepdim=True)
    entropy = (torch.log(total) - weighted / total)[:, 0]
    logprob = (torch.gather(x, 1, s["tokens"].long()[:, None]) - lse)[:, 0]
    value, index = _best(x, k)
    index = torch.where(value == float("-inf"), torch.full_like(index, -1), index)
    return {"logprob": logprob, "entropy": entropy, "top_logprob": value - lse, "top_index": index.to(torch.int32)}


def run(state):
    if own:
        return _run_own(state)
    return {"attend": _plain_attend, "append": _plain_append, "copy": _plain_copy, "score": _plain_score}[state["case"]["kind"]](state)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------
def _exact_attend(s):
    case = s["case"]
    B, x, h, d, page = (case[k] for k in ("B", "beam", "heads", "d", "page"))
    g = h // case["kv_heads"]
    out = torch.zeros((B, x, h, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, x, h), float("-inf"), dtype=torch.float64, device="cuda")
    for b, length in enumerate(s["lengths"].tolist()):
        first = max(0, length - case["window"]) if case["window"] else 0
        t = torch.arange(first, length, device="cuda")
        where = s["table"][b].long()[torch.div(t, page, rounding_mode="floor")]
        for i in range(h):
            k = s["K"][where, t % page, i // g].double()
            v = s["V"][where, t % page, i // g].double()
            z = s["q"][b, :, i].double() @ k.T / math.sqrt(d)
            if case["softcap"]:
                z = torch.tanh(z / case["softcap"]) * case["softcap"]
            if s["slopes"] is not None:
                z = z + s["slopes"][i].double() * (t - (length - 1)).double()
            lse[b, :, i] = torch.logsumexp(z, 1)
            out[b, :, i] = torch.softmax(z, 1) @ v
    if not case["segment"]:
        return {"out": out}
    return {"out": out.reshape(B * x, h * d), "lse": lse.reshape(B * x, h)}


def _exact_score(s):
    x, k = s["logits"], s["case"]["k"]
    rows = x.shape[0]
    made = {"logprob": [], "entropy": [], "top_logprob": [], "top_index": []}
    for r in range(rows):
        row = x[r].double()
        logp = row - torch.logsumexp(row, 0)
        p = torch.exp(logp)
        value, index = torch.sort(row, descending=True, stable=True)
        value, index = value[:k], index[:k]
        made["logprob"].append(logp[int(s["tokens"][r])])
        made["entropy"].append(-(p * logp)[p > 0].sum())
        made["top_logprob"].append(logp[index])
        made["top_index"].append(torch.where(torch.isinf(value), torch.full_like(index, -1), index))
    return {name: torch.stack(parts) for name, parts in made.items()}


def exact(case, seed):
    if case["kind"] in ("append", "copy"):
        return None                                                            # moved, not computed
    s = prepare(case, seed)
    return _exact_attend(s) if case["kind"] == "attend" else _exact_score(s)


def work(case):
    kind, e = case["kind"], _BYTES[case["dtype"]]
    if kind == "score":
        rows, V = case["rows"], case["vocab"]
        # an exponential, two sums and the comparisons of every logit
        return {"bytes": float(rows) * (V * e + 4 + 8 + 8 * case["k"]), "flops": 8.0 * rows * V}
    row = 2.0 * case["kv_heads"] * case["d"] * e                               # a position's keys and values
    if kind == "copy":
        # counts are uniform over [1, page]
        return {"bytes": case["pairs"] * (2.0 * row * (case["page"] + 1) / 2 + 12), "flops": 0.0}
    if kind == "append":
        moved = sum(min(n, case["T"]) for n in _lengths_sorted(case)) if case["ragged"] else case["B"] * case["T"]
        return {"bytes": moved * (2.0 * row + 4) + case["B"] * 8, "flops": 0.0}
    rows = float(case["B"] * case["beam"] * case["heads"])
    read = sum(min(n, case["window"] or n) for n in _lengths_sorted(case))
    return {"bytes": read * (row + 4.0 / case["page"]) + rows * (case["d"] * (e + _BYTES[case["out"]]) + 4.0 * case["segment"]),
            "flops": 4.0 * case["heads"] * case["beam"] * case["d"] * read}
