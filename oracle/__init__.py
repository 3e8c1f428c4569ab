"""fp64 CPU oracle for the multi-head-attention decode step (TEST INFRASTRUCTURE).

Only tests, the smoke check and the benchmark's ``cpu_baseline`` leg may import
this package.  It shares no code with the HIP path and never imports it.

The arithmetic lives in ``mha_oracle.c`` (plain C, double precision); this
module compiles it with gcc on first use and marshals numpy arrays to it.

``mha_reference``  multi-head attention by its definition (Eq. 1, Eq. 2/6).
``el_reference``   the same quantity in the evaluation order of Eq. 9; used by
                   the tests to check the losslessness identity on the oracle.
``segment_reference``  per-(row, head) log-sum-exp of the scores and head outputs of ordinary attention
                   over one key set, by definition (Eq. 1, Eq. 6/7), for the joint softmax of
                   section 3.2; ``join_segments_reference`` joins them and applies W^O.
``check_inputs_reference``  what a decode step assumes about its inputs, counted by definition.
``paged_attend_reference``, ``paged_append_reference``, ``paged_copy_reference``  attention of one new token over pages
                   of projected keys and values, and what moves them, position by position.
``quantized_append_reference``, ``quantized_copy_reference``, ``quantized_values``, ``nearest_codes``  the paged cache in 8 bits.
``plan_pages_reference``  the table of the next step, one sequence after the other.
``sample_tokens_reference``  the token that a random number draws from what the filters leave, and how close that was.
``score_tokens_reference``  log-probability, entropy and best alternatives of rows of logits, by definition.
``gather_batch_reference``  the state gather between decode steps (section 3.1.1's
                   state, re-ordered / compacted by the search), by its definition.
"""
from __future__ import annotations

import ctypes
import os
import subprocess
import threading

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_SRC = os.path.join(_HERE, "mha_oracle.c")
_LIB = os.path.join(_HERE, "libmha_oracle.so")
_lock = threading.Lock()
_lib = None


def build(force: bool = False, out: str | None = None, extra_flags=()) -> str:
    """Compile mha_oracle.c into libmha_oracle.so next to it (gcc, OpenMP).  With `out`, into that file
    instead, with `extra_flags` added (the sanitizer test builds an instrumented copy this way)."""
    lib = out or _LIB
    if force or out or not os.path.exists(lib) or os.path.getmtime(lib) < os.path.getmtime(_SRC):
        tmp = lib + ".tmp.%d" % os.getpid()
        cmd = ["gcc", "-O2", "-fopenmp", "-fno-fast-math", "-ffp-contract=off", "-shared", "-fPIC", *extra_flags,
               "-o", tmp, _SRC, "-lm"]
        subprocess.run(cmd, check=True)
        os.replace(tmp, lib)
    return lib


def _load():
    global _lib
    with _lock:
        if _lib is None:
            # MHA_ORACLE_LIB: a library built by build(out=...) to load instead (same source, other compiler flags)
            lib = ctypes.CDLL(os.environ.get("MHA_ORACLE_LIB") or build())
            dp = ctypes.POINTER(ctypes.c_double)
            ip = ctypes.POINTER(ctypes.c_int32)
            sig = [ctypes.c_int] * 6 + [dp, ip, dp] + [dp] * 8 + [dp]
            for name in ("mha_oracle", "el_oracle"):
                fn = getattr(lib, name)
                fn.argtypes = sig
                fn.restype = ctypes.c_int
            lib.oracle_num_threads.restype = ctypes.c_int
            _lib = lib
    return _lib


def num_threads() -> int:
    """Threads the oracle's OpenMP loop over batch elements will use."""
    return int(_load().oracle_num_threads())


def _f64(a, shape, name):
    if a is None:
        return None
    a = np.ascontiguousarray(np.asarray(a, dtype=np.float64))
    if a.shape != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {a.shape}")
    return a


def _ptr(a):
    return None if a is None else a.ctypes.data_as(ctypes.POINTER(ctypes.c_double))


def _call(fn_name, H, lengths, queries, Wq, bq, Wk, bk, Wv, bv, Wo, bo, heads, d_k):
    H = np.asarray(H)
    queries = np.asarray(queries)
    if H.ndim != 3 or queries.ndim != 3:
        raise ValueError("H must be [B, n, d_m] and queries [B, beam, d_m]")
    B, n, d_m = H.shape
    beam = queries.shape[1]
    hd = heads * d_k
    H = _f64(H, (B, n, d_m), "H")
    queries = _f64(queries, (B, beam, d_m), "queries")
    Wq = _f64(Wq, (d_m, hd), "Wq")
    Wk = _f64(Wk, (d_m, hd), "Wk")
    Wv = _f64(Wv, (d_m, hd), "Wv")
    Wo = _f64(Wo, (hd, d_m), "Wo")
    bq = _f64(bq, (hd,), "bq")
    bk = _f64(bk, (hd,), "bk")
    bv = _f64(bv, (hd,), "bv")
    bo = _f64(bo, (d_m,), "bo")
    lp = None
    if lengths is not None:
        lengths = np.ascontiguousarray(np.asarray(lengths, dtype=np.int32))
        if lengths.shape != (B,):
            raise ValueError("lengths must be [B]")
        lp = lengths.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    out = np.empty((B, beam, d_m), dtype=np.float64)
    rc = getattr(_load(), fn_name)(B, beam, n, heads, d_m, d_k, _ptr(H), lp, _ptr(queries),
                                   _ptr(Wq), _ptr(bq), _ptr(Wk), _ptr(bk), _ptr(Wv), _ptr(bv),
                                   _ptr(Wo), _ptr(bo), _ptr(out))
    if rc != 0:
        raise ValueError(f"{fn_name} rejected its arguments (code {rc}); lengths must lie in [1, n]")
    return out


def mha_reference(H, lengths, queries, Wq, bq, Wk, bk, Wv, bv, Wo, bo, *, heads, d_k):
    """Eq. 6: sum_i softmax(Q_i K_i^T / sqrt(d_k)) V_i W_i^O (+ b^O), in float64.

    H [B,n,d_m]; lengths [B] or None; queries [B,beam,d_m]; Wq/Wk/Wv [d_m,h*d_k];
    Wo [h*d_k,d_m]; biases may be None.  Returns out [B,beam,d_m] float64.
    """
    return _call("mha_oracle", H, lengths, queries, Wq, bq, Wk, bk, Wv, bv, Wo, bo, heads, d_k)


def el_reference(H, lengths, queries, Wq, bq, Wk, bk, Wv, bv, Wo, bo, *, heads, d_k):
    """Eq. 9: the expanded-query evaluation order, in float64 (oracle self-check only)."""
    return _call("el_oracle", H, lengths, queries, Wq, bq, Wk, bk, Wv, bv, Wo, bo, heads, d_k)


def gather_batch_reference(H_src, lengths_src, index, H_dst_before):
    """State maintenance by its definition, one row at a time (section 3.1.1: the state is H itself).

    H_dst[i, t, :] = H_src[index[i], t, :] for t < lengths_src[index[i]]; other rows keep what
    ``H_dst_before`` held; lengths_dst[i] = lengths_src[index[i]].  An index outside [0, B_src)
    leaves its destination untouched and reports length 0.  Arrays are copied bit for bit
    (any dtype); returns (H_dst, lengths_dst).
    """
    H_src = np.asarray(H_src)
    out = np.array(H_dst_before, copy=True)
    n = H_src.shape[1]
    lens = np.full(H_src.shape[0], n, dtype=np.int32) if lengths_src is None else np.asarray(lengths_src, dtype=np.int32)
    new_lens = np.zeros(len(index), dtype=np.int32)
    for i, src in enumerate(index):
        src = int(src)
        if src < 0 or src >= H_src.shape[0]:
            continue
        new_lens[i] = lens[src]
        for t in range(int(lens[src])):
            out[i, t, :] = H_src[src, t, :]
    return out, new_lens


def segment_reference(H, lengths, queries, Wq, bq, Wk, bk, Wv, bv, *, heads, d_k):
    """Ordinary attention over one key set, left unjoined (section 3.2 combines such pieces under one softmax).

    Per query row m = b*beam + j and head i, with K_i = H_b W_i^K + b_i^K, V_i = H_b W_i^V + b_i^V (Eq. 6) and
    s_t = Q_i K_i[t]^T / sqrt(d_k) for t < lengths[b] (Eq. 1):
        lse[m, i] = log sum_t exp(s_t)            seg_A[m, i*d_k:(i+1)*d_k] = softmax(s) V_i
    Everything in float64; returns (seg_A [B*beam, h*d_k], lse [B*beam, h]).
    """
    H = np.asarray(H, dtype=np.float64)
    q = np.asarray(queries, dtype=np.float64)
    B, n, d_m = H.shape
    beam = q.shape[1]
    hd = heads * d_k
    zeros = np.zeros(hd)
    bq, bk, bv = [zeros if b is None else np.asarray(b, dtype=np.float64) for b in (bq, bk, bv)]
    Wq, Wk, Wv = [np.asarray(W, dtype=np.float64) for W in (Wq, Wk, Wv)]
    lens = np.full(B, n, dtype=np.int64) if lengths is None else np.asarray(lengths, dtype=np.int64)
    seg_A = np.zeros((B * beam, hd))
    lse = np.zeros((B * beam, heads))
    for b in range(B):
        Hb = H[b, :lens[b]]
        K = Hb @ Wk + bk
        V = Hb @ Wv + bv
        for j in range(beam):
            Q = q[b, j] @ Wq + bq
            for i in range(heads):
                cols = slice(i * d_k, (i + 1) * d_k)
                s = K[:, cols] @ Q[cols] / np.sqrt(d_k)
                m = s.max()
                e = np.exp(s - m)
                lse[b * beam + j, i] = m + np.log(e.sum())
                seg_A[b * beam + j, cols] = (e / e.sum()) @ V[:, cols]
    return seg_A, lse


def join_segments_reference(segments, Wo, bo, *, heads, d_k):
    """One softmax over the union of the segments' keys, then Eq. 2's output projection.

    segments: list of (seg_A, lse) as segment_reference returns them, all over the same query rows.
    A softmax over a union of key sets is the mixture of the per-set softmaxes with weights
    proportional to each set's sum of exponentials, exp(lse_s).  Returns out [rows, d_m] float64.
    """
    Wo = np.asarray(Wo, dtype=np.float64)
    rows = segments[0][0].shape[0]
    A = np.zeros((rows, heads * d_k))
    for r in range(rows):
        for i in range(heads):
            cols = slice(i * d_k, (i + 1) * d_k)
            M = max(l[r, i] for _, l in segments)
            w = np.array([np.exp(l[r, i] - M) for _, l in segments])
            w /= w.sum()
            for (sA, _), ws in zip(segments, w):
                A[r, cols] += ws * sA[r, cols]
    out = A @ Wo
    if bo is not None:
        out = out + np.asarray(bo, dtype=np.float64)
    return out


def check_inputs_reference(H, lengths, n=None):
    """Counts of what the decode step assumes about its inputs (section 3.1 needs a non-empty softmax; the 16-bit
    path needs fp16-representable magnitudes), one element at a time over the valid rows only.

    H [B, n, d_m] as float32/float64 VALUES of the stored elements (NaN/Inf allowed); lengths [B] or None.
    Returns [lengths outside [1, n], non-finite elements, finite elements with |v| > 65504, elements examined];
    a length outside [0, n] is clamped for the walk.
    """
    H = np.asarray(H)
    B, n_rows, d_m = H.shape
    n = n_rows if n is None else n
    lens = np.full(B, n, dtype=np.int64) if lengths is None else np.asarray(lengths, dtype=np.int64)
    bad_len = nonfinite = large = seen = 0
    for b in range(B):
        if lens[b] < 1 or lens[b] > n:
            bad_len += 1
        for t in range(int(min(max(lens[b], 0), n))):
            row = H[b, t].astype(np.float64)
            fin = np.isfinite(row)
            nonfinite += int((~fin).sum())
            large += int((np.abs(row[fin]) > 65504.0).sum())
            seen += d_m
    return [bad_len, nonfinite, large, seen]


def paged_attend_reference(K, V, table, lengths, queries, *, scale, n=None, softcap=0.0, window=0, slopes=None):
    """Attention of one new token over pages of projected keys and values, one (row, head) at a time.

    K, V [pages, page_size, kv_heads, d], queries [B, x, heads, d] as values of the stored elements; table [B, columns];
    lengths [B], n the nearer end for what lies outside [0, n].  Positions in a page outside the pool do not exist.
    Returns float64 out [B, x, heads, d] and lse [B, x, heads] (nothing attended: 0 and -inf), and for error bounds
    {"spread": sum_t p_t |V_t| like out, "qk": max_t scale sum_c |q_c k_tc|, "s": the largest |score| or cap or bias that
    a score is made of, "n": positions}, like lse.
    """
    pages, page_size, kv_heads, d = K.shape
    B, x, heads, _ = queries.shape
    n = table.shape[1] * page_size if n is None else n
    out, lse = np.zeros((B, x, heads, d)), np.full((B, x, heads), -np.inf)
    info = {"spread": np.zeros_like(out), "qk": np.zeros_like(lse), "s": np.zeros_like(lse), "n": np.zeros_like(lse)}
    for b in range(B):
        length = int(min(max(lengths[b], 0), n))
        places = []
        for t in range(max(0, length - window) if window else 0, length):
            page = int(table[b, t // page_size])
            if 0 <= page < pages:
                places.append((t, page, t % page_size))
        if not places:
            continue
        t, page, at = (np.array(c) for c in zip(*places))
        for i in range(heads):
            g = i // (heads // kv_heads)
            k, v = K[page, at, g].astype(np.float64), V[page, at, g].astype(np.float64)
            for j in range(x):
                q = queries[b, j, i].astype(np.float64)
                s = scale * (k @ q)
                parts = [np.abs(s).max()]
                info["qk"][b, j, i] = abs(scale) * (np.abs(k) @ np.abs(q)).max()
                if softcap:
                    s = softcap * np.tanh(s / softcap)
                    parts.append(softcap)
                if slopes is not None:
                    bias = float(slopes[i]) * (length - 1 - t)
                    s = s - bias
                    parts += [np.abs(bias).max(), np.abs(s).max()]
                m = s.max()
                if m == -np.inf:
                    continue
                e = np.exp(s - m)
                p = e / e.sum()
                lse[b, j, i] = m + np.log(e.sum())
                out[b, j, i] = (p[:, None] * v)[p > 0].sum(0)
                info["spread"][b, j, i] = (p[:, None] * np.abs(v))[p > 0].sum(0)
                info["s"][b, j, i], info["n"][b, j, i] = max(parts), len(places)
    return out, lse, info


def paged_append_reference(K, V, table, lengths, counts, K_new, V_new):
    """K, V with token i < counts[b] of K_new, V_new [B, T, kv_heads, d] at position lengths[b] - counts[b] + i, token by
    token; positions that do not exist are dropped."""
    K, V = K.copy(), V.copy()
    pages, page_size = K.shape[:2]
    B, T = K_new.shape[:2]
    for b in range(B):
        count = T if counts is None else int(min(max(counts[b], 0), T))
        for i in range(count):
            t = int(lengths[b]) - count + i
            if 0 <= t < table.shape[1] * page_size and 0 <= table[b, t // page_size] < pages:
                K[table[b, t // page_size], t % page_size] = K_new[b, i]
                V[table[b, t // page_size], t % page_size] = V_new[b, i]
    return K, V


def paged_copy_reference(K, V, src, dst, counts):
    """K, V with positions [0, counts[i]) of page dst[i] taken from page src[i], pair by pair."""
    K2, V2 = K.copy(), V.copy()
    pages, page_size = K.shape[:2]
    for i in range(len(src)):
        if 0 <= src[i] < pages and 0 <= dst[i] < pages:
            c = page_size if counts is None else int(min(max(counts[i], 0), page_size))
            K2[dst[i], :c], V2[dst[i], :c] = K[src[i], :c], V[src[i], :c]
    return K2, V2


def score_tokens_reference(logits, tokens, k):
    """(logprob, entropy, top_logprob, top_index) of float64 rows, and for error bounds sum_v p_v |x_v - max| per row."""
    rows, vocab = logits.shape
    logprob, entropy, away = np.zeros(rows), np.zeros(rows), np.zeros(rows)
    top_logprob, top_index = np.full((rows, k), -np.inf), np.full((rows, k), -1, dtype=np.int64)
    for r in range(rows):
        x = logits[r].astype(np.float64)
        allowed = x > -np.inf                                        # (False for NaN)
        broken = bool(np.isnan(x).any() or (x == np.inf).any())
        m = log_S = 0.0
        if broken:
            log_S = entropy[r] = np.nan
        elif allowed.any():
            m = x.max()
            d = x[allowed] - m                                       # (of any size: the sums are relative to the largest)
            log_S = np.log(np.exp(d).sum())
            p = np.exp(d - log_S)
            entropy[r] = log_S - (p * d).sum()
            away[r] = -(p * d).sum()
        if tokens is not None:
            t = int(tokens[r])
            logprob[r] = 0.0 if t < 0 else np.nan if t >= vocab else (x[t] - m) - log_S
        which = np.nonzero(allowed)[0]                               # ascending: a stable sort leaves equal ones in this order
        for i, v in enumerate(which[np.argsort(-x[which], kind="stable")[:k]]):
            top_logprob[r, i], top_index[r, i] = (x[v] - m) - log_S, v
    return logprob, entropy, top_logprob, top_index, away


# ---- the paged cache in 8 bits -------------------------------------------------------------------------------------------
LARGEST_CODE = {"e4m3": 448.0, "int8": 127.0}


def e4m3_values():
    """The 256 values of an e4m3 code, from its bits: sign, 4 bits of exponent (bias 7), 3 of mantissa; no infinities, all ones is NaN."""
    values = np.zeros(256)
    for code in range(256):
        exponent, mantissa = code >> 3 & 15, code & 7
        size = (8 + mantissa) * 2.0 ** (exponent - 10) if exponent else mantissa * 2.0 ** -9
        values[code] = np.nan if exponent == 15 and mantissa == 7 else size
        if code & 128:
            values[code] = -values[code]
    return values


def quantized_values(codes, fmt):
    """Codes (uint8 bits of e4m3, or int8) as numbers."""
    return codes.astype(np.float64) if fmt == "int8" else e4m3_values()[codes]


def nearest_codes(y, fmt):
    """The code nearest to each y, of two the even one; beyond the largest, the largest; NaN: NaN, or 0 among whole numbers."""
    y = np.asarray(y, dtype=np.float64)
    if fmt == "int8":
        return np.where(np.isnan(y), 0, np.rint(np.clip(y, -127, 127))).astype(np.int8)
    size, x = e4m3_values()[:127], np.minimum(np.abs(np.nan_to_num(y, nan=0.0, posinf=448.0, neginf=-448.0)), 448.0)
    above = np.clip(np.searchsorted(size, x), 1, 126)                          # size[above - 1] < x <= size[above], x = 0 apart
    below = above - 1
    down, up = x - size[below], size[above] - x
    code = np.where(down < up, below, np.where(up < down, above, np.where(below % 2 == 0, below, above)))
    return np.where(np.isnan(y), 127, code | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def quantized_append_reference(codes, scale, table, lengths, counts, new, block, fmt):
    """(codes, scale) with token i < counts[b] of new [B, T, kv_heads, d] (float32 values) at position lengths[b] - counts[b] + i, block by block, in the
    fp32 arithmetic of the definition.  codes [pages, page_size, kv_heads, d], scale [pages, kv_heads, page_size // block] float32."""
    codes, scale = codes.copy(), scale.copy()
    pages, page_size, kv_heads, _ = codes.shape
    f = np.float32
    inverse_largest = f(1.0 / LARGEST_CODE[fmt])
    B, T = new.shape[:2]
    with np.errstate(all="ignore"):
        for b in range(B):
            count = T if counts is None else int(min(max(counts[b], 0), T))
            start = int(lengths[b]) - count
            groups = {}
            for i in range(count):
                t = start + i
                if 0 <= t < table.shape[1] * page_size and 0 <= table[b, t // page_size] < pages:
                    groups.setdefault(t // block, []).append((i, t))
            for k, tokens in groups.items():
                base = k * block
                page, first = int(table[b, base // page_size]), base % page_size
                had = min(max(start - base, 0), block)
                for h in range(kv_heads):
                    x = np.stack([new[b, i, h] for i, _ in tokens]).astype(f)
                    size = np.abs(x[np.isfinite(x)])
                    needed = max(f(size.max(initial=f(0))) * inverse_largest, f(2.0 ** -126))
                    old = scale[page, h, first // block]
                    now = old if had and not needed > old else needed
                    inverse = f(1) / f(now)
                    if had and needed > old:
                        value = quantized_values(codes[page, first:first + had, h], fmt).astype(f)
                        codes[page, first:first + had, h] = nearest_codes((value * old) * inverse, fmt)
                    for (_, t), row in zip(tokens, x):
                        codes[page, t % page_size, h] = nearest_codes(row * inverse, fmt)
                    scale[page, h, first // block] = now
    return codes, scale


def quantized_copy_reference(codes, scale, src, dst, counts, block):
    """(codes, scale) with positions [0, counts[i]) of page dst[i], and the scales of the blocks that they begin or fill, taken from page src[i]."""
    codes2, scale2 = codes.copy(), scale.copy()
    pages, page_size = codes.shape[:2]
    for i in range(len(src)):
        if 0 <= src[i] < pages and 0 <= dst[i] < pages:
            c = page_size if counts is None else int(min(max(counts[i], 0), page_size))
            codes2[dst[i], :c] = codes[src[i], :c]
            scale2[dst[i], :, :-(-c // block)] = scale[src[i], :, :-(-c // block)]
    return codes2, scale2


# ---- the table of the next step ------------------------------------------------------------------------------------------
def plan_pages_reference(table, lengths, counts, parents, reserved, pages, page_size, T, exclusive=False):
    """dict of table, lengths, granted, slots, copies, free, as whole numbers, one sequence after the other.  exclusive: a page that is written is kept only if one
    entry names it."""
    B_old, columns = table.shape
    parents = list(range(B_old)) if parents is None else [int(p) for p in parents]
    B = len(parents)
    had, rows, asked = [], [], []
    for b, p in enumerate(parents):
        there = 0 <= p < B_old
        n = min(max(int(lengths[p]), 0), columns * page_size) if there else 0
        held = -(-n // page_size)
        row = [int(table[p, j]) if j < held and 0 <= table[p, j] < pages else -1 for j in range(columns)] if there else [-1] * columns
        c = T if counts is None else min(max(int(counts[b]), 0), T)
        had.append(n)
        rows.append(row)
        asked.append(c if n + c <= columns * page_size else 0)
    users = {}                                                                 # page: (positions used, writes, sequence) of each that names it
    for b in range(B):
        held = -(-had[b] // page_size)
        for j in range(held):
            if rows[b][j] >= 0:
                writes = asked[b] > 0 and had[b] % page_size != 0 and j == held - 1
                users.setdefault(rows[b][j], []).append((min(page_size, had[b] - j * page_size), writes, b))
    free = [p for p in range(pages) if p not in users and not (reserved is not None and reserved[p])]
    available, wanted = len(free), 0
    out = {"table": np.full((B, columns), -1), "lengths": np.zeros(B, int), "granted": np.zeros(B, int), "slots": np.full((B, T), -1),
           "copies": np.stack([np.full(B, -1), np.full(B, -1), np.zeros(B, int)])}
    taken = 0
    for b in range(B):
        held, then = -(-had[b] // page_size), -(-(had[b] + asked[b]) // page_size)
        replaced = False
        if asked[b] > 0 and had[b] % page_size != 0:
            page = rows[b][held - 1]
            if page < 0 or (reserved is not None and reserved[page]):
                replaced = True
            elif exclusive:
                replaced = len(users[page]) > 1
            else:
                most = max(e for e, _, _ in users[page])
                keeper = min([s for e, w, s in users[page] if e == most and w], default=None)
                replaced = keeper != b
        need = then - held + replaced if asked[b] > 0 else 0
        wanted += need
        if need and wanted > available:
            asked[b] = 0
        row = list(rows[b])
        if asked[b] > 0 and need:
            mine = free[wanted - need:wanted]
            taken = wanted
            if replaced:
                page, own = row[held - 1], mine.pop(0)
                if page >= 0:
                    out["copies"][:, b] = page, own, had[b] % page_size
                row[held - 1] = own
            row[held:then] = mine
        out["table"][b] = row
        out["granted"][b], out["lengths"][b] = asked[b], had[b] + asked[b]
        for i in range(asked[b]):
            t = had[b] + i
            out["slots"][b, i] = row[t // page_size] * page_size + t % page_size
    out["free"] = available - taken
    return out


# ---- sampling ------------------------------------------------------------------------------------------------------------
def sample_tokens_reference(logits, uniform, temperature, top_k, top_p, min_p):
    """(tokens, logprob, margin) of float64 rows with a setting of each row; margin: how far the decisions (which token, where the filters cut) are from going
    the other way, relative to the sums that decide them."""
    rows, vocab = logits.shape
    tokens, logprob, margin = np.full(rows, -1), np.zeros(rows), np.full(rows, np.inf)
    for r in range(rows):
        x = logits[r].astype(np.float64)
        t, k, p, q, u = float(temperature[r]), int(top_k[r]), float(top_p[r]), float(min_p[r]), float(uniform[r])
        if np.isnan(x).any() or (x == np.inf).any():
            logprob[r] = np.nan
            continue
        order = np.argsort(-x, kind="stable")
        order = order[x[order] > -np.inf]
        if len(order) == 0:
            logprob[r] = -np.inf
            continue
        if not t > 0:
            tokens[r] = order[0]
            continue
        w = np.exp((x[order] - x[order[0]]) / t)
        n = min(k, len(order)) if k > 0 else len(order)
        before = np.concatenate([[0.0], np.cumsum(w[:n])])
        if p < 1:
            margin[r] = min(margin[r], np.abs(before[1:n] - p * before[n]).min(initial=np.inf) / before[n])
            n = max(1, int((before[:n] < p * before[n]).sum()))
        if q > 0:
            margin[r] = min(margin[r], np.abs(w[1:n] / q - 1).min(initial=np.inf))
            n = max(1, int((w[:n] >= q).sum()))
        left = np.sort(order[:n])
        weights = np.exp((x[left] - x[order[0]]) / t)
        upto = np.cumsum(weights)
        past = np.nonzero(upto > u * upto[-1])[0]
        at = int(past[0]) if len(past) else n - 1
        margin[r] = min(margin[r], np.abs(upto[:-1] / upto[-1] - u).min(initial=np.inf))
        tokens[r], logprob[r] = left[at], np.log(weights[at] / upto[-1])
    return tokens, logprob, margin
