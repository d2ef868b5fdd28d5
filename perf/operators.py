"""Performance cases of the token-record operators: writing K and V rows into record pools (with
8-bit quantisation), reading them back, and attention of chunks of new tokens over such pools.

Three kinds of case:
  write   rows of new tokens into the token slots of a pool (hisparse_write_tokens)
  read    token slots of a pool back into rows (hisparse_read_tokens)
  attend  attention of each request's newest tokens over its cache (hisparse_chunk_attention):
          form "pages", a pool of pages shared by all requests and a block table, causal; or form
          "slots", a slot cache per (request, kv head) and a slot vector per unit, one new token

Layouts: "grouped", K 128 | V 128 per token and kv head; "latent", 512 latent dims (also the value)
and 64 rotary dims. Types: "bf16" and "fp8" (e4m3 with one power-of-two scale per token and part;
the rotary dims stay bf16).
"""
import math
import random

import torch

own = False

LAYOUT = {"grouped": {"k": 128, "v": 128, "d_qk": 128, "d_v": 128, "scale": 1.0 / math.sqrt(128.0)},
          "latent": {"k": 512, "v": 64, "d_qk": 576, "d_v": 512, "scale": 1.0 / math.sqrt(192.0)}}


def _tokens(name, kind, layout, type_, tpr, heads, tokens, pad=0, fused=False):
    """pad: tokens without a slot. fused: rows that are slices of a wider projection."""
    return {"name": name, "kind": kind, "layout": layout, "type": type_, "tpr": tpr,
            "heads": heads, "tokens": tokens, "pad": pad, "fused": fused}


def _pages(name, layout, type_, tpr, requests, heads, q_heads, chunk, context, ragged=0, window=0,
           tail=0):
    """chunk, context: new tokens and all tokens of the longest request. ragged: 0, or the number
    that the requests' lengths are drawn from. tail: rows behind the last request."""
    return {"name": name, "kind": "attend", "form": "pages", "layout": layout, "type": type_,
            "tpr": tpr, "requests": requests, "heads": heads, "q_heads": q_heads, "chunk": chunk,
            "context": context, "ragged": ragged, "window": window, "tail": tail}


def _slots(name, layout, type_, tpr, requests, heads, q_heads, k, capacity, pad=0):
    """pad: trailing padding entries of each unit's slot vector."""
    return {"name": name, "kind": "attend", "form": "slots", "layout": layout, "type": type_,
            "tpr": tpr, "requests": requests, "heads": heads, "q_heads": q_heads, "k": k,
            "capacity": capacity, "pad": pad}


def listed():
    return [
        # The records of one decode step: a token of each of 32 requests, latent records. The
        # smallest call, all latency.
        _tokens("write_step_latent_fp8", "write", "latent", "fp8", 1, 1, 32),
        # A long prompt into 16-token pages of 8 kv heads, straight from the fused projection.
        _tokens("write_prompt_pages_fp8", "write", "grouped", "fp8", 16, 8, 32768, fused=True),
        # A batch of prompts padded to a common length, 64-token blocks.
        _tokens("write_blocks_padded_fp8", "write", "grouped", "fp8", 64, 4, 5003, pad=411),
        # A layer's top-2048 records of 32 requests as rows, for a consumer that takes bf16.
        _tokens("read_selected_latent_fp8", "read", "latent", "fp8", 1, 1, 65536),
        # One request's pages read back, odd length, some slots missing.
        _tokens("read_pages_fp8", "read", "grouped", "fp8", 16, 8, 2001, pad=37),
        # Sparse decode of one short request on a small model: the smallest attention call.
        _slots("decode_tiny_latent_fp8", "latent", "fp8", 1, 1, 1, 16, 128, 512),
        # Sparse decode of a full batch over 8-bit latent records, top-2048 tokens.
        _slots("decode_latent_fp8", "latent", "fp8", 1, 32, 1, 128, 2048, 4096),
        # Page selection: 8 requests x 8 kv heads, 256 pages of 16 tokens.
        _slots("decode_pages_fp8", "grouped", "fp8", 16, 8, 8, 4, 256, 384, pad=3),
        # Verification of drafted tokens: up to 4 per request, contexts of different length.
        _pages("verify_latent_fp8", "latent", "fp8", 64, 8, 1, 128, 4, 8192, ragged=5),
        # A chunk of a prompt over its cached part, latent attention with 128 heads.
        _pages("prompt_latent_bf16", "latent", "bf16", 64, 1, 1, 128, 512, 8192),
        # A chunk of a long prompt, 64 query heads on 4 kv heads: the largest case.
        _pages("prompt_blocks_bf16", "grouped", "bf16", 64, 1, 4, 16, 2048, 16384),
        # A mixed batch as a scheduler builds it: decoding requests beside prompt chunks, rows
        # behind the last request, 8-bit pages.
        _pages("mixed_pages_fp8", "grouped", "fp8", 16, 12, 8, 4, 1024, 8192, ragged=9, tail=19),
    ]


MOST_SCORES = 2048 * 64 * 16384      # of the largest listed case
MOST_FLOPS = 2 * MOST_SCORES * 256
MOST_ELEMS = 32 * 1024 * 1024 * 8    # cached elements of an attention case


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("write", "read", "slots", "slots", "pages", "pages", "pages"))
    layout = rng.choice(("grouped", "grouped", "latent"))
    type_ = rng.choice(("fp8", "fp8", "bf16"))
    grouped = layout == "grouped"
    tpr = rng.choice((1, 4, 16, 32, 64)) if grouped else rng.choice((1, 1, 16, 64))
    heads = rng.choice((1, 2, 4, 8)) if grouped else 1
    if kind in ("write", "read"):
        tokens = _log(rng, 1, 32768)
        pad = rng.choice((0, 0, rng.randint(0, tokens // 8)))
        c = _tokens("", kind, layout, type_, tpr, heads, tokens, pad=pad,
                    fused=rng.random() < 0.5)
    elif kind == "slots":
        requests = _log(rng, 1, 32)
        q_heads = (rng.choice((1, 4, 8, 16, rng.randint(1, 32))) if grouped else
                   rng.choice((16, 32, 64, 128, rng.randint(1, 128))))
        k = max(1, _log(rng, 1, 4096) // tpr)
        c = _slots("", layout, type_, tpr, requests, heads, q_heads, k, k + k // 2 + 1,
                   pad=rng.choice((0, 0, rng.randint(0, k - 1))))
    else:
        requests, chunk = _log(rng, 1, 32), _log(rng, 1, 2048)
        q_heads = (rng.choice((1, 4, 8, 16, rng.randint(1, 24))) if grouped else
                   rng.choice((16, 64, 128, rng.randint(1, 128))))
        context = max(chunk, _log(rng, 16, 32768))
        d = LAYOUT[layout]
        while (requests * heads * q_heads * chunk * context > MOST_SCORES
               or 2 * requests * heads * q_heads * chunk * context * (d["d_qk"] + d["d_v"])
               > MOST_FLOPS
               or requests * heads * context * (d["k"] + d["v"]) > MOST_ELEMS):
            if requests > 1 and rng.random() < 0.5:
                requests = (requests + 1) // 2
            elif chunk > 1 and rng.random() < 0.5:
                chunk = (chunk + 1) // 2
            else:
                context = max(chunk, (context + 1) // 2)
        c = _pages("", layout, type_, tpr, requests, heads, q_heads, chunk, context,
                   ragged=rng.choice((0, rng.randint(1, 999))),
                   window=rng.choice((0, 0, 0, _log(rng, 1, context))),
                   tail=rng.choice((0, rng.randint(0, 40))))
    del c["name"]
    return c


def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(seed * 64 + salt)


def _randn(seed, salt, shape, dtype=torch.float32):
    return torch.randn(shape, generator=_gen(seed, salt), device="cuda", dtype=dtype)


def _perm(seed, salt, n):
    return torch.argsort(torch.rand(n, generator=_gen(seed, salt), device="cuda"), stable=True)


# -- record pools ---------------------------------------------------------------------------

def _record_bytes(case):
    """One record: the tokens' rows, for 8 bits then their rotary dims and their scales."""
    d, n = LAYOUT[case["layout"]], case["tpr"]
    if case["type"] == "bf16":
        per = 2 * (d["k"] + d["v"])
    else:
        per = 264 if case["layout"] == "grouped" else 512 + 128 + 4
    return (n * per + 15) // 16 * 16


def _views(case, pool):
    """The parts of a uint8 pool [..., record bytes]: the rows of its tokens [..., tpr, elems] as
    they are stored, and for 8 bits the scales [..., tpr, parts] and the rotary dims."""
    n, grouped = case["tpr"], case["layout"] == "grouped"
    if case["type"] == "bf16":
        elems = 256 if grouped else 576
        return {"records": pool[..., :2 * n * elems].view(torch.bfloat16).unflatten(-1, (n, elems))}
    elems = 256 if grouped else 512
    at = n * elems
    v = {"records": pool[..., :at].view(torch.float8_e4m3fn).unflatten(-1, (n, elems))}
    if not grouped:
        v["rope"] = pool[..., at:at + n * 128].view(torch.bfloat16).unflatten(-1, (n, 64))
        at += n * 128
    parts = 2 if grouped else 1
    v["scales"] = pool[..., at:at + 4 * n * parts].view(torch.float32).unflatten(-1, (n, parts))
    return v


def _quantised(x):
    """float32 [..., dims] -> e4m3 values and the scales [..., 1] they are multiples of."""
    amax = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1, keepdim=True)
    m, e = torch.frexp(amax)  # amax = m 2^e, m in [0.5, 1): the least 2^e' with amax <= 448 2^e'
    e = (e - 9 + (m > 0.875)).clamp(min=-117)
    scale = torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), 1.0)
    return (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), scale


def _parts(case, k, v):
    """Rows k and v (bf16) as the parts of a record."""
    if case["type"] == "bf16":
        return {"records": torch.cat((k, v), -1)}
    qk, sk = _quantised(k.float())
    if case["layout"] == "latent":
        return {"records": qk, "rope": v, "scales": sk}
    qv, sv = _quantised(v.float())
    return {"records": torch.cat((qk.view(torch.uint8), qv.view(torch.uint8)), -1)
            .view(torch.float8_e4m3fn), "scales": torch.cat((sk, sv), -1)}


def _rows(case, parts):
    """float32 rows k and v of the parts of a record."""
    d, x = LAYOUT[case["layout"]], parts["records"].float()
    if case["type"] == "bf16":
        return x[..., :d["k"]], x[..., d["k"]:]
    if case["layout"] == "latent":
        return x * parts["scales"], parts["rope"].float()
    return x[..., :128] * parts["scales"][..., :1], x[..., 128:] * parts["scales"][..., 1:]


def _raw(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _new_rows(case, seed, salt, lead):
    """bf16 K and V rows [lead..., dims]: some channels larger than others, as keys have them, and
    tokens of different size."""
    d = LAYOUT[case["layout"]]
    out = []
    for i, part in enumerate(("k", "v")):
        x = _randn(seed, salt + 2 * i, (*lead, d[part]), torch.bfloat16)
        spread = torch.exp(0.3 * _randn(seed, salt + 2 * i + 1, (d[part],))).to(torch.bfloat16)
        out.append(x * spread)
    return out


def _filled(case, seed, lead):
    """A uint8 pool [lead..., record bytes] whose every token holds a row."""
    pool = torch.zeros((*lead, _record_bytes(case)), dtype=torch.uint8, device="cuda")
    views = _views(case, pool)
    k, v = _new_rows(case, seed, 8, (*lead, case["tpr"]))
    for name, part in _parts(case, k, v).items():
        _raw(views[name]).copy_(_raw(part))
    return pool


def _slot_list(case, seed):
    """int64 [tokens]: distinct token slots of whole pages in a shuffled order, or of single
    tokens; the last `pad` tokens have none."""
    n, tpr = case["tokens"], case["tpr"]
    pages = (n + tpr - 1) // tpr + 3
    t = torch.arange(n, device="cuda")
    slots = _perm(seed, 1, pages)[t // tpr] * tpr + t % tpr
    if case["pad"]:
        slots[n - case["pad"]:] = -1
    return slots, pages


def _row_buffers(case, fill):
    """K and V rows [tokens][heads][dims], of their own or as slices of one wider buffer."""
    d, n, h = LAYOUT[case["layout"]], case["tokens"], case["heads"]
    if case["fused"]:
        wide = torch.zeros((n, h * (d["k"] + d["v"]) + 256), dtype=torch.bfloat16, device="cuda")
        k = wide[:, 256:256 + h * d["k"]].unflatten(1, (h, d["k"]))
        v = wide[:, 256 + h * d["k"]:].unflatten(1, (h, d["v"]))
    else:
        k, v = (torch.zeros((n, h, d[p]), dtype=torch.bfloat16, device="cuda") for p in "kv")
    if fill is not None:
        k.copy_(fill[0])
        v.copy_(fill[1])
    return k, v


# -- attention cases ------------------------------------------------------------------------

def _lengths(case):
    """New tokens and all tokens of every request."""
    R, C, T = case["requests"], case["chunk"], case["context"]
    if not case["ragged"]:
        return [C] * R, [T] * R
    rng = random.Random(case["ragged"])
    new = [C] + [_log(rng, 1, C) if rng.random() < 0.5 else 1 for _ in range(R - 1)]
    return new, [T] + [n + rng.randint(0, T - C) for n in new[1:]]


def _prepare_pages(case, seed, s):
    d, R, h, tpr = LAYOUT[case["layout"]], case["requests"], case["heads"], case["tpr"]
    new, kv = _lengths(case)
    per = (max(kv) + tpr - 1) // tpr
    s["pool"] = _filled(case, seed, (R * per + 2, h))
    table = _perm(seed, 2, R * per + 2)[:R * per].to(torch.int32).view(R, per)
    used = torch.tensor([(t + tpr - 1) // tpr for t in kv], device="cuda")
    s["table"] = torch.where(torch.arange(per, device="cuda")[None] < used[:, None], table,
                             torch.full_like(table, -1))
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s["start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device="cuda")
    s["total"] = starts[-1] + case["tail"]


def _prepare_slots(case, seed, s):
    R, h, k, B = case["requests"], case["heads"], case["k"], case["capacity"]
    s["pool"] = _filled(case, seed, (R, h, B))
    u = torch.rand((R, h, B), generator=_gen(seed, 2), device="cuda")
    s["table"] = torch.argsort(u, dim=-1, stable=True)[..., :k].to(torch.int32).contiguous()
    if case["pad"]:
        s["table"][..., k - case["pad"]:] = -1
    s["start"] = s["kv_len"] = None
    s["total"] = R


def prepare(case, seed):
    d = LAYOUT[case["layout"]]
    s = {"case": case}
    if case["kind"] == "attend":
        (_prepare_pages if case["form"] == "pages" else _prepare_slots)(case, seed, s)
        H = case["heads"] * case["q_heads"]
        s["q"] = _randn(seed, 4, (s["total"], H, d["d_qk"]), torch.bfloat16)
        s["out"] = torch.zeros((s["total"], H, d["d_v"]), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros((s["total"], H), dtype=torch.float32, device="cuda")
        return s
    s["slots"], pages = _slot_list(case, seed)
    if case["kind"] == "write":
        s["pool"] = torch.zeros((pages, case["heads"], _record_bytes(case)), dtype=torch.uint8,
                                device="cuda")
        lead = (case["tokens"], case["heads"])
        s["k"], s["v"] = _row_buffers(case, _new_rows(case, seed, 8, lead))
    else:
        s["pool"] = _filled(case, seed, (pages, case["heads"]))
        s["k"], s["v"] = _row_buffers(case, None)
    return s


# -- the plain forms ------------------------------------------------------------------------

def _write_plain(s):
    case, views, slots = s["case"], _views(s["case"], s["pool"]), s["slots"]
    # a token without a slot stands in for one that has one: the same values to the same place
    t = torch.where(slots >= 0, torch.arange(slots.numel(), device=slots.device),
                    torch.argmax((slots >= 0).int()))
    rec, off = slots[t] // case["tpr"], slots[t] % case["tpr"]
    for name, part in _parts(case, s["k"][t], s["v"][t]).items():
        _raw(views[name])[rec, :, off] = _raw(part)
    return views


def _read_plain(s):
    case, slots = s["case"], s["slots"]
    rec, off = slots.clamp(min=0) // case["tpr"], slots.clamp(min=0) % case["tpr"]
    views = _views(case, s["pool"])
    parts = {n: _raw(v)[rec, :, off].view(v.dtype) for n, v in views.items()}
    ok = (slots >= 0)[:, None, None]
    for to, rows in zip((s["k"], s["v"]), _rows(case, parts)):
        to.copy_(torch.where(ok, rows, 0.0))
    return {"k": s["k"], "v": s["v"]}


def _attend_plain(s):
    case = s["case"]
    d, R, h, g, tpr = (LAYOUT[case["layout"]], case["requests"], case["heads"], case["q_heads"],
                       case["tpr"])
    pages = case["form"] == "pages"
    table = s["table"].long()
    if pages:
        table = table[:, None].expand(R, h, table.shape[1])
        rec = table.clamp(min=0)
        head = torch.arange(h, device=rec.device)[None, :, None].expand_as(rec)
        at = (rec, head)
        start, kv = s["start"].long(), s["kv_len"].long()
        new, C = start[1:] - start[:-1], case["chunk"]
    else:
        rec = table.clamp(min=0)
        req = torch.arange(R, device=rec.device)[:, None, None].expand_as(rec)
        head = torch.arange(h, device=rec.device)[None, :, None].expand_as(rec)
        at = (req, head, rec)
        start = torch.arange(R + 1, device=rec.device)
        kv = torch.full((R,), rec.shape[2] * tpr, device=rec.device)
        new, C = torch.ones_like(kv), 1
    parts = {n: _raw(v)[at].view(v.dtype).flatten(2, 3)
             for n, v in _views(case, s["pool"]).items()}          # [R][h][T][elems]
    k, v = _rows(case, parts)
    if case["layout"] == "latent":
        k, v = torch.cat((k, v), -1), k
    T = k.shape[2]
    j = torch.arange(T, device=k.device)
    i = torch.arange(C, device=k.device)
    live = i[None] < new[:, None]                                   # [R][C]
    row = (start[:-1, None] + i[None]).clamp(max=s["total"] - 1)
    last = (kv - new)[:, None] + i[None] if pages else (kv - 1)[:, None]   # newest visible token
    seen = (j < kv[:, None, None]) & (j <= last[..., None])         # [R][C][T]
    if pages and case["window"]:
        seen = seen & (j > last[..., None] - case["window"])
    seen = (seen[:, None] & (table >= 0).repeat_interleave(tpr, 2)[:, :, None])[:, :, None]
    q = s["q"][row].float().unflatten(2, (h, g)).permute(0, 2, 3, 1, 4)    # [R][h][g][C][dqk]
    x = (q.flatten(2, 3) @ k.transpose(2, 3)).unflatten(2, (g, C)) * d["scale"]
    x = x.masked_fill(~seen, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m > -math.inf, m, 0.0))
    l = p.sum(-1, keepdim=True)
    o = (p.flatten(2, 3) @ v).unflatten(2, (g, C)) / torch.where(l > 0, l, 1.0)
    lse = (m + torch.log(l)).squeeze(-1)
    # the rows of live tokens; a dead one stands in for its request's first
    i0 = torch.where(live, i[None], 0)
    r = torch.arange(R, device=k.device)[:, None].expand_as(i0)
    to = start[:-1, None] + i0
    s["out"][to] = o.permute(0, 3, 1, 2, 4)[r, i0].flatten(2, 3).to(torch.bfloat16)
    s["lse"][to] = lse.permute(0, 3, 1, 2)[r, i0].flatten(2, 3)
    return {"out": s["out"], "lse": s["lse"]}


# -- the framework's calls ------------------------------------------------------------------

def _kv_desc(hs, case, pool):
    layout = hs.HISPARSE_KV_GROUPED if case["layout"] == "grouped" else hs.HISPARSE_KV_LATENT
    type_ = hs.HISPARSE_KV_BF16 if case["type"] == "bf16" else hs.HISPARSE_KV_FP8
    if pool.dim() == 3:  # [record][head]
        return hs.KvDesc(layout, type_, case["tpr"], pool.shape[2], pool.shape[0],
                         pool.stride(0), pool.stride(1), 0)
    return hs.KvDesc(layout, type_, case["tpr"], pool.shape[3], pool.shape[2], pool.stride(2),
                     pool.stride(1), pool.stride(0))


def _call(s):
    from paper_2608_07009_amd import hisparse as hs
    case, stream = s["case"], torch.cuda.current_stream()
    if "kv" not in s:  # what a program sets up once
        s["kv"] = _kv_desc(hs, case, s["pool"])
        if case["kind"] == "write":
            s["views"] = _views(case, s["pool"])
        if case["kind"] == "attend":
            pages, t = case["form"] == "pages", s["table"]
            s["chunk"] = hs.ChunkDesc(
                case["requests"], case["heads"], case["q_heads"], s["total"],
                case["chunk"] if pages else 1, t.shape[-1], s["q"].stride(0), s["out"].stride(0),
                t.stride(0), 0 if pages else t.stride(1), case["window"] if pages else 0, 0,
                LAYOUT[case["layout"]]["scale"], hs.HISPARSE_CHUNK_CAUSAL if pages else 0)
            n = hs.hisparse_chunk_workspace_bytes(s["kv"], s["chunk"])
            s["ws"] = torch.empty(n, dtype=torch.uint8, device=s["pool"].device)
    if case["kind"] == "write":
        hs.hisparse_write_tokens(s["kv"], case["heads"], case["tokens"], s["k"], s["k"].stride(0),
                                 s["v"], s["v"].stride(0), s["slots"], s["pool"], stream)
        return s["views"]
    if case["kind"] == "read":
        hs.hisparse_read_tokens(s["kv"], case["heads"], case["tokens"], s["pool"], s["slots"],
                                s["k"], s["k"].stride(0), s["v"], s["v"].stride(0), stream)
        return {"k": s["k"], "v": s["v"]}
    hs.hisparse_chunk_attention(s["kv"], s["chunk"], s["pool"], s["table"], s["start"],
                                s["kv_len"], s["q"], s["out"], s["lse"], s["ws"],
                                s["ws"].numel(), stream)
    return {"out": s["out"], "lse": s["lse"]}


def run(s):
    if own:
        return _call(s)
    return {"write": _write_plain, "read": _read_plain, "attend": _attend_plain}[
        s["case"]["kind"]](s)


# -- what a pass cannot do without ----------------------------------------------------------

def _token_bytes(case):
    """Bytes of one token of one kv head in a record."""
    grouped = case["layout"] == "grouped"
    if case["type"] == "bf16":
        return 512 if grouped else 1152
    return 264 if grouped else 644


def _visible(n, kv, window):
    """Visible (new token, cached token) pairs of one request and the cached tokens any of its new
    tokens sees."""
    pairs = sum(min(kv - n + i + 1, window or kv) for i in range(n))
    return pairs, min(kv, (window + n - 1) if window else kv)


def work(case):
    d = LAYOUT[case["layout"]]
    if case["kind"] != "attend":
        n = case["tokens"] - case["pad"]
        rows = 2 * (d["k"] + d["v"])
        return {"bytes": 8 * case["tokens"] + n * case["heads"] * (rows + _token_bytes(case)),
                "flops": 0}
    if case["form"] == "slots":
        n = case["requests"] * case["heads"] * (case["k"] - case["pad"]) * case["tpr"]
        pairs, tokens, rows = n * case["q_heads"], n, case["requests"]
    else:
        pairs = tokens = 0
        new, kv = _lengths(case)
        for a, b in zip(new, kv):
            p, t = _visible(a, b, case["window"])
            pairs += p * case["heads"] * case["q_heads"]
            tokens += t * case["heads"]
        rows = sum(new)
    io = rows * case["heads"] * case["q_heads"] * (2 * d["d_qk"] + 2 * d["d_v"] + 4)
    return {"bytes": tokens * _token_bytes(case) + io, "flops": 2 * pairs * (d["d_qk"] + d["d_v"])}


# -- the same results from their definition, in 64 bits --------------------------------------

def _e4m3_value(b):
    """The numbers that e4m3 bytes stand for."""
    b = b.to(torch.int64)
    e, m = (b >> 3) & 15, (b & 7).double()
    x = torch.where(e > 0, (8.0 + m) * torch.exp2((e - 10).double()), m * 2.0 ** -9)
    x = torch.where((b & 127) == 127, math.nan, x)
    return torch.where(b > 127, -x, x)


def _to_e4m3_grid(y):
    """float64 values rounded to the nearest e4m3 number (ties to even), at most 448."""
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -40))).clamp(min=-6.0)
    step = torch.exp2(e - 3.0)
    return (torch.round(y / step) * step).clamp(-448.0, 448.0)


def _token_rows(case, record):
    """float64 K and V rows [..., tpr, dims] of records given as bytes."""
    n, grouped = case["tpr"], case["layout"] == "grouped"
    word = lambda a, b, t: record[..., a:b].contiguous().view(t).double()  # noqa: E731
    if case["type"] == "bf16":
        e, cut = (256, 128) if grouped else (576, 512)
        x = word(0, 2 * e * n, torch.bfloat16).unflatten(-1, (n, e))
        return x[..., :cut], x[..., cut:]
    e = 256 if grouped else 512
    x = _e4m3_value(record[..., :e * n]).unflatten(-1, (n, e))
    if grouped:
        sc = word(e * n, (e + 8) * n, torch.float32).unflatten(-1, (n, 2))
        return x[..., :128] * sc[..., 0, None], x[..., 128:] * sc[..., 1, None]
    rope = word(e * n, (e + 128) * n, torch.bfloat16).unflatten(-1, (n, 64))
    return x * word((e + 128) * n, (e + 132) * n, torch.float32)[..., None], rope


def _exact_write(case, s):
    slots = s["slots"]
    t = torch.nonzero(slots >= 0).flatten()
    rec, off = slots[t] // case["tpr"], slots[t] % case["tpr"]
    out = {n: torch.zeros(v.shape, dtype=torch.float64, device="cuda")
           for n, v in _views(case, s["pool"]).items()}
    if case["type"] == "bf16":
        out["records"][rec, :, off] = torch.cat((s["k"][t], s["v"][t]), -1).double()
        return out
    rows, scales = [], []
    for x in (s["k"][t].double(), s["v"][t].double())[:2 if case["layout"] == "grouped" else 1]:
        scale = torch.exp2(torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 448.0)))
        rows.append(_to_e4m3_grid(x / scale))
        scales.append(scale)
    out["records"][rec, :, off] = torch.cat(rows, -1)
    out["scales"][rec, :, off] = torch.cat(scales, -1)
    if case["layout"] == "latent":
        out["rope"][rec, :, off] = s["v"][t].double()
    return out


def _exact_read(case, s):
    slots = s["slots"]
    k, v = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (s["k"], s["v"]))
    t = torch.nonzero(slots >= 0).flatten()
    rk, rv = _token_rows(case, s["pool"])      # [page][head][tpr][dims]
    rec, off = slots[t] // case["tpr"], slots[t] % case["tpr"]
    k[t], v[t] = rk[rec, :, off], rv[rec, :, off]
    return {"k": k, "v": v}


def _exact_attend(case, s):
    d, R, h, g = LAYOUT[case["layout"]], case["requests"], case["heads"], case["q_heads"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    pages = case["form"] == "pages"
    new, kv = _lengths(case) if pages else ([1] * R, [(case["k"] - case["pad"]) * case["tpr"]] * R)
    begin = 0
    for r in range(R):
        n, T = new[r], kv[r]
        for u in range(h):
            if pages:
                rec = s["table"][r, :(T + case["tpr"] - 1) // case["tpr"]].long()
                records = s["pool"][rec, u]
            else:
                records = s["pool"][r, u, s["table"][r, u, :case["k"] - case["pad"]].long()]
            k, v = (x.flatten(0, 1)[:T] for x in _token_rows(case, records))
            if case["layout"] == "latent":
                k, v = torch.cat((k, v), -1), k.contiguous()
            kt = k.t().contiguous()
            i = torch.arange(T - n, T, device="cuda")[:, None]
            j = torch.arange(T, device="cuda")[None]
            hidden = (j > i) | (j <= i - (case["window"] or T) if pages else j > i)
            for e in range(u * g, (u + 1) * g):
                x = s["q"][begin:begin + n, e].double() @ kt * d["scale"]
                x = x.masked_fill(hidden, -math.inf)
                lse[begin:begin + n, e] = torch.logsumexp(x, 1)
                out[begin:begin + n, e] = torch.softmax(x, 1) @ v
        begin += n
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    return {"write": _exact_write, "read": _exact_read, "attend": _exact_attend}[case["kind"]](
        case, s)
