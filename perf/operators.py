"""The paged 8-bit cache: its operators as cases that can be timed and compared, in plain torch and through the library.

A page holds P positions of a layer for all KV heads: the codes of K (a standard layer) or K' (a shared one), the codes of V, and a
scale for every block of 16 positions and head.  Page bytes, in order (a layer's pool is [n_pages, page_bytes]):
  K codes   [Hkv][P][d], or K' [Hkv][P/16][r][16] (the 16 positions of a block side by side), padded to 128 bytes
  V codes   [Hkv][P][d]
  scales    [Hkv][P/16][2] fp32: K's (or K''s) and V's; the page is padded to 128 bytes
A code is an int8 (value = code * scale, scale = amax / 127) or an e4m3 (amax / 448).  Sequence b's position j lies in page
table[b][j / P].  Four operators:

  append   rows of new tokens quantised into the pages (blocks that are partly filled keep one scale: what they hold is
           rescaled when it grows), and the rows read back as a program that hands a sequence to another cache does
  anchor   a new token's attention over a standard layer's pages (softmax(q K^T / sqrt(d)) V), with the score row for the
           shared layer behind it
  shared   the same for a shared layer: scores = Integrate(Align(previous row), q' K'^T / sqrt(r)), softmax, V
  pages    the bookkeeping: beams taking over one another's pages and writing to copies of those that they share; moving
           the pages in use to the front of the pool
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 16
FLOAT = {"f32": torch.float32, "bf16": torch.bfloat16}
L7 = {"Hq": 32, "Hkv": 32, "d": 128, "r": 21, "m": 64}    # LLaMA2-7B-shaped
L8 = {"Hq": 32, "Hkv": 8, "d": 128, "r": 21, "m": 64}     # LLaMA3-8B-shaped (grouped queries)
L13 = {"Hq": 40, "Hkv": 40, "d": 128, "r": 21, "m": 80}   # LLaMA2-13B-shaped
LP = {"Hq": 32, "Hkv": 32, "d": 128, "r": 20, "m": 256}   # the paper's default layer (concatenating aligner)
SHAPES = {"7b": L7, "8b": L8, "13b": L13, "paper": LP}


def _case(op, shape, **more):
    return dict(op=op, shape=shape, **more)


def _append(shape, kind, B, n, before, fmt="s8", page=64, ragged=False, **name):
    return _case("append", shape, kind=kind, B=B, n=n, before=before, fmt=fmt, page=page, ragged=ragged, **name)


def _attend(op, shape, B, L, fmt="s8", page=64, ragged=False, rows="f32", **name):
    return _case(op, shape, B=B, L=L, fmt=fmt, page=page, ragged=ragged, rows=rows, **name)


def listed():
    return [
        # one decode step's K' and V of 64 sequences into a shared layer, blocks half full
        _append("13b", "shared", 64, 1, 1111, page=16, name="append_token_13b"),
        # prompts of odd lengths behind what their sequences hold already, e4m3, grouped KV heads
        _append("8b", "shared", 12, 1777, 333, fmt="e4m3", ragged=True, name="append_ragged_prompts_8b"),
        # a batch of prompts into a standard layer of the 7B shape
        _append("7b", "standard", 8, 2048, 0, name="append_prompts_7b"),
        # one user's chat turn: a single sequence, a short context, where launches and latency count
        _attend("anchor", "8b", 1, 333, page=16, name="anchor_one_sequence_8b"),
        # continuous batching: sequences of every length in one call, idle slots among them
        _attend("anchor", "7b", 16, 2900, fmt="e4m3", ragged=True, rows="none", name="anchor_ragged_7b"),
        # long documents with grouped queries: few sequences, the context split over the whole card
        _attend("anchor", "8b", 2, 65537, rows="bf16", name="anchor_long_8b"),
        # a large batch of the 13B shape: bound by HBM
        _attend("anchor", "13b", 64, 4096, rows="none", name="anchor_batch_13b"),
        # one sequence through a shared layer of the 7B shape
        _attend("shared", "7b", 1, 333, page=16, name="shared_one_sequence_7b"),
        # the paper's default layer (concatenating aligner, hidden width 256) over a ragged batch, 2-byte score rows
        _attend("shared", "paper", 12, 1901, fmt="e4m3", ragged=True, rows="bf16", name="shared_ragged_paper_default"),
        # the batch of the 13B shape through a shared layer
        _attend("shared", "13b", 64, 4096, name="shared_batch_13b"),
        # a beam-search step: 16 prompts of 4 beams change places, then each writes to a page of its own (32 layers)
        _case("beam", "8b", groups=16, beams=4, L=1000, layers=32, fmt="s8", page=16, name="beam_step_8b"),
        # a pool in which two of five sequences have ended, compacted
        _case("compact", "8b", B=40, L=1500, layers=16, fmt="s8", page=32, name="compact_8b"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "anchor", "anchor", "anchor", "shared", "shared", "shared", "beam", "compact"])
    fmt, page, ragged = rng.choice(["s8", "e4m3"]), rng.choice([16, 32, 64, 128]), rng.random() < 0.5
    if op == "append":
        n = rng.choice([1, _log(rng, 1, 64), _log(rng, 64, 4096)])
        return _append(rng.choice(["7b", "8b", "13b", "paper"]), rng.choice(["standard", "shared"]), _log(rng, 1, max(1, min(64, 16384 // n))),
                       n, rng.randrange(0, 2000), fmt, page, ragged)
    if op in ("anchor", "shared"):
        shape = rng.choice(["7b", "8b", "13b"] + ["paper"] * (op == "shared"))
        heads = SHAPES[shape]["Hkv"] if op == "anchor" else 40   # a shared layer's cost is not that of its KV heads alone
        L = _log(rng, 1, 65536)
        most = 64 * 4096 * 40 // (L * heads)
        return _attend(op, shape, _log(rng, 1, max(1, min(64, most))), L, fmt, page, ragged, rng.choice(["f32", "bf16", "none"]))
    if op == "beam":
        return _case("beam", rng.choice(["7b", "8b"]), groups=_log(rng, 1, 16), beams=rng.choice([2, 3, 4, 5]), L=_log(rng, 8, 1000),
                     layers=rng.choice([8, 16, 32]), fmt=fmt, page=rng.choice([16, 32]))
    return _case("compact", rng.choice(["7b", "8b"]), B=_log(rng, 3, 40), L=_log(rng, 40, 1500), layers=rng.choice([4, 8, 16]), fmt=fmt,
                 page=rng.choice([16, 32]))


# ------------------------------------------------------------------ page layout
def _up(n, to=128):
    return -(-n // to) * to


def _layout(shape, kind, P):
    """(key width, offset of V, offset of the scales, bytes of a page)."""
    Hkv, d = shape["Hkv"], shape["d"]
    kw = d if kind == "standard" else shape["r"]
    v = _up(Hkv * P * kw)
    s = v + Hkv * P * d
    return kw, v, s, _up(s + Hkv * (P // BLOCK) * 8)


def _views(pool, shape, kind, P):
    """K and V codes as bytes [n_pages, P/16, Hkv, 16, width] and scales [n_pages, P/16, Hkv, 2], all views of the pool."""
    Hkv, d, nb = shape["Hkv"], shape["d"], P // BLOCK
    kw, v_at, s_at, _ = _layout(shape, kind, P)
    k = pool[:, :Hkv * P * kw]
    k = k.unflatten(1, (Hkv, nb, BLOCK, kw)) if kind == "standard" else k.unflatten(1, (Hkv, nb, kw, BLOCK)).transpose(3, 4)
    v = pool[:, v_at:s_at].unflatten(1, (Hkv, nb, BLOCK, d))
    s = pool[:, s_at:s_at + Hkv * nb * 8].view(torch.float32).unflatten(1, (Hkv, nb, 2))
    return k.transpose(1, 2), v.transpose(1, 2), s.transpose(1, 2)


def _values(codes, fmt, dtype=torch.float32):
    return codes.view(torch.int8 if fmt == "s8" else torch.float8_e4m3fn).to(dtype)


def _codes(y, fmt):
    """y, in units of the scale, as codes (bytes)."""
    if fmt == "s8":
        return y.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _largest(fmt, like):
    return torch.full((), 127.0 if fmt == "s8" else 448.0, device=like.device, dtype=like.dtype)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _tokens(g, B, n, H, w):
    """Rows as a model's projections give them: N(0, 1), some columns louder, some tokens too."""
    x = _normal(g, B, n, H, w)
    x *= 1 + 3 * (torch.arange(w, device="cuda") % 16 == 5)
    return x * (0.25 * _normal(g, B, n, 1, 1)).exp()


def _fill(pool, shape, kind, P, fmt, g):
    """A pool of pages as the append leaves them when every block is full."""
    views = _views(pool, shape, kind, P)
    step = max(1, (1 << 27) // (shape["Hkv"] * P * shape["d"]))
    for at in range(0, pool.shape[0], step):
        for i in (0, 1):
            codes, scales = views[i][at:at + step], views[2][at:at + step, ..., i]
            x = _tokens(g, codes.shape[0], codes.shape[1], codes.shape[2] * BLOCK, codes.shape[4]).view(codes.shape)
            s = x.abs().amax((3, 4)) / _largest(fmt, x)
            codes.copy_(_codes(x / s[..., None, None], fmt))
            scales.copy_(s)


def _lengths(c, g, most):
    """Ragged batches: spread over [most / 8, most] and one of them full, every sixth an idle slot of length 0."""
    B = c["B"]
    if not c["ragged"]:
        return torch.full((B,), most, dtype=torch.int32, device="cuda")
    lens = (most * (0.125 + 0.875 * torch.rand(B, generator=g, device="cuda"))).to(torch.int32).clamp(min=1)
    at = torch.arange(B, device="cuda")
    return torch.where(at % 6 == 4, 0, torch.where(at == 0, most, lens)).to(torch.int32)


def _table(g, B, per_row, spare):
    """Pages as a pool in use hands them out: in no order, a few of them free."""
    n_pages = B * per_row + spare
    table = torch.randperm(n_pages, generator=g, device="cuda")[:B * per_row].to(torch.int32).view(B, per_row)
    return n_pages, table


def _kinds(layers):
    """Layers 0-3 and every 4th thereafter are standard, the rest shared."""
    return ["standard" if l < 4 or l % 4 == 3 else "shared" for l in range(layers)]


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    shape, P = SHAPES[c["shape"]], c["page"]
    s = {"case": c, "shape": shape}
    if c["op"] in ("beam", "compact"):
        return _prepare_pages(s, g)
    kind = c.get("kind") or ("standard" if c["op"] == "anchor" else "shared")
    B, Hq, Hkv, d = c["B"], shape["Hq"], shape["Hkv"], shape["d"]
    most = c["before"] + c["n"] if c["op"] == "append" else c["L"]
    s["kind"] = kind
    n_pages, s["table"] = _table(g, B, -(-most // P), 3)
    s["pool"] = torch.zeros((n_pages, _layout(shape, kind, P)[3]), dtype=torch.uint8, device="cuda")
    _fill(s["pool"], shape, kind, P, c["fmt"], g)
    if c["op"] == "append":
        n, kw = c["n"], _layout(shape, kind, P)[0]
        s["k"] = _tokens(g, B, n, Hkv, kw).bfloat16()
        s["v"] = _tokens(g, B, n, Hkv, d).bfloat16()
        before = torch.randint(0, c["before"] + 1, (B,), generator=g, device="cuda") if c["ragged"] else torch.full((B,), c["before"], device="cuda")
        s["before"] = before.to(torch.int32)
        s["new"] = _lengths(c, g, n)
        # what is read back begins with the block that the new rows begin in
        s["first"] = s["before"] // BLOCK * BLOCK
        s["read"] = torch.where(s["new"] > 0, s["before"] - s["first"] + s["new"], 0).to(torch.int32)
        s["k_out"] = torch.zeros((B, n + BLOCK, Hkv, kw), dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.zeros((B, n + BLOCK, Hkv, d), dtype=torch.bfloat16, device="cuda")
        return s
    s["lens"] = _lengths(c, g, c["L"])
    L_row = _up(c["L"], 8)
    if c["rows"] != "none":
        s["row"] = torch.zeros((B, Hq, L_row), dtype=FLOAT[c["rows"]], device="cuda")
    s["o"] = torch.empty((B, 1, Hq, d), dtype=torch.bfloat16, device="cuda")
    if c["op"] == "anchor":
        s["q"] = _normal(g, B, 1, Hq, d).bfloat16()
        return s
    r, m = shape["r"], shape["m"]
    s["qp"] = _normal(g, B, 1, Hq, r).bfloat16()
    s["prev"] = _normal(g, B, Hq, L_row).to(FLOAT["f32" if c["rows"] == "none" else c["rows"]])
    h_in = Hq if c["shape"] != "paper" else 2 * Hq
    s["w1"] = (_normal(g, h_in, m) * h_in ** -0.5).bfloat16()
    s["w2"] = (_normal(g, m, Hq) * m ** -0.5).bfloat16()
    return s


def _prepare_pages(s, g):
    c, shape = s["case"], s["shape"]
    P, L = c["page"], c["L"]
    s["kinds"] = _kinds(c["layers"])
    per_row = -(-(L + 1) // P)
    if c["op"] == "beam":
        # a prompt's full pages are shared by its beams; the page being written is each beam's own
        G, K = c["groups"], c["beams"]
        full = L // P
        n_pages = G * full + 3 * G * K
        ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        table = torch.full((G * K, per_row + 1), -1, dtype=torch.int32, device="cuda")
        table[:, :full] = ids[:G * full].view(G, full).repeat_interleave(K, 0)
        if L % P:
            table[:, full] = ids[G * full:G * full + G * K]
        s["lens"] = torch.full((G * K,), L, dtype=torch.int32, device="cuda")
        parent = torch.randint(0, K, (G, K), generator=g, device="cuda") + K * torch.arange(G, device="cuda")[:, None]
        s["parent"] = parent.view(-1).to(torch.int32)
        s["new"] = torch.ones(G * K, dtype=torch.int32, device="cuda")
    else:
        B = c["B"]
        n_pages, table = _table(g, B, per_row, 5)
        lens = torch.where(torch.arange(B, device="cuda") % 5 < 2, 0, L).to(torch.int32)     # two of five sequences have ended
        table = torch.where(lens[:, None] > 0, table, -1)
        table[:, -(-L // P):] = -1
        s["lens"] = lens
    s["table"] = table
    held = table[table >= 0].long()
    s["refs"] = torch.zeros(n_pages, dtype=torch.int32, device="cuda").index_add_(0, held, torch.ones_like(held, dtype=torch.int32))
    s["pools"] = [torch.randint(0, 256, (n_pages, _layout(shape, k, P)[3]), generator=g, device="cuda", dtype=torch.uint8) for k in s["kinds"]]
    s["table0"], s["refs0"] = s["table"].clone(), s["refs"].clone()
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return {"append": _run_append, "anchor": _run_attend, "shared": _run_attend, "beam": _run_beam, "compact": _run_compact}[s["case"]["op"]](s)


def _layer(s):
    """The library's handle on the pool, made by the first pass and kept with it."""
    if "layer" not in s:
        from paper_2408_01890_b200 import binding as lb
        c, shape = s["case"], s["shape"]
        kind = lb.CACHE_STANDARD if s["kind"] == "standard" else lb.CACHE_SHARED
        s["lb"] = lb
        s["layer"] = lb.PagedLayer(kind, shape["Hkv"], c["page"], shape["d"], shape["r"] if s["kind"] == "shared" else 0,
                                   dtype=lb.S8 if c["fmt"] == "s8" else lb.E4M3, pool=s["pool"])
        if c["op"] == "anchor":
            s["workspace"] = lb.paged_decode_workspace(s["layer"], c["B"], shape["Hq"], c["L"])
        if c["op"] == "shared":
            s["workspace"] = lb.paged_decode_workspace(s["layer"], c["B"], shape["Hq"], c["L"])
            s["link"] = lb.Link(s["qp"], None, s["w1"], s["w2"], act=lb.ACT_RELU,
                                integrate=lb.INTEGRATE_CONCAT if c["shape"] == "paper" else lb.INTEGRATE_ADD)
    return s["lb"], s["layer"]


def _run_append(s):
    if own:
        lb, layer = _layer(s)
        lb.lisa_paged_append(layer, s["table"], s["k"], s["v"], s["before"], s["new"])
        lb.lisa_paged_read(layer, s["table"], s["first"], s["k_out"], s["v_out"], s["read"])
    else:
        _plain_append(s)
        _plain_read(s)
    return {"k": s["k_out"], "v": s["v_out"], "scales": _views(s["pool"], s["shape"], s["kind"], s["case"]["page"])[2]}


def _blocks(s, first, count, n):
    """The blocks of positions [first, first + count), count <= n: (touched, page, block of the page), all [B, blocks], and each of their
    positions relative to `first` [B, blocks, 16]."""
    P, table = s["case"]["page"], s["table"]
    nb = (n + 2 * BLOCK - 2) // BLOCK
    blk = first.long()[:, None] // BLOCK + torch.arange(nb, device="cuda")
    rel = blk[..., None] * BLOCK + torch.arange(BLOCK, device="cuda") - first.long()[:, None, None]
    touched = ((rel >= 0) & (rel < count.long()[:, None, None])).any(-1)
    page = table.gather(1, (blk * BLOCK // P).clamp(max=table.shape[1] - 1)).long()
    return touched, torch.where(touched, page, 0), blk % (P // BLOCK), rel


def _plain_append(s):
    c, fmt = s["case"], s["case"]["fmt"]
    touched, page, within, rel = _blocks(s, s["before"], s["new"], c["n"])
    is_new = ((rel >= 0) & (rel < s["new"].long()[:, None, None]))[:, :, None, :, None]
    is_old = (rel < 0)[:, :, None, :, None]
    views = _views(s["pool"], s["shape"], s["kind"], c["page"])
    row = torch.arange(c["B"], device="cuda")[:, None, None]
    for i, rows in enumerate((s["k"], s["v"])):
        x = rows[row, rel.clamp(0, c["n"] - 1)].float().transpose(2, 3)                # [B, blocks, H, 16, w]
        codes = views[i][page, within]
        grown = torch.where(is_new, x.abs(), 0).amax((3, 4)) / _largest(fmt, x)
        held = torch.where(is_old.any(3)[..., 0], views[2][page, within][..., i], 0)
        scale = torch.maximum(held, grown)
        scale = torch.where(scale.isfinite(), scale, torch.nan)
        some = (scale > 0)[..., None, None]
        kept = _codes(torch.where(some, _values(codes, fmt) * (held / scale)[..., None, None], 0), fmt)
        new = _codes(torch.where(some, x / scale[..., None, None], 0), fmt)
        codes = torch.where(is_new, new, torch.where(is_old, kept, codes))
        views[i].index_put_((page[touched], within[touched]), codes[touched])
        views[2][..., i].index_put_((page[touched], within[touched]), scale[touched])


def _plain_read(s):
    c = s["case"]
    n = c["n"] + BLOCK
    B = c["B"]
    touched, page, within, rel = _blocks(s, s["first"], s["read"], n)
    views = _views(s["pool"], s["shape"], s["kind"], c["page"])
    pos = torch.arange(n, device="cuda")
    valid = (pos < s["read"].long()[:, None])[..., None, None]
    for i, out in enumerate((s["k_out"], s["v_out"])):
        x = _values(views[i][page, within], c["fmt"]) * views[2][page, within][..., i][..., None, None]     # [B, blocks, H, 16, w]
        x = x.transpose(2, 3).flatten(1, 2)[:, :n]
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, n - x.shape[1]))
        out.copy_(torch.where(valid, x.to(out.dtype), out))


def _gather(s, i, dtype=torch.float32, rows=slice(None)):
    """The sequences' rows out of the pages, dequantised: [B, Hkv, L, width]."""
    c = s["case"]
    views = _views(s["pool"], s["shape"], s["kind"], c["page"])
    table = s["table"][rows].long()
    x = _values(views[i][table], c["fmt"], dtype) * views[2][table][..., i][..., None, None].to(dtype)     # [B, pages, blocks, H, 16, w]
    return x.flatten(1, 2).transpose(1, 2).flatten(2, 3)[:, :, :c["L"]]


def _scores(s, dtype=torch.float32, rows=slice(None)):
    """Pre-softmax scores [B, Hq, L] of the sequences `rows`."""
    c, shape = s["case"], s["shape"]
    Hq, Hkv, L = shape["Hq"], shape["Hkv"], c["L"]
    q = (s["q"] if c["op"] == "anchor" else s["qp"])[rows, 0].to(dtype)
    q = q.unflatten(1, (Hkv, Hq // Hkv))
    a = (q @ _gather(s, 0, dtype, rows).transpose(2, 3)).flatten(1, 2) / math.sqrt(q.shape[-1])
    if c["op"] == "anchor":
        return a
    prev = s["prev"][rows, :, :L].to(dtype)
    x = prev if c["shape"] != "paper" else torch.cat([prev, a], 1)
    y = ((x.transpose(1, 2) @ s["w1"].to(dtype)).relu() @ s["w2"].to(dtype)).transpose(1, 2)
    return y if c["shape"] == "paper" else y + a


def _attend_rows(s, dtype=torch.float32, rows=slice(None)):
    """(scores, o) of the sequences `rows`; a sequence without positions has o = 0."""
    c, shape = s["case"], s["shape"]
    a = _scores(s, dtype, rows)
    on = (torch.arange(c["L"], device="cuda") < s["lens"][rows, None])[:, None]
    z = torch.where(on, a, -torch.inf)
    p = torch.where(on, (z - z.amax(-1, keepdim=True)).exp(), 0)
    o = p.unflatten(1, (shape["Hkv"], -1)) @ _gather(s, 1, dtype, rows)
    den = p.sum(-1)[..., None]
    return a, on, torch.where(den > 0, o.flatten(1, 2) / torch.where(den > 0, den, 1), 0)


def _run_attend(s):
    c = s["case"]
    row = s.get("row")
    if own:
        lb, layer = _layer(s)
        lens = s["lens"] if c["ragged"] else None
        if c["op"] == "anchor":
            lb.lisa_attn_anchor_paged(s["q"], layer, s["table"], L=c["L"], seq_lens=lens, out=s["o"], out_scores=row, workspace=s["workspace"])
        else:
            lb.lisa_attn_shared_decode_paged(s["prev"], s["link"], layer, s["table"], L=c["L"], seq_lens=lens, out=s["o"], out_scores=row,
                                             workspace=s["workspace"])
    else:
        a, on, o = _attend_rows(s)
        s["o"].copy_(o[:, None])
        if row is not None:
            row[..., :c["L"]] = torch.where(on, a.to(row.dtype), row[..., :c["L"]])
    return {"o": s["o"]} if row is None else {"o": s["o"], "row": row}


def _pages(s):
    """The library's handles on the tables and the pools, made by the first pass and kept with them."""
    if "pages" not in s:
        from paper_2408_01890_b200 import binding as lb
        c, shape = s["case"], s["shape"]
        s["lb"] = lb
        s["cache"] = lb.PagedCache.of([lb.PagedLayer(lb.CACHE_STANDARD if k == "standard" else lb.CACHE_SHARED, shape["Hkv"], c["page"], shape["d"],
                                                     0 if k == "standard" else shape["r"], dtype=lb.S8 if c["fmt"] == "s8" else lb.E4M3, pool=p)
                                       for k, p in zip(s["kinds"], s["pools"])])
        s["pages"] = lb.Pages(s["table"], s["lens"], s["refs"], c["page"])
    return s["lb"], s["pages"], s["cache"]


def _run_beam(s):
    if own:
        lb, pages, cache = _pages(s)
        lb.lisa_pages_fork(pages, s["parent"])
        lb.lisa_pages_reserve(pages, cache, s["new"])
    else:
        _plain_fork(s)
        _plain_reserve(s)
    return {"table": s["table"], "lens": s["lens"], "refs": s["refs"], "pools": s["pools"]}


def _held(table, n_pages):
    """How many entries of the table name each page."""
    at = torch.where(table >= 0, table, n_pages).flatten().long()
    return torch.zeros(n_pages + 1, dtype=torch.int32, device="cuda").index_add_(0, at, torch.ones_like(at, dtype=torch.int32))[:n_pages]


def _plain_fork(s):
    """Row i takes over the pages and the length of row parent[i] (none where that is -1)."""
    parent, table, refs = s["parent"].long(), s["table"], s["refs"]
    taken = torch.where((parent >= 0)[:, None], table[parent.clamp(min=0)], -1)
    refs += _held(taken, refs.shape[0]) - _held(table, refs.shape[0])
    s["lens"].copy_(torch.where(parent >= 0, s["lens"][parent.clamp(min=0)], 0))
    table.copy_(taken)


def _plain_reserve(s):
    """Every row gets the pages that its next `new` positions need, the lowest free ones first, row by row; a partly filled page that
    others hold as well is exchanged for a copy (by all of its writers, or all but the last if nobody else holds it)."""
    table, refs, P = s["table"], s["refs"], s["case"]["page"]
    lens, new = s["lens"].long(), s["new"].long()
    B, slots = table.shape
    have, need = (lens + P - 1) // P, (lens + new + P - 1) // P
    last = torch.where((lens % P > 0) & (new > 0), table.gather(1, (have - 1).clamp(min=0)[:, None])[:, 0], -1).long()
    same = (last[:, None] == last[None]) & (last >= 0)[:, None]
    before = same.tril(-1).sum(1)
    copy = (last >= 0) & (refs[last.clamp(min=0)] - before > 1)
    wanted = copy.long() + need - have
    at = wanted.cumsum(0) - wanted
    free = torch.nonzero(refs == 0)[:, 0]
    if int(wanted.sum()) > free.numel():
        return
    slot = torch.arange(slots, device="cuda")
    fresh = (slot >= have[:, None]) & (slot < need[:, None])
    copied = copy[:, None] & (slot == have[:, None] - 1)
    which = at[:, None] + torch.where(copied, 0, copy.long()[:, None] + slot - have[:, None])
    taken = free[which.clamp(0, max(0, free.numel() - 1))]
    table.copy_(torch.where(fresh | copied, taken, table.long()).to(torch.int32))
    refs.index_add_(0, last[copy], torch.full_like(last[copy], -1, dtype=torch.int32))
    refs[taken[fresh | copied]] = 1
    src, dst = last[copy], taken[copied]
    for pool in s["pools"]:
        pool[dst] = pool[src]


def _run_compact(s):
    # the pool is fragmented again, as it was: the tables alone, the pages move from where they lie
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    if own:
        lb, pages, cache = _pages(s)
        lb.lisa_pages_compact(pages, cache)
    else:
        _plain_compact(s)
    return {"table": s["table"], "refs": s["refs"], "pools": s["pools"]}


def _plain_compact(s):
    """The pages in use that lie behind as many pages as are in use move into the free ones before, both in ascending order."""
    table, refs = s["table"], s["refs"]
    used = refs > 0
    n = int(used.sum())
    dst, src = torch.nonzero(~used[:n])[:, 0], torch.nonzero(used[n:])[:, 0] + n
    for pool in s["pools"]:
        pool[dst] = pool[src]
    to = torch.arange(refs.shape[0], device="cuda").index_put_((src,), dst)
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], -1))
    refs[dst] = refs[src]
    refs[src] = 0


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, shape = dict(case), SHAPES[case["shape"]]
    Hq, Hkv, d, P = shape["Hq"], shape["Hkv"], shape["d"], c["page"]
    share = (5 / 6) * (0.5625 if c.get("ragged") else 1.2)     # mean length over the longest
    if c["op"] == "append":
        kw = _layout(shape, c["kind"], P)[0]
        values = c["B"] * c["n"] * share * Hkv * (kw + d)
        return {"bytes": values * 2 + values + values + values * 2, "flops": 4 * values}
    if c["op"] in ("anchor", "shared"):
        kw = d if c["op"] == "anchor" else shape["r"]
        positions = c["B"] * c["L"] * share
        row = 0 if c["rows"] == "none" else 4 if c["rows"] == "f32" else 2
        bytes_ = positions * (Hkv * (kw + d + 8 / BLOCK) + Hq * row) + c["B"] * Hq * (kw + d) * 2
        flops = positions * Hq * 2 * (kw + d)
        if c["op"] == "shared":
            bytes_ += positions * Hq * (row or 4)
            flops += positions * 2 * shape["m"] * Hq * (3 if c["shape"] == "paper" else 2)
        return {"bytes": bytes_, "flops": flops}
    page = sum(_layout(shape, k, P)[3] for k in _kinds(c["layers"]))
    if c["op"] == "beam":
        K = c["beams"]
        distinct = K * (1 - (1 - 1 / K) ** K)               # beams that go on, of K drawn with replacement
        copies = c["groups"] * (K - distinct) * (c["L"] % P > 0)
        entries = c["groups"] * K * (-(-c["L"] // P))
        return {"bytes": 2 * copies * page + 3 * 4 * entries, "flops": entries}
    per_row = -(-c["L"] // P)
    ended = sum(b % 5 < 2 for b in range(c["B"]))
    held, all_ = (c["B"] - ended) * per_row, c["B"] * per_row
    moved = held * (1 - held / (all_ + 5))                  # pages in use lie anywhere in the pool
    return {"bytes": 2 * moved * page + 3 * 4 * c["B"] * per_row, "flops": moved}


# ------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    c = dict(case)
    if c["op"] in ("beam", "compact"):
        return None
    s = prepare(case, seed)
    if c["op"] == "append":
        return _exact_append(s)
    row = s.get("row")
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device="cuda")
    out = None if row is None else row.double()
    for b in range(c["B"]):
        n = int(s["lens"][b])
        if n == 0:
            continue
        o[b, 0], a = _exact_sequence(s, b, n)
        if out is not None:
            out[b, :, :n] = a
    return {"o": o} if out is None else {"o": o, "row": out}


def _exact_cached(s, b, i, n):
    """[Hkv, n, width] of sequence b."""
    c = s["case"]
    views = _views(s["pool"], s["shape"], s["kind"], c["page"])
    page = s["table"][b, :-(-n // c["page"])].long()
    x = _values(views[i][page], c["fmt"], torch.float64)
    x = torch.einsum("pbhtw,pbh->hpbtw", x, views[2][page][..., i].double())
    return x.reshape(x.shape[0], -1, x.shape[-1])[:, :n]


def _exact_sequence(s, b, n):
    c, shape = s["case"], s["shape"]
    K, V = _exact_cached(s, b, 0, n), _exact_cached(s, b, 1, n)
    G = shape["Hq"] // shape["Hkv"]
    q = (s["q"] if c["op"] == "anchor" else s["qp"])[b, 0].double()
    a = torch.einsum("hx,hnx->hn", q, K.repeat_interleave(G, 0)) * q.shape[-1] ** -0.5
    if c["op"] == "shared":
        prev = s["prev"][b, :, :n].double()
        w1, w2 = s["w1"].double(), s["w2"].double()
        if c["shape"] == "paper":
            hidden = torch.einsum("hn,hu->un", prev, w1[:shape["Hq"]]) + torch.einsum("hn,hu->un", a, w1[shape["Hq"]:])
            a = torch.einsum("un,ug->gn", hidden.clamp(min=0), w2)
        else:
            a = a + torch.einsum("un,ug->gn", torch.einsum("hn,hu->un", prev, w1).clamp(min=0), w2)
    return torch.einsum("hn,hnx->hx", torch.softmax(a, -1), V.repeat_interleave(G, 0)), a


def _exact_append(s):
    """A sequence at a time: the rows that the touched blocks hold afterwards, in 64 bits, each block's scale from its largest value."""
    c = s["case"]
    fmt, P, top = c["fmt"], c["page"], 127.0 if c["fmt"] == "s8" else 448.0
    views = _views(s["pool"], s["shape"], s["kind"], P)
    scales = views[2].double()
    outs = [s["k_out"].double(), s["v_out"].double()]
    for b in range(c["B"]):
        n, at = int(s["new"][b]), int(s["before"][b]) % BLOCK
        if n == 0:
            continue
        nb = -(-(at + n) // BLOCK)
        blk = int(s["first"][b]) // BLOCK + torch.arange(nb, device="cuda")
        page, within = s["table"][b, blk * BLOCK // P].long(), blk % (P // BLOCK)
        for i, rows in enumerate((s["k"], s["v"])):
            H, w = rows.shape[2:]
            held = scales[page[0], within[0], :, i].clone()                                        # [H]
            old = _values(views[i][page[0], within[0]], fmt, torch.float64)[:, :at]                # [H, at, w]
            x = torch.zeros((nb * BLOCK, H, w), dtype=torch.float64, device="cuda")
            x[at:at + n] = rows[b, :n].double()
            x = x.view(nb, BLOCK, H, w)
            scale = x.abs().amax((1, 3)) / top                                                     # [nb, H]
            if at:
                scale[0] = torch.maximum(scale[0], held)
                x[0, :at] = (old * held[:, None, None]).transpose(0, 1)
            y = x / scale[:, None, :, None]
            y = y.round() if fmt == "s8" else y.clamp(-448, 448).to(torch.float8_e4m3fn).double()
            outs[i][b, :at + n] = (y * scale[:, None, :, None]).view(-1, H, w)[:at + n]
            scales[page, within, :, i] = scale
    return {"k": outs[0], "v": outs[1], "scales": scales}
