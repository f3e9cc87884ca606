"""The operators of a compressed model's decode step: FC layers with 4-bit weights, attention of
one new token over a paged cache of keys and values, and the care of that cache's pages.

A case is a dict of plain values.  Its "kind" says what one pass is:
  q4       one FC layer with 4-bit weights and group scales, feature-major activations
  q4prep   the weights of a pruned layer quantised to 4 bits and read back
  attn     the new token's key and value of every sequence written into the cache, and its
           attention over the sequence's pages
  beam     one step of a beam search: sequences fork to the beams that go on, and each gets
           room for its next token (a shared last page is copied)
  compact  sequences end, and the pages that are left move to the front of the cache
Where `own` is false a pass is computed in elementary torch operations, in 32 bits.
"""

import math
import random

import torch

own = False

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f32": 4}


def _q4(name, rows, cols, batch, group, dt="bf16", out="bf16", bias=True, relu=False):
    return {"name": name, "kind": "q4", "rows": rows, "cols": cols, "batch": batch, "group": group, "dt": dt, "out": out,
            "bias": bias, "relu": relu}


def _attn(name, batch, ctx, kv, heads, dim, page, dt="bf16", slots_first=False, ragged=True, empty=0, window=0):
    return {"name": name, "kind": "attn", "batch": batch, "ctx": ctx, "kv": kv, "heads": heads, "dim": dim, "page": page,
            "dt": dt, "slots_first": slots_first, "ragged": ragged, "empty": empty, "window": window}


def listed():
    return [
        # a classifier of 1000 classes for one token, in single precision: the smallest call,
        # where latency counts
        _q4("q4_1000x2048_b1_f32", 1000, 2048, 1, 32, "f32", "f32"),
        # one layer of a large fully connected stack for one token: reading the weights is all
        _q4("q4_4096_b1", 4096, 4096, 1, 128),
        # a few sequences, odd sizes everywhere (ragged last group, tile and row), fp32 scores
        _q4("q4_4099x1003_b13_f32out", 4099, 1003, 13, 32, "bf16", "f32"),
        # the widening layer of a feed-forward block for 64 sequences
        _q4("q4_16384x4096_b64_relu", 16384, 4096, 64, 64, relu=True),
        # preparing layers for deployment: a column-pruned conv layer, and a dense fp32 FC layer
        {"name": "q4prep_512x4608_pruned", "kind": "q4prep", "rows": 512, "cols": 4608, "group": 64, "dt": "bf16", "rate": 4},
        {"name": "q4prep_4096_f32", "kind": "q4prep", "rows": 4096, "cols": 4096, "group": 128, "dt": "f32", "rate": 1},
        # the first tokens of one short conversation: latency
        _attn("attn_b1_ctx77_d64", 1, 77, 2, 8, 64, 16),
        # ordinary serving: 32 conversations of different lengths, four query heads a key head
        _attn("attn_b32_ctx2048_ragged", 32, 2048, 8, 32, 128, 16),
        # one very long document
        _attn("attn_b1_ctx131072", 1, 131072, 8, 64, 128, 64, ragged=False),
        # single precision, a key head per query head, odd pages, a sliding window whose old
        # pages are gone, sequences without a token
        _attn("attn_b7_ctx1531_window_f32", 7, 1531, 12, 12, 80, 7, "f32", True, True, 2, 1000),
        # 8 prompts whose 4 beams each go on, 12 layers: four beams copy each prompt's last page
        {"name": "beam_8x4_layers12", "kind": "beam", "parents": 8, "beams": 4, "ctx": 700, "layers": 12, "kv": 8,
         "dim": 128, "page": 16, "dt": "bf16", "slots_first": False, "tokens": 1},
        # half of 96 sequences end; what is left moves to the front (8 layers)
        {"name": "compact_96_layers8", "kind": "compact", "seqs": 96, "ctx": 640, "ended": 48, "layers": 8, "kv": 8,
         "dim": 128, "page": 16, "dt": "bf16", "slots_first": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any sizes between the listed ones, odd ones among them."""
    kind = rng.choice(["q4"] * 4 + ["q4prep"] + ["attn"] * 5 + ["beam", "compact"])
    dt = rng.choice(["bf16"] * 3 + ["f32"])
    if kind == "q4":
        c = _q4("", _log(rng, 48, 16384), _log(rng, 48, 16384), _log(rng, 1, 64), rng.choice([32, 64, 128]), dt,
                "f32" if dt == "f32" else rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.7, rng.random() < 0.4)
        while c["rows"] * c["cols"] > 1 << 26:
            c["rows"] = c["rows"] // 2 + 1
        if rng.random() < 0.5:   # half of the layers have round sizes, as most models' do
            c["rows"], c["cols"] = (128 * (c[k] // 256 * 2 + 1) for k in ("rows", "cols"))
    elif kind == "q4prep":
        c = {"kind": kind, "rows": _log(rng, 32, 4096), "cols": _log(rng, 32, 4608), "group": rng.choice([32, 64, 128]),
             "dt": dt, "rate": rng.choice([1, 2, 4, 8])}
    elif kind == "attn":
        kv = rng.choice([1, 2, 4, 8, 8, 12])
        heads = kv * rng.choice([1, 1, 2, 3, 4, 4, 6, 8, 8, 16])
        c = _attn("", _log(rng, 1, 64), _log(rng, 1, 131072), kv, heads, rng.choice([64, 64, 80, 96, 128, 128, 128, 256]),
                  rng.choice([1, 7, 16, 16, 16, 32, 64, 100, 256]), dt, rng.random() < 0.4, rng.random() < 0.7)
        while c["batch"] > 1 and _attn_bytes(c) > 4e8:
            c["batch"] = c["batch"] // 2
        while _attn_bytes(c) > 4e8:
            c["ctx"] = c["ctx"] // 2 + 1
        c["empty"] = rng.randint(0, c["batch"] // 4)
        c["window"] = rng.choice([0, 0, 0, max(1, c["ctx"] // 3)])
    elif kind == "beam":
        c = {"kind": kind, "parents": _log(rng, 1, 12), "beams": rng.randint(2, 5), "ctx": _log(rng, 20, 700),
             "layers": _log(rng, 1, 16), "kv": rng.choice([1, 2, 4, 8]), "dim": rng.choice([64, 80, 128]),
             "page": rng.choice([7, 16, 16, 32, 64]), "dt": dt, "slots_first": rng.random() < 0.4,
             "tokens": rng.choice([1, 1, 1, 4, 9])}
    else:
        c = {"kind": kind, "seqs": _log(rng, 4, 96), "ctx": _log(rng, 20, 640), "ended": 0, "layers": _log(rng, 1, 8),
             "kv": rng.choice([1, 2, 4, 8]), "dim": rng.choice([64, 80, 128]), "page": rng.choice([7, 16, 16, 32, 64]),
             "dt": dt, "slots_first": rng.random() < 0.4}
        c["ended"] = max(1, int(c["seqs"] * rng.uniform(0.2, 0.8)))
        c["layers"] = max(1, c["layers"] // (2 if dt == "f32" else 1))
    c.pop("name", None)
    return c


# ---- what the sizes of a case say ----------------------------------------------------------

def _lens(case):
    """Cached tokens of every sequence, by the case alone (the new token of "attn" included)."""
    rng = random.Random(case["ctx"])
    if case["kind"] == "attn":
        n = [case["ctx"]] + [rng.randint(1, case["ctx"]) if case["ragged"] else case["ctx"]
                             for _ in range(case["batch"] - 1)]
        return n[:len(n) - case["empty"]] + [0] * case["empty"]
    if case["kind"] == "beam":   # the prompts, then the beams, which begin empty
        return [rng.randint(case["ctx"] // 2, case["ctx"]) for _ in range(case["parents"])] + \
            [0] * (case["parents"] * case["beams"])
    return [rng.randint(1, case["ctx"]) for _ in range(case["seqs"])]


def _seen(case):
    """Tokens that each sequence of an "attn" case attends to."""
    return [min(n, case["window"]) if case["window"] else n for n in _lens(case)]


def _attn_bytes(c):
    return 2 * sum(_seen({**c, "empty": 0, "window": 0})) * c["kv"] * c["dim"] * ESIZE[c["dt"]]


def _ceil(a, b):
    return -(-a // b)


def _groups(case):
    return _ceil(case["cols"], case["group"])


def _rows16(case):
    return _ceil(case["rows"], 16) * 16


def _code_stride(case):
    """Bytes of a row of codes: two to a byte, rows begin at multiples of 16."""
    return _ceil(_ceil(case["cols"], 2), 16) * 16


def work(case):
    kind = case["kind"]
    if kind in ("q4", "q4prep"):
        rows, cols = case["rows"], case["cols"]
        packed = rows * _ceil(cols, 2) + 2 * rows * _groups(case)
        if kind == "q4prep":   # weights and mask in, codes and scales out and in, weights out
            return {"bytes": rows * cols * (2 * ESIZE[case["dt"]] + (case["rate"] > 1)) + 2 * packed,
                    "flops": 4.0 * rows * cols}
        io = case["batch"] * (cols * ESIZE[case["dt"]] + rows * ESIZE[case["out"]]) + 4 * rows * case["bias"]
        return {"bytes": packed + io, "flops": 2.0 * rows * cols * case["batch"]}
    e = ESIZE[case["dt"]]
    if kind == "attn":
        row = case["kv"] * case["dim"] * e
        io = case["batch"] * (2 * case["heads"] * case["dim"] * e + 4 * case["heads"]) + 4 * case["batch"] * row
        return {"bytes": 2 * sum(_seen(case)) * row + io + 4 * sum(_ceil(n, case["page"]) for n in _seen(case)),
                "flops": 4.0 * sum(_seen(case)) * case["heads"] * case["dim"]}
    slot = 2 * case["layers"] * case["kv"] * case["dim"] * e   # a token's keys and values in all layers
    if kind == "beam":
        lens = _lens(case)[:case["parents"]]
        copied = case["beams"] * sum(n % case["page"] for n in lens)
        tables = 2 * 4 * case["beams"] * sum(_ceil(n, case["page"]) for n in lens)
        return {"bytes": 2 * copied * slot + tables + 8, "flops": 0}
    pages = [_ceil(n, case["page"]) for n in _lens(case)]
    left = sum(pages) * (case["seqs"] - case["ended"]) // case["seqs"]
    moved = left * case["ended"] // case["seqs"]   # live pages are spread evenly
    return {"bytes": 2 * moved * case["page"] * slot + 4 * 3 * sum(pages), "flops": 0}


# ---- inputs ------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(gen, *shape, dt="f32", scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(TORCH[dt])


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _tables(case, lens, gen, spare):
    """Page table of sequences of these lengths, whose pages lie anywhere in the cache; the number
    of pages; references to each."""
    page = case["page"]
    most = max(max(lens) + case.get("tokens", 0), 1)
    width, total = _ceil(most, page), sum(_ceil(n, page) for n in lens)
    pages = total + spare
    order = torch.randperm(pages, generator=gen, device="cuda")[:total]
    need = (_ints(lens) + page - 1) // page
    used = torch.arange(width, device="cuda")[None, :] < need[:, None]
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    table[used] = order.to(torch.int32)
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[order] = 1
    return table, pages, refs


def _cache(case, planes, pages, gen):
    inner = (case["page"], case["kv"]) if case["slots_first"] else (case["kv"], case["page"])
    data = torch.empty(planes, pages, *inner, case["dim"], dtype=TORCH[case["dt"]], device="cuda")
    for plane in data:
        plane.normal_(generator=gen)
    return data


def _activations(gen, case, heads):
    """[batch, heads, dim] of the library's feature-major activations."""
    fm = _randn(gen, heads * case["dim"], case["batch"], dt=case["dt"])
    return fm.view(heads, case["dim"], case["batch"]).permute(2, 0, 1)


def prepare(case, seed):
    gen, kind = _gen(seed), case["kind"]
    s = {"case": case}
    if kind in ("q4", "q4prep"):
        w = _randn(gen, case["rows"], case["cols"], scale=math.sqrt(2.0 / case["cols"]))
        codes = torch.zeros(case["rows"], _code_stride(case), dtype=torch.uint8, device="cuda")
        scales = torch.zeros(_groups(case), _rows16(case), dtype=torch.bfloat16, device="cuda")
        if kind == "q4prep":
            w = w.to(TORCH[case["dt"]])
            mask = None
            if case["rate"] > 1:   # whole columns kept and removed in blocks of 16 rows
                keep = torch.rand(_ceil(case["rows"], 16), case["cols"], generator=gen, device="cuda") * case["rate"] < 1
                mask = keep.repeat_interleave(16, 0)[:case["rows"]].to(torch.uint8).contiguous()
            return {**s, "w": w, "mask": mask, "codes": codes, "scales": scales, "back": torch.empty_like(w)}
        _quantize(w, None, case["group"], codes, scales)
        # activations inside a network
        return {**s, "codes": codes, "scales": scales, "x": _randn(gen, case["cols"], case["batch"], dt=case["dt"]),
                "bias": _randn(gen, case["rows"], scale=0.1) if case["bias"] else None,
                "y": torch.empty(case["rows"], case["batch"], dtype=TORCH[case["out"]], device="cuda")}
    lens = _lens(case)
    if kind == "attn":
        table, pages, _ = _tables(case, lens, gen, 3)
        if case["window"]:   # pages that no window reaches again have been given back
            gone = (_ints(lens) - case["window"]).clamp(min=0) // case["page"]
            table[torch.arange(table.shape[1], device="cuda")[None, :] < gone[:, None]] = -1
        fm = torch.empty(case["heads"] * case["dim"], case["batch"], dtype=TORCH[case["dt"]], device="cuda")
        s.update(table=table, lens=_ints(lens), pos=_ints([n - 1 for n in lens]), data=_cache(case, 2, pages, gen),
                 q=_activations(gen, case, case["heads"]), k=_activations(gen, case, case["kv"]),
                 v=_activations(gen, case, case["kv"]), y=fm.view(case["heads"], case["dim"], -1).permute(2, 0, 1),
                 lse=torch.empty(case["batch"], case["heads"], device="cuda"))
    else:
        n = case["parents"] * case["beams"] if kind == "beam" else 0
        spare = n * (2 + _ceil(case["tokens"], case["page"])) if kind == "beam" else 5
        table, pages, refs = _tables(case, lens, gen, spare)
        # what the tables were before the pass, and the ones that the pass changes
        before = torch.cat([table.flatten(), _ints(lens), refs])
        s.update(before=before, now=before.clone(), shape=table.shape, pages=pages,
                 data=_cache(case, 2 * case["layers"], pages, gen))
        if kind == "beam":   # beam j of prompt i
            s["parents"] = _ints([i // case["beams"] for i in range(n)])
            s["children"] = _ints([case["parents"] + i for i in range(n)])
            s.update(counts=_ints([case["tokens"]] * n), pos=torch.empty(n, dtype=torch.int32, device="cuda"))
        else:
            s["ended"] = torch.randperm(case["seqs"], generator=gen, device="cuda")[:case["ended"]].to(torch.int32)
            s["info"] = torch.empty(2, dtype=torch.int32, device="cuda")
    if own:   # the handle and the scratch memory that a program keeps
        import paper_2111_11581_amd as B
        cache = B.CacheShape.of(s["data"][0], B.SLOT_MAJOR if case["slots_first"] else B.HEAD_MAJOR)
        need = B.bsp_attention_workspace(cache, case["batch"], case["heads"], s["table"].shape[1]) if kind == "attn" else \
            B.bsp_cache_scratch(cache, *s["shape"], max(1, case.get("parents", 0) * case.get("beams", 0)))
        s.update(cache=cache, scratch=torch.empty(need, dtype=torch.uint8, device="cuda"))
    return s


# ---- the plain forms: 4-bit weights --------------------------------------------------------------

def _quantize(w, mask, group, codes, scales):
    rows, cols = w.shape
    n = scales.shape[0]
    w = w.float() if mask is None else torch.where(mask != 0, w.float(), 0.0)
    w = torch.nn.functional.pad(w, (0, n * group - cols)).view(rows, n, group)
    s = (w.abs().amax(2) / 7.0).to(torch.bfloat16)
    scales[:, :rows] = s.t()
    q = torch.where(s[..., None] == 0, 0.0, torch.round(w / s.float()[..., None]).clamp(-7, 7))
    q = torch.nn.functional.pad((q + 8).view(rows, -1)[:, :cols].to(torch.uint8), (0, 2 * codes.shape[1] - cols))
    codes.copy_(q[:, 0::2] | (q[:, 1::2] << 4))


def _dequantize(codes, scales, rows, cols, group):
    q = torch.stack([codes & 15, codes >> 4], 2).view(rows, -1)[:, :cols].float() - 8.0
    return q * scales[:, :rows].float().t().repeat_interleave(group, 1)[:, :cols]


# ---- the plain forms: attention --------------------------------------------------------------------

def _plain_append(case, data, table, pos, k, v):
    at = (pos >= 0).nonzero()[:, 0]
    where = pos[at].long()
    page = table[at, where // case["page"]].long()
    slot = where % case["page"]
    for plane, new in ((data[0], k), (data[1], v)):
        if case["slots_first"]:
            plane[page, slot] = new[at]
        else:
            plane[page, :, slot] = new[at]


def _tokens(case, plane, table):
    """[batch, kv, tokens, dim] in 32 bits of the pages in the table."""
    t = plane[table.clamp(min=0).long()]   # [batch, width, ...]
    t = t.permute(0, 3, 1, 2, 4) if case["slots_first"] else t.permute(0, 2, 1, 3, 4)
    return t.float().reshape(t.shape[0], case["kv"], -1, case["dim"])


def _plain_attention(case, q, data, table, lens, y, lse):
    batch, kv, dim = case["batch"], case["kv"], case["dim"]
    k = _tokens(case, data[0], table)
    qt = q.float().reshape(batch, kv, -1, dim).transpose(2, 3).contiguous()
    s = torch.matmul(k, qt) * (1.0 / math.sqrt(dim))   # [batch, kv, tokens, group]
    del k
    at = torch.arange(s.shape[2], device="cuda")[None, :]
    valid = (at < lens[:, None]) & (table >= 0).repeat_interleave(case["page"], 1)
    if case["window"]:
        valid &= at >= lens[:, None] - case["window"]
    s = s.masked_fill(~valid[:, None, :, None], -math.inf)
    top = s.amax(2, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(s - top)
    total = p.sum(2, keepdim=True)
    o = torch.matmul(p.transpose(2, 3).contiguous(), _tokens(case, data[1], table))
    o = torch.where(total.transpose(2, 3) > 0, o / total.transpose(2, 3), 0.0)
    y.copy_(o.reshape(batch, -1, dim))
    lse.copy_((top + torch.log(total)).reshape(batch, -1))


# ---- the plain forms: pages ------------------------------------------------------------------------

def _views(state, flat):
    """Table, lengths and references in one array."""
    seqs, width = state["shape"]
    return flat[:seqs * width].view(seqs, width), flat[seqs * width:seqs * width + seqs], flat[seqs * width + seqs:]


def _count(refs, entries, by):
    refs.index_add_(0, entries.clamp(min=0).flatten(), torch.where(entries >= 0, by, 0).to(torch.int32).flatten())


def _plain_fork(table, lens, refs, parents, children):
    new, old = table[parents], table[children]
    _count(refs, new, 1)
    _count(refs, old, -1)
    table[children] = new
    lens[children] = lens[parents]


def _plain_extend(case, data, table, lens, refs, rows, counts, pos):
    page, width = case["page"], table.shape[1]
    have = lens[rows]
    part, last = have % page, (have // page).clamp(max=width - 1)
    old = table[rows, last]
    shared = (counts > 0) & (part > 0) & (refs[old.clamp(min=0)] > 1)
    start, end = (have + page - 1) // page, (have + counts + page - 1) // page
    need = torch.where(counts > 0, end - start, 0) + shared.int()
    first = need.cumsum(0) - need
    free = torch.sort((refs > 0).to(torch.uint8), stable=True).indices.to(torch.int32)   # lowest free page first
    ok = (need.sum() <= (refs == 0).sum()) & (end.max() <= width)
    entry = torch.arange(width, device="cuda", dtype=torch.int32)[None, :]
    fresh = (counts[:, None] > 0) & (entry >= start[:, None]) & (entry < end[:, None])
    copied = shared[:, None] & (entry == last[:, None])
    rank = first[:, None] + torch.where(copied, 0, shared[:, None].int() + entry - start[:, None])
    given = free[rank.clamp(0, free.numel() - 1).long()]
    taken = (fresh | copied) & ok
    i = (shared & ok).nonzero()[:, 0]
    src, dst = old[i].long(), given[i, last[i].long()].long()
    slot = torch.arange(page, device="cuda")
    used = slot[None, :] < part[i][:, None]
    used = used[None, :, :, None, None] if case["slots_first"] else used[None, :, None, :, None]
    data[:, dst] = torch.where(used, data[:, src], data[:, dst])
    _count(refs, torch.where(taken, given, -1), 1)
    _count(refs, torch.where(shared & ok, old, -1), -1)
    table[rows] = torch.where(taken, given, table[rows])
    pos.copy_(torch.where(ok, have, -1))
    lens[rows] = have + torch.where(ok, counts, 0)


def _plain_release(table, lens, refs, rows):
    _count(refs, table[rows], -1)
    table[rows] = -1
    lens[rows] = 0


def _plain_compact(data, table, refs, info):
    live, ids = refs > 0, torch.arange(refs.numel(), device="cuda")
    used = live.sum()
    src, dst = (live & (ids >= used)).nonzero()[:, 0], (~live & (ids < used)).nonzero()[:, 0]
    data[:, dst] = data[:, src]
    ids[src] = dst
    table.copy_(torch.where(table >= 0, ids[table.clamp(min=0)].to(torch.int32), -1))
    refs[dst] = refs[src]
    refs[src] = 0
    info.copy_(torch.stack([used, torch.full_like(used, src.numel())]))


# ---- one pass ----------------------------------------------------------------------------------------

def _own_run(case, st):
    import paper_2111_11581_amd as B
    code = {"bf16": B.BF16, "f32": B.F32}
    kind = case["kind"]
    if kind == "q4":
        B.bsp_q4_linear(case["rows"], case["cols"], case["group"], case["batch"], code[case["dt"]], code[case["out"]],
                        st["x"], st["codes"], st["scales"], st["bias"], case["relu"], st["y"])
    elif kind == "q4prep":
        shape = (case["rows"], case["cols"], case["group"], code[case["dt"]])
        B.bsp_q4_quantize(*shape, st["w"], st["mask"], st["codes"], st["scales"])
        B.bsp_q4_dequantize(*shape, st["codes"], st["scales"], st["back"])
    elif kind == "attn":
        keys, values = st["data"][0], st["data"][1]
        B.bsp_cache_append(st["cache"], st["k"], st["v"], keys, values, st["table"], st["pos"])
        B.bsp_attention(st["cache"], st["q"], keys, values, st["table"], st["lens"], st["y"],
                        1.0 / math.sqrt(case["dim"]), window=case["window"], lse=st["lse"], workspace=st["scratch"])
    else:
        st["now"].copy_(st["before"])
        table, lens, refs = _views(st, st["now"])
        if kind == "beam":
            B.bsp_cache_fork(table, lens, refs, st["parents"], st["children"], st["scratch"])
            B.bsp_cache_extend(st["cache"], st["data"], table, lens, refs, st["children"], st["counts"], st["pos"],
                               st["scratch"])
        else:
            B.bsp_cache_release(table, lens, refs, st["ended"])
            B.bsp_cache_compact(st["cache"], st["data"], table, refs, st["info"], st["scratch"])


def _plain_run(case, st):
    kind = case["kind"]
    if kind == "q4":
        y = torch.matmul(_dequantize(st["codes"], st["scales"], case["rows"], case["cols"], case["group"]), st["x"].float())
        y = y if st["bias"] is None else y + st["bias"][:, None]
        st["y"].copy_(y.clamp(min=0) if case["relu"] else y)
    elif kind == "q4prep":
        _quantize(st["w"], st["mask"], case["group"], st["codes"], st["scales"])
        st["back"].copy_(_dequantize(st["codes"], st["scales"], case["rows"], case["cols"], case["group"]))
    elif kind == "attn":
        _plain_append(case, st["data"], st["table"], st["pos"], st["k"], st["v"])
        _plain_attention(case, st["q"], st["data"], st["table"], st["lens"], st["y"], st["lse"])
    else:
        st["now"].copy_(st["before"])
        table, lens, refs = _views(st, st["now"])
        if kind == "beam":
            _plain_fork(table, lens, refs, st["parents"], st["children"])
            _plain_extend(case, st["data"], table, lens, refs, st["children"], st["counts"], st["pos"])
        else:
            _plain_release(table, lens, refs, st["ended"])
            _plain_compact(st["data"], table, refs, st["info"])


def _outputs(case, st):
    """What a pass leaves behind: the cache and its tables are outputs where it writes them.  Codes
    are given as the weights that they stand for."""
    if case["kind"] == "q4":
        return {"y": st["y"]}
    if case["kind"] == "q4prep":
        return {"weights": st["back"], "scales": st["scales"]}
    if case["kind"] == "attn":
        return {"y": st["y"], "lse": st["lse"], "cache": st["data"]}
    table, lens, refs = _views(st, st["now"])
    more = {"pos": st["pos"]} if case["kind"] == "beam" else {"info": st["info"]}
    return {"table": table, "lens": lens, "refs": refs, "cache": st["data"], **more}


def run(state):
    (_own_run if own else _plain_run)(state["case"], state)
    return _outputs(state["case"], state)


# ---- the same in 64 bits, sequence by sequence ----------------------------------------------------------

def _exact_weights(st, case):
    """Weights of the codes, from their definition."""
    r = torch.arange(case["rows"], device="cuda")[:, None]
    k = torch.arange(case["cols"], device="cuda")[None, :]
    n = (st["codes"][r, k // 2].to(torch.int64) >> (4 * (k % 2))) % 16
    return (n - 8).double() * st["scales"].double()[k // case["group"], r]


def _exact_q4prep(st, case):
    w = st["w"].double() * (1 if st["mask"] is None else st["mask"].double())
    rows, cols, g = case["rows"], case["cols"], case["group"]
    scales, out = torch.zeros_like(st["scales"], dtype=torch.float64), torch.zeros_like(w)
    for i, c in enumerate(range(0, cols, g)):
        block = w[:, c:c + g]
        s = (block.abs().max(1).values / 7).to(torch.bfloat16).double()
        scales[i, :rows] = s
        out[:, c:c + g] = torch.where(s[:, None] > 0, (block / s[:, None]).round().clamp(-7, 7) * s[:, None], 0.0)
    return {"weights": out, "scales": scales}


def _exact_attn(st, case):
    page, group, dim = case["page"], case["heads"] // case["kv"], case["dim"]
    data = st["data"].double()
    keys, values = (p if case["slots_first"] else p.transpose(1, 2) for p in (data[0], data[1]))   # [page, slot, kv, dim]
    table, lens = st["table"].tolist(), st["lens"].tolist()
    y = torch.zeros(case["batch"], case["heads"], dim, dtype=torch.float64, device="cuda")
    lse = torch.full((case["batch"], case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        if not n:
            continue
        p, slot = table[b][(n - 1) // page], (n - 1) % page
        keys[p, slot], values[p, slot] = st["k"][b].double(), st["v"][b].double()
        at = torch.arange(max(0, n - case["window"]) if case["window"] else 0, n, device="cuda")
        own_pages = st["table"][b].long()[at // page]
        k, v = keys[own_pages, at % page], values[own_pages, at % page]   # [tokens, kv, dim]
        for j in range(case["kv"]):
            s = (k[:, j] @ st["q"][b, j * group:(j + 1) * group].double().t()) / math.sqrt(dim)
            lse[b, j * group:(j + 1) * group] = torch.logsumexp(s, 0)
            y[b, j * group:(j + 1) * group] = torch.softmax(s, 0).t() @ v[:, j]
    return {"y": y, "lse": lse, "cache": data}


def _exact_pages(st, case):
    table, lens, refs = (v.tolist() for v in _views(st, st["before"]))
    data, page = st["data"].double(), case["page"]
    if case["kind"] == "beam":
        parents, children, pos = st["parents"].tolist(), st["children"].tolist(), []
        for p, c in zip(parents, children):   # no beam is a prompt, so one after the other
            table[c], lens[c] = list(table[p]), lens[p]
            for e in table[c]:
                if e >= 0:
                    refs[e] += 1
        at_first = list(refs)
        free = iter([i for i, n in enumerate(at_first) if n == 0])
        for c in children:
            n, more = lens[c], case["tokens"]
            if n % page and at_first[table[c][n // page]] > 1:
                src, dst = table[c][n // page], next(free)
                for s in range(n % page):
                    if case["slots_first"]:
                        data[:, dst, s] = data[:, src, s]
                    else:
                        data[:, dst, :, s] = data[:, src, :, s]
                table[c][n // page], refs[dst] = dst, 1
                refs[src] -= 1
            for e in range(_ceil(n, page), _ceil(n + more, page)):
                table[c][e] = next(free)
                refs[table[c][e]] = 1
            pos.append(n)
            lens[c] = n + more
        extra = {"pos": _ints(pos)}
    else:
        for r in st["ended"].tolist():
            for e in table[r]:
                if e >= 0:
                    refs[e] -= 1
            table[r], lens[r] = [-1] * len(table[r]), 0
        used = sum(n > 0 for n in refs)
        src = [i for i, n in enumerate(refs) if n > 0 and i >= used]
        dst = [i for i, n in enumerate(refs) if n == 0 and i < used]
        to = dict(zip(src, dst))
        for a, b in to.items():
            data[:, b] = data[:, a]
            refs[a], refs[b] = 0, refs[a]
        table = [[to.get(e, e) for e in row] for row in table]
        extra = {"info": _ints([used, len(src)])}
    return {"table": _ints(table), "lens": _ints(lens), "refs": _ints(refs), "cache": data, **extra}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "q4":
        y = _exact_weights(st, case) @ st["x"].double()
        y = y if st["bias"] is None else y + st["bias"].double()[:, None]
        return {"y": torch.relu(y) if case["relu"] else y}
    return {"q4prep": _exact_q4prep, "attn": _exact_attn}.get(case["kind"], _exact_pages)(st, case)
