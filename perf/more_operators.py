"""The operators around a compressed model's FC layers when many continuations of one prompt are
sampled together: rotary positions with norms of queries and keys, attention of sequences that share
their first tokens, and the choice of the next token.

A case is a dict of plain values.  Its "kind" says what one pass is:
  rope     queries and keys of n tokens normed by head and rotated by their positions; with "append"
           the keys and values go into a paged cache, else it is one array [tokens, heads, dim]
  prefix   attention of one new token of every sequence over a paged cache, where the sequences of a
           group share the pages of their first tokens
  sample   one token of every row of logits, after temperature, top-k, top-p and min-p, from given
           random numbers
Where `own` is false a pass is computed in elementary torch operations: in 32 bits, and in 64 the
angles of rotations and the sums that a token is chosen by.
"""

import math
import random

import numpy as np
import torch

own = False

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f32": 4}
EPS = 1e-6   # of the norms


def _rope(name, n, heads, kv, dim, rot, layout="half", dt="bf16", append=True, norm=True, scaling="", start=0, seqs=1,
          page=16, slots_first=False, fm=False, skipped=0):
    return {"name": name, "kind": "rope", "n": n, "heads": heads, "kv": kv, "dim": dim, "rot": rot, "layout": layout, "dt": dt,
            "append": append, "norm": norm, "scaling": scaling, "start": start, "seqs": seqs, "page": page,
            "slots_first": slots_first, "fm": fm, "skipped": skipped}


def _prefix(name, groups, batch, shared, own_tokens, kv, heads, dim, page, dt="bf16", slots_first=False, ragged=True, empty=0,
            window=0):
    return {"name": name, "kind": "prefix", "groups": groups, "batch": batch, "shared": shared, "own": own_tokens, "kv": kv,
            "heads": heads, "dim": dim, "page": page, "dt": dt, "slots_first": slots_first, "ragged": ragged, "empty": empty,
            "window": window}


def _sample(name, batch, vocab, cut, dt="f32", fm=True, masked=False, spread=3.0):
    return {"name": name, "kind": "sample", "batch": batch, "vocab": vocab, "cut": cut, "dt": dt, "fm": fm, "masked": masked,
            "spread": spread}


def listed():
    return [
        # one token of one short conversation: the smallest call, where latency counts
        _rope("rope_b1_d64", 1, 8, 2, 64, 64, norm=False, start=77),
        # one token of each of 32 conversations, feature-major as the FC layers leave it, norms of
        # queries and keys, long contexts by a scaled rotation
        _rope("rope_b32_d128_norm", 32, 32, 8, 128, 128, scaling="turns", start=30000, seqs=32, fm=True),
        # a prompt of odd length, pairs side by side
        _rope("rope_prompt4097_interleaved", 4097, 32, 8, 128, 128, "interleaved", scaling="index"),
        # single precision, part of an odd head rotated, far positions, one array (no cache)
        _rope("rope_far_f32_part", 1003, 12, 12, 80, 40, dt="f32", append=False, scaling="linear", start=900000),
        # four beams of a short prompt: latency
        _prefix("prefix_4x100_d64", 1, 4, 100, 20, 2, 8, 64, 16),
        # 32 continuations of one prompt, four query heads a key head
        _prefix("prefix_32x4096", 1, 32, 4096, 256, 8, 32, 128, 16),
        # several prompts with their continuations, of different numbers and lengths
        _prefix("prefix_8groups_61", 8, 61, 2000, 500, 8, 32, 128, 64, slots_first=True, empty=3),
        # single precision, a key head per query head, odd pages, a sliding window
        _prefix("prefix_3groups_f32_window", 3, 11, 900, 400, 12, 12, 80, 7, "f32", window=1000, empty=1),
        # a long document that 64 continuations share, eight query heads a key head
        _prefix("prefix_64x32768", 1, 64, 32768, 128, 8, 64, 128, 64, ragged=False),
        # one token from a small vocabulary
        _sample("sample_1x1000", 1, 1000, "p"),
        # a few rows of an odd vocabulary, scores in half the bytes (ties everywhere), masked tokens
        _sample("sample_13x49999_bf16", 13, 49999, "kpm", "bf16", fm=False, masked=True),
        # a batch over a large vocabulary, all cuts
        _sample("sample_64x131072", 64, 131072, "kpm"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any sizes between the listed ones, odd ones among them."""
    kind = rng.choice(["rope", "prefix", "sample"])
    dt = rng.choice(["bf16", "bf16", "f32"])
    kv = rng.choice([1, 2, 4, 8, 8, 12])
    heads = kv * rng.choice([1, 1, 2, 3, 4, 4, 6, 8])
    dim = rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
    if kind == "rope":
        append = rng.random() < 0.75
        n = _log(rng, 1, 4097)
        while n * heads * dim * ESIZE[dt] > 1 << 25:
            n = n // 2 + 1
        c = _rope("", n, heads, kv, dim, rng.choice([dim, dim, dim, dim // 2, dim // 4, 2 * rng.randint(1, dim // 2)]),
                  rng.choice(["half", "half", "interleaved"]), dt, append, rng.random() < 0.5,
                  rng.choice(["", "", "linear", "turns", "index"]), rng.choice([0, _log(rng, 1, 900000)]),
                  n if n <= 64 and rng.random() < 0.7 else rng.randint(1, min(4, n)), rng.choice([1, 7, 16, 16, 16, 64, 100]),
                  rng.random() < 0.4, rng.random() < (0.7 if n <= 64 else 0.2), rng.choice([0, 0, n // 7]))
    elif kind == "prefix":
        batch = _log(rng, 1, 64)
        c = _prefix("", rng.choice([1, 1, 1, rng.randint(1, min(8, batch))]), batch, _log(rng, 1, 32768), _log(rng, 1, 600),
                    kv, heads, dim, rng.choice([1, 7, 16, 16, 16, 32, 64, 100]), dt, rng.random() < 0.4, rng.random() < 0.7)
        # no more operations than the largest listed case, which fp32 reaches eight times sooner
        while 4.0 * c["batch"] * c["heads"] * c["dim"] * (c["shared"] + c["own"]) * (8 if dt == "f32" else 1) > 6.9e10 or \
                2.0 * (c["groups"] * c["shared"] + c["batch"] * c["own"]) * kv * dim * ESIZE[dt] > 2.6e8:
            c["shared"], c["own"] = c["shared"] // 2 + 1, c["own"] // 2 + 1
        c["empty"] = rng.randint(0, c["batch"] // 4)
        c["window"] = rng.choice([0, 0, 0, max(1, (c["shared"] + c["own"]) // 2)])
    else:
        c = _sample("", _log(rng, 1, 64), _log(rng, 100, 131072), rng.choice(["", "k", "p", "m", "kp", "kpm", "kpm"]), dt,
                    rng.random() < 0.6, rng.random() < 0.3, rng.choice([1.0, 2.0, 3.0, 3.0, 5.0]))
    c.pop("name", None)
    return c


# ---- what the sizes of a case say ----------------------------------------------------------

def _ceil(a, b):
    return -(-a // b)


def _tokens(case):
    """(sequence, position) of every token of a "rope" case; the skipped ones have position -1."""
    n, seqs = case["n"], case["seqs"]
    rng = random.Random(n)
    # one token a sequence: sequences of different lengths; else stretches of prompts
    at = [(i, case["start"] + rng.randint(0, case["page"])) for i in range(n)] if seqs == n else \
        [(i * seqs // n, case["start"] + i - _ceil(i * seqs // n * n, seqs)) for i in range(n)]
    for i in rng.sample(range(n), case["skipped"]):
        at[i] = (at[i][0], -1)
    return at


def _groups(case):
    """Of a "prefix" case: where groups begin in the batch, their shared tokens, every length."""
    rng = random.Random(case["shared"] * 64 + case["batch"])
    cuts = sorted(rng.sample(range(1, case["batch"]), case["groups"] - 1))
    starts = [0] + cuts + [case["batch"]]
    shared = [rng.randint(_ceil(case["shared"], 4), case["shared"]) if g and case["ragged"] else case["shared"]
              for g in range(case["groups"])]
    lens = []
    for g in range(case["groups"]):
        for _ in range(starts[g], starts[g + 1]):
            lens.append(shared[g] + (rng.randint(1, case["own"]) if case["ragged"] else case["own"]))
    for b in rng.sample(range(case["batch"]), case["empty"]):
        lens[b] = 0
    return starts, shared, lens


def _first(case, n):
    return max(0, n - case["window"]) if case["window"] else 0


def work(case):
    kind = case["kind"]
    if kind == "sample":
        n = case["batch"] * case["vocab"]
        return {"bytes": n * ESIZE[case["dt"]] + 28 * case["batch"], "flops": 4.0 * n}
    e = ESIZE[case["dt"]]
    row = case["kv"] * case["dim"] * e
    if kind == "rope":
        put = sum(p >= 0 for _, p in _tokens(case)) if case["append"] else 0
        q = case["n"] * case["heads"] * case["dim"]
        k = case["n"] * case["kv"] * case["dim"] if case["append"] else 0
        return {"bytes": 2 * q * e + 2 * k * e + 2 * put * row + 8 * case["n"], "flops": (3.0 + 4.0 * case["norm"]) * (q + k)}
    starts, shared, lens = _groups(case)
    read = 0   # tokens whose keys and values have to be read
    for g, s in enumerate(shared):
        members = [n for n in lens[starts[g]:starts[g + 1]] if n]
        if members:
            read += max(0, min(s, max(members)) - min(_first(case, n) for n in members))
            read += sum(max(0, n - max(s, _first(case, n))) for n in members)
    seen = sum(n - _first(case, n) for n in lens)
    return {"bytes": 2 * read * row + case["batch"] * case["heads"] * (2 * case["dim"] * e + 4) + 4 * _ceil(read, case["page"]),
            "flops": 4.0 * seen * case["heads"] * case["dim"]}


# ---- what a program has in hand --------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _randn(gen, *shape, scale=1.0, dt="f32"):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(TORCH[dt])


def _array(gen, case, n, heads, fill=True):
    """[n, heads, dim], feature-major underneath or token by token."""
    shape = (heads, case["dim"], n) if case.get("fm", True) else (n, heads, case["dim"])
    a = _randn(gen, *shape, dt=case["dt"]) if fill else torch.empty(shape, dtype=TORCH[case["dt"]], device="cuda")
    return a.permute(2, 0, 1) if case.get("fm", True) else a


def _cache(case, pages, gen):
    inner = (case["page"], case["kv"]) if case["slots_first"] else (case["kv"], case["page"])
    data = torch.empty(2, pages, *inner, case["dim"], dtype=TORCH[case["dt"]], device="cuda")
    for plane in data:
        plane.normal_(generator=gen)
    return data


# (factor, tokens that the model was trained with, low, high) of the ways to lengthen a context
SCALING = {"linear": (4.0, 0.0, 0.0, 0.0), "turns": (8.0, 8192.0, 1.0, 4.0), "index": (4.0, 32768.0, 1.0, 32.0)}
BASE = 500000.0


def _attention_factor(case):
    return 0.1 * math.log(SCALING["index"][0]) + 1.0 if case["scaling"] == "index" else 1.0


def _freqs(case):
    """Radians that every pair turns by a token, in 64 bits."""
    rot = case["rot"]
    f = [BASE ** (-2.0 * i / rot) for i in range(rot // 2)]
    if not case["scaling"]:
        return f
    factor, length, low, high = SCALING[case["scaling"]]
    if case["scaling"] == "linear":
        keep = [0.0] * len(f)
    elif case["scaling"] == "turns":
        keep = [min(max((length * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]
    else:
        def index(turns):
            return rot * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(BASE))
        a, b = max(math.floor(index(high)), 0), min(math.ceil(index(low)), rot - 1)
        b = b if b != a else a + 0.001
        keep = [1.0 - min(max((i - a) / (b - a), 0.0), 1.0) for i in range(len(f))]
    return [x * (r + (1 - r) / factor) for x, r in zip(f, keep)]


def _prepare_rope(case, seed):
    gen = _gen(seed)
    s = {"case": case, "q": _array(gen, case, case["n"], case["heads"]), "q_out": _array(gen, case, case["n"], case["heads"], False)}
    at = _tokens(case)
    s["pos"], s["rows"] = _ints([p for _, p in at]), _ints([r for r, _ in at])
    for name in ("q_norm", "k_norm"):
        s[name] = 1 + _randn(gen, case["dim"], scale=0.2) if case["norm"] else None
    if case["append"]:
        s["k"], s["v"] = (_array(gen, case, case["n"], case["kv"]) for _ in range(2))
        entries = sorted({(r, p // case["page"]) for r, p in at if p >= 0})
        width = max([e for _, e in entries], default=0) + 1
        pages = len(entries) + 2   # of what lies before the tokens only the places in the table are there
        order = torch.randperm(pages, generator=gen, device="cuda")[:len(entries)].to(torch.int32)
        s["table"] = torch.full((case["seqs"], width), -1, dtype=torch.int32, device="cuda")
        if entries:
            where = torch.tensor(entries, device="cuda")
            s["table"][where[:, 0], where[:, 1]] = order
        s["data"] = _cache(case, pages, gen)
    if own:
        import paper_2111_11581_amd as B
        s["rope"] = B.Rope(B.ROPE_HALF if case["layout"] == "half" else B.ROPE_INTERLEAVED, case["rot"], _attention_factor(case))
        scaling = None
        if case["scaling"]:
            ramp = {"linear": B.RAMP_NONE, "turns": B.RAMP_TURNS, "index": B.RAMP_INDEX}[case["scaling"]]
            scaling = B.RopeScaling(*SCALING[case["scaling"]], ramp)
        s["freqs"] = torch.tensor(B.bsp_rope_freqs(case["rot"], BASE, scaling), dtype=torch.float64, device="cuda")
        if case["append"]:
            s["cache"] = B.CacheShape.of(s["data"][0], B.SLOT_MAJOR if case["slots_first"] else B.HEAD_MAJOR)
    else:
        s["freqs"] = torch.tensor(_freqs(case), dtype=torch.float64, device="cuda")
    return s


def _prepare_prefix(case, seed):
    gen = _gen(seed)
    starts, shared, lens = _groups(case)
    page, width = case["page"], _ceil(max(max(lens), max(shared)), case["page"])
    rows, used = [[-1] * width for _ in lens], 0
    for g, s in enumerate(shared):
        whole = s // page   # full pages are shared; a last page that is not full each sequence has for itself
        first = list(range(used, used + whole))
        used += whole
        for b in range(starts[g], starts[g + 1]):
            mine = max(0, _ceil(lens[b], page) - whole)
            rows[b][:whole + mine] = first + list(range(used, used + mine))
            used += mine
    pages = used + 3
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    rows = torch.tensor(rows, device="cuda")
    table = torch.where(rows >= 0, order[rows.clamp(min=0)], -1)
    for g in range(case["groups"]):
        if case["window"]:   # pages that no window reaches again have been given back
            alive = [_first(case, n) for n in lens[starts[g]:starts[g + 1]] if n]
            table[starts[g]:starts[g + 1], :min(alive, default=0) // page] = -1
    fm = torch.empty(case["heads"] * case["dim"], case["batch"], dtype=TORCH[case["dt"]], device="cuda")
    s = {"case": case, "table": table, "lens": _ints(lens), "data": _cache(case, pages, gen),
         "q": _array(gen, case, case["batch"], case["heads"]), "y": fm.view(case["heads"], case["dim"], -1).permute(2, 0, 1),
         "lse": torch.empty(case["batch"], case["heads"], device="cuda"), "starts": _ints(starts),
         # what is shared in whole pages, as a fork and the copy of its last page leave it
         "shared": _ints([n // page * page for n in shared])}
    if own:
        import paper_2111_11581_amd as B
        s["cache"] = B.CacheShape.of(s["data"][0], B.SLOT_MAJOR if case["slots_first"] else B.HEAD_MAJOR)
        need = B.bsp_attention_prefix_workspace(s["cache"], case["batch"], case["heads"], case["groups"], width)
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    else:
        s["members"] = [(starts[g], starts[g + 1], shared[g] // page * page) for g in range(case["groups"])]
    return s


def _prepare_sample(case, seed):
    gen, n, vocab = _gen(seed), case["batch"], case["vocab"]
    x = _randn(gen, n, vocab, scale=case["spread"])
    x.scatter_add_(1, torch.randint(vocab, (n, 4), generator=gen, device="cuda"), 2 * case["spread"] * torch.rand(n, 4, generator=gen, device="cuda"))
    if case["masked"]:   # a grammar allows some tokens only; one row none
        x.masked_fill_(torch.rand(n, vocab, generator=gen, device="cuda") < 0.3, -math.inf)
        x[n // 2] = x[n // 2] if n == 1 else -math.inf
    x = x.to(TORCH[case["dt"]])

    def rand(lo, hi):
        return lo + (hi - lo) * torch.rand(n, generator=gen, device="cuda")
    temperature = rand(0.5, 1.3)
    if n > 4:   # one row asks for the likeliest token
        temperature[3] = 0.0
    s = {"case": case, "logits": x.t().contiguous().t() if case["fm"] else x, "temperature": temperature, "u": rand(0, 1),
         "top_k": torch.randint(0, 200, (n,), generator=gen, device="cuda").to(torch.int32) if "k" in case["cut"] else None,
         "top_p": rand(0.6, 1.0) if "p" in case["cut"] else None, "min_p": rand(0.0, 0.1) if "m" in case["cut"] else None,
         "tokens": torch.empty(n, dtype=torch.int32, device="cuda"), "logp": torch.empty(n, device="cuda")}
    if own:
        import paper_2111_11581_amd as B
        s["workspace"] = torch.empty(B.bsp_sample_workspace(n, vocab), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    return {"rope": _prepare_rope, "prefix": _prepare_prefix, "sample": _prepare_sample}[case["kind"]](case, seed)


# ---- the plain forms -------------------------------------------------------------------------

def _pairs(case):
    """Dimensions of the first and of the second half of every rotated pair."""
    i = torch.arange(case["rot"] // 2, device="cuda")
    return (2 * i, 2 * i + 1) if case["layout"] == "interleaved" else (i, i + case["rot"] // 2)


def _plain_rotate(case, st, x, norm):
    x = x.float()
    if norm is not None:
        x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + EPS) * norm
    angle = st["pos"].double()[:, None] * st["freqs"]
    cos, sin = ((f(angle).float() * _attention_factor(case))[:, None] for f in (torch.cos, torch.sin))
    first, second = _pairs(case)
    a, b = x[:, :, first], x[:, :, second]
    y = x.clone()
    y[:, :, first], y[:, :, second] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_rope(case, st):
    st["q_out"].copy_(_plain_rotate(case, st, st["q"], st["q_norm"]))
    if case["append"]:
        at = (st["pos"] >= 0).nonzero()[:, 0]
        pos = st["pos"][at].long()
        page, slot = st["table"][st["rows"][at].long(), pos // case["page"]].long(), pos % case["page"]
        k = _plain_rotate(case, st, st["k"], st["k_norm"]).to(TORCH[case["dt"]])
        for plane, new in ((st["data"][0], k[at]), (st["data"][1], st["v"][at])):
            if case["slots_first"]:
                plane[page, slot] = new
            else:
                plane[page, :, slot] = new


def _pages(case, plane, table):
    """[rows of the table, kv, tokens, dim] in 32 bits."""
    t = plane[table.clamp(min=0).long()]
    t = t.permute(0, 3, 1, 2, 4) if case["slots_first"] else t.permute(0, 2, 1, 3, 4)
    return t.float().reshape(t.shape[0], case["kv"], -1, case["dim"])


def _valid(case, table, lens, begin):
    """[rows, tokens] from token `begin` on: which of them a sequence attends to."""
    at = begin + torch.arange(table.shape[1] * case["page"], device="cuda")[None, :]
    ok = (at < lens[:, None]) & (table >= 0).repeat_interleave(case["page"], 1)
    return ok & (at >= lens[:, None] - case["window"]) if case["window"] else ok


def _plain_prefix(case, st):
    kv, dim, page = case["kv"], case["dim"], case["page"]
    group = case["heads"] // kv
    for lo, hi, shared in st["members"]:
        m, table, lens = hi - lo, st["table"][lo:hi], st["lens"][lo:hi]
        cut = shared // page
        q = st["q"][lo:hi].float().reshape(m, kv, group, dim) / math.sqrt(dim)
        parts = []
        if cut:   # the shared pages once, for the queries of all members
            k, v = (_pages(case, p, table[:1, :cut])[0] for p in (st["data"][0], st["data"][1]))
            qs = q.permute(1, 3, 0, 2).reshape(kv, dim, m * group).contiguous()
            s = torch.matmul(k, qs).reshape(kv, -1, m, group)
            ok = _valid(case, table[:1, :cut].expand(m, -1), lens, 0)
            s = s.masked_fill(~ok.t()[None, :, :, None], -math.inf)
            parts.append((s.permute(2, 0, 3, 1), v, True))
        if cut < table.shape[1]:
            k, v = (_pages(case, p, table[:, cut:]) for p in (st["data"][0], st["data"][1]))
            s = torch.matmul(k, q.transpose(2, 3).contiguous()).transpose(2, 3)   # [m, kv, group, tokens]
            ok = _valid(case, table[:, cut:], lens, shared)
            parts.append((s.masked_fill(~ok[:, None, None, :], -math.inf), v, False))
        top = torch.stack([s.amax(3) for s, _, _ in parts]).amax(0)[..., None]
        top = torch.where(top == -math.inf, 0.0, top)
        total, out = 0.0, 0.0
        for s, v, common in parts:
            p = torch.exp(s - top)
            total = total + p.sum(3, keepdim=True)
            if common:
                o = torch.matmul(p.permute(1, 0, 2, 3).reshape(kv, m * group, -1), v)
                out = out + o.reshape(kv, m, group, dim).transpose(0, 1)
            else:
                out = out + torch.matmul(p.contiguous(), v)
        out = torch.where(total > 0, out / total, 0.0)
        st["y"][lo:hi] = out.reshape(m, -1, dim).to(st["y"].dtype)
        st["lse"][lo:hi] = (top + torch.log(total)).reshape(m, -1)


def _plain_sample(case, st):
    n, vocab = case["batch"], case["vocab"]
    x = st["logits"].double()
    greedy = st["temperature"] <= 0
    t = torch.where(greedy, 1.0, st["temperature"].double())[:, None]
    top = x.amax(1, keepdim=True)
    none = top[:, 0] == -math.inf
    w = torch.exp((x - torch.where(top == -math.inf, 0.0, top)) / t)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices   # equal ones: the lowest index first
    ranked = w.gather(1, order)
    rank = torch.arange(vocab, device="cuda")[None, :]
    live = rank < (x > -math.inf).sum(1, keepdim=True)
    keep = live
    if st["top_k"] is not None:
        k = st["top_k"][:, None]
        keep = keep & ((k <= 0) | (rank < k))
    if st["top_p"] is not None:
        mass = torch.where(keep, ranked, 0.0)
        before = mass.cumsum(1) - mass
        keep = keep & ((before < st["top_p"].double()[:, None] * mass.sum(1, keepdim=True)) | (rank == 0))
    if st["min_p"] is not None:
        keep = keep & (ranked >= st["min_p"].double()[:, None])
    keep = keep & (~greedy[:, None] | (rank == 0)) & live
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ranked, 0.0))
    upto = kept.cumsum(1)
    total = upto[:, -1:]
    token = (upto <= st["u"].double()[:, None] * total).sum(1, keepdim=True).clamp(max=vocab - 1)
    logp = torch.log(kept.gather(1, token) / total)[:, 0]
    st["tokens"].copy_(torch.where(none, -1, token[:, 0]))
    st["logp"].copy_(torch.where(none, -math.inf, logp))


# ---- one pass --------------------------------------------------------------------------------

def _own_run(case, st):
    import paper_2111_11581_amd as B
    code = {"bf16": B.BF16, "f32": B.F32}
    if case["kind"] == "sample":
        B.bsp_sample(code[case["dt"]], st["logits"], st["u"], st["tokens"], st["temperature"], st["top_k"], st["top_p"],
                     st["min_p"], st["logp"], st["workspace"])
    elif case["kind"] == "prefix":
        B.bsp_attention_prefix(st["cache"], st["q"], st["data"][0], st["data"][1], st["table"], st["lens"], st["starts"],
                               st["shared"], st["y"], 1.0 / math.sqrt(case["dim"]), window=case["window"], lse=st["lse"],
                               workspace=st["workspace"])
    elif case["append"]:
        B.bsp_cache_append_rotary(st["cache"], st["rope"], st["freqs"], st["q"], st["k"], st["v"], st["q_out"], st["data"][0],
                                  st["data"][1], st["table"], st["pos"], st["rows"], st["q_norm"], st["k_norm"], EPS)
    else:
        B.bsp_rotary(code[case["dt"]], st["rope"], st["freqs"], st["q"], st["pos"], st["q_out"], st["q_norm"], EPS)


def run(state):
    """One pass; the cache is an output where it is written."""
    case = state["case"]
    (_own_run if own else {"rope": _plain_rope, "prefix": _plain_prefix, "sample": _plain_sample}[case["kind"]])(case, state)
    if case["kind"] == "sample":
        return {"tokens": state["tokens"], "logp": state["logp"]}
    if case["kind"] == "prefix":
        return {"y": state["y"], "lse": state["lse"]}
    return {"q": state["q_out"], **({"cache": state["data"]} if case["append"] else {})}


# ---- the same in 64 bits, from the definitions -----------------------------------------------

def _exact_rotate(case, x, norm, pos):
    """Pair by pair as complex numbers."""
    y = x.double().clone()
    if norm is not None:
        y = y / (y.square().mean(2, keepdim=True) + EPS).sqrt() * norm.double()
    half = case["rot"] // 2
    for i, f in enumerate(_freqs(case)):
        a, b = (2 * i, 2 * i + 1) if case["layout"] == "interleaved" else (i, i + half)
        turned = torch.complex(y[:, :, a], y[:, :, b]) * torch.polar(torch.full_like(pos, _attention_factor(case)), pos * f)[:, None]
        y[:, :, a], y[:, :, b] = turned.real, turned.imag
    return y


def _exact_rope(case, st):
    pos = st["pos"].double()
    out = {"q": _exact_rotate(case, st["q"], st["q_norm"], pos)}
    if case["append"]:
        data, k, v = st["data"].double(), _exact_rotate(case, st["k"], st["k_norm"], pos), st["v"].double()
        planes = data if case["slots_first"] else data.transpose(2, 3)   # [2, page, slot, kv, dim]
        table = st["table"].tolist()
        for i, (r, p) in enumerate(_tokens(case)):
            if p >= 0:
                planes[0, table[r][p // case["page"]], p % case["page"]] = k[i]
                planes[1, table[r][p // case["page"]], p % case["page"]] = v[i]
        out["cache"] = data
    return out


def _exact_prefix(case, st):
    page, group = case["page"], case["heads"] // case["kv"]
    y = torch.zeros(case["batch"], case["heads"], case["dim"], dtype=torch.float64, device="cuda")
    lse = torch.full((case["batch"], case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    keys, values = (p if case["slots_first"] else p.transpose(1, 2) for p in (st["data"][0], st["data"][1]))
    for b, n in enumerate(st["lens"].tolist()):   # every sequence by its own table, as if nothing were shared
        at = torch.arange(_first(case, n), n, device="cuda")
        if n == 0:
            continue
        mine = st["table"][b].long()[at // page]
        k, v = keys[mine, at % page].double(), values[mine, at % page].double()   # [tokens, kv, dim]
        for j in range(case["kv"]):
            s = (st["q"][b, j * group:(j + 1) * group].double() @ k[:, j].t()) / math.sqrt(case["dim"])
            lse[b, j * group:(j + 1) * group] = torch.logsumexp(s, 1)
            y[b, j * group:(j + 1) * group] = torch.softmax(s, 1) @ v[:, j]
    return {"y": y, "lse": lse}


def _exact_sample(case, st):
    x, u, t = (st[k].double().cpu().numpy() for k in ("logits", "u", "temperature"))
    cut = {k: None if st[k] is None else st[k].double().cpu().numpy() for k in ("top_k", "top_p", "min_p")}
    tokens, logp = np.full(len(x), -1), np.full(len(x), -np.inf)
    for b, row in enumerate(x):
        best = row.max()
        if best == -np.inf:
            continue
        if t[b] <= 0:
            tokens[b], logp[b] = row.argmax(), 0.0
            continue
        order = np.lexsort((np.arange(len(row)), -row))
        order = order[row[order] > -np.inf]
        if cut["top_k"] is not None and cut["top_k"][b] > 0:
            order = order[:int(cut["top_k"][b])]
        w = np.exp((row[order] - best) / t[b])
        n = len(order)
        if cut["top_p"] is not None:
            n = min(n, max(1, int(np.searchsorted(np.cumsum(w), cut["top_p"][b] * w.sum())) + 1))
        if cut["min_p"] is not None:
            n = min(n, max(1, int((w >= cut["min_p"][b]).sum())))
        by_index = np.sort(order[:n])
        w = np.exp((row[by_index] - best) / t[b])
        i = min(int(np.searchsorted(np.cumsum(w), u[b] * w.sum(), side="right")), n - 1)
        tokens[b], logp[b] = by_index[i], np.log(w[i] / w.sum())
    return {"tokens": _ints(tokens.tolist()), "logp": torch.from_numpy(logp).cuda()}


def exact(case, seed):
    return {"rope": _exact_rope, "prefix": _exact_prefix, "sample": _exact_sample}[case["kind"]](case, prepare(case, seed))
