"""A small decoder over compressed weights, as the decode operators are used together: FC layers pruned
and quantised to 4 bits, keys and values in a paged cache, a beam search whose beams share pages, and
sampling of several continuations of a prompt, which share its pages and read them together.

    python -m paper_2111_11581_amd.decode [--prompts 4] [--beams 4] [--tokens 32] [--dtype bf16] ...
    python -m paper_2111_11581_amd.decode --samples 16 [--temperature 0.8] [--top-k 50] [--top-p 0.95] [--min-p 0] ...

Weights are random (this is a program to read and to time, not a model).  Activations are
feature-major [features][sequences], as the FC layers take them; attention reads and writes them in
place by strides.  A step never waits for the device.
"""

from __future__ import annotations

import argparse
import math
import time

import torch

from . import BF16, COL, F32, Scheme, bsp_prune
from .layers import TORCH_DT, PagedCache, QuantLayer, Rotary, Sampler


class Decoder:
    """``layers`` of attention and a ReLU feed-forward part, with RMS norms and learned positions, or with
    ``rotary`` positions and norms of queries and keys by head."""

    def __init__(self, layers=2, heads=8, kv_heads=2, head_dim=64, ffn=1024, vocab=1000, longest=512, group=64,
                 rate=2, dtype: int = BF16, seed=0, rotary: Rotary | None = None):
        self.heads, self.kv_heads, self.head_dim, self.vocab, self.longest = heads, kv_heads, head_dim, vocab, longest
        self.dtype, self.torch_dtype = dtype, TORCH_DT[dtype]
        gen = torch.Generator(device="cuda").manual_seed(seed)
        hidden, inner = heads * head_dim, (heads + 2 * kv_heads) * head_dim

        def randn(*shape, scale):
            return torch.randn(*shape, device="cuda", generator=gen) * scale

        def layer(rows, cols):
            w = randn(rows, cols, scale=1 / math.sqrt(cols)).to(self.torch_dtype)
            mask = None
            if rate > 1:   # of every block of 16 rows and 64 columns, one column in `rate` is kept
                mask = torch.empty(rows * cols, dtype=torch.uint8, device="cuda")
                bsp_prune(Scheme(rows, cols, 16, 64, COL, rate), dtype, w, mask)
            return QuantLayer(rows, cols, group, dtype, w, mask)

        self.embedding = randn(vocab, hidden, scale=1.0)
        self.places = randn(longest, hidden, scale=0.5)
        self.blocks = [{"qkv": layer(inner, hidden), "out": layer(hidden, hidden), "up": layer(ffn, hidden),
                        "down": layer(hidden, ffn)} for _ in range(layers)]
        self.head = layer(vocab, hidden)
        self.rotary = rotary
        if rotary is not None:
            for block in self.blocks:
                block.update(q_norm=1 + randn(head_dim, scale=0.2), k_norm=1 + randn(head_dim, scale=0.2))

    def cache(self, seqs: int, pages: int, page_size: int = 16) -> PagedCache:
        return PagedCache(len(self.blocks), seqs, -(-self.longest // page_size), pages, page_size, self.kv_heads,
                          self.head_dim, self.dtype)

    def _linear(self, layer, x, relu=False, out_dt=None):
        out_dt = self.dtype if out_dt is None else out_dt
        y = torch.empty(layer.rows, x.shape[1], dtype=TORCH_DT[out_dt], device="cuda")
        layer.linear(x, y, x.shape[1], self.dtype, out_dt, relu=relu)
        return y

    def _norm(self, x):
        return (x * torch.rsqrt(x.square().mean(0, keepdim=True) + 1e-6)).to(self.torch_dtype)

    def step(self, cache: PagedCache, tokens, rows, groups=None):
        """One more token of each of the sequences rows (int32, on the device, as tokens); -> fp32
        logits [vocab][sequences] of the tokens after them.  groups: (starts, shared, prefix_rows) of
        sequences that share their first tokens, as PagedCache.attend_prefix takes them."""
        n, h, d = tokens.numel(), self.heads, self.head_dim
        pos = torch.empty_like(rows)
        cache.extend(rows, torch.ones_like(rows), pos)
        x = self.embedding[tokens]   # the residual, in fp32
        if self.rotary is None:
            x = x + self.places[pos.clamp(0, self.longest - 1)]
        x = x.t().contiguous()

        def split(a):   # [heads * dim][sequences] as [sequences, heads, dim]
            return a.view(-1, d, n).permute(2, 0, 1)

        for i, block in enumerate(self.blocks):
            qkv = self._linear(block["qkv"], self._norm(x))
            q, k, v = (split(a) for a in qkv.split([h * d, self.kv_heads * d, self.kv_heads * d]))
            if self.rotary is None:
                cache.append(i, k, v, pos, rows)
            else:
                cache.append_rotary(i, self.rotary, q, k, v, q, pos, rows, block["q_norm"], block["k_norm"])
            seen = torch.empty(h * d, n, dtype=self.torch_dtype, device="cuda")
            if groups is None:
                cache.attend(i, q, split(seen), 1 / math.sqrt(d), rows)
            else:
                starts, shared, prefix_rows = groups
                cache.attend_prefix(i, q, split(seen), 1 / math.sqrt(d), starts, shared, rows, prefix_rows)
            x = x + self._linear(block["out"], seen)
            x = x + self._linear(block["down"], self._linear(block["up"], self._norm(x), relu=True))
        return self._linear(self.head, self._norm(x), out_dt=F32)


def ints(values) -> torch.Tensor:
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _check(model: Decoder, prompts, new, each: int, what: str):
    n = len(prompts)
    if n == 0 or each < 1 or len(new) != n or min(new) < 1 or min(map(len, prompts)) < 1:
        raise ValueError(f"{what} needs prompts of at least one token, and at least one new token for each")
    if max(len(p) + t for p, t in zip(prompts, new)) > model.longest + 1:
        raise ValueError(f"sequences are limited to {model.longest} tokens")


def _read(model: Decoder, cache: PagedCache, prompts, rows):
    """The prompts, a token of each at a time, in sequences rows; -> logits [prompts][vocab] after their last tokens."""
    last = [None] * len(prompts)
    for t in range(max(map(len, prompts))):
        on = [i for i, p in enumerate(prompts) if t < len(p)]
        logits = model.step(cache, ints([prompts[i][t] for i in on]), ints([rows[i] for i in on]))
        for j, i in enumerate(on):
            if t == len(prompts[i]) - 1:
                last[i] = logits[:, j]
    return torch.stack(last)


def sample(model: Decoder, prompts, new, samples: int, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0,
           min_p: float = 0.0, seed: int = 0, page_size: int = 16):
    """``samples`` continuations of every prompt (a list of tokens), new[i] tokens of prompt i; -> tokens (per
    prompt [samples][new[i]]), the log probabilities that they were drawn with (the same) and the cache."""
    _check(model, prompts, new, samples, "sample")
    n = len(prompts)
    if n * samples > 1024:
        raise ValueError("sample draws up to 1024 continuations, which attention over shared prefixes takes at a time")
    pages = sum(-(-len(p) // page_size) + samples * (-(-t // page_size) + 2) for p, t in zip(prompts, new))
    cache = model.cache(n * (1 + samples), pages, page_size)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    sampler = Sampler(n * samples, model.vocab)

    def draw(logits):   # [rows, vocab]
        m = logits.shape[0]
        tokens, logp = torch.empty(m, dtype=torch.int32, device="cuda"), torch.empty(m, device="cuda")

        def each(value, dtype=torch.float32):
            return torch.full((m,), value, dtype=dtype, device="cuda")
        sampler.sample(logits, torch.rand(m, generator=gen, device="cuda"), tokens, F32, each(temperature),
                       each(top_k, torch.int32) if top_k > 0 else None, each(top_p) if top_p < 1 else None,
                       each(min_p) if min_p > 0 else None, logp)
        return tokens, logp

    def rows_of(running):
        return ints([n + i * samples + j for i in running for j in range(samples)])

    # every prompt once, in the sequence of its number; its continuations share its pages
    tokens, logp = draw(_read(model, cache, prompts, range(n)).repeat_interleave(samples, 0))
    cache.fork(ints(list(range(n))).repeat_interleave(samples), rows_of(range(n)))
    running, found = list(range(n)), [None] * n
    history, weights = tokens.view(n, samples, 1), logp.view(n, samples, 1)
    for made in range(1, max(new) + 1):
        ended = [i for i in running if new[i] == made]
        if ended:
            for i in ended:
                found[i] = (history[running.index(i)], weights[running.index(i)])
            cache.release(torch.cat([rows_of(ended), ints(ended)]))
            keep = [at for at, i in enumerate(running) if new[i] > made]
            running = [running[at] for at in keep]
            if not running:
                break
            history, weights = history[keep], weights[keep]
        groups = (ints([k * samples for k in range(len(running) + 1)]), ints([len(prompts[i]) for i in running]), ints(running))
        logits = model.step(cache, history[:, :, -1].flatten(), rows_of(running), groups)
        tokens, logp = draw(logits.t())
        shape = (len(running), samples, 1)
        history, weights = torch.cat([history, tokens.view(shape)], 2), torch.cat([weights, logp.view(shape)], 2)
    return [h for h, _ in found], [w for _, w in found], cache


def beam_search(model: Decoder, prompts, new, beams: int, page_size: int = 16):
    """The ``beams`` likeliest continuations found of every prompt (a list of tokens), new[i] tokens
    of prompt i; -> tokens (per prompt [beams][new[i]]), their log probabilities (per prompt [beams])
    and the cache."""
    _check(model, prompts, new, beams, "beam_search")
    if beams > model.vocab:
        raise ValueError("beam_search finds no more beams than there are tokens")
    n = len(prompts)
    pages = sum(beams * (-(-(len(p) + t) // page_size) + 1) for p, t in zip(prompts, new))
    cache = model.cache(n * beams, pages, page_size)

    last = _read(model, cache, prompts, [i * beams for i in range(n)])   # in the first beam of each
    scores, tokens = torch.log_softmax(last, 1).topk(beams)   # [prompts][beams]
    heads = ints([i * beams for i in range(n)])
    cache.fork(heads.repeat_interleave(beams - 1), ints([i * beams + j for i in range(n) for j in range(1, beams)]))

    running, found = list(range(n)), [None] * n
    history = tokens[:, :, None]
    for made in range(1, max(new) + 1):
        ended = [i for i in running if new[i] == made]
        if ended:   # their pages go back, and what is left moves to the front
            for i in ended:
                at = running.index(i)
                found[i] = (history[at], scores[at])
            cache.release(ints([i * beams + j for i in ended for j in range(beams)]))
            cache.compact()
            keep = [at for at, i in enumerate(running) if new[i] > made]
            running = [running[at] for at in keep]
            if not running:
                break
            history, scores, tokens = history[keep], scores[keep], tokens[keep]
        rows = ints([[i * beams + j for j in range(beams)] for i in running])
        logits = model.step(cache, tokens.flatten().int(), rows.flatten())
        total = scores[:, :, None] + torch.log_softmax(logits, 0).t().reshape(len(running), beams, -1)
        scores, best = total.flatten(1).topk(beams)
        parent, tokens = best // model.vocab, best % model.vocab
        cache.fork(rows.gather(1, parent).flatten(), rows.flatten())
        history = torch.cat([history.gather(1, parent[:, :, None].expand(-1, -1, made)), tokens[:, :, None]], 2)
    return [h for h, _ in found], [s for _, s in found], cache


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, default in (("prompts", 4), ("beams", 4), ("tokens", 32), ("layers", 2), ("heads", 8), ("kv-heads", 2),
                          ("head-dim", 64), ("ffn", 1024), ("vocab", 1000), ("rate", 2), ("seed", 0), ("samples", 0), ("top-k", 0)):
        ap.add_argument(f"--{name}", type=int, default=default)
    for name, default in (("temperature", 1.0), ("top-p", 1.0), ("min-p", 0.0)):
        ap.add_argument(f"--{name}", type=float, default=default)
    ap.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    a = ap.parse_args(argv)
    model = Decoder(a.layers, a.heads, a.kv_heads, a.head_dim, a.ffn, a.vocab, rate=a.rate,
                    dtype=BF16 if a.dtype == "bf16" else F32, seed=a.seed, rotary=Rotary(a.head_dim) if a.samples else None)
    prompts = [[(7 * i + 3 * j) % a.vocab for j in range(3 + 5 * i)] for i in range(a.prompts)]
    new = [max(1, a.tokens - 2 * i) for i in range(a.prompts)]

    def run(new):
        if a.samples:
            return sample(model, prompts, new, a.samples, a.temperature, a.top_k, a.top_p, a.min_p, a.seed)
        return beam_search(model, prompts, new, a.beams)

    run([min(2, t) for t in new])   # code and memory are loaded
    torch.cuda.synchronize()
    start = time.perf_counter()
    tokens, scores, cache = run(new)
    torch.cuda.synchronize()
    seconds = time.perf_counter() - start
    which = "one of the continuations" if a.samples else "best continuation"
    for i, (t, s) in enumerate(zip(tokens, scores)):
        print(f"prompt {i}: {len(prompts[i])} tokens, {which} {t[0].tolist()[:8]}... log probability {s[0].sum().item():.3f}")
    steps = max(map(len, prompts)) + max(new) - 1
    print(f"{steps} steps in {seconds * 1e3:.1f} ms ({seconds / steps * 1e6:.0f} us each); "
          f"{int((cache.refs > 0).sum())} pages in use at the end")


if __name__ == "__main__":
    main()
