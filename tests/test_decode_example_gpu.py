"""The decoder that uses the decode operators together, against the same model computed in 64 bits
without a cache: every sequence's logits from all of its tokens at once."""

import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def D():
    import torch   # first: the library then runs on torch's HIP runtime
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2111_11581_amd import decode
    return decode


def plain_logits(model, tokens):
    """Logits [vocab][tokens] of one sequence."""
    import torch

    def w(layer):
        return layer.dequantize().double().cpu()

    def norm(x):
        return x * torch.rsqrt(x.square().mean(0, keepdim=True) + 1e-6)

    n, h, kv, d = len(tokens), model.heads, model.kv_heads, model.head_dim
    x = (model.embedding.double().cpu()[tokens] + model.places.double().cpu()[:n]).t()
    later = torch.ones(n, n, dtype=torch.bool).triu(1)
    for block in model.blocks:
        q, k, v = (w(block["qkv"]) @ norm(x)).split([h * d, kv * d, kv * d])
        q = q.view(h, d, n)
        k, v = (a.view(kv, d, n).repeat_interleave(h // kv, 0) for a in (k, v))
        score = (q.transpose(1, 2) @ k / math.sqrt(d)).masked_fill(later, -math.inf)
        x = x + w(block["out"]) @ (v @ score.softmax(2).transpose(1, 2)).reshape(h * d, n)
        x = x + w(block["down"]) @ (w(block["up"]) @ norm(x)).relu()
    return w(model.head) @ norm(x)


# fp32: a chain of some thirty fp32 sums of up to 200 terms, 2^-24 each; bf16: some ten roundings of
# 2^-9 in a row, whose errors add up as their squares
TOLERANCE = {"f32": 2e-5, "bf16": 3e-2}


def small(D, dt, **kw):
    c = dict(layers=2, heads=4, kv_heads=2, head_dim=24, ffn=200, vocab=77, longest=60, group=32, rate=2, seed=3)
    c.update(kw)
    return D.Decoder(dtype=D.F32 if dt == "f32" else D.BF16, **c)


def close(got, want, dt):
    import torch
    err = (got.double().cpu() - want).norm() / want.norm()
    assert err < TOLERANCE[dt], float(err)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [{}, dict(heads=3, kv_heads=3, head_dim=40, ffn=65, rate=1), dict(kv_heads=1, layers=1, group=128)])
def test_sequences_that_fork_and_end(D, dt, kw):
    model = small(D, dt, **kw)
    cache = model.cache(6, 40, page_size=5)
    text = {r: [] for r in range(6)}

    def step(tokens, rows):
        logits = model.step(cache, D.ints(tokens), D.ints(rows))
        for j, (t, r) in enumerate(zip(tokens, rows)):
            text[r] = text[r] + [t]
            close(logits[:, j], plain_logits(model, text[r])[:, -1], dt)

    for t in range(7):
        step([t, 70 - t, 5], [0, 3, 5])
    cache.fork(D.ints([0, 0, 3]), D.ints([1, 2, 4]))
    text[1] = text[2] = text[0]
    text[4] = text[3]
    for t in range(4):
        step([10 + t, 20 + t, 30, 40, 50 + t], [2, 0, 1, 4, 3])
    cache.release(D.ints([0, 5]))
    text[0] = text[5] = []
    cache.compact()
    cache.fork(D.ints([2, 1]), D.ints([1, 2]))   # two change places
    text[1], text[2] = text[2], text[1]
    for t in range(3):
        step([60, 61, 62, t], [1, 2, 3, 5])


@pytest.mark.parametrize("beams", [1, 4])
def test_beam_search_scores(D, beams):
    """What a beam is said to be worth is what its tokens are worth, and no beam is found twice."""
    import torch
    model = small(D, "f32")
    prompts, new = [[1, 2, 3], [4], [5, 6, 7, 8, 9, 10, 11, 12]], [6, 1, 9]
    tokens, scores, cache = D.beam_search(model, prompts, new, beams, page_size=4)
    assert int(cache.refs.sum()) == 0 and int(cache.lens.sum()) == 0
    for p, n, ts, ss in zip(prompts, new, tokens, scores):
        assert ts.shape == (beams, n) and len({tuple(t) for t in ts.tolist()}) == beams
        for t, s in zip(ts.tolist(), ss.tolist()):
            logp = plain_logits(model, p + t[:-1]).log_softmax(0)
            want = sum(float(logp[tok, len(p) - 1 + i]) for i, tok in enumerate(t))
            assert abs(s - want) < 1e-3   # n sums of terms of some units, 2e-5 of them each
    one = plain_logits(model, prompts[1])[:, -1].log_softmax(0)
    assert torch.allclose(scores[1].double().cpu(), one.topk(beams).values, atol=1e-3)


def test_refusals(D):
    model = small(D, "bf16")
    for prompts, new, beams in (([], [], 1), ([[]], [1], 1), ([[1]], [0], 1), ([[1]], [1, 1], 1), ([[1]], [1], 0),
                                ([[1]], [1], 78), ([[1] * 50], [12], 2)):
        with pytest.raises(ValueError):
            D.beam_search(model, prompts, new, beams)


def test_command(D, capsys):
    D.main(["--prompts", "2", "--beams", "2", "--tokens", "4", "--dtype", "f32", "--layers", "1"])
    assert "0 pages in use" in capsys.readouterr().out
