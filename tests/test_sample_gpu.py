"""Sampling against its definition: tokens exactly, log probabilities to their rounding."""

import numpy as np
import pytest

from tests import decode_model as M
from tests import sampling_model as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch   # first: the library then runs on torch's HIP runtime
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2111_11581_amd as B
    B.lib()
    return B


def device(a, dtype=None):
    import torch
    return None if a is None else torch.tensor(np.asarray(a), dtype=dtype or torch.float32, device="cuda")


def logits_of(a, dt, layout):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda().to(torch.bfloat16 if dt == "bf16" else torch.float32)
    if layout == "features":
        return t.t().contiguous().t()
    if layout == "gaps":
        room = torch.zeros(a.shape[0], 2 * a.shape[1] + 3, dtype=t.dtype, device="cuda")
        out = room[:, 1:1 + 2 * a.shape[1]:2]
        out.copy_(t)
        return out
    if layout == "odd":
        room = torch.zeros(a.shape[0], a.shape[1] + 1, dtype=t.dtype, device="cuda")
        out = room[:, 1:]
        out.copy_(t)
        return out
    return t


def check(B, l, u, dt="f32", layout="rows", temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
    import torch
    n, vocab = l.shape
    l = M.bf16(l) if dt == "bf16" else np.asarray(l, np.float32)
    f32 = [None if a is None else np.asarray(a, np.float32) for a in (u, temperature, top_p, min_p)]
    tokens, logp = torch.full((n,), -99, dtype=torch.int32, device="cuda"), torch.full((n,), 7.0, device="cuda")
    ws = torch.full((max(16, B.bsp_sample_workspace(n, vocab)),), 0xff, dtype=torch.uint8, device="cuda")
    x = logits_of(l, dt, layout)
    args = [device(a) for a in f32] + [device(top_k, torch.int32)]
    torch.cuda.synchronize()
    B.bsp_sample(B.BF16 if dt == "bf16" else B.F32, x, args[0], tokens, args[1], args[4], args[2], args[3], logp, ws, stream)
    torch.cuda.synchronize()
    again = torch.full((n,), -99, dtype=torch.int32, device="cuda")   # without log probabilities, and the same once more
    B.bsp_sample(B.BF16 if dt == "bf16" else B.F32, x, args[0], again, args[1], args[4], args[2], args[3], None, ws, stream)
    torch.cuda.synchronize()
    assert torch.equal(tokens, again)
    for b in range(n):
        one = [None if a is None else float(a[b]) for a in f32]
        want, lp, w = S.sample(l[b], one[0], 1.0 if one[1] is None else one[1], 0 if top_k is None else int(top_k[b]),
                               1.0 if one[2] is None else one[2], 0.0 if one[3] is None else one[3])
        assert int(tokens[b]) == want, (b, one, int(tokens[b]), want)
        # a weight is a whole multiple of 2^-43, and the log is rounded to fp32
        got = float(logp[b])
        assert got == lp if want < 0 else abs(got - lp) <= S.U24 * abs(lp) + 2.0 ** -43 / w + 2.0 ** -40, (b, got, lp)
    return tokens


VOCABS = [1, 2, 3, 63, 64, 65, 100, 1000, 1023, 1024, 1025, 4099, 16384, 20001, 32768, 32769, 50000]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", VOCABS)
def test_vocabularies_and_cuts(B, vocab, dt):
    rng = np.random.default_rng(vocab)
    for layout, n in (("rows", 12), ("features", 5), ("gaps", 2), ("odd", 3)):
        l = rng.standard_normal((n, vocab)) * 3
        some = dict(temperature=rng.uniform(0.3, 2, n), top_k=rng.integers(-1, min(2 * vocab, 300), n), top_p=rng.uniform(0.05, 1.0, n),
                    min_p=rng.uniform(0, 0.2, n))
        for names in ((), ("temperature",), ("top_k",), ("top_p",), ("min_p",), ("temperature", "top_k", "top_p"), tuple(some)):
            check(B, l, rng.random(n), dt, layout, **{k: some[k] for k in names})


@pytest.mark.parametrize("vocab", [131072, 200003, 262144, 1 << 20])
def test_large_vocabularies(B, vocab):
    rng = np.random.default_rng(vocab)
    for dt, layout in (("f32", "rows"), ("bf16", "features")):
        n = 3
        l = rng.standard_normal((n, vocab)) * 2
        check(B, l, rng.random(n), dt, layout)
        check(B, l, rng.random(n), dt, layout, temperature=[0.5, 1.0, 1.5], top_k=[0, 1000, vocab - 1], top_p=[0.9, 0.999, 0.5], min_p=[0, 0, 1e-3])


@pytest.mark.parametrize("vocab", [77, 5000, 70000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_ties(B, vocab, dt):
    """Few different values: the lower index goes first, and a cut may fall among equals."""
    rng = np.random.default_rng(vocab)
    n = 16
    l = rng.integers(-2, 3, (n, vocab)).astype(np.float64)
    l[:2] = 0.25
    l[2] = np.where(rng.random(vocab) < 0.5, 0.0, -0.0)
    for k in (1, 2, 7, vocab // 3, vocab - 1, vocab, vocab + 1):
        check(B, l, rng.random(n), dt, top_k=[k] * n)
    for p in (0.0, 1e-9, 0.25, 0.5, 0.75, 0.999):
        check(B, l, rng.random(n), dt, top_p=[p] * n)
        check(B, l, rng.random(n), dt, top_p=[p] * n, top_k=rng.integers(1, vocab, n))
    check(B, l, rng.random(n), dt, min_p=[1.0] * n)
    check(B, l, rng.random(n), dt, min_p=np.exp(-1.0) * np.ones(n) * 0.999)


@pytest.mark.parametrize("vocab", [50, 3000, 66000])
def test_masked_and_infinite(B, vocab):
    rng = np.random.default_rng(vocab)
    n = 14
    l = rng.standard_normal((n, vocab)) * 2
    l[0] = -np.inf
    l[1] = np.nan
    l[2, :] = -np.inf
    l[2, vocab - 1] = -5.0
    l[3, ::2] = -np.inf
    l[4, 5:9] = np.inf
    l[5, 1::3] = np.nan
    l[6, :] = -3.0e38
    l[6, 7] = 3.0e38
    l[7] = -3.4028234663852886e38
    l[8, 3] = np.inf
    l[9] = np.where(rng.random(vocab) < 0.9, -np.inf, l[9])
    l[10, :] = 1e-40
    cuts = dict(top_k=rng.integers(0, 20, n), top_p=rng.uniform(0.5, 1, n), min_p=rng.uniform(0, 0.1, n))
    for layout in ("rows", "features"):
        for t in (None, np.full(n, 0.7), np.full(n, 1e-30), np.full(n, 1e30), np.full(n, np.inf), np.zeros(n), np.full(n, -1.0)):
            check(B, l, rng.random(n), layout=layout, temperature=t)
            check(B, l, rng.random(n), layout=layout, temperature=t, **cuts)


def test_edges_of_the_arguments(B):
    rng = np.random.default_rng(8)
    l = rng.standard_normal((7, 999))
    check(B, l, [0.0, 1.0, 2.0, -1.0, np.nan, 1 - 2.0 ** -24, 2.0 ** -140])
    check(B, l, rng.random(7), top_p=[0, -1, 1, 2, np.nan, 2.0 ** -149, 1 - 2.0 ** -24])
    check(B, l, rng.random(7), min_p=[0, -1, 1, 2, np.nan, 2.0 ** -149, np.inf])
    check(B, l, rng.random(7), top_k=[0, -5, 1, 2 ** 31 - 1, -2 ** 31, 999, 998])
    check(B, l, rng.random(7), temperature=[0, -0.0, np.nan, 2.0 ** -149, np.inf, -np.inf, 3e38])


def test_frequencies(B):
    """Every token is taken for its part of the numbers 0 to 1: all of 4096 even steps."""
    l = np.log(np.array([0.5, 0.25, 0.0, 0.125, 0.125]) + 0.0, where=np.array([1, 1, 0, 1, 1], bool), out=np.full(5, -np.inf))
    n = 4096
    t = check(B, np.tile(l, (n, 1)), (np.arange(n) + 0.5) / n)
    assert [int((t == i).sum()) for i in range(5)] == [2048, 1024, 0, 512, 512]


def test_many_rows(B):
    rng = np.random.default_rng(9)
    check(B, rng.standard_normal((700, 257)) * 2, rng.random(700), layout="features", top_p=rng.random(700))
    check(B, rng.standard_normal((300, 4000)) * 2, rng.random(300), top_k=rng.integers(1, 50, 300), top_p=rng.random(300))


def test_adversarial_spreads(B):
    """Mass in one place, mass everywhere, values that differ in their last bits, values that span everything."""
    rng = np.random.default_rng(10)
    for vocab in (3000, 40000, 100000):
        l = np.zeros((8, vocab))
        l[0] = np.nextafter(np.float32(1), np.float32(2)) - 1 + np.float32(1) - rng.integers(0, 50, vocab) * 2.0 ** -24
        l[1] = rng.uniform(-1e30, 1e30, vocab)
        l[2] = -np.arange(vocab) * 1e-3
        l[3] = np.arange(vocab) * 1e-5
        l[4, rng.integers(vocab)] = 80.0
        l[5] = -np.exp(rng.uniform(-60, 60, vocab))
        l[6] = rng.choice([0.0, -20.0, -29.0, -30.0, -31.0], vocab)
        l[7] = rng.standard_normal(vocab) * 1e-6
        for k in (None, np.full(8, 17), np.full(8, vocab // 2)):
            for p in (None, np.full(8, 0.5), np.full(8, 0.99)):
                check(B, l, rng.random(8), top_k=k, top_p=p)


def test_streams_and_graphs(B):
    import torch
    rng = np.random.default_rng(11)
    for n, vocab in ((4, 1000), (4, 60000)):
        l = rng.standard_normal((n, vocab)) * 2
        check(B, l, rng.random(n), stream=torch.cuda.Stream(), top_k=[5] * n)
        x, u = logits_of(l, "f32", "features"), device(np.zeros(n))
        tokens, logp = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
        p = device(np.full(n, 0.9))
        graphs, spaces = [], []
        for _ in range(2):   # two graphs, each with its own workspace
            spaces.append(torch.full((max(16, B.bsp_sample_workspace(n, vocab)),), 0xff, dtype=torch.uint8, device="cuda"))
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1]):
                B.bsp_sample(B.F32, x, u, tokens, top_p=p, logp=logp, workspace=spaces[-1])
        for turn in range(4):
            r = rng.random(n).astype(np.float32)
            l = rng.standard_normal((n, vocab)).astype(np.float32) * (turn + 1)
            x.copy_(torch.from_numpy(l))
            u.copy_(torch.from_numpy(r))
            graphs[turn % 2].replay()
            torch.cuda.synchronize()
            for b in range(n):
                assert int(tokens[b]) == S.sample(l[b], r[b], top_p=float(np.float32(0.9)))[0]


@pytest.mark.parametrize("vocab", [1000, 9000, 40000])
def test_where_min_p_cuts(B, vocab):
    """Logits of every spread around the cut: some next to it, all of them far above or below, across zero, one float apart."""
    rng = np.random.default_rng(vocab)
    for t in (1e-6, 0.7, 30.0, 1e5, 1e30, 2.0 ** -140):
        for scale in (1e-3, 1.0, 40.0, 1e6):
            p = np.array([1e-42, 1e-20, 1e-3, 0.5, 1 - 2.0 ** -23, 1.5], np.float32)
            l = (rng.standard_normal((6, vocab)) * scale).astype(np.float32)
            l[:, :64] = l.max(1, keepdims=True) + (np.log(p.astype(np.float64)) * t).clip(-1e30, 0)[:, None].astype(np.float32)
            for i in range(64):   # a run of neighbours across the cut
                for _ in range(2):
                    l[:, i:64] = np.nextafter(l[:, i:64], np.float32(-np.inf if i % 2 else np.inf))
            check(B, l, rng.random(6), temperature=[t] * 6, min_p=p)
            check(B, l, rng.random(6), temperature=[t] * 6, min_p=p, top_k=[40] * 6, top_p=[0.9] * 6)
