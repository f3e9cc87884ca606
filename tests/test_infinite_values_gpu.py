"""Attention over values of Inf: what it answers is what the definition does, Inf, or NaN where both are attended to or
a NaN is."""

import numpy as np
import pytest

from tests import decode_model as M
from tests import sampling_model as S
from tests import test_prefix_attention_gpu as P
from tests.test_paged_attention_gpu import B, Setup   # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


def spoil(s, at, rng):
    """Values (by `at(b)`: pages and slots that sequence b attends to) of Inf in dimension 0 of one token, -Inf in 1,
    both in 2, NaN in 3, Inf in 4 of several tokens, in 5 of the last one and in 6 of the first."""
    inf = np.inf
    for b in range(s.n if hasattr(s, "n") else len(s.lens)):
        tokens = at(b)
        if not tokens:
            continue

        def put(dim, value, *which):
            for i in which:
                s.values[tokens[i][0], tokens[i][1], :, dim] = value
        n = len(tokens)
        one, two = int(rng.integers(0, n)), int(rng.integers(0, n))
        put(0, inf, one), put(1, -inf, two), put(2, inf, one), put(3, np.nan, two), put(5, inf, n - 1), put(6, -inf, 0)
        if one != two:
            put(2, -inf, two)
        put(4, inf, *rng.integers(0, n, 5))


def same(got, ref, bound):
    """Alike where ref is not finite, and within the bound where it is."""
    odd = ~np.isfinite(ref)
    assert np.array_equal(got[odd], ref[odd], equal_nan=True), (got[odd], ref[odd])
    assert (np.abs(got[~odd] - ref[~odd]) <= bound[~odd]).all()
    return odd


def check(s, y, lse, scale, window=0):
    """As Setup.check, with the bounds of finite values."""
    y, lse, spoiled = y.double().cpu().numpy(), lse.double().cpu().numpy(), 0
    for i, n in enumerate(s.lens):
        for h in range(s.heads):
            j = h // (s.heads // s.kv)
            with np.errstate(invalid="ignore"):
                ref, l, size, _, qk = M.attention(s.q[i, h], s.keys[:, :, j], s.values[:, :, j], s.table[i], s.page, n, window, scale)
                small = 2 * 2 * (s.dim + 4) * M.U24 * qk + (2 * n + 64) * M.U24
                p, u = (2.0 ** -8, 2.0 ** -8) if s.dt == "bf16" else (0.0, M.U24)
                spoiled += same(y[i, h], ref, u * np.abs(ref) + (1 + u) * (p + small) * size).sum()
            assert lse[i, h] == l if l == -np.inf else abs(lse[i, h] - l) <= 2 * (s.dim + 4) * M.U24 * qk + (n + 64) * M.U24 + 4 * M.U24 * abs(l)
    assert spoiled > 0


def tokens_of(s, b, window=0):
    n = s.lens[b]
    at = [(s.table[b, t // s.page], t % s.page) for t in range(max(0, n - window) if window else 0, n)]
    return [(p, t) for p, t in at if p >= 0]


@pytest.mark.parametrize("order", ["heads", "slots"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 40, 64, 96, 128, 136, 256])
@pytest.mark.parametrize("lens", [[0, 1, 2, 31, 33, 129], [1, 3000, 0, 700, 1500]])
def test_attention(B, lens, dim, dt, order):
    s = Setup(B, lens, 2, 6, dim, 16, dt, order, seed=dim)
    spoil(s, lambda b: tokens_of(s, b), np.random.default_rng(dim))
    s.dvalues = s.plane(s.values, 0)
    check(s, *s.run(dim ** -0.5), dim ** -0.5)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attention_windows_and_holes(B, dt):
    """Nothing of what lies before the window, past the end or in no page."""
    for lens, window in (([40, 100, 7], 30), ([2500, 1300, 20], 1100)):
        s = Setup(B, lens, 2, 4, 64, 7, dt, "heads", seed=window, holes=0.1)
        spoil(s, lambda b: tokens_of(s, b, window), np.random.default_rng(window))
        s.dvalues = s.plane(s.values, 0)
        check(s, *s.run(0.125, window), 0.125, window)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n", [60, 2000])
def test_attention_of_probabilities_that_are_almost_nothing(B, dt, n):
    """A value of Inf whose probability is 2^-200 or so: below what fp32 holds, but above 0."""
    s = Setup(B, [n, n], 1, 2, 64, 16, dt, "heads", seed=n)
    s.q[:] = 1.0
    s.keys[np.isfinite(s.keys)] = 0.0
    page, slot = s.table[0, 5 // 16], 5 % 16
    s.keys[page, slot] = -2.0      # a score of -128, times 1.125: e^-144
    s.values[page, slot, :, :4] = np.inf
    s.values[page, slot, :, 4] = -np.inf
    s.dkeys, s.dvalues = s.plane(s.keys, 0), s.plane(s.values, 0)
    y, lse = s.run(1.125)
    check(s, y, lse, 1.125)
    assert np.isinf(y[0, :, :5].float().cpu().numpy()).all() and y[1].isfinite().all()


# ---- sequences that share their first tokens ----

def check_prefix(s, y, lse, scale, window=0):
    y, lse, spoiled = y.double().cpu().numpy(), lse.double().cpu().numpy(), 0
    group = s.heads // s.kv
    for b in range(s.n):
        at = s.tokens(b, window)
        if not at:
            assert (y[b] == 0).all() and (lse[b] == -np.inf).all()
            continue
        p, t = np.array(at).T
        for j in range(s.kv):
            h = slice(j * group, (j + 1) * group)
            with np.errstate(invalid="ignore"):
                ref, l, size, qk = S.attention(s.q[b, h], s.keys[p, t, j], s.values[p, t, j], scale)
                score = 2 * (s.dim + 4) * S.U24 * qk[:, None]
                u, cut = (2.0 ** -8, 2.0 ** -15) if s.dt == "bf16" else (S.U24, 0.0)
                spoiled += same(y[b, h], ref, u * np.abs(ref) + (1 + u) * (cut + 2 * score + (2 * len(at) + 64) * S.U24) * size).sum()
            assert (np.abs(lse[b, h] - l) <= score[:, 0] + (len(at) + 64) * S.U24 + 4 * S.U24 * np.abs(l)).all()
    assert spoiled > 0


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 64, 96, 128, 256])
@pytest.mark.parametrize("sizes,shared,longest,window,least", [
    ([1, 3, 0, 2], [33, 100, 5, 64], 40, 0, 0), ([3, 4], [60, 90], 50, 70, 0),              # short tables
    ([1, 3, 0, 2], [33, 100, 5, 64], 40, 0, 2100), ([3, 9], [2200, 300], 300, 0, 0),        # by a plan
    ([10, 33, 70], [1500, 900, 2300], 200, 0, 2100), ([30, 5], [3000, 2900], 300, 2500, 0)])
def test_prefix(B, sizes, shared, longest, window, least, dim, dt):
    rng = np.random.default_rng(dim + longest)
    P.Setup.least = least
    try:
        s = P.Setup(B, sizes, shared, [rng.integers(-20, longest, m) for m in sizes], 1, 3, dim, 16, dt, seed=dim, extra=1, holes=0.03)
    finally:
        P.Setup.least = 0
    few = rng.permutation(s.n)[:3]   # what most members share stays finite but for a few dimensions
    spoil(s, lambda b: s.tokens(b, window)[-40:] if b in few else [], rng)
    for b in few[:1]:
        for t in s.tokens(b, window)[:3]:
            s.values[t][:, 7] = np.inf
    s.data = [s.plane(a) for a in (s.keys, s.values)]
    check_prefix(s, *s.run(dim ** -0.5, window), dim ** -0.5, window)
    check_prefix(s, *s.run(dim ** -0.5, window, feature_major=True), dim ** -0.5, window)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("least", [0, 2100])
def test_prefix_of_other_rows(B, least, dt):
    """Shared tokens in the pages of a sequence of their own, which alone has the Inf."""
    P.Setup.least = least
    try:
        s = P.Setup(B, [3, 2], [60, 90], [[5, 9, 1], [30, 7]], 2, 4, 64, 16, dt, seed=3, prefix_rows=True)
    finally:
        P.Setup.least = 0
    for t, dim, value in ((3, 0, np.inf), (59, 1, -np.inf), (20, 2, np.nan)):
        s.values[s.table[s.prefix_rows[0], t // 16], t % 16, :, dim] = value
    s.data = [s.plane(a) for a in (s.keys, s.values)]
    check_prefix(s, *s.run(0.125), 0.125)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("least", [0, 2100])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_keys(B, value, least, dt):
    """A score of NaN or Inf makes all of y NaN, one of -Inf is of no weight."""
    import torch
    P.Setup.least = least
    try:
        s = P.Setup(B, [3, 2], [60, 90], [[5, 9, 1], [30, 7]], 2, 4, 64, 16, dt, seed=4)
    finally:
        P.Setup.least = 0
    s.keys[s.table[0, 1], 3, :, 5] = value   # token 19 of the first group
    s.keys[s.table[3, 0], 0, :, 9] = value
    s.data = [s.plane(a) for a in (s.keys, s.values)]
    y, lse = s.run(0.125)
    z, lse2 = torch.empty_like(y), torch.empty_like(lse)
    ws = torch.empty(max(16, B.bsp_attention_workspace(s.cache, s.n, s.heads, s.width)), dtype=torch.uint8, device="cuda")
    B.bsp_attention(s.cache, torch.from_numpy(s.q).to(s.tdt).cuda(), *s.data, s.ints(s.table), s.ints(s.lens), z, 0.125, 0, None, lse2, ws)
    torch.cuda.synchronize()
    odd = 0
    for b in range(s.n):
        p, t = np.array(s.tokens(b, 0)).T
        for h in range(s.heads):
            k, v = s.keys[p, t, h // 2].astype(np.float64), s.values[p, t, h // 2]
            score = k @ s.q[b, h].astype(np.float64)
            spoiled = bool((np.isnan(score) | (score == np.inf)).any())
            odd += spoiled
            on = score > -np.inf
            for got in (y, z):
                got = got[b, h].double().cpu().numpy()
                if spoiled:
                    assert np.isnan(got).all()
                    continue
                ref, _, size, qk = S.attention(s.q[b, h][None], k[on], v[on], 0.125)
                score_error = 2 * (s.dim + 4) * S.U24 * qk[0]
                u, cut = (2.0 ** -8, 2.0 ** -15) if dt == "bf16" else (S.U24, 0.0)
                assert (np.abs(got - ref[0]) <= u * np.abs(ref[0]) + (1 + u) * (cut + 2 * score_error + (2 * len(p) + 64) * S.U24) * size[0]).all()
    assert odd > 0 and (odd == s.n * s.heads) == np.isnan(value)
