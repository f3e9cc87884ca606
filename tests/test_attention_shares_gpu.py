"""The ways in which attention's work is cut up: whole units, pieces, equal shares, at the lengths where
one gives way to the other, and tables much wider than what the sequences fill."""

import numpy as np
import pytest

from tests.test_paged_attention_gpu import LENS, B, Setup   # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


class Wide(Setup):
    """A table with room for `tokens` tokens of every sequence."""

    def __init__(self, B, lens, kv, heads, dim, page, dt, order, tokens, **kw):
        super().__init__(B, lens, kv, heads, dim, page, dt, order, **kw)
        width = max(self.width, -(-tokens // page))
        table = np.full((len(lens), width), -1, np.int64)
        table[:, :self.width] = self.table
        self.table, self.width, self.dtable = table, width, self.ints(table)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("window,holes", [(0, 0.0), (100, 0.0), (33, 0.3), (0, 0.8)])
@pytest.mark.parametrize("kv,heads,dim", [(2, 6, 64), (1, 1, 80), (2, 4, 128), (1, 18, 256)])
def test_short_sequences_in_wide_tables(B, kv, heads, dim, window, holes, dt):
    s = Wide(B, LENS, kv, heads, dim, 16, dt, "heads", 5000, seed=dim + window, holes=holes)
    s.check(*s.run(dim ** -0.5, window), dim ** -0.5, window)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n,longest,kv,heads", [(20, 2500, 4, 4), (100, 300, 3, 6), (300, 60, 2, 2), (1024, 20, 1, 1), (1025, 20, 1, 1)])
def test_ragged_sequences(B, n, longest, kv, heads, dt):
    """More pieces than workgroups: equal shares, that begin and end inside sequences."""
    rng = np.random.default_rng(n)
    lens = rng.integers(0, longest, n)
    lens[rng.random(n) < 0.2] = 0
    lens[n // 2] = longest
    s = Wide(B, lens.tolist(), kv, heads, 16, 16, dt, "slots", 3000, seed=n)
    s.check(*s.run(0.25), 0.25)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [6 * 64, 6 * 64 + 65, 6 * 128, 6 * 128 + 1, 7 * 128, 7 * 128 + 1])
def test_lengths_about_the_first_cut(B, tokens, dt):
    s = Wide(B, [tokens, 1, 0, tokens // 2], 1, 3, 24, 1, dt, "heads", tokens, seed=tokens)
    s.check(*s.run(0.2), 0.2)


@pytest.mark.parametrize("tokens", [65535, 65536, 65537, 70000])
def test_a_piece_for_each_workgroup_and_one_more(B, tokens):
    s = Setup(B, [tokens], 1, 1, 8, 64, "f32", "heads", seed=tokens)
    s.check(*s.run(0.3), 0.3)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_long_sequence_whose_scores_are_all_nan_at_one_end(B, dt):
    """NaN in one token, in a segment of its own: the whole row of that head group is NaN, no other."""
    import torch
    s = Setup(B, [3000, 2000], 2, 4, 64, 16, dt, "heads", seed=8)
    s.dkeys[int(s.table[0, 170]), 1] = float("nan")   # tokens 2720 .. 2735 of the second key head
    y, lse = s.run(0.125)
    bad = torch.isnan(y).any(2)
    assert bad.tolist() == [[False, False, True, True], [False] * 4]
    assert torch.isnan(lse).tolist() == bad.tolist()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [40, 64, 80, 128, 136, 256])
@pytest.mark.parametrize("tokens", [0, 3000])
def test_caches_too_large_to_stay(B, dim, tokens, dt):
    """Few tokens far apart, in the whole and cut."""
    s = Wide(B, [1, 17, 0, 300, 130], 2, 6, dim, 16, dt, "heads", tokens, seed=dim, page_gap=1 << 20)
    s.check(*s.run(dim ** -0.5), dim ** -0.5)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [8 * 64, 9 * 64 - 1, 9 * 64, 9 * 64 + 1, 8 * 128, 9 * 128 - 1, 9 * 128, 9 * 128 + 1])
def test_lengths_about_a_few_steps(B, tokens, dt):
    s = Wide(B, [tokens, 0, 1, tokens - 1, tokens // 2], 1, 3, 24, 1, dt, "heads", tokens, seed=tokens)
    s.check(*s.run(0.2), 0.2)
