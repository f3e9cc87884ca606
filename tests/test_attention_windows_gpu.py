"""Windows of attention where the work is cut up: their first tokens lie inside pages, pieces and shares."""

import numpy as np
import pytest

from tests import decode_model as M
from tests.test_attention_shares_gpu import Wide
from tests.test_paged_attention_gpu import B, Setup   # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


class Far(Setup):
    """Sequences whose last tokens lie in two pages each, after a long part of the table that is gone."""

    def __init__(self, B, lens, width, page, dt, window, seed):
        import torch
        rng = np.random.default_rng(seed)
        self.B, self.lens, self.kv, self.heads, self.dim, self.page, self.dt, self.order = B, lens, 1, 2, 8, page, dt, "heads"
        self.width, self.window = width, window
        rnd = M.bf16 if dt == "bf16" else (lambda a: a)
        self.keys, self.values = (rnd(rng.standard_normal((2, page, 1, 8)).astype(np.float32)) for _ in range(2))
        self.q = rnd(rng.standard_normal((len(lens), 2, 8)).astype(np.float32))
        self.table = np.full((len(lens), width), -1, np.int64)
        for b, n in enumerate(lens):
            last = (n - 1) // page
            self.table[b, last] = b % 2
            if last:
                self.table[b, last - 1] = 1 - b % 2
        self.tdt = torch.bfloat16 if dt == "bf16" else torch.float32
        self.dkeys, self.dvalues = self.plane(self.keys, 0), self.plane(self.values, 0)
        self.cache = B.CacheShape.of(self.dkeys)
        self.dtable, self.dlens = self.ints(self.table), self.ints(lens)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_over_very_long_tables(B, dt):
    """64 sequences in tables for 2^30 tokens each."""
    rng = np.random.default_rng(5)
    lens = rng.integers(1, 1 << 30, 64)
    lens[:4] = [1, 4095, 4097, 1 << 30]
    s = Far(B, lens.tolist(), 1 << 14, 1 << 16, dt, 4096, 5)
    s.check(*s.run(0.35, 4096), 0.35, 4096)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("holes", [0.0, 0.3])
@pytest.mark.parametrize("window", [1000, 1153, 2000])
@pytest.mark.parametrize("page", [7, 16])
def test_in_pieces(B, page, window, holes, dt):
    """Few sequences: a piece of four blocks for each workgroup."""
    lens = [1, 5000, 999, 1000, 1001, 1153, 1154, 0, 2000, 2001, 3777]
    s = Wide(B, lens, 2, 6, 64, page, dt, "heads", 5000, seed=window + page, holes=holes)
    s.check(*s.run(0.125, window), 0.125, window)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("holes", [0.0, 0.3])
@pytest.mark.parametrize("n,kv,window", [(40, 4, 1153), (40, 4, 2000), (36, 8, 1100), (36, 8, 2200)])
def test_in_equal_shares(B, n, kv, window, holes, dt):
    """More pieces than workgroups; with fewer than 256 sequences times key heads, and with more."""
    rng = np.random.default_rng(n + window)
    lens = rng.integers(1, 3000, n)
    lens[:6] = [0, 1, window - 1, window, window + 1, 5000]
    s = Wide(B, lens.tolist(), kv, kv, 16, 16, dt, "slots", 5000, seed=window, holes=holes)
    s.check(*s.run(0.25, window), 0.25, window)
