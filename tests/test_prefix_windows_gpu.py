"""Windows over shared prefixes where the work is planned: they begin before, within, at the end of and past what is
shared."""

import numpy as np
import pytest

from tests.test_prefix_attention_gpu import B, Setup   # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


def tasks(s, window):
    """(all tasks, those of what groups share) of a call, as its plan leaves them at the front of the workspace."""
    import torch
    need = s.B.bsp_attention_prefix_workspace(s.cache, s.n, s.heads, len(s.shared), s.width)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    q = torch.from_numpy(s.q).to(s.tdt).cuda()
    y = torch.empty_like(q)
    s.B.bsp_attention_prefix(s.cache, q, *s.data, *[s.ints(a) for a in (s.table, s.lens, s.starts, s.shared)], y, 0.125, window, None, None,
                             None, ws)
    torch.cuda.synchronize()
    return ws[:8].view(torch.int32).tolist()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_what_no_window_reaches_is_no_work(B, dt):
    s = Setup(B, [6, 2], [3000, 1700], [[1500, 1501, 1600, 2000, 1500, 1900], [1500, 1499]], 2, 4, 64, 16, dt, seed=1)
    for window, reached in ((1499, 0), (1500, 1), (1501, 2), (0, 2)):
        count, shared = tasks(s, window)
        assert count > 0 and (shared > 0) == (reached > 0), (window, count, shared)
        s.check(*s.run(0.125, window), 0.125, window)
    alone = tasks(s, 1499)
    s.starts, s.shared = [0], []
    assert alone == tasks(s, 1499)   # as if nothing were shared


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim,order", [(64, "heads"), (80, "slots"), (128, "heads"), (256, "slots")])
def test_windows_by_a_plan(B, dim, order, dt):
    """Above 2048 tokens, which are planned whatever the number of sequences."""
    rng = np.random.default_rng(dim)
    sizes, shared = [1, 4, 9, 0, 3], [2600, 2300, 3100, 50, 2200]
    own = [[40], [0, 1, 700, 2500], list(rng.integers(-800, 300, 9)), [], [2400, 2150, 2101]]
    s = Setup(B, sizes, shared, own, 1, 3, dim, 16, dt, order, seed=dim, extra=1, holes=0.02)
    for window in (2049, 2100, 2101, 2400, 2500, 2599, 2600, 2601, 3000, 3399, 10 ** 6, 2 ** 31 - 1):
        s.check(*s.run(dim ** -0.5, window, feature_major=window % 2 == 0), dim ** -0.5, window)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 72, 128, 256])
def test_column_blocks_in_windows(B, dim, dt):
    """Every number of columns that is worked on in another way, windows that begin within what is shared, where some
    members' tokens end before the others', and past it for some."""
    rng = np.random.default_rng(dim + 1)
    sizes = [1, 4, 8, 9, 16, 17, 33, 71]
    shared = [int(x) for x in rng.integers(2100, 2900, len(sizes))]
    s = Setup(B, sizes, shared, [rng.integers(-40 if i % 2 else 0, 300, m) for i, m in enumerate(sizes)], 1, 4, dim, 16, dt,
              "slots" if dim == 72 else "heads", seed=dim, holes=0.02)
    for window in (2060, 2500):
        s.check(*s.run(dim ** -0.5, window), dim ** -0.5, window)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("kv,heads,dim,members", [(8, 8, 64, 40), (5, 20, 40, 30), (8, 16, 136, 20)])
def test_several_key_heads_of_own_tokens_in_windows(B, kv, heads, dim, members, dt):
    rng = np.random.default_rng(kv)
    s = Setup(B, [members, 3], [2300, 2160], [rng.integers(0, 200, members), rng.integers(-50, 300, 3)], kv, heads, dim, 16, dt, seed=kv)
    for window in (2080, 2200, 2350):
        s.check(*s.run(dim ** -0.5, window), dim ** -0.5, window)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("members,group,window", [(3, 2, 0), (24, 4, 0), (70, 4, 0), (24, 4, 2250), (70, 3, 2250)])
def test_what_one_member_attends_to_changes_nothing_of_another(B, members, group, window, dt):
    """Results of a member that does not attend to a token are the same bit by bit whatever that token holds: neither the
    tasks nor their sums go by the values of other sequences."""
    import torch
    rng = np.random.default_rng(members + window)
    s = Setup(B, [members], [2300], [[100, 40] + list(rng.integers(-900, 100, members - 2))], 1, group, 64, 16, dt, seed=members)
    before = [t.cpu() for t in s.run(0.125, window)]
    longest, checked = int(np.argmax(s.lens)), 0
    for at, value in ((s.lens[0] - 1, float("nan")), (2250, float("inf")), (2299, float("nan")), (160, float("nan")), (s.lens[longest] - 1, -1e30)):
        keys, values = s.keys.copy(), s.values.copy()
        page, slot = s.table[longest if at == s.lens[longest] - 1 else 0, at // 16], at % 16
        keys[page, slot] = values[page, slot] = value
        t = Setup.__new__(Setup)
        t.__dict__.update(s.__dict__)
        t.data = [t.plane(a) for a in (keys, values)]
        y, lse = (a.cpu() for a in t.run(0.125, window))
        for b in range(s.n):
            if (page, slot) not in s.tokens(b, window):
                assert torch.equal(y[b], before[0][b]) and torch.equal(lse[b], before[1][b]), (b, at)
                checked += 1
    assert checked > 0
