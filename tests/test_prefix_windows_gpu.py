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
