"""What the decode operators keep of their operands' bits, where cancelling sums would show fewer."""

import numpy as np
import pytest

from tests import decode_model as M
from tests.test_paged_attention_gpu import B, Setup   # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,kv,heads,dim", [([2, 9, 40, 300], 2, 6, 64), ([33, 500], 1, 3, 128), ([3000, 1], 1, 4, 64),
                                               ([70], 2, 2, 256)])
def test_bf16_probabilities_keep_16_bits(B, lens, kv, heads, dim):
    """Values whose weighted sums nearly cancel.  The scores' error, of fp32 sums, and the sums' own as in
    Setup.check; a probability kept to 16 bits errs by 2^-16 of it at most; the output is rounded
    once, by 2^-8 of it.  Probabilities of 8 bits would err by 2^-8 of the values."""
    s = Setup(B, lens, kv, heads, dim, 16, "bf16", "heads", seed=dim)
    for b, n in enumerate(lens):   # of neighbours the same value with the other sign
        for t in range(1, n, 2):
            s.values[s.table[b, t // 16], t % 16] = -s.values[s.table[b, (t - 1) // 16], (t - 1) % 16]
            near = s.keys[s.table[b, (t - 1) // 16], (t - 1) % 16]
            s.keys[s.table[b, t // 16], t % 16] = M.bf16(near + 0.02 * np.sign(near))
    s.dkeys, s.dvalues = s.plane(s.keys, 0), s.plane(s.values, 0)
    scale = dim ** -0.5
    y, lse = s.run(scale)
    s.check(y, lse, scale)
    y = y.double().cpu().numpy()
    for b, n in enumerate(lens):
        for h in range(heads):
            j = h // (heads // kv)
            ref, _, size, _, qk = M.attention(s.q[b, h], s.keys[:, :, j], s.values[:, :, j], s.table[b], 16, n, 0, scale)
            small = 2 * 2 * (dim + 4) * M.U24 * qk + (2 * n + 64) * M.U24
            assert (np.abs(y[b, h] - ref) <= 2.0 ** -8 * np.abs(ref) + 1.01 * (2.0 ** -16 + small) * size).all(), (b, h)
