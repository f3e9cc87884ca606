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


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,group", [(40, 300, 32), (64, 1003, 64), (100, 4096, 128)])
@pytest.mark.parametrize("batch", [1, 2, 5, 16, 33, 64])
def test_weights_of_0_take_no_part(B, rows, cols, group, batch, dt):
    """Pruned columns whose activations are 2^60 times the rest.  fp32 sums of exact products, in any
    order: (cols + 4) 2^-24 of the sum of |w x|, which those columns are not in, with a factor of 2."""
    import torch
    rng = np.random.default_rng(rows + batch)
    mask = (rng.random((rows, cols)) < 0.5).astype(np.uint8)
    large = rng.permutation(cols)[:7]
    mask[:, large] = 0
    n, scales = M.q4_quantize(rng.standard_normal((rows, cols)).astype(np.float32) * 0.05, mask, group)
    x = rng.standard_normal((cols, batch)).astype(np.float32)
    x[large] *= 2.0 ** 60
    x = M.bf16(x) if dt == "bf16" else x
    y = torch.empty(rows, batch, device="cuda")
    B.bsp_q4_linear(rows, cols, group, batch, B.BF16 if dt == "bf16" else B.F32, B.F32,
                    torch.from_numpy(x).to(torch.bfloat16 if dt == "bf16" else torch.float32).cuda(),
                    torch.from_numpy(M.q4_bytes(n)).cuda(), torch.from_numpy(M.q4_scales(scales)).bfloat16().cuda(), None, False, y)
    w = M.q4_weights(n, scales, group)
    ref, size = w @ x.astype(np.float64), np.abs(w) @ np.abs(x.astype(np.float64))
    assert (np.abs(y.double().cpu().numpy() - ref) <= 2 * (cols + 4) * M.U24 * size).all()


@pytest.mark.parametrize("batch", [1, 6, 40])
def test_an_infinite_bf16_activation_counts_by_its_weight(B, batch):
    import torch
    rows, cols, group = 48, 260, 64
    rng = np.random.default_rng(batch)
    n, scales = rng.integers(0, 16, (rows, cols)), np.full((M.ceil(cols, group), rows), 0.5, np.float32)
    x = M.bf16(rng.standard_normal((cols, batch)).astype(np.float32))
    x[200, batch // 2] = -np.inf
    y = torch.empty(rows, batch, device="cuda")
    B.bsp_q4_linear(rows, cols, group, batch, B.BF16, B.F32, torch.from_numpy(x).bfloat16().cuda(),
                    torch.from_numpy(M.q4_bytes(n)).cuda(), torch.from_numpy(M.q4_scales(scales)).bfloat16().cuda(), None, False, y)
    with np.errstate(invalid="ignore"):
        want = (M.q4_weights(n, scales, group)[:, 200] * -np.inf).astype(np.float32)
    assert np.array_equal(y.cpu().numpy()[:, batch // 2], want, equal_nan=True)


def test_odd_batches_up_to_the_last_byte_of_4_gb(B):
    """x of 2^32 - 4 bytes: 32-bit offsets of bytes reach within 16 of their end.  As many rows as it
    takes for 33 vectors to be one tile: 67 GB of codes."""
    import torch
    rows, batch, cols, group = 2049, 33, 65075262, 128
    assert batch * cols == 2 ** 31 - 2
    nc, ns = B.bsp_q4_sizes(rows, cols, group)
    if torch.cuda.mem_get_info()[0] < nc + (16 << 30):
        pytest.skip("not enough memory left")
    x = torch.zeros(cols, batch, dtype=torch.bfloat16, device="cuda")
    near = torch.arange(1, 8 * batch + 1, device="cuda").view(8, batch)
    x[-8:] = (near % 251 - 125).bfloat16()
    codes = torch.full((nc,), 0x88, dtype=torch.uint8, device="cuda")
    at = (cols - 8) // 2
    codes.view(rows, -1)[:, at:at + 4] = torch.tensor([0xA9, 0xCB, 0xED, 0x7F], dtype=torch.uint8, device="cuda")
    scales, y = torch.ones(ns, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, batch, device="cuda")
    B.bsp_q4_linear(rows, cols, group, batch, B.BF16, B.F32, x, codes, scales, None, False, y)
    w = torch.tensor([9, 10, 11, 12, 13, 14, 15, 7], dtype=torch.float64) - 8
    want = w @ x[-8:].double().cpu()
    assert torch.equal(y.double().cpu(), want.expand(rows, -1))
    del x, codes, scales
    torch.cuda.empty_cache()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,cols,batch", [(4112, 300, 16), (8200, 203, 13), (16400, 140, 61), (16400, 140, 64), (16400, 600, 64)])
def test_fp32_layers_of_many_tiles(B, rows, cols, batch, group):
    """More tiles than workgroups run at once, and so many that a workgroup has two waves."""
    import torch
    rng = np.random.default_rng(rows + cols)
    n, scales = M.q4_quantize(rng.standard_normal((rows, cols)).astype(np.float32) * 0.05, None, group)
    x, bias = rng.standard_normal((cols, batch)).astype(np.float32), rng.standard_normal(rows).astype(np.float32) * 0.1
    room = torch.full((cols * batch + 64,), float("nan"), device="cuda")
    room[:cols * batch] = torch.from_numpy(x).cuda().view(-1)
    y = torch.empty(rows, batch, device="cuda")
    B.bsp_q4_linear(rows, cols, group, batch, B.F32, B.F32, room[:cols * batch], torch.from_numpy(M.q4_bytes(n)).cuda(),
                    torch.from_numpy(M.q4_scales(scales)).bfloat16().cuda(), torch.from_numpy(bias).cuda(), False, y)
    w = M.q4_weights(n, scales, group)
    ref = w @ x.astype(np.float64) + bias[:, None]
    size = np.abs(w) @ np.abs(x.astype(np.float64)) + np.abs(bias)[:, None]
    assert (np.abs(y.double().cpu().numpy() - ref) <= 2 * (cols + 4) * M.U24 * size).all()
