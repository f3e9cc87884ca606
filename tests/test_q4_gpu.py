"""FC layers with 4-bit weights against their definition in 64 bits."""

import numpy as np
import pytest

from tests import decode_model as M

pytestmark = pytest.mark.gpu
DT = {"f32": 0, "bf16": 1}


@pytest.fixture(scope="module")
def B():
    import torch   # first: the library then runs on torch's HIP runtime
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2111_11581_amd as B
    B.lib()
    return B


def tens(a, dt):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to({"f32": torch.float32, "bf16": torch.bfloat16}[dt]).cuda()


def weights(rows, cols, group, seed, mask=None):
    rng = np.random.default_rng(seed)
    w = rng.standard_normal((rows, cols)).astype(np.float32) * 0.05
    return M.q4_quantize(w, mask, group)


def on_device(n, scales):
    import torch
    return torch.from_numpy(M.q4_bytes(n)).cuda(), tens(M.q4_scales(scales), "bf16")


def run_linear(B, n, scales, group, x, dt, out, bias, relu, stream=None):
    import torch
    rows, cols = n.shape
    codes, sc = on_device(n, scales)
    y = torch.full((rows, x.shape[1]), float("nan"), dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    B.bsp_q4_linear(rows, cols, group, x.shape[1], DT[dt], DT[out], x, codes, sc, bias, relu, y, stream)
    return y


def check_linear(got, n, scales, group, x, out, bias, relu):
    """Each element's own bound: fp32 sums of exact products of magnitude up to (16 + 15 + 24) s |x| in
    any order, then the output's rounding.  With 16 rows or more (so that no column cancels) also each
    column's rel-L2: fp32 1e-5, bf16 5e-3."""
    w = M.q4_weights(n, scales, group)
    ref = w @ x
    size = M.q4_weights(np.full_like(n, 8 + 55), scales, group) @ np.abs(x)
    if bias is not None:
        ref, size = ref + bias[:, None], size + np.abs(bias)[:, None]
    if relu:
        ref = np.maximum(ref, 0)
    assert np.isfinite(got).all()
    u = 2.0 ** -8 if out == "bf16" else 0.0
    assert (np.abs(got - ref) <= u * np.abs(ref) + (1 + u) * 2 * (n.shape[1] + 4) * M.U24 * size).all()
    if n.shape[0] < 16:
        return
    tol = 5e-3 if out == "bf16" else 1e-5
    err = np.linalg.norm(got - ref, axis=0)
    assert (err <= tol * np.linalg.norm(ref, axis=0) + 1e-30).all(), (err / np.linalg.norm(ref, axis=0)).max()


def inputs(rows, cols, batch, dt, seed):
    rng = np.random.default_rng(seed + 7)
    x = rng.standard_normal((cols, batch)).astype(np.float32)
    x = M.bf16(x) if dt == "bf16" else x
    return x, rng.standard_normal(rows).astype(np.float32) * 0.1


SHAPES = [(1, 1), (1, 33), (16, 128), (17, 129), (40, 64), (33, 200), (64, 500), (100, 1003), (256, 1024), (31, 4100),
          (515, 2047), (2050, 384)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("batch", [1, 2, 3, 4, 7, 8, 13, 16, 17, 20, 33, 64, 67, 100])
def test_linear_bf16(B, rows, cols, batch):
    group = [32, 64, 128][(rows + cols + batch) % 3]
    n, scales = weights(rows, cols, group, rows + cols)
    x, bias = inputs(rows, cols, batch, "bf16", batch)
    out = ["bf16", "f32"][(rows + batch) % 2]
    b = bias if batch % 2 else None
    y = run_linear(B, n, scales, group, tens(x, "bf16"), "bf16", out, None if b is None else tens(b, "f32"), batch % 3 == 0)
    check_linear(y.double().cpu().numpy(), n, scales, group, x.astype(np.float64), out, b, batch % 3 == 0)


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("batch", [1, 2, 5, 8, 16, 19, 48, 65])
def test_linear_f32(B, rows, cols, batch):
    group = [32, 64, 128][(rows + 2 * cols + batch) % 3]
    n, scales = weights(rows, cols, group, rows + 2 * cols)
    x, bias = inputs(rows, cols, batch, "f32", batch)
    out = ["f32", "f32", "bf16"][(rows + batch) % 3]
    y = run_linear(B, n, scales, group, tens(x, "f32"), "f32", out, tens(bias, "f32"), False)
    check_linear(y.double().cpu().numpy(), n, scales, group, x.astype(np.float64), out, bias, False)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("batch", [1, 4, 11, 64])
def test_every_code_at_every_place(B, group, batch):
    """All codes, 0 too (which no quantiser gives), against one-hot activations: each output is one weight."""
    rows, cols = 32, 300
    rng = np.random.default_rng(group)
    n = rng.integers(0, 16, (rows, cols))
    scales = M.bf16(2.0 ** rng.integers(-6, 6, (M.ceil(cols, group), rows)))
    w = M.q4_weights(n, scales, group)
    for first in range(0, cols, batch):
        x = np.zeros((cols, batch), np.float32)
        for j in range(batch):
            if first + j < cols:
                x[first + j, j] = 1
        for dt in ("bf16", "f32"):
            y = run_linear(B, n, scales, group, tens(x, dt), dt, "f32", None, False).double().cpu().numpy()
            want = w @ x.astype(np.float64)
            assert np.array_equal(y, want), (first, dt)


def test_padding_is_not_read_as_values(B):
    """Codes and scales past the last column and row hold anything."""
    import torch
    rows, cols, group, batch = 21, 75, 32, 3
    n, scales = weights(rows, cols, group, 3)
    x, _ = inputs(rows, cols, batch, "bf16", 1)
    codes, sc = on_device(n, scales)
    codes[:, 38:] = 0xA7
    codes[:, 37] |= 0xF0
    sc[:, rows:] = float("nan")
    y = torch.empty(rows, batch, device="cuda")
    for dt in ("bf16", "f32"):
        B.bsp_q4_linear(rows, cols, group, batch, DT[dt], 0, tens(x, dt), codes, sc, None, False, y)
        check_linear(y.double().cpu().numpy(), n, scales, group, x.astype(np.float64), "f32", None, False)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("dt,batch", [("bf16", 1), ("f32", 1), ("bf16", 6), ("f32", 6), ("bf16", 40), ("f32", 40)])
def test_one_bad_activation_spoils_its_column_only(B, bad, dt, batch):
    rows, cols, group = 48, 260, 64
    n, scales = weights(rows, cols, group, 5)
    x, _ = inputs(rows, cols, batch, "bf16", 2)
    x[200, batch // 2] = bad
    y = run_linear(B, n, scales, group, tens(x, dt), dt, "f32", None, False).cpu().numpy()
    assert not np.isfinite(y[:, batch // 2]).any()
    assert np.isfinite(np.delete(y, batch // 2, 1)).all()


@pytest.mark.parametrize("batch", [1, 5, 16])
def test_f32_activations_count_in_full(B, batch):
    """Activations with 24 significant bits: rounding them to 16 or to 8 would show."""
    rows, cols, group = 64, 512, 128
    n, scales = weights(rows, cols, group, 11)
    x = (1 + np.random.default_rng(1).integers(0, 1 << 23, (cols, batch)) * 2.0 ** -23).astype(np.float32)
    y = run_linear(B, n, scales, group, tens(x, "f32"), "f32", "f32", None, False).double().cpu().numpy()
    w = M.q4_weights(n, scales, group)
    size = M.q4_weights(np.full_like(n, 8 + 55), scales, group) @ np.abs(x.astype(np.float64))
    assert (np.abs(y - w @ x.astype(np.float64)) <= 2 * (cols / 128 + 260) * M.U24 * size).all()


@pytest.mark.parametrize("batch", [1, 3, 8, 64])
def test_unaligned_activations_and_outputs(B, batch):
    """Views that begin one element into an array."""
    import torch
    rows, cols, group = 37, 256, 64
    n, scales = weights(rows, cols, group, 21)
    codes, sc = on_device(n, scales)
    x, _ = inputs(rows, cols, batch, "bf16", 4)
    for dt in ("bf16", "f32"):
        room = torch.empty(cols * batch + 1, dtype=tens(x, dt).dtype, device="cuda")
        xs = room[1:].view(cols, batch)
        xs.copy_(tens(x, dt))
        guard = torch.full((rows * batch + 2,), 7.0, device="cuda")
        y = guard[1:-1].view(rows, batch)
        B.bsp_q4_linear(rows, cols, group, batch, DT[dt], 0, xs, codes, sc, None, False, y)
        check_linear(y.double().cpu().numpy(), n, scales, group, x.astype(np.float64), "f32", None, False)
        assert guard[0] == 7 and guard[-1] == 7


def test_same_twice_and_on_another_stream(B):
    import torch
    rows, cols, group, batch = 300, 2000, 64, 9
    n, scales = weights(rows, cols, group, 9)
    x, bias = inputs(rows, cols, batch, "bf16", 3)
    xd, bd = tens(x, "bf16"), tens(bias, "f32")
    first = run_linear(B, n, scales, group, xd, "bf16", "bf16", bd, True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = run_linear(B, n, scales, group, xd, "bf16", "bf16", bd, True)
    third = run_linear(B, n, scales, group, xd, "bf16", "bf16", bd, True, s)
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), second.view(torch.int16))
    assert torch.equal(first.view(torch.int16), third.view(torch.int16))


def test_empty_batch(B):
    n, scales = weights(20, 40, 32, 1)
    x, _ = inputs(20, 40, 0, "bf16", 1)
    assert run_linear(B, n, scales, 32, tens(x, "bf16"), "bf16", "bf16", None, False).shape == (20, 0)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (16, 32), (17, 257), (64, 1000), (250, 640)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [False, True])
def test_quantize_and_back(B, rows, cols, group, dt, masked):
    """Codes, scales and the weights read back equal the definition's bit for bit."""
    import torch
    rng = np.random.default_rng(rows * cols + group)
    w = rng.standard_normal((rows, cols)).astype(np.float32)
    w[:, : cols // 3] = 0            # groups of zeros
    w[0] *= 1e-30
    w = M.bf16(w) if dt == "bf16" else w
    mask = rng.integers(0, 3, (rows, cols)).astype(np.uint8) if masked else None
    n, scales = M.q4_quantize(w, mask, group)
    nc, ns = B.bsp_q4_sizes(rows, cols, group)
    codes = torch.full((nc,), 0xEE, dtype=torch.uint8, device="cuda")
    sc = torch.full((ns,), 9.0, dtype=torch.bfloat16, device="cuda")
    B.bsp_q4_quantize(rows, cols, group, DT[dt], tens(w, dt), None if mask is None else torch.from_numpy(mask).cuda(),
                      codes, sc)
    assert np.array_equal(codes.cpu().numpy(), M.q4_bytes(n).ravel())
    assert np.array_equal(sc.float().cpu().numpy(), M.q4_scales(scales).ravel())
    if masked:
        assert (M.q4_weights(n, scales, group)[mask == 0] == 0).all()
    back = torch.empty(rows, cols, dtype=torch.float32 if dt == "f32" else torch.bfloat16, device="cuda")
    B.bsp_q4_dequantize(rows, cols, group, DT[dt], codes, sc, back)
    want = M.q4_weights(n, scales, group).astype(np.float32)
    assert np.array_equal(back.float().cpu().numpy(), M.bf16(want) if dt == "bf16" else want)


def test_a_pruned_layer_in_4_bits(B):
    """Pruned by bsp_prune, quantised with its mask: removed weights are 0, and the layer's outputs are
    those of the pruned layer read back and run by bsp_linear."""
    import torch
    from paper_2111_11581_amd.layers import PackedLayer
    rows, cols, batch = 64, 256, 5
    w = tens(np.random.default_rng(2).standard_normal((rows, cols)).astype(np.float32), "f32")
    scheme = B.Scheme(rows, cols, 16, 32, B.COL, 4)
    mask = torch.empty(rows * cols, dtype=torch.uint8, device="cuda")
    B.bsp_prune(scheme, B.F32, w, mask)
    nc, ns = B.bsp_q4_sizes(rows, cols, 64)
    codes, sc = torch.empty(nc, dtype=torch.uint8, device="cuda"), torch.empty(ns, dtype=torch.bfloat16, device="cuda")
    B.bsp_q4_quantize(rows, cols, 64, B.F32, w, mask, codes, sc)
    back = torch.empty_like(w)
    B.bsp_q4_dequantize(rows, cols, 64, B.F32, codes, sc, back)
    assert (back.view(-1)[mask == 0] == 0).all()
    x = tens(np.random.default_rng(3).standard_normal((cols, batch)).astype(np.float32), "f32")
    y4, y = torch.empty(rows, batch, device="cuda"), torch.empty(rows, batch, device="cuda")
    B.bsp_q4_linear(rows, cols, 64, batch, B.F32, B.F32, x, codes, sc, None, False, y4)
    PackedLayer(scheme, B.F32, back, mask=mask).linear(x, y, batch, B.F32)
    assert torch.allclose(y4, y, rtol=1e-4, atol=1e-4 * float(y.abs().max()))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("batch", [1, 13, 64])
def test_in_a_graph(B, batch, dt):
    """Captured once, replayed with other activations and the program's own work in between."""
    import torch
    rows, cols, group = 600, 1003, 64
    nc, ns = B.bsp_q4_sizes(rows, cols, group)
    gen = torch.Generator(device="cuda").manual_seed(batch)
    codes = torch.randint(0, 256, (nc,), dtype=torch.uint8, device="cuda", generator=gen)
    scales = torch.rand(ns, device="cuda", generator=gen).bfloat16()
    code, tdt = (B.BF16, torch.bfloat16) if dt == "bf16" else (B.F32, torch.float32)
    x = torch.zeros(cols, batch, dtype=tdt, device="cuda")
    y, eager = torch.empty(rows, batch, device="cuda"), torch.empty(rows, batch, device="cuda")

    def call(to):
        B.bsp_q4_linear(rows, cols, group, batch, code, B.F32, x, codes, scales, None, True, to)

    call(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(y)
    for _ in range(4):
        x.copy_(torch.randn(cols, batch, device="cuda", generator=gen))
        y.fill_(float("nan"))
        call(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager) and eager.abs().sum() > 0


def between_nan(B, x, dt, before):
    """x on the device, `before` elements after the start of an array of NaN that goes on after it."""
    import torch
    room = torch.full((before + x.size + 64,), float("nan"), dtype=torch.bfloat16 if dt == "bf16" else torch.float32, device="cuda")
    out = room[before:before + x.size].view(x.shape)
    out.copy_(tens(x, dt))
    return out


@pytest.mark.parametrize("before", [0, 2, 3])
@pytest.mark.parametrize("cols", [1, 2, 3, 5, 31, 127, 128, 129, 131, 255, 257])
@pytest.mark.parametrize("batch", [3, 5, 7, 9, 15, 17, 25, 31, 33, 41, 63, 65])
def test_odd_batches(B, batch, cols, before):
    """Rows of bf16 vectors that begin in the middle of a word, up to the last of x."""
    rows, group = 20, [32, 64, 128][cols % 3]
    n, scales = weights(rows, cols, group, cols)
    x, _ = inputs(rows, cols, batch, "bf16", batch)
    y = run_linear(B, n, scales, group, between_nan(B, x, "bf16", before), "bf16", "f32", None, False)
    check_linear(y.double().cpu().numpy(), n, scales, group, x.astype(np.float64), "f32", None, False)


@pytest.mark.parametrize("rows,cols", [(4100, 300), (4112, 2050), (8200, 1003), (16400, 140)])
@pytest.mark.parametrize("batch", [3, 13, 16, 30, 31, 33, 61, 64])
def test_more_tiles_than_workgroups_at_once(B, rows, cols, batch):
    group = [32, 64, 128][batch % 3]
    n, scales = weights(rows, cols, group, rows)
    x, bias = inputs(rows, cols, batch, "bf16", batch)
    y = run_linear(B, n, scales, group, between_nan(B, x, "bf16", 0), "bf16", "f32", tens(bias, "f32"), False)
    check_linear(y.double().cpu().numpy(), n, scales, group, x.astype(np.float64), "f32", bias, False)
