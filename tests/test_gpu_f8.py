"""Matrices in 8 bits with a power of two for each block of 128, and their products, on the GPU against plain 64-bit forms."""
import pytest
import torch

import f8_util as ref
import paper_2309_01507_amd as lpmm
from conftest import progress
from f8_util import DEV

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")


def matrix(rows, cols, dtype, seed, spread=1.5):
    """Rows and columns of different size"""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * (spread * torch.randn(rows, 1, generator=g)).exp()
    return (x * (spread * torch.randn(1, cols, generator=g)).exp()).to(dtype)


def check_quant(x, tile, on_gpu=None, what=""):
    xd = x.to(DEV) if on_gpu is None else on_gpu
    want, scales = ref.quantize(x, tile)
    want_t, scales_t = ref.quantize(x.t(), tile)
    q = lpmm.lpmm_f8_quant(xd, tile)
    p, pt = lpmm.lpmm_f8_quant_both(xd, tile)
    for m, v, s in ((q, want, scales), (p, want, scales), (pt, want_t, scales_t)):
        got, got_scales = ref.unpack(m)
        assert torch.equal(got_scales, s) and ref.same(got, v), f"{what} {tuple(x.shape)} tile {tile}"
        for dtype in (F32, BF16):
            back = lpmm.lpmm_f8_dequant(m, dtype).cpu().double()
            assert ref.same(back, v), f"{what}: back to {dtype}"
    return q


SHAPES = [(1, 1), (1, 128), (3, 127), (2, 129), (128, 128), (127, 130), (129, 257), (300, 77), (16, 1000), (1000, 16), (260, 520)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_there_and_back(rows, cols, tile, dtype):
    check_quant(matrix(rows, cols, dtype, rows + cols), tile)


@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_every_code_and_border(dtype, tile):
    """Each code, each point half way between two (which bf16 holds), and their neighbours; for several powers, and largest elements at the power's border"""
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    points = torch.cat([codes, (codes[1:] + codes[:-1]) / 2])
    fine = torch.cat([points, points * (1 + 2.0 ** -7), points * (1 - 2.0 ** -8), torch.tensor([2.0 ** -11, 2.0 ** -10, 1.5 * 2.0 ** -10, 449.0, 463.0])])
    fine = torch.cat([fine, -fine]).to(dtype).float()
    for e in (-60, -3, 0, 1, 40):
        for top in (448.0, 450.0, 224.0, 226.0):
            x = torch.zeros(-(-fine.numel() // 100), 127)
            kept = torch.where(fine.abs() <= top, fine, torch.zeros_like(fine))
            for r in range(x.shape[0]):
                part = kept[r * 100:(r + 1) * 100]
                x[r, :part.numel()] = part
            x[:, 126] = top
            check_quant((x * 2.0 ** e).to(dtype), tile, what=f"2^{e}, {top}")


@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_unusual_values(dtype, tile):
    """Zeros, infinities, NaN, the type's largest and least numbers"""
    x = matrix(9, 300, dtype, 4, 0.3)
    x[0] = 0.0
    x[1, 5], x[1, 6] = INF, -INF
    x[2, 200] = NAN
    x[3, :128] = INF
    x[4, :128] = NAN
    x[5] *= 1e-30
    x[6, ::3] = -0.0
    check_quant(x, tile)
    big, small = torch.finfo(dtype).max, torch.finfo(dtype).tiny
    x = torch.zeros(6, 200, dtype=dtype)
    x[0, 3], x[0, 4] = big / 2, big / 300
    x[1, 3], x[1, 4] = small, small * 200
    x[2, :3] = torch.tensor([small / 8, small / 16, -small / 4]).to(dtype)          # below the normal numbers
    for r in range(6):                                                              # one kind a block
        check_quant(x[r:r + 1].clone(), tile)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_anywhere(dtype):
    x = matrix(70, 333, dtype, 5)
    for gap, off in ((1, 1), (3, 5), (4, 0)):
        room = torch.full((70 * (333 + gap) + off,), NAN, dtype=dtype, device=DEV)
        view = room[off:off + 70 * (333 + gap)].view(70, 333 + gap)[:, :333]
        view.copy_(x)
        for tile in (1, 128):
            q = check_quant(x, tile, view, f"{gap} {off}")
        out = torch.full_like(room, 77.0)
        to = out[off:off + 70 * (333 + gap)].view(70, 333 + gap)[:, :333]
        lpmm.lpmm_f8_dequant(q, out=to)
        assert torch.equal(to, lpmm.lpmm_f8_dequant(q, dtype))
        to.fill_(77.0)
        assert bool((out == 77.0).all()), "around the rows"


def product_of(m, n, k, dtype, tiles, seed, what=""):
    x, w = matrix(m, k, F32, seed, 0.7), matrix(n, k, F32, seed + 1, 0.7)
    a, b = lpmm.lpmm_f8_quant(x.to(DEV), tiles[0]), lpmm.lpmm_f8_quant(w.to(DEV), tiles[1])
    c = lpmm.lpmm_f8_matmul(a, b, dtype)
    ref.check_product(c, ref.unpack(a)[0], ref.unpack(b)[0], f"{m} x {n} x {k} {what}")
    return c


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tiles", [(1, 128), (1, 1), (128, 1), (128, 128)])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (5, 3, 100), (33, 65, 129), (128, 128, 128), (130, 257, 384), (64, 300, 1000), (257, 129, 2050)])
def test_products(m, n, k, tiles, dtype):
    product_of(m, n, k, dtype, tiles, m + n + k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(1000, 700, 640), (17, 5000, 300), (2, 2, 40000), (600, 2000, 1100), (5000, 33, 257)])
def test_larger_products(m, n, k, dtype):
    product_of(m, n, k, dtype, (1, 128), m)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(4100, 2600, 300), (2053, 2100, 515), (100, 32001, 260), (300, 9000, 130)])
def test_tiles_of_every_size(m, n, k, dtype):
    """256 x 256, 128 x 128 and 64 x 128, with edges in both directions"""
    product_of(m, n, k, dtype, (1, 128), m)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(17, 8100, 4100), (200, 2100, 8300), (330, 4100, 9300), (512, 4096, 9250)])
def test_sums_in_parts(m, n, k, dtype):
    product_of(m, n, k, dtype, (1, 128), m)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,n,k", [(1, 16384, 130), (3, 16400, 260), (16, 20001, 515), (2, 70000, 40)])
def test_few_tokens_and_many_rows(t, n, k, dtype):
    x, w = matrix(t, k, dtype, t, 0.7), matrix(n, k, F32, n, 0.7)
    q = lpmm.lpmm_f8_quant(w.to(DEV), 128)
    ref.check_product(lpmm.lpmm_f8_linear(x.to(DEV), q), ref.quantize(x, 1)[0], ref.unpack(q)[0], f"{t} x {n} x {k}")


def test_many_blocks_down():
    """More than 65535 blocks below each other"""
    rows = 128 * 65536 + 5
    x = torch.ones(rows, 3, dtype=BF16, device=DEV)
    x[-5:] = 3 * 2.0 ** 20
    q = lpmm.lpmm_f8_quant(x, 128)
    assert torch.equal(lpmm.lpmm_f8_dequant(q, BF16), x)
    assert bool((q.scales[:-1, 0] == q.scales[0, 0]).all()) and int(q.scales[-1, 0]) == ref.scale_of(x[-5:].double().cpu())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t", [1, 2, 7, 16, 17, 31, 64, 100, 200])
def test_linear(t, dtype):
    for n, k in ((1, 1), (15, 127), (100, 200), (333, 1000), (77, 4100)):
        x, w = matrix(t, k, dtype, t + n + k, 0.7), matrix(n, k, F32, t + n + k + 1, 0.7)
        q = lpmm.lpmm_f8_quant(w.to(DEV), 128)
        y = lpmm.lpmm_f8_linear(x.to(DEV), q)
        assert y.dtype == dtype
        ref.check_product(y, ref.quantize(x, 1)[0], ref.unpack(q)[0], f"{t} x {n} x {k}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t", [3, 40])
def test_linear_rows_anywhere(t, dtype):
    """x and y with gaps and off their boundaries; what lies around y stays; weights in blocks of 1 x 128 too"""
    n, k = 130, 515
    x, w = matrix(t, k, dtype, 1, 0.7), matrix(n, k, F32, 2, 0.7)
    for tile in (128, 1):
        q = lpmm.lpmm_f8_quant(w.to(DEV), tile)
        want = lpmm.lpmm_f8_linear(x.to(DEV), q)
        ref.check_product(want, ref.quantize(x, 1)[0], ref.unpack(q)[0], f"tile {tile}")
        xs = torch.full((t, k + 3), NAN, dtype=dtype, device=DEV)[:, 1:1 + k]
        xs.copy_(x)
        room = torch.full((t, n + 5), 77.0, dtype=dtype, device=DEV)
        y = lpmm.lpmm_f8_linear(xs, q, room[:, 3:3 + n])
        assert torch.equal(y, want) and bool((room[:, :3] == 77.0).all()) and bool((room[:, 3 + n:] == 77.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_is_not_finite_is_carried_through(dtype):
    for t in (2, 40):
        x, w = matrix(t, 300, dtype, 8, 0.5), matrix(150, 300, F32, 9, 0.5)
        x[1, 7] = NAN
        w[3, 299] = INF
        x[0] = 0.0
        q = lpmm.lpmm_f8_quant(w.to(DEV), 128)
        y = lpmm.lpmm_f8_linear(x.to(DEV), q).cpu()
        assert bool(y[1].isnan().all()) and bool(y[:, 3].isnan().all())
        ref.check_product(y, ref.quantize(x, 1)[0], ref.unpack(q)[0], f"{t}")


def test_blocks_far_apart_in_size():
    """Neighbouring blocks' powers 2^60 apart: each is applied to its own block."""
    g = torch.Generator().manual_seed(3)
    x, w = torch.randn(50, 512, generator=g), torch.randn(140, 512, generator=g)
    for j, e in enumerate((-30, 0, 30, -5)):
        x[:, j * 128:(j + 1) * 128] *= 2.0 ** e
        w[:, j * 128:(j + 1) * 128] *= 2.0 ** -e * (1 + j)
    for dtype in (F32, BF16):
        for t in (5, 50):
            q = lpmm.lpmm_f8_quant(w.to(DEV), 128)
            y = lpmm.lpmm_f8_linear(x[:t].to(dtype).to(DEV), q)
            ref.check_product(y, ref.quantize(x[:t].to(dtype), 1)[0], ref.unpack(q)[0], f"{t} {dtype}")


def test_empty():
    q = lpmm.lpmm_f8_quant(torch.randn(20, 130, device=DEV), 128)
    assert lpmm.lpmm_f8_linear(torch.empty(0, 130, device=DEV), q).shape == (0, 20)
    none = lpmm.lpmm_f8_quant(torch.empty(0, 130, device=DEV))
    assert lpmm.lpmm_f8_matmul(none, q).shape == (0, 20) and lpmm.lpmm_f8_matmul(q, none).shape == (20, 0)
    assert lpmm.lpmm_f8_dequant(none).shape == (0, 130)
    with pytest.raises(lpmm.LpmmError):
        lpmm.lpmm_f8_quant_both(torch.empty(0, 130, device=DEV))


def test_beyond_32_bits():
    """More than 2^31 codes, and results: the last rows"""
    n, k = 600_011, 4096
    progress("weights of 2.4e9 codes")
    q = lpmm.new_f8(n, k, 128)
    q.codes.zero_()
    q.scales.fill_(127)
    last = matrix(130, k, F32, 3, 0.3)
    part = lpmm.lpmm_f8_quant(last.to(DEV), 1)
    q.codes[n - 130:] = part.codes
    ones = torch.zeros_like(part.scales)
    ones[:, :130] = 127
    w = ref.unpack(lpmm.MatF8(130, k, 1, part.codes, ones))[0]
    for t, dtype in ((2, BF16), (2, F32), (40, BF16)):
        x = matrix(t, k, dtype, 4, 0.3)
        y = lpmm.lpmm_f8_linear(x.to(DEV), q)
        assert bool((y[:, :n - 130] == 0).all())
        ref.check_product(y[:, n - 130:], ref.quantize(x, 1)[0], w, f"{t}")
    progress("back to 2.4e9 values")
    back = lpmm.lpmm_f8_dequant(q, BF16)
    assert torch.equal(back[n - 130:].cpu().double(), w) and not bool(back[:n - 130].any())
    again = lpmm.lpmm_f8_quant(back, 128)
    assert torch.equal(lpmm.lpmm_f8_dequant(again, BF16)[n - 2:], lpmm.lpmm_f8_dequant(lpmm.lpmm_f8_quant(back[(n - 1) // 128 * 128:], 128), BF16)[-2:])


@pytest.mark.parametrize("t", [4, 100])
def test_on_a_stream_and_captured(t):
    """The same bits on another stream and from a captured graph, replayed with other inputs in between"""
    n, k = 200, 1000
    x, q = matrix(t, k, BF16, 1).to(DEV), lpmm.lpmm_f8_quant(matrix(n, k, F32, 2).to(DEV), 128)
    sets = [x.clone(), (x * 2).flip(0).contiguous(), x.flip(1).contiguous()]
    want = [lpmm.lpmm_f8_linear(v, q) for v in sets]
    y = torch.empty(t, n, dtype=BF16, device=DEV)
    room = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    lpmm.lpmm_f8_linear(x, q, y, room, stream=s)
    s.synchronize()
    assert torch.equal(y, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lpmm.lpmm_f8_linear(x, q, y)
        p, pt = lpmm.lpmm_f8_quant_both(x)
        c = lpmm.lpmm_f8_matmul(pt, pt, F32)
    for i in (0, 1, 2, 1, 0):
        x.copy_(sets[i])
        graph.replay()
        assert torch.equal(y, want[i])
        eager = lpmm.lpmm_f8_quant_both(sets[i])
        assert torch.equal(p.codes, eager[0].codes) and torch.equal(pt.scales, eager[1].scales)
        assert torch.equal(c, lpmm.lpmm_f8_matmul(eager[1], eager[1], F32))
        torch.randn(1000, device=DEV).sum().item()


def test_refusals():
    q = lpmm.lpmm_f8_quant(torch.randn(20, 130, device=DEV), 128)
    x = torch.randn(30, 130, device=DEV)
    need = lpmm.lib().lpmm_f8_linear_workspace_bytes(30, 20, 130)
    assert need > 0
    with pytest.raises(lpmm.LpmmError, match="workspace"):
        lpmm.lpmm_f8_linear(x, q, workspace=torch.empty(need - 1, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        lpmm.lpmm_f8_linear(x.cpu(), q)
    with pytest.raises(ValueError):
        lpmm.lpmm_f8_linear(x, q, y=torch.empty(30, 20, device=DEV, dtype=BF16))
    with pytest.raises(ValueError):
        lpmm.lpmm_f8_matmul(q, lpmm.lpmm_f8_quant(x[:, :128]))


# ---- the layer -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,w_dtype", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("t", [1, 9, 150])
def test_layer_and_gradients(t, dtype, w_dtype):
    """y, dx and dW against their formulas, each from its own 8-bit operands"""
    n, k = 140, 270
    x, w, dy = matrix(t, k, dtype, 1, 0.6), matrix(n, k, w_dtype, 2, 0.6), matrix(t, n, dtype, 3, 0.6)
    layer = lpmm.F8Linear.from_weight(w.to(DEV))
    xd = x.to(DEV).requires_grad_()
    y = layer(xd)
    dx, dw = torch.autograd.grad(y, (xd, layer.weight), dy.to(DEV))
    assert y.dtype == dx.dtype == dtype and dw.dtype == w_dtype
    val = lambda m, tile=1: ref.quantize(m, tile)[0]
    qw = val(w, 128)
    ref.check_product(y, val(x), qw, "y")
    ref.check_product(dx, val(dy), qw.t().contiguous(), "dx")
    ref.check_product(dw, val(dy.t()), val(x.t()), "dW")
    # one of the two alone gives the same values
    dx1, = torch.autograd.grad(lpmm.f8_linear(xd, layer.weight.detach()), xd, dy.to(DEV))
    dw1, = torch.autograd.grad(layer(x.to(DEV)), layer.weight, dy.to(DEV))
    ref.check_product(dx1, val(dy), qw.t().contiguous(), "dx alone")
    assert torch.equal(dw1, dw)


@pytest.mark.parametrize("dtype,w_dtype", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("t,n,k", [(1, 1, 1), (130, 257, 100), (20, 40, 515)])
def test_training_calls(t, n, k, dtype, w_dtype):
    """Tensors with gaps and off their boundaries, each choice of gradients, and the second call repeated"""
    x, w, dy = matrix(t, k, dtype, 1, 0.6), matrix(n, k, w_dtype, 2, 0.6), matrix(t, n, dtype, 3, 0.6)
    rooms = []

    def apart(rows, cols, dtype, value=None):
        room = torch.full((rows, cols + 5), 77.0, dtype=dtype, device=DEV)
        rooms.append((room, cols))
        if value is not None:
            room[:, 1:1 + cols] = value.to(DEV)
        return room[:, 1:1 + cols]

    val = lambda m, tile=1: ref.quantize(m, tile)[0]
    qw = val(w, 128)
    xs, ws, dys = apart(t, k, dtype, x), apart(n, k, w_dtype, w), apart(t, n, dtype, dy)
    first = None
    for grads in (lpmm.F8_DX | lpmm.F8_DW, lpmm.F8_DX, lpmm.F8_DW):
        y, kept = lpmm.lpmm_f8_train_forward(xs, ws, grads, apart(t, n, dtype))
        ref.check_product(y, val(x), qw, "y")
        copy = kept.clone()
        dx, dw = lpmm.lpmm_f8_train_backward(dys, kept, k, w_dtype, grads, apart(t, k, dtype) if grads & lpmm.F8_DX else None, apart(n, k, w_dtype) if grads & lpmm.F8_DW else None)
        again = lpmm.lpmm_f8_train_backward(dys, kept, k, w_dtype, grads)
        assert torch.equal(kept, copy)
        if grads & lpmm.F8_DX:
            ref.check_product(dx, val(dy), qw.t().contiguous(), "dx")
            assert torch.equal(dx, again[0])
        else:
            assert dx is again[0] is None
        if grads & lpmm.F8_DW:
            ref.check_product(dw, val(dy.t()), val(x.t()), "dW")
            assert torch.equal(dw, again[1]) and dw.dtype == w_dtype
        else:
            assert dw is again[1] is None
        first = first or (y, dx, dw)
        assert torch.equal(y, first[0]) and (dx is None or torch.equal(dx, first[1])) and (dw is None or torch.equal(dw, first[2]))
    y, kept = lpmm.lpmm_f8_train_forward(xs, ws, 0)
    assert kept is None and torch.equal(y, first[0]) and lpmm.lpmm_f8_train_backward(dys, kept, k, grads=0) == (None, None)
    for room, cols in rooms:
        assert bool((room[:, 0] == 77).all()) and bool((room[:, 1 + cols:] == 77).all()), "around the rows"


def test_training_calls_captured():
    """On another stream with its own memory, and captured and replayed with other values between"""
    t, n, k = 70, 130, 200
    sets = [(matrix(t, k, BF16, s).to(DEV), matrix(n, k, F32, s + 9).to(DEV), matrix(t, n, BF16, s + 5).to(DEV)) for s in (1, 2, 3)]

    def step(x, w, dy, stream=None, y=None, kept=None, dx=None, dw=None, room=None):
        y, kept = lpmm.lpmm_f8_train_forward(x, w, y=y, kept=kept, workspace=room, stream=stream)
        return (y, *lpmm.lpmm_f8_train_backward(dy, kept, k, dx=dx, dw=dw, workspace=room, stream=stream))

    want = [step(*s) for s in sets]
    L = lpmm.lib()
    kept = torch.empty(L.lpmm_f8_train_kept_bytes(t, n, k, 3), dtype=torch.uint8, device=DEV)
    room = torch.empty(L.lpmm_f8_train_workspace_bytes(t, n, k), dtype=torch.uint8, device=DEV)
    outs = [torch.empty_like(o) for o in want[0]]
    x, w, dy = (v.clone() for v in sets[0])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    step(x, w, dy, s, outs[0], kept, outs[1], outs[2], room)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(x, w, dy)
    for i in (0, 1, 2, 1, 0):
        for to, v in zip((x, w, dy), sets[i]):
            to.copy_(v)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
        torch.randn(1000, device=DEV).sum().item()
    with pytest.raises(ValueError):
        lpmm.lpmm_f8_train_forward(x, w, stream=s)               # memory of the current stream for another
    with pytest.raises(lpmm.LpmmError):
        lpmm.lpmm_f8_train_forward(x, w, kept=kept[:-1])
    with pytest.raises(lpmm.LpmmError):
        lpmm.lpmm_f8_train_backward(dy, kept, k, workspace=room[8:])
    with pytest.raises(ValueError):
        lpmm.lpmm_f8_train_backward(dy, kept.cpu(), k)


def test_layer_without_gradients():
    """No gradients wanted: nothing is kept, and the product is as close"""
    layer = lpmm.F8Linear(300, 70)
    x = matrix(50, 300, BF16, 1).to(DEV).requires_grad_()
    val = ref.quantize(x.detach().cpu(), 1)[0], ref.quantize(layer.weight.detach().cpu(), 128)[0]
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            y = layer(x)
        assert y.grad_fn is None and not y.requires_grad
        ref.check_product(y, *val, str(mode))


def test_gradients_against_differences():
    """Whole numbers up to 15 with a 15 in every block are 8-bit values as they are, both ways round: the layer is linear among them, and a
    difference is the gradient's."""
    g = torch.Generator().manual_seed(6)
    t, n, k = 20, 30, 200
    whole = lambda r, c: torch.randint(-7, 8, (r, c), generator=g).float()
    x, w, dy = whole(t, k), whole(n, k), whole(t, n)
    x[0], x[:, 0], x[:, 128], w[0, 0], w[0, 128], dy[0], dy[:, 0] = 15, 15, 15, 15, 15, 15, 15
    xd, wd, dyd = x.to(DEV).requires_grad_(), w.to(DEV).requires_grad_(), dy.to(DEV)
    loss = lambda a, b: (lpmm.f8_linear(a, b).double() * dyd.double()).sum()
    dx, dw = torch.autograd.grad(loss(xd, wd), (xd, wd))
    for _ in range(5):
        sx, sw = whole(t, k).to(DEV).clamp(-1, 1), whole(n, k).to(DEV).clamp(-1, 1)
        sx[0], sx[:, 0], sx[:, 128], sw[0, 0], sw[0, 128] = 0, 0, 0, 0, 0
        assert float(loss(xd + sx, wd) - loss(xd, wd)) == float((dx.double() * sx.double()).sum())
        assert float(loss(xd, wd + sw) - loss(xd, wd)) == float((dw.double() * sw.double()).sum())


def test_layer_shapes_and_states():
    torch.manual_seed(0)
    layer = lpmm.F8Linear(100, 33)
    other = lpmm.F8Linear(100, 33)
    other.load_state_dict(layer.state_dict())
    x = torch.randn(2, 3, 100, device=DEV, requires_grad=True)
    y = layer(x)
    assert y.shape == (2, 3, 33) and torch.equal(y, other(x))
    y.sum().backward()                                       # a gradient that arrives expanded
    first, first_x = layer.weight.grad.clone(), x.grad.clone()
    layer.weight.grad = x.grad = None
    (layer(x).permute(2, 0, 1) * torch.ones(33, 2, 3, device=DEV)).sum().backward()        # and one that arrives transposed
    assert torch.equal(layer.weight.grad, first) and torch.equal(x.grad, first_x)
    empty = torch.empty(0, 100, device=DEV, requires_grad=True)
    layer.weight.grad = None
    layer(empty).sum().backward()
    assert empty.grad.shape == (0, 100) and not bool(layer.weight.grad.any())
    one = layer(torch.randn(100, device=DEV))
    assert one.shape == (33,)
    with pytest.raises(ValueError):
        layer(torch.randn(5, 99, device=DEV))


def test_more_rows_than_a_launch_has_workgroups():
    """Every matrix that lpmm_f8_sizes takes is brought to 8 bits: beyond 2^25 rows of one block, which end within a workgroup's four"""
    rows = 4 * 2 ** 23 + 5
    i = torch.arange(rows, device=DEV)
    x = ((i % 7 + 1).float() * torch.exp2((i % 11 - 5).float())).to(BF16)[:, None].expand(rows, 2).contiguous()
    x[-1, 1] = 448 * 2.0 ** 9
    q = lpmm.lpmm_f8_quant(x)
    assert torch.equal(lpmm.lpmm_f8_dequant(q, BF16)[:-1], x[:-1])
    for part in (slice(0, 9), slice(rows // 2, rows // 2 + 9), slice(rows - 9, rows)):
        want, scales = ref.quantize(x[part].cpu(), 1)
        assert torch.equal(q.scales[0, part].cpu().long(), scales[:, 0])
        assert ref.same(lpmm.lpmm_f8_dequant(lpmm.lpmm_f8_quant(x[part]), F32).cpu().double(), want)
        assert torch.equal(q.codes[part], lpmm.lpmm_f8_quant(x[part]).codes)
    assert q.scales[0, rows:].tolist() == [0, 0, 0] and bool((q.codes[:, 2:] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,n,k", [(1, 24576, 4100), (8, 24575, 4096), (8, 24577, 5000), (9, 32768, 4096), (3, 32769, 4001), (11, 24576, 4096), (12, 24576, 4096), (16, 24575, 4000), (16, 24577, 4000),
                                   (16, 65536, 4096), (16, 65537, 4096), (13, 50257, 2560), (5, 16384, 8192)])
def test_few_tokens_next_to_the_rules_borders(t, n, k, dtype):
    """Whichever kernel takes them, rows of W at the start, at the end, and where tiles meet"""
    progress(f"{t} x {n} x {k} {dtype}")
    x, w = matrix(t, k, dtype, t + k, 0.7), matrix(n, k, BF16, n, 0.7)
    q = lpmm.lpmm_f8_quant(w.to(DEV), 128)
    y = lpmm.lpmm_f8_linear(x.to(DEV), q)
    some = torch.cat([torch.arange(40), torch.arange(n // 2, n // 2 + 300), torch.arange(n - 70, n)]).to(DEV)
    values = lpmm.lpmm_f8_dequant(q)[some].cpu().double()
    ref.check_product(y[:, some], ref.quantize(x, 1)[0], values, f"{t} x {n} x {k}")
    assert torch.equal(y, lpmm.lpmm_f8_linear(x.to(DEV), q)) and bool(torch.isfinite(y).all())


def cut_off(a, b):
    """How much the matrix instructions on 8 bits may lose of each of a's rows times each of b's, from the codes: of each eight neighbouring products, up to seven times 2^-13 of the largest
    2^(ea + eb), with the exponents of the codes, -6 for those below the normal numbers, and of products that are not 0"""
    def exponents(m):
        codes = m.codes.cpu().long() & 127
        scales = m.scales.cpu().double()
        scales = scales[:, :m.rows].t() if m.tile == 1 else scales[:, :codes.shape[1] // 128].repeat_interleave(128, 0)[:m.rows]
        e = ((codes >> 3).clamp(min=1) - 7).double() + (scales - 127).repeat_interleave(128, 1)
        return torch.where(codes > 0, e, torch.full_like(e, -INF))
    ea, eb = exponents(a), exponents(b)
    return torch.stack([torch.exp2((ea[i] + eb).view(b.rows, -1, 8).amax(2) - 13).sum(1) * 7 for i in range(a.rows)])


def check_cut(x, w, what):
    """x: in bf16 too.  Few tokens and tiles; rounding to bf16, what is cut off, and a rounding of fp32 for each term"""
    w = w.to(DEV)
    b = lpmm.lpmm_f8_quant(w, 128)
    a = lpmm.lpmm_f8_quant(x.to(DEV))
    va, vb = ref.unpack(a)[0], ref.unpack(b)[0]
    want, size = va @ vb.t().contiguous(), va.abs() @ vb.abs().t().contiguous()
    lost = cut_off(a, b)
    for form, got in (("tiles", lpmm.lpmm_f8_matmul(a, b)), ("linear", lpmm.lpmm_f8_linear(x.to(DEV).bfloat16(), b))):
        ref.assert_within(got, want, 2.0 ** -8 * want.abs() + (1 + 2.0 ** -8) * (lost + x.shape[1] * 2.0 ** -24 * size), f"{what} {form}")
    ref.check_product(lpmm.lpmm_f8_matmul(a, b, F32), va, vb, f"{what} fp32")
    return want, lost


@pytest.mark.parametrize("m,n,k,spread", [(3, 70, 1000, 1.0), (16, 33, 515, 4.0), (40, 70, 640, 4.0), (40, 50, 300, 8.0)])
def test_what_results_of_16_bits_lose(m, n, k, spread):
    """Elements that spread over codes below the normal numbers, with zeros among them"""
    g = torch.Generator().manual_seed(m + n)
    x, w = (torch.randn(r, k, generator=g) * (spread * torch.randn(r, k, generator=g)).exp() for r in (m, n))
    x[x < 0] = 0.0
    check_cut(x.bfloat16().float(), w, f"{m} x {n} x {k} {spread}")


@pytest.mark.parametrize("t", [2, 20])
def test_the_most_that_results_of_16_bits_lose(t):
    """Of a product whose code is the least of all, 2^-9 times 256, and seven of just below 2^-11 beside it these are lost, 2^-7.3 of the sum; a block's largest codes meet zeros.  And sums
    that cancel: nothing of them is left but what fp32 keeps."""
    x, w = torch.zeros(t, 256), torch.zeros(5, 256)
    x[:, 8], w[:, 8] = 2.0 ** -9, 256.0
    x[:, 9:16], w[:, 9:16] = 1.875 * 2.0 ** -6, 2.0 ** -6
    x[:, 100], w[:, 120] = 448.0, 448.0
    want, lost = check_cut(x, w, "least code")
    assert 2.0 ** -8 < float((lost / want)[0, 0]) < 2.0 ** -7
    x, w = torch.zeros(t, 256), torch.zeros(5, 256)
    x[:, :8], w[:, 2:8] = 2.0 ** -7, 2.0 ** -7
    x[:, 0] = x[:, 1] = w[:, 0] = 16.0
    w[:, 1] = -16.0
    want, lost = check_cut(x, w, "cancels")
    assert bool((want == 6 * 2.0 ** -14).all()) and bool((lost > want).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("blocks", [1, 2, 4, 5, 9, 10])
def test_large_tiles_of_any_number_of_blocks(blocks, dtype):
    """256 x 256: the loop over two blocks a turn not at all, once and many times, and one or two blocks behind it"""
    product_of(4100, 2600, 128 * blocks - 3, dtype, (1, 128), blocks)
