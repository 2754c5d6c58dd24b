"""Matrices in MXFP4 on the GPU: quantisation and its inverse bit for bit, products against float64."""
import math

import pytest
import torch

import mx4_reference as ref
from paper_2601_17768_amd import binding as B
from paper_2601_17768_amd.mx4 import Mx4Matrix

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def values(rows, cols, dtype, seed=0, spread=True):
    g = torch.Generator().manual_seed(seed * 1000003 + rows * 4099 + cols)
    x = torch.randn(rows, cols, generator=g)
    if spread:                                                # every magnitude that the type has room for
        x = x * torch.exp2(torch.randint(-60, 60, (rows, (cols + 31) // 32), generator=g).float()).repeat_interleave(32, 1)[:, :cols]
    return x.to(dtype)


def same(got, want):
    got, want = got.cpu().double(), want.double()
    assert got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (1, 32), (3, 33), (16, 256), (17, 255), (15, 257), (5, 700), (688, 256), (33, 4096)])
def test_quantize_and_values(rows, cols, dtype):
    x = values(rows, cols, dtype)
    m = Mx4Matrix.quantize(x.to(DEV))
    want = ref.quantized(x)
    same(m.values(torch.bfloat16), want)
    same(m.values(torch.float32), want)


def test_every_rounding_tie_and_special_value():
    t = torch.tensor([4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9, 5.05, 0.2, 0.3])
    blocks = [torch.cat((t, -t, torch.zeros(8))) * s for s in (1.0, 2.0 ** -100, 2.0 ** 100, 2.0 ** -126, 2.0 ** 125)]
    blocks += [torch.zeros(32), torch.full((32,), 2.0 ** -133), torch.full((32,), 2.0 ** -127), torch.full((32,), 3.0e38)]
    blocks += [torch.cat((torch.tensor([2.0 ** -126, -(2.0 ** -127), 2.0 ** -128]), torch.zeros(29)))]
    for bad in (math.inf, -math.inf, math.nan):
        blocks.append(torch.cat((torch.ones(31), torch.tensor([bad]))))
    x = torch.cat(blocks)[None]
    for dtype in (torch.bfloat16, torch.float32):
        m = Mx4Matrix.quantize(x.to(dtype).to(DEV))
        same(m.values(torch.float32), ref.quantized(x.to(dtype)))
        same(m.values(torch.bfloat16), ref.quantized(x.to(dtype)))


def test_every_bf16_value():
    """Blocks of a value and its magnitude's neighbours under a leading value that fixes the scale: all mantissas at each level."""
    bits = torch.arange(1 << 16, dtype=torch.int32)
    x = (bits << 16).view(torch.float32)
    x = torch.where(torch.isfinite(x), x, 0.0)
    lead = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -120, max=2.0 ** 118))) + 2)
    for shift in (1.0, 0.5, 0.25, 0.125):                     # the value at 1, 1/2, 1/4, 1/8 of the block's largest power of two
        block = torch.zeros(1 << 16, 32)
        block[:, 0], block[:, 7] = lead * shift, x
        block = block.to(torch.bfloat16)
        m = Mx4Matrix.quantize(block.to(DEV))
        same(m.values(torch.float32), ref.quantized(block))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_apart_and_off_alignment(dtype):
    x = values(20, 75, dtype)
    for offset, stride in ((0, 80), (1, 77), (3, 83)):
        buf = torch.full((offset + 20 * stride,), 7.0, dtype=dtype, device=DEV)
        view = buf[offset:].view(20, stride)[:, :75]
        view.copy_(x)
        m = Mx4Matrix.quantize(view)
        same(m.values(torch.float32), ref.quantized(x))
        view.fill_(9.0)
        m.values(out=view)
        same(view, ref.quantized(x))
        assert bool((buf[offset:].view(20, stride)[:, 75:] == 7.0).all()) and bool((buf[:offset] == 7.0).all())


def product_tolerance(x, w, out_dtype):
    """fp32 sums of k exact products, in any order, are off by at most k roundings of what has been summed so far (2^-23 of it each, a
    matrix instruction may truncate); then one rounding to the output type."""
    x, w = x.double(), w.double()
    k = x.shape[1]
    want = x @ w.T
    tol = k * 2.0 ** -23 * (x.abs() @ w.abs().T) + 1e-37
    return want, tol + want.abs() * torch.finfo(out_dtype).eps / 2


SIZES = [(1, 16, 32), (1, 1, 1), (2, 17, 31), (3, 40, 33), (5, 100, 256), (16, 64, 512), (17, 48, 288), (32, 688, 256), (33, 250, 700),
         (64, 128, 1024), (65, 130, 520), (100, 300, 96), (128, 512, 256), (129, 4112, 64), (200, 96, 2080), (257, 1000, 320), (300, 48, 4096),
         (513, 528, 160), (1000, 272, 736), (4, 8200, 128), (24, 4096, 512)]


@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,n,k", SIZES)
def test_product(rows, n, k, out_dtype):
    x, w = values(rows, k, torch.bfloat16, 1, False), values(n, k, torch.bfloat16, 2, False) * 0.02
    m = Mx4Matrix.quantize(w.to(DEV))
    got = m.matmul(x.to(DEV), out_dtype).cpu().double()
    want, tol = product_tolerance(x, ref.quantized(w), out_dtype)
    err = (got - want).abs()
    assert bool((err <= tol).all()), f"largest error {float(err.max()):.3e}, tolerance there {float(tol.flatten()[err.argmax()]):.3e}"


# every tile and number of parts that the choice takes on 256 CUs, with plain rows (columns a multiple of 32) and packed ones
TILES = [(130, 33000, 260), (130, 33000, 288), (70, 33000, 260), (70, 33000, 288), (70, 16400, 260), (70, 16400, 288), (265, 1000, 8200),
         (265, 1000, 8192), (525, 6000, 260), (525, 6000, 288), (130, 2000, 8200), (130, 2000, 8192), (9, 33000, 260), (20, 33000, 288),
         (35, 4112, 8200), (35, 4112, 8192), (35, 16400, 260), (45, 16400, 288), (130, 1000, 8200), (130, 1000, 8192), (35, 8200, 545),
         (35, 8200, 544), (130, 500, 8200), (130, 500, 8192), (9, 16400, 260), (20, 16400, 288), (70, 1000, 8200), (70, 1000, 8192),
         (20, 8200, 8192), (9, 4112, 4100), (9, 4112, 4096), (9, 40, 8200), (20, 40, 8192), (9, 40, 4100), (20, 40, 4096), (1, 40, 8200),
         (5, 5000, 1090), (16, 20, 31), (1, 3, 1), (12, 40, 4100), (16, 33000, 287), (16, 33000, 4095), (7, 60, 257), (2, 8200, 223),
         (8, 5000, 1088), (9, 8200, 1090), (16, 8200, 1088), (3, 9000, 2050), (8, 33000, 1024 + 64), (20, 33000, 260), (20, 4112, 4100),
         (20, 40, 8200), (20, 40, 4100), (20, 16400, 260), (24, 33000, 33), (9, 14336, 260), (6, 24000, 96),
         (3, 61000, 40), (20, 5000, 288), (30, 9000, 1024), (32, 16000, 2048), (17, 15000, 4100), (31, 300, 64), (17, 16, 33), (65536, 48, 96), (65536, 17, 1030), (30000, 16, 4128)]


@pytest.mark.parametrize("rows,n,k", TILES)
def test_product_by_every_tile(rows, n, k):
    g = torch.Generator(device=DEV).manual_seed(rows + n + k)
    x = torch.randn(rows, k, generator=g, device=DEV).to(torch.bfloat16)
    m = Mx4Matrix.quantize(torch.randn(n, k, generator=g, device=DEV))
    w = m.values(torch.float32)                               # (bit for bit: the tests above)
    out = torch.full((rows + 1, n + 3), 7.0, device=DEV)
    m.matmul(x, out=out[:rows, :n])
    want, tol = product_tolerance(x, w, torch.float32)
    assert bool(((out[:rows, :n].double() - want).abs() <= tol).all())
    assert bool((out[rows] == 7.0).all()) and bool((out[:, n:] == 7.0).all())


def test_product_without_a_workspace_sums_in_one_piece():
    x, w = values(24, 4096, torch.bfloat16, 1, False).to(DEV), values(100, 4096, torch.bfloat16, 2, False).to(DEV)
    m, out = Mx4Matrix.quantize(w), torch.empty(24, 100, device=DEV)
    B.llm42_mx4_matmul(m.data, x, out)
    want, tol = product_tolerance(x, m.values(torch.float32), torch.float32)
    assert bool(((out.double() - want).abs() <= tol).all())


def test_product_by_one_hot_rows_returns_the_matrix():
    """Conversion and layout: every column of the matrix, bit for bit, whatever its scale."""
    w = values(45, 288, torch.bfloat16, 3)
    m = Mx4Matrix.quantize(w.to(DEV))
    got = m.matmul(torch.eye(288, dtype=torch.bfloat16, device=DEV), torch.float32)
    same(got.T, ref.quantized(w))


@pytest.mark.parametrize("rows,n,k", [(3, 50, 64), (70, 50, 64), (3, 50, 75), (130, 270, 75), (1, 33, 40)])
def test_product_of_rows_apart_and_off_alignment(rows, n, k):
    x, w = values(rows, k, torch.bfloat16, 1, False), values(n, k, torch.bfloat16, 2, False)
    m = Mx4Matrix.quantize(w.to(DEV))
    for dtype in (torch.bfloat16, torch.float32):
        want, tol = product_tolerance(x, ref.quantized(w), dtype)
        for offset, stride in ((0, k + (-k) % 8 + 8), (1, k + 3), (8, k)):
            buf = torch.full((offset + rows * stride + 8,), math.nan, dtype=torch.bfloat16, device=DEV)
            xv = buf[offset:offset + rows * stride].view(rows, stride)[:, :k]
            xv.copy_(x)
            ob = torch.full((offset + rows * (n + 5),), 7.0, dtype=dtype, device=DEV)
            ov = ob[offset:].view(rows, n + 5)[:, :n]
            m.matmul(xv, out=ov)
            assert bool(((ov.cpu().double() - want).abs() <= tol).all()), (offset, stride)
            assert bool((ob[offset:].view(rows, n + 5)[:, n:] == 7.0).all()) and bool((ob[:offset] == 7.0).all())


def test_nan_and_infinity_reach_the_rows_and_columns_that_hold_them_alone():
    x, w = values(40, 96, torch.bfloat16, 1, False), values(70, 96, torch.bfloat16, 2, False)
    x[3, 5], x[39, 95], w[69, 90] = math.nan, math.inf, math.inf
    got = Mx4Matrix.quantize(w.to(DEV)).matmul(x.to(DEV), torch.float32).cpu()
    bad = ~torch.isfinite(got)
    want = torch.zeros(40, 70, dtype=torch.bool)
    want[3], want[39], want[:, 69] = True, True, True
    # (an infinite activation times a weight of zero is NaN, times any other it is infinite: not finite either way)
    assert torch.equal(bad, want)
    assert bool(torch.isnan(got[3]).all()) and bool(torch.isnan(got[:, 69]).all())


@pytest.mark.parametrize("rows", [1, 24, 100])
def test_replays_and_streams_give_the_same_bits(rows):
    x, w = values(rows, 512, torch.bfloat16, 1, False).to(DEV), values(300, 512, torch.bfloat16, 2, False).to(DEV)
    m = Mx4Matrix.quantize(w)
    out = torch.zeros(rows, 300, dtype=torch.float32, device=DEV)
    want = m.matmul(x, torch.float32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = m.matmul(x, torch.float32)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(on_side, want)
    m.matmul(x, out=out)
    product_magnitude = x.float().abs() @ m.values(torch.float32).abs().T
    graph = torch.cuda.CUDAGraph()
    data = m.data
    with torch.cuda.graph(graph):
        Mx4Matrix.quantize(w, data)
        m.matmul(x, out=out)
    for scale in (1.0, -2.0, 0.5):
        w.copy_(values(300, 512, torch.bfloat16, 2, False) * scale)
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        # (not want * scale bit for bit: a matrix instruction does not round a sum and its negative alike)
        assert torch.equal(out, Mx4Matrix.quantize(w).matmul(x, torch.float32))
        assert bool(((out - want * scale).abs() <= abs(scale) * 512 * 2.0 ** -23 * product_magnitude).all())


def test_a_matrix_of_more_than_4_gib():
    """Its last rows and their offsets beyond 32 bits, in values, product and codes."""
    n, k = (1 << 21) + 40, 4096
    src = torch.empty(n, k, dtype=torch.bfloat16, device=DEV)
    src[:48], src[-48:] = values(48, k, torch.bfloat16, 1, False).to(DEV), values(48, k, torch.bfloat16, 2, False).to(DEV)
    m = Mx4Matrix.quantize(src)
    assert m.data.numel() > 2 ** 32
    small = [Mx4Matrix.quantize(src[:48].contiguous()), Mx4Matrix.quantize(src[-40:].contiguous())]
    assert torch.equal(m.data[:small[0].data.numel()], small[0].data) and torch.equal(m.data[-small[1].data.numel():], small[1].data)
    m.values(out=src)
    same(src[-40:].cpu(), small[1].values().cpu())
    for rows in (3, 24, 70):
        x = values(rows, k, torch.bfloat16, 3, False).to(DEV)
        got = m.matmul(x, torch.float32)
        for a, part in ((got[:, :48], small[0]), (got[:, -40:], small[1])):
            want, tol = product_tolerance(x, part.values(torch.float32), torch.float32)
            assert bool(((a.double() - want).abs() <= tol).all())


def test_product_of_rows_far_apart():
    """More than 2^26 elements: beyond 16 rows packed first, which needs the workspace."""
    far = (1 << 26) + 8
    x = torch.zeros(16 * far + 64, dtype=torch.bfloat16, device=DEV).as_strided((17, 64), (far, 1))
    x.copy_(values(17, 64, torch.bfloat16, 1, False))
    m = Mx4Matrix.quantize(values(20, 64, torch.bfloat16, 2, False).to(DEV))
    for rows in (2, 16, 17):
        want, tol = product_tolerance(x[:rows].contiguous(), m.values(torch.float32), torch.float32)
        assert bool(((m.matmul(x[:rows], torch.float32).double() - want).abs() <= tol).all())
    with pytest.raises(B.Llm42Error) as e:
        B.llm42_mx4_matmul(m.data, x, torch.zeros(17, 20, device=DEV))
    assert e.value.status == B.LLM42_EWORKSPACE


@pytest.mark.parametrize("rows,n,k", [(24, 100, 4096), (24, 100, 4100), (9, 40, 8200), (3, 50, 75)])
def test_product_stays_within_its_workspace(rows, n, k):
    x, w = values(rows, k, torch.bfloat16, 1, False).to(DEV), values(n, k, torch.bfloat16, 2, False).to(DEV)
    m, need = Mx4Matrix.quantize(w), B.llm42_mx4_matmul_workspace_bytes(rows, n, k)
    ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device=DEV)
    assert torch.equal(m.matmul(x, torch.float32, workspace=ws[:need]), m.matmul(x, torch.float32)) and bool((ws[need:] == 77).all())


def test_the_binding_refuses():
    w = torch.zeros(32, 64, dtype=torch.bfloat16, device=DEV)
    m = Mx4Matrix.quantize(w)
    for x in (torch.zeros(2, 63, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 64, device=DEV), torch.zeros(2, 64, dtype=torch.bfloat16),
              torch.zeros(64, 2, dtype=torch.bfloat16, device=DEV).T):
        with pytest.raises(ValueError):
            m.matmul(x)
    with pytest.raises(ValueError):
        m.values(out=torch.zeros(32, 65, device=DEV))
    with pytest.raises(ValueError):
        Mx4Matrix.quantize(w.half())
    with pytest.raises(B.Llm42Error):
        Mx4Matrix.quantize(w, torch.zeros(4000, dtype=torch.uint8, device=DEV))
