"""Microscaled 4-bit floating point on the GPU: quantisation and its inverse bit for bit against the definition in 64 bits, the
product against the product of the values that codes and scales stand for, in 64 bits.

Tolerance of a product: its terms are exact, and the tensor core adds 64 of them (in groups of 32 with one pair of scales) at a
time to an fp32 accumulator; each of these additions, and each of up to 8 that join the parts of a split sum, is off by at most a
step (2^-23, it may truncate) of a value that is at most sum |x w|.  So an output is within (d_in / 32 + 12) 2^-23 sum |x w|, plus
2^-24 of itself for the bias, plus half a step where it is rounded to bf16."""
import math

import pytest

import paper_2210_03858_b200 as bcq
from paper_2210_03858_b200 import build as bcq_build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


@pytest.fixture(scope="module", autouse=True)
def _built():
    bcq_build.build_library()
    yield
    bcq.check_device()
    assert bcq.device_timeout_flag() == 0


def ref_quantize(x):
    """(codes [rows][cols], exponents + 127 [rows][blocks]) from the definition."""
    rows, cols = x.shape
    v = torch.zeros((rows, -(-cols // 32) * 32), dtype=torch.float64, device=x.device)
    v[:, :cols] = x.double()
    v = v.view(rows, -1, 32)
    top = v.abs().amax(dim=2, keepdim=True)
    bad = ~torch.isfinite(v).all(dim=2, keepdim=True)
    mantissa, e = torch.frexp(torch.where(bad | (top == 0), 1.0, top))    # mantissa in [1/2, 1)
    e = torch.where(top == 0, -127, (e - 1 - 2).clamp(min=-127))
    a = torch.where(bad, 0.0, torch.ldexp(v.abs(), -e))
    code = torch.zeros_like(a, dtype=torch.int32)
    for i in range(7):  # the point halfway between magnitudes i and i + 1 goes to the even one
        half = (MAGNITUDES[i] + MAGNITUDES[i + 1]) / 2
        code += ((a > half) if i % 2 == 0 else (a >= half)).int()
    code += 8 * (torch.signbit(v) & ~bad).int()
    s = torch.where(bad, 255, e + 127)[:, :, 0]
    return code.view(rows, -1)[:, :cols], s


def unpack(M):
    """(codes [rows][cols], scales [rows][blocks]) of a container, and whether all that is behind rows and columns is 0."""
    code = torch.stack((M.codes & 15, M.codes >> 4), dim=2).view(M.rows, -1).int()
    a = -(-M.cols // 128)
    s = M.scales.permute(0, 3, 2, 1, 4).reshape(-1, 4 * a).int()
    blocks = -(-M.cols // 32)
    clean = not bool(code[:, M.cols:].any()) and not bool(s[M.rows:].any()) and not bool(s[:, blocks:].any())
    return code[:, :M.cols], s[:M.rows, :blocks], clean


def values_of(M):
    code, s, _ = unpack(M)
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float64, device="cuda")
    f = torch.where(s == 255, math.nan, torch.exp2(s.double() - 127))
    return table[code.long()] * f.repeat_interleave(32, dim=1)[:, :M.cols]


def spread(rows, cols, dtype, seed, offset=0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, cols), generator=g, device="cuda") * torch.exp2(torch.randint(-20, 20, (rows, 1), generator=g, device="cuda").float())
    buf = torch.full((rows * (cols + pad) + offset,), math.nan, dtype=dtype, device="cuda")
    out = buf[offset:].view(rows, cols + pad)[:, :cols]
    out.copy_(x)
    return out


def check_quantize(x):
    M = bcq.mx_quantize(x)
    code, s, clean = unpack(M)
    ref_code, ref_s = ref_quantize(x)
    assert torch.equal(s, ref_s.int()) and clean
    assert torch.equal(code, ref_code)
    for dtype in (F32, BF16):
        v = bcq.mx_dequantize(M, out_dtype=dtype)
        assert v.dtype == dtype and torch.equal(torch.nan_to_num(v.double(), 9e9), torch.nan_to_num(values_of(M), 9e9))
    return M


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,pad,offset", [(1, 1, 0, 0), (1, 31, 0, 1), (3, 33, 0, 0), (5, 128, 0, 0), (127, 129, 7, 0), (128, 256, 0, 0),
                                                  (129, 1000, 0, 0), (129, 1000, 24, 8), (300, 1001, 0, 3), (2, 16384, 0, 0), (777, 640, 0, 0),
                                                  (40000, 64, 0, 0)])
def test_quantize_sizes(dtype, rows, cols, pad, offset):
    check_quantize(spread(rows, cols, dtype, rows + cols, offset, pad))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantize_every_rounding_border(dtype):
    # multiples of 1/64 from -8 to 8 are 13 steps to each side of every border; the block's largest fixes its scale
    grid = torch.arange(-512, 513, device="cuda").float() / 64
    rows = []
    for top in (4.0, 5.0, 6.0, 7.0, 7.96875):
        inside = grid[grid.abs() <= top]
        inside = torch.nn.functional.pad(inside, (0, -len(inside) % 31)).view(-1, 31)
        rows.append(torch.cat((inside, torch.full((len(inside), 1), top, device="cuda")), dim=1))
    x = torch.cat(rows)
    for e in (-140, -128, -127, -126, -20, 0, 100, 124):
        check_quantize(torch.ldexp(x.double(), torch.tensor(e, device="cuda")).float().to(dtype))
    check_quantize(torch.nextafter(x, torch.tensor(9.0, device="cuda")).to(dtype))
    check_quantize(torch.nextafter(x, torch.tensor(-9.0, device="cuda")).to(dtype))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantize_zeros_extremes_and_values_that_are_none(dtype):
    x = torch.zeros((9, 100), device="cuda")
    x[1, ::2] = -0.0
    x[2, 5] = torch.finfo(dtype).max
    x[3, 40] = -torch.finfo(dtype).max
    x[4] = torch.finfo(dtype).smallest_normal
    x[5, 3:9] = 2.0 ** -133
    x[6, 33] = math.nan
    x[6, 34] = 3.0
    x[7, 99] = math.inf
    x[7, 10] = 1.0
    x[8, 64] = -math.inf
    M = check_quantize(x.to(dtype))
    _, s, _ = unpack(M)
    assert (s == 255).nonzero().tolist() == [[6, 1], [7, 3], [8, 2]]


# ---------------------------------------------------------------- product

def check_linear(n, d_in, d_out, dtype=F32, bias=False, seed=0, x_dtype=BF16):
    g = torch.Generator(device="cuda").manual_seed(seed + n + d_in)
    X = bcq.mx_quantize(torch.randn((n, d_in), generator=g, device="cuda").to(x_dtype))
    W = bcq.mx_quantize(torch.randn((d_out, d_in), generator=g, device="cuda") * torch.exp2(torch.randint(-9, 9, (d_out, 1), generator=g, device="cuda").float()))
    b = torch.randn(d_out, generator=g, device="cuda") if bias else None
    buf = torch.full((n + 2, d_out + 5), 7.0, dtype=dtype, device="cuda")
    out = buf[1:n + 1, 2:d_out + 2]
    assert bcq.mx_linear(X, W, bias=b, out=out) is out
    x, w = values_of(X), values_of(W)
    ref, size = x @ w.t(), x.abs() @ w.abs().t()
    if bias:
        ref, size = ref + b.double(), size + b.double().abs()
    tol = (d_in / 32 + 12) * 2.0 ** -23 * size + (torch.finfo(dtype).eps / 2 if dtype == BF16 else 2.0 ** -24) * ref.abs() * 1.01
    off = (out.double() - ref).abs() - tol
    assert torch.isfinite(out).all() and float(off.max()) <= 0, float(off.max())
    # nothing around the result is touched
    buf[1:n + 1, 2:d_out + 2] = 7.0
    assert bool((buf == 7).all())
    again = bcq.mx_linear(X, W, bias=b, out_dtype=dtype)
    assert torch.equal(again, bcq.mx_linear(X, W, bias=b, out_dtype=dtype))
    return X, W


def test_linear_of_one_tile():
    # the smallest whole tile first: 128 outputs, 16 tokens, one step
    check_linear(16, 256, 128)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 33, 64, 65, 128, 129, 256, 300])
@pytest.mark.parametrize("d_in,d_out", [(1, 1), (32, 5), (33, 130), (128, 128), (129, 64), (256, 300), (384, 257), (1000, 1528), (4104, 700)])
def test_linear_sizes(n, d_in, d_out):
    check_linear(n, d_in, d_out, F32 if n % 2 else BF16, bias=(n + d_in) % 3 == 0)


@pytest.mark.parametrize("n,d_in,d_out", [(1, 16384, 4096), (4, 4096, 12288), (16, 1600, 6400), (512, 1024, 1024), (2048, 1600, 6400),
                                          (700, 5120, 5000), (4000, 640, 20000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_linear_larger(n, d_in, d_out, dtype):
    check_linear(n, d_in, d_out, dtype, bias=True)


def test_linear_takes_values_and_keeps_nan_apart():
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((20, 500), generator=g, device="cuda").bfloat16()
    w = torch.randn((300, 500), generator=g, device="cuda")
    W = bcq.mx_quantize(w)
    y = bcq.mx_linear(x, W)
    assert torch.equal(y, bcq.mx_linear(bcq.mx_quantize(x), W))
    x2, w2 = x.clone(), w.clone()
    x2[7, 499] = math.inf
    w2[200, 3] = math.nan
    y2 = bcq.mx_linear(x2, bcq.mx_quantize(w2))
    touched = torch.zeros((20, 300), dtype=torch.bool, device="cuda")
    touched[7], touched[:, 200] = True, True
    assert torch.isnan(y2[touched]).all() and torch.equal(y2[~touched], y[~touched])
    assert bcq.mx_linear(x[:0], W).shape == (0, 300)


def test_operands_that_cannot_be_passed_on():
    x = torch.randn((4, 64), device="cuda")
    M = bcq.mx_quantize(x)
    for bad, error in ((x.half(), TypeError), (x[0], ValueError), (x.t(), ValueError), (x.cpu(), ValueError), (3, TypeError)):
        with pytest.raises(error):
            bcq.mx_quantize(bad)
    with pytest.raises(bcq.BcqError):
        bcq.mx_quantize(x[:1].expand(4, 64))
    with pytest.raises(ValueError):
        bcq.MxMatrix(M.codes, M.scales, 4, 200)
    with pytest.raises(ValueError):
        bcq.MxMatrix(M.codes[:3], M.scales, 4, 64)
    with pytest.raises(TypeError):
        bcq.MxMatrix(M.codes.int(), M.scales, 4, 64)
    with pytest.raises(ValueError):
        bcq.mx_linear(M, bcq.mx_quantize(torch.randn((4, 65), device="cuda")))
    with pytest.raises(TypeError):
        bcq.mx_linear(M, M, out_dtype=torch.float16)
    for bad, error in ((torch.zeros(5, device="cuda"), ValueError), (torch.zeros(4, device="cuda", dtype=BF16), TypeError)):
        with pytest.raises(error):
            bcq.mx_linear(M, M, bias=bad)
    for bad, error in ((torch.zeros((4, 5), device="cuda"), ValueError), (torch.zeros((4, 4), device="cuda").half(), TypeError),
                       (torch.zeros((4, 4), device="cuda").t()[:, ::1].t()[:, :4].t(), ValueError)):
        with pytest.raises(error):
            bcq.mx_linear(M, M, out=bad)
    assert torch.equal(bcq.mx_linear(M, M), bcq.mx_linear(M, M, out=torch.empty((4, 4), device="cuda")))


def test_mx_on_a_side_stream_and_in_a_graph():
    g = torch.Generator(device="cuda").manual_seed(4)
    x, x2 = (torch.randn((40, 1024), generator=g, device="cuda").bfloat16() for _ in range(2))
    W = bcq.mx_quantize(torch.randn((4096, 1024), generator=g, device="cuda"))
    expect = bcq.mx_linear(x, W)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = bcq.mx_linear(x, W)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(expect, got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = bcq.mx_linear(x, W)
    x.copy_(x2)
    got.zero_()
    graph.replay()
    graph.replay()
    assert torch.equal(got, bcq.mx_linear(x2, W)) and not torch.equal(got, expect)
