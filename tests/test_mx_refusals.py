"""What the microscaled operators refuse before anything is launched, and the sizes of their container.  No GPU is needed."""
import ctypes as C

import pytest

import paper_2210_03858_b200 as bcq
from paper_2210_03858_b200 import build as bcq_build

P, NULL, ODD = C.c_void_p(256), C.c_void_p(0), C.c_void_p(264)


@pytest.fixture(scope="module", autouse=True)
def _built():
    bcq_build.build_library()


def quantize(rows=4, cols=100, x=P, ld=100, dtype=1, codes=P, scales=P):
    return bcq.lib().bcq_mx_quantize(rows, cols, x, ld, dtype, codes, scales, None)


def dequantize(rows=4, cols=100, x=P, ld=100, dtype=1, codes=P, scales=P):
    return bcq.lib().bcq_mx_dequantize(rows, cols, codes, scales, x, ld, dtype, None)


def linear(d_out=8, d_in=100, n=4, xc=P, xs=P, wc=P, ws=P, bias=NULL, y=P, ldy=8, dtype=0):
    return bcq.lib().bcq_mx_linear(d_out, d_in, n, xc, xs, wc, ws, bias, y, ldy, dtype, None)


def test_container_sizes():
    lib = bcq.lib()
    assert lib.bcq_mx_codes_bytes(3, 1) == 3 * 64 and lib.bcq_mx_codes_bytes(3, 129) == 3 * 128
    assert lib.bcq_mx_scales_bytes(1, 1) == 512 and lib.bcq_mx_scales_bytes(129, 129) == 2048
    assert lib.bcq_mx_codes_bytes(0, 5) == 0 and lib.bcq_mx_scales_bytes(5, 0) == 0
    assert lib.bcq_mx_codes_bytes(2 ** 31 - 1, 2 ** 20) == (2 ** 31 - 1) * 2 ** 19


@pytest.mark.parametrize("call", [quantize, dequantize])
def test_values(call):
    assert call(rows=-1) == -2 and call(cols=0) == -2 and call(ld=99) == -2
    assert call(cols=2 ** 20 + 1, ld=2 ** 21) == -4 and call(dtype=2) == -4
    assert call(x=NULL) == -1 and call(codes=NULL) == -1 and call(scales=NULL) == -1
    assert call(codes=ODD) == -3 and call(scales=ODD) == -3 and call(x=C.c_void_p(257)) == -3 and call(x=C.c_void_p(258), dtype=0) == -3
    assert call(rows=0, x=NULL, codes=NULL, scales=NULL) == 0


def test_linear():
    assert linear(d_out=0) == -2 and linear(d_in=0) == -2 and linear(n=-1) == -2 and linear(ldy=7) == -2
    assert linear(d_in=2 ** 20 + 1) == -4 and linear(dtype=3) == -4
    for name in ("xc", "xs", "wc", "ws", "y"):
        assert linear(**{name: NULL}) == -1, name
    for name in ("xc", "xs", "wc", "ws"):
        assert linear(**{name: ODD}) == -3, name
    assert linear(bias=C.c_void_p(258)) == -3 and linear(y=C.c_void_p(257)) == -3
    assert linear(n=0, xc=NULL, xs=NULL, y=NULL) == 0


def test_tensors_on_the_host_are_refused():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        bcq.mx_quantize(torch.zeros(2, 32))
    with pytest.raises(ValueError):
        bcq.MxMatrix(torch.zeros((2, 64), dtype=torch.uint8), torch.zeros((1, 1, 32, 4, 4), dtype=torch.uint8), 2, 32)
