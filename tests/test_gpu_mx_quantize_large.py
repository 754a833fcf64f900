"""The quantizer on either side of 128 tiles of 128 x 128, up to which two workgroups take a tile, one for the rows' side and
one for the columns', and beyond which one takes both: every code and scale equal to the definition's in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_08040_amd as fq
from tests import gpu_util as gu
from tests import mx_ref as ref
from tests.test_gpu_mx_quantize import check_side, make

# tiles: 128 (the most with two workgroups each), 136, 192, 129, 129, 143
SHAPES = [(2048, 1024), (2049, 1021), (1930, 1501), (16390, 70), (45, 16500), (1281, 1537)]


def quantized(call, rows, cols, sides):
    q = fq.MxTensor(rows, cols, sides)
    q.storage.fill_(0xA5)
    call(q)
    torch.cuda.synchronize()
    return q


def check(bits, call, rule, random):
    rows, cols = bits.shape
    both = quantized(call, rows, cols, fq.FQ_MX_BOTH)
    check_side(both, bits, False, rule, random)
    check_side(both, bits, True, rule, random)
    one, other = quantized(call, rows, cols, fq.FQ_MX_ROWS), quantized(call, rows, cols, fq.FQ_MX_COLS)
    for q, t in ((one, ""), (other, "_t")):
        for f in ("codes", "scales"):
            assert torch.equal(q.view(f + t), both.view(f + t)), f + t


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("rule", [fq.FQ_MX_FLOOR, fq.FQ_MX_COVER])
def test_nearest(rows, cols, rule):
    bits = make(rows, cols, rows + cols)
    bits[rows // 2, cols // 2], bits[rows - 1, 0], bits[0, cols - 1] = 0x7F80, 0xFFC0, 0x7F81
    x = gu.to_device_bf16(bits)
    gu.announce(f"mx quantize {rows}x{cols} rule {rule}")
    check(bits, lambda q: fq.fq_mx_quantize(x, out=q, rule=rule), rule, None)


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_stochastic(rows, cols):
    bits = make(rows, cols, 5 * rows + cols)
    x = gu.to_device_bf16(bits)
    gu.announce(f"mx quantize_sr {rows}x{cols}")
    check(bits, lambda q: fq.fq_mx_quantize_sr(x, 2 ** 63 + 11, out=q), ref.COVER, ref.random16(rows, cols, 2 ** 63 + 11))


@pytest.mark.parametrize("rows,cols", [(130, 300), (1930, 1501)])
def test_a_slice_of_a_larger_matrix(rows, cols):
    """An odd pitch and a base off 16 bytes, on either side of 128 tiles."""
    bits = make(rows, cols, rows)
    wide = torch.full((rows, cols + 14), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 3:3 + cols] = gu.to_device_bf16(bits)
    gu.announce(f"mx quantize a slice {rows}x{cols}")
    check(bits, lambda q: fq.fq_mx_quantize(wide[:, 3:3 + cols], out=q), ref.FLOOR, None)


@pytest.mark.parametrize("rows,cols", [(70, 90), (1930, 1501)])
def test_zeros_keep_their_signs(rows, cols):
    """A group whose largest magnitude is 0 has scale byte 0 and codes 0 with the elements' signs."""
    bits = make(rows, cols, 3)
    bits[:] = (bits & 0x8000)
    bits[::3] = 0x8000
    x = gu.to_device_bf16(bits)
    q = fq.fq_mx_quantize(x, sides=fq.FQ_MX_BOTH)
    check_side(q, bits, False, ref.FLOOR)
    check_side(q, bits, True, ref.FLOOR)
    assert not q.view("scales").any() and not q.view("scales_t").any()
    back = fq.fq_mx_dequantize(q)
    assert not back.any() and torch.equal(back.signbit(), x.signbit())
