"""Microscaled quantization and the way back on the GPU: every code and scale equal to the definition's in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2503_08040_amd as fq
from tests import gpu_util as gu
from tests import mx_ref as ref

SIDES = {"rows": fq.FQ_MX_ROWS, "columns": fq.FQ_MX_COLS, "both": fq.FQ_MX_BOTH}


def make(rows, cols, seed):
    """bf16 bits over many magnitudes, zeros, values between the codes, group maxima on either side of 1.5 2^E."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-20, 20, (rows, 1))) * np.exp(rng.standard_normal((rows, cols)))
    x[rng.random((rows, cols)) < 0.05] = 0.0
    x[rng.random((rows, cols)) < 0.01] = -0.0
    ties = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, -2.5], (rows, cols))
    take = rng.random((rows, 1)) < 0.3
    x = np.where(take, ties, x).astype(np.float32)
    x[rng.random(rows) < 0.05] = 0.0
    return (x.view(np.uint32) >> 16).astype(np.uint16)


def check_side(q, bits, columns, rule, random=None):
    b = bits.T if columns else bits
    u = None if random is None else (random.T if columns else random)
    codes, scales = ref.quantize(b, rule, u)
    t = "_t" if columns else ""
    got, full = ref.untile_codes(q.view("codes" + t).cpu().numpy(), *b.shape)
    assert np.array_equal(got, codes)
    full[:b.shape[0], :b.shape[1]] = 0
    assert not full.any()
    got, full = ref.untile_scales(q.view("scales" + t).cpu().numpy(), *b.shape)
    assert np.array_equal(got, scales)
    full[:got.shape[0], :got.shape[1]] = 0
    assert not full.any()
    return ref.values(codes, scales).T if columns else ref.values(codes, scales)


SHAPES = [(1, 1), (1, 4096), (2, 31), (31, 2), (33, 97), (64, 128), (129, 257), (200, 392), (513, 1), (384, 640)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("sides", SIDES)
def test_nearest(rows, cols, sides):
    bits = make(rows, cols, rows + cols)
    x = gu.to_device_bf16(bits)
    for rule in (fq.FQ_MX_FLOOR, fq.FQ_MX_COVER):
        gu.announce(f"mx quantize {rows}x{cols} {sides} rule {rule}")
        q = fq.MxTensor(rows, cols, SIDES[sides])
        q.storage.fill_(0xA5)
        fq.fq_mx_quantize(x, out=q, rule=rule)
        torch.cuda.synchronize()
        for side in (fq.FQ_MX_ROWS, fq.FQ_MX_COLS):
            if SIDES[sides] & side:
                want = check_side(q, bits, side == fq.FQ_MX_COLS, rule)
                for dt in (torch.bfloat16, torch.float32):
                    got = fq.fq_mx_dequantize(q, side, out_dtype=dt)
                    assert got.dtype == dt and np.array_equal(got.double().cpu().numpy(), want)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 515), (65, 33), (96, 128), (131, 300)])
@pytest.mark.parametrize("seed", [0, 2 ** 64 - 1, 0x123456789ABCDEF])
def test_stochastic(rows, cols, seed):
    bits = make(rows, cols, 7 * rows + cols)
    gu.announce(f"mx quantize_sr {rows}x{cols} seed {seed}")
    random = ref.random16(rows, cols, seed)
    one = {}
    for sides in SIDES:
        q = one[sides] = fq.fq_mx_quantize_sr(gu.to_device_bf16(bits), seed, sides=SIDES[sides])
        torch.cuda.synchronize()
        for columns in (False, True):
            if SIDES[sides] & (2 if columns else 1):
                check_side(q, bits, columns, ref.COVER, random)
    assert torch.equal(one["rows"].view("codes"), one["both"].view("codes"))
    assert torch.equal(one["columns"].view("codes_t"), one["both"].view("codes_t"))


@pytest.mark.parametrize("sr", [False, True])
def test_every_bf16_value(sr):
    """All 65536 bit patterns, 32 in a row each with a leader that sets the scale: infinities and NaNs leave their group
    NaN and the neighbouring groups alone; subnormal groups have the smallest scale."""
    bits = np.arange(65536, dtype=np.uint16).reshape(-1, 64)
    bits = np.concatenate([bits, bits[::-1], np.roll(bits, 5, axis=1)])
    rng = np.random.default_rng(1)
    shuffled = rng.permutation(np.arange(65536, dtype=np.uint16)).reshape(-1, 64)
    finite = shuffled[:, :32].copy()
    finite[(finite & 0x7F80) == 0x7F80] = 0x0001
    tiny = rng.integers(0, 0x0300, (64, 64)).astype(np.uint16) | (rng.integers(0, 2, (64, 64)) << 15).astype(np.uint16)
    for b in (bits, shuffled, finite, tiny):
        gu.announce(f"mx every value {b.shape} sr {sr}")
        x = gu.to_device_bf16(b)
        if sr:
            q, random = fq.fq_mx_quantize_sr(x, 3, sides=fq.FQ_MX_BOTH), ref.random16(*b.shape, 3)
        else:
            q, random = fq.fq_mx_quantize(x, sides=fq.FQ_MX_BOTH), None
        torch.cuda.synchronize()
        for columns in (False, True):
            want = check_side(q, b, columns, ref.COVER if sr else ref.FLOOR, random)
            side = fq.FQ_MX_COLS if columns else fq.FQ_MX_ROWS
            for dt in (torch.bfloat16, torch.float32):
                got = fq.fq_mx_dequantize(q, side, out_dtype=dt).double().cpu().numpy()
                over = np.abs(want) >= 2.0 ** 128
                assert np.array_equal(got, np.where(over, np.copysign(np.inf, want), want), equal_nan=True)


def test_strides_and_alignment():
    """A slice of a larger matrix, odd pitches, bases off 16 bytes; the neighbours of a strided output stay."""
    rows, cols = 70, 203
    bits = make(rows, cols, 11)
    want = fq.fq_mx_quantize(gu.to_device_bf16(bits), sides=fq.FQ_MX_BOTH)
    deq = fq.fq_mx_dequantize(want)
    for pad, off in [(0, 1), (5, 0), (5, 8), (21, 3)]:
        wide = torch.full((rows, cols + pad + off), 3.0, dtype=torch.bfloat16, device="cuda")
        wide[:, off:off + cols] = gu.to_device_bf16(bits)
        gu.announce(f"mx strides pad {pad} offset {off}")
        q = fq.fq_mx_quantize(wide[:, off:off + cols], sides=fq.FQ_MX_BOTH)
        for f in ("codes", "scales", "codes_t", "scales_t"):
            assert torch.equal(q.view(f), want.view(f)), (pad, off, f)
        for dt in (torch.bfloat16, torch.float32):
            for side in (fq.FQ_MX_ROWS, fq.FQ_MX_COLS):
                out = torch.full((rows, cols + pad + off), 7.0, dtype=dt, device="cuda")
                fq.fq_mx_dequantize(q, side, out=out[:, off:off + cols])
                ref_ = fq.fq_mx_dequantize(want, side, out_dtype=dt)
                assert torch.equal(out[:, off:off + cols], ref_)
                assert (out[:, :off] == 7.0).all() and (out[:, off + cols:] == 7.0).all()
    assert torch.equal(fq.fq_mx_dequantize(want, out=torch.empty_like(deq)), deq)


def test_columns_side_is_the_rows_side_of_the_transpose():
    bits = make(300, 517, 2)
    x = gu.to_device_bf16(bits)
    c = fq.fq_mx_quantize(x, sides=fq.FQ_MX_COLS)
    r = fq.fq_mx_quantize(x.T.contiguous())
    assert torch.equal(c.view("codes_t"), r.view("codes")) and torch.equal(c.view("scales_t"), r.view("scales"))


def test_empty():
    for rows, cols in [(0, 40), (40, 0), (0, 0)]:
        q = fq.fq_mx_quantize(torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda"), sides=fq.FQ_MX_BOTH)
        assert fq.fq_mx_dequantize(q).shape == (rows, cols)
    torch.cuda.synchronize()
