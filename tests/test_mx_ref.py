"""The 64-bit statement of the microscaled format that the GPU tests compare with: hand-worked groups, bounds, and
mistakes that have to show."""
import numpy as np
import pytest

from tests import golden_io
from tests import mx_ref as ref

F32 = np.float32


def bits(values):
    return (np.asarray(values, F32).view(np.uint32) >> 16).astype(np.uint16)


def group(values):
    row = np.zeros(32, F32)
    row[:len(values)] = values
    return bits(row)[None]


def test_ties_go_to_the_even_code():
    # largest magnitude 4: s = 0, so the values are in units of the grid
    x = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -0.25, -0.75, -2.5]
    codes, scales = ref.quantize(group(x))
    assert scales[0, 0] == 127
    assert codes[0, :10].tolist() == [6, 0, 2, 2, 4, 4, 6, 8, 10, 12]
    codes, _ = ref.quantize(group([4.0, 5.0, 7.5]))            # 5 is half way between 4 and 6, 7.5 is cut off
    assert codes[0, :3].tolist() == [6, 6, 7]


def test_the_two_rules():
    for m, floor, cover in [(4.0, 127, 127), (6.0, 127, 127), (6.03125, 127, 128), (7.9375, 127, 128), (8.0, 128, 128)]:
        b = group([m])
        assert ref.quantize(b, ref.FLOOR)[1][0, 0] == floor and ref.quantize(b, ref.COVER)[1][0, 0] == cover, m
    assert ref.quantize(group([7.5]), ref.FLOOR)[0][0, 0] == 7       # 6
    assert ref.quantize(group([7.5]), ref.COVER)[0][0, 0] == 6       # 4, times 2: 7.5 is nearer to 8


def test_smallest_and_non_finite():
    tiny = np.array([[1] + [0] * 31], np.uint16)                # 2^-133
    codes, scales = ref.quantize(tiny)
    assert scales[0, 0] == 0 and codes[0, 0] == 0               # 2^-133 / 2^-127
    codes, scales = ref.quantize(np.array([[64] + [0] * 31], np.uint16))          # 2^-127
    assert scales[0, 0] == 0 and codes[0, 0] == 2
    for v in (0x7F80, 0xFF80, 0x7FC0, 0x7F81):
        b = np.full((1, 40), 0x3F80, np.uint16)
        b[0, 5] = v
        codes, scales = ref.quantize(b)
        assert scales[0].tolist() == [255, 125] and not codes[0, :32].any() and (codes[0, 32:] == 6).all()
        assert np.isnan(ref.values(codes, scales)[0, :32]).all() and (ref.values(codes, scales)[0, 32:] == 1.0).all()


@pytest.mark.parametrize("rule", [ref.FLOOR, ref.COVER])
def test_error_bounds(rule):
    rng = np.random.default_rng(rule)
    b = bits(rng.standard_normal((64, 100)) * np.exp(3 * rng.standard_normal((64, 100))))
    x, v = ref.bf16_values(b), ref.values(*ref.quantize(b, rule))
    s = np.repeat(np.ldexp(1.0, ref.quantize(b, rule)[1].astype(int) - 127), 32, axis=1)[:, :100]
    t = np.abs(x) / s
    half = np.where(t <= 2, 0.25, np.where(t <= 4, 0.5, 1.0))
    inside = t <= 6
    assert (np.abs(x - v)[inside] <= (half * s)[inside]).all()
    assert inside.all() if rule == ref.COVER else (np.abs(v)[~inside] == 6 * s[~inside]).all()


def test_philox_known_answers():
    _, kat = golden_io.load("philox4x32_10_kat.txt")
    for c, k, want in zip(kat["ctr"], kat["key"], kat["out"]):
        got = ref.philox([int(v) for v in c], int(k[0]) | int(k[1]) << 32)
        assert [int(v) for v in got] == [int(v) for v in want]


def test_stochastic_rounding_is_unbiased_and_exact_values_stay():
    b = np.tile(group([4.3125, 3.2, 0.2, 1.1, -2.7, 5.9, 0.013]), (4000, 1))
    r = np.stack([ref.random16(4000, 32, s) for s in (1, 2)])
    v = np.stack([ref.values(*ref.quantize(b, ref.COVER, k)) for k in r]).reshape(-1, 32)
    x = ref.bf16_values(b[:1])[0]
    # 8000 draws of a step of at most 2: a standard error of 1 / sqrt(8000); the cut to 2^-17 is below it
    assert (np.abs(v.mean(axis=0) - x) < 5 / np.sqrt(8000)).all()
    assert not np.array_equal(r[0], r[1])
    on_grid = np.tile(group([6.0, 4.0, -3.0, 2.0, 1.5, 1.0, 0.5]), (50, 1))
    v = ref.values(*ref.quantize(on_grid, ref.COVER, ref.random16(50, 32, 3)))
    assert np.array_equal(v, ref.bf16_values(on_grid))


def test_storage_order_is_a_bijection():
    rng = np.random.default_rng(0)
    for R, C in [(1, 1), (17, 129), (70, 300)]:
        strips, quads, nkb = -(-R // 16), -(-R // 64), -(-C // 128)
        stored = np.arange(strips * nkb * 1024, dtype=np.int64).reshape(strips, nkb, 1024)
        r, c = np.meshgrid(np.arange(strips * 16), np.arange(nkb * 128), indexing="ij")
        byte = stored[r // 16, c // 128, (r % 16 + 16 * (c % 128 // 32)) * 16 + c % 32 // 2]
        assert sorted((byte * 2 + c % 2).ravel().tolist()) == list(range(2 * stored.size))
        sc = rng.integers(0, 256, (quads, nkb, 256)).astype(np.uint8)
        _, full = ref.untile_scales(sc, R, C)
        assert sorted(full.ravel().tolist()) == sorted(sc.ravel().tolist())


def test_planted_mistakes_show():
    """Half-up ties, the other rule's scale, swapped halves of a word: each differs from the definition on inputs like
    the GPU tests'."""
    rng = np.random.default_rng(5)
    b = bits(rng.standard_normal((16, 256)).astype(F32))
    codes, scales = ref.quantize(b)
    x = ref.bf16_values(b)
    t = np.abs(x) / np.repeat(np.ldexp(1.0, scales.astype(int) - 127), 32, axis=1)
    half_up = np.searchsorted((ref.GRID[1:] + ref.GRID[:-1]) / 2, t, side="right")
    assert (half_up != (codes & 7)).any()
    assert (ref.quantize(b, ref.COVER)[1] != scales).any()
    r = ref.random16(16, 256, 9)
    swapped = r.reshape(16, -1, 2)[:, :, ::-1].reshape(16, 256)
    assert (ref.quantize(b, ref.COVER, r)[0] != ref.quantize(b, ref.COVER, swapped)[0]).any()
