"""What the header says of the parts of a value in the layer for a few tokens, by their definition (no kernel runs here)."""
import numpy as np
import pytest

from tests import parts_reference as pr

# times that another of the 32 may be as large: {bits: {type: power of two}}
EXACT = {8: {"bf16": 26, "fp16": 23}, 4: {"bf16": 11, "fp16": 8}}
MANTISSA = {"bf16": 7, "fp16": 10}


def _beside(ratio, bits_of_value, seed, rows=16000):
    """Groups of one value in [1, 2) and 31 others, up to `ratio` times smaller, with so many bits behind the point."""
    g = np.random.default_rng(seed)
    small = 2.0 ** -g.integers(0, ratio + 1, (rows, 32))
    v = small * (1 + np.floor(g.random((rows, 32)) * 2.0**bits_of_value) * 2.0**-bits_of_value) * g.choice([-1.0, 1.0], (rows, 32))
    v[:, 7] = 1 + np.floor(g.random(rows) * 2.0**bits_of_value) * 2.0**-bits_of_value
    return v * 2.0 ** g.integers(-20, 20, (rows, 1))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("size", [2, 4])
def test_what_is_left_out_at_most(bits, size):
    parts = pr.PARTS[bits][size]
    for ratio in (2, 10, 20, 30):
        v = _beside(ratio, 23, ratio)
        off = np.abs(pr.split(v, bits, parts) - v)
        assert (off <= pr.bound(v, bits, parts)).all()
        amax = np.abs(v).max(1, keepdims=True)
        stated = np.maximum(2.0**-24 * np.abs(v), 2.0**-36 * amax) if bits == 8 else 2.0 ** (-25 if size == 4 else -19) * amax
        assert (off <= stated).all()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_of_16_bits_are_exact_beside_larger_ones(bits, dtype):
    parts, ratio = pr.PARTS[bits][2], EXACT[bits][dtype]
    v = _beside(ratio, MANTISSA[dtype], 3)
    v = v[np.abs(v).max(1) / np.abs(v).min(1) <= 2.0**ratio]
    assert len(v) > 500 and np.array_equal(pr.split(v, bits, parts), v)
    wider = _beside(ratio + 4, MANTISSA[dtype], 4)
    assert not np.array_equal(pr.split(wider, bits, parts), wider)
