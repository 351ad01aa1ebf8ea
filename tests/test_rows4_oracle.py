"""What the oracle of rows in 4 bits makes of values that are held already."""
import numpy as np

from oracle import rows_oracle as ro
from oracle.compactor_oracle import bf16_bits_to_f64


def parameters(rows):
    p = bf16_bits_to_f64(np.ascontiguousarray(rows[..., 64:]).view(np.uint16)).reshape(rows.shape[:-1] + (4, 2))
    return p[..., 0], p[..., 1]


def test_holding_what_is_held():
    """The least value stays to the bit (its code is 0, and no other value is rounded past it).  The step does not grow where the greatest value, lo +
    s c with c <= 15, is a bf16; where it had to be rounded, by 2^-9 of at most the group's range, by no more than one unit of its four bits."""
    rng = np.random.default_rng(0)
    x = ro.f64_to_bf16_bits(rng.standard_normal((3000, 128)) * np.exp(rng.standard_normal((3000, 1)) * 3))
    held = ro.hold4(x)
    v = ro.values4(held)
    again = ro.hold4(ro.f64_to_bf16_bits(v))
    (s, lo), (s2, lo2) = parameters(held), parameters(again)
    np.testing.assert_array_equal(lo2, lo)
    greatest = v.reshape(3000, 4, 32).max(-1)
    rounded = bf16_bits_to_f64(ro.f64_to_bf16_bits(greatest)) != greatest
    assert rounded.any() and not rounded.all()
    assert np.all(np.abs(greatest) <= 15 * s) and np.all(s2 <= np.where(rounded, 1.125, 1.0) * s)
    # whole numbers from one step up are held as they are, over and over
    y = np.tile(np.arange(16.0), (5, 8)) * 2.0 ** np.arange(-2, 3)[:, None] - 6
    held = ro.hold4(ro.f64_to_bf16_bits(y))
    np.testing.assert_array_equal(ro.values4(held), y)
    np.testing.assert_array_equal(ro.hold4(ro.f64_to_bf16_bits(ro.values4(held))), held)
