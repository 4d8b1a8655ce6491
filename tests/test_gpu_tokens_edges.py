"""Token writes and reads at the edges: values that leave 32 bits on the way into 4-bit rows, values that are not finite, calls
without tokens."""
import numpy as np
import pytest

from attention_sim import to64
from paper_2608_13263_b200 import binding as vt
from test_gpu_tokens import GEOMETRIES, Writer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exponents", [(-30, -30), (-60, -45), (-28, 0)])
@pytest.mark.parametrize("geometry", [GEOMETRIES[3], GEOMETRIES[6]], ids=["128", "64"])
def test_4_bit_rows_saturate_beyond_32_bits(geometry, exponents):
    """Finite values whose multiple by 2^-exponent is not a 32-bit number are held as the largest, not as NaN."""
    w = Writer(np.random.default_rng(50), geometry, 40, exponents=exponents, scale=3e29, weights=False)
    w.write()
    w.check()
    w.close()
