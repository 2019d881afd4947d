"""More refusals of the dense operators, on the host: temperatures whose reciprocal is no float32."""
import pytest

import paper_2112_15345_amd as hg
from test_dense_refusals import LIB, distill


@pytest.mark.parametrize("temperature", [2.0 ** -126 * 0.99, 1e-39, 2.0 ** -149])
def test_temperatures_below_the_normal_numbers(temperature):
    assert distill(temperature=temperature) == hg.HG_EUNSUPPORTED
    assert b"temperature" in LIB.hg_last_error()
