"""Limits of the sampling and the norm at the C ABI, without a GPU: the library refuses before it looks at a pointer."""
import pytest

import paper_2401_13660_amd as mb


@pytest.mark.parametrize("temperature,code", [(2.0 ** -127, -5), (4e-39, -5), (3e-39, -5), (1e-45, -5), (2.0 ** -127 * 1.01, 0), (2.0 ** -126, 0), (3.4e38, 0)])
def test_smallest_temperature(temperature, code):
    assert mb.load_library().mb_sample(0, 5, 0, temperature, 0, 1.0, 0.0, *[None] * 9) == code
