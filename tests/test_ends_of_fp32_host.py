"""Numbers of a configuration at the ends of fp32 that the kernels' arithmetic does not hold are refused when the handle is made."""
import ctypes as C

import pytest

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200 import build as ffbuild


@pytest.fixture(scope="module", autouse=True)
def _built():
    ffbuild.build()


@pytest.mark.parametrize("status,eps", [(0, 2.0 ** -126), (1, 2.0 ** -127), (1, 1e-44), (0, 2.9e38)])
def test_layer_norm_eps(status, eps):
    """Below 2^-126 eps itself, and the squares that it is added to, have lost digits: 1e-44 is 2 % off."""
    lib, c, h = B.library(), B.ff_layer_norm_config_t(64, 0, 0, eps), C.c_void_p()
    assert lib.ff_layer_norm_create(C.byref(c), C.byref(h)) == status and bool(h) == (status == 0)
    lib.ff_layer_norm_destroy(h)


@pytest.mark.parametrize("status,scale", [(0, 2.0 ** -126), (0, 2e38), (1, 2.4e38), (1, 2.99e38)])
def test_cross_attention_scale(status, scale):
    """Times log2(e), as the kernels count, the scale has to be finite: else scores of zero are no numbers."""
    lib, c = B.library(), B.ff_cross_attention_config_t(64, 8, 8, scale)
    assert lib.ff_cross_attention_validate(C.byref(c)) == status
