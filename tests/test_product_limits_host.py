"""Refusals of a product's bound on its waits, on the host."""
import pytest

import paper_2004_14180_b200 as qb
from test_layer_host import PRODUCT, PRODUCT_BASE, SIZE, call, lib  # noqa: F401


@pytest.mark.parametrize("kw,code", [(dict(wait_polls=-1), SIZE), (dict(test_missing_blocks=-1), SIZE), (dict(test_missing_blocks=256), SIZE),
                                     (dict(wait_polls=1 << 20, test_missing_blocks=255), 0)])
def test_bounds_of_waits(lib, kw, code):  # noqa: F811
    assert call(lib.qadam_row_product, PRODUCT, PRODUCT_BASE, **kw) == code
    assert qb.ST_TIMEOUT
