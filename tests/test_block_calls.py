"""Refusals of the Python calls on 8-bit block matrices that come before any tensor is looked at (no GPU)."""
import pytest


@pytest.fixture(scope="module")
def mad():
    pytest.importorskip("torch")
    import paper_2106_10860_amd as m
    return m


def test_a_product_by_depth_needs_offsets(mad):
    """Without them it is the dense product, which by='depth' did not ask for."""
    some = mad.BlockMatrix._made(None, None, 1)
    with pytest.raises(ValueError, match="offsets"):
        mad.maddness_block_product(some, some, by="depth")
