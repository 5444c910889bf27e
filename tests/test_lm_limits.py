"""Sizes at the ends of what the calls of the language-model layer take (CPU)."""
import pytest

SHAPE = -2


@pytest.fixture(scope="module")
def L():
    from test_abi import _lib_path
    _lib_path()
    import paper_1805_11046_amd as m
    return m.binding._lib


@pytest.mark.parametrize("R,C", [((1 << 28) - 1, 1), ((1 << 28) - 15, 60)])
def test_row_copies_of_more_blocks_than_a_launch_holds_are_refused(L, R, C):
    # 16 threads a block in workgroups of 256: 2^32 threads from 2^28 - 15 blocks on
    blocks = R * -(-C // 128)
    assert (1 << 28) - 16 < blocks < 1 << 28 and R * C <= 1 << 34
    assert L.q8t_fp8_quantize(16, 0, R, C, 0, 0, 0, 0, None, 16, 16, None, None, None) == SHAPE
