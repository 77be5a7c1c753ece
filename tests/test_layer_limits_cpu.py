"""CPU checks of the selective state-space layer's calls: sizes that the outputs' types could not hold."""
import pytest


@pytest.fixture(scope="module")
def qlib():
    from paper_1607_04683_gb300 import build, qnn
    build.build()
    return qnn.lib()


@pytest.mark.parametrize("cols,sums,status", [(8421504, 16, 0), (8421505, 16, 1), (8421505, None, 0), (1 << 24, None, 0),
                                              ((1 << 24) + 1, None, 1)])
def test_norm_refuses_sums_past_32_bits(qlib, cols, sums, status):
    assert (2 ** 31 - 1) // 255 == 8421504
    assert qlib.qnn_rmsnorm_quantize(16, cols, None, 0, 0, 16, 1e-5, 0, cols, None, 0, 16, cols, 16, sums, None, 0,
                                     None) == status
