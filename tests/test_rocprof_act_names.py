"""rocprof_summary names the matrix products with an activation as plans do."""
import pytest

from paper_2006_10226_amd.rocprof_summary import group_of


@pytest.mark.parametrize("symbol,group", [
    ("void qnn::conv_flow_kernel<256, 256, 2, 4, 4, 1, false, false, true, true, true>(qnn::ConvArgs)",
     "conv_dma_flow tile=256x256x64 threads=512 stages=4 +act +add"),
    ("void qnn::conv_flow_kernel<64, 128, 2, 2, 1, 1, true, false, false, false, true>(qnn::ConvArgs)",
     "conv_dma_flow tile=64x128x64 threads=256 stages=1s +act"),
    ("void qnn::conv_flow_kernel<64, 128, 2, 2, 1, 1, true, false, false, true, false>(qnn::ConvArgs)",
     "conv_dma_flow tile=64x128x64 threads=256 stages=1s +add"),
    ("void qnn::conv_small_kernel<1, 2, false, true, false, true>(qnn::ConvArgs)",
     "conv_dma_small tile=16x32x64 threads=512 stages=1 +act"),
])
def test_names(symbol, group):
    assert group_of(symbol) == group
