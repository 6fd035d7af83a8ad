"""The largest matrices that the conversions take, without a GPU: what is refused for its size and what is not."""
import pytest

import paper_2605_05888_amd as hub
from test_few_refusals import dequantize, quantize


@pytest.mark.parametrize("call", [quantize, dequantize])
@pytest.mark.parametrize("fmt,group", [(hub.Q4_FP4, 32), (hub.Q4_INT4, 32), (hub.Q4_INT4, 64), (hub.Q4_INT4, 128)])
@pytest.mark.parametrize("cols", [64, 192, 4096, (1 << 22) - 64])
def test_rows_times_columns_stay_below_2_to_the_36(call, fmt, group, cols):
    most = ((1 << 36) - 1) // cols
    sizes = dict(fmt=fmt, group=group, cols=cols, w=None)
    assert call(rows=most, **sizes) == -1 and "NULL" in hub.last_error()  # (only the pointer is wrong)
    assert call(rows=most + 1, **sizes) == -1 and "2^36" in hub.last_error()
