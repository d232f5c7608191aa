"""The range of laser_attend's scale, through the C ABI without a device."""
import math

from paper_2606_31580_amd import laser as L
from test_kv_rows_abi import _attend, _kv, _msg, _rows


def test_scales_that_leave_fp32():
    """Scores are kept in units of log 2: a scale whose multiple by log2(e) = 1.44 is infinite would make 0 x inf of a
    product of zero."""
    _, kv = _kv()
    L._call("laser_kv_add_seq", kv, 0, 40)
    q, span = _rows(64, 4), [L.attend_span(0, 4, 10)]
    largest = 2.0 ** 128 * (1 - 2.0 ** -24)
    for scale in (0.7 * largest, -0.7 * largest, largest, math.inf, -math.inf, math.nan):
        assert _attend(kv, span, q, q, scale=scale) == L.ERR_INVALID_ARG and "scale" in _msg()
    for scale in (0.69 * largest, -0.69 * largest, 0.0, 2.0 ** -149):
        assert _attend(kv, span, q, q, scale=scale) == L.ERR_STATE and "finalized" in _msg()
