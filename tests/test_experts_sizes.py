"""Sizes near 2^31 of the operators of a layer of experts: what the encoders refuse, since a kernel would count past 32 bits."""
import pytest

from tests.test_experts_host import OK, TOO_LARGE, encode

LAST = 2 ** 31 - 1


@pytest.mark.parametrize("kw,want", [
    (dict(rows=LAST - 255, n=8, out_stride=8), OK), (dict(rows=LAST - 254, n=8, out_stride=8), TOO_LARGE), (dict(rows=LAST, n=8, out_stride=8), TOO_LARGE),
    (dict(n=LAST - 255, out_stride=LAST, w_stride=(1 << 38, 16), k=16, x_stride=16), OK), (dict(n=LAST - 254, out_stride=LAST, w_stride=(1 << 38, 16), k=16, x_stride=16), TOO_LARGE),
    (dict(n=LAST, out_stride=LAST, w_stride=(1 << 38, 16), k=16, x_stride=16), TOO_LARGE)])
def test_scaled_matmul_sizes(kw, want):
    """Numbers of tiles are formed by adding a tile's rows (128) or columns (256) less one."""
    assert encode("scaled_matmul", **kw)[0] == want


@pytest.mark.parametrize("name,kw", [
    ("combine", dict(cols=LAST, y_stride=LAST, out_stride=LAST, base_stride=LAST)), ("combine", dict(rows=LAST)),
    ("quantize", dict(rows=2, cols=LAST - 15, out_rows=6, x_stride=LAST, codes_stride=LAST + 1, scales_stride=1 << 25)),
    ("quantize", dict(rows=LAST, cols=16, x_stride=16, copies=0, out_rows=LAST, codes_stride=16, scales_stride=1))])
def test_sizes_that_are_taken(name, kw):
    assert encode(name, **kw)[0] == OK
