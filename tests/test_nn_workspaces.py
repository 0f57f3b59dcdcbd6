"""Workspaces that are large enough but not where they have to be, without a GPU."""
import ctypes

import pytest

from paper_2010_13972_amd import gts, nn

P = 1 << 20    # an address that is never read


@pytest.mark.parametrize("dtype,size", [(0, 4), (2, 2), (3, 2)])
@pytest.mark.parametrize("act", [0, 3])
def test_a_misaligned_workspace_is_invalid(dtype, size, act):
    """Of exactly the size the query gives, for whatever extents: the status is that of a bad
    address, not of a size."""
    for rows in (1, 40, 700, 5000):
        for inputs in (8, 512, 1030):
            for outputs in (16, 520, 1001):
                n = ctypes.c_int64(0)
                for aligned in (0, 1):
                    assert nn._L().gts_linear_backward_workspace_bytes(rows, inputs, outputs, dtype, aligned,
                                                                       n) == gts.GTS_OK
                    ld = {w: -(-w // 8) * 8 for w in (inputs, outputs)}
                    a = nn._LinearGrad(rows=rows, inputs=inputs, outputs=outputs, dtype=dtype, act=act, dy=P,
                                       ld_dy=ld[outputs], pre=P, ld_pre=ld[outputs], x=P, ld_x=ld[inputs], w=P,
                                       ld_w=ld[inputs], dx=P, ld_dx=ld[inputs], dw=P, ld_dw=ld[inputs], db=P)
                    status = nn._L().gts_linear_backward(a, P + 8, n, None)
                    assert status == gts.GTS_EINVAL, (rows, inputs, outputs, aligned, gts.last_error())
                    status = nn._L().gts_linear_backward(a, P, 16, None)
                    assert status == gts.GTS_EBUFSIZE, (rows, inputs, outputs, aligned)
