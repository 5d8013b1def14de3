"""Limits of the few-bit calls that the host checks by itself (CPU; nothing is launched)."""
import numpy as np
import pytest

import paper_2402_10876_amd as tw

P = 0x10000        # never dereferenced


def _status(f, *a):
    with pytest.raises(tw.TwError) as e:
        f(*a)
    return e.value.status


@pytest.mark.parametrize("M", [(1 << 27) + 1, 1 << 28, (1 << 31) - 16])
def test_scaled_int8_product_of_more_than_the_most_tokens(M):
    """M <= 2^27 holds for every few-bit call; 2^27 itself goes on to the next check (the weight is not uploaded)."""
    w = tw.tw_pack_i8_host(np.ones((1, 70), np.int8), np.ones((1, 70), np.uint8), 64)
    ld = -(-M // 16) * 16
    assert _status(tw.tw_gemm_i8_scaled, P, M, ld, w, P, P, 2 * P, ld) == 3
    assert _status(tw.tw_gemm_i8_scaled, P, 1 << 27, 1 << 27, w, P, P, 2 * P, 1 << 27) == 6
    w.free()
