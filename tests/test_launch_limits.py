"""Batches whose attention would take a launch of 2^32 threads or more are refused by the plan, before anything is stored."""
import ctypes

import numpy as np
import pytest

from paper_2601_12784_amd import binding as B

MOST = (2 ** 32 - 1) // 768   # workgroups of 768 threads


@pytest.mark.parametrize("hkv", [1, 4])
def test_extend_plans_stop_at_the_largest_launch(hkv):
    n = MOST // hkv
    for count, ok in ((n, True), (n + 1, False)):
        one = np.ones(count, np.int32)
        desc = B.make_desc(count, hkv, hkv, 64, 1, count, 0.1)
        info = B.sf_extend_info()
        want = 0 if ok else B.UNSUPPORTED
        assert B.lib().sf_extend_attn_plan(ctypes.byref(desc), one.ctypes.data, one.ctypes.data, None, 0, ctypes.byref(info)) == want
        counts = np.zeros(5, np.int32)
        st = B.lib().sf_debug_extend_plan(ctypes.byref(desc), one.ctypes.data, one.ctypes.data, 256, 1, None, 0, counts.ctypes.data)
        assert st == (B.CAPACITY if ok else B.UNSUPPORTED)
        if ok:   # what the store launch of such a plan counts to fits 32 bits
            assert info.num_items == counts[1] == count * hkv and int(counts[3]) * 256 < 2 ** 31
