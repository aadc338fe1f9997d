"""A call without the workspace that it needs is refused like one with too little of it."""
import numpy as np
import pytest

import paper_2505_21594_amd as ee
from tests.device import Dev


def test_no_workspace():
    z, rs = Dev(np.zeros((3, 100), np.float32)), Dev(np.array([0, 3], np.int32))
    x, u, one, i = Dev(np.zeros(3, np.int32)), Dev(np.zeros(3, np.float32)), Dev(np.ones(1, np.float32)), Dev(np.zeros(1, np.int32))
    with pytest.raises(ee.EEError) as e:
        ee.ee_accept_drafts(z, rs, x, None, u, u, one, i, i, workspace=None)
    assert e.value.code == ee.EE_EINVAL and "workspace" in str(e.value)
    k, v = Dev(np.zeros((200, 1, 16, 1, 64), np.uint16)), Dev(np.zeros((200, 1, 1, 64, 16), np.uint16))
    cache, q = ee.PagedCache(k, v, Dev(np.zeros((1, 200), np.int32))), Dev(np.zeros((1, 1, 64), np.float32))
    assert ee.ee_attend_workspace(cache, Dev(np.array([0, 1], np.int32)), q) > 0
    with pytest.raises(ee.EEError) as e:
        ee.ee_attend(cache, Dev(np.array([0, 1], np.int32)), i, q, q, scale=1.0)
    assert e.value.code == ee.EE_EINVAL and "workspace" in str(e.value)
