"""Strides of dimensions of one: they say nothing, whatever they are."""
import ctypes

import numpy as np
import pytest

import paper_2505_21594_amd as ee
from tests import operators_ref as ref
from tests.device import Dev, bf16_values, decode, encode
from tests.test_operators_checks import append_args, attend_args, cache, refused


def test_strides_of_one_row_or_head_are_not_checked():
    """(Each call is refused in the end, for a null array: it would have none of these addresses read.)"""
    lib = ee.load_library()
    one = dict(n_rows=1, q_stride=1, k_stride=-3, v_stride=7, q_out_stride=2)
    refused(lib.ee_kv_append(ctypes.byref(cache()), ctypes.byref(append_args(k=0, **one)), None), "null")
    refused(lib.ee_attend(ctypes.byref(cache()), ctypes.byref(attend_args(n_rows=1, q_stride=1, out_stride=-5, q=0)), None, 0, None), "null")
    head = dict(n_heads=1, q_head_stride=1, k_head_stride=3, v_head_stride=-1, q_out_head_stride=5)
    refused(lib.ee_kv_append(ctypes.byref(cache(n_kv_heads=1)), ctypes.byref(append_args(k=0, **head)), None), "null")
    refused(lib.ee_attend(ctypes.byref(cache(n_kv_heads=1)), ctypes.byref(attend_args(n_heads=1, q_head_stride=3, out_head_stride=1, q=0)), None, 0, None), "null")
    for kw in (dict(n_rows=2, k_stride=1), dict(n_heads=2, q_head_stride=1), dict(k_head_stride=4)):
        refused(lib.ee_kv_append(ctypes.byref(cache()), ctypes.byref(append_args(k=0, **kw)), None), "alignment")


def test_contiguous_pools_whatever_the_strides_of_ones():
    k, v, table = np.zeros((1, 1, 16, 1, 64), np.uint16), np.zeros((1, 1, 1, 64, 16), np.uint16), np.zeros((3, 1), np.int32)
    k, v, table = Dev(k).view(k.shape, (5, 1, 64, 3, 1)), Dev(v).view(v.shape, (1, 7, 9, 16, 1)), Dev(table).view((3, 1), (1, 8))
    ee.PagedCache(k, v, table)
    for bad in ((k.view((1, 1, 16, 1, 64), (1, 1, 128, 1, 1)), v, table), (k, v.view((1, 1, 1, 64, 16), (1, 1, 1, 1, 64)), table), (k, v, table.view((3, 1), (2, 1)))):
        with pytest.raises(ValueError):
            ee.PagedCache(*bad)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,heads,kv_heads", [(1, 4, 2), (3, 1, 1), (1, 1, 1)])
def test_odd_strides_of_ones(rows, heads, kv_heads):
    c = ref.Case(840, [rows], [40], kv_heads, 64, 1).fill()
    x = c.rng.standard_normal((rows, heads + 2 * kv_heads, 64)).astype(np.float32)
    parts = [np.ascontiguousarray(x[:, a:b]) for a, b in ((0, heads), (heads, heads + kv_heads), (heads + kv_heads, heads + 2 * kv_heads))]

    def odd(a):
        return Dev(a).view(a.shape, (3 if a.shape[0] == 1 else a.shape[1] * 64, 5 if a.shape[1] == 1 else 64, 1))

    q, k, v = (odd(a) for a in parts)
    pools = Dev(c.k_pool), Dev(c.v_pool)
    pool = ee.PagedCache(*pools, Dev(c.table))
    rs, kl, q_out = Dev(c.row_start), Dev(c.kv_len), Dev(np.zeros_like(parts[0]))
    ee.ee_kv_append(pool, rs, kl, q, k, v, q_out.view(q_out.shape, odd(parts[0]).stride()))
    assert (q_out.numpy() == parts[0]).all()
    c.k_pool, c.v_pool = pools[0].numpy(), pools[1].numpy()
    assert (bf16_values(c.k_pool[c.table[0, 39 // 16], :, 39 % 16, 0]) == decode(encode(bf16_values(encode(parts[1][-1], "bf16")), "fp32"))).all()
    out = Dev(np.zeros_like(parts[0]))
    ws = Dev(np.zeros(max(ee.ee_attend_workspace(pool, rs, q, max_kv=40), 1), np.uint8))
    ee.ee_attend(pool, rs, kl, q, out.view(out.shape, odd(parts[0]).stride()), scale=0.125, max_kv=40, workspace=ws)
    want, tol = ref.attend(c, parts[0].astype(np.float64), 0.125, "fp32", "fp32")
    assert (np.abs(out.numpy() - want) <= tol).all()
