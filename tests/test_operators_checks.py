"""Refusals of the operators on device memory (argument checks run before anything touches a GPU), and their reference forms."""
import ctypes

import numpy as np
import pytest

import paper_2505_21594_amd as ee
from paper_2505_21594_amd import binding
from paper_2505_21594_amd.binding import AcceptArgsC, AppendArgsC, AttendArgsC, PagedCacheC
from tests import operators_ref as ref

P = 1 << 20   # an address that nothing reads


def cache(**kw):
    c = PagedCacheC(0, 2, 64, 1, 8, 3, 4, 0, P, P, P)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def append_args(**kw):
    a = AppendArgsC(ee.BF16, ee.FP32, 4, 5, 16, 0, 1e-5, 0, P, P, P, P, P, 2 * P, 512, 64, 512, 64, 512, 64, 256, 64, P, P, P)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def attend_args(**kw):
    a = AttendArgsC(ee.BF16, ee.FP32, 4, 5, 0, 0, 0, 0.125, P, P, 0, 0, P, P, 256, 64, 256, 64)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def accept_args(**kw):
    a = AcceptArgsC(0, ee.FP32, 2, 6, 100, 0, P, P, 100, P, P, 100, P, P, P, P, P)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def refused(rc, word):
    assert rc == ee.EE_EINVAL
    assert word in ee.load_library().ee_last_error().decode()


CACHE = [(dict(device=-1), "device"), (dict(head_dim=96), "head_dim"), (dict(head_dim=0), "head_dim"), (dict(terms=3), "terms"), (dict(n_kv_heads=0), "n_kv_heads"),
         (dict(n_kv_heads=3), "multiple"), (dict(n_pages=0), "n_pages"), (dict(table_stride=0), "table_stride"), (dict(n_seqs=-1), "n_seqs"), (dict(k_pool=0), "null"),
         (dict(v_pool=P + 8), "16-byte"), (dict(page_table=0), "null"), (dict(page_table=P + 2), "4-byte")]


@pytest.mark.parametrize("kw,word", CACHE)
def test_cache_is_checked(kw, word):
    lib = ee.load_library()
    refused(lib.ee_kv_append(ctypes.byref(cache(**kw)), ctypes.byref(append_args()), None), word)
    refused(lib.ee_attend(ctypes.byref(cache(**kw)), ctypes.byref(attend_args()), None, 0, None), word)


@pytest.mark.parametrize("kw,word", [(dict(dtype=3), "type"), (dict(q_out_dtype=-1), "type"), (dict(n_heads=3), "multiple"), (dict(n_rows=-1), "n_rows"),
                                     (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(rope_pairs=2), "rope_pairs"), (dict(rope_len=0), "rope_len"),
                                     (dict(k_stride=508), "alignment"), (dict(q_stride=-512), "alignment"), (dict(q_out_head_stride=2), "alignment"),
                                     (dict(q=0), "null"), (dict(v=0), "null"), (dict(q_out=0), "null"), (dict(q=P + 2), "16-byte"), (dict(rope=P + 4), "16-byte"),
                                     (dict(q_out=P), "same type"), (dict(row_start=0), "null"), (dict(kv_len=P + 1), "4-byte")])
def test_append_is_checked(kw, word):
    refused(ee.load_library().ee_kv_append(ctypes.byref(cache()), ctypes.byref(append_args(**kw)), None), word)


@pytest.mark.parametrize("kw,word", [(dict(dtype=7), "type"), (dict(n_heads=0), "n_heads"), (dict(n_heads=5), "multiple"), (dict(scale=0.0), "scale"),
                                     (dict(scale=float("inf")), "scale"), (dict(scale=float("nan")), "scale"), (dict(n_groups=4), "n_groups"), (dict(n_groups=-1), "n_groups"),
                                     (dict(n_groups=1), "null"), (dict(max_kv=-1), "max_kv"), (dict(q=0), "null"), (dict(out=P + 8), "16-byte"),
                                     (dict(q_stride=250), "alignment"), (dict(n_rows=(1 << 24) + 1), "n_rows")])
def test_attend_is_checked(kw, word):
    refused(ee.load_library().ee_attend(ctypes.byref(cache()), ctypes.byref(attend_args(**kw)), None, 0, None), word)


def test_attend_workspace_is_checked():
    lib = ee.load_library()
    c, a, n = cache(table_stride=4096), attend_args(n_rows=1), ctypes.c_size_t(5)
    assert lib.ee_attend_workspace(ctypes.byref(c), ctypes.byref(a), ctypes.byref(n)) == ee.EE_OK and n.value > 0
    refused(lib.ee_attend(ctypes.byref(c), ctypes.byref(a), P, n.value - 1, None), "workspace")
    refused(lib.ee_attend(ctypes.byref(c), ctypes.byref(a), P + 128, n.value, None), "workspace")
    refused(lib.ee_attend(ctypes.byref(c), ctypes.byref(a), None, n.value, None), "workspace")
    refused(lib.ee_attend_workspace(ctypes.byref(cache(terms=0)), ctypes.byref(a), ctypes.byref(n)), "terms")
    assert lib.ee_attend_workspace(ctypes.byref(c), ctypes.byref(a), None) == ee.EE_EINVAL


@pytest.mark.parametrize("kw,word", [(dict(device=-2), "device"), (dict(dtype=9), "type"), (dict(vocab=0), "vocab"), (dict(n_seqs=-1), "n_seqs"), (dict(n_rows=70000), "n_rows"),
                                     (dict(row_start=0), "null"), (dict(logits=0), "null"), (dict(drafts=0), "null"), (dict(accept_len=0), "null"), (dict(temperature=0), "null"),
                                     (dict(logits_stride=99), "stride"), (dict(probs_stride=50), "stride"), (dict(u=0), "together"), (dict(u=0, v=0), "draft_probs"),
                                     (dict(logits=P + 2), "aligned"), (dict(v=P + 2), "4-byte")])
def test_accept_is_checked(kw, word):
    refused(ee.load_library().ee_accept_drafts(ctypes.byref(accept_args(**kw)), P, 1 << 20, None), word)


def test_accept_workspace_is_checked():
    lib, n = ee.load_library(), ctypes.c_size_t()
    assert lib.ee_accept_workspace(ctypes.byref(accept_args()), ctypes.byref(n)) == ee.EE_OK and n.value > 0
    refused(lib.ee_accept_drafts(ctypes.byref(accept_args()), P, n.value - 1, None), "workspace")
    refused(lib.ee_accept_drafts(ctypes.byref(accept_args()), None, n.value, None), "workspace")


def test_nothing_to_do_is_fine():
    lib = ee.load_library()
    assert lib.ee_kv_append(ctypes.byref(cache(n_seqs=0)), ctypes.byref(append_args()), None) == ee.EE_OK
    assert lib.ee_kv_append(ctypes.byref(cache()), ctypes.byref(append_args(n_rows=0)), None) == ee.EE_OK
    assert lib.ee_attend(ctypes.byref(cache()), ctypes.byref(attend_args(n_rows=0)), None, 0, None) == ee.EE_OK
    assert lib.ee_accept_drafts(ctypes.byref(accept_args(n_seqs=0)), None, 0, None) == ee.EE_OK
    for call in (lambda: lib.ee_kv_append(None, None, None), lambda: lib.ee_attend(None, None, None, 0, None), lambda: lib.ee_accept_drafts(None, None, 0, None)):
        refused(call(), "null")


def test_struct_layouts_match_header():
    assert ctypes.sizeof(PagedCacheC) == 8 * 4 + 3 * 8
    assert ctypes.sizeof(AppendArgsC) == 8 * 4 + 6 * 8 + 8 * 8 + 3 * 8
    assert ctypes.sizeof(AttendArgsC) == 8 * 4 + 6 * 8 + 4 * 8
    assert ctypes.sizeof(AcceptArgsC) == 6 * 4 + 11 * 8
    for fmt, c in ((binding._APPEND_PACK, AppendArgsC), (binding._ATTEND_PACK, AttendArgsC), (binding._ACCEPT_PACK, AcceptArgsC)):
        kinds = [f[1] for f in c._fields_]
        values = [0.5 + i if k is ctypes.c_float else i + 1 for i, k in enumerate(kinds)]
        got = c.from_buffer_copy(fmt(*values))
        assert [getattr(got, f[0]) for f in c._fields_] == values


def test_reference_forms_agree_with_themselves():
    """The attention's reference against a direct softmax over one sequence, and a mistake planted in it."""
    c = ref.Case(1, [2], [20], 1, 64, 2).fill()
    q = np.random.default_rng(0).standard_normal((2, 1, 64))
    out, tol = ref.attend(c, q, 0.125, "fp32", "fp32")
    K, V = c.keys(0)[0][:, 0], c.values(0)[:, 0]
    for i, n in enumerate((19, 20)):
        e = np.exp(K[:n] @ q[i, 0] * 0.125)
        assert np.allclose(out[i, 0], e @ V[:n] / e.sum(), rtol=1e-12)
    c.lens[0] = 19                                     # one position fewer: far outside the tolerance
    assert (np.abs(ref.attend(c, q, 0.125, "fp32", "fp32")[0] - out) > tol).any()


def test_binding_checks_shapes():
    from tests.device import Dev
    k, v = Dev(np.zeros((8, 2, 16, 1, 64), np.uint16)), Dev(np.zeros((8, 2, 1, 64, 16), np.uint16))
    table = Dev(np.zeros((3, 4), np.int32))
    ee.PagedCache(k, v, table)
    for bad in ((v, k, table), (k, Dev(np.zeros((8, 2, 2, 64, 16), np.uint16)), table), (k, v, Dev(np.zeros((3, 4), np.float32))),
                (k, v, table.view((3, 2), (4, 1))), (k.view((8, 2, 16, 1, 32), k.stride()), v, table)):
        with pytest.raises(ValueError):
            ee.PagedCache(*bad)
