"""A pass that failed, and the prompt that comes behind it."""
import pytest

import eegen
import paper_2505_21594_amd as ee

pytestmark = pytest.mark.gpu


def tokens(seed, n):
    return list(eegen.prompt_tokens(seed, n, eegen.TINY.vocab, session=0))


def test_continue_says_that_the_last_pass_failed(model_dir):
    """Rows behind a pass that failed would stand where nobody expects them: EE_CONTINUE reports it, a fresh prompt gives it up.  (The failure is the
    result block's word, written by the host.)"""
    p = f"{model_dir}/gpu_tiny_continue.bin"
    eegen.write_model(p, eegen.TINY, 96, gains="uniform")
    m = ee.Model(p)
    s = m.session(200, max_gamma=4)
    try:
        s.ee_prefill(tokens(957, 30))
        s.ee_verify([1, 2, 3, 4], [2])
        ee.ee_device_synchronize(0)
        s._res.contents.device_status = 1
        with pytest.raises(ee.EEError) as e:
            s.ee_prefill([5, 6], flags=ee.CONTINUE)
        assert e.value.code == ee.EE_EDEVICE and s.ee_kv_len() == 30
        s.ee_prefill([5, 6], flags=ee.CONTINUE)                  # (said once)
        assert s.ee_kv_len() == 32
        s.ee_verify([1, 2, 3, 4], [2])
        ee.ee_device_synchronize(0)
        s._res.contents.device_status = 1
        s.ee_prefill(tokens(958, 20))
        assert s.ee_kv_len() == 20
    finally:
        s.free()
        m.free()
