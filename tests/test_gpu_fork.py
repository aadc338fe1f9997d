"""Sessions forked from one prefix: the copies are exact, and a batch that reads common pages once matches the oracle."""
import dataclasses

import numpy as np
import pytest

import eegen
import paper_2505_21594_amd as ee
from oracle import oracle as eo
from tests.parity import check_pass, gpu_logits, oracle_greedy, oracle_prefill

pytestmark = pytest.mark.gpu

EXITS = [2]


@pytest.fixture(scope="module", params=[64, 128])
def tiny(model_dir, request):
    hd = request.param
    p = f"{model_dir}/gpu_tiny_fork_{hd}.bin"
    eegen.write_model(p, dataclasses.replace(eegen.TINY, n_heads=eegen.TINY.d_model // hd, head_dim=hd), 91, gains="uniform")
    g = ee.Model(p, max_rows=48)
    yield g, eo.Model(p)
    g.free()


def tokens(o, seed, n, session=0):
    return list(eegen.prompt_tokens(seed, n, o.vocab, session=session))


@pytest.mark.parametrize("scatter", [False, True])
@pytest.mark.parametrize("n,more", [(64, 1), (37, 20), (200, 70), (16, 3)])
def test_fork_and_continue_equal_a_prefill(tiny, n, more, scatter):
    """prefix, fork, rest of the prompt: the same tokens as a prompt in one piece, and the oracle's logits."""
    g, o = tiny
    prompt = tokens(o, 900, n + more)
    a, b, whole, os_ = g.session(400), g.session(400, flags=ee.KEEP_LOGITS), g.session(400), o.session(400)
    try:
        if scatter:
            a.ee_session_option(ee.OPT_SCATTER_PAGES, 1)
            b.ee_session_option(ee.OPT_SCATTER_PAGES, 1)
        a.ee_prefill(prompt[:n] + tokens(o, 901, 9))             # (positions behind the fork are others)
        a.ee_session_fork(n, b)
        assert b.ee_kv_len() == n
        with pytest.raises(ee.EEError):
            b.ee_pending()
        with pytest.raises(ee.EEError):
            b.ee_verify([1, 2])
        first = b.ee_prefill(prompt[n:], flags=ee.CONTINUE)
        fo, margin = oracle_prefill(os_, prompt)
        if margin >= 1e-2:
            assert first == fo == whole.ee_prefill(prompt)
        b.ee_set_pending(fo)
        assert b.ee_kv_len() == n + more
        d = oracle_greedy(os_, 4)
        ro = os_.verify(d, EXITS, want_logits=True)
        b.ee_verify(d, EXITS)
        b.ee_wait_final()
        check_pass(ro, b.final_result(), gpu_logits(b, 1), d, "after fork")
        assert a.ee_kv_len() == n + 9                            # the source is as it was
    finally:
        for s in (a, b, whole):
            s.free()


def test_continue_behind_embeddings_and_held_token(tiny):
    g, o = tiny
    emb = eegen.embedding_prefix(902, 30, o.d_model, session=0)
    t = tokens(o, 903, 40)
    s, os_ = g.session(200, flags=ee.KEEP_LOGITS), o.session(200)
    try:
        s.ee_prefill(t[:5], emb=emb)
        s.ee_prefill(t[5:], flags=ee.CONTINUE | ee.HOLD_LAST)
        assert s.ee_kv_len() == 30 + 39 and s.ee_pending() == t[-1]
        s.ee_prefill([7], flags=ee.CONTINUE | ee.HOLD_LAST)      # nothing to cache: only another pending token
        assert s.ee_kv_len() == 69 and s.ee_pending() == 7
        s.ee_set_pending(t[-1])
        os_.prefill(t, flags=eo.HOLD_LAST, emb=emb)
        ro = os_.verify([1, 2, 3], EXITS, want_logits=True)
        s.ee_verify([1, 2, 3], EXITS)
        s.ee_wait_final()
        check_pass(ro, s.final_result(), gpu_logits(s, 1), [1, 2, 3], "continue")
    finally:
        s.free()


# prefixes: (parent session or -1, positions taken from it, own tokens behind them) per session
FAMILIES = {
    "one image": [(-1, 0, 70), (0, 70, 5), (0, 70, 9), (0, 70, 1)],
    "two prompts and a stranger": [(-1, 0, 100), (0, 96, 20), (-1, 0, 50), (2, 50, 3), (2, 33, 40), (-1, 0, 12)],
    "a fork of a fork": [(-1, 0, 64), (0, 64, 30), (1, 90, 5), (1, 80, 2), (0, 40, 7)],
    "less than a page": [(-1, 0, 15), (0, 15, 4), (0, 10, 6)],
    "long": [(-1, 0, 600), (0, 600, 150), (0, 590, 20)],
}


@pytest.mark.parametrize("option", [0, 1, 2])
@pytest.mark.parametrize("name", FAMILIES)
def test_batch_of_forks(tiny, name, option):
    """Three committed rounds, every session's logits against the oracle; the sources' caches grow beside their forks'."""
    g, o = tiny
    family, gamma = FAMILIES[name], 4
    sess, osess, prompts = [], [], []
    try:
        for b, (parent, n, own) in enumerate(family):
            gs, os_ = g.session(900, max_gamma=gamma, flags=ee.KEEP_LOGITS), o.session(900)
            mine = tokens(o, 910, own, session=b)
            prompts.append((prompts[parent][:n] if parent >= 0 else []) + mine)
            if parent >= 0:
                sess[parent].ee_session_fork(n, gs)
                gs.ee_prefill(mine, flags=ee.CONTINUE)
            else:
                gs.ee_prefill(mine)
            fo, _ = oracle_prefill(os_, prompts[-1])
            gs.ee_set_pending(fo)
            sess.append(gs)
            osess.append(os_)
        sess[0].ee_session_option(ee.OPT_SHARED_ATT, option)
        for rnd in range(3):
            drafts = [eegen.corrupt_drafts(np.array(oracle_greedy(osess[b], gamma), dtype=np.int32), 0.3, o.vocab, 911, rnd, session=b) for b in range(len(sess))]
            ee.ee_verify_batch(sess, drafts, EXITS)
            for b, s in enumerate(sess):
                s.ee_wait_final()
                ro = osess[b].verify(drafts[b], EXITS, want_logits=True)
                rg = s.final_result()
                exempt, err = check_pass(ro, rg, gpu_logits(s, 1), drafts[b], f"{name} round {rnd} session {b}")
                assert err < 5e-4
                if exempt and (rg.accept_len != ro.accept_len or rg.next_token != ro.next_token):
                    s.ee_kv_truncate(osess[b].kv_len)
                    s.ee_set_pending(osess[b].pending)
                assert s.ee_kv_len() == osess[b].kv_len and s.ee_pending() == osess[b].pending
    finally:
        for s in sess:
            s.free()


def test_what_was_cut_off_is_not_shared(tiny):
    """Truncated below the fork and filled with other tokens, two sessions have only what both still hold."""
    g, o = tiny
    base = tokens(o, 920, 80)
    tails = [tokens(o, 921, 45, session=b) for b in range(2)]
    sess = [g.session(300, max_gamma=4, flags=ee.KEEP_LOGITS) for _ in range(2)]
    osess = [o.session(300) for _ in range(2)]
    try:
        sess[0].ee_prefill(base)
        sess[0].ee_session_fork(80, sess[1])
        for b in range(2):
            sess[b].ee_kv_truncate(40)
            sess[b].ee_prefill(tails[b], flags=ee.CONTINUE)
            fo, _ = oracle_prefill(osess[b], base[:40] + tails[b])
            sess[b].ee_set_pending(fo)
        sess[0].ee_session_option(ee.OPT_SHARED_ATT, 2)
        drafts = [oracle_greedy(osess[b], 4) for b in range(2)]
        ee.ee_verify_batch(sess, drafts, EXITS)
        for b in range(2):
            sess[b].ee_wait_final()
            check_pass(osess[b].verify(drafts[b], EXITS, want_logits=True), sess[b].final_result(), gpu_logits(sess[b], 1), drafts[b], f"session {b}")
    finally:
        for s in sess:
            s.free()


def test_more_forks_than_are_remembered(tiny):
    """A source of many forks of different lengths still shares its longest ones, and its first ones stay right."""
    g, o = tiny
    base = tokens(o, 925, 340)
    sess = [g.session(500, max_gamma=4, flags=ee.KEEP_LOGITS) for _ in range(4)]
    osess = [o.session(500) for _ in range(4)]
    cut = [340, 17, 300, 340]
    try:
        sess[0].ee_prefill(base)
        sess[0].ee_session_fork(17, sess[1])
        for n in range(34, 300, 11):
            sess[0].ee_session_fork(n, sess[2])
        sess[0].ee_session_fork(300, sess[2])
        sess[2].ee_session_fork(200, sess[3])
        sess[0].ee_session_fork(340, sess[3])
        for b in range(4):
            more = tokens(o, 926, 3 + b, session=b)
            sess[b].ee_prefill(more, flags=ee.CONTINUE)
            fo, _ = oracle_prefill(osess[b], base[:cut[b]] + more)
            sess[b].ee_set_pending(fo)
        sess[0].ee_session_option(ee.OPT_SHARED_ATT, 2)
        drafts = [oracle_greedy(osess[b], 4) for b in range(4)]
        ee.ee_verify_batch(sess, drafts, EXITS)
        for b in range(4):
            sess[b].ee_wait_final()
            check_pass(osess[b].verify(drafts[b], EXITS, want_logits=True), sess[b].final_result(), gpu_logits(sess[b], 1), drafts[b], f"session {b}")
    finally:
        for s in sess:
            s.free()


def test_source_freed_first_and_sampled_batch(tiny):
    g, o = tiny
    a = g.session(300, max_gamma=4, flags=ee.SAMPLING)
    kids = [g.session(300, max_gamma=4, flags=ee.SAMPLING) for _ in range(3)]
    try:
        base = tokens(o, 930, 100)
        a.ee_prefill(base)
        for i, k in enumerate(kids):
            a.ee_session_fork(100, k)
            k.ee_prefill(tokens(o, 931, 3 + i), flags=ee.CONTINUE)
        a.free()
        out = []
        rng = np.random.default_rng(1)
        probs = [np.full((4, o.vocab), 1.0 / o.vocab, np.float32) for _ in kids]
        u, v = [rng.random(4, dtype=np.float32) for _ in kids], [rng.random(5, dtype=np.float32) for _ in kids]
        for option in (1, 2):
            kids[0].ee_session_option(ee.OPT_SHARED_ATT, option)
            marks = [(k.ee_kv_len(), k.ee_pending()) for k in kids]
            ee.ee_verify_sampled_batch(kids, [[1, 2, 3, 4]] * 3, probs, u, v, [1.0] * 3, EXITS)
            got = []
            for k, (n, p) in zip(kids, marks):
                k.ee_wait_final()
                r = k.final_result()
                got.append((r.accept_len, r.next_token, tuple(r.final_tokens), r.final_conf))
                k.ee_kv_truncate(n)
                k.ee_set_pending(p)
            out.append(got)
        for x, y in zip(*out):
            assert np.allclose(x[3], y[3], rtol=1e-4)
    finally:
        for k in kids:
            k.free()


def test_fork_refusals(tiny, model_dir):
    g, o = tiny
    a, b, small = g.session(200), g.session(200), g.session(40)
    try:
        with pytest.raises(ee.EEError) as e:
            a.ee_session_fork(1, b)                              # nothing cached
        assert e.value.code == ee.EE_EINVAL
        a.ee_prefill(tokens(o, 940, 60))
        for n in (0, -1, 61):
            with pytest.raises(ee.EEError) as e:
                a.ee_session_fork(n, b)
            assert e.value.code == ee.EE_EINVAL
        with pytest.raises(ee.EEError):
            a.ee_session_fork(10, a)
        with pytest.raises(ee.EEError) as e:
            a.ee_session_fork(60, small)
        assert e.value.code == ee.EE_ECAPACITY
        a.ee_session_fork(39, small)
        with pytest.raises(ee.EEError) as e:
            small.ee_prefill([1, 2], flags=ee.CONTINUE)
        assert e.value.code == ee.EE_ECAPACITY and small.ee_kv_len() == 39
        with pytest.raises(ee.EEError):
            a.ee_session_option(ee.OPT_SHARED_ATT, 3)
        p2 = f"{model_dir}/gpu_tiny_fork2.bin"
        eegen.write_model(p2, eegen.TINY, 92, gains="uniform")
        g2 = ee.Model(p2)
        c = g2.session(100)
        with pytest.raises(ee.EEError):
            a.ee_session_fork(5, c)
        c.free()
        g2.free()
    finally:
        for s in (a, b, small):
            s.free()
