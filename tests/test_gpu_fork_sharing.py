"""Verify batches over forked sessions: when common pages are read once.

Reading common pages once sums in another order than reading them for every session, and each way gives the same bits whenever it is taken: the
bits of a batch's confidences and logits say which way it went."""
import dataclasses

import numpy as np
import pytest

import eegen
import paper_2505_21594_amd as ee

pytestmark = pytest.mark.gpu

EXITS = [1]
GAMMA = 4


@pytest.fixture(scope="module")
def models(model_dir):
    made = {}

    def get(heads, hd):
        if (heads, hd) not in made:
            p = f"{model_dir}/gpu_sharing_{heads}_{hd}.bin"
            cfg = dataclasses.replace(eegen.TINY, n_layers=2, d_model=heads * hd, n_heads=heads, head_dim=hd, d_ffn=512, vocab=512, exit_layers=(1,))
            eegen.write_model(p, cfg, 95, gains="uniform")
            made[heads, hd] = ee.Model(p, max_rows=48)
        return made[heads, hd]

    yield get
    for m in made.values():
        m.free()


def tokens(m, seed, n, session=0):
    return list(eegen.prompt_tokens(seed, n, 512, session=session))


def forks(m, n_sess, common, own=41):
    """Sessions with `common` positions of the first, and their own behind them."""
    s = [m.session(common + own + 60, max_gamma=GAMMA, flags=ee.KEEP_LOGITS) for _ in range(n_sess)]
    s[0].ee_prefill(tokens(m, 950, common))
    for k in s[1:]:
        s[0].ee_session_fork(common, k)
    for i, k in enumerate(s):
        k.ee_prefill(tokens(m, 951, own, session=i), flags=ee.CONTINUE)
    return s


def one_pass(sess, option, gamma=GAMMA):
    """Logits and confidences of one pass; the sessions are as they were before it."""
    sess[0].ee_session_option(ee.OPT_SHARED_ATT, option)
    before = [(s.ee_kv_len(), s.ee_pending()) for s in sess]
    ee.ee_verify_batch(sess, [[3, 1, 4, 1][:gamma]] * len(sess), EXITS)
    out = []
    for s, (n, p) in zip(sess, before):
        s.ee_wait_final()
        out.append(np.concatenate([s.ee_debug_logits(1).ravel(), s.final_result().final_conf]))
        s.ee_kv_truncate(n)
        s.ee_set_pending(p)
    return np.stack(out)


def same(a, b):
    return (a.view(np.uint32) == b.view(np.uint32)).all()


# heads, head size, sessions, common positions, drafts, the faster way by at least 7 % (1: read for every session, 2: once)
FASTER = [
    (4, 64, 8, 4096, 4, 1),
    (20, 64, 8, 512, 4, 1),
    (20, 64, 8, 1024, 4, 2),
    (20, 64, 4, 2048, 4, 2),
    (4, 64, 16, 4096, 2, 2),
    (32, 128, 2, 512, 4, 1),
    (32, 128, 2, 2048, 4, 2),
    (32, 128, 8, 128, 4, 1),
    (32, 128, 8, 256, 4, 2),
]


@pytest.mark.parametrize("heads,hd,n_sess,common,gamma,faster", FASTER)
def test_the_default_takes_the_faster_way(models, heads, hd, n_sess, common, gamma, faster):
    sess = forks(models(heads, hd), n_sess, common)
    try:
        each, once = one_pass(sess, 1, gamma), one_pass(sess, 2, gamma)
        assert same(each, one_pass(sess, 1, gamma)) and same(once, one_pass(sess, 2, gamma))
        assert not same(each, once)
        assert np.abs(each - once).max() < 1e-3
        chosen = one_pass(sess, 0, gamma)
        assert same(chosen, each if faster == 1 else once)
    finally:
        for s in sess:
            s.free()


def test_common_pages_are_read_once_and_no_others(models):
    """Shared where whole pages are in common, not below a page, and not what a session has cut off and replaced."""
    m = models(4, 64)
    for common, shared in ((64, True), (17, True), (16, True), (15, False)):
        sess = forks(m, 2, common)
        try:
            each, once = one_pass(sess, 1), one_pass(sess, 2)
            assert same(each, once) != shared
            for s in sess:                                       # cut below a page and filled up again: nothing is in common
                s.ee_kv_truncate(10)
            for i, s in enumerate(sess):
                s.ee_prefill(tokens(m, 952, common + 31, session=i), flags=ee.CONTINUE)
            assert same(one_pass(sess, 1), one_pass(sess, 2))
        finally:
            for s in sess:
                s.free()


def test_a_longer_fork_stays_shared_after_many(models):
    """Of more forks than a session remembers the longest is still read once: the short ones' sessions alone are not."""
    m = models(4, 64)
    src = m.session(500, max_gamma=GAMMA, flags=ee.KEEP_LOGITS)
    kids = [m.session(500, max_gamma=GAMMA, flags=ee.KEEP_LOGITS) for _ in range(2)]
    try:
        src.ee_prefill(tokens(m, 953, 340))
        src.ee_session_fork(20, kids[0])
        for n in range(34, 300, 11):
            src.ee_session_fork(n, kids[1])
        src.ee_session_fork(320, kids[1])
        for i, s in enumerate([src] + kids):
            s.ee_prefill(tokens(m, 954, 9, session=i), flags=ee.CONTINUE)
        long_pair, short_pair = [src, kids[1]], [src, kids[0]]
        assert not same(one_pass(long_pair, 1), one_pass(long_pair, 2))
        assert same(one_pass(short_pair, 1), one_pass(short_pair, 2))    # (24 longer forks have taken its place)
    finally:
        for s in [src] + kids:
            s.free()


def test_sampled_batch_draws_the_same_tokens(models):
    """The two ways' logits differ by roundings, far less than the distances of these draws from their borders: the same drafts are kept, the same tokens follow."""
    m = models(4, 64)
    rng = np.random.default_rng(3)
    src = m.session(400, max_gamma=GAMMA, flags=ee.SAMPLING)
    kids = [m.session(400, max_gamma=GAMMA, flags=ee.SAMPLING) for _ in range(4)]
    try:
        src.ee_prefill(tokens(m, 955, 200))
        for i, k in enumerate(kids):
            src.ee_session_fork(200, k)
            k.ee_prefill(tokens(m, 956, 3 + i, session=i), flags=ee.CONTINUE)
        probs = [np.full((GAMMA, 512), 1.0 / 512, np.float32) for _ in kids]
        drafts = [list(rng.integers(512, size=GAMMA)) for _ in kids]
        for rep in range(4):
            u, v = [rng.random(GAMMA, dtype=np.float32) for _ in kids], [rng.random(GAMMA + 1, dtype=np.float32) for _ in kids]
            out = []
            for option in (1, 2):
                kids[0].ee_session_option(ee.OPT_SHARED_ATT, option)
                before = [(k.ee_kv_len(), k.ee_pending()) for k in kids]
                ee.ee_verify_sampled_batch(kids, drafts, probs, u, v, [1.0] * len(kids), EXITS)
                got = []
                for k, (n, p) in zip(kids, before):
                    k.ee_wait_final()
                    r = k.final_result()
                    got.append((r.accept_len, r.next_token, list(r.final_tokens)))
                    k.ee_kv_truncate(n)
                    k.ee_set_pending(p)
                out.append(got)
            assert out[0] == out[1], f"draw {rep}"
    finally:
        for s in [src] + kids:
            s.free()
