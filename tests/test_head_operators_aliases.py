"""Arrays that calls of the operators around the LM head may not share (argument checks, no GPU)."""
import ctypes

import paper_2505_21594_amd as ee
from tests.test_head_operators_checks import P, distill_args, refused


def test_the_loss_is_not_written_where_its_weights_are_read():
    for vocab in (100, 140001):                              # one launch, and two of which parts of a row read d_loss beside the one that writes the loss
        args = distill_args(vocab=vocab, logits_stride=vocab, d_logits_stride=vocab, loss=3 * P, d_loss=3 * P)
        refused(ee.load_library().ee_distill(ctypes.byref(args), P, 1 << 30, None), "loss and d_loss")
