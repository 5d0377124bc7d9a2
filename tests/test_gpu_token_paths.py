"""GPU tests of the token operators on the paths that only certain sizes, numbers and calls take: exponents at the ends of fp32's range, confident
rows, sorted gradients with strides and far offsets, gradients of few rows, vocabularies in pieces, calls beyond the last-level cache.

Tolerances as in test_gpu_tokens.py; where a test has bounds of its own, their derivation stands there.
"""
import numpy as np
import pytest

from oracle import tokens as otk
from tests.test_gpu_sequence import HALF, E, _np, _randn, _round, _strided, _within, gpu  # noqa: F401
from tests.test_gpu_tokens import _check_head, _head_inputs, _ints, _words, _workspace

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------- vocabulary loss
LARGE = (1210, 2730, 3040)           # fp32 logits from pairs of fp16 terms, the vocabulary ends inside a tile


@pytest.mark.parametrize("what", ["rows of h", "weight", "both"])
def test_head_loss_products_below_the_normal_range(gpu, what):
    """Ordinary numbers on one side and tiny ones on the other: the logits are zero but for 2^-99, losses and gradients those of equal probabilities."""
    torch, pb = gpu
    h, w, labels, g = _head_inputs(torch, *LARGE, "f32")
    labels[:30] = torch.arange(30)
    if what != "weight":
        h[:40] *= 1e-32
    if what != "rows of h":
        w *= 1e-32
    _check_head(torch, pb, h, w, labels, g, "f32", ("tiny", what))


def test_head_loss_large_numbers_that_never_meet(gpu):
    """Products of the largest numbers pass fp32, but h has them where the weight is zero and the other way round: every logit is zero, exactly."""
    torch, pb = gpu
    rows, vocab, d = LARGE
    h, w, labels, g = _head_inputs(torch, rows, vocab, d, "f32")
    h, w = h * 1e30, w * 1e30
    h[:, 1520:], w[:, :1520] = 0.0, 0.0
    loss, dh, dw = torch.empty(rows, device="cuda"), torch.empty_like(h), torch.empty_like(w)
    print("head_loss numbers that never meet", flush=True)
    pb.head_loss(h, w, labels, loss, _workspace(torch, pb.head_loss_workspace_bytes(rows, vocab, d, h.dtype, True)), row_weight=g, dh=dh, dweight=dw)
    # |h| |w|^T is zero, and with it every error of a logit: the bounds are those of the softmax and of the gradients' products
    r = otk.head_loss(_np(h), _np(w), labels.cpu().numpy(), _np(g))
    _within(_np(loss), r["loss"], r["loss_err"], "loss")
    _within(_np(dh), r["dh"], _round(r["dh"], r["dh_err"], "f32"), "dh")
    _within(_np(dw), r["dweight"], _round(r["dweight"], r["dweight_err"], "f32"), "dweight")
