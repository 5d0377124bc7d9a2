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


# -------------------------------------------------------------------------------------- distillation from top logits
@pytest.mark.parametrize("vocab,dtype", [(9000, "f32"), (50021, "f32"), (262144, "f32"), (1 << 21, "f32"), (131072, "bf16"), (1 << 21, "bf16"), ((1 << 21) + 1, "f16")])
@pytest.mark.parametrize("temperature", [1.0, 2.0])
def test_topk_distill_of_confident_rows(gpu, vocab, dtype, temperature):
    """One logit, or two equal ones, far above the rest: the sum of exponentials stays that of the first batch through all later ones.

    lse = (m + log2 s) ln 2 with m the maximum in units of log 2: rounded when the two are added and when they are multiplied, by 2^-24 of lse each, the two
    constants are off by half of that together, a pair's logit is subtracted and added to (two more), its share multiplied and summed: at most 8
    times 2^-24 of lse, and 64 for what does not grow with it (the hardware's logarithm near 1, joining 16 waves of 64 threads).  A probability's exponent
    has no errors but those of lse.  How long the row is does not matter."""
    torch, pb = gpu
    tops = torch.tensor([100.0, 117.5, 251.0, 500.0, 100.0, 117.5, 251.0, 500.0])
    rows = len(tops)
    z = _randn(torch, 1, rows, vocab, dtype=dtype)
    z[:, 3] = tops.to(z.dtype).cuda()
    z[4:, vocab - 5] = z[4:, 3]                    # two
    at, t = torch.tensor([[3, vocab // 2]] * rows, device="cuda"), torch.tensor([[5.0, float("-inf")]] * rows, device="cuda")
    t[::2, 1] = 5.0
    g = torch.ones(rows, device="cuda")
    loss, only, dz = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(z)
    print("topk_distill confident", vocab, dtype, temperature, flush=True)
    pb.topk_distill(z, t, at, loss, temperature=temperature, row_weight=g, dlogits=dz)
    pb.topk_distill(z, t, at, only, temperature=temperature)
    r = otk.topk_distill(_np(z), _np(t), at.cpu().numpy(), temperature)
    off = (8 * tops.numpy() / temperature + 64) * E
    _within(_np(loss), r["loss"], temperature ** 2 * off, "loss")
    _within(_np(only), r["loss"], temperature ** 2 * off, "loss alone")
    _within(_np(dz), r["dlogits"], _round(r["dlogits"], temperature * (off[:, None] + 2 * otk.LEAST), dtype), "dlogits")


# ------------------------------------------------------------------------------------------------------------ refusals
def test_binding_refuses_missing_tensors(gpu):
    torch, pb = gpu
    w, y, tok = torch.zeros(10, 8, device="cuda"), torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    ws, loss = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"), torch.zeros(4, device="cuda")
    z, t, at = torch.zeros(4, 10, device="cuda"), torch.zeros(4, 2, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    calls = [(pb.embed_forward, (tok, w, y)), (pb.embed_backward, (tok, y, w, ws)), (pb.head_loss, (y, w, tok, loss, ws)), (pb.topk_distill, (z, t, at, loss)), (pb.rmsnorm_forward, (y, loss.new_zeros(8), torch.empty_like(y)))]
    for call, args in calls:
        for i in range(len(args)):
            with pytest.raises(pb.PbkdError):
                call(*args[:i], None, *args[i + 1:])
                print("not refused:", call.__name__, i)


# ---------------------------------------------------------------------------------------------------- the token student
def test_token_student_imitates_from_strided_tensors(gpu):
    """The teacher's logits as slices of longer lists, and stored token by token: the gradients of contiguous ones."""
    torch, pb = gpu
    from paper_2012_03096_amd.tokens import TokenStudent
    student = TokenStudent(300, 64, seed=3)
    tokens, teacher = _ints(torch, 1, 0, 300, 3, 11), _randn(torch, 2, 3, 11, 8, scale=3.0)
    at = torch.stack([torch.randperm(300, generator=torch.Generator().manual_seed(k))[:8] for k in range(33)]).view(3, 11, 8).cuda()
    at[1, 2] = -1
    mean = student.imitate_gradients(tokens, teacher[..., :5].contiguous(), at[..., :5].contiguous())
    want = [mean] + [g.clone() for g in student.grads + student.blocks[0].grads]
    turned = [t[..., :5].transpose(0, 1).contiguous().transpose(0, 1) for t in (teacher, at)]
    for given in ((teacher[..., :5], at[..., :5]), turned):
        mean = student.imitate_gradients(tokens, *given)
        assert all(torch.equal(a, b) for a, b in zip(want, [mean] + student.grads + student.blocks[0].grads))


def test_token_student_takes_slices_of_a_text(gpu):
    """Tokens and labels as neighbouring slices of one tensor, and single columns of it."""
    torch, pb = gpu
    from paper_2012_03096_amd.tokens import TokenStudent
    student, text = TokenStudent(300, 64, seed=3), _ints(torch, 1, 0, 300, 3, 12)

    def results(x, y, one, label):
        state = student.new_state(3)
        mean = student.learn_gradients(x, y)
        out = [mean] + [g.clone() for g in student.grads + student.blocks[0].grads]
        return out + [student.score(x, y), student.score(one, label), *student.top_logits(x, 4), student.answer(one[:, 0], state), *state]
    strided = results(text[:, :-1], text[:, 1:], text[:, 3:4], text[:, 4:5])
    dense = results(*(t.contiguous() for t in (text[:, :-1], text[:, 1:], text[:, 3:4], text[:, 4:5])))
    assert all(torch.equal(a, b) for a, b in zip(strided, dense))


def test_token_student_keeps_a_training_pass_sums_in_its_blocks(gpu, monkeypatch):
    """A training pass stores each residual sum in the block that reads it again, and asks for no other room."""
    torch, pb = gpu
    from paper_2012_03096_amd import tokens as module
    student, totals, forward = module.TokenStudent(300, 64, blocks=3, seed=3), [], module.SequenceBlock._forward

    def spy(self, x, residual, lengths, state, state_out, training, total=None):
        totals.append(total)
        return forward(self, x, residual, lengths, state, state_out, training, total=total)
    monkeypatch.setattr(module.SequenceBlock, "_forward", spy)
    x = _ints(torch, 1, 0, 300, 2, 9)
    student.learn_gradients(x, x)
    assert totals == [None] * 3
