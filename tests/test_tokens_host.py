"""CPU-only checks of the token operators: the oracle's gradients against differences of its forward pass, and what the library and the binding
refuse.  Every refused call here returns before any device work."""
import numpy as np
import pytest

from oracle import tokens as otk
from paper_2012_03096_amd import binding as pb


def _difference(f, x, i, h=1e-5):
    a, b = x.copy(), x.copy()
    a.flat[i] += h
    b.flat[i] -= h
    return (f(a) - f(b)) / (2 * h)


def test_oracle_embed_gradients_match_differences():
    rng = np.random.default_rng(1)
    tokens, w, dy = np.array([2, 0, -1, 2, 4, 9, 2]), rng.standard_normal((5, 3)), rng.standard_normal((7, 3))
    dw, _, count = otk.embed_backward(tokens, dy, 5, 1.5)
    assert count.tolist() == [1, 0, 3, 0, 1]
    for i in range(w.size):
        assert abs(dw.flat[i] - _difference(lambda v: (otk.embed(tokens, v, 1.5) * dy).sum(), w, i)) < 1e-8


def test_oracle_head_gradients_match_differences():
    rng = np.random.default_rng(2)
    h, w, g = rng.standard_normal((5, 4)), rng.standard_normal((7, 4)), rng.standard_normal(5)
    labels = np.array([3, -100, 6, 7, 0])
    loss = lambda h_, w_: (otk.head_loss(h_, w_, labels, g)["loss"] * g).sum()                       # noqa: E731
    r = otk.head_loss(h, w, labels, g)
    assert (r["loss"][[1, 3]] == 0).all() and (r["dh"][[1, 3]] == 0).all()
    for i in range(h.size):
        assert abs(r["dh"].flat[i] - _difference(lambda v: loss(v, w), h, i)) < 1e-8
    for i in range(w.size):
        assert abs(r["dweight"].flat[i] - _difference(lambda v: loss(h, v), w, i)) < 1e-8


@pytest.mark.parametrize("temperature", [1.0, 2.5])
def test_oracle_distill_gradients_match_differences(temperature):
    rng = np.random.default_rng(3)
    z, t, g = rng.standard_normal((4, 6)), rng.standard_normal((4, 3)), rng.standard_normal(4)
    at = np.array([[0, 5, 2], [1, 1, 4], [-1, 6, 3], [-1, -1, 9]])
    t[0, 1] = -np.inf
    loss = lambda v: (otk.topk_distill(v, t, at, temperature, g)["loss"] * g).sum()                  # noqa: E731
    r = otk.topk_distill(z, t, at, temperature, g)
    assert r["loss"][3] == 0 and (r["dlogits"][3] == 0).all() and (r["loss"][:3] > 0).all()
    for i in range(z.size):
        assert abs(r["dlogits"].flat[i] - _difference(loss, z, i)) < 1e-8


def test_oracle_distill_is_the_divergence_of_softmaxes():
    """A teacher known everywhere: T^2 KL of the two softmaxes."""
    rng = np.random.default_rng(4)
    z, t = rng.standard_normal((3, 8)), rng.standard_normal((3, 8))
    at = np.stack([rng.permutation(8) for _ in range(3)])
    full = np.zeros_like(t)
    np.put_along_axis(full, at, t, 1)
    p, q = (np.exp(x / 2) / np.exp(x / 2).sum(1, keepdims=True) for x in (z, full))
    assert np.allclose(otk.topk_distill(z, t, at, 2.0)["loss"], 4 * (q * np.log(q / p)).sum(1))


def _desc(fmt, **at):
    v = [0] * len(fmt.unpack(bytes(fmt.size)))
    for i, x in at.items():
        v[int(i[1:])] = x
    return fmt.pack(*v)


def test_library_refuses_bad_embeddings():
    L = pb.lib()
    f = lambda **k: L.pbkd_embed_forward(_desc(pb._EMBED, **k), None)               # noqa: E731
    assert L.pbkd_embed_forward(None, None) == pb.EINVAL
    # rows, vocab, d, dtype, index, scale, tokens, weight, y, strides of weight and y
    ok = dict(_0=4, _1=10, _2=8, _3=pb.F32, _4=pb.I64, _5=1.0, _6=64, _7=64, _8=64, _9=8, _10=8)
    assert f(**{**ok, "_0": 0}) == pb.OK
    assert f(**{**ok, "_0": -1}) == pb.ESHAPE and f(**{**ok, "_1": 0}) == pb.ESHAPE and f(**{**ok, "_2": 0}) == pb.ESHAPE
    assert f(**{**ok, "_0": (1 << 23) + 1}) == pb.EUNSUPPORTED and f(**{**ok, "_1": (1 << 22) + 1}) == pb.EUNSUPPORTED and f(**{**ok, "_2": 65537}) == pb.EUNSUPPORTED
    assert f(**{**ok, "_3": pb.E4M3}) == pb.EINVAL and f(**{**ok, "_4": pb.F32}) == pb.EINVAL
    for k in ("_6", "_7", "_8"):
        assert f(**{**ok, k: 0}) == pb.EINVAL and f(**{**ok, k: 66}) == pb.EINVAL
    assert f(**{**ok, "_6": 68}) == pb.EINVAL                                        # 64-bit tokens
    assert f(**{**ok, "_9": -8}) == pb.EINVAL and f(**{**ok, "_10": 7}) == pb.ESHAPE
    b = lambda **k: L.pbkd_embed_backward(_desc(pb._EMBED_GRAD, **k), None)         # noqa: E731
    assert L.pbkd_embed_backward(None, None) == pb.EINVAL
    need = L.pbkd_embed_workspace_bytes(4, 10, 8)
    assert need > 0
    for bad in ((-1, 10, 8), (4, 0, 8), (4, 10, 0), ((1 << 23) + 1, 10, 8), (4, (1 << 22) + 1, 8), (4, 10, 65537)):
        assert L.pbkd_embed_workspace_bytes(*bad) == 0
    # rows, vocab, d, dtype, index, scale, accumulate, tokens, dy, dweight, strides of dy and dweight, workspace
    ok = dict(_0=4, _1=10, _2=8, _3=pb.BF16, _4=pb.I32, _5=1.0, _7=64, _8=64, _9=64, _10=8, _11=8, _12=256, _13=need)
    assert b(**{**ok, "_0": 0, "_6": 1}) == pb.OK                                    # nothing to add
    for k in ("_7", "_8", "_9"):
        assert b(**{**ok, k: 0}) == pb.EINVAL and b(**{**ok, k: 65}) == pb.EINVAL
    assert b(**{**ok, "_10": -1}) == pb.EINVAL and b(**{**ok, "_11": 7}) == pb.ESHAPE
    assert b(**{**ok, "_12": 0}) == pb.ENOMEM and b(**{**ok, "_12": 128}) == pb.ENOMEM and b(**{**ok, "_13": need - 1}) == pb.ENOMEM
    assert b(**{**ok, "_3": 7}) == pb.EINVAL and b(**{**ok, "_4": 7}) == pb.EINVAL


def test_library_refuses_bad_vocabulary_losses():
    L = pb.lib()
    f = lambda **k: L.pbkd_head_loss(_desc(pb._HEAD_LOSS, **k), None)               # noqa: E731
    assert L.pbkd_head_loss(None, None) == pb.EINVAL
    size = L.pbkd_head_loss_workspace_bytes
    need = size(4, 10, 8, pb.BF16, 1)
    assert need > size(4, 10, 8, pb.BF16, 0) > 0
    for bad in ((-1, 10, 8, 0, 0), (4, 0, 8, 0, 0), (4, 10, 0, 0, 0), ((1 << 21) + 1, 10, 8, 0, 0), (4, (1 << 22) + 1, 8, 0, 0), (4, 10, 65537, 0, 0), (4, 10, 8, 3, 0)):
        assert size(*bad) == 0
    # rows, vocab, d, dtype, index, h, weight, labels, row_weight, loss, lse, dh, dweight, strides of h weight dh dweight, workspace
    ok = dict(_0=4, _1=10, _2=8, _3=pb.BF16, _4=pb.I64, _5=64, _6=64, _7=64, _9=64, _11=64, _12=64, _13=8, _14=8, _15=8, _16=8, _17=256, _18=need)
    assert f(**{**ok, "_0": -1}) == pb.ESHAPE and f(**{**ok, "_1": 0}) == pb.ESHAPE and f(**{**ok, "_2": 0}) == pb.ESHAPE
    assert f(**{**ok, "_0": (1 << 21) + 1}) == pb.EUNSUPPORTED and f(**{**ok, "_1": (1 << 22) + 1}) == pb.EUNSUPPORTED and f(**{**ok, "_2": 65537}) == pb.EUNSUPPORTED
    assert f(**{**ok, "_3": pb.E4M3}) == pb.EINVAL and f(**{**ok, "_4": 0}) == pb.EINVAL
    for k in ("_5", "_6", "_7", "_9", "_11", "_12"):
        assert f(**{**ok, k: 0}) == pb.EINVAL and f(**{**ok, k: 65}) == pb.EINVAL
    assert f(**{**ok, "_8": 66}) == pb.EINVAL and f(**{**ok, "_10": 66}) == pb.EINVAL
    assert f(**{**ok, "_13": -8}) == pb.EINVAL and f(**{**ok, "_14": -8}) == pb.EINVAL
    assert f(**{**ok, "_15": 7}) == pb.ESHAPE and f(**{**ok, "_16": 7}) == pb.ESHAPE
    assert f(**{**ok, "_17": 0}) == pb.ENOMEM and f(**{**ok, "_17": 64}) == pb.ENOMEM and f(**{**ok, "_18": need - 1}) == pb.ENOMEM
    assert f(**{**ok, "_0": 0, "_11": 0, "_12": 0}) == pb.OK


def test_library_refuses_bad_distillations():
    L = pb.lib()
    f = lambda **k: L.pbkd_topk_distill(_desc(pb._TOPK_DISTILL, **k), None)         # noqa: E731
    assert L.pbkd_topk_distill(None, None) == pb.EINVAL
    # rows, vocab, top, dtype, teacher's, index, temperature, logits, teacher, at, row_weight, loss, dlogits, strides of logits and dlogits
    ok = dict(_0=4, _1=10, _2=3, _3=pb.F16, _4=pb.F32, _5=pb.I32, _6=2.0, _7=64, _8=64, _9=64, _11=64, _12=128, _13=10, _14=10)
    assert f(**{**ok, "_0": 0}) == pb.OK
    assert f(**{**ok, "_0": -1}) == pb.ESHAPE and f(**{**ok, "_1": 0}) == pb.ESHAPE and f(**{**ok, "_2": 0}) == pb.ESHAPE
    assert f(**{**ok, "_2": 1025}) == pb.EUNSUPPORTED and f(**{**ok, "_0": (1 << 21) + 1}) == pb.EUNSUPPORTED
    assert f(**{**ok, "_1": (1 << 30) + 1, "_13": 1 << 31, "_14": 1 << 31}) == pb.EUNSUPPORTED
    assert f(**{**ok, "_3": 3}) == pb.EINVAL and f(**{**ok, "_4": 3}) == pb.EINVAL and f(**{**ok, "_5": 3}) == pb.EINVAL
    for bad in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
        assert f(**{**ok, "_6": bad}) == pb.EINVAL
    for k in ("_7", "_8", "_9", "_11"):
        assert f(**{**ok, k: 0}) == pb.EINVAL and f(**{**ok, k: 65}) == pb.EINVAL
    assert f(**{**ok, "_10": 66}) == pb.EINVAL and f(**{**ok, "_12": 65}) == pb.EINVAL
    assert f(**{**ok, "_13": -1}) == pb.EINVAL and f(**{**ok, "_14": 9}) == pb.ESHAPE
    assert f(**{**ok, "_12": 64, "_14": 12}) == pb.EINVAL and "stride" in pb.last_error()


def test_binding_refuses_tensors_on_the_host():
    torch = pytest.importorskip("torch")
    w, y, t = torch.zeros(10, 8), torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    ws, loss = torch.zeros(1024, dtype=torch.uint8), torch.zeros(4)
    for call in (lambda: pb.embed_forward(t, w, y), lambda: pb.embed_backward(t, y, w, ws), lambda: pb.head_loss(y, w, t, loss, ws),
                 lambda: pb.topk_distill(y, y[:, :2].contiguous(), t[:, None].expand(4, 2).contiguous(), loss), lambda: pb.embed_forward(t, w.double(), y.double())):
        with pytest.raises(pb.PbkdError):
            call()


def test_binding_refuses_missing_tensors_without_a_gpu():
    torch = pytest.importorskip("torch")
    y, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: pb.embed_forward(t, None, y), lambda: pb.embed_backward(t, y, None, None), lambda: pb.head_loss(None, y, t, y[:, 0], None),
                 lambda: pb.topk_distill(None, y, t, y[:, 0]), lambda: pb.rmsnorm_forward(None, y[0], y)):
        with pytest.raises(pb.PbkdError, match="missing"):
            call()
