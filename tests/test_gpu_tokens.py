"""GPU tests of the token operators against the 64-bit oracle (oracle/tokens.py), element by element.

Tolerances, from the arithmetic: an output is rounded once to its type (half a unit: 2^-24, 2^-8, 2^-11 of the value for
float32, bfloat16, float16; float16 also 2^-25 below its normal range), on top of what the oracle's bounds (its *_err arrays) allow for fp32
sums.  The vocabulary loss multiplies the logits' gradient in the operands' type: half a unit of each value more, carried through the product
by the oracle; below float16's normal range half a step is 2^-25 where the largest row weight lies above 2^13, so 2^-38 of it.
"""
import numpy as np
import pytest

from oracle import tokens as otk
from tests.test_gpu_sequence import HALF, E, _np, _randn, _round, _strided, _type, _within, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def _ints(torch, seed, lo, hi, *shape, dtype="i64"):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(lo, hi, shape, generator=g).to({"i32": torch.int32, "i64": torch.int64}[dtype]).cuda()


def _words(torch, seed, n, vocab, dtype="i64"):
    """Tokens of which few make up most, with some outside the vocabulary."""
    g = torch.Generator().manual_seed(seed)
    t = (torch.exp(torch.rand(n, generator=g, dtype=torch.float64) * np.log(vocab + 1.0)) - 1).long().clamp(0, vocab - 1)
    t[torch.rand(n, generator=g) < 0.1] = -100
    t[torch.rand(n, generator=g) < 0.05] = vocab
    return t.to({"i32": torch.int32, "i64": torch.int64}[dtype]).cuda()


def _workspace(torch, n):
    assert n > 0
    return torch.full((n,), 255, device="cuda", dtype=torch.uint8)


# ------------------------------------------------------------------------------------------------------- embedding
EMBED = [(1, 1, 1), (1, 300, 16), (7, 5, 33), (64, 1000, 129), (33, 3, 2048), (700, 40, 515), (3000, 5000, 64), (5000, 700, 72), (2500, 20000, 100), (40, 9, 5000),
         (255, 4, 100), (256, 300, 40), (257, 300, 40), (256, 20000, 2100), (20000, 30, 24), (18000, 9000, 520)]


@pytest.mark.parametrize("rows,vocab,d", EMBED)
@pytest.mark.parametrize("dtype,index", [("f32", "i64"), ("bf16", "i32"), ("f16", "i64")])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed(gpu, rows, vocab, d, dtype, index, accumulate):
    torch, pb = gpu
    tokens, w, dy = _words(torch, 1, rows, vocab, index), _randn(torch, 2, vocab, d, dtype=dtype), _randn(torch, 3, rows, d, dtype=dtype)
    print("embed", rows, vocab, d, dtype, index, accumulate, flush=True)
    y = torch.full((rows, d), float("nan"), dtype=w.dtype, device="cuda")
    pb.embed_forward(tokens, w, y, scale=1.25)
    ref = otk.embed(tokens.cpu().numpy(), _np(w), 1.25)
    _within(_np(y), ref, _round(ref, E * np.abs(ref), dtype), "y")
    dy[tokens < 0] = float("nan")                     # padding has no influence
    before = _randn(torch, 4, vocab, d, dtype=dtype) if accumulate else torch.full((vocab, d), float("nan"), dtype=w.dtype, device="cuda")
    dw = before.clone()
    ws = _workspace(torch, pb.embed_workspace_bytes(rows, vocab, d))
    pb.embed_backward(tokens, dy, dw, ws, scale=1.25, accumulate=accumulate)
    ref, err, count = otk.embed_backward(tokens.cpu().numpy(), _np(dy), vocab, 1.25, _np(before) if accumulate else None)
    bound = _round(ref, err, dtype)
    if accumulate:
        bound[count == 0] = 0.0                       # rows that do not occur stay as they are
    _within(_np(dw), ref, bound, "dweight")
    again = before.clone()
    ws.fill_(0)
    pb.embed_backward(tokens, dy, again, ws, scale=1.25, accumulate=accumulate)
    assert torch.equal(dw, again)


@pytest.mark.parametrize("rows,vocab", [(200, 1), (256, 70000), (4096, 1), (4096, 4096), (20000, 70000), (3000, 1 << 20)])
@pytest.mark.parametrize("kind", ["one", "two in turn", "multiples", "falling", "none"])
def test_embed_backward_orders_of_tokens(gpu, rows, vocab, kind):
    """One token everywhere, tokens of one workgroup's share only, tokens in falling order, padding only."""
    torch, pb = gpu
    i = torch.arange(rows)
    tokens = {"one": torch.full((rows,), vocab - 1), "two in turn": (i % 2) * (vocab - 1), "multiples": i * 256 % vocab, "falling": (vocab - 1 - i).clamp(-1),
              "none": torch.full((rows,), -1)}[kind]
    dy = _randn(torch, 1, rows, 16)
    dw = torch.full((vocab, 16), float("nan"), device="cuda")
    print("embed_backward", rows, vocab, kind, flush=True)
    pb.embed_backward(tokens.cuda(), dy, dw, _workspace(torch, pb.embed_workspace_bytes(rows, vocab, 16)))
    ref, err, _ = otk.embed_backward(tokens.numpy(), _np(dy), vocab)
    _within(_np(dw), ref, err, "dweight")


def test_embed_gradient_is_the_slope_of_the_loss(gpu):
    torch, pb = gpu
    tokens, w, dy = _words(torch, 1, 50, 6), _randn(torch, 2, 6, 5), _randn(torch, 3, 50, 5)
    y, dw = torch.empty(50, 5, device="cuda"), torch.empty(6, 5, device="cuda")
    pb.embed_backward(tokens, dy, dw, _workspace(torch, pb.embed_workspace_bytes(50, 6, 5)), scale=2.0)

    def loss(x):
        pb.embed_forward(tokens, x, y, scale=2.0)
        return float((y.double() * dy.double()).sum())
    for i in range(30):
        a, b = w.clone(), w.clone()
        a.view(-1)[i] += 0.5
        b.view(-1)[i] -= 0.5
        # the loss is linear; its 250 terms are rounded to 2^-24 of at most 2 |w| |dy|
        assert abs(float(dw.view(-1)[i]) - (loss(a) - loss(b))) < 250 * 2 * 4 * 4 * 2 ** -23


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_embed_strides_and_shapes(gpu, dtype):
    torch, pb = gpu
    tokens, w, dy = _words(torch, 1, 60, 33), _randn(torch, 2, 33, 77, dtype=dtype), _randn(torch, 3, 60, 77, dtype=dtype)
    y, dw, ws = torch.empty_like(dy), torch.empty_like(w), _workspace(torch, pb.embed_workspace_bytes(60, 33, 77))
    pb.embed_forward(tokens, w, y, scale=3.0)
    pb.embed_backward(tokens, dy, dw, ws)
    ys, dws = _strided(torch, torch.zeros_like(y), 5, 3), _strided(torch, torch.zeros_like(w), 9, 1)
    pb.embed_forward(tokens, _strided(torch, w, 3, 1), ys, scale=3.0)
    pb.embed_backward(tokens, _strided(torch, dy, 1, 2), dws, ws)
    assert torch.equal(ys, y) and torch.equal(dws, dw)
    for t, pad in ((ys, 3), (dws, 1)):
        assert torch.isnan(t._base[:, :pad]).all() and torch.isnan(t._base[:, pad + 77:]).all()
    y3, dw3 = torch.empty(4, 15, 77, dtype=w.dtype, device="cuda"), torch.empty_like(w)
    pb.embed_forward(tokens.view(4, 15), w, y3, scale=3.0)
    pb.embed_backward(tokens.view(4, 15), dy.view(4, 15, 77), dw3, ws)
    assert torch.equal(y3.view(60, 77), y) and torch.equal(dw3, dw)


def test_embed_without_tokens(gpu):
    torch, pb = gpu
    w, y, none = torch.ones(7, 9, device="cuda"), torch.empty(0, 9, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    pb.embed_forward(none, w, y)
    ws = _workspace(torch, pb.embed_workspace_bytes(0, 7, 9))
    pb.embed_backward(none, y, w, ws, accumulate=True)
    assert (w == 1).all()
    pb.embed_backward(none, y, w, ws)
    assert (w == 0).all()


def test_embed_offsets_beyond_32_bits(gpu):
    """A table of 2.2G elements: its last rows are read and written."""
    torch, pb = gpu
    vocab, d = 1 << 20, 2112
    w = torch.zeros(vocab, d, dtype=torch.bfloat16, device="cuda")
    w[-3:] = _randn(torch, 1, 3, d, dtype="bf16")
    tokens = torch.tensor([vocab - 1, 0, vocab - 3, vocab - 1, vocab], device="cuda")
    y = torch.empty(5, d, dtype=torch.bfloat16, device="cuda")
    pb.embed_forward(tokens, w, y)
    assert torch.equal(y, torch.stack([w[-1], w[0], w[-3], w[-1], torch.zeros_like(w[0])]))
    dy = _randn(torch, 2, 5, d, dtype="bf16")
    pb.embed_backward(tokens, dy, w, _workspace(torch, pb.embed_workspace_bytes(5, vocab, d)))
    assert torch.equal(w[-1], (dy[0].float() + dy[3].float()).bfloat16()) and torch.equal(w[-3], dy[2]) and torch.equal(w[0], dy[1])
    assert (w[1:-3] == 0).all() and (w[-2] == 0).all()


# ------------------------------------------------------------------------------------------------- vocabulary loss
HEAD = [(1, 1, 1), (1, 7, 3), (3, 64, 64), (64, 130, 128), (65, 257, 100), (33, 1000, 192), (130, 513, 65), (64, 4096, 256), (257, 300, 576), (300, 2500, 192), (40, 333, 1000)]


def _check_head(torch, pb, h, w, labels, g, dtype, what, gradients=True, out=None):
    """Calls head_loss twice and compares with the oracle; returns the outputs."""
    rows, (vocab, d) = h.shape[0], w.shape
    new = lambda t: torch.full(t.shape, float("nan"), dtype=t.dtype, device="cuda")                 # noqa: E731
    print("head_loss", what, flush=True)
    results = []
    for fill in (255, 0):
        ws = torch.full((pb.head_loss_workspace_bytes(rows, vocab, d, h.dtype, gradients),), fill, device="cuda", dtype=torch.uint8)
        loss, lse = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")
        dh, dw = (new(h), new(w)) if gradients else (None, None)
        pb.head_loss(h, w, labels, loss, ws, lse=lse, row_weight=g, dh=dh, dweight=dw)
        results.append((loss, lse, dh, dw))
    for a, b in zip(*results):
        assert a is None or torch.equal(a, b), "the same bits again"
    loss, lse, dh, dw = results[0]
    r = otk.head_loss(_np(h), _np(w), labels.cpu().numpy(), None if g is None else _np(g), HALF[dtype], 2.0 ** -38 if dtype == "f16" else 0.0, pairs=dtype == "f32" and rows * vocab * d >= 1e10)
    _within(_np(loss), r["loss"], r["loss_err"], "loss")
    _within(_np(lse), r["lse"], r["lse_err"], "lse")
    if gradients:
        _within(_np(dh), r["dh"], _round(r["dh"], r["dh_err"], dtype), "dh")
        _within(_np(dw), r["dweight"], _round(r["dweight"], r["dweight_err"], dtype), "dweight")
    return results[0]


def _head_inputs(torch, rows, vocab, d, dtype, index="i64"):
    h, w = _randn(torch, 1, rows, d, dtype=dtype), _randn(torch, 2, vocab, d, scale=2.0 * d ** -0.5, dtype=dtype)
    g = (0.5 + torch.rand(rows, generator=torch.Generator().manual_seed(4))).cuda() / rows
    return h, w, _words(torch, 3, rows, vocab, index), g


@pytest.mark.parametrize("rows,vocab,d", HEAD)
@pytest.mark.parametrize("dtype,index", [("f32", "i32"), ("bf16", "i64"), ("f16", "i32")])
@pytest.mark.parametrize("gradients", [False, True])
def test_head_loss(gpu, rows, vocab, d, dtype, index, gradients):
    torch, pb = gpu
    h, w, labels, g = _head_inputs(torch, rows, vocab, d, dtype, index)
    _check_head(torch, pb, h, w, labels, g, dtype, (rows, vocab, d, dtype, gradients), gradients)


# large tiles for the losses, for the weight's gradient, for h's gradient
@pytest.mark.parametrize("rows,vocab,d,dtype", [(1600, 8200, 128, "bf16"), (1500, 8300, 70, "f16"), (70, 8200, 1600, "bf16"), (3100, 700, 4100, "bf16"), (8000, 6000, 40, "f32"),
                                                (1300, 10000, 64, "f32")])
def test_head_loss_of_large_tiles_and_pieces(gpu, rows, vocab, d, dtype):
    torch, pb = gpu
    h, w, labels, g = _head_inputs(torch, rows, vocab, d, dtype)
    _check_head(torch, pb, h, w, labels, g, dtype, (rows, vocab, d, dtype))


def test_head_loss_vocabulary_in_pieces(gpu):
    """16000 rows of fp32: dz of 6500 places takes two pieces, the second one not a multiple of a slice."""
    torch, pb = gpu
    h, w, labels, g = _head_inputs(torch, 16000, 6500, 24, "f32")
    _check_head(torch, pb, h, w, labels, g, "f32", "two pieces")


@pytest.mark.parametrize("dtype,d", [("bf16", 2990), ("f32", 2990)])
def test_head_loss_losses_in_pieces(gpu, dtype, d):
    """A weight that is laid out for the losses, in two pieces."""
    torch, pb = gpu
    h, w, labels, g = _head_inputs(torch, 5, 100500, d, dtype)
    labels[0] = 100499
    _check_head(torch, pb, h, w, labels, g, dtype, ("losses in pieces", dtype), gradients=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_head_loss_ignored_labels(gpu, dtype):
    """No label at all; labels at the ends; rows to be ignored that hold NaN; weights of very different sizes, and none."""
    torch, pb = gpu
    h, w, labels, g = _head_inputs(torch, 70, 300, 96, dtype)
    labels[0], labels[1], labels[2] = 0, 299, 300
    g[5], g[6], g[7] = 0.0, 1e-9, -2.0
    first = _check_head(torch, pb, h, w, labels, g, dtype, "ends")
    _check_head(torch, pb, h, w, labels, None, dtype, "no weights")
    live = (labels >= 0) & (labels < 300)
    bad = torch.where(live[:, None], h, float("nan"))
    again = [torch.empty_like(t) for t in first]
    ws = _workspace(torch, pb.head_loss_workspace_bytes(70, 300, 96, h.dtype, True))
    pb.head_loss(bad, w, labels, again[0], ws, lse=again[1], row_weight=g, dh=again[2], dweight=again[3])
    assert torch.equal(again[0], first[0]) and torch.equal(again[2], first[2]) and torch.equal(again[3], first[3])
    assert torch.equal(again[1][live], first[1][live])
    none = torch.full_like(labels, -1)
    pb.head_loss(bad, w, none, again[0], ws, row_weight=g, dh=again[2], dweight=again[3])
    assert (again[0] == 0).all() and (again[2] == 0).all() and (again[3] == 0).all()


def test_head_loss_far_logits(gpu):
    """Logits of hundreds: the sum of exponentials stays in range, one place has all the probability."""
    torch, pb = gpu
    h, w, labels, _ = _head_inputs(torch, 40, 500, 64, "f32")
    h *= 100.0
    labels[:20] = (h[:20] @ w.t()).argmax(1)
    _check_head(torch, pb, h, w, labels, None, "f32", "far logits")


def test_head_loss_rows_do_not_scale_each_other(gpu):
    """A large fp32 call: rows to be ignored hold NaN, infinities or numbers of 1e30; the others' results are those without them, bit for bit."""
    torch, pb = gpu
    rows, vocab, d = 1210, 2730, 3040
    h, w, labels, g = _head_inputs(torch, rows, vocab, d, "f32")
    labels[:40] = -1
    results = []
    for junk in (0.0, float("nan"), float("inf"), 1e30):
        h[:40] = junk
        out = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(h), torch.empty_like(w)
        pb.head_loss(h, w, labels, out[0], _workspace(torch, pb.head_loss_workspace_bytes(rows, vocab, d, h.dtype, True)), lse=out[1], row_weight=g, dh=out[2], dweight=out[3])
        results.append(out)
    for out in results[1:]:
        assert torch.equal(out[0], results[0][0]) and torch.equal(out[1][40:], results[0][1][40:]) and torch.equal(out[2], results[0][2]) and torch.equal(out[3], results[0][3])
    assert bool((results[0][0][:40] == 0).all()) and bool((results[0][2][:40] == 0).all())


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e12, 1e18])
def test_head_loss_numbers_of_any_size(gpu, size):
    """fp32 operands of large calls are scaled for the logits: tiny and huge ones whose products are ordinary, rows of far smaller numbers beside
    them, zeros; small calls do without."""
    torch, pb = gpu
    for rows, vocab, d in ((40, 500, 96), (1210, 2730, 3040)):
        h, w, labels, g = _head_inputs(torch, rows, vocab, d, "f32")
        h, w = h * size, w / size
        h[:10] *= 2.0 ** -20
        h[10], w[3] = 0.0, 0.0
        _check_head(torch, pb, h, w, labels, g, "f32", ("sizes", size, rows))
        if rows == 40 or size == 1e12:
            _check_head(torch, pb, torch.zeros_like(h), w, labels, g, "f32", "zeros")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_head_loss_what_is_not_finite(gpu, dtype):
    """A NaN in a row that counts reaches its own loss and gradient, and the weight's gradient, but no other row."""
    torch, pb = gpu
    h, w, labels, _ = _head_inputs(torch, 20, 100, 64, dtype)
    labels[:] = torch.arange(20)
    h[3, 5] = float("nan")
    loss, dh, dw = torch.empty(20, device="cuda"), torch.empty_like(h), torch.empty_like(w)
    pb.head_loss(h, w, labels, loss, _workspace(torch, pb.head_loss_workspace_bytes(20, 100, 64, h.dtype, True)), dh=dh, dweight=dw)
    bad = torch.arange(20, device="cuda") == 3
    assert torch.equal(torch.isnan(loss), bad) and torch.equal(torch.isnan(dh).all(1), bad) and not torch.isnan(dh[~bad]).any() and torch.isnan(dw).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 100), ("f32", 70)])
def test_head_loss_strides(gpu, dtype, d):
    """Rows inside wider ones, at 16-byte steps (read as they lie) and at odd ones (laid out first): the same bits."""
    torch, pb = gpu
    h, w, labels, g = _head_inputs(torch, 90, 333, d, dtype)
    first = _check_head(torch, pb, h, w, labels, g, dtype, ("strides", d))
    for pad, shift in ((8, 8), (5, 3)):
        dh, dw = _strided(torch, torch.zeros_like(h), pad, shift), _strided(torch, torch.zeros_like(w), pad, shift)
        loss = torch.empty(90, device="cuda")
        ws = _workspace(torch, pb.head_loss_workspace_bytes(90, 333, d, h.dtype, True))
        pb.head_loss(_strided(torch, h, pad, shift), _strided(torch, w, pad, shift), labels, loss, ws, row_weight=g, dh=dh, dweight=dw)
        assert torch.equal(loss, first[0]) and torch.equal(dh, first[2]) and torch.equal(dw, first[3])
        for t in (dh, dw):
            assert torch.isnan(t._base[:, :shift]).all() and torch.isnan(t._base[:, shift + d:]).all()


def test_head_loss_shapes_and_no_rows(gpu):
    torch, pb = gpu
    h, w, labels, g = _head_inputs(torch, 24, 50, 64, "bf16")
    ws = _workspace(torch, pb.head_loss_workspace_bytes(24, 50, 64, h.dtype, True))
    a, b = (torch.empty(24, device="cuda"), torch.empty_like(h), torch.empty_like(w)), (torch.empty(24, device="cuda"), torch.empty_like(h), torch.empty_like(w))
    pb.head_loss(h, w, labels, a[0], ws, row_weight=g, dh=a[1], dweight=a[2])
    pb.head_loss(h.view(4, 6, 64), w, labels.view(4, 6), b[0], ws, row_weight=g, dh=b[1].view(4, 6, 64), dweight=b[2])
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    pb.head_loss(h[:0], w, labels[:0], a[0][:0], ws, dh=a[1][:0], dweight=a[2])
    assert (a[2] == 0).all()


# -------------------------------------------------------------------------------------- distillation from top logits
DISTILL = [(1, 1, 1), (3, 7, 3), (2, 100, 100), (5, 2047, 17), (4, 8192, 64), (3, 8193, 65), (2, 50001, 300), (3, 131072, 1024), (300, 512, 9)]


def _distill_inputs(torch, rows, vocab, top, dtype, teacher, index="i64"):
    z = _randn(torch, 1, rows, vocab, scale=3.0, dtype=dtype)
    t = _randn(torch, 2, rows, top, scale=3.0, dtype=teacher)
    at = _ints(torch, 3, -1, vocab + 1, rows, top, dtype=index)        # some outside, some twice
    g = (0.5 + torch.rand(rows, generator=torch.Generator().manual_seed(4))).cuda()
    return z, t, at, g


def _check_distill(torch, pb, z, t, at, g, temperature, dtype, what):
    rows = z.shape[0]
    print("topk_distill", what, flush=True)
    loss, dz, only = torch.full((rows,), float("nan"), device="cuda"), torch.full_like(z, float("nan")), torch.full((rows,), float("nan"), device="cuda")
    pb.topk_distill(z, t, at, loss, temperature=temperature, row_weight=g, dlogits=dz)
    pb.topk_distill(z, t, at, only, temperature=temperature)
    r = otk.topk_distill(_np(z), _np(t), at.cpu().numpy(), temperature, None if g is None else _np(g))
    # a call without a gradient sums a row in another order: either loss keeps the bound
    _within(_np(loss), r["loss"], r["loss_err"], "loss")
    _within(_np(only), r["loss"], r["loss_err"], "loss alone")
    _within(_np(dz), r["dlogits"], _round(r["dlogits"], r["dlogits_err"], dtype), "dlogits")
    place, again = z.clone(), torch.empty_like(loss)
    pb.topk_distill(place, t, at, again, temperature=temperature, row_weight=g, dlogits=place)
    assert torch.equal(torch.nan_to_num(place, 7.0), torch.nan_to_num(dz, 7.0)) and torch.equal(torch.nan_to_num(again, 7.0), torch.nan_to_num(loss, 7.0))
    return loss, dz


@pytest.mark.parametrize("rows,vocab,top", DISTILL)
@pytest.mark.parametrize("dtype,teacher,index", [("f32", "f32", "i32"), ("bf16", "bf16", "i64"), ("f16", "f32", "i32"), ("bf16", "f16", "i64")])
@pytest.mark.parametrize("temperature", [1.0, 2.5])
def test_topk_distill(gpu, rows, vocab, top, dtype, teacher, index, temperature):
    torch, pb = gpu
    z, t, at, g = _distill_inputs(torch, rows, vocab, top, dtype, teacher, index)
    _check_distill(torch, pb, z, t, at, g, temperature, dtype, (rows, vocab, top, dtype, teacher, temperature))


@pytest.mark.parametrize("vocab,dtype", [(8192, "f32"), (700, "f16"), (16384, "bf16")])
def test_topk_distill_one_repeated_place_among_many(gpu, vocab, dtype):
    torch, pb = gpu
    rows, top = 4, 301
    z, t, _, g = _distill_inputs(torch, rows, vocab, top, dtype, "f32")
    at = torch.stack([torch.randperm(vocab, generator=torch.Generator().manual_seed(r))[:top] for r in range(rows)]).cuda()
    at[1, 300] = at[1, 0]                          # the first and the last pair
    at[2, 257] = at[2, 256]                        # neighbours
    at[3, :150] = torch.arange(150, device="cuda")
    at[3, 150:300] = (torch.arange(150, device="cuda") + 8192) % vocab ^ (1 if vocab > 8192 else 0)
    _check_distill(torch, pb, z, t, at, g, 1.5, dtype, ("one place twice", vocab, dtype))


@pytest.mark.parametrize("vocab", [300, 20000])
def test_topk_distill_rows_without_pairs_and_repeated_places(gpu, vocab):
    torch, pb = gpu
    z, t, at, g = _distill_inputs(torch, 8, vocab, 40, "f32", "f32")
    at[0] = -1                                     # nothing known
    at[1] = 17                                     # one place, forty times
    t[2] = float("-inf")                           # nothing above -infinity
    t[3, 1:] = float("-inf")                       # one pair
    at[4] = torch.arange(40, device="cuda") % 3    # three places in turn
    t[5, 0] = 200.0                                # one has all the weight
    at[5] = torch.arange(40, device="cuda")
    z[6, ::2] = float("-inf")                      # places the student excludes ...
    at[6] = torch.arange(40, device="cuda") * 2 + 1
    z[7, 5] = float("-inf")                        # ... of which the teacher wants one
    at[7] = torch.arange(40, device="cuda")
    loss, dz = _check_distill(torch, pb, z, t, at, g, 2.0, "f32", ("edges", vocab))
    loss, dz = _np(loss), _np(dz)
    assert (loss[[0, 2]] == 0).all() and (dz[[0, 2]] == 0).all() and loss[7] == np.inf and np.isfinite(dz).all() and (dz[6, ::2] == 0).all()
    # p and q each sum to one: the gradient sums to zero, up to the rounding of its terms (magnitudes sum to at most 2 g T)
    assert (np.abs(dz.sum(1)) < (64 + vocab / 64) * E * 2 * 3).all()


def test_topk_distill_what_is_not_finite(gpu):
    """NaN or +infinity among a row's logits, or nothing but -infinity: that row is NaN, no other."""
    torch, pb = gpu
    z, t, at, g = _distill_inputs(torch, 5, 9000, 4, "bf16", "f32")
    at.clamp_(0, 8999)
    z[1, 77], z[2, 8999], z[3] = float("nan"), float("inf"), float("-inf")
    at[2] = torch.arange(4)
    loss, dz = torch.empty(5, device="cuda"), torch.empty_like(z)
    pb.topk_distill(z, t, at, loss, dlogits=dz)
    bad = torch.tensor([False, True, True, True, False], device="cuda")
    assert torch.equal(torch.isnan(loss), bad) and not torch.isnan(dz[~bad]).any() and torch.isnan(dz[bad]).any(1).all()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("vocab", [77, 9001])
def test_topk_distill_strides_and_shapes(gpu, dtype, vocab):
    torch, pb = gpu
    z, t, at, g = _distill_inputs(torch, 6, vocab, 5, dtype, "f32")
    loss, dz = _check_distill(torch, pb, z, t, at, g, 1.5, dtype, ("strides", vocab))
    a, b = torch.empty_like(loss), _strided(torch, torch.zeros_like(z), 7, 3)
    pb.topk_distill(_strided(torch, z, 5, 1), t, at, a, temperature=1.5, row_weight=g, dlogits=b)
    assert torch.equal(a, loss) and torch.equal(b, dz) and torch.isnan(b._base[:, :3]).all() and torch.isnan(b._base[:, 3 + vocab:]).all()
    c = torch.empty_like(z)
    pb.topk_distill(z.view(2, 3, vocab), t.view(2, 3, 5), at.view(2, 3, 5), a, temperature=1.5, row_weight=g, dlogits=c.view(2, 3, vocab))
    assert torch.equal(a, loss) and torch.equal(c, dz)
    pb.topk_distill(z[:0], t[:0], at[:0], a[:0])


def test_topk_distill_gradient_is_the_slope_of_the_loss(gpu):
    torch, pb = gpu
    z, t, at, g = _distill_inputs(torch, 3, 9, 4, "f32", "f32")
    loss, dz = torch.empty(3, device="cuda"), torch.empty_like(z)
    pb.topk_distill(z, t, at, loss, temperature=2.0, row_weight=g, dlogits=dz)
    step = 2.0 ** -7
    for i in range(27):
        r = []
        for s in (step, -step):
            x = z.clone()
            x.view(-1)[i] += s
            pb.topk_distill(x, t, at, loss, temperature=2.0, row_weight=g)
            r.append(float((loss.double() * g.double()).sum()))
        # losses of at most 60 are off by 64 roundings; the third derivative of a log-sum is below 1 / T, times T^2 g step^2 / 6
        assert abs(float(dz.view(-1)[i]) - (r[0] - r[1]) / (2 * step)) < 64 * E * 60 / step + 2 * 1.5 * step ** 2


def test_topk_distill_offsets_beyond_32_bits(gpu):
    torch, pb = gpu
    rows, vocab = 33000, 66000                     # 2.2G logits
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    z[-2:] = _randn(torch, 1, 2, vocab, dtype="bf16")
    at, t = torch.zeros(rows, 2, dtype=torch.int32, device="cuda"), torch.zeros(rows, 2, device="cuda")
    at[-2:] = torch.tensor([[65999, 3], [-1, 65998]])
    last = z[-2:].clone()
    loss, two, dlast = torch.empty(rows, device="cuda"), torch.empty(2, device="cuda"), torch.empty_like(last)
    pb.topk_distill(last, t[-2:].contiguous(), at[-2:].contiguous(), two, dlogits=dlast)
    pb.topk_distill(z, t, at, loss, dlogits=z)
    assert torch.equal(loss[-2:], two) and torch.equal(z[-2:], dlast) and bool((loss[:-2] == loss[0]).all()) and bool((z[:-2] == z[0]).all())


# ---------------------------------------------------------------------------------------- streams, graphs, refusals
def _all_calls(torch, pb):
    """(what to run, its outputs): every operator once, as a training step strings them together."""
    tokens, labels = _words(torch, 1, 300, 900), _words(torch, 2, 300, 900)
    w, g = _randn(torch, 3, 900, 128, dtype="bf16"), torch.full((300,), 1 / 300, device="cuda")
    x, dx, dw, loss, kd = (torch.empty(300, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(300, 128, dtype=torch.bfloat16, device="cuda"), torch.empty_like(w),
                           torch.empty(300, device="cuda"), torch.empty(300, device="cuda"))
    z, t, at, _ = _distill_inputs(torch, 300, 900, 12, "bf16", "bf16")
    dz = torch.empty_like(z)
    ws = _workspace(torch, max(pb.embed_workspace_bytes(300, 900, 128), pb.head_loss_workspace_bytes(300, 900, 128, w.dtype, True)))

    def run(stream=None):
        pb.embed_forward(tokens, w, x, scale=0.1, stream=stream)
        pb.head_loss(x, w, labels, loss, ws, row_weight=g, dh=dx, dweight=dw, stream=stream)
        pb.embed_backward(tokens, dx, dw, ws, scale=0.1, accumulate=True, stream=stream)
        pb.topk_distill(z, t, at, kd, temperature=2.0, row_weight=g, dlogits=dz, stream=stream)
    return run, (x, dx, dw, loss, kd, dz)


def test_token_operators_on_another_stream(gpu):
    torch, pb = gpu
    run, out = _all_calls(torch, pb)
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    for t in out:
        t.fill_(0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    run(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, out))
    for t in out:
        t.fill_(0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, out))


def test_token_operators_on_two_streams_at_once(gpu):
    torch, pb = gpu
    calls = [_all_calls(torch, pb) for _ in range(2)]          # each with a workspace of its own
    calls[0][0]()
    torch.cuda.synchronize()
    want = [t.clone() for t in calls[0][1]]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for (run, _), stream in zip(calls, streams):
            run(stream)
    torch.cuda.synchronize()
    for _, out in calls:
        assert all(torch.equal(a, b) for a, b in zip(want, out))


def test_token_operators_in_a_graph(gpu):
    torch, pb = gpu
    run, out = _all_calls(torch, pb)
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for t in out:
            t.fill_(0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))
        run()                                       # and eagerly in between
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))


def test_binding_refuses_wrong_tensors(gpu):
    torch, pb = gpu
    w, y, tok = torch.zeros(10, 8, device="cuda"), torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    ws, loss = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"), torch.zeros(4, device="cuda")
    z, t, at = torch.zeros(4, 10, device="cuda"), torch.zeros(4, 2, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    bad = [
        lambda: pb.embed_forward(tok.float(), w, y), lambda: pb.embed_forward(tok[::2], w, y[:2]), lambda: pb.embed_forward(tok, w, y.half()), lambda: pb.embed_forward(tok, w, y[:3]),
        lambda: pb.embed_forward(tok, w[0], y), lambda: pb.embed_forward(tok, w.t(), y), lambda: pb.embed_forward(tok.cpu(), w, y), lambda: pb.embed_forward(tok, w[:, :0], y[:, :0]),
        lambda: pb.embed_backward(tok, y, w, ws[:100]), lambda: pb.embed_backward(tok, y, w, None), lambda: pb.embed_backward(tok, y.bfloat16(), w, ws),
        lambda: pb.embed_backward(tok, y[:3], w, ws), lambda: pb.embed_backward(tok, y, w, ws[4:]),
        lambda: pb.head_loss(y, w, tok, loss, ws, dh=y), lambda: pb.head_loss(y, w, tok, loss, None), lambda: pb.head_loss(y, w, tok[:3], loss, ws),
        lambda: pb.head_loss(y, w.bfloat16(), tok, loss, ws), lambda: pb.head_loss(y, w[:, :7], tok, loss, ws), lambda: pb.head_loss(y, w, tok, loss.double(), ws),
        lambda: pb.head_loss(y, w, tok, None, ws), lambda: pb.head_loss(y, w, tok, loss, ws, lse=loss[:2]), lambda: pb.head_loss(y, w, tok, loss, ws, row_weight=loss.bfloat16()),
        lambda: pb.head_loss(y, w, tok, loss, ws, dh=y[:3], dweight=w), lambda: pb.head_loss(y, w, tok, loss, ws[:256]),
        lambda: pb.topk_distill(z, t, at.float(), loss), lambda: pb.topk_distill(z, t, at[:, :1], loss), lambda: pb.topk_distill(z, t[:3], at[:3], loss),
        lambda: pb.topk_distill(z, t.double(), at, loss), lambda: pb.topk_distill(z, t, at, loss[:3]), lambda: pb.topk_distill(z, t, at, loss, dlogits=z.half()),
        lambda: pb.topk_distill(z, t, at, loss, temperature=0.0), lambda: pb.topk_distill(z[:, :0], t, at, loss), lambda: pb.topk_distill(z, t[:, :0], at[:, :0], loss),
        lambda: pb.topk_distill(z.double(), t, at, loss), lambda: pb.topk_distill(z[0], t[0, 0], at[0, 0], loss[:1]), lambda: pb.embed_forward(tok.view(2, 2), w, y), lambda: pb.topk_distill(z, t.cpu(), at, loss),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(pb.PbkdError):
            call()
            print("not refused:", i)
    with pytest.raises(pb.PbkdError):
        pb.head_loss_workspace_bytes(4, 10, 8, torch.float64, False)


# ---------------------------------------------------------------------------------------------------- the token student
def _reference_student(torch, student, tokens, dtype):
    """The student's formulas in torch operations, differentiable: (leaves in the order of the student's gradients, h)."""
    table, norm = student.table.to(dtype).requires_grad_(), student.norm.to(dtype).clone().requires_grad_()
    leaves = [table, norm]

    def rms(x, w):
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
    live = ((tokens >= 0) & (tokens < student.vocab))[..., None]
    out, stream = torch.where(live, table[tokens.clamp(0, student.vocab - 1)], torch.zeros((), dtype=dtype, device="cuda")) * student.scale, None
    for block in student.blocks:
        w = [block.norm.to(dtype).clone(), block.copies[1].to(dtype), block.bias.to(dtype).clone(), block.copies[3].to(dtype)]
        w = [t.requires_grad_() for t in w]
        leaves += w
        s = out if stream is None else out + stream
        u, gate, o = (rms(s, w[0]) @ w[1].t()).split(student.d, -1)
        a, state, ys = torch.sigmoid(gate + w[2]), torch.zeros_like(u[:, 0]), []
        for i in range(u.shape[1]):
            state = a[:, i] * state + torch.sigmoid(-(gate[:, i] + w[2])) * u[:, i]
            ys.append(state)
        stream, out = s, (torch.stack(ys, 1) * o * torch.sigmoid(o)) @ w[3].t()
    return leaves, rms(out + stream, norm).view(-1, student.d)


@pytest.mark.parametrize("blocks", [1, 2])
@pytest.mark.parametrize("way", ["learn", "imitate"])
def test_token_student_gradients(gpu, blocks, way):
    """All operators in a training step, against automatic differentiation of the same formulas in float64.  Between the table and a gradient lie at most
    30 bf16 tensors (15 of a block and its backward pass, twice), each off by at most 2^-8 of its norm, and no step here makes a
    relative error larger than it was by more than its share of the sum it enters: 30 * 2^-8 = 0.12 of a gradient's norm."""
    torch, pb = gpu
    from paper_2012_03096_amd.tokens import TokenStudent
    student = TokenStudent(300, 64, blocks=blocks, seed=3)
    tokens, labels = _ints(torch, 1, 0, 300, 4, 25), _ints(torch, 2, 0, 300, 4, 25)
    tokens[0, 20:], labels[0, 19:], labels[2, 3] = -1, -100, 300
    leaves, h = _reference_student(torch, student, tokens, torch.float64)
    logits = h @ leaves[0].t()
    if way == "learn":
        mean = student.learn_gradients(tokens, labels)
        want = torch.nn.functional.cross_entropy(logits, torch.where((labels >= 0) & (labels < 300), labels, -100).view(-1), ignore_index=-100)
    else:
        teacher, at = _randn(torch, 4, 4, 25, 8, scale=3.0), torch.stack([torch.randperm(300)[:8] for _ in range(100)]).view(4, 25, 8).cuda()
        at[1, 2] = -1
        mean = student.imitate_gradients(tokens, teacher, at, temperature=2.0)
        some = (at >= 0).all(-1).view(-1)
        q = torch.softmax(teacher.view(-1, 8).double() / 2, 1)
        log_p = torch.log_softmax(logits / 2, 1).gather(1, at.view(-1, 8).clamp_min(0))
        want = (4 * (q * (torch.log(q) - log_p)).sum(1) * some).sum() / some.sum()
    want.backward()
    want = want.detach()
    got = student.grads + [g for block in student.blocks for g in block.grads]
    assert len(got) == len(leaves)
    assert abs(float(mean) - float(want)) < 0.12 * float(want)
    for i, (g, leaf) in enumerate(zip(got, leaves)):
        off = float((g.double() - leaf.grad).norm() / leaf.grad.norm())
        print(way, blocks, i, f"{off:.4f}", flush=True)
        assert off < 0.12, (i, off)


def test_token_student_steps_scores_and_answers(gpu):
    torch, pb = gpu
    from paper_2012_03096_amd.tokens import TokenStudent
    student, other = TokenStudent(500, 64, blocks=2, seed=1), TokenStudent(500, 64, seed=2)
    x, y = _ints(torch, 1, 0, 500, 3, 17), _ints(torch, 2, 0, 500, 3, 17)
    before = [p.clone() for p in student.params + student.blocks[1].params]
    student.learn(x, y, 1e-3)
    assert all(bool((a != b).any()) for a, b in zip(before, student.params + student.blocks[1].params))
    values, at = student.top_logits(x, 5)
    assert torch.isfinite(other.imitate(x, values, at, 1e-3)) and at.dtype == torch.int32
    score = student.score(x, y)
    logits = (student._forward(x, False) @ student.table.t()).float()
    # the logits themselves were rounded to bf16 here: half a step of the largest, twice
    want = torch.nn.functional.cross_entropy(logits, y.view(-1), reduction="none")
    assert float((score.view(-1) - want).abs().max()) < 2 * 2.0 ** -8 * float(logits.abs().max()) + 1e-4
    state = student.new_state(3)
    alone = torch.stack([student.answer(x[:, t].contiguous(), state) for t in range(17)], 1)
    # 12 bf16 tensors up to the logits, each off by at most 2^-8 of its norm
    assert float((alone.view(-1, 500).float() - logits).norm() / logits.norm()) < 12 * 2.0 ** -8


def test_token_student_demonstration_runs(gpu):
    from paper_2012_03096_amd import tokens
    losses, off = tokens.demo(vocab=300, d=64, batch=4, length=20, steps=4, report=2)
    assert len(losses) == 6 and np.isfinite(losses).all() and off < 12 * 2.0 ** -8
