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


# ------------------------------------------------------------------------------------------------------- embedding
# Up to 256 tokens take one launch for the gradient, more are sorted first: what follows is about the latter.
def _embed_gradient(torch, tokens, dy, vocab, scale, before=None):
    """(dweight, bound, tokens that occur) on the GPU, in 64 bits; the bound is the oracle's."""
    live = (tokens >= 0) & (tokens < vocab)
    at, rows = tokens[live].long(), dy[live].double()
    dw, size = (torch.zeros(vocab, dy.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at, r) for r in (rows, rows.abs()))
    count = torch.bincount(at, minlength=vocab)
    dw, err = dw * scale, (count[:, None] + 2) * E * size * abs(scale)
    if before is not None:
        dw = dw + before.double()
        err = err + E * (dw.abs() + before.double().abs())
    return dw, err, count


def _near(torch, got, ref, bound, dtype, what):
    """got, of this type, is ref to within bound and its rounding, everywhere."""
    bound = bound + (ref.abs() + bound) * HALF[dtype] * 1.001 + (2.0 ** -25 if dtype == "f16" else 0.0)
    bad = ~((got.double() - ref).abs() <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[:3].tolist(), got[bad][:3], ref[bad][:3], bound[bad][:3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [600, 20000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_sorted_gradient_strides(gpu, dtype, rows, accumulate):
    """Some tokens are longer than a piece, some of a dy's and a gradient's rows lie inside wider ones."""
    torch, pb = gpu
    vocab, d = 133, 77
    tokens, dy, first = _words(torch, 1, rows, vocab), _randn(torch, 2, rows, d, dtype=dtype), _randn(torch, 3, vocab, d, dtype=dtype)
    ws = _workspace(torch, pb.embed_workspace_bytes(rows, vocab, d))
    dense, strided = first.clone(), _strided(torch, first, 9, 1)
    print("embed_backward strides", dtype, rows, accumulate, flush=True)
    pb.embed_backward(tokens, dy, dense, ws, scale=0.75, accumulate=accumulate)
    pb.embed_backward(tokens, _strided(torch, dy, 1, 2), strided, ws, scale=0.75, accumulate=accumulate)
    ref, err, count = _embed_gradient(torch, tokens, dy, vocab, 0.75, first if accumulate else None)
    _near(torch, dense, ref, err, dtype, "dweight")
    assert torch.equal(strided, dense) and torch.isnan(strided._base[:, :1]).all() and torch.isnan(strided._base[:, 1 + d:]).all()
    # one row of dy for all tokens, as the gradient of a sum has it
    same = dy[:1].expand(rows, d)
    pb.embed_backward(tokens, same, dense, ws)
    pb.embed_backward(tokens, same.contiguous(), strided, ws)
    assert same.stride(0) == 0 and torch.equal(strided, dense)


def test_embed_sorted_gradient_is_the_slope_of_the_loss(gpu):
    torch, pb = gpu
    tokens, w, dy = _words(torch, 1, 300, 6), _randn(torch, 2, 6, 5), _randn(torch, 3, 300, 5)
    y, dw = torch.empty(300, 5, device="cuda"), torch.empty(6, 5, device="cuda")
    pb.embed_backward(tokens, dy, dw, _workspace(torch, pb.embed_workspace_bytes(300, 6, 5)), scale=2.0)

    def loss(x):
        pb.embed_forward(tokens, x, y, scale=2.0)
        return float((y.double() * dy.double()).sum())
    for i in range(30):
        a, b = w.clone(), w.clone()
        a.view(-1)[i] += 0.5
        b.view(-1)[i] -= 0.5
        # the loss is linear; of its terms 300 at most have this number, each rounded to 2^-24 of at most 2 * 4 * 4 when it is formed and when it is added
        assert abs(float(dw.view(-1)[i]) - (loss(a) - loss(b))) < 300 * 2 * 4 * 4 * 2 * E


def test_embed_sorted_gradient_offsets_beyond_32_bits(gpu):
    """A table of 2.2G elements, written in its first and last rows; one token is longer than a piece."""
    torch, pb = gpu
    vocab, d, rows = 1 << 20, 2112, 300
    dw = torch.full((vocab, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    tokens = torch.randint(vocab - 9, vocab - 1, (rows,), generator=torch.Generator().manual_seed(1))
    tokens[::3], tokens[1], tokens[2] = vocab - 1, 0, vocab
    dy = _randn(torch, 2, rows, d, dtype="bf16")
    print("embed_backward far table", flush=True)
    pb.embed_backward(tokens.cuda(), dy, dw, _workspace(torch, pb.embed_workspace_bytes(rows, vocab, d)))
    at = torch.where(tokens == 0, 0, tokens - (vocab - 10)).cuda()                     # tokens by their place among the first and the last nine rows
    ref, err, count = _embed_gradient(torch, torch.where(tokens.cuda() < vocab, at, -1), dy, 10, 1.0)
    assert int(count[9]) == 100 and int(count[0]) == 1
    _near(torch, torch.cat([dw[:1], dw[-9:]]), ref, err, "bf16", "dweight")
    assert bool((dw[1:-9] == 0).all())


def test_embed_activations_beyond_32_bits(gpu):
    """2.2G elements of y and dy, padding but for tokens at the ends and between."""
    torch, pb = gpu
    rows, vocab, d = (1 << 20) + 700, 50, 2112
    tokens = torch.full((rows,), -1, dtype=torch.int32)
    places = torch.cat([torch.arange(200), torch.arange(rows // 2, rows // 2 + 9), torch.arange(rows - 400, rows)])
    tokens[places] = _words(torch, 1, len(places), vocab, "i32").cpu()
    tokens[-1] = 49
    w, tokens = _randn(torch, 2, vocab, d, dtype="bf16"), tokens.cuda()
    y, dw = torch.full((rows, d), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.empty_like(w)
    print("embed far activations", flush=True)
    pb.embed_forward(tokens, w, y)
    live = (tokens >= 0) & (tokens < vocab)
    # every row: the table's own numbers where there is a token, zeros elsewhere
    assert bool((y[~live] == 0).all()) and torch.equal(y[live], w[tokens[live].long()])
    y[live] = _randn(torch, 3, int(live.sum()), d, dtype="bf16")
    pb.embed_backward(tokens, y, dw, _workspace(torch, pb.embed_workspace_bytes(rows, vocab, d)))
    ref, err, _ = _embed_gradient(torch, tokens[live], y[live], vocab, 1.0)
    _near(torch, dw, ref, err, "bf16", "dweight")


# past the caches: wide rows with a tail, narrow rows of which four go to a thread
@pytest.mark.parametrize("rows,vocab,d,dtype", [(33000, 40000, 4100, "bf16"), (33000, 40000, 4096, "f16"), (33000, 9000, 2050, "f32"), (2200000, 1000, 64, "bf16"), (600000, 70001, 250, "f32")])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_beyond_the_last_level_cache(gpu, rows, vocab, d, dtype, accumulate):
    torch, pb = gpu
    gen = torch.Generator(device="cuda").manual_seed(5)
    new = lambda n: torch.randn(n, d, generator=gen, device="cuda").to({"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype])     # noqa: E731
    tokens, w, dy, dw = _words(torch, 1, rows, vocab), new(vocab), new(rows), new(vocab)
    y = torch.full_like(dy, float("nan"))
    assert y.nbytes > 256e6
    print("embed beyond the cache", rows, vocab, d, dtype, accumulate, flush=True)
    pb.embed_forward(tokens, w, y, scale=1.25)
    live = ((tokens >= 0) & (tokens < vocab))[:, None]
    # 1.25 times a 16-bit number is exact in 32 bits and rounded once to the type; of an fp32 number it is the one rounding
    assert torch.equal(y, torch.where(live, (w[tokens.clamp(0, vocab - 1)].float() * 1.25).to(w.dtype), 0.0))
    ref, err, count = _embed_gradient(torch, tokens, dy, vocab, 1.25, dw if accumulate else None)
    before = dw.clone()
    pb.embed_backward(tokens, dy, dw, _workspace(torch, pb.embed_workspace_bytes(rows, vocab, d)), scale=1.25, accumulate=accumulate)
    _near(torch, dw, ref, err, dtype, "dweight")
    if accumulate:
        assert torch.equal(dw[count == 0], before[count == 0])


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


# few rows: tiles of 128 x 32 and 128 x 64, dz in two terms (three of fp32)
@pytest.mark.parametrize("rows,vocab,d,dtype", [(16, 25000, 256, "bf16"), (48, 25000, 256, "bf16"), (32, 24700, 256, "f16"), (64, 25100, 200, "f16"), (17, 25000, 70, "f32"),
                                                (33, 25003, 100, "f32"), (1, 25000, 64, "bf16"), (30, 24700, 2100, "f16")])
@pytest.mark.parametrize("gradients", [False, True])
def test_head_loss_of_few_rows_of_a_large_vocabulary(gpu, rows, vocab, d, dtype, gradients):
    torch, pb = gpu
    h, w, labels, g = _head_inputs(torch, rows, vocab, d, dtype)
    labels[-1] = vocab - 1
    _check_head(torch, pb, h, w, labels, g, dtype, (rows, vocab, d, dtype, gradients), gradients)


def _head_reference(torch, h, w, labels, g, dtype, gradients):
    """The oracle's values and bounds (oracle.tokens.head_loss has their derivation) on the GPU, in 64 bits, a range of rows at a time."""
    (n, d), v = h.shape, w.shape[0]
    half, least, pairs = HALF[dtype], 2.0 ** -38 if dtype == "f16" else 0.0, dtype == "f32" and n * v * d >= 1e10
    w = w.double()
    aw, wt = w.abs(), w.t().contiguous()
    awt = aw.t().contiguous()
    live = (labels >= 0) & (labels < v)
    at, g = torch.where(live, labels, 0).long()[:, None], torch.where(live, g.double(), 0.0)[:, None]
    parts = {k: [] for k in ("loss", "loss_err", "lse", "lse_err", "dh", "dh_err")}
    dw, dw_err = (torch.zeros_like(w), torch.zeros_like(w)) if gradients else (None, None)
    step = max(1, (1 << 26) // v)
    for i in range(0, n, step):
        s = slice(i, i + step)
        x, a, gi, on = h[s].double(), at[s], g[s], live[s][:, None]
        ax = x.abs()
        z, size = x @ wt, ax @ awt
        zerr = (2 * d + 32) * E * size
        if pairs:
            zerr = 3 * zerr + 3 * 2.0 ** -22 * size + 2.0 ** -38 * 1.01 * (ax.amax(1, keepdim=True) * aw.sum(1)[None] + aw.max() * ax.sum(1, keepdim=True))
        lse = torch.logsumexp(z, 1, keepdim=True)
        p = torch.exp(z - lse)
        perr = zerr + (8 + 2 * (z - lse).abs()) * E
        lse_err = (p * perr).sum(1, keepdim=True) + (160 + v / 2048) * E + 2 * E * lse.abs()
        label = z.gather(1, a)
        parts["lse"].append(lse[:, 0])
        parts["lse_err"].append(lse_err[:, 0])
        parts["loss"].append(torch.where(on, lse - label, 0.0)[:, 0])
        parts["loss_err"].append(torch.where(on, lse_err + zerr.gather(1, a) + 2 * E * (lse.abs() + label.abs()), 0.0)[:, 0])
        if not gradients:
            continue
        hot = torch.zeros_like(p).scatter_(1, a, on.double())
        dz = gi * (p - hot)
        off = gi.abs() * (p * (perr + lse_err) + 2 * E * (p + hot))
        off = off + (dz.abs() + off) * torch.where(hot > 0, max(half * half, E), half) + torch.where(gi != 0, least * float(g.abs().max()), 0.0) + 2 * otk.LEAST * gi.abs()
        x, ax = torch.where(on, x, 0.0), torch.where(on, ax, 0.0)
        parts["dh"].append(dz @ w)
        parts["dh_err"].append(off @ aw + (2 * v + 64) * E * (dz.abs() @ aw) + v * otk.LEAST)
        dw += dz.t().contiguous() @ x
        dw_err += off.t().contiguous() @ ax + (2 * n + 64) * E * (dz.abs().t().contiguous() @ ax)
    r = {k: torch.cat(t) for k, t in parts.items() if t}
    return {**r, "dweight": dw, "dweight_err": dw_err + n * otk.LEAST} if gradients else r


def _check_head_on_gpu(torch, pb, rows, vocab, d, dtype, gradients, stride=None):
    gen = torch.Generator(device="cuda").manual_seed(7)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    h = torch.randn(rows, d, generator=gen, device="cuda").to(dt)
    w = torch.full((vocab, stride or d), float("nan"), dtype=dt, device="cuda")[:, :d]
    w.copy_(torch.randn(vocab, d, generator=gen, device="cuda") * 2.0 * d ** -0.5)
    g = (0.5 + torch.rand(rows, generator=gen, device="cuda")) / rows
    labels = _words(torch, 3, rows, vocab)
    # a vocabulary is cut at multiples of 256: labels on both sides of each
    cuts = torch.arange(256, vocab, 256, device="cuda")
    sides = torch.cat([cuts, cuts - 1, torch.tensor([vocab - 1], device="cuda")])[-rows:]
    labels[:len(sides)] = sides
    out = [torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")] + [torch.full_like(t, float("nan")) for t in (h, w)]
    ws = torch.full((pb.head_loss_workspace_bytes(rows, vocab, d, dt, gradients),), 255, device="cuda", dtype=torch.uint8)
    print("head_loss", rows, vocab, d, dtype, gradients, flush=True)
    more = dict(dh=out[2], dweight=out[3]) if gradients else {}
    pb.head_loss(h, w, labels, out[0], ws, lse=out[1], row_weight=g, **more)
    r = _head_reference(torch, h, w, labels, g, dtype, gradients)
    for name, got in zip(("loss", "lse") + (("dh", "dweight") if gradients else ()), out):
        if got.dtype is torch.float32:
            bad = ~((got.double() - r[name]).abs() <= r[name + "_err"] + (got.double().abs() * 2 * E if name[0] == "d" else 0.0))
            assert not bool(bad.any()), (name, int(bad.sum()), bad.nonzero()[:3].tolist(), got[bad][:3], r[name][bad][:3])
        else:
            _near(torch, got, r[name], r[name + "_err"], dtype, name)
    ws.fill_(0)
    again = [torch.empty_like(t) for t in out]
    more = dict(dh=again[2], dweight=again[3]) if gradients else {}
    pb.head_loss(h, w, labels, again[0], ws, lse=again[1], row_weight=g, **more)
    assert all(torch.equal(a, b) for a, b in zip(out[:4 if gradients else 2], again))


# dz of the whole vocabulary would pass its share of the workspace: two or three pieces, the last one shorter and no multiple of a slice.  W as it lies,
# in rows with gaps, laid out; sums of dh in parts and in one; fp32 in triples and in pairs, whose tiles are 256 x 256 here
@pytest.mark.parametrize("rows,vocab,d,dtype,stride", [(16000, 20000, 128, "bf16", None), (16001, 20011, 64, "f16", None), (16000, 20011, 128, "bf16", 144), (16000, 20011, 72, "f16", None),
                                                       (15999, 40007, 64, "bf16", 67), (16000, 19999, 1100, "bf16", None), (16000, 6500, 100, "f32", None), (16000, 12511, 24, "f32", None),
                                                       (4097, 30011, 90, "f32", None), (5000, 20003, 1030, "f32", None)])
def test_head_loss_gradients_in_pieces(gpu, rows, vocab, d, dtype, stride):
    torch, pb = gpu
    _check_head_on_gpu(torch, pb, rows, vocab, d, dtype, True, stride)


# a weight that is laid out for the losses alone: 128 x 64 and 256 x 256 tiles, pairs of fp16 terms and 16-bit numbers, in pieces
@pytest.mark.parametrize("rows,vocab,d,dtype", [(40, 100501, 2990, "f32"), (300, 120003, 2560, "f32"), (300, 120003, 2565, "bf16"), (2000, 32771, 1024, "f32")])
def test_head_loss_losses_of_large_calls(gpu, rows, vocab, d, dtype):
    torch, pb = gpu
    _check_head_on_gpu(torch, pb, rows, vocab, d, dtype, False)


# W as it lies, in one piece: 256 x 256, 128 x 128 and 64 x 64 tiles, dh in parts, sums of dW short and long
@pytest.mark.parametrize("rows,vocab,d,dtype", [(256, 24700, 2112, "bf16"), (4096, 12000, 256, "f16"), (2500, 12300, 1024, "bf16"), (1210, 2731, 3008, "bf16"), (700, 50001, 512, "f16")])
def test_head_loss_gradients_of_large_tiles(gpu, rows, vocab, d, dtype):
    torch, pb = gpu
    _check_head_on_gpu(torch, pb, rows, vocab, d, dtype, True)


@pytest.mark.parametrize("rows,vocab,d,dtype", [(65, 300, 64, "bf16"), (130, 1000, 100, "f16"), (700, 2500, 512, "bf16"), (4096, 20000, 512, "bf16"), (3000, 33000, 1030, "f16"), (2048, 9000, 2048, "bf16"), (1000, 10000, 300, "f16")])
@pytest.mark.parametrize("weights", ["means", "of all sizes"])
def test_head_loss_gradients_are_off_by_their_own_rounding(gpu, rows, vocab, d, dtype, weights):
    """16-bit gradients against those in 64 bits, in the 2-norm: hardly more off than the exact ones rounded once to the type.

    Rounding leaves r = |round(x) - x| / |x|.  dz is rounded where v is not the label, which leaves at most half a step of each such number: random signs in sums over rows (columns) make
    that at most 2 half / sqrt(12) of the norm of those numbers' part, which is sqrt(sum over v of p^2) of g |h| beside the label's 1 - p.  Here no probability is above a
    quarter but for the label's own, so that the part is below sqrt(1 / 4) of what the label gives, and the whole below sqrt(r^2 + (r / 2)^2) = 1.12 r up to how roundings are distributed: 1.15 r."""
    torch, pb = gpu
    gen = torch.Generator(device="cuda").manual_seed(11)
    dt = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    h, w = torch.randn(rows, d, generator=gen, device="cuda").to(dt), (torch.randn(vocab, d, generator=gen, device="cuda") * d ** -0.5).to(dt)
    g = (0.5 + torch.rand(rows, generator=gen, device="cuda")) / rows
    if weights == "of all sizes":
        g = g * 2.0 ** torch.randint(-6, 1, (rows,), generator=gen, device="cuda")
    labels = _words(torch, 3, rows, vocab)
    # scaled so that the gradients are ordinary fp16 numbers, whose smallest steps do not count here
    g = g * rows
    loss, dh, dw = torch.empty(rows, device="cuda"), torch.empty_like(h), torch.empty_like(w)
    print("head_loss as exact as rounding", rows, vocab, d, dtype, weights, flush=True)
    pb.head_loss(h, w, labels, loss, _workspace(torch, pb.head_loss_workspace_bytes(rows, vocab, d, dt, True)), row_weight=g, dh=dh, dweight=dw)
    x, y = h.double(), w.double()
    live = (labels >= 0) & (labels < vocab)
    p = torch.softmax(x @ y.t().contiguous(), 1)
    assert float(p.max()) < 0.25
    p[live.nonzero()[:, 0], labels[live]] -= 1.0
    p *= torch.where(live, g.double(), 0.0)[:, None]
    for name, got, ref in (("dh", dh, p @ y), ("dweight", dw, p.t().contiguous() @ x)):
        off, least = (float((t.double() - ref).norm() / ref.norm()) for t in (got, ref.to(dt)))
        print(name, f"{off:.6f} {least:.6f}", flush=True)
        assert off < 1.15 * least, (name, off, least)


# dz at the labels in fp32: rows found among all by one launch (up to 2048), or sorted; whole vectors of a row and tails; sums that go on over pieces of the sorted list
@pytest.mark.parametrize("rows,vocab,d,dtype", [(700, 5000, 264, "bf16"), (2048, 1003, 520, "f16"), (2049, 3000, 136, "f16"), (5000, 2001, 91, "bf16"), (17000, 400, 128, "bf16")])
@pytest.mark.parametrize("kind", ["words", "one", "two in turn", "all", "none"])
def test_head_loss_labels_of_every_kind(gpu, rows, vocab, d, dtype, kind):
    torch, pb = gpu
    assert rows * vocab * d > 8e8
    h, w, labels, g = _head_inputs(torch, rows, vocab, d, dtype)
    i = torch.arange(rows, device="cuda")
    labels = {"words": labels, "one": torch.full_like(labels, vocab - 1), "two in turn": i % 2 * (vocab - 1), "all": i * 7 % vocab, "none": torch.full_like(labels, -1)}[kind]
    live = (labels >= 0) & (labels < vocab)

    def run(h, w, labels, dh, dw):
        loss = torch.full((rows,), float("nan"), device="cuda")
        pb.head_loss(h, w, labels, loss, _workspace(torch, pb.head_loss_workspace_bytes(rows, vocab, d, w.dtype, True)), row_weight=g, dh=dh, dweight=dw)
        return loss, dh, dw
    print("head_loss labels", rows, vocab, d, dtype, kind, flush=True)
    new = lambda t: torch.full_like(t, float("nan"))                                                 # noqa: E731
    first = run(h, w, labels, new(h), new(w))
    r = _head_reference(torch, h, w, labels, g, dtype, True)
    assert bool(((first[0].double() - r["loss"]).abs() <= r["loss_err"]).all())
    _near(torch, first[1], r["dh"], r["dh_err"], dtype, "dh")
    _near(torch, first[2], r["dweight"], r["dweight_err"], dtype, "dweight")
    # 32-bit labels, rows to be ignored that hold NaN, rows inside wider ones: the same bits
    bad = torch.where(live[:, None], h, float("nan"))
    dh, dw = _strided(torch, torch.zeros_like(h), 3, 5), _strided(torch, torch.zeros_like(w), 5, 3)
    again = run(_strided(torch, bad, 5, 3), w, labels.int(), dh, dw)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    for t, shift in ((dh, 5), (dw, 3)):
        assert torch.isnan(t._base[:, :shift]).all() and torch.isnan(t._base[:, shift + d:]).all()


@pytest.mark.parametrize("rows,vocab,d", [(600, 2000, 1024), (3000, 2000, 256)])
def test_head_loss_labels_in_a_graph_and_on_two_streams(gpu, rows, vocab, d):
    torch, pb = gpu
    calls = []
    for k in range(2):                                   # the second with other labels, and a workspace of its own
        h, w, labels, g = _head_inputs(torch, rows, vocab, d, "bf16")
        labels = labels if k == 0 else labels.flip(0).contiguous()
        out = torch.empty(rows, device="cuda"), torch.empty_like(h), torch.empty_like(w)
        calls.append((h, w, labels, g, out, _workspace(torch, pb.head_loss_workspace_bytes(rows, vocab, d, h.dtype, True))))

    def run(k, stream=None):
        h, w, labels, g, out, ws = calls[k]
        pb.head_loss(h, w, labels, out[0], ws, row_weight=g, dh=out[1], dweight=out[2], stream=stream)
    want = []
    for k in range(2):
        run(k)
        torch.cuda.synchronize()
        want.append([t.clone() for t in calls[k][4]])
    assert not torch.equal(want[0][2], want[1][2])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for k in range(2):
            run(k, streams[k])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for k in range(2) for a, b in zip(want[k], calls[k][4]))
    # one workspace after the other: what the call before left in it has no influence
    calls[1] = calls[1][:5] + (calls[0][5],)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(0)
        run(1)
    for _ in range(3):
        for k in range(2):
            for t in calls[k][4]:
                t.fill_(0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for k in range(2) for a, b in zip(want[k], calls[k][4]))
        run(0)
        torch.cuda.synchronize()


@pytest.mark.parametrize("rows", [700, 2100])
def test_head_loss_labels_of_rows_that_are_not_finite(gpu, rows):
    """A NaN in a row that counts reaches its own loss and gradient and the weight's, one in a row without a label nothing; a row of weight zero gives nothing."""
    torch, pb = gpu
    vocab, d = 5000, 264
    h, w, labels, g = _head_inputs(torch, rows, vocab, d, "bf16")
    labels[3], labels[5], labels[7] = 17, -1, 4999
    labels[8:20] = 4999
    h[5, 9], g[7:20] = float("nan"), 0.0
    loss, dh, dw = torch.empty(rows, device="cuda"), torch.empty_like(h), torch.empty_like(w)
    ws = _workspace(torch, pb.head_loss_workspace_bytes(rows, vocab, d, h.dtype, True))
    pb.head_loss(h, w, labels, loss, ws, row_weight=g, dh=dh, dweight=dw)
    assert torch.isfinite(loss).all() and torch.isfinite(dh).all() and torch.isfinite(dw).all() and (dh[5] == 0).all() and (dh[7:20] == 0).all()
    h[3, 5] = float("nan")
    pb.head_loss(h, w, labels, loss, ws, row_weight=g, dh=dh, dweight=dw)
    bad = torch.arange(rows, device="cuda") == 3
    assert torch.equal(torch.isnan(loss), bad) and torch.equal(torch.isnan(dh).all(1), bad) and not torch.isnan(dh[~bad]).any() and torch.isnan(dw).all()


@pytest.mark.parametrize("rows,vocab,d,dtype", [(40, 300, 96, "bf16"), (300, 1000, 128, "bf16"), (300, 1000, 100, "f16"), (4000, 9000, 256, "bf16"), (300, 1000, 70, "f32")])
def test_head_loss_gradients_in_place(gpu, rows, vocab, d, dtype):
    """A gradient may lie where its tensor does."""
    torch, pb = gpu
    h, w, labels, g = _head_inputs(torch, rows, vocab, d, dtype)
    loss = _check_head(torch, pb, h, w, labels, g, dtype, ("apart", rows, dtype))[0]
    ws = _workspace(torch, pb.head_loss_workspace_bytes(rows, vocab, d, h.dtype, True))
    r = otk.head_loss(_np(h), _np(w), labels.cpu().numpy(), _np(g), HALF[dtype], 2.0 ** -38 if dtype == "f16" else 0.0)
    for both in ((True, False), (False, True), (True, True)):
        x, y, again = h.clone(), w.clone(), torch.empty_like(loss)
        a, b = x if both[0] else torch.empty_like(x), y if both[1] else torch.empty_like(y)
        pb.head_loss(x, y, labels, again, ws, row_weight=g, dh=a, dweight=b)
        assert torch.equal(again, loss)
        _within(_np(a), r["dh"], _round(r["dh"], r["dh_err"], dtype), "dh")
        _within(_np(b), r["dweight"], _round(r["dweight"], r["dweight_err"], dtype), "dweight")


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


def _distill_reference(torch, z, t, at, temperature, g):
    """The oracle's values and bounds (oracle.tokens.topk_distill) on the GPU, in 64 bits, a range of rows at a time: losses, dlogits in ranges."""
    n, v = z.shape
    top, step = at.shape[1], max(1, (1 << 26) // v)
    for i in range(0, n, step):
        s = slice(i, i + step)
        x, c, a = z[s].double() / temperature, t[s].double() / temperature, at[s].long()
        known = (a >= 0) & (a < v)
        a = torch.where(known, a, 0)
        some = known.any(1)
        lse = torch.logsumexp(x, 1)
        lse_err = (32 + v / 1024 + 4 * x.abs().amax(1)) * E
        log_q = torch.where(known, c, -torch.inf)
        log_q = log_q - torch.where(some, torch.logsumexp(log_q, 1), 0.0)[:, None]
        q = torch.exp(log_q)
        xj = x.gather(1, a)
        qerr = ((16 + top / 64 + 6 * torch.where(known, c.abs(), 0.0).amax(1)) * E)[:, None]
        loss = torch.where(known, q * (log_q - xj + lse[:, None]), 0.0).sum(1) * temperature ** 2
        size = torch.where(known, q * (log_q.abs() + xj.abs() + lse.abs()[:, None]), 0.0)
        loss_err = torch.where(some, temperature ** 2 * ((size * ((top / 64 + 16) * E + qerr)).sum(1) + lse_err), 0.0)
        p = torch.exp(x - lse[:, None])
        c = torch.where(some, g[s].double() * temperature, 0.0)[:, None]
        derr = (p * (lse_err[:, None] + (8 + 4 * x.abs()) * E)).scatter_add_(1, a, q * (qerr + top * E))
        dz = p.scatter_add_(1, a, -q) * c
        yield s, loss, loss_err, dz, (derr + 2 * otk.LEAST) * c.abs() + 4 * E * dz.abs()


# past the caches, in each number of threads a row; rows that begin between two words
@pytest.mark.parametrize("rows,vocab,top,dtype", [(40000, 4096, 33, "bf16"), (9000, 8191, 40, "f32"), (9001, 15001, 100, "f16"), (1100, 131071, 64, "f16"), (1001, 131072, 300, "bf16"),
                                                  (700, 100003, 7, "f32")])
def test_topk_distill_beyond_the_last_level_cache(gpu, rows, vocab, top, dtype):
    torch, pb = gpu
    gen = torch.Generator(device="cuda").manual_seed(5)
    z = (torch.randn(rows, vocab, generator=gen, device="cuda") * 3.0).to({"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype])
    assert z.nbytes > 256e6
    t, at = torch.randn(rows, top, generator=gen, device="cuda") * 3.0, torch.randint(-1, vocab + 1, (rows, top), generator=gen, device="cuda", dtype=torch.int32)
    at[rows // 2] = -1
    g = 0.5 + torch.rand(rows, generator=gen, device="cuda")
    loss, only, dz = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda"), torch.full_like(z, float("nan"))
    print("topk_distill beyond the cache", rows, vocab, top, dtype, flush=True)
    pb.topk_distill(z, t, at, loss, temperature=2.0, row_weight=g, dlogits=dz)
    pb.topk_distill(z, t, at, only, temperature=2.0)
    seen = 0
    for s, ref, err, dref, derr in _distill_reference(torch, z, t, at, 2.0, g):
        for got in (loss, only):
            bad = ~((got[s].double() - ref).abs() <= err)
            assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3].tolist(), got[s][bad][:3], ref[bad][:3], err[bad][:3])
        _near(torch, dz[s], dref, derr, dtype, "dlogits")
        seen += len(ref)
    assert seen == rows


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
