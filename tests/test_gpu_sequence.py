"""GPU tests of the sequence operators against the 64-bit oracle (oracle/sequence.py), element by element.

Tolerances, from the arithmetic: an output is rounded once to its type (half a unit: 2^-24, 2^-8, 2^-11 of the value for
float32, bfloat16, float16; float16 also 2^-25 below its normal range), on top of the fp32 error of what is rounded.
For the norm that is a few roundings and a sum of squares (at most 64 products in a row, then a tree): 64 * 2^-24 of the value.
For the recurrence and the gradients the oracle carries a bound along with the values (its *_err arrays), in which a
step's error decays as the state does.  Codes of the 8-bit outputs are compared with the exact quotient: to nearest within half a
step of the grid, random ones one of the two neighbours, up to what fp32 leaves of the quotient (1e-5 of a step and more).
"""
import numpy as np
import pytest

from oracle import sequence as osq

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # 2^-p, p bits of significand
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}
E = osq.EPS32


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2012_03096_amd import binding
    binding.lib()
    return torch, binding


def _type(torch, name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _within(got, ref, bound, what):
    got, ref, bound = np.asarray(got), np.asarray(ref), np.broadcast_to(bound, np.shape(ref))
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    same = (np.isnan(got) & np.isnan(ref)) | (got == ref)
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - ref) <= bound))
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], ref[bad][:3], bound[bad][:3])


def _round(ref, err, dtype):
    """Bound of an output of this type whose unrounded value is off by err."""
    return err + (np.abs(ref) + err) * HALF[dtype] * 1.001 + TINY[dtype]


def _randn(torch, seed, *shape, scale=1.0, dtype="f32"):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(_type(torch, dtype)).cuda()


def _strided(torch, t, pad, shift=0):
    """The same values with `pad` elements behind each row and `shift` in front of all; the gaps hold NaN."""
    n = t.shape[-1]
    buf = torch.full((*t.shape[:-1], n + pad + shift), float("nan"), dtype=t.dtype, device=t.device)
    v = buf[..., shift:shift + n]
    v.copy_(t)
    return v


# ------------------------------------------------------------------------------------------------------------ norm
NORM_SIZES = [(1, 1), (1, 16), (3, 7), (5, 511), (4, 513), (6, 1024), (3, 2047), (2, 2048), (9, 2049), (7, 4096), (3, 8191), (2, 16384), (1025, 64), (9001, 40)]


def _check_codes(torch, q, scale, y, what):
    """q, scale against the exact y: the row's scale, and each code next to y / scale."""
    top = np.maximum(np.abs(y).max(-1), osq.TINY) / 448.0
    _within(scale, top, 80 * E * top, what + " scale")
    x = y / top[:, None]
    _within(q, x, 0.5 * osq.e4m3_spacing(x) * (1 + 1e-4) + np.abs(x) * 1e-5, what + " codes")


@pytest.mark.parametrize("rows,d", NORM_SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("residual", [False, True])
def test_rmsnorm_forward(gpu, rows, d, dtype, residual):
    torch, pb = gpu
    x, w = _randn(torch, 1, rows, d, dtype=dtype), 1.0 + _randn(torch, 2, d, scale=0.3)
    r = _randn(torch, 3, rows, d, scale=4.0, dtype=dtype) if residual else None
    y, s, _ = osq.rmsnorm(_np(x), _np(w), _np(r) if residual else None)
    out, total = torch.full_like(x, float("nan")), torch.full_like(x, float("nan")) if residual else None
    print("rmsnorm_forward", rows, d, dtype, residual, flush=True)
    pb.rmsnorm_forward(x, w, out, residual=r, total=total)
    torch.cuda.synchronize()
    _within(_np(out), y, _round(y, 64 * E * np.abs(y), dtype), "y")
    if residual:
        _within(_np(total), s, _round(s, E * np.abs(s), dtype), "total")
    q, scale = torch.empty(rows, d, device="cuda", dtype=torch.float8_e4m3fn), torch.full((rows,), float("nan"), device="cuda")
    total8 = torch.empty_like(total) if residual else None
    pb.rmsnorm_forward(x, w, q, residual=r, total=total8, scale=scale)
    torch.cuda.synchronize()
    _check_codes(torch, _np(q), _np(scale), y, "e4m3")
    assert not residual or torch.equal(total, total8)


@pytest.mark.parametrize("rows,d", NORM_SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("into_total", [False, True])
def test_rmsnorm_backward(gpu, rows, d, dtype, into_total):
    torch, pb = gpu
    s, w, dy = _randn(torch, 1, rows, d, scale=3.0, dtype=dtype), 1.0 + _randn(torch, 2, d, scale=0.3), _randn(torch, 3, rows, d, dtype=dtype)
    ds = _randn(torch, 4, rows, d, dtype=dtype) if into_total else None
    dx_ref, dw_ref, ex, ew = osq.rmsnorm_backward(_np(s), _np(w), _np(dy), _np(ds) if into_total else None)
    dx, dw = torch.full_like(s, float("nan")), torch.full((d,), float("nan"), device="cuda")
    ws = torch.full((pb.rmsnorm_workspace_bytes(rows, d),), 255, device="cuda", dtype=torch.uint8)
    print("rmsnorm_backward", rows, d, dtype, into_total, flush=True)
    pb.rmsnorm_backward(s, w, dy, dx, dw, ws, dtotal=ds)
    torch.cuda.synchronize()
    _within(_np(dx), dx_ref, _round(dx_ref, ex, dtype), "dx")
    _within(_np(dw), dw_ref, ew, "dweight")
    dx2, dw2 = torch.empty_like(dx), torch.empty_like(dw)
    ws.fill_(0)
    pb.rmsnorm_backward(s, w, dy, dx2, dw2, ws, dtotal=ds)
    torch.cuda.synchronize()
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [33, 520, 2500])
def test_rmsnorm_strides_and_places(gpu, dtype, d):
    """Rows inside wider ones at odd shifts, three dimensions, outputs that are the inputs, gaps left alone."""
    torch, pb = gpu
    rows = 13
    x, r, w = _randn(torch, 1, rows, d, dtype=dtype), _randn(torch, 2, rows, d, dtype=dtype), 1.0 + _randn(torch, 3, d, scale=0.3)
    y, total = torch.empty_like(x), torch.empty_like(x)
    pb.rmsnorm_forward(x, w, y, residual=r, total=total)
    xs, rs, ys, ts = (_strided(torch, t, 5, 3) for t in (x, r, torch.zeros_like(x), torch.zeros_like(x)))
    pb.rmsnorm_forward(xs, w, ys, residual=rs, total=ts)
    assert torch.equal(ys, y) and torch.equal(ts, total)
    for t in (ys, ts):
        b = t._base
        assert torch.isnan(b[:, :3]).all() and torch.isnan(b[:, 3 + d:]).all()
    a, b = x.clone(), r.clone()
    pb.rmsnorm_forward(a, w, a, residual=b, total=b)              # the residual stream in place, y in x's place
    assert torch.equal(a, y) and torch.equal(b, total)
    y3 = torch.empty(1, rows, d, dtype=x.dtype, device="cuda")
    pb.rmsnorm_forward(x[None], w, y3, residual=r[None])
    assert torch.equal(y3[0], y)
    dy, ds = _randn(torch, 4, rows, d, dtype=dtype), _randn(torch, 5, rows, d, dtype=dtype)
    ws = torch.empty(pb.rmsnorm_workspace_bytes(rows, d), device="cuda", dtype=torch.uint8)
    dx, dw, dw2 = torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    pb.rmsnorm_backward(total, w, dy, dx, dw, ws, dtotal=ds)
    for place in (dy.clone(), ds.clone()):
        first = place.clone()
        is_dy = torch.equal(first, dy)
        pb.rmsnorm_backward(total, w, place if is_dy else dy, place, dw2, ws, dtotal=ds if is_dy else place)
        assert torch.equal(place, dx) and torch.equal(dw, dw2)
    dxs = _strided(torch, torch.zeros_like(x), 7, 1)
    pb.rmsnorm_backward(_strided(torch, total, 1, 1), w, _strided(torch, dy, 2, 5), dxs, dw2, ws, dtotal=_strided(torch, ds, 9))
    assert torch.equal(dxs, dx) and torch.equal(dw, dw2) and torch.isnan(dxs._base[:, 1 + d:]).all()


def test_rmsnorm_rows_of_zeros_and_what_is_not_finite(gpu):
    torch, pb = gpu
    d = 300
    x, w = _randn(torch, 1, 5, d), torch.ones(d, device="cuda")
    x[1] = 0.0
    x[2, 7] = float("nan")
    x[3, 11] = float("inf")
    x[4] = 1e-30
    y = torch.empty_like(x)
    pb.rmsnorm_forward(x, w, y)
    q, scale = torch.empty(5, d, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(5, device="cuda")
    pb.rmsnorm_forward(x, w, q, scale=scale)
    y, q, s = _np(y), _np(q), _np(scale)
    assert np.isfinite(y[0]).all() and (y[1] == 0).all() and np.isnan(y[2]).all()
    inf = np.arange(d) == 11
    assert np.isnan(y[3][inf]).all() and (y[3][~inf] == 0).all()
    _within(y[4], np.full(d, 1e-27), 1e-32, "tiny row")
    assert (q[1] == 0).all() and np.isnan(q[2]).all() and np.isnan(q[3][inf]).all() and (q[3][~inf] == 0).all()
    assert np.isfinite(s).all() and (s > 0).all() and np.abs(q[4] * s[4] - 1e-27).max() < 1e-31


@pytest.mark.parametrize("x_scale,w_scale", [(1e15, 1e30), (1e16, 1e-20), (1e-15, 1e-25), (1e-17, 1e35), (1e-12, 1e-29)])
@pytest.mark.parametrize("d", [40, 300, 9000])
def test_rmsnorm_8_bits_of_far_magnitudes(gpu, x_scale, w_scale, d):
    """The sum times the weight would pass fp32's range, or fall under it, where the output is far from both ends."""
    torch, pb = gpu
    x, w = _randn(torch, 1, 6, d, scale=x_scale), _randn(torch, 2, d, scale=w_scale)
    y, _, _ = osq.rmsnorm(_np(x), _np(w), eps=0.0)
    q, scale = torch.empty(6, d, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(6, device="cuda")
    pb.rmsnorm_forward(x, w, q, scale=scale, eps=0.0)
    torch.cuda.synchronize()
    _check_codes(torch, _np(q), _np(scale), y, "e4m3")


def test_rmsnorm_without_rows(gpu):
    torch, pb = gpu
    x, w, dw = torch.empty(0, 8, device="cuda"), torch.ones(8, device="cuda"), torch.full((8,), 3.0, device="cuda")
    pb.rmsnorm_forward(x, w, torch.empty_like(x))
    pb.rmsnorm_backward(x, w, x, torch.empty_like(x), dw, torch.empty(pb.rmsnorm_workspace_bytes(0, 8), device="cuda", dtype=torch.uint8))
    assert (dw == 0).all()


# ------------------------------------------------------------------------------------------------------ recurrence
REC_SIZES = [(1, 1, 1), (2, 17, 5), (3, 16, 64), (1, 64, 4), (2, 65, 66), (1, 128, 64), (2, 129, 130), (3, 300, 36), (5, 64, 3), (1, 2500, 68), (2, 1000, 7), (1, 5003, 2)]


def _rec_inputs(torch, b, t, d, dtype, gated, ragged, state, bias=True):
    q = {"u": _randn(torch, 1, b, t, d, dtype=dtype), "gate": _randn(torch, 2, b, t, d, scale=2.0, dtype=dtype)}
    q["out_gate"] = _randn(torch, 3, b, t, d, dtype=dtype) if gated else None
    q["bias"] = (torch.rand(d, generator=torch.Generator().manual_seed(4)) * 7 - 1).cuda() if bias else None
    q["lengths"] = torch.tensor([[t, 0, 1, t // 2, t - 1][i % 5] for i in range(b)], dtype=torch.int32).cuda() if ragged else None
    q["state"] = _randn(torch, 5, b, d) if state else None
    return q


def _oracle(q, **more):
    a = {k: (v.cpu().numpy() if k == "lengths" else _np(v)) if v is not None else None for k, v in q.items()}
    a.update(more)
    return a


def _forward(torch, pb, q, want_saved=True, fill=float("nan"), **kw):
    b, t, d = q["u"].shape
    out = {"y": torch.full((b, t, d), fill, dtype=q["u"].dtype, device="cuda"), "state": torch.full((b, d), fill, device="cuda"),
           "saved": torch.full((pb.recurrence_saved_bytes(b, t, d),), 255, dtype=torch.uint8, device="cuda") if want_saved else None,
           "workspace": torch.full((pb.recurrence_workspace_bytes(b, t, d),), 255, dtype=torch.uint8, device="cuda")}
    pb.recurrence_forward(**q, y=out["y"], state_out=out["state"], saved=out["saved"], workspace=out["workspace"], **kw)
    return out


def _backward(torch, pb, q, f, dy, dstate_out, want_bias=True, **kw):
    b, t, d = q["u"].shape
    nan = lambda *s, dtype=torch.float32: torch.full(s, float("nan"), dtype=dtype, device="cuda")     # noqa: E731
    g = {k: nan(b, t, d, dtype=q["u"].dtype) for k in ("du", "dgate")}
    g["dout_gate"] = nan(b, t, d, dtype=q["u"].dtype) if q["out_gate"] is not None else None
    g["dbias"], g["dstate"] = nan(d) if want_bias else None, nan(b, d)
    a = {k: v for k, v in q.items() if k != "state"}
    f["workspace"].fill_(255)
    pb.recurrence_backward(**a, dy=dy, saved=f["saved"], dstate_out=dstate_out, workspace=f["workspace"], **g, **kw)
    return g


@pytest.mark.parametrize("b,t,d", REC_SIZES)
@pytest.mark.parametrize("dtype,gated,ragged,state", [("f32", True, True, True), ("f32", False, False, False), ("bf16", True, False, True),
                                                      ("bf16", False, True, False), ("f16", True, True, False)])
def test_recurrence_forward_and_backward(gpu, b, t, d, dtype, gated, ragged, state):
    torch, pb = gpu
    q = _rec_inputs(torch, b, t, d, dtype, gated, ragged, state)
    print("recurrence", b, t, d, dtype, gated, ragged, state, flush=True)
    out = _forward(torch, pb, q)
    ref = osq.recurrence(**_oracle(q))
    torch.cuda.synchronize()
    _within(_np(out["y"]), ref["y"], _round(ref["y"], ref["y_err"], dtype), "y")
    _within(_np(out["state"]), ref["state"], ref["state_err"] + E * np.abs(ref["state"]), "state")
    dy, dT = _randn(torch, 6, b, t, d, dtype=dtype), _randn(torch, 7, b, d) if state else None
    g = _backward(torch, pb, q, out, dy, dT)
    want = osq.recurrence_backward(**_oracle(q, dy=_np(dy), dstate_out=_np(dT) if state else None))
    torch.cuda.synchronize()
    for k in ("du", "dgate") + (("dout_gate",) if gated else ()):
        _within(_np(g[k]), want[k], _round(want[k], want[k + "_err"], dtype), k)
    for k in ("dbias", "dstate"):
        _within(_np(g[k]), want[k], want[k + "_err"] + E * np.abs(want[k]), k)
    again = _forward(torch, pb, q)
    g2 = _backward(torch, pb, q, again, dy, dT)
    torch.cuda.synchronize()
    assert torch.equal(out["y"], again["y"]) and torch.equal(out["state"], again["state"])
    assert all(torch.equal(g[k], g2[k]) for k in g if g[k] is not None)
    bare = _forward(torch, pb, q, want_saved=False)
    assert torch.equal(out["y"], bare["y"])


@pytest.mark.parametrize("b,t,d", [(3, 23, 70), (2, 24, 64), (3, 25, 70), (5, 8, 1), (1100, 33, 122), (1040, 64, 127), (1030, 65, 129), (513, 63, 256)])
@pytest.mark.parametrize("dtype,gated,ragged,state", [("f32", True, True, True), ("bf16", False, True, False), ("f16", True, False, True)])
def test_recurrence_of_short_pieces(gpu, b, t, d, dtype, gated, ragged, state):
    """Around the lengths and numbers of sequences up to which a thread takes the tokens one after the other."""
    test_recurrence_forward_and_backward(gpu, b, t, d, dtype, gated, ragged, state)


@pytest.mark.parametrize("b,t,d", [(4, 15, 66), (7, 16, 64), (3, 17, 129), (260, 31, 65), (5, 32, 64), (4, 33, 70), (300, 16, 515), (6, 47, 3)])
@pytest.mark.parametrize("dtype,gated,ragged,state", [("f32", False, True, True), ("bf16", True, False, True), ("bf16", True, True, False), ("f16", False, False, False)])
def test_recurrence_of_sequences_shorter_than_a_tile(gpu, b, t, d, dtype, gated, ragged, state):
    """Around the lengths at which the backward pass takes tiles of one, two and four waves."""
    test_recurrence_forward_and_backward(gpu, b, t, d, dtype, gated, ragged, state)


@pytest.mark.parametrize("b,t,d", [(1, 8191, 64), (1, 8192, 64), (2, 8321, 70), (3, 9001, 5), (1, 12345, 1), (5, 8200, 130)])
@pytest.mark.parametrize("dtype,gated,ragged,state", [("bf16", True, True, True), ("f16", False, False, True), ("f16", True, False, False), ("f32", True, True, False)])
def test_recurrence_of_long_chains(gpu, b, t, d, dtype, gated, ragged, state):
    """Few long sequences, from 8192 tokens of 16 bits on in taller tiles."""
    test_recurrence_forward_and_backward(gpu, b, t, d, dtype, gated, ragged, state)


@pytest.mark.parametrize("t,d", [(5, 6), (130, 70), (700, 64)])
def test_recurrence_gradient_is_the_slope_of_the_loss(gpu, t, d):
    """A step along the kernels' gradient changes the (64-bit) loss by the gradient's square, to first order."""
    torch, pb = gpu
    q = _rec_inputs(torch, 2, t, d, "f32", True, False, True)
    dy, dT = _randn(torch, 6, 2, t, d), _randn(torch, 7, 2, d)
    g = _backward(torch, pb, q, _forward(torch, pb, q), dy, dT)
    a = _oracle(q)

    def loss(eps):
        m = {**a, "u": a["u"] + eps * _np(g["du"]), "gate": a["gate"] + eps * _np(g["dgate"]), "out_gate": a["out_gate"] + eps * _np(g["dout_gate"]),
             "bias": a["bias"] + eps * _np(g["dbias"]), "state": a["state"] + eps * _np(g["dstate"])}
        f = osq.recurrence(**m)
        return (f["y"] * _np(dy)).sum() + (f["state"] * _np(dT)).sum()

    square = sum((_np(v) ** 2).sum() for v in g.values())
    h = 1e-3 / np.sqrt(square)
    assert abs((loss(h) - loss(-h)) / (2 * h) - square) < 1e-4 * square


@pytest.mark.parametrize("t", [16, 200])
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf")])
def test_recurrence_what_lies_behind_a_sequence_has_no_influence(gpu, t, junk):
    torch, pb = gpu
    b, d = 5, 70
    q = _rec_inputs(torch, b, t, d, "bf16", True, True, True)
    dy, dT = _randn(torch, 6, b, t, d, dtype="bf16"), _randn(torch, 7, b, d)
    f = _forward(torch, pb, q)
    g = _backward(torch, pb, q, f, dy, dT)
    gone = torch.arange(t, device="cuda")[None, :] >= q["lengths"][:, None]
    bad = {k: v.masked_fill(gone[:, :, None], junk) if k in ("u", "gate", "out_gate") else v for k, v in q.items()}
    f2 = _forward(torch, pb, bad)
    g2 = _backward(torch, pb, bad, f2, dy.masked_fill(gone[:, :, None], junk), dT)
    assert torch.equal(f["y"], f2["y"]) and torch.equal(f["state"], f2["state"])
    assert all(torch.equal(g[k], g2[k]) for k in g)
    assert (f["y"][gone] == 0).all() and all((g[k][gone] == 0).all() for k in ("du", "dgate", "dout_gate"))
    assert torch.equal(f["state"][1], q["state"][1]) and torch.equal(g["dstate"][1], dT[1])     # no token at all
    wild = {**q, "lengths": torch.tensor([t + 100, -5, 1, t // 2, t - 1], dtype=torch.int32).cuda()}
    f3 = _forward(torch, pb, wild)
    assert torch.equal(f["y"], f3["y"]) and torch.equal(f["state"], f3["state"])


def test_recurrence_gates_at_their_ends(gpu):
    """gate = -inf takes the new value exactly, gate = +inf keeps the state exactly, over tiles; large states are forgotten."""
    torch, pb = gpu
    b, t, d = 1, 400, 8
    u, gate, state = _randn(torch, 1, b, t, d), torch.full((b, t, d), float("inf"), device="cuda"), torch.full((b, d), 1e30, device="cuda")
    gate[:, 37] = -float("inf")
    y = torch.empty_like(u)
    pb.recurrence_forward(u, gate, y, state=state, workspace=torch.empty(pb.recurrence_workspace_bytes(b, t, d), dtype=torch.uint8, device="cuda"))
    assert (y[:, :37] == state[:, None]).all() and (y[:, 37:] == u[:, 37:38]).all()
    gate[:], gate[:, 0] = 30.0, -float("inf")                       # a memory of 1e13 tokens
    pb.recurrence_forward(u, gate, y, state=state, workspace=torch.empty(pb.recurrence_workspace_bytes(b, t, d), dtype=torch.uint8, device="cuda"))
    assert ((y - u[:, :1]).abs() < 1e-6 * u[:, :1].abs() + 1e-9).all()
    u[:, 100, 3] = float("nan")
    gate[:] = 0.0
    pb.recurrence_forward(u, gate, y, state=state, workspace=torch.empty(pb.recurrence_workspace_bytes(b, t, d), dtype=torch.uint8, device="cuda"))
    assert torch.isnan(y[:, 100:, 3]).all() and torch.isfinite(y[:, :100]).all() and torch.isfinite(y[..., :3]).all() and torch.isfinite(y[..., 4:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("b,t,d", [(3, 9, 10), (2, 200, 67), (2, 140, 128)])
def test_recurrence_strides(gpu, dtype, b, t, d):
    """Column ranges of one projection's output, tokens in front of sequences, odd shifts; gradients into one buffer and in place."""
    torch, pb = gpu
    q = _rec_inputs(torch, b, t, d, dtype, True, True, True)
    dy, dT = _randn(torch, 6, b, t, d, dtype=dtype), _randn(torch, 7, b, d)
    f = _forward(torch, pb, q)
    g = _backward(torch, pb, q, f, dy, dT)
    z = torch.cat([q["u"], q["gate"], q["out_gate"]], 2)
    cols = lambda x: {"u": x[..., :d], "gate": x[..., d:2 * d], "out_gate": x[..., 2 * d:]}                       # noqa: E731
    for view in (z, z.transpose(0, 1).contiguous().transpose(0, 1), _strided(torch, z, 3, 1)):
        v = {**q, **cols(view)}
        y = _strided(torch, torch.zeros_like(dy), 1, 2)
        state, saved, ws = torch.empty_like(q["state"]), torch.empty_like(f["saved"]), torch.empty_like(f["workspace"])
        pb.recurrence_forward(**v, y=y, state_out=state, saved=saved, workspace=ws)
        assert torch.equal(y, f["y"]) and torch.equal(state, f["state"]) and torch.isnan(y._base[..., 2 + d:]).all()
        dz = torch.full_like(view, float("nan"))
        c = cols(dz)
        db, ds = torch.empty(d, device="cuda"), torch.empty_like(dT)
        a = {k: x for k, x in v.items() if k != "state"}
        pb.recurrence_backward(**a, dy=dy, saved=saved, du=c["u"], dgate=c["gate"], dout_gate=c["out_gate"], dbias=db, dstate_out=dT, dstate=ds, workspace=ws)
        assert torch.equal(dz, torch.cat([g["du"], g["dgate"], g["dout_gate"]], 2)) and torch.equal(db, g["dbias"]) and torch.equal(ds, g["dstate"])
    w = z.clone()
    c = cols(w)
    pb.recurrence_backward(**{k: x for k, x in {**q, **c}.items() if k != "state"}, dy=dy, saved=f["saved"], du=c["u"], dgate=c["gate"], dout_gate=c["out_gate"],
                           dbias=db, dstate_out=dT, dstate=ds, workspace=f["workspace"])
    assert torch.equal(w, torch.cat([g["du"], g["dgate"], g["dout_gate"]], 2))
    state = q["state"].clone()
    pb.recurrence_forward(**{**q, "state": state}, y=y, state_out=state, workspace=f["workspace"])
    assert torch.equal(state, f["state"])
    e = dy.clone()
    pb.recurrence_backward(**{k: x for k, x in q.items() if k != "state"}, dy=e, saved=f["saved"], du=e, dgate=torch.empty_like(e), dout_gate=torch.empty_like(e),
                           dstate_out=dT, workspace=f["workspace"])
    assert torch.equal(e, g["du"])


@pytest.mark.parametrize("dtype,gated", [("f32", True), ("bf16", False), ("f16", True)])
def test_recurrence_token_by_token_and_in_pieces(gpu, dtype, gated):
    """Single steps and pieces of any length reach what one call over all tokens reaches (within the oracle's bounds)."""
    torch, pb = gpu
    b, t, d = 3, 300, 67
    q = _rec_inputs(torch, b, t, d, dtype, gated, False, True)
    ref = osq.recurrence(**_oracle(q))
    y, state = torch.empty_like(q["u"]), q["state"].clone()
    for i in range(t):
        pb.recurrence_step(q["u"][:, i], q["gate"][:, i], state, y[:, i], out_gate=q["out_gate"][:, i] if gated else None, bias=q["bias"])
    _within(_np(y), ref["y"], _round(ref["y"], ref["y_err"], dtype), "steps")
    _within(_np(state), ref["state"], ref["state_err"] + E * np.abs(ref["state"]), "steps' state")
    ws = torch.empty(pb.recurrence_workspace_bytes(b, t, d), dtype=torch.uint8, device="cuda")
    state.copy_(q["state"])
    at = 0
    for n in (1, 2, 13, 16, 17, 127, t - 176):
        cut = {k: q[k][:, at:at + n] if q[k] is not None else None for k in ("u", "gate", "out_gate")}
        pb.recurrence_forward(**cut, bias=q["bias"], y=y[:, at:at + n], state=state, state_out=state, workspace=ws)
        at += n
    assert at == t
    _within(_np(y), ref["y"], _round(ref["y"], ref["y_err"], dtype), "pieces")
    idle, other = state.clone(), torch.empty_like(state)
    active = torch.tensor([1, 0, 1], dtype=torch.int32).cuda()
    pb.recurrence_step(q["u"][:, 0], q["gate"][:, 0], idle, y[:, 0], out_gate=q["out_gate"][:, 0] if gated else None, bias=q["bias"], active=active, state_out=other)
    assert torch.equal(idle, state) and torch.equal(other[1], state[1]) and (y[1, 0] == 0).all() and not torch.equal(other[0], state[0])


def test_recurrence_without_tokens(gpu):
    torch, pb = gpu
    u, state = torch.empty(2, 0, 5, device="cuda"), _randn(torch, 1, 2, 5)
    ws = torch.empty(pb.recurrence_workspace_bytes(2, 0, 5), dtype=torch.uint8, device="cuda")
    saved = torch.empty(pb.recurrence_saved_bytes(2, 0, 5), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(state)
    pb.recurrence_forward(u, u, u, state=state, state_out=out, workspace=ws, saved=saved)
    assert torch.equal(out, state)
    pb.recurrence_forward(u, u, u, state_out=out, workspace=ws)
    assert (out == 0).all()
    db, ds = torch.ones(5, device="cuda"), torch.empty_like(state)
    pb.recurrence_backward(u, u, u, saved, u, u, dbias=db, dstate_out=state, dstate=ds, workspace=ws)
    assert (db == 0).all() and torch.equal(ds, state)
    none = torch.empty(0, 4, 5, device="cuda")
    pb.recurrence_forward(none, none, none, workspace=ws)


def test_recurrence_many_sequences_sum_into_the_bias(gpu):
    """More rows of partial sums than one pass of the column sums takes."""
    torch, pb = gpu
    b, t, d = 1500, 3, 6
    q = _rec_inputs(torch, b, t, d, "f32", False, False, False)
    dy = _randn(torch, 6, b, t, d)
    g = _backward(torch, pb, q, _forward(torch, pb, q), dy, None)
    want = osq.recurrence_backward(**_oracle(q, dy=_np(dy)))
    _within(_np(g["dbias"]), want["dbias"], want["dbias_err"], "dbias")


def test_recurrence_offsets_beyond_32_bits(gpu):
    """Sequences more than 2^32 bytes (and 2^31 elements) apart."""
    torch, pb = gpu
    b, t, d = 2, 150, 66
    q = _rec_inputs(torch, b, t, d, "bf16", True, False, False)
    dy = _randn(torch, 6, b, t, d, dtype="bf16")
    f = _forward(torch, pb, q)
    g = _backward(torch, pb, q, f, dy, None)
    far = (1 << 31) + 12345
    need = lambda: torch.empty(far + 8 * t * d, dtype=torch.bfloat16, device="cuda")       # noqa: E731
    buf = need()
    views = [buf.as_strided((b, t, d), (far, d, 1), k * t * d) for k in range(8)]
    for v, k in zip(views, ("u", "gate", "out_gate")):
        v.copy_(q[k])
    views[3].copy_(dy)
    y, du, dg, do = views[4:8]
    pb.recurrence_forward(views[0], views[1], y, out_gate=views[2], bias=q["bias"], saved=f["saved"], workspace=f["workspace"])
    pb.recurrence_backward(views[0], views[1], views[3], f["saved"], du, dg, out_gate=views[2], dout_gate=do, bias=q["bias"], workspace=f["workspace"])
    assert torch.equal(y, f["y"]) and torch.equal(du, g["du"]) and torch.equal(dg, g["dgate"]) and torch.equal(do, g["dout_gate"])


# ----------------------------------------------------------------------------------------------------------- AdamW
SIZES = [1, 3, 255, 256, 257, 1023, 4095, 4096, 4097, 10007]


def _adamw_setup(torch, sizes, param, grad, bits, shift=0, seed=1):
    """Parameters, gradients and states of a training under way; shift: all of them start at odd places."""
    cut = lambda t: t[shift:]                                                              # noqa: E731
    ps = [cut(_randn(torch, seed + i, n + shift, dtype=param)) for i, n in enumerate(sizes)]
    gs = [cut(_randn(torch, seed + 50 + i, n + shift, scale=0.1, dtype=grad)) for i, n in enumerate(sizes)]
    states = []
    for i, n in enumerate(sizes):
        m, v = _randn(torch, seed + 100 + i, n + shift, scale=0.03), _randn(torch, seed + 150 + i, n + shift, scale=0.1).square()
        if bits == 32:
            states.append((cut(m), cut(v)))
            continue
        blocks = -(-n // 256)
        code = lambda x: (x.abs().clamp(max=1.0) * 448).to(torch.float8_e4m3fn)            # noqa: E731
        sign = torch.sign(m)
        states.append((cut((code(m * 10).float() * sign).to(torch.float8_e4m3fn)), cut(code(v.sqrt() * 3)), _randn(torch, seed + 200 + i, blocks).abs() * 1e-4 + 1e-5,
                       _randn(torch, seed + 250 + i, blocks).abs() * 1e-3 + 1e-4))
    return ps, gs, states


def _blocks(x, n):
    return np.repeat(x, 256)[:n]


def _check_adamw(torch, before, grads, opt, decays, lr, bits, param, copies=None, betas=(0.9, 0.999), eps=1e-8, scale=1.0, seed=None):
    """before: clones of (param, states) from before the step."""
    first = 0
    for i, (p0, s0) in enumerate(before):
        n, step = p0.numel(), opt.steps
        m0, v0 = _np(s0[0]), _np(s0[1])
        if bits == 8:
            m0, v0 = m0 * _blocks(_np(s0[2]), n), (v0 * _blocks(_np(s0[3]), n)) ** 2
        g = _np(grads[i])
        p, m, v = osq.adamw(_np(p0), g, m0, v0, lr, step, betas, eps, decays[i], scale)
        em = 8 * E * (np.abs(betas[0] * m0) + np.abs((1 - betas[0]) * g * scale))
        ev = 8 * E * v
        move = np.abs(p - _np(p0) * (1 - lr * decays[i]))
        with np.errstate(divide="ignore", invalid="ignore"):
            ep = 3 * E * np.abs(p) + 24 * E * move + lr / (1 - betas[0] ** step) * np.where(em > 0, em / (np.sqrt(v / (1 - betas[1] ** step)) + eps), 0.0)
        noise = osq.element_hash(n, step if seed is None else seed, first)
        got = _np(opt.params[i])
        if param == "f32":
            _within(got, p, ep, f"param {i}")
            if copies is not None:
                assert torch.equal(copies[i], opt.params[i].to(torch.bfloat16))
        else:
            q = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(p), 2.0 ** -126))) - 7)
            want = np.sign(p) * np.floor(np.abs(p) / q + (noise & 0xFFFF) / 65536.0) * q
            _within(got, p, q * (1 + 1e-3) + ep, f"param {i}")
            near = np.abs((np.abs(p) / q + (noise & 0xFFFF) / 65536.0 + 0.5) % 1 - 0.5) < 1e-3      # where fp32 may fall on either side
            assert near.mean() < 0.02 or n < 1000
            _within(got[~near], want[~near], 1e-30, f"rounding of param {i}")
        s = opt.states[i]
        if bits == 32:
            _within(_np(s[0]), m, em, f"m {i}")
            _within(_np(s[1]), v, ev, f"v {i}")
        else:
            pad = lambda x: np.concatenate([x, np.zeros(-n % 256)]).reshape(-1, 256)       # noqa: E731
            r = np.sqrt(v)
            for k, (x, name) in enumerate(((m, "m"), (r, "v"))):
                top = np.maximum(np.abs(pad(x)).max(1), osq.TINY) / 448.0
                _within(_np(s[2 + k]), top, 16 * E * top, f"{name} scale {i}")
                y, code = x / _blocks(top, n), _np(s[k])
                grid = osq.e4m3_spacing(y)
                if k == 0:
                    _within(code, y, 0.5 * grid * (1 + 1e-3) + em / _blocks(top, n), f"m codes {i}")
                else:
                    t = y / grid + (noise >> 12) / 2.0 ** 20
                    want = np.where(y > 0, np.maximum(np.floor(t) * grid, 2.0 ** -9), 0.0)
                    near = np.abs((t + 0.5) % 1 - 0.5) < 1e-4
                    _within(code, y, np.maximum(grid, 2.0 ** -9) * (1 + 1e-3), f"v codes {i}")
                    _within(code[~near], want[~near], 1e-30, f"v codes' rounding {i}")
        first += -(-n // 256) * 256


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("shift", [0, 1])
def test_adamw_step(gpu, bits, param, grad, shift):
    torch, pb = gpu
    ps, gs, states = _adamw_setup(torch, SIZES, param, grad, bits, shift)
    copies = [torch.empty(n + shift, dtype=torch.bfloat16, device="cuda")[shift:] for n in SIZES] if param == "f32" else None
    decays = [0.1 if i % 2 else 0.0 for i in range(len(SIZES))]
    opt = pb.AdamW(ps, state_bits=bits, states=states, copies=copies, weight_decay=decays, steps=41)
    for _ in range(2):
        before = [(p.clone(), tuple(x.clone() for x in s)) for p, s in zip(ps, states)]
        print("adamw", bits, param, grad, shift, opt.steps, flush=True)
        opt.step(gs, 0.01, grad_scale=0.5)
        torch.cuda.synchronize()
        _check_adamw(torch, before, gs, opt, [np.float64(np.float32(x)) for x in decays], 0.01, bits, param, copies, scale=0.5)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_from_nothing(gpu, bits):
    """The first steps on states made here, of more tensors than one launch takes, some without gradients or elements."""
    torch, pb = gpu
    sizes = [(37 * i) % 700 for i in range(100)]
    ps, gs, _ = _adamw_setup(torch, sizes, "f32", "f32", bits)
    gs = [None if i % 9 == 4 else g for i, g in enumerate(gs)]
    opt = pb.AdamW(ps, state_bits=bits, weight_decay=0.01)
    for _ in range(3):
        before = [(p.clone(), tuple(x.clone() for x in s)) for p, s in zip(ps, opt.states)]
        opt.step(gs, 0.003)
        torch.cuda.synchronize()
        full = [g if g is not None else torch.zeros_like(p) for g, p in zip(gs, ps)]
        for i, (p0, s0) in enumerate(before):
            if gs[i] is None:
                assert torch.equal(p0, ps[i]) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(s0, opt.states[i]))
        keep = [i for i in range(100) if gs[i] is not None and sizes[i]]
        assert keep and opt.steps
        first, wd = 0, np.float64(np.float32(0.01))
        for i, n in enumerate(sizes):
            if i in keep and bits == 32:
                p, m, v = osq.adamw(_np(before[i][0]), _np(full[i]), *(_np(x) for x in before[i][1]), 0.003, opt.steps, weight_decay=wd)
                _within(_np(ps[i]), p, 3 * E * np.abs(p) + 1e-7 * 0.003 + 40 * E * 0.02, f"param {i}")
                _within(_np(opt.states[i][0]), m, 8 * E * (np.abs(m) + np.abs(_np(full[i]))), f"m {i}")
            first += n
    assert first


def test_adamw_random_rounding_is_fair_and_never_reaches_zero(gpu):
    """sqrt(v) of one block's worth of values, over many seeds: the mean of the codes is the value; tiny ones stay above zero."""
    torch, pb = gpu
    n, rounds = 256, 400
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    v0 = torch.linspace(2.0 ** -9, 448.0, n, device="cuda").to(torch.float8_e4m3fn)
    total, x = np.zeros(n), None
    for seed in range(rounds):
        st = [(torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), v0.clone(), torch.zeros(1, device="cuda"), torch.ones(1, device="cuda"))]
        opt = pb.AdamW([p], state_bits=8, states=st, betas=(0.9, 0.9))
        opt.step([g], 0.0, seed=seed)
        total += _np(st[0][1]) * _np(st[0][3])
    x = _np(v0) * np.sqrt(0.9)
    grid = osq.e4m3_spacing(x / x.max() * 448) * x.max() / 448
    assert (np.abs(total / rounds - x) <= 5 * 0.5 * grid / np.sqrt(rounds) + 1e-5 * x).all()      # five sigma of a coin's mean
    g[0], v0 = 1e6, torch.full((n,), 2.0 ** -9, device="cuda").to(torch.float8_e4m3fn)
    v0[5] = 0.0
    st = [(torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), v0, torch.zeros(1, device="cuda"), torch.ones(1, device="cuda"))]
    pb.AdamW([p], state_bits=8, states=st).step([g], 0.0)
    c = _np(st[0][1])
    assert c[0] == 448 and c[5] == 0 and (np.delete(c, [0, 5]) == 2.0 ** -9).all()


def test_adamw_codes_are_those_of_separate_operations(gpu):
    """The 8-bit states of fp32 arithmetic with every product, sum, root and quotient rounded by itself, code for code: products
    fused into their sums would move about four codes in a million over the middle between two, here some ten."""
    torch, pb = gpu
    f, n, b1, b2, scale = np.float32, 3 * 1048576 + 77, 0.9, 0.999, 0.37
    ps, gs, states = _adamw_setup(torch, [n], "f32", "bf16", 8, seed=9)
    m8, v8, sm, sv = [x.clone() for x in states[0]]
    opt = pb.AdamW(ps, state_bits=8, states=states, betas=(b1, b2), steps=6)
    opt.step(gs, 0.01, grad_scale=scale)
    at = lambda t: np.repeat(t.cpu().numpy(), 256)[:n]                                     # noqa: E731
    g = gs[0].float().cpu().numpy() * f(scale)
    m, v = m8.float().cpu().numpy() * at(sm), v8.float().cpu().numpy() * at(sv)
    m = m * f(b1) + g * f(1 - b1)
    root = np.sqrt((v * v) * f(b2) + (g * g) * f(1 - b2))
    up = (osq.element_hash(n, 7) >> 12).astype(np.uint32)
    for k, x in ((0, m), (1, root)):
        top = np.abs(np.concatenate([x, np.zeros(-n % 256, f)]).reshape(-1, 256)).max(1)
        assert x.dtype == top.dtype == f
        assert (states[0][2 + k].cpu().numpy() == top * f(1 / 448)).all()
        x = np.minimum(x * np.repeat(f(1) / top * f(448), 256)[:n], f(448))
        if k == 1:
            low = np.where(x < f(2.0 ** -6), f(2.0 ** -6), f(0))
            r = ((((x + low).view(np.uint32) + up) & np.uint32(0xFFF00000)).view(f)) - low
            x = np.where(x > 0, np.maximum(r, f(2.0 ** -9)), f(0))
        want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8)
        assert torch.equal(states[0][k].cpu().view(torch.uint8), want)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", ["f32", "bf16"])
def test_adamw_steps_are_those_of_separate_operations(gpu, bits, param):
    """Parameters and 32-bit states of fp32 arithmetic with every product, sum, root and quotient rounded by itself, bit for bit, so
    that random rounding to bf16 decides alike.  (The 8-bit kernels' roots and quotients miss the nearest number about once in
    2^21 times: one unit of the last place of an fp32 parameter's move, below one of the parameter's own.)"""
    torch, pb = gpu
    f, n, b1, b2, lr, wd, step = np.float32, 1048576 + 77, 0.9, 0.999, 0.01, np.float64(np.float32(0.1)), 7
    ps, gs, states = _adamw_setup(torch, [n], param, "f32", bits, seed=19)
    p = ps[0].float().cpu().numpy()
    m, v = [x.float().cpu().numpy() for x in states[0][:2]]
    if bits == 8:
        at = lambda t: np.repeat(t.cpu().numpy(), 256)[:n]                                 # noqa: E731
        m, v = m * at(states[0][2]), np.square(v * at(states[0][3]))
    pb.AdamW(ps, state_bits=bits, states=states, betas=(b1, b2), weight_decay=wd, steps=step - 1).step(gs, lr)
    g = gs[0].cpu().numpy()
    m, v = m * f(b1) + g * f(1 - b1), v * f(b2) + (g * g) * f(1 - b2)
    move = m / (np.sqrt(v) * f(1 / np.sqrt(1 - b2 ** step)) + f(1e-8)) * f(lr / (1 - b1 ** step))
    p = p * f(1 - lr * wd) - move
    assert p.dtype == move.dtype == f
    if param == "bf16":
        p = ((p.view(np.uint32) + (osq.element_hash(n, step) & 0xFFFF).astype(np.uint32)) & np.uint32(0xFFFF0000)).view(f)
    got = ps[0].float().cpu().numpy()
    if bits == 32:
        assert (got == p).all() and (states[0][0].cpu().numpy() == m).all() and (states[0][1].cpu().numpy() == v).all()
    else:
        other = np.abs(got.astype(np.float64) - p) / (np.spacing(np.abs(p)) if param == "f32" else 2.0 ** -7 * np.abs(p) + 1e-30)
        assert (other > 0).sum() <= n * 2.0 ** -18 and other.max() <= 1


def test_adamw_not_finite(gpu):
    torch, pb = gpu
    p, g = torch.ones(600, device="cuda"), torch.ones(600, device="cuda")
    g[3], g[300] = float("nan"), float("inf")
    opt = pb.AdamW([p])
    opt.step([g], 0.1)
    bad = _np(p)
    assert np.isnan(bad[3]) and np.isnan(bad[300]) and np.isfinite(np.delete(bad, [3, 300])).all()
    p8 = torch.ones(600, device="cuda")
    opt = pb.AdamW([p8], state_bits=8)
    opt.step([g], 0.1)
    assert torch.equal(torch.isnan(p8), torch.isnan(p)) and np.isnan(_np(opt.states[0][0])[3])
    assert np.isfinite(_np(opt.states[0][0])[512:]).all() and np.isfinite(_np(opt.states[0][2])[2])


# -------------------------------------------------------------------------------------------------- all of them
def test_sequence_operators_on_another_stream(gpu):
    """Each call runs on the stream it is given: a long chain of work in front of it there is waited for, on a tensor made there."""
    torch, pb = gpu
    s, d, b, t = torch.cuda.Stream(), 512, 4, 300
    big = torch.randn(4096, 4096, device="cuda")
    x0, w = _randn(torch, 1, b * t, d), torch.ones(d, device="cuda")
    y_ref = torch.empty_like(x0)
    pb.rmsnorm_forward(x0, w, y_ref)
    q = {"u": x0.view(b, t, d), "gate": y_ref.view(b, t, d)}
    h_ref, ws = torch.empty_like(q["u"]), torch.empty(pb.recurrence_workspace_bytes(b, t, d), dtype=torch.uint8, device="cuda")
    pb.recurrence_forward(**q, y=h_ref, workspace=ws)
    p_ref = x0.clone()
    pb.AdamW([p_ref]).step([h_ref], 0.1)
    torch.cuda.synchronize()
    x, y, h, p = torch.zeros_like(x0), torch.zeros_like(x0), torch.zeros_like(h_ref), x0.clone()
    opt = pb.AdamW([p])
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(20):
            big = big @ big * 1e-3
        x.copy_(x0)
    pb.rmsnorm_forward(x, w, y, stream=s)
    pb.recurrence_forward(x.view(b, t, d), y.view(b, t, d), h, workspace=ws, stream=s)
    opt.step([h], 0.1, stream=s)
    s.synchronize()
    assert torch.equal(y, y_ref) and torch.equal(h, h_ref) and torch.equal(p, p_ref)


def test_sequence_operators_in_a_graph(gpu):
    """Captured once and replayed on new inputs, with eager work in between: the eager results."""
    torch, pb = gpu
    b, t, d = 2, 400, 96
    u, gate, x, w = _randn(torch, 1, b, t, d), _randn(torch, 2, b, t, d), _randn(torch, 3, b * t, d), torch.ones(d, device="cuda")
    y, n, dx, dw = torch.empty_like(u), torch.empty_like(x), torch.empty_like(x), torch.empty(d, device="cuda")
    ws, saved = (torch.empty(f(b, t, d), dtype=torch.uint8, device="cuda") for f in (pb.recurrence_workspace_bytes, pb.recurrence_saved_bytes))
    nws = torch.empty(pb.rmsnorm_workspace_bytes(b * t, d), dtype=torch.uint8, device="cuda")
    du, dg, db = torch.empty_like(u), torch.empty_like(u), torch.empty(d, device="cuda")

    def work(stream=None):
        pb.rmsnorm_forward(x, w, n, stream=stream)
        pb.recurrence_forward(u, n.view(b, t, d), y, saved=saved, workspace=ws, stream=stream)
        pb.recurrence_backward(u, n.view(b, t, d), gate, saved, du, dg, dbias=db, workspace=ws, stream=stream)
        pb.rmsnorm_backward(x, w, dg.view(b * t, d), dx, dw, nws, stream=stream)

    work()
    torch.cuda.synchronize()
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        work()
    for k in range(4):
        x.copy_(_randn(torch, 10 + k, b * t, d))
        u.copy_(_randn(torch, 20 + k, b, t, d))
        work()
        want = [v.clone() for v in (n, y, du, dg, db, dx, dw)]
        for v in (n, y, du, dg, db, dx, dw):
            v.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, (n, y, du, dg, db, dx, dw))), k


def test_binding_refusals(gpu):
    torch, pb = gpu
    x, w = torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda")
    u = torch.zeros(2, 4, 8, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    bad = [lambda: pb.rmsnorm_forward(x, w, torch.empty(4, 9, device="cuda")),
           lambda: pb.rmsnorm_forward(x, w.double(), torch.empty_like(x)),
           lambda: pb.rmsnorm_forward(x, w[:4], torch.empty_like(x)),
           lambda: pb.rmsnorm_forward(x, w, torch.empty_like(x), residual=x.bfloat16()),
           lambda: pb.rmsnorm_forward(x.t().contiguous().t(), w, torch.empty_like(x)),
           lambda: pb.rmsnorm_forward(x, w, torch.empty(4, 8, device="cuda", dtype=torch.float8_e4m3fn)),
           lambda: pb.rmsnorm_forward(x, w, torch.empty_like(x), scale=torch.empty(4, device="cuda")),
           lambda: pb.rmsnorm_forward(x, w.cpu(), torch.empty_like(x)),
           lambda: pb.rmsnorm_backward(x, w, x, torch.empty_like(x), torch.empty(8, device="cuda"), ws[:64]),
           lambda: pb.recurrence_forward(u, u[:1], torch.empty_like(u), workspace=ws),
           lambda: pb.recurrence_forward(u, u, torch.empty_like(u)),
           lambda: pb.recurrence_forward(u, u, torch.empty_like(u), lengths=torch.zeros(2, device="cuda"), workspace=ws),
           lambda: pb.recurrence_forward(u, u, torch.empty_like(u), state=torch.zeros(2, 9, device="cuda"), workspace=ws),
           lambda: pb.recurrence_forward(u, u, torch.empty_like(u), saved=ws[:8], workspace=ws),
           lambda: pb.recurrence_forward(u, u, u[:, :1].expand(2, 4, 8), workspace=ws),
           lambda: pb.recurrence_backward(u, u, u, ws, torch.empty_like(u), torch.empty_like(u), out_gate=u, workspace=ws),
           lambda: pb.recurrence_step(u[:, 0], u[:, 0], torch.zeros(2, 8, device="cuda", dtype=torch.bfloat16), torch.empty(2, 8, device="cuda")),
           lambda: pb.AdamW([x.half()]),
           lambda: pb.AdamW([x], states=[(x, x, x)]),
           lambda: pb.AdamW([x], copies=[x]),
           lambda: pb.AdamW([x], weight_decay=[0.1, 0.1]),
           lambda: pb.AdamW([x]).step([x, x], 0.1),
           lambda: pb.AdamW([x]).step([x[:2]], 0.1),
           lambda: pb.AdamW([x]).step([x.double()], 0.1),
           lambda: pb.AdamW([x]).step([x], float("nan"))]
    for i, f in enumerate(bad):
        with pytest.raises(pb.PbkdError):
            f()
            pytest.fail(f"call {i} was not refused")


def test_sequence_block_learns_and_answers_token_by_token(gpu):
    """The example's student: the local loss on a frozen block's labels falls to a tenth, and the answers token by token are those
    of the pass over all tokens, up to the roundings of bf16 (three products and a norm on the way: 2^-6 of the output's size)."""
    torch, pb = gpu
    from paper_2012_03096_amd import sequence
    losses, off = sequence.demo(d=64, batch=16, length=200, steps=400, lr=1e-2, report=399)
    assert losses[-1] < 0.1 * losses[0] and np.isfinite(losses).all()
    assert off < 2.0 ** -6
    block = sequence.SequenceBlock(64, seed=5)
    x = _randn(torch, 8, 2, 40, 64, dtype="bf16")
    r = _randn(torch, 9, 2, 40, 64, dtype="bf16")
    whole = block.forward(x, residual=r)
    state, pieces, at = torch.zeros(2, 64, device="cuda"), [], 0
    for n in (7, 1, 32):
        pieces.append(block.forward(x[:, at:at + n].contiguous(), residual=r[:, at:at + n].contiguous(), state=state, state_out=state))
        at += n
    assert float((torch.cat(pieces, 1).float() - whole.float()).norm() / whole.float().norm()) < 2.0 ** -6


# ------------------------------------------- calls beyond the last-level cache: the same bits as in smaller pieces
def test_rmsnorm_of_many_rows(gpu):
    torch, pb = gpu
    rows, d, cut = 60001, 1280, 23456
    x, r = (torch.randn(rows, d, device="cuda").bfloat16() for _ in range(2))
    w = 1.0 + _randn(torch, 3, d, scale=0.3)
    y, total, q, scale = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, d, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(rows, device="cuda")
    pb.rmsnorm_forward(x, w, y, residual=r, total=total)
    pb.rmsnorm_forward(x, w, q, residual=r, total=total, scale=scale)
    dx, dw = torch.empty_like(x), torch.empty(d, device="cuda")
    ws = torch.empty(pb.rmsnorm_workspace_bytes(rows, d), device="cuda", dtype=torch.uint8)
    pb.rmsnorm_backward(total, w, x, dx, dw, ws, dtotal=r)
    for part in (slice(0, 1000), slice(cut, cut + 1001), slice(rows - 7, rows)):
        a, b, e, f, g = torch.empty_like(x[part]), torch.empty_like(x[part]), torch.empty_like(q[part]), torch.empty_like(scale[part]), torch.empty_like(x[part])
        pb.rmsnorm_forward(x[part], w, a, residual=r[part], total=b)
        pb.rmsnorm_forward(x[part], w, e, residual=r[part], scale=f)
        pb.rmsnorm_backward(b, w, x[part], g, torch.empty_like(dw), ws, dtotal=r[part])
        assert torch.equal(a, y[part]) and torch.equal(b, total[part]) and torch.equal(e.view(torch.uint8), q[part].view(torch.uint8)) and torch.equal(f, scale[part])
        assert torch.equal(g, dx[part])
    ref = torch.zeros(d, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(ref)
    for i in range(0, rows, 8192):
        s, dy = total[i:i + 8192].double(), x[i:i + 8192].double()
        t = dy * s * torch.rsqrt((s * s).mean(1, keepdim=True) + 1e-6)
        ref, size = ref + t.sum(0), size + t.abs().sum(0)
    _within(_np(dw), ref.cpu().numpy(), ((64 + rows / 32) * E * size).cpu().numpy(), "dweight")


@pytest.mark.parametrize("gated", [True, False])
def test_recurrence_of_much_data(gpu, gated):
    torch, pb = gpu
    b, t, d = 6, 9000, 1280
    make = lambda: torch.randn(b, t, d, device="cuda").bfloat16()                                    # noqa: E731
    q = {"u": make(), "gate": make(), "out_gate": make() if gated else None, "bias": torch.rand(d, device="cuda") * 6, "state": torch.randn(b, d, device="cuda"),
         "lengths": torch.tensor([t, t - 1, 4000, 0, t, 1], dtype=torch.int32).cuda()}
    f = _forward(torch, pb, q)
    dy, dT = make(), torch.randn(b, d, device="cuda")
    g = _backward(torch, pb, q, f, dy, dT)
    for i in range(b):                               # one sequence a call stays below the cache's size
        one = {k: (v if k == "bias" else v[i:i + 1]) if v is not None else None for k, v in q.items()}
        f1 = _forward(torch, pb, one)
        g1 = _backward(torch, pb, one, f1, dy[i:i + 1], dT[i:i + 1])
        assert torch.equal(f1["y"], f["y"][i:i + 1]) and torch.equal(f1["state"], f["state"][i:i + 1])
        assert all(torch.equal(g1[k], g[k][i:i + 1]) for k in ("du", "dgate", "dstate") + (("dout_gate",) if gated else ()))


@pytest.mark.parametrize("bits,param,grad", [(32, "f32", "f32"), (8, "f32", "bf16"), (8, "bf16", "bf16")])
def test_adamw_of_many_elements(gpu, bits, param, grad):
    torch, pb = gpu
    n, cut = 40_000_123, 256 * 54321
    make = lambda kind, s: (torch.randn(n, device="cuda") * s).to(_type(torch, kind))                # noqa: E731
    p, g = make(param, 0.1), make(grad, 0.01)
    blocks = -(-n // 256)
    if bits == 32:
        st = [make("f32", 0.003), make("f32", 0.01).square()]
    else:
        st = [(torch.randn(n, device="cuda") * 60).clamp(-448, 448).to(torch.float8_e4m3fn), (torch.rand(n, device="cuda") * 448).to(torch.float8_e4m3fn),
              torch.rand(blocks, device="cuda") * 1e-4 + 1e-6, torch.rand(blocks, device="cuda") * 1e-4 + 1e-6]
    p2, st2 = p.clone(), [x.clone() for x in st]
    c, c2 = ([torch.empty(n, dtype=torch.bfloat16, device="cuda") for _ in range(2)] if param == "f32" else (None, None))
    pb.AdamW([p], state_bits=bits, states=[tuple(st)], copies=[c] if c is not None else None, weight_decay=0.1).step([g], 0.01)
    for a, e in ((0, cut), (cut, n)):                # the second piece with the elements' numbers of the whole
        for a2 in range(a, e, 256 * 30000):          # pieces below the cache's size
            e2 = min(e, a2 + 256 * 30000)
            piece = [x[a2:e2] for x in st2[:2]] + [x[a2 // 256:-(-e2 // 256)] for x in st2[2:]]
            opt = pb.AdamW([p2[a2:e2]], state_bits=bits, states=[tuple(piece)], copies=[c2[a2:e2]] if c2 is not None else None, weight_decay=0.1)
            opt._table["first"] = a2
            opt.step([g[a2:e2]], 0.01)
    assert torch.equal(p, p2) and all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(st, st2))
    assert c is None or torch.equal(c, c2)


# ------------------------------------------------------------------------------- tensors that move between steps
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_follows_its_tensors(gpu, bits):
    """A parameter's data, states and copies are exchanged between steps: the step works on the new ones, as an optimizer that always
    had them does, and writes nothing into the old ones."""
    torch, pb = gpu
    sizes = [300, 4097, 1]
    ps, gs, states = _adamw_setup(torch, sizes, "f32", "f32", bits)
    copies = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in sizes]
    opt = pb.AdamW(ps, state_bits=bits, states=states, copies=copies, weight_decay=0.1)
    ref = pb.AdamW([p.clone() for p in ps], state_bits=bits, states=[tuple(x.clone() for x in s) for s in states], weight_decay=0.1)
    raw = lambda t: t.view(torch.uint8).clone()                                            # noqa: E731
    for k in range(4):
        old = []
        if k == 1:
            old = [(p.data, raw(p.data)) for p in ps]
            for p in ps:
                p.data = p.data.clone()
        elif k == 2:
            old = [(x, raw(x)) for x in opt.states[1]] + [(c, raw(c)) for c in copies]
            opt.states[1] = tuple(x.clone() for x in opt.states[1])
            for i, n in enumerate(sizes):
                copies[i] = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
        elif k == 3:
            opt.params[0], copies[2] = ps[0].clone(), None
            old = [(ps[0], raw(ps[0]))]
        opt.step(gs, 0.01)
        ref.step(gs, 0.01)
        assert all(torch.equal(a, b) for a, b in zip(opt.params, ref.params)), k
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for s, t in zip(opt.states, ref.states) for a, b in zip(s, t)), k
        assert all(torch.equal(c, p.to(torch.bfloat16)) for c, p in zip(copies, opt.params) if c is not None), k
        assert all(torch.equal(t.view(torch.uint8), was) for t, was in old), k
    ps[1].data = torch.zeros(4096, device="cuda")
    with pytest.raises(pb.PbkdError):
        opt.step(gs, 0.01)
    assert opt.steps == 4


@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf"), 3.0])
@pytest.mark.parametrize("residual", [True, False])
def test_sequence_block_what_lies_behind_a_sequence_has_no_influence(gpu, junk, residual):
    """Steps on a padded batch: loss, gradients, weights and states are those of a batch that is padded with zeros, bit for bit."""
    torch, pb = gpu
    from paper_2012_03096_amd import sequence
    b, t, d = 5, 50, 64
    lengths = torch.tensor([t, 0, 1, 23, t - 1], dtype=torch.int32).cuda()
    gone = (torch.arange(t, device="cuda")[None] >= lengths[:, None])[:, :, None]
    x, r, target = (_randn(torch, k, b, t, d, dtype="bf16") for k in (1, 2, 3))
    seen = []
    for fill in (0.0, junk):
        block = sequence.SequenceBlock(d, seed=5)
        given = x.masked_fill(gone, fill)
        was = given.clone()
        loss = [block.distill_step(given, target.masked_fill(gone, fill), 1e-2, residual=r.masked_fill(gone, fill) if residual else None, lengths=lengths) for _ in range(3)]
        assert torch.equal(given.view(torch.int16), was.view(torch.int16))
        seen.append([float(v) for v in loss] + [v.clone() for v in (*block.grads, *block.params, *block.copies, *(s.view(torch.uint8) for st in block.optimizer.states for s in st))])
    assert np.isfinite(seen[0][:3]).all() and seen[0][:3] == seen[1][:3]
    assert all(torch.isfinite(v.float()).all() for v in seen[1][3:15]) and all(torch.equal(a, c) for a, c in zip(seen[0][3:], seen[1][3:]))


# ------------------------------------------------------------------------ 8-bit states of what is not finite
@pytest.mark.parametrize("bits", [0x7FC00000, 0x7F800001, 0x7FFF0000, 0x7FFFFFFF, 0xFFC00000, 0xFFFF0000, 0xFFFFFFFF])
def test_adamw_8_bits_of_any_nan(gpu, bits):
    """A gradient of NaN, whatever its sign and mantissa, leaves NaN in both states and the parameter, by any random number."""
    torch, pb = gpu
    g = torch.from_numpy(np.full(256, bits, np.uint32).view(np.float32)).cuda()
    for seed in range(8):
        p = torch.ones(256, device="cuda")
        opt = pb.AdamW([p], state_bits=8)
        opt.step([g], 0.1, seed=seed)
        assert torch.isnan(opt.states[0][0].float()).all() and torch.isnan(opt.states[0][1].float()).all() and torch.isnan(p).all(), seed


@pytest.mark.parametrize("bad,param,grad", [(b, p, g) for b in (float("inf"), -float("inf"), float("nan"), 1e20)
                                            for p, g in (("f32", "f32"), ("f32", "bf16"), ("bf16", "f16")) if b != 1e20 or g != "f16"])
def test_adamw_8_bits_beside_what_is_not_finite(gpu, bad, param, grad):
    """One gradient of a block is infinite, NaN or has a square past fp32's range: its own element is lost (the last one's second moment
    only), the others' parameters, codes and scales are those beside a zero in its place, in this step and the next."""
    torch, pb = gpu
    n, at = 600, [3, 300, 599]

    def run(value):
        p, g, g2 = (_randn(torch, k, n, scale=0.1) for k in (1, 2, 3))
        p[at], g[at], g2[at] = 0.0, value, 0.0
        p, g, g2 = p.to(_type(torch, param)), g.to(_type(torch, grad)), g2.to(_type(torch, grad))
        opt = pb.AdamW([p], state_bits=8)
        out = []
        for v in (g, g2):
            opt.step([v], 0.01)
            out.append([x.clone() for x in (p, *opt.states[0])])
        return out

    keep = np.delete(np.arange(n), at)
    for k, (a, z) in enumerate(zip(run(bad), run(0.0))):
        for j, name in enumerate(("param", "m", "v", "m_scale", "v_scale")):
            if bad == 1e20 and name in ("m", "m_scale"):
                continue                           # a finite first moment counts for its scale
            x, y = _np(a[j]), _np(z[j])
            if name.endswith("scale"):
                assert (x == y).all() and np.isfinite(x).all(), (k, name)
            else:
                assert name == "param" and bad == 1e20 and k == 1 or (x[keep] == y[keep]).all(), (k, name)
                assert np.isfinite(x[keep]).all(), (k, name)
                lost = np.isnan(x[at])
                assert lost.all() if name == "v" or bad != 1e20 or name == "param" and k == 1 else True, (k, name)


def test_adamw_8_bits_of_the_largest_numbers(gpu):
    """First moments around fp32's largest number, where the reciprocal of their maximum is below its normal range."""
    torch, pb = gpu
    f = torch.linspace(0.0, 1.0, 256, device="cuda") * 3.4e38
    p = torch.zeros(256, device="cuda")
    opt = pb.AdamW([p], state_bits=8, betas=(0.0, 0.999))
    opt.step([f], 0.0)
    x = _np(f) / _np(f).max() * 448.0
    _within(_np(opt.states[0][0]), x, 0.5 * osq.e4m3_spacing(x) * (1 + 1e-3), "codes")
    _within(_np(opt.states[0][2]), [_np(f).max() / 448.0], 4 * E * 1e36, "scale")


@pytest.mark.parametrize("param", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [1e-8, 0.0])
def test_adamw_8_bits_move_at_the_ends_of_the_range(gpu, param, eps):
    """The first step from nothing is the same with states in 8 as in 32 bits, also where the quotient's denominator is infinite
    (a gradient whose square passes fp32's range: no move) or zero, and where the gradient is."""
    torch, pb = gpu
    g = _randn(torch, 1, 512)
    g[:8] = torch.tensor([1e20, -1e20, 3.4e38, 0.0, -0.0, 1e-30, float("inf"), float("nan")])
    p, q = (_randn(torch, 2, 512, dtype=param) for _ in range(2))
    pb.AdamW([p], weight_decay=0.1, eps=eps).step([g], 0.01)
    pb.AdamW([q], weight_decay=0.1, eps=eps, state_bits=8).step([g], 0.01)
    a, b = _np(p), _np(q)
    assert (np.isnan(a[:8]) == np.isnan(b[:8])).all() and (np.isnan(a[:8]) == [False, False, False, eps == 0.0, eps == 0.0, False, True, True]).all(), (a[:8], b[:8])
    _within(b, a, np.abs(a) * (2 * E if param == "f32" else 2.0 ** -7) + 0.01 * 4 * E, "parameters")


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_is_refused_in_a_capture(gpu, bits):
    """A replayed step would not count on.  The refusal leaves the capture, and the optimizer, as they were."""
    torch, pb = gpu
    x, w = _randn(torch, 1, 4, 64), torch.ones(64, device="cuda")
    y, g, p = torch.zeros_like(x), _randn(torch, 2, 300), _randn(torch, 3, 300)
    opt, ref = (pb.AdamW([q], state_bits=bits) for q in (p, p.clone()))
    pb.rmsnorm_forward(x, w, y)
    want, before = y.clone(), p.clone()
    torch.cuda.synchronize()
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        with pytest.raises(pb.PbkdError) as refused:
            opt.step([g], 0.1)
        pb.rmsnorm_forward(x, w, y)
    assert refused.value.status == pb.EUNSUPPORTED and opt.steps == 0
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(p, before)
    for _ in range(2):
        opt.step([g], 0.1)
        ref.step([g], 0.1, stream=s)
        torch.cuda.synchronize()
    assert opt.steps == 2 and torch.equal(p, ref.params[0])


def test_sequence_block_keeps_no_more_than_the_largest_batch_takes(gpu):
    """Batches of many sizes, in any order, take no more memory than the largest did, and answer as a new block does."""
    torch, pb = gpu
    from paper_2012_03096_amd import sequence
    block = sequence.SequenceBlock(64, seed=5)
    x = _randn(torch, 1, 6, 700, 64, dtype="bf16")
    target, steps = torch.zeros_like(x), [(6, 700, True), (6, 700, False)] + [(b, t, k % 3 == 0) for k, (b, t) in enumerate((1 + k % 6, 1 + 37 * k % 699) for k in range(40))]
    most = None
    for b, t, training in steps:
        cut = x[:b, :t].contiguous()
        if training:
            block.distill_step(cut, target[:b, :t].contiguous(), 0.0)
        out = block.forward(cut)
        if most is not None and b * t < 500:
            assert torch.equal(out, sequence.SequenceBlock(64, seed=5).forward(cut)), (b, t)
        torch.cuda.synchronize()
        if t == 700:
            del out, cut
            most = torch.cuda.memory_allocated()
            continue
        del out, cut
        assert torch.cuda.memory_allocated() <= most, (b, t)


def test_sequence_block_writes_no_sum_that_nobody_reads(gpu, monkeypatch):
    torch, pb = gpu
    from paper_2012_03096_amd import sequence
    seen = []
    norm = pb.rmsnorm_forward
    monkeypatch.setattr(pb, "rmsnorm_forward", lambda *a, **kw: (seen.append(kw.get("total")), norm(*a, **kw))[1])
    block, x = sequence.SequenceBlock(64, seed=5), _randn(torch, 1, 2, 40, 64, dtype="bf16")
    block.forward(x)
    block.forward(x, residual=x)
    block.distill_step(x, x, 1e-3)
    assert seen == [None, None, None]
    block.distill_step(x, x, 1e-3, residual=x)
    assert seen[3] is not None and torch.equal(seen[3], x + x)


def test_sequence_blocks_in_a_chain_with_a_residual_stream(gpu):
    """Two blocks behind each other: the stream is the sum of all that went before, and the answers token by token, residual and all, are
    those of the pass over all tokens (up to the roundings of bf16, 2^-6 of the output's size)."""
    torch, pb = gpu
    from paper_2012_03096_amd import sequence
    b, t, d = 3, 40, 64
    one, two = sequence.SequenceBlock(d, seed=5), sequence.SequenceBlock(d, seed=6)
    x, r = _randn(torch, 8, b, t, d, dtype="bf16"), _randn(torch, 9, b, t, d, dtype="bf16")
    s = torch.empty_like(x)
    first = one.forward(x, residual=r, total=s)
    assert torch.equal(first, one.forward(x, residual=r)) and torch.equal(s, x + r)
    was = s.clone()
    second = two.forward(first, residual=s, total=s)                      # the stream in place
    assert torch.equal(s, first + was) and torch.equal(second, two.forward(first, residual=was))
    alone = torch.empty_like(x)
    one.forward(x, total=alone)
    assert torch.equal(alone, x)
    states, out, stream = [torch.zeros(b, d, device="cuda") for _ in range(2)], torch.empty_like(x), torch.empty_like(x)
    for i in range(t):
        a = torch.empty(b, d, dtype=x.dtype, device="cuda")
        h = one.step(x[:, i].contiguous(), states[0], residual=r[:, i].contiguous(), total=a)
        assert torch.equal(a, was[:, i])
        out[:, i] = two.step(h, states[1], residual=a, total=a)
        stream[:, i] = a
    for got, want in ((out, second), (stream, s)):
        assert float((got.float() - want.float()).norm() / want.float().norm()) < 2.0 ** -6


# ------------------------------------------------------------------------------------------- paths by size and count
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("dtype,b,t,d", [("bf16", 9, 4163, 2048), ("f16", 9, 4163, 2048), ("f32", 4, 4321, 1312)])
def test_recurrence_of_much_data_in_many_chains(gpu, dtype, b, t, d, gated):
    """More than the last-level cache holds in tiles of four waves: 16-bit types in more than 128 chains, and fp32, its last slice half a
    one.  The same bits as one sequence a call, which stays below the cache's size and takes the same tiles."""
    torch, pb = gpu
    size = 4 if dtype == "f32" else 2
    assert b * t * d * size * 3 > 256e6 > t * d * size * 7 and d * size % 128 == 0 and (dtype == "f32" or b * -(-d // 64) > 128) and t < 8192
    kind = _type(torch, dtype)
    make = lambda: torch.randn(b, t, d, device="cuda").to(kind)                                     # noqa: E731
    q = {"u": make(), "gate": make(), "out_gate": make() if gated else None, "bias": torch.rand(d, device="cuda") * 6, "state": torch.randn(b, d, device="cuda"),
         "lengths": torch.tensor([t, 0, 1, t // 2, t - 1, 129, 64, 2049, t][:b], dtype=torch.int32).cuda()}
    print("recurrence of much data", dtype, b, t, d, gated, flush=True)
    f = _forward(torch, pb, q)
    dy, dT = make(), torch.randn(b, d, device="cuda")
    g = _backward(torch, pb, q, f, dy, dT)
    part = torch.zeros(d, dtype=torch.float64, device="cuda")
    for i in range(b):
        one = {k: (v if k == "bias" else v[i:i + 1]) if v is not None else None for k, v in q.items()}
        f1 = _forward(torch, pb, one)
        g1 = _backward(torch, pb, one, f1, dy[i:i + 1], dT[i:i + 1])
        assert torch.equal(f1["y"], f["y"][i:i + 1]) and torch.equal(f1["state"], f["state"][i:i + 1]), i
        assert all(torch.equal(g1[k], g[k][i:i + 1]) for k in ("du", "dgate", "dstate") + (("dout_gate",) if gated else ())), i
        part += g1["dbias"].double()
    # each is a sum of at most 64 tokens in a thread, then of 4163 / 64 rows a sequence
    size = g["dgate"].double().abs().sum((0, 1)) * (1 + 2 * HALF[dtype])
    _within(_np(g["dbias"]), part.cpu().numpy(), (2 * (64 + b * t / 64) * E * size).cpu().numpy(), "dbias")


@pytest.mark.parametrize("bits,param,grad", [(8, "f32", "f32"), (8, "bf16", "bf16"), (32, "f32", "bf16"), (32, "bf16", "f32")])
def test_adamw_of_more_tensors_than_one_launch_takes(gpu, bits, param, grad):
    """A hundred tensors, some without elements, some without gradients, from nothing and under way: every parameter, state and scale, and
    the random numbers by the elements' places across the launches."""
    import types
    torch, pb = gpu
    sizes = [(37 * i) % 700 for i in range(100)]
    absent = [i % 9 == 4 for i in range(100)]
    assert sum(1 for n, a in zip(sizes, absent) if n and not a) > 80 and 0 in sizes
    for start in (0, 41):
        ps, gs, states = _adamw_setup(torch, sizes, param, grad, bits)
        decays = [0.1 if i % 2 else 0.0 for i in range(100)]
        opt = pb.AdamW(ps, state_bits=bits, states=states if start else None, weight_decay=decays, steps=start)
        for _ in range(2):
            before = [(p.clone(), tuple(x.clone() for x in s)) for p, s in zip(ps, opt.states)]
            opt.step([None if a else g for a, g in zip(absent, gs)], 0.01)
            torch.cuda.synchronize()
            for i in range(100):
                if absent[i]:
                    assert torch.equal(before[i][0], ps[i]) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before[i][1], opt.states[i]))
            # what had no gradient stands in the check as zeros that stay zeros, so that the elements behind it keep their numbers
            zero = lambda t: torch.zeros_like(t.view(torch.uint8)).view(t.dtype)                    # noqa: E731
            tiny = lambda s: tuple(zero(x) if k < 2 else torch.full_like(x, osq.TINY / 448.0) for k, x in enumerate(s))          # noqa: E731
            told = types.SimpleNamespace(steps=opt.steps, params=[zero(p) if a else p for a, p in zip(absent, ps)],
                                         states=[tiny(s) if a else s for a, s in zip(absent, opt.states)])
            was = [(zero(p), tiny(s)) if a else (p, s) for a, (p, s) in zip(absent, before)]
            _check_adamw(torch, was, [zero(g) if a else g for a, g in zip(absent, gs)], told, [np.float64(np.float32(x)) for x in decays], 0.01, bits, param)
