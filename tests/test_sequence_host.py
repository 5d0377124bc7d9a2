"""CPU-only checks of the sequence operators: the oracle's gradients against differences of its forward pass, its e4m3 table, and what
the library and the binding refuse.  Every refused call here returns before any device work."""
import ctypes

import numpy as np
import pytest

from oracle import sequence as osq
from paper_2012_03096_amd import binding as pb


def _difference(f, x, i, h=1e-5):
    a, b = x.copy(), x.copy()
    a.flat[i] += h
    b.flat[i] -= h
    return (f(a) - f(b)) / (2 * h)


@pytest.mark.parametrize("residual", [False, True])
def test_oracle_norm_gradients_match_differences(residual):
    rng = np.random.default_rng(1)
    x, r, w = rng.standard_normal((3, 5)), rng.standard_normal((3, 5)), rng.standard_normal(5)
    dy, ds = rng.standard_normal((3, 5)), rng.standard_normal((3, 5))
    res = r if residual else None

    def loss(x_, w_):
        y, s, _ = osq.rmsnorm(x_, w_, res)
        return (y * dy).sum() + ((s * ds).sum() if residual else 0.0)

    _, s, _ = osq.rmsnorm(x, w, res)
    dx, dw, _, _ = osq.rmsnorm_backward(s, w, dy, ds if residual else None)
    for i in range(x.size):
        assert abs(dx.flat[i] - _difference(lambda v: loss(v, w), x, i)) < 1e-8
    for i in range(w.size):
        assert abs(dw.flat[i] - _difference(lambda v: loss(x, v), w, i)) < 1e-8


@pytest.mark.parametrize("gated", [False, True])
def test_oracle_recurrence_gradients_match_differences(gated):
    rng = np.random.default_rng(2)
    b, t, d = 3, 6, 2
    q = {k: rng.standard_normal((b, t, d)) for k in ("u", "gate", "out_gate", "dy")}
    bias, state, dT = rng.standard_normal(d), rng.standard_normal((b, d)), rng.standard_normal((b, d))
    lengths = np.array([6, 0, 4])
    if not gated:
        q["out_gate"] = None

    def loss(**kw):
        a = dict(u=q["u"], gate=q["gate"], out_gate=q["out_gate"], bias=bias, state=state)
        a.update(kw)
        f = osq.recurrence(a["u"], a["gate"], a["out_gate"], a["bias"], lengths, a["state"])
        return (f["y"] * q["dy"]).sum() + (f["state"] * dT).sum()

    g = osq.recurrence_backward(q["u"], q["gate"], q["dy"], q["out_gate"], bias, lengths, state, dT)
    pairs = [("u", q["u"], "du"), ("gate", q["gate"], "dgate"), ("bias", bias, "dbias"), ("state", state, "dstate")]
    pairs += [("out_gate", q["out_gate"], "dout_gate")] if gated else []
    for name, x, out in pairs:
        for i in range(x.size):
            assert abs(g[out].flat[i] - _difference(lambda v: loss(**{name: v}), x, i)) < 1e-8, (name, i)


def test_oracle_adamw_is_the_gradient_scaled_for_the_first_step():
    p, g = np.array([1.0, -2.0, 0.5]), np.array([0.1, -3.0, 0.0])
    q, m, v = osq.adamw(p, g, np.zeros(3), np.zeros(3), 0.01, 1, weight_decay=0.1)
    assert np.allclose(q, p * (1 - 0.001) - 0.01 * np.sign(g), atol=1e-8)     # m/(1-b1) = g, sqrt(v/(1-b2)) = |g|
    assert np.allclose(m, 0.1 * g) and np.allclose(v, 0.001 * g * g)


def test_oracle_e4m3_table():
    torch = pytest.importorskip("torch")
    got = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(osq.e4m3_values(), got, equal_nan=True)


def _desc(fmt, **at):
    """Bytes of a descriptor with the given fields (by position) set."""
    n = len(fmt.unpack(bytes(fmt.size)))
    v = [0] * n
    for i, x in at.items():
        v[int(i[1:])] = x
    return fmt.pack(*v)


def test_library_refuses_bad_norms():
    L = pb.lib()
    f = lambda **k: L.pbkd_rmsnorm_forward(_desc(pb._RMSNORM, **k), None)                                                       # noqa: E731
    assert L.pbkd_rmsnorm_forward(None, None) == pb.EINVAL
    ok = dict(_0=4, _1=8, _2=pb.F32, _3=pb.F32, _4=1e-6, _5=64, _7=64, _9=64, _11=8, _14=8)
    assert f(**{**ok, "_0": -1}) == pb.ESHAPE
    assert f(**{**ok, "_1": 0}) == pb.ESHAPE
    assert f(**{**ok, "_1": 16385}) == pb.EUNSUPPORTED
    assert f(**{**ok, "_2": pb.E4M3}) == pb.EINVAL
    assert f(**{**ok, "_3": pb.BF16}) == pb.EINVAL
    assert f(**{**ok, "_4": -1.0}) == pb.EINVAL
    assert f(**{**ok, "_4": float("nan")}) == pb.EINVAL
    assert f(**{**ok, "_5": 0}) == pb.EINVAL
    assert f(**{**ok, "_5": 66}) == pb.EINVAL and "aligned" in pb.last_error()
    assert f(**{**ok, "_3": pb.E4M3}) == pb.EINVAL                                  # no scale
    assert f(**{**ok, "_14": 7}) == pb.ESHAPE                                       # rows of y overlap
    assert f(**{**ok, "_11": -8}) == pb.EINVAL
    assert f(**{**ok, "_8": 64, "_13": 8}) == pb.EINVAL                             # total and y the same
    assert f(**{**ok, "_0": 0}) == pb.OK                                            # no rows: nothing to do
    b = lambda **k: L.pbkd_rmsnorm_backward(_desc(pb._RMSNORM_GRAD, **k), None)     # noqa: E731
    assert L.pbkd_rmsnorm_backward(None, None) == pb.EINVAL
    need = L.pbkd_rmsnorm_workspace_bytes(4, 8)
    assert need > 0 and L.pbkd_rmsnorm_workspace_bytes(4, 0) == 0 and L.pbkd_rmsnorm_workspace_bytes(-1, 8) == 0 and L.pbkd_rmsnorm_workspace_bytes(1, 16385) == 0
    ok = dict(_0=4, _1=8, _2=pb.F32, _3=1e-6, _4=64, _5=64, _7=64, _8=128, _9=64, _10=8, _11=8, _13=8, _14=256, _15=need)
    assert b(**{**ok, "_15": need - 1}) == pb.ENOMEM
    assert b(**{**ok, "_14": 128}) == pb.ENOMEM
    assert b(**{**ok, "_14": 0}) == pb.ENOMEM
    assert b(**{**ok, "_9": 0}) == pb.EINVAL
    assert b(**{**ok, "_8": 0}) == pb.EINVAL
    assert b(**{**ok, "_13": 7}) == pb.ESHAPE
    assert b(**{**ok, "_2": 7}) == pb.EINVAL


def test_library_refuses_bad_recurrences():
    L = pb.lib()
    need, keep = L.pbkd_recurrence_workspace_bytes(2, 40, 8), L.pbkd_recurrence_saved_bytes(2, 40, 8)
    assert need > 0 and keep > 0
    for bad in ((-1, 4, 8), (2, -1, 8), (2, 4, 0), (1 << 30, 4, 4), (2, 1 << 31, 8), (1 << 23, 4, 1)):
        assert L.pbkd_recurrence_workspace_bytes(*bad) == 0 and L.pbkd_recurrence_saved_bytes(*bad) == 0
    f = lambda **k: L.pbkd_recurrence_forward(_desc(pb._RECURRENCE, **k), None)     # noqa: E731
    s = lambda **k: L.pbkd_recurrence_step(_desc(pb._RECURRENCE, **k), None)        # noqa: E731
    assert L.pbkd_recurrence_forward(None, None) == pb.EINVAL and L.pbkd_recurrence_step(None, None) == pb.EINVAL
    # batch, channels, len, dtype, u, gate, out_gate, bias, lengths, state, state_out, y, (batch, token) strides of u, gate, out_gate, y, ...
    ok = dict(_0=2, _1=8, _2=40, _3=pb.F32, _4=64, _5=64, _11=64, _12=320, _13=8, _14=320, _15=8, _18=320, _19=8, _22=256, _23=need)
    assert f(**{**ok, "_0": -1}) == pb.ESHAPE
    assert f(**{**ok, "_1": 0}) == pb.ESHAPE
    assert f(**{**ok, "_2": -1}) == pb.ESHAPE
    assert f(**{**ok, "_2": 1 << 31}) == pb.EUNSUPPORTED
    assert f(**{**ok, "_3": pb.E4M3}) == pb.EINVAL
    assert f(**{**ok, "_4": 0}) == pb.EINVAL
    assert f(**{**ok, "_5": 62}) == pb.EINVAL
    assert f(**{**ok, "_13": -8}) == pb.EINVAL
    assert f(**{**ok, "_19": 7}) == pb.ESHAPE
    assert f(**{**ok, "_18": 300}) == pb.ESHAPE
    assert f(**{**ok, "_20": 64, "_21": keep - 1}) == pb.ENOMEM
    assert f(**{**ok, "_22": 0}) == pb.ENOMEM
    assert f(**{**ok, "_23": need - 1}) == pb.ENOMEM
    assert f(**{**ok, "_0": 0}) == pb.OK
    assert s(**{**ok, "_2": 1}) == pb.EINVAL and "state" in pb.last_error()
    b = lambda **k: L.pbkd_recurrence_backward(_desc(pb._RECURRENCE_GRAD, **k), None)   # noqa: E731
    assert L.pbkd_recurrence_backward(None, None) == pb.EINVAL
    # ..., u, gate, out_gate, dy, bias, lengths, dstate_out, du, dgate, dout_gate, dbias, dstate, strides of u gate out_gate dy du dgate dout_gate, saved, workspace
    ok = dict(_0=2, _1=8, _2=40, _3=pb.F32, _4=64, _5=64, _7=64, _11=64, _12=64, _16=320, _17=8, _18=320, _19=8, _22=320, _23=8, _24=320, _25=8, _26=320, _27=8,
              _30=64, _31=keep, _32=256, _33=need)
    assert b(**{**ok, "_30": 0}) == pb.EINVAL
    assert b(**{**ok, "_6": 64}) == pb.EINVAL and "together" in pb.last_error()
    assert b(**{**ok, "_31": keep - 1}) == pb.ENOMEM
    assert b(**{**ok, "_33": need - 1}) == pb.ENOMEM
    assert b(**{**ok, "_25": 7}) == pb.ESHAPE
    assert b(**{**ok, "_7": 0}) == pb.EINVAL
    assert b(**{**ok, "_12": 0}) == pb.EINVAL
    assert b(**{**ok, "_3": 9}) == pb.EINVAL


def test_library_refuses_bad_adamw_steps():
    L = pb.lib()

    def call(n=1, args=None, elements=100, **fields):
        t = np.zeros(1, pb._ADAMW_TENSOR)
        t["n"], t["param"], t["grad"], t["m"], t["v"] = elements, 64, 64, 64, 64
        for k, x in fields.items():
            t[k] = x
        a = dict(lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, scale=1.0, step=1, bits=32, seed=0)
        a.update(args or {})
        return L.pbkd_adamw_step(n, t.ctypes.data_as(ctypes.c_void_p), pb._ADAMW_ARGS.pack(*a.values()), None)

    assert call(n=-1) == pb.EINVAL
    assert L.pbkd_adamw_step(1, None, bytes(pb._ADAMW_ARGS.size), None) == pb.EINVAL
    assert L.pbkd_adamw_step(0, None, None, None) == pb.EINVAL
    for args in (dict(bits=16), dict(step=0), dict(b1=1.0), dict(b2=-0.1), dict(b1=float("nan")), dict(eps=-1.0), dict(lr=float("nan")), dict(scale=float("nan"))):
        assert call(args=args) == pb.EINVAL, args
    assert call(n=0) == pb.OK and call(elements=0) == pb.OK
    assert call(elements=-1) == pb.ESHAPE and call(elements=(1 << 34) + 1) == pb.EUNSUPPORTED
    for fields in (dict(param=0), dict(grad=0), dict(m=0), dict(v=66), dict(param=66), dict(grad=63), dict(param_dtype=pb.F16), dict(grad_dtype=5), dict(copy=63),
                   dict(copy=64, param_dtype=pb.BF16), dict(weight_decay=-1.0), dict(weight_decay=np.nan)):
        assert call(**fields) == pb.EINVAL, fields
    assert call(args=dict(bits=8)) == pb.EINVAL                                     # no scales


def test_binding_refuses_tensors_that_are_not_on_a_gpu():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 4, 8)
    with pytest.raises(pb.PbkdError):
        pb.rmsnorm_forward(x, torch.ones(8), torch.empty_like(x))
    with pytest.raises(pb.PbkdError):
        pb.recurrence_forward(x, x, torch.empty_like(x))
    with pytest.raises(pb.PbkdError):
        pb.recurrence_step(x[:, 0], x[:, 0], torch.zeros(2, 8), torch.empty(2, 8))
    with pytest.raises(pb.PbkdError):
        pb.AdamW([x])
    with pytest.raises(pb.PbkdError):
        pb.rmsnorm_forward(x.double(), torch.ones(8), x)
    with pytest.raises(pb.PbkdError):
        pb.AdamW([], state_bits=4)


class _Recorder:
    """Stands in for the library: keeps the table of each step that reaches it (host tensors: nothing may run on their addresses)."""

    def __init__(self):
        self.tables = []

    def pbkd_adamw_step(self, n, table, args, stream):
        self.tables.append(np.frombuffer((ctypes.c_char * (n * pb._ADAMW_TENSOR.itemsize)).from_address(table), pb._ADAMW_TENSOR).copy())
        return 0


@pytest.fixture
def recorded(monkeypatch):
    torch = pytest.importorskip("torch")
    pb._types()
    seen = _Recorder()
    monkeypatch.setattr(pb, "_lib", seen)
    monkeypatch.setattr(pb, "_current_device", lambda: -1)
    monkeypatch.setattr(pb, "_first", lambda t, name: (seen, pb._CODES.get(t.dtype), t.dtype, t.shape, -1))
    return torch, seen


def _adamw_on_host(torch, bits, copies=True):
    params = [torch.zeros(6, 50), torch.zeros(300)]
    kind = torch.float32 if bits == 32 else torch.float8_e4m3fn
    states = [tuple([torch.zeros(300).to(kind), torch.zeros(300).to(kind)] + ([] if bits == 32 else [torch.zeros(2), torch.zeros(2)])) for _ in params]
    return pb.AdamW(params, state_bits=bits, states=states, copies=[p.bfloat16() for p in params] if copies else None)


def _addresses(opt):
    names = ("m", "v", "m_scale", "v_scale")[:len(opt.states[0])]
    out = {"param": [p.data_ptr() for p in opt.params], **{k: [s[i].data_ptr() for s in opt.states] for i, k in enumerate(names)}}
    if opt.copies is not None:
        out["copy"] = [c.data_ptr() if c is not None else 0 for c in opt.copies]
    return out


class _Stream:
    cuda_stream = 0


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_goes_to_where_its_tensors_are(recorded, bits):
    """A parameter's data, a state or a copy that was exchanged for another tensor of the same type and size: the next step takes the
    new one (the old one's memory may belong to somebody else by then)."""
    torch, seen = recorded
    opt = _adamw_on_host(torch, bits)
    grads = [torch.zeros(6, 50), torch.zeros(300)]

    def step():
        opt.step(grads, 0.1, stream=_Stream)
        table, want = seen.tables[-1], _addresses(opt)
        for k, v in want.items():
            assert table[k].tolist() == v, k
        assert table["n"].tolist() == [300, 300]

    step()
    opt.params[0].data = torch.ones(6, 50)
    step()
    opt.params[1] = torch.ones(300)
    step()
    opt.states[1] = tuple(x.clone() for x in opt.states[1])
    step()
    opt.copies[0] = torch.zeros(6, 50, dtype=torch.bfloat16)
    step()
    opt.copies[1] = None
    step()
    opt.params[1].set_(torch.zeros(1000), 700, (300,))
    step()


@pytest.mark.parametrize("change", ["shorter", "shorter at its place", "longer", "type", "layout", "copy", "state", "state type", "count"])
def test_adamw_refuses_tensors_that_are_not_what_they_were(recorded, change):
    torch, seen = recorded
    opt = _adamw_on_host(torch, 32)
    grads = [torch.zeros(6, 50), torch.zeros(300)]
    opt.step(grads, 0.1, stream=_Stream)
    p = opt.params[0]
    if change == "shorter":
        p.data = torch.zeros(5, 50)
    elif change == "shorter at its place":
        p.data = p.data[:5]
        grads[0] = torch.zeros(5, 50)
    elif change == "longer":
        p.resize_(7, 50)
    elif change == "type":
        p.data = p.data.bfloat16()
    elif change == "layout":
        p.data = p.data.view(50, 6).t()
    elif change == "copy":
        opt.copies[0] = torch.zeros(6, 49, dtype=torch.bfloat16)
    elif change == "state":
        opt.states[0] = (torch.zeros(299), opt.states[0][1])
    elif change == "state type":
        opt.states[0] = (torch.zeros(300, dtype=torch.float64), opt.states[0][1])
    else:
        opt.params.append(torch.zeros(3))
    with pytest.raises(pb.PbkdError):
        opt.step(grads, 0.1, stream=_Stream)
    assert len(seen.tables) == 1 and opt.steps == 1


def test_adamw_tells_the_library_each_steps_gradients(recorded):
    """Their addresses, types and elements, step by step, as types change and gradients come and go."""
    torch, seen = recorded
    opt = _adamw_on_host(torch, 32, copies=False)
    a, b, h = torch.zeros(6, 50), torch.zeros(300), torch.zeros(300, dtype=torch.bfloat16)
    for grads in ([a, b], [a, h], (a, h), [None, h], [a, None], [None, None], [a, b], [a.half(), b.clone()], [a.half(), b]):
        opt.step(grads, 0.1, stream=_Stream)
        table = seen.tables[-1]
        assert table["n"].tolist() == [0 if g is None else 300 for g in grads]
        assert table["grad"].tolist() == [0 if g is None else g.data_ptr() for g in grads]
        assert table["grad_dtype"].tolist() == [pb.F32 if g is None else pb._CODES[g.dtype] for g in grads]
    for grads in ([a, b.double()], [a[:5], b], [a.t(), b], [a], [None, b.double()], [None, b[:299]]):
        with pytest.raises(pb.PbkdError):
            opt.step(grads, 0.1, stream=_Stream)
    assert opt.steps == 9 == len(seen.tables)
    opt.step([a, b], 0.1, stream=_Stream)
    assert seen.tables[-1]["n"].tolist() == [300, 300] and seen.tables[-1]["grad_dtype"].tolist() == [pb.F32, pb.F32]
