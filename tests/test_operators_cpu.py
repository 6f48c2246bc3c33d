"""What needs no GPU of the operators of gated pre-norm blocks: every refusal (each comes before anything is enqueued), workspace sizes,
the frequency tables, and the 64-bit statements themselves against differences."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import operators_oracle as P
from paper_2505_04802_amd import binding as B

p = 1 << 20                     # an address that is never followed: aligned to everything the library asks for
F32, BF16, E4M3 = B.RESLIM_F32, B.RESLIM_BF16, B.RESLIM_E4M3
EINVAL, ESHAPE, EWS, OK = B.RESLIM_EINVAL, B.RESLIM_ESHAPE, B.RESLIM_EWORKSPACE, B.RESLIM_OK


def _norm(x=p, delta=p, gamma=p, eps=1e-6, rows=4, D=64, stream=F32, act=BF16, yt=BF16, sum_=p, y=p, scale=None):
    return B.load().reslim_rmsnorm_fwd(x, delta, gamma, eps, rows, D, stream, act, yt, sum_, y, scale, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), EINVAL), (dict(gamma=None), EINVAL), (dict(y=None), EINVAL), (dict(rows=-1), ESHAPE), (dict(rows=1 << 31), ESHAPE),
    (dict(D=0), ESHAPE), (dict(D=16385), ESHAPE), (dict(eps=-1.0), EINVAL), (dict(eps=math.nan), EINVAL), (dict(eps=math.inf), EINVAL),
    (dict(stream=BF16, act=F32), EINVAL), (dict(stream=E4M3), EINVAL), (dict(act=E4M3, yt=E4M3), EINVAL), (dict(stream=7), EINVAL),
    (dict(yt=F32), EINVAL), (dict(yt=E4M3), EINVAL), (dict(scale=p), EINVAL), (dict(x=p + 2), EINVAL), (dict(delta=p + 1), EINVAL),
    (dict(sum_=p + 1), EINVAL), (dict(gamma=p + 2), EINVAL), (dict(yt=E4M3, scale=p + 2), EINVAL)])
def test_rmsnorm_refusals(kw, code):
    assert _norm(**kw) == code
    assert b"reslim_rmsnorm_fwd" in B.load().reslim_last_error(None)


def test_rmsnorm_of_no_rows_touches_nothing():
    assert _norm(rows=0, x=None, y=None, delta=None, sum_=None) == OK


def _norm_bwd(s=p, dy=p, gamma=p, eps=1e-6, d_sum=p, rows=4, D=64, stream=F32, act=BF16, dx=p, dd=p, dg=p, ws=p, n=1 << 30):
    return B.load().reslim_rmsnorm_bwd(s, dy, gamma, eps, d_sum, rows, D, stream, act, dx, dd, dg, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(s=None), EINVAL), (dict(dy=None), EINVAL), (dict(gamma=None), EINVAL), (dict(dx=None), EINVAL), (dict(dg=None), EINVAL), (dict(rows=-1), ESHAPE),
    (dict(D=16385), ESHAPE), (dict(stream=BF16, act=F32), EINVAL), (dict(ws=None), EWS), (dict(ws=p + 128), EWS), (dict(n=4 * 64 * 4 - 1), EWS),
    (dict(dx=p + 2), EINVAL), (dict(dy=p + 1), EINVAL), (dict(dd=p + 1), EINVAL), (dict(d_sum=p + 2), EINVAL), (dict(dg=p + 2), EINVAL)])
def test_rmsnorm_bwd_refusals(kw, code):
    assert _norm_bwd(**kw) == code


def test_rmsnorm_workspace():
    assert B.reslim_rmsnorm_bwd_workspace_bytes(0, 100) == 0
    assert B.reslim_rmsnorm_bwd_workspace_bytes(3, 100) == 1280                       # 1200 bytes to the next 256
    assert B.reslim_rmsnorm_bwd_workspace_bytes(10 ** 6, 4096) == 768 * 4096 * 4
    for rows, D in ((-1, 4), (1, 0), (1, 16385)):
        with pytest.raises(B.ReslimError):
            B.reslim_rmsnorm_bwd_workspace_bytes(rows, D)
    assert B.load().reslim_rmsnorm_bwd_workspace_bytes(1, 4, None) == EINVAL


def _rot(name="reslim_rotary_fwd", x=p, out=2 * p, pos=p, freq=p, tokens=5, xs=192, os=128, period=5, heads=2, dh=64, rot=64, axes=1, layout=1, amp=1.0, dt=BF16):
    return getattr(B.load(), name)(x, out, pos, freq, tokens, xs, os, period, heads, dh, rot, axes, layout, amp, dt, None)


@pytest.mark.parametrize("name", ["reslim_rotary_fwd", "reslim_rotary_bwd"])
@pytest.mark.parametrize("kw,code", [
    (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(pos=None), EINVAL), (dict(freq=None), EINVAL), (dict(tokens=-1), ESHAPE), (dict(period=0), ESHAPE),
    (dict(heads=0), ESHAPE), (dict(heads=4), ESHAPE), (dict(dh=63), ESHAPE), (dict(dh=1026, rot=64, heads=1, xs=2000, os=2000), ESHAPE), (dict(rot=66), ESHAPE),
    (dict(rot=1), ESHAPE), (dict(rot=0), ESHAPE), (dict(rot=62, axes=2), ESHAPE), (dict(axes=3), EINVAL), (dict(layout=2), EINVAL), (dict(layout=-1), EINVAL),
    (dict(dt=E4M3), EINVAL), (dict(xs=127), ESHAPE), (dict(os=127), ESHAPE), (dict(amp=math.nan), EINVAL), (dict(amp=math.inf), EINVAL), (dict(out=p), EINVAL),
    (dict(x=p + 1), EINVAL), (dict(freq=p + 4), EINVAL), (dict(pos=p + 2), EINVAL), (dict(layout=0, x=p + 2), EINVAL), (dict(layout=0, xs=193), EINVAL),
    (dict(layout=0, os=129), EINVAL), (dict(dt=F32, x=p + 2), EINVAL)])
def test_rotary_refusals(name, kw, code):
    assert _rot(name, **kw) == code
    assert name.encode() in B.load().reslim_last_error(None)


def test_rotary_of_no_tokens_touches_nothing():
    assert _rot(tokens=0, x=None, out=None, pos=None, freq=None, period=0) == OK


@pytest.mark.parametrize("rot,axes", [(2, 1), (64, 1), (128, 2), (4, 2), (96, 1)])
@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "by_parts"])
def test_frequencies(rot, axes, scaling):
    base, factor, length = 10000.0, 8.0, 4096.0
    got, amp = B.reslim_rotary_frequencies(rot, axes, base, scaling, factor, length)
    d = rot // axes
    b = base * factor ** (d / (d - 2)) if scaling == "base" and d > 2 else base
    f = np.array([b ** (-2.0 * j / d) for j in range(d // 2)])
    if scaling == "linear":
        f = f / factor
    if scaling == "by_parts":
        keep = np.clip((length * f / (2 * math.pi) - 1) / 31, 0, 1)
        f = keep * f + (1 - keep) * f / factor
    # a power, a product, a quotient and the blend: a few half steps of 2^-53 each, the power's exponent up to 10 of them
    assert np.allclose(got, np.tile(f, axes), rtol=64 * 2.0 ** -53, atol=0)
    assert amp == (np.float32(0.1 * math.log(factor) + 1) if scaling == "by_parts" else 1.0)
    if scaling == "base" and d > 2:          # the slowest pair is interpolated by the whole factor, the fastest not at all
        assert got[0] == 1.0 and math.isclose(got[d // 2 - 1] * factor, base ** (-(d - 2) / d), rel_tol=1e-12)


@pytest.mark.parametrize("kw", [dict(rot=3), dict(rot=0), dict(rot=6, axes=2), dict(rot=1026), dict(axes=3), dict(base=1.0), dict(base=math.nan), dict(base=math.inf),
                                dict(scaling="linear", factor=0.5), dict(scaling="base", factor=math.inf), dict(scaling="by_parts", factor=2.0, original_length=0.0)])
def test_frequency_refusals(kw):
    with pytest.raises(B.ReslimError):
        B.reslim_rotary_frequencies(**{"rot": 64, **kw})
    lib = B.load()
    a, f = C.c_float(), np.empty(32)
    assert lib.reslim_rotary_frequencies(64, 1, 1e4, 4, 1.0, 1.0, f.ctypes.data, C.byref(a)) == EINVAL
    assert lib.reslim_rotary_frequencies(64, 1, 1e4, 0, 1.0, 1.0, None, C.byref(a)) == EINVAL


def _weights(w_in=p, scale=None, b_in=p, w_out=p, b_out=p):
    return C.byref(B.GatedMlpWeightsC(w_in=w_in, in_scale=scale, b_in=b_in, w_out=w_out, b_out=b_out))


def _fwd(x=p, xs=None, w=None, gate=0, rows=4, D=128, R=192, dt=BF16, y=p, ws=p, n=1 << 30, **kw):
    return B.load().reslim_gated_mlp_fwd(x, xs, w or _weights(**kw), gate, rows, D, R, dt, y, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(w_in=None), EINVAL), (dict(w_out=None), EINVAL), (dict(gate=2), EINVAL), (dict(gate=-1), EINVAL), (dict(dt=3), EINVAL),
    (dict(rows=-1), ESHAPE), (dict(D=0), ESHAPE), (dict(R=0), ESHAPE), (dict(D=96), ESHAPE), (dict(R=100), ESHAPE), (dict(D=16448), ESHAPE), (dict(R=65600), ESHAPE),
    (dict(dt=E4M3, xs=p, scale=p, D=192), ESHAPE), (dict(dt=E4M3, xs=p), EINVAL), (dict(dt=E4M3, scale=p), EINVAL), (dict(xs=p), EINVAL), (dict(scale=p), EINVAL),
    (dict(dt=F32, rows=4000001), ESHAPE), (dict(dt=F32, rows=3999999, R=9000), ESHAPE), (dict(dt=F32, rows=3999999, D=16000), ESHAPE), (dict(rows=2000000001), ESHAPE),
    (dict(x=p + 8), EINVAL), (dict(w_in=p + 8), EINVAL), (dict(w_out=p + 2), EINVAL), (dict(b_in=p + 4), EINVAL), (dict(b_out=p + 8), EINVAL),
    (dict(y=p + 8), EINVAL), (dict(dt=F32, x=p + 2), EINVAL), (dict(ws=None), EWS), (dict(ws=p + 16), EWS), (dict(n=1), EWS)])
def test_gated_refusals(kw, code):
    assert _fwd(**kw) == code
    assert b"reslim_gated_mlp_fwd" in B.load().reslim_last_error(None)


def test_gated_null_struct_and_no_rows():
    lib = B.load()
    assert lib.reslim_gated_mlp_fwd(p, None, None, 0, 4, 128, 192, BF16, p, p, 1 << 30, None) == EINVAL
    assert _fwd(rows=0, x=None, y=None, ws=None, n=0) == OK
    assert lib.reslim_gated_mlp_fwd_train(None, _weights(), 0, 0, 128, 192, BF16, None, None, None, None, 0, None) == OK
    for fn in (lambda: B.reslim_gated_mlp_workspace_bytes(4, 96, 64, torch.bfloat16), lambda: B.reslim_gated_mlp_workspace_bytes(-1, 64, 64, torch.bfloat16),
               lambda: B.reslim_gated_mlp_bwd_workspace_bytes(4, 128, 64, torch.float8_e4m3fn, torch.float32),
               lambda: B.reslim_gated_mlp_bwd_workspace_bytes(4, 128, 64, torch.float32, torch.bfloat16)):
        with pytest.raises(B.ReslimError):
            fn()
    assert lib.reslim_gated_mlp_workspace_bytes(4, 64, 64, BF16, None) == EINVAL
    with pytest.raises(ValueError):
        B.reslim_gated_mlp_workspace_bytes(4, 64, 64, torch.float16)


@pytest.mark.parametrize("kw,code", [
    (dict(gu=None), EINVAL), (dict(h=None), EINVAL), (dict(y=None), EINVAL), (dict(gu=p + 8), EINVAL), (dict(dt=E4M3, D=128), EINVAL), (dict(gate=5), EINVAL)])
def test_gated_train_refusals(kw, code):
    a = {"gu": p, "h": p, "y": p, "dt": BF16, "D": 128, "gate": 0, **kw}
    w = _weights(scale=p) if a["dt"] == E4M3 else _weights()
    assert B.load().reslim_gated_mlp_fwd_train(p, w, a["gate"], 4, a["D"], 192, a["dt"], a["gu"], a["h"], a["y"], p, 1 << 30, None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), EINVAL), (dict(gu=None), EINVAL), (dict(h=None), EINVAL), (dict(dy=None), EINVAL), (dict(gwi=None), EINVAL), (dict(gwo=None), EINVAL), (dict(dx=p + 8), EINVAL),
    (dict(gwi=p + 8), EINVAL), (dict(gbi=p + 4), EINVAL), (dict(gt=E4M3), EINVAL), (dict(dt=F32, gt=BF16), EINVAL), (dict(dt=E4M3), EINVAL), (dict(D=100), ESHAPE), (dict(gate=9), EINVAL)])
def test_gated_bwd_refusals(kw, code):
    a = {"x": p, "gu": p, "h": p, "dy": p, "gwi": p, "gbi": p, "gwo": p, "gbo": p, "dx": p, "gt": F32, "dt": BF16, "D": 128, "gate": 0, **kw}
    g = C.byref(B.GatedMlpGradsC(w_in=a["gwi"], b_in=a["gbi"], w_out=a["gwo"], b_out=a["gbo"]))
    w = _weights(scale=p) if a["dt"] == E4M3 else _weights()
    assert B.load().reslim_gated_mlp_bwd(a["x"], a["gu"], a["h"], a["dy"], w, a["gate"], 4, a["D"], 192, a["dt"], a["gt"], a["dx"], g, p, 1 << 40, None) == code


def test_binding_refuses_tensors_that_are_not_on_the_gpu():
    x = torch.zeros(2, 64)
    with pytest.raises(ValueError, match="not on the current GPU"):
        B.reslim_rmsnorm_fwd(x, torch.ones(64), torch.empty_like(x))
    with pytest.raises(ValueError, match="not on the current GPU"):
        B.reslim_gated_mlp_fwd(x, {"w_in": torch.zeros(128, 64), "w_out": torch.zeros(64, 64)}, x, None)
    with pytest.raises(ValueError, match="not on the current GPU"):
        B.reslim_rotary_fwd(x[None], x[None], torch.zeros(1, 1, dtype=torch.int32), torch.zeros(32, dtype=torch.float64), heads=2)
    with pytest.raises(ValueError, match="layout"):
        B.reslim_rotary_fwd(x[None], x[None], None, None, heads=2, layout="other")


# ------------------------------------------------------------------ the oracle against differences (64 bits: step 1e-5, error about 1e-9 of the slope)
def _slope(f, x, v, h=1e-5):
    return float((f(x + h * v) - f(x - h * v)) / (2 * h))


def test_oracle_gradients_against_differences():
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    x, dy, gamma, up = r(5, 12), r(5, 12), r(12), r(5, 12)
    loss = lambda x, gamma: (P.rmsnorm(x, None, gamma, 1e-6)[1] * dy).sum() + (x * up).sum()  # noqa: E731
    dx, dgamma, _, _ = P.rmsnorm_bwd(x, dy, gamma, 1e-6, up)
    for v in (r(5, 12), r(5, 12)):
        assert math.isclose(_slope(lambda t: loss(t, gamma), x, v), float((dx * v).sum()), rel_tol=1e-6, abs_tol=1e-7)
    v = r(12)
    assert math.isclose(_slope(lambda t: loss(x, t), gamma, v), float((dgamma * v).sum()), rel_tol=1e-6, abs_tol=1e-7)
    for gate in ("silu", "gelu"):
        w = {"w_in": r(14, 6), "w_out": r(6, 7), "b_in": r(14), "b_out": r(6)}
        x, dy = r(4, 6), r(4, 6)
        run = lambda x, w: P.gated_mlp(x, w, gate, torch.float32)  # noqa: E731
        f = run(x, w)
        grads = P.gated_mlp_bwd(x, f["gu"], f["h"], dy, w, gate, torch.float32, torch.float32)
        v = r(4, 6)
        assert math.isclose(_slope(lambda t: (run(t, w)["y"] * dy).sum(), x, v), float((grads["dx"] * v).sum()), rel_tol=1e-6, abs_tol=1e-7)
        for n in w:
            v = r(*w[n].shape)
            assert math.isclose(_slope(lambda t: (run(x, {**w, n: t})["y"] * dy).sum(), w[n], v), float((grads[n] * v).sum()), rel_tol=1e-6, abs_tol=1e-7), n


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("axes", [1, 2])
def test_oracle_rotation_is_undone_by_its_gradient(layout, axes):
    g = torch.Generator().manual_seed(5)
    x = torch.randn(6, 3, 20, generator=g, dtype=torch.float64)
    pos = torch.randint(0, 1000, (axes, 6), generator=g).to(torch.int32)
    f = torch.from_numpy(B.reslim_rotary_frequencies(12, axes)[0])
    y, _ = P.rotary(x, pos, f, 3, layout, 1.0)
    back, _ = P.rotary(y, pos, f, 3, layout, 1.0, backwards=True)
    assert torch.allclose(back, x, rtol=0, atol=1e-13) and torch.equal(y[..., 12:], x[..., 12:])
    assert torch.allclose(y.square().sum(-1), x.square().sum(-1), rtol=1e-13)
