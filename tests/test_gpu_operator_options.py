"""Outputs of the operators of gated pre-norm blocks that a call may leave out: what remains is the same."""
import math

import pytest
import torch

from paper_2505_04802_amd import binding as B

pytestmark = pytest.mark.gpu
F, H, Q = torch.float32, torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def _float32():
    """Other modules make float64 torch's default for the whole session."""
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


def _bits(t):
    return t.view(torch.uint8)


@pytest.mark.parametrize("stream,act", [(F, F), (F, H), (H, H)], ids=["f32", "f32_bf16", "bf16"])
@pytest.mark.parametrize("D", [33, 64, 1000, 4096])
def test_norm_without_the_sum(D, stream, act):
    x, delta, gamma = torch.randn(9, D, device="cuda").to(stream), torch.randn(9, D, device="cuda").to(act), torch.randn(D, device="cuda")
    for yt in (act, Q):
        out = []
        for keep in (True, False):
            y, scale = torch.empty(9, D, dtype=yt, device="cuda"), torch.empty(9, device="cuda") if yt == Q else None
            B.reslim_rmsnorm_fwd(x, gamma, y, delta=delta, sum_out=torch.empty_like(x) if keep else None, y_scale=scale)
            out.append((y, scale))
        assert torch.equal(_bits(out[0][0]), _bits(out[1][0])) and (yt != Q or torch.equal(out[0][1], out[1][1]))


@pytest.mark.parametrize("stream,act", [(F, F), (F, H), (H, H)], ids=["f32", "f32_bf16", "bf16"])
@pytest.mark.parametrize("D", [33, 64, 1000, 4096])
def test_norm_gradient_without_the_addends(D, stream, act):
    s, dy, gamma = torch.randn(70, D, device="cuda").to(stream), torch.randn(70, D, device="cuda").to(act), torch.randn(D, device="cuda")
    ws = torch.full((B.reslim_rmsnorm_bwd_workspace_bytes(70, D),), 255, dtype=torch.uint8, device="cuda")
    got = []
    for dd in (torch.empty_like(dy), None):
        dx, dg = torch.empty_like(s), torch.full_like(gamma, math.nan)
        B.reslim_rmsnorm_bwd(s, dy, gamma, dx, dg, ws, d_delta=dd)
        got.append((dx, dg))
        assert dd is None or torch.equal(dd, dx.to(act))      # fp32 rounded once more, or the same type
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("act", [F, H], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 100, 1500])
def test_gated_gradient_without_dx_or_biases(act, rows):
    D, R = 192, 320
    x, gu, h, dy = (torch.randn(rows, n, device="cuda").to(act) for n in (D, 2 * R, R, D))
    w = {"w_in": torch.randn(2 * R, D, device="cuda").to(act), "w_out": torch.randn(D, R, device="cuda").to(act)}
    ws = torch.full((B.reslim_gated_mlp_bwd_workspace_bytes(rows, D, R, act, act),), 255, dtype=torch.uint8, device="cuda")
    shapes = {"w_in": (2 * R, D), "w_out": (D, R), "b_in": (2 * R,), "b_out": (D,)}
    whole = None
    for names, want_dx in ((("w_in", "w_out", "b_in", "b_out"), True), (("w_in", "w_out", "b_in"), False), (("w_in", "w_out", "b_out"), True), (("w_in", "w_out"), False)):
        g, dx = {n: torch.full(shapes[n], math.nan, dtype=act, device="cuda") for n in names}, torch.full_like(x, math.nan) if want_dx else None
        B.reslim_gated_mlp_bwd(x, gu, h, dy, w, dx, g, ws, gate="gelu")
        whole = whole or (g, dx)
        assert all(bool(torch.isfinite(t).all()) and torch.equal(t, whole[0][n]) for n, t in g.items()) and (dx is None or torch.equal(dx, whole[1]))
