"""Rows of the gated feed-forward layer do not depend on where a call's products are cut: the output map's and the input gradient's rows past the whole rounds of
256 x 256 tiles go to a launch of their own, and the same rows in other calls get the same bits from whichever kernel takes them."""
import math

import pytest
import torch

from oracle import operators_oracle as P
from paper_2505_04802_amd import binding as B

pytestmark = pytest.mark.gpu
H = torch.bfloat16
AT = 16384                                       # rows of the whole rounds at 2048 columns on 256 compute units
ROWS = [16500, 18000, 20000]                     # the rest goes to 64 x 64, 128 x 128 and 128 x 256 tiles
D, R_OUT, R_DX = 2048, 2048, 1024                # contractions of 2048 either way
PARTS = [(0, AT), (0, AT - 1), (AT - 1700, None), (3000, 15000), (9000, None)]      # rows of calls whose product is not cut there, or not cut at all


@pytest.fixture(autouse=True)
def _float32():
    """Other modules make float64 torch's default for the whole session."""
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


def _layer(R):
    g = torch.Generator(device="cuda").manual_seed(R)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    return {"w_in": (r(2 * R, D) / math.sqrt(D)).to(H), "w_out": (r(D, R) / math.sqrt(R)).to(H), "b_in": 0.3 * r(2 * R), "b_out": 0.3 * r(D)}, r


def _room(n):
    return torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("rows", ROWS)
def test_output_map(rows):
    w, r = _layer(R_OUT)
    x = r(rows, D).to(H)

    def forward(x):
        y = torch.full_like(x, math.nan)
        B.reslim_gated_mlp_fwd(x, w, y, _room(B.reslim_gated_mlp_workspace_bytes(x.shape[0], D, R_OUT, H)))
        return y

    y = forward(x)
    for a, b in PARTS:
        assert torch.equal(forward(x[a:b].contiguous()), y[a:b]), (a, b)
    at = torch.cat([torch.arange(AT - 8, AT + 8), torch.arange(rows - 8, rows)]).cuda()
    want = P.gated_mlp(x[at], w, "silu", H)
    assert P.worst(y[at], want["y"], want["y_bound"] * 1.01 + 1e-30) <= 1


@pytest.mark.parametrize("rows", ROWS)
def test_input_gradient(rows):
    w, r = _layer(R_DX)
    x, gu, h, dy = (r(rows, n).to(H) for n in (D, 2 * R_DX, R_DX, D))

    def gradient(*t):
        dx = torch.full_like(t[0], math.nan)
        grads = {"w_in": torch.empty_like(w["w_in"]), "w_out": torch.empty_like(w["w_out"])}
        B.reslim_gated_mlp_bwd(*t, w, dx, grads, _room(B.reslim_gated_mlp_bwd_workspace_bytes(t[0].shape[0], D, R_DX, H, H)))
        return dx

    dx = gradient(x, gu, h, dy)
    for a, b in PARTS:
        assert torch.equal(gradient(*(t[a:b].contiguous() for t in (x, gu, h, dy))), dx[a:b]), (a, b)
    at = torch.cat([torch.arange(AT - 8, AT + 8), torch.arange(rows - 8, rows)]).cuda()
    want = P.gated_mlp_bwd(x[at], gu[at], h[at], dy[at], w, "silu", H, H)
    assert P.worst(dx[at], want["dx"], want["dx_bound"] * 1.01 + 1e-30) <= 1
