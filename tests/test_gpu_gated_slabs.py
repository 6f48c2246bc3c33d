"""Contractions of one to three slabs through the gated feed-forward layer's larger kernels, where a work-group's tiles follow each other after a slab or two."""
import math

import pytest
import torch

from oracle import operators_oracle as P
from paper_2505_04802_amd import binding as B

pytestmark = pytest.mark.gpu
H, Q = torch.bfloat16, torch.float8_e4m3fn

E4M3 = [(12000, 128, 4096), (1500, 384, 4096), (3000, 384, 4096)]      # persistent 256 x 256 with one slab and with three, 128 x 256 with three
BF16 = [(700, 192, 1024), (20000, 64, 128), (20000, 192, 128), (66000, 64, 64), (100000, 192, 4096)]      # 128 x 128 tiles with one and three; the last: 256 x 256


@pytest.fixture(autouse=True)
def _float32():
    """Other modules make float64 torch's default for the whole session."""
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


def _room(n):
    return torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda")


def _rows(rows):
    """Rows at the ends and around the borders of the first tiles and of the last ones."""
    last = (rows - 1) // 256 * 256
    return torch.cat([torch.arange(a, b) for a, b in ((0, 8), (120, 136), (248, 264), (rows // 2, rows // 2 + 8), (last - 8, last + 1), (rows - 8, rows))]).unique().cuda()


@pytest.mark.parametrize("gate", ["silu", "gelu"])
@pytest.mark.parametrize("rows,D,R", E4M3)
def test_e4m3(rows, D, R, gate):
    g = torch.Generator(device="cuda").manual_seed(rows + D)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, w_in = r(rows, D), r(2 * R, D) / math.sqrt(D)
    xs, ws = x.abs().amax(1) / 448, w_in.abs().amax(1) / 448
    x8 = (x / xs[:, None]).to(Q)
    w = {"w_in": (w_in / ws[:, None]).to(Q), "in_scale": ws, "w_out": (r(D, R) / math.sqrt(R)).to(H), "b_in": 0.3 * r(2 * R), "b_out": 0.3 * r(D)}
    y = torch.full((rows, D), math.nan, dtype=H, device="cuda")
    B.reslim_gated_mlp_fwd(x8, w, y, _room(B.reslim_gated_mlp_workspace_bytes(rows, D, R, Q)), gate=gate, x_scale=xs)
    assert bool(torch.isfinite(y).all())
    at = _rows(rows)
    want = P.gated_mlp(x8[at], w, gate, H, xs[at])
    assert P.worst(y[at], want["y"], want["y_bound"] * 1.01 + 1e-30) <= 1


@pytest.mark.parametrize("rows,D,R", BF16)
def test_bf16(rows, D, R):
    g = torch.Generator(device="cuda").manual_seed(rows + D)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, w = r(rows, D).to(H), {"w_in": (r(2 * R, D) / math.sqrt(D)).to(H), "w_out": (r(D, R) / math.sqrt(R)).to(H), "b_in": 0.3 * r(2 * R)}
    gu, h, y, dx = (torch.full((rows, n), math.nan, dtype=H, device="cuda") for n in (2 * R, R, D, D))
    B.reslim_gated_mlp_fwd_train(x, w, gu, h, y, _room(B.reslim_gated_mlp_workspace_bytes(rows, D, R, H)), gate="silu")
    dy = r(rows, D).to(H)
    grads = {"w_in": torch.empty_like(w["w_in"]), "w_out": torch.empty_like(w["w_out"])}
    B.reslim_gated_mlp_bwd(x, gu, h, dy, w, dx, grads, _room(B.reslim_gated_mlp_bwd_workspace_bytes(rows, D, R, H, H)), gate="silu")
    assert all(bool(torch.isfinite(t).all()) for t in (gu, h, y, dx, *grads.values()))
    at = _rows(rows)
    want = P.gated_mlp(x[at], w, "silu", H)
    for n, t in (("gu", gu), ("h", h), ("y", y)):
        assert P.worst(t[at], want[n], want[n + "_bound"] * 1.01 + 1e-30) <= 1, n
    want = P.gated_mlp_bwd(x[at], gu[at], h[at], dy[at], w, "silu", H, H)
    assert P.worst(dx[at], want["dx"], want["dx_bound"] * 1.01 + 1e-30) <= 1
