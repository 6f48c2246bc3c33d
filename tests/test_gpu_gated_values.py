"""Values at which the gated feed-forward layer can go wrong: gates at the infinities and far below zero."""
import math

import pytest
import torch

from oracle import operators_oracle as P
from paper_2505_04802_amd import binding as B

pytestmark = pytest.mark.gpu
F, H = torch.float32, torch.bfloat16


@pytest.fixture(autouse=True)
def _float32():
    """Other modules make float64 torch's default for the whole session."""
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


def _room(n):
    return torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda")


def _layer(gates, act, rows=1):
    """A layer whose gate projections are `gates` for every row and whose up projections are 1; W_out's row 0 is ones, so that dh = dy[:, 0]."""
    R, D = gates.numel(), 64
    w = {"w_in": torch.zeros(2 * R, D, dtype=act, device="cuda"), "w_out": torch.zeros(D, R, dtype=act, device="cuda"), "b_in": torch.cat([gates, torch.ones_like(gates)])}
    w["w_out"][0] = 1
    x = torch.ones(rows, D, dtype=act, device="cuda")
    return x, w


def _run(x, w, gate):
    rows, D = x.shape
    R = w["w_out"].shape[1]
    gu, h, y = (torch.full((rows, n), 7.0, dtype=x.dtype, device="cuda") for n in (2 * R, R, D))
    B.reslim_gated_mlp_fwd_train(x, w, gu, h, y, _room(B.reslim_gated_mlp_workspace_bytes(rows, D, R, x.dtype)), gate=gate)
    dy = torch.zeros(rows, D, dtype=x.dtype, device="cuda")
    dy[0, 0] = 1                                     # the gradient of one row
    grads = {"w_in": torch.empty(2 * R, D, device="cuda"), "w_out": torch.empty(D, R, device="cuda"), "b_in": torch.empty(2 * R, device="cuda")}
    B.reslim_gated_mlp_bwd(x, gu, h, dy, w, None, grads, _room(B.reslim_gated_mlp_bwd_workspace_bytes(rows, D, R, x.dtype, F)), gate=gate)
    return gu, h, grads["b_in"][:R]


# rows: 64 x 64 tiles, 128 x 128, and the persistent kernels
@pytest.mark.parametrize("rows", [1, 700, 5000])
@pytest.mark.parametrize("gate", ["silu", "gelu"])
@pytest.mark.parametrize("act", [H, F], ids=["bf16", "f32"])
def test_infinite_gates_give_what_the_definition_gives(act, gate, rows):
    g = torch.randn(704, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    at = {3: math.inf, 64: -math.inf, 130: math.nan, 703: -math.inf, 640: math.inf}
    for k, v in at.items():
        g[k] = v
    x, w = _layer(g, act, rows)
    gu, h, _ = _run(x, w, gate)
    want = P.act(g.double(), gate)
    assert [math.isnan(float(want[k])) for k in at] == [False, True, True, True, False]
    for r in {0, rows // 2, rows - 1}:
        assert torch.equal(torch.isnan(h[r]), torch.isnan(want)) and torch.equal(torch.isinf(h[r]), torch.isinf(want)), r
        fine = torch.isfinite(want)
        assert P.worst(h[r][fine], want[fine], P.FAST[act] * g[fine].double().abs().clamp(min=1.0) + P.half(act) * want[fine].abs()) <= 1


@pytest.mark.parametrize("gate", ["silu", "gelu"])
@pytest.mark.parametrize("act", [H, F], ids=["bf16", "f32"])
def test_slopes_at_infinite_gates(act, gate):
    g = torch.tensor([math.inf, -math.inf, math.nan, 1.0, -1.0], device="cuda").repeat(64)
    x, w = _layer(g, act)
    _, _, dg = _run(x, w, gate)
    want = P.act_slope(g.double(), gate)
    assert torch.equal(torch.isnan(dg), torch.isnan(want)) and bool(torch.isnan(want[:3]).all()) and bool(torch.isfinite(dg[3:5]).all())


@pytest.mark.parametrize("rows", [1, 700, 5000])
def test_gelu_far_below_zero(rows):
    """bf16: relative to the value down to where it leaves fp32, and nothing left of it further down."""
    g = -torch.cat([torch.linspace(0.5, 13.0, 640, device="cuda"), torch.linspace(14.0, 1e4, 64, device="cuda")])
    x, w = _layer(g, H, rows)
    gu, h, dg = _run(x, w, "gelu")
    v = g.double()
    cdf = 0.5 * torch.special.erfc(-v / math.sqrt(2.0))
    want = v * cdf
    # the tail to 1.6e-3 (1.5e-5 down to -5) and the bf16 result's half step; 1e-36: fp32's subnormal values
    assert P.worst(h[0], want, (P.half(H) * 1.01 + 1.7e-3) * want.abs() + 1e-36) <= 1
    assert torch.equal(h[-1], h[0]) and not bool(h[0, 640:].any())
    v = gu[0, :704].double()
    cdf, pdf = 0.5 * torch.special.erfc(-v / math.sqrt(2.0)), torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
    slope = cdf + v * pdf
    err = 1.7e-3 * cdf * (v < -5) + 1.6e-5 * cdf + P.E * (v * v + 4) * (v * pdf).abs()
    assert P.worst(dg, slope, err * 1.01 + P.half(H) * 1.01 * slope.abs() + 1e-36) <= 1
    assert bool((dg[(g < -5) & (g > -12)] < 0).all())
