"""The gated feed-forward layer, forward and gradient, against the 64-bit statement: elementwise within bounds that count every rounding, and in
the 2-norm.  One row to several tiles, feature counts that end inside every tile, every type, biases present and absent."""
import math

import pytest
import torch

from oracle import operators_oracle as P
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


def _gen(*seed):
    return torch.Generator(device="cuda").manual_seed(sum(s * 1000003 ** i for i, s in enumerate(seed)) % (1 << 40))


def _case(rows, D, R, act, bias, x_type=None, seed=0):
    g = _gen(rows, D, R, seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    w = {"w_in": r(2 * R, D) / math.sqrt(D), "w_out": (r(D, R) / math.sqrt(R)).to(act)}
    x, x_scale = r(rows, D), None
    if bias:
        w["b_in"], w["b_out"] = 0.3 * r(2 * R), 0.3 * r(D)
    if x_type == Q:
        w["in_scale"], x_scale = w["w_in"].abs().amax(1) / 448, x.abs().amax(1) / 448
        w["w_in"], x = (w["w_in"] / w["in_scale"][:, None]).to(Q), (x / x_scale[:, None]).to(Q)
    else:
        w["w_in"], x = w["w_in"].to(act), x.to(act)
    return x, x_scale, w


def _room(n):
    return torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda")      # NaN wherever it is read unwritten


def _forward(x, w, act, gate, x_scale=None, **kw):
    R = w["w_out"].shape[1]
    y = torch.full(x.shape, math.nan, dtype=act, device="cuda")
    B.reslim_gated_mlp_fwd(x, w, y, _room(B.reslim_gated_mlp_workspace_bytes(*x.shape, R, x.dtype)), gate=gate, x_scale=x_scale, **kw)
    return y


def _train(x, w, gate):
    R = w["w_out"].shape[1]
    gu, h, y = (torch.full((x.shape[0], n), math.nan, dtype=x.dtype, device="cuda") for n in (2 * R, R, x.shape[1]))
    B.reslim_gated_mlp_fwd_train(x, w, gu, h, y, _room(B.reslim_gated_mlp_workspace_bytes(*x.shape, R, x.dtype)), gate=gate)
    return gu, h, y


def _backward(x, gu, h, dy, w, gate, gt, bias=True, want_dx=True):
    R, D = h.shape[1], x.shape[1]
    grads = {"w_in": torch.full((2 * R, D), math.nan, dtype=gt, device="cuda"), "w_out": torch.full((D, R), math.nan, dtype=gt, device="cuda")}
    if bias:
        grads["b_in"], grads["b_out"] = torch.full((2 * R,), math.nan, dtype=gt, device="cuda"), torch.full((D,), math.nan, dtype=gt, device="cuda")
    dx = torch.full_like(x, math.nan) if want_dx else None
    B.reslim_gated_mlp_bwd(x, gu, h, dy, w, dx, grads, _room(B.reslim_gated_mlp_bwd_workspace_bytes(x.shape[0], D, R, x.dtype, gt)), gate=gate)
    return {**grads, "dx": dx} if want_dx else grads


def _near(got, want, bound, dtype, name):
    over, rel = P.worst(got, want, bound * 1.01 + 1e-30), P.rel2(got, want)
    print(f"  {name}: {over:.3f} of the elementwise bound, 2-norm {rel:.2e}", flush=True)
    assert over <= 1, name
    # at most three independent roundings to the type on the way to a result, each at most half a step, a third of its square on average:
    # half a step in all; fp32 adds the sums' rounding, some 30 half steps (products of up to 4096 terms, exponential or error function)
    assert rel <= (P.half(dtype) * 1.01 if dtype != F else 40 * P.E), name


SIZES = [(1, 64, 64), (2, 128, 192), (16, 256, 704), (17, 64, 320), (31, 320, 832), (33, 192, 64), (64, 512, 1344), (65, 128, 256), (127, 1024, 2752), (129, 320, 192),
         (197, 320, 832), (256, 64, 128), (300, 1088, 1472), (515, 448, 1216)]

# sizes for the kernels beside the 64 x 64 tiles, and for slices of k
LARGE = [(400, 1024, 2752), (1001, 1024, 2752), (1300, 1024, 2752), (590, 2048, 5504), (2030, 1024, 2752), (4100, 1024, 2752), (100, 4096, 10944), (999, 2048, 5504)]


@pytest.mark.parametrize("gate", ["silu", "gelu"])
@pytest.mark.parametrize("rows,D,R", SIZES + LARGE)
def test_forward_bf16(rows, D, R, gate):
    for bias in (False, True):
        x, _, w = _case(rows, D, R, H, bias)
        want = P.gated_mlp(x, w, gate, H)
        y = _forward(x, w, H, gate)
        _near(y, want["y"], want["y_bound"], H, "y")
        gu, h, y2 = _train(x, w, gate)
        _near(gu, want["gu"], want["gu_bound"], H, "gu")
        _near(h, want["h"], want["h_bound"], H, "h")
        _near(y2, want["y"], want["y_bound"], H, "y of the training forward")
        assert torch.equal(y, _forward(x, w, H, gate))


@pytest.mark.parametrize("gate", ["silu", "gelu"])
@pytest.mark.parametrize("rows,D,R", [(1, 128, 64), (3, 256, 704), (16, 512, 320), (40, 128, 192), (64, 1024, 2752), (130, 384, 832), (257, 640, 1216), (1000, 256, 128),
                                       (700, 2048, 5504), (2030, 1024, 2752)])
def test_forward_e4m3(rows, D, R, gate):
    for bias in (False, True):
        x, xs, w = _case(rows, D, R, H, bias, Q)
        want = P.gated_mlp(x, w, gate, H, xs)
        _near(_forward(x, w, H, gate, xs), want["y"], want["y_bound"], H, "y")


@pytest.mark.parametrize("gate", ["silu", "gelu"])
@pytest.mark.parametrize("gt", [H, F], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,D,R", SIZES + LARGE)
def test_backward_bf16(rows, D, R, gt, gate):
    x, _, w = _case(rows, D, R, H, True)
    gu, h, _ = _train(x, w, gate)
    dy = torch.randn(rows, D, generator=_gen(rows, 5), device="cuda").to(H)
    want = P.gated_mlp_bwd(x, gu, h, dy, w, gate, H, gt)
    got = _backward(x, gu, h, dy, w, gate, gt)
    for n, t in got.items():
        assert P.worst(t, want[n], want[n + "_bound"] * 1.01 + 1e-30) <= 1, n
        # dx and dW_in read [dg | du] rounded to bf16 whatever the gradient's type; dW_out and its bias read nothing rounded on the way
        rounded = t.dtype == H or n in ("dx", "w_in", "b_in")
        assert P.rel2(t, want[n]) <= (P.half(H) * 1.01 if rounded else 40 * P.E), n
    again = _backward(x, gu, h, dy, w, gate, gt)
    assert all(torch.equal(got[n], again[n]) for n in got)
    bare = _backward(x, gu, h, dy, {k: v for k, v in w.items() if k[0] == "w"}, gate, gt, bias=False, want_dx=False)
    assert set(bare) == {"w_in", "w_out"} and all(torch.equal(bare[n], got[n]) for n in bare)


# any sizes: operands whose rows start off 16 bytes, features that end inside tiles of 32 and 64, contractions that end inside slabs
@pytest.mark.parametrize("gate", ["silu", "gelu"])
@pytest.mark.parametrize("rows,D,R", [(1, 1, 1), (1, 24, 48), (2, 7, 5), (5, 33, 31), (64, 128, 344), (129, 65, 130), (200, 100, 66), (333, 513, 257), (1100, 40, 70), (700, 36, 32)])
def test_fp32(rows, D, R, gate):
    for bias in (False, True):
        x, _, w = _case(rows, D, R, F, bias)
        want = P.gated_mlp(x, w, gate, F)
        y = _forward(x, w, F, gate)
        gu, h, y2 = _train(x, w, gate)
        assert torch.equal(y, y2)
        for n, t in (("gu", gu), ("h", h), ("y", y)):
            _near(t, want[n], want[n + "_bound"], F, n)
        dy = torch.randn(rows, D, generator=_gen(rows, 6), device="cuda")
        want = P.gated_mlp_bwd(x, gu, h, dy, w, gate, F, F)
        got = _backward(x, gu, h, dy, w, gate, F, bias=bias)
        for n, t in got.items():
            assert P.worst(t, want[n], want[n + "_bound"] * 1.01 + 1e-30) <= 1, n


def test_fp32_off_16_bytes():
    x, _, w = _case(70, 64, 96, F, True)
    off = lambda t: torch.empty(t.numel() + 1, device="cuda")[1:].view(t.shape).copy_(t)  # noqa: E731
    got, want = _train(off(x), {n: off(t) for n, t in w.items()}, "silu"), _train(x, w, "silu")
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_many_rows_go_through_the_persistent_kernels():
    """Enough tiles for several rounds of a work-group a compute unit, the last one partly filled, at the widths of the medium grid."""
    rows, D, R = 20000, 1024, 2752
    x, _, w = _case(rows, D, R, H, True)
    gu, h, y = _train(x, w, "silu")
    dy = (0.01 * torch.randn(rows, D, generator=_gen(1), device="cuda")).to(H)
    want = P.gated_mlp(x, w, "silu", H)
    for n, t in (("gu", gu), ("h", h), ("y", y)):
        _near(t, want[n], want[n + "_bound"], H, n)
    del want
    for gt in (H, F):
        got, want = _backward(x, gu, h, dy, w, "silu", gt), P.gated_mlp_bwd(x, gu, h, dy, w, "silu", H, gt)
        for n, t in got.items():
            assert P.worst(t, want[n], want[n + "_bound"] * 1.01 + 1e-30) <= 1, n
    x8, xs, w8 = _case(rows, D, R, H, True, Q)
    want = P.gated_mlp(x8, w8, "gelu", H, xs)
    _near(_forward(x8, w8, H, "gelu", xs), want["y"], want["y_bound"], H, "y of e4m3")


@pytest.mark.parametrize("rows", [16500, 18000, 20000])
def test_rows_past_the_whole_rounds_of_tiles(rows):
    """The output map's product and the input gradient's are cut behind row 16,384, for either of the three kernels that the rest may get."""
    D, R = 2048, 1024
    x, _, w = _case(rows, D, R, H, True)
    gu, h, y = _train(x, w, "silu")
    dy = torch.randn(rows, D, generator=_gen(rows), device="cuda").to(H)
    got = _backward(x, gu, h, dy, w, "silu", H)
    at = torch.cat([torch.arange(0, 40), torch.arange(16384 - 40, 16384 + 100), torch.arange(rows - 40, rows)]).cuda()
    want = P.gated_mlp(x[at], w, "silu", H)
    _near(y[at], want["y"], want["y_bound"], H, "y")
    want = P.gated_mlp_bwd(x[at], gu[at], h[at], dy[at], w, "silu", H, H)
    assert P.worst(got["dx"][at], want["dx"], want["dx_bound"] * 1.01 + 1e-30) <= 1
    cut = 16384 + 64
    for rest in (slice(0, cut), slice(cut - 300, rows)):      # whole and part again, in calls that are cut elsewhere: the same bits
        a, b = _train(x[rest].contiguous(), w, "silu"), (gu[rest], h[rest])
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("x_type,rows", [(H, 3), (H, 70), (H, 700), (F, 70), (Q, 3), (Q, 70)])
def test_a_row_does_not_touch_others_and_nothing_behind_the_last_is_written(x_type, rows):
    act = F if x_type == F else H
    x, xs, w = _case(rows, 256, 320, act, True, x_type)
    clean = _forward(x, w, act, "gelu", xs)
    bad = x.clone()
    bad[rows // 2, 3] = math.nan
    y = torch.full((rows + 300, 256), 7.0, dtype=act, device="cuda")
    B.reslim_gated_mlp_fwd(bad, w, y[:rows], _room(B.reslim_gated_mlp_workspace_bytes(rows, 256, 320, x.dtype)), gate="gelu", x_scale=xs)
    keep = torch.arange(rows, device="cuda") != rows // 2
    assert torch.equal(y[:rows][keep], clean[keep]) and bool(torch.isnan(y[rows // 2]).all()) and bool((y[rows:] == 7).all())
    if x_type != Q:
        gu, h = (torch.full((rows + 300, n), 7.0, dtype=act, device="cuda") for n in (640, 320))
        B.reslim_gated_mlp_fwd_train(x, w, gu[:rows], h[:rows], y[:rows], _room(B.reslim_gated_mlp_workspace_bytes(rows, 256, 320, x.dtype)), gate="gelu")
        assert torch.equal(y[:rows], clean) and all(bool((t[rows:] == 7).all()) for t in (gu, h, y))
        dx = torch.full((rows + 300, 256), 7.0, dtype=act, device="cuda")
        grads = {"w_in": torch.empty_like(w["w_in"]), "w_out": torch.empty_like(w["w_out"])}
        B.reslim_gated_mlp_bwd(x, gu[:rows], h[:rows], clean, w, dx[:rows], grads, _room(B.reslim_gated_mlp_bwd_workspace_bytes(rows, 256, 320, act, act)), gate="gelu")
        assert bool(torch.isfinite(dx).all()) and bool((dx[rows:] == 7).all())


@pytest.mark.parametrize("gate", ["silu", "gelu"])
@pytest.mark.parametrize("act", [H, F], ids=["bf16", "f32"])
def test_activation_over_its_whole_range(act, gate):
    """One row whose gate takes every size through the bias: w_in = 0, u = 1, so that h = act(g) and dg = dh act'(g)."""
    R = 4096
    g = torch.cat([torch.linspace(-30, 30, R - 8, device="cuda"), torch.tensor([0.0, -0.0, 1e-20, -1e-20, 80.0, -80.0, 3e4, -3e4], device="cuda")])
    w = {"w_in": torch.zeros(2 * R, 64, dtype=act, device="cuda"), "w_out": torch.zeros(64, R, dtype=act, device="cuda"), "b_in": torch.cat([g, torch.ones_like(g)])}
    w["w_out"][0] = 1
    x = torch.ones(1, 64, dtype=act, device="cuda")
    gu, h, _ = _train(x, w, gate)
    held = gu[0, :R].double()
    want = P.act(g.double(), gate)
    assert P.worst(h[0], want, 4e-6 * g.double().abs().clamp(min=1e-3) + P.half(act) * want.abs() + 2e-6 * (act == H) + 1e-30) <= 1
    dy = torch.zeros(1, 64, dtype=act, device="cuda")
    dy[0, 0] = 1
    got = _backward(x, gu, h, dy, w, gate, F)
    slope = P.act_slope(held, gate)
    assert P.worst(got["b_in"][:R], slope, 4e-6 * held.abs().clamp(min=1.0) + P.half(act) * slope.abs()) <= 1


def test_no_rows():
    for act in (H, F):
        x, _, w = _case(0, 64, 128, act, True)
        gu, h, y = _train(x, w, "silu")
        for gt in {act, F}:
            assert all(bool((t == 0).all()) for n, t in _backward(x, gu, h, y, w, "silu", gt).items())


def test_rows_behind_two_to_the_31_elements():
    rows, D, R = 420000, 64, 2560
    x, _, w = _case(8, D, R, H, True)
    x = x.repeat(rows // 8, 1)
    gu, h, y = _train(x, w, "silu")
    print("forward done", flush=True)
    for t in (gu, h, y):                                    # every group of eight rows is the first one
        assert torch.equal(t[:8], t[-8:]) and torch.equal(t[:8], t[209720:209728])
    want = P.gated_mlp(x[:8], w, "silu", H)
    for n, t in (("gu", gu), ("h", h), ("y", y)):
        _near(t[:8], want[n], want[n + "_bound"], H, n)
    dy = torch.zeros_like(y)
    dy[-3:] = 1.0
    got = _backward(x, gu, h, dy, w, "silu", F)
    print("backward done", flush=True)
    want = P.gated_mlp_bwd(x[-3:], gu[-3:], h[-3:], dy[-3:], w, "silu", H, F)
    for n, t in got.items():
        assert P.worst(t[-3:] if n == "dx" else t, want[n], want[n + "_bound"] * 1.01 + 1e-30) <= 1, n
    assert bool((got["dx"][:-3] == 0).all())


@pytest.mark.parametrize("rows", [5, 200])
def test_another_stream_and_captured_graphs_that_share_nothing_but_weights(rows):
    x, _, w = _case(rows, 192, 320, H, True)
    dy = torch.randn(rows, 192, device="cuda").to(H)
    st = torch.cuda.Stream()
    y = torch.empty_like(x)
    room = [_room(B.reslim_gated_mlp_workspace_bytes(rows, 192, 320, H)) for _ in range(2)]
    st.wait_stream(torch.cuda.current_stream())
    B.reslim_gated_mlp_fwd(x, w, y, room[0], stream=st)
    st.synchronize()
    assert torch.equal(y, _forward(x, w, H, "silu"))
    sets = []
    for k in range(2):
        s = {"x": x.clone(), "gu": torch.empty(rows, 640, dtype=H, device="cuda"), "h": torch.empty(rows, 320, dtype=H, device="cuda"), "y": torch.empty_like(x),
             "dx": torch.empty_like(x), "grads": {n: torch.empty_like(t, dtype=F) for n, t in w.items()}, "graph": torch.cuda.CUDAGraph(),
             "room": _room(B.reslim_gated_mlp_bwd_workspace_bytes(rows, 192, 320, H, F))}
        with torch.cuda.graph(s["graph"]):
            B.reslim_gated_mlp_fwd_train(s["x"], w, s["gu"], s["h"], s["y"], room[k])
            B.reslim_gated_mlp_bwd(s["x"], s["gu"], s["h"], dy, w, s["dx"], s["grads"], s["room"])
        sets.append(s)
    for seed in range(3):
        for k, s in enumerate(sets):
            s["x"].copy_(_case(rows, 192, 320, H, True, seed=10 * seed + k + 1)[0])
        for s in sets:
            s["graph"].replay()
        torch.cuda.synchronize()
        for s in sets:
            gu, h, y = _train(s["x"], w, "silu")
            assert torch.equal(s["y"], y) and torch.equal(s["gu"], gu)
            want = _backward(s["x"], gu, h, dy, w, "silu", F)
            assert torch.equal(s["dx"], want["dx"]) and all(torch.equal(t, want[n]) for n, t in s["grads"].items())


def test_two_calls_at_once():
    x, _, w = _case(600, 256, 704, H, True)
    z, _, v = _case(90, 512, 320, H, True, seed=4)
    want = _forward(x, w, H, "silu"), _forward(z, v, H, "gelu")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    ys = [torch.empty_like(x), torch.empty_like(z)]
    rooms = [_room(B.reslim_gated_mlp_workspace_bytes(600, 256, 704, H)), _room(B.reslim_gated_mlp_workspace_bytes(90, 512, 320, H))]
    torch.cuda.synchronize()
    for _ in range(10):
        B.reslim_gated_mlp_fwd(x, w, ys[0], rooms[0], gate="silu", stream=streams[0])
        B.reslim_gated_mlp_fwd(z, v, ys[1], rooms[1], gate="gelu", stream=streams[1])
    torch.cuda.synchronize()
    assert torch.equal(ys[0], want[0]) and torch.equal(ys[1], want[1])


def test_binding_refuses():
    x, _, w = _case(4, 64, 128, H, True)
    y, ws = torch.empty_like(x), _room(1 << 16)
    for kw in (dict(x=x.float()), dict(x=x[:, :32]), dict(y=y.float()), dict(w={**w, "w_in": w["w_in"][:200]}), dict(w={**w, "b_in": w["b_in"].to(H)}),
               dict(w={**w, "w_out": w["w_out"].t()}), dict(x_scale=torch.ones(3, device="cuda")), dict(gate="relu")):
        a = {"x": x, "y": y, "w": w, "x_scale": None, "gate": "silu", **kw}
        with pytest.raises((ValueError, B.ReslimError)):
            B.reslim_gated_mlp_fwd(a["x"], a["w"], a["y"], ws, gate=a["gate"], x_scale=a["x_scale"])
    with pytest.raises(B.ReslimError):
        B.reslim_gated_mlp_fwd(x, w, y, ws, x_scale=torch.ones(4, device="cuda"))      # scales without 8-bit rows
    with pytest.raises(B.ReslimError):
        B.reslim_gated_mlp_fwd(x, w, y, None)
