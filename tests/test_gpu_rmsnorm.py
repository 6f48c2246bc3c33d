"""RMS norm with the residual's addition and its gradient against the 64-bit statement, elementwise, within derived bounds: widths on either
side of every boundary between the kernel's shapes, rows that start off 16 bytes, every type, one row to several for each work-group."""
import math

import pytest
import torch

from oracle import operators_oracle as P
from paper_2505_04802_amd import binding as B

pytestmark = pytest.mark.gpu
F, H, Q = torch.float32, torch.bfloat16, torch.float8_e4m3fn
EPS = 1e-6
WIDTHS = [1, 3, 4, 8, 60, 64, 65, 100, 256, 257, 260, 512, 895, 1000, 1024, 1025, 1032, 2048, 2056, 4096, 4097, 4104, 8192, 8200, 16383, 16384]


@pytest.fixture(autouse=True)
def _float32():
    """Other modules make float64 torch's default for the whole session."""
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


def _off(t, n):
    """The same values `n` elements into an allocation."""
    return torch.empty(t.numel() + n, dtype=t.dtype, device="cuda")[n:].view(t.shape).copy_(t)


def _inputs(rows, D, stream, act, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 31 * D + rows)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    return (r(rows, D) * torch.exp(r(D))).to(stream), (0.5 * r(rows, D)).to(act), 1.0 + 0.3 * r(D)


def _forward(x, delta, gamma, yt, eps=EPS, **kw):
    y = torch.empty(x.shape, dtype=yt, device="cuda")
    s = torch.empty_like(x)
    scale = torch.empty(x.shape[0], device="cuda") if yt == Q else None
    B.reslim_rmsnorm_fwd(x, gamma, y, eps=eps, delta=delta, sum_out=s, y_scale=scale, **kw)
    return s, y, scale


def _check_forward(x, delta, gamma, s, y, scale, eps=EPS):
    want_s, want = P.rmsnorm(x, delta, gamma, eps)
    assert P.worst(s, want_s, (P.half(x.dtype) + P.E) * want_s.abs() + 1e-40) <= 1
    # s: one half step; mean: half of (16 + 6 + 16 additions), root, quotient and the two products
    near = 40 * P.E * want.abs()
    if y.dtype == Q:
        top = want.abs().amax(1)
        assert P.worst(scale, top / 448, 44 * P.E * top / 448 + 1e-40) <= 1
        assert bool((y.double().abs().amax(1)[top > 0] == 448).all())
        # half a step of the value, or of the smallest numbers (2^-9 apart)
        assert P.worst(y.double() * scale.double()[:, None], want, near + 46 * P.E * want.abs() + P.half(Q) * want.abs() + 2.0 ** -10 * (top / 448)[:, None] * 1.001 + 1e-40) <= 1
    else:
        assert P.worst(y, want, near + P.half(y.dtype) * want.abs() + 1e-40) <= 1


@pytest.mark.parametrize("stream,act", [(F, F), (F, H), (H, H)], ids=["f32", "f32_bf16", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_forward(D, stream, act):
    for rows in (1, 5, 66):
        x, delta, gamma = _inputs(rows, D, stream, act)
        for yt in (act, Q):
            for add in (delta, None):
                if add is None and yt == Q and stream != act:
                    continue                       # without an addend the activation type is the stream's
                _check_forward(x, add, gamma, *_forward(x, add, gamma, yt))


@pytest.mark.parametrize("stream,act", [(F, F), (F, H), (H, H)], ids=["f32", "f32_bf16", "bf16"])
@pytest.mark.parametrize("D", [8, 72, 1024, 4096, 16384])
def test_rows_that_start_off_16_bytes_give_what_aligned_ones_give(D, stream, act):
    x, delta, gamma = _inputs(7, D, stream, act)
    for yt in (act, Q):
        s, y, scale = _forward(_off(x, 1), _off(delta, 3), _off(gamma, 1), yt)
        _check_forward(x, delta, gamma, s, y, scale)


def _backward(s, dy, gamma, d_sum, apart, eps=EPS):
    dx, dgamma = torch.empty_like(s), torch.full_like(gamma, math.nan)
    dd = torch.empty_like(dy) if apart else None
    ws = torch.full((max(B.reslim_rmsnorm_bwd_workspace_bytes(*s.shape), 256),), 255, dtype=torch.uint8, device="cuda")
    B.reslim_rmsnorm_bwd(s, dy, gamma, dx, dgamma, ws, eps=eps, d_sum=d_sum, d_delta=dd)
    return dx, dd, dgamma


def _check_backward(s, dy, gamma, d_sum, dx, dd, dgamma, eps=EPS):
    want, want_g, bound, bound_g = P.rmsnorm_bwd(s, dy, gamma, eps, d_sum)
    assert P.worst(dx, want, bound * 1.01 + P.half(dx.dtype) * want.abs() + 1e-40) <= 1
    if dd is not None:
        assert P.worst(dd, want, bound * 1.01 + P.half(dd.dtype) * want.abs() + 1e-40) <= 1
    assert P.worst(dgamma, want_g, bound_g + 1e-40) <= 1


@pytest.mark.parametrize("stream,act", [(F, F), (F, H), (H, H)], ids=["f32", "f32_bf16", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_backward(D, stream, act):
    for rows in (1, 2, 67):
        s, dy, gamma = _inputs(rows, D, stream, act)
        d_sum = torch.randn_like(s)
        for add in (d_sum, None):
            _check_backward(s, dy, gamma, add, *_backward(s, dy, gamma, add, stream != act))


@pytest.mark.parametrize("rows,D,stream", [(2500, 320, F), (5001, 72, H), (3000, 1500, F), (1025, 4096, H), (1100, 33, F)])
def test_backward_of_several_rows_a_work_group(rows, D, stream):
    s, dy, gamma = _inputs(rows, D, stream, H)
    d_sum = torch.randn_like(s)
    one = _backward(s, dy, gamma, d_sum, stream != H)
    _check_backward(s, dy, gamma, d_sum, *one)
    for a, b in zip(one, _backward(s, dy, gamma, d_sum, stream != H)):
        assert a is None or torch.equal(a, b)      # sums in a fixed order


def test_backward_off_16_bytes():
    for stream, D in ((F, 1024), (H, 512), (F, 16384)):
        s, dy, gamma = _inputs(9, D, stream, H)
        _check_backward(s, dy, gamma, s, *_backward(_off(s, 1), _off(dy, 1), _off(gamma, 1), _off(s, 3), stream != H))


@pytest.mark.parametrize("D", [64, 1000, 4096, 77])
def test_in_place_is_the_same_and_nothing_else_is_written(D):
    x, delta, gamma = _inputs(6, D, F, H)
    s, y, _ = _forward(x, delta, gamma, H)
    big = torch.full((10, D), 7.0, device="cuda")
    big[2:8] = x
    out = torch.full((10, D), 7.0, dtype=H, device="cuda")
    B.reslim_rmsnorm_fwd(big[2:8], gamma, out[2:8], eps=EPS, delta=delta, sum_out=big[2:8])
    assert torch.equal(big[2:8], s) and torch.equal(out[2:8], y)
    assert bool((big[:2] == 7).all()) and bool((big[8:] == 7).all()) and bool((out[:2] == 7).all()) and bool((out[8:] == 7).all())
    dx, dd, dg = _backward(x, delta, gamma, s, True)
    big[2:8] = s
    dg2, dd2 = torch.empty_like(gamma), torch.full((10, D), 7.0, dtype=H, device="cuda")
    ws = torch.empty(max(B.reslim_rmsnorm_bwd_workspace_bytes(6, D), 256), dtype=torch.uint8, device="cuda")
    B.reslim_rmsnorm_bwd(x, delta, gamma, big[2:8], dg2, ws, eps=EPS, d_sum=big[2:8], d_delta=dd2[2:8])
    assert torch.equal(big[2:8], dx) and torch.equal(dd2[2:8], dd) and torch.equal(dg2, dg)
    assert bool((big[:2] == 7).all()) and bool((big[8:] == 7).all()) and bool((dd2[8:] == 7).all())


@pytest.mark.parametrize("D", [64, 4096, 130])
def test_a_row_that_is_not_finite_or_zero_keeps_to_itself(D):
    x, delta, gamma = _inputs(8, D, F, H)
    clean = _forward(x, delta, gamma, H)[1]
    clean8, scale8 = _forward(x, delta, gamma, Q)[1:]
    for value in (math.nan, math.inf, -math.inf, 3e38):
        bad = x.clone()
        bad[3, D // 2] = value
        _, y, _ = _forward(bad, delta, gamma, H)
        keep = [0, 1, 2, 4, 5, 6, 7]
        assert torch.equal(y[keep], clean[keep])
        _, y8, s8 = _forward(bad, delta, gamma, Q)
        assert torch.equal(y8.view(torch.uint8)[keep], clean8.view(torch.uint8)[keep]) and torch.equal(s8[keep], scale8[keep])
        if not math.isfinite(value):
            assert bool(torch.isnan(y[3, D // 2])) and bool(torch.isnan(y8[3, D // 2].float() * s8[3]))
        dx = _backward(bad, delta, gamma, None, False)[0]
        assert torch.equal(dx[keep], _backward(x, delta, gamma, None, False)[0][keep])
    zero = x.clone()
    zero[3] = 0
    _, y8, s8 = _forward(zero, None, gamma, Q)
    assert bool((y8[3].float() == 0).all()) and float(s8[3]) == 0.0
    assert bool((_forward(zero, None, gamma, F)[1][3] == 0).all())


def test_values_at_the_ends_of_the_range():
    gamma = torch.ones(256, device="cuda")
    for size in (1e-30, 1e-18, 1e18):                # squares below the smallest numbers, and large ones
        x = torch.randn(4, 256, device="cuda") * size
        _check_forward(x, None, gamma, *_forward(x, None, gamma, F))
    tiny = torch.randn(4, 256, device="cuda") * 1e-38      # 448 / max overflows: the factor stops at the largest number
    _, y, scale = _forward(tiny, None, 1e-3 * gamma, Q)
    assert bool(torch.isfinite(y.float()).all()) and bool(torch.isfinite(scale).all())


def test_no_rows():
    gamma = torch.ones(96, device="cuda")
    x = torch.empty(0, 96, device="cuda")
    _forward(x, None, gamma, F)
    dgamma = torch.full_like(gamma, 5.0)
    B.reslim_rmsnorm_bwd(x, x, gamma, x, dgamma, None)
    assert bool((dgamma == 0).all())


def test_rows_behind_two_to_the_31_elements():
    rows, D = 140000, 16384
    x = torch.empty(rows, D, dtype=H, device="cuda").normal_()
    gamma = torch.randn(D, device="cuda")
    s, y, scale = _forward(x, x, gamma, Q)
    print("forward done", flush=True)
    for at in (slice(0, 3), slice(131070, 131075), slice(rows - 3, rows)):
        _check_forward(x[at], x[at], gamma, s[at], y[at], scale[at])
    del y
    dx, dgamma = s, torch.empty_like(gamma)          # in place of the forward's sum: not read by this call
    ws = torch.empty(B.reslim_rmsnorm_bwd_workspace_bytes(rows, D), dtype=torch.uint8, device="cuda")
    B.reslim_rmsnorm_bwd(x, x, gamma, dx, dgamma, ws, eps=EPS)
    print("backward done", flush=True)
    for at in (slice(0, 3), slice(131070, 131075), slice(rows - 3, rows)):
        want, _, bound, _ = P.rmsnorm_bwd(x[at], x[at], gamma, EPS, None)
        assert P.worst(dx[at], want, bound * 1.01 + P.half(H) * want.abs() + 1e-40) <= 1


@pytest.mark.parametrize("stream,act", [(F, F), (F, H), (H, H)], ids=["f32", "f32_bf16", "bf16"])
@pytest.mark.parametrize("D", [1, 3, 7, 61, 257, 1021, 2047, 4093, 8189, 9001, 16383])
def test_a_row_that_ends_inside_a_piece_takes_nothing_from_the_next(D, stream, act):
    rows = 2000 // (D // 1000 + 1)
    x, delta, gamma = _inputs(rows, D, stream, act)
    d_sum = torch.randn_like(x)
    wild = torch.zeros(rows, 1, device="cuda")
    wild[1::2], wild[3::4] = math.nan, math.inf
    for yt in (act, Q):
        clean, mixed = x.clone(), x + wild.to(stream)
        for t in (clean, mixed):
            t.y, t.scale = torch.empty(rows, D, dtype=yt, device="cuda"), torch.empty(rows, device="cuda") if yt == Q else None
            B.reslim_rmsnorm_fwd(t, gamma, t.y, eps=EPS, delta=delta, sum_out=t, y_scale=t.scale)        # in place
        for a, b in ((clean, mixed), (clean.y.view(torch.uint8), mixed.y.view(torch.uint8))) + (((clean.scale, mixed.scale),) if yt == Q else ()):
            assert torch.equal(a[::2], b[::2])
    clean, mixed = _backward(x, delta, gamma, d_sum, True), _backward(x + wild.to(stream), delta, gamma, d_sum + wild.to(stream), True)
    assert torch.equal(clean[0][::2], mixed[0][::2]) and torch.equal(clean[1][::2], mixed[1][::2])


def test_more_rows_than_a_launch_has_threads():
    n = 68_000_000                                   # a wave each: 4.35e9 threads
    x, y, scale = torch.ones(n, 64, dtype=H, device="cuda"), torch.zeros(n, 64, dtype=Q, device="cuda"), torch.zeros(n, device="cuda")
    B.reslim_rmsnorm_fwd(x, torch.ones(64, device="cuda"), y, eps=0.0, y_scale=scale)
    torch.cuda.synchronize()
    assert bool((y.view(torch.uint8).view(-1, 4096)[::17] == 0x7E).all()) and bool((scale == scale[0]).all()) and abs(float(scale[0]) * 448 - 1) <= 4 * P.E


def test_another_stream_and_a_captured_graph():
    x, delta, gamma = _inputs(300, 1024, F, H)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    y, s = torch.empty(300, 1024, dtype=H, device="cuda"), torch.empty_like(x)
    B.reslim_rmsnorm_fwd(x, gamma, y, eps=EPS, delta=delta, sum_out=s, stream=st)
    st.synchronize()
    assert torch.equal(y, _forward(x, delta, gamma, H)[1])
    dx, dd, dg = torch.empty_like(x), torch.empty_like(delta), torch.empty_like(gamma)
    ws = torch.empty(B.reslim_rmsnorm_bwd_workspace_bytes(300, 1024), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.reslim_rmsnorm_fwd(x, gamma, y, eps=EPS, delta=delta, sum_out=s)
        B.reslim_rmsnorm_bwd(s, y, gamma, dx, dg, ws, eps=EPS, d_sum=x, d_delta=dd)
    for seed in range(3):
        nx, nd, _ = _inputs(300, 1024, F, H, seed + 1)
        x.copy_(nx)
        delta.copy_(nd)
        graph.replay()
        torch.cuda.synchronize()
        es, ey, _ = _forward(nx, nd, gamma, H)
        assert torch.equal(s, es) and torch.equal(y, ey)
        for a, b in zip((dx, dd, dg), _backward(es, ey, gamma, nx, True)):
            assert torch.equal(a, b)


def test_binding_refuses():
    x, delta, gamma = _inputs(4, 64, F, H)
    y = torch.empty(4, 64, dtype=H, device="cuda")
    for kw in (dict(x=x[:, :32]), dict(y=y[:2]), dict(gamma=gamma.double()), dict(gamma=gamma[:8]), dict(delta=delta[:, ::2]), dict(sum_out=x.to(H)), dict(x=x.half())):
        a = {"x": x, "gamma": gamma, "y": y, "delta": delta, "sum_out": None, **kw}
        with pytest.raises(ValueError):
            B.reslim_rmsnorm_fwd(a["x"], a["gamma"], a["y"], delta=a["delta"], sum_out=a["sum_out"])
    with pytest.raises(B.ReslimError):
        B.reslim_rmsnorm_fwd(x, gamma, torch.empty(4, 64, dtype=Q, device="cuda"))      # no y_scale


@pytest.mark.parametrize("D", [48, 513, 4096])
@pytest.mark.parametrize("size", [1.0, 1e-30, 1e-35, 1e-36, 1e-37, 1e-38, 1e-40, 1e-42])
def test_e4m3_of_rows_at_the_end_of_fp32(size, D):
    """Rows whose largest magnitude is too small for 448 / max: they still span the 8-bit range."""
    x = torch.randn(5, D, generator=torch.Generator(device="cuda").manual_seed(D), device="cuda")
    gamma = torch.full((D,), size, device="cuda")
    y, scale = torch.empty(5, D, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(5, device="cuda")
    B.reslim_rmsnorm_fwd(x, gamma, y, y_scale=scale)
    _, want = P.rmsnorm(x, None, gamma, 1e-6)
    top = want.abs().amax(1, keepdim=True)
    assert bool((y.float().abs().amax(1) == 448).all())
    # y gamma rounded among fp32's subnormal values, 2^-150; half a step of e4m3, 2^-4 of the value or 2^-10 of the scale; a scale among the subnormal values is off by
    # up to 2^-150, 448 times that at the top; the norm's sums and products some 40 half steps of fp32
    bound = want.abs() * (2.0 ** -4 + 64 * P.E) + top / 448 * 2.0 ** -10 + 450 * 2.0 ** -150
    assert P.worst(y.double() * scale.double()[:, None], want, bound * 1.01) <= 1
