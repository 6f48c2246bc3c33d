"""Rotary positions and their gradient against the 64-bit statement, elementwise, within the derived bound: both layouts, one and two axes, part
of the head, odd numbers of heads and tokens, strided and offset tensors, positions up to 2^31 - 1."""
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


def _table(rot, axes, **kw):
    f, amp = B.reslim_rotary_frequencies(rot, axes, **kw)
    return torch.from_numpy(f).cuda(), amp


def _x(tokens, heads, dh, dtype, seed=0):
    return torch.randn(tokens, heads, dh, generator=torch.Generator(device="cuda").manual_seed(seed + tokens), device="cuda").to(dtype)


def _positions(axes, period, top=200000, seed=0):
    return torch.randint(0, top, (axes, period), generator=torch.Generator(device="cuda").manual_seed(seed + 7), device="cuda").to(torch.int32)


def _check(x, out, positions, freq, heads, layout, amplitude, backwards=False):
    want, bound = P.rotary(x, positions, freq, heads, layout, amplitude, backwards)
    assert P.worst(out, want, bound * 1.01 + P.half(out.dtype) * want.abs() + 1e-40) <= 1
    assert torch.equal(out[..., 2 * freq.numel():], x[:, :heads, 2 * freq.numel():])


# head sizes whose pieces are whole 16 bytes, and ones that are not
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [H, F], ids=["bf16", "f32"])
@pytest.mark.parametrize("dh,rot,axes", [(64, 64, 1), (64, 64, 2), (128, 64, 1), (128, 128, 2), (80, 20, 1), (96, 24, 2), (256, 256, 1), (64, 16, 1), (64, 8, 2), (6, 4, 1), (10, 2, 1),
                                         (34, 20, 2), (1024, 1022, 1), (720, 720, 2)])
def test_rotation(dh, rot, axes, dtype, layout):
    freq, _ = _table(rot, axes)
    for tokens, heads, more, period in ((1, 1, 0, 1), (3, 5, 2, 2), (131, 3, 3, 131), (70, 12, 6, 35)):
        x = _x(tokens, heads + more, dh, dtype)
        pos = _positions(axes, period)
        for call, back in ((B.reslim_rotary_fwd, False), (B.reslim_rotary_bwd, True)):
            out = torch.full((tokens, heads, dh), math.nan, dtype=dtype, device="cuda")
            call(x, out, pos, freq, heads=heads, layout=layout, amplitude=1.25)
            _check(x, out, pos, freq, heads, layout, 1.25, back)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [H, F], ids=["bf16", "f32"])
def test_in_place_strided_and_offset(dtype, layout):
    freq, amp = _table(64, 1, scaling="by_parts", factor=16.0, original_length=4096.0)
    pos = _positions(1, 50)
    x = _x(50, 9, 96, dtype)
    want = torch.empty(50, 6, 96, dtype=dtype, device="cuda")
    B.reslim_rotary_fwd(x, want, pos, freq, heads=6, layout=layout, amplitude=amp)
    _check(x, want, pos, freq, 6, layout, amp)
    y = x.clone()
    B.reslim_rotary_fwd(y, y, pos, freq, heads=6, layout=layout, amplitude=amp)
    assert torch.equal(y[:, :6], want) and torch.equal(y[:, 6:], x[:, 6:])
    # into the first heads of a wider tensor whose other heads, and whose tokens in front and behind, stay
    wide = torch.full((54, 8, 96), 3.0, dtype=dtype, device="cuda")
    B.reslim_rotary_fwd(x, wide[2:52], pos, freq, heads=6, layout=layout, amplitude=amp)
    assert torch.equal(wide[2:52, :6], want) and bool((wide[2:52, 6:] == 3).all()) and bool((wide[:2] == 3).all()) and bool((wide[52:] == 3).all())
    # two elements into an allocation, every second token of it: not on 16 bytes
    flat = torch.empty(2 + 100 * 9 * 96, dtype=dtype, device="cuda")
    off = flat[2:].view(100, 9, 96)[::2].copy_(x)
    out = torch.empty_like(want)
    B.reslim_rotary_fwd(off, out, pos, freq, heads=6, layout=layout, amplitude=amp)
    _check(x, out, pos, freq, 6, layout, amp)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_and_negative_positions(layout):
    freq, _ = _table(128, 1)
    pos = torch.tensor([[0, 1, -1, 1 << 20, (1 << 20) + 1, 2 ** 31 - 1, -(2 ** 31)]], dtype=torch.int32, device="cuda")
    x = _x(7, 4, 128, F)
    out = torch.empty_like(x)
    B.reslim_rotary_fwd(x, out, pos, freq, heads=4, layout=layout)
    want, bound = P.rotary(x, pos, freq, 4, layout, 1.0)
    # the angle, its turns and the constant 1 / 2 pi are each off by up to 2^-53 of 2^31 radians, and so is the angle of the statement
    assert P.worst(out, want, bound + 2.0 ** 31 * 4 * 2.0 ** -53 * 2 * x.double().abs().amax() + 1e-40) <= 1
    assert torch.equal(out[0], x[0])


def test_values_that_are_not_finite_stay_in_their_pair():
    freq, _ = _table(64, 1)
    pos = _positions(1, 9)
    x = _x(9, 4, 64, H)
    clean = torch.empty_like(x)
    B.reslim_rotary_fwd(x, clean, pos, freq, heads=4, layout="half")
    bad = x.clone()
    bad[4, 2, 5], bad[6, 1, 40] = math.nan, math.inf
    out = torch.empty_like(x)
    B.reslim_rotary_fwd(bad, out, pos, freq, heads=4, layout="half")
    same = torch.ones_like(x, dtype=torch.bool)
    for t, h, k in ((4, 2, 5), (6, 1, 40)):
        same[t, h, k % 32] = same[t, h, k % 32 + 32] = False
    assert torch.equal(out[same], clean[same]) and not bool(torch.isfinite(out[~same]).any())


def test_gradient_is_the_transpose():
    """<rotate(x), d> = <x, gradient(d)>: what a gradient of a linear map has to satisfy."""
    freq, _ = _table(48, 2)
    pos, x, d = _positions(2, 40), _x(40, 5, 64, F), _x(40, 5, 64, F, seed=9)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    B.reslim_rotary_fwd(x, y, pos, freq, heads=5, layout="interleaved", amplitude=0.75)
    B.reslim_rotary_bwd(d, dx, pos, freq, heads=5, layout="interleaved", amplitude=0.75)
    # the unturned features are copied on both sides; errors of the elements add up to at most the bounds' sum
    a, b = (y.double() * d.double()).sum(), (x.double() * dx.double()).sum()
    assert abs(float(a - b)) <= 26 * P.E * float((x.double().abs() * 2).sum() * d.double().abs().amax())


def test_tokens_behind_two_to_the_31_elements():
    tokens, heads, dh = 290000, 116, 64
    x = torch.empty(tokens, heads, dh, dtype=H, device="cuda").normal_()
    freq, _ = _table(64, 1)
    pos = _positions(1, 1000)
    sample = [slice(0, 2), slice(289261, 289265), slice(tokens - 2, tokens)]      # 2^31 elements end in token 289,262
    kept = [x[at].clone() for at in sample]
    B.reslim_rotary_fwd(x, x, pos, freq, heads=heads, layout="half")
    for at, was in zip(sample, kept):
        t = torch.arange(at.start, at.stop, device="cuda") % 1000
        _check(was, x[at], pos[:, t].contiguous(), freq, heads, "half", 1.0)


def test_more_tokens_than_a_launch_has_threads():
    tokens, dh = 67_200_000, 62                      # 31 threads each, eight tokens to a work-group: a second launch from 2^26 on
    x = torch.empty(tokens, 1, dh, dtype=H, device="cuda").normal_()
    freq, _ = _table(62, 1)
    pos = _positions(1, 1001)
    sample = [slice(0, 2), slice(2 ** 26 - 2, 2 ** 26 + 2), slice(tokens - 2, tokens)]
    kept = [x[at].clone() for at in sample]
    B.reslim_rotary_fwd(x, x, pos, freq, heads=1, layout="half")
    for at, was in zip(sample, kept):
        t = torch.arange(at.start, at.stop, device="cuda") % 1001
        _check(was, x[at], pos[:, t].contiguous(), freq, 1, "half", 1.0)


def test_no_tokens():
    x = torch.empty(0, 4, 64, dtype=H, device="cuda")
    B.reslim_rotary_fwd(x, x, torch.empty(1, 0, dtype=torch.int32, device="cuda"), _table(64, 1)[0], heads=4)


def test_another_stream_and_a_captured_graph():
    freq, _ = _table(64, 2)
    pos, x = _positions(2, 77), _x(154, 12, 64, H)
    want, out = torch.empty(154, 8, 64, dtype=H, device="cuda"), torch.empty(154, 8, 64, dtype=H, device="cuda")
    B.reslim_rotary_fwd(x, want, pos, freq, heads=8)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    B.reslim_rotary_fwd(x, out, pos, freq, heads=8, stream=st)
    st.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.reslim_rotary_fwd(x, out, pos, freq, heads=8)
    for seed in range(3):
        x.copy_(_x(154, 12, 64, H, seed + 1))
        pos.copy_(_positions(2, 77, seed=seed))
        graph.replay()
        torch.cuda.synchronize()
        B.reslim_rotary_fwd(x, want, pos, freq, heads=8)
        assert torch.equal(out, want)


def test_binding_refuses():
    freq, _ = _table(64, 1)
    pos, x = _positions(1, 4), _x(4, 6, 64, H)
    ok = dict(x=x, out=torch.empty(4, 4, 64, dtype=H, device="cuda"), pos=pos, freq=freq, heads=4)
    for kw in (dict(heads=7), dict(x=x[..., :32]), dict(x=x[:, ::2]), dict(out=ok["out"].float()), dict(out=ok["out"][:3]), dict(pos=pos.long()), dict(freq=freq.float()),
               dict(out=torch.empty(4, 4, 32, dtype=H, device="cuda")), dict(pos=pos[0])):
        a = {**ok, **kw}
        with pytest.raises((ValueError, B.ReslimError)):
            B.reslim_rotary_fwd(a["x"], a["out"], a["pos"], a["freq"], heads=a["heads"])
    with pytest.raises(B.ReslimError):
        B.reslim_rotary_fwd(x, x[:, :4].contiguous(), pos, _table(128, 1)[0], heads=4)      # more features than a head has


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [H, F], ids=["bf16", "f32"])
@pytest.mark.parametrize("dh,rot", [(70, 64), (66, 32), (18, 16), (130, 128)])
def test_in_place_beside_features_that_end_inside_a_piece(dh, rot, dtype, layout):
    freq, _ = _table(rot, 1)
    pos, x = _positions(1, 37), _x(37, 7, dh, dtype)
    y = x.clone()
    B.reslim_rotary_fwd(y, y, pos, freq, heads=5, layout=layout)
    _check(x, y[:, :5], pos, freq, 5, layout, 1.0)
    assert torch.equal(y[:, 5:], x[:, 5:])
