"""The operators in a run as they are used: a pre-norm block with RMS norm, rotary positions by patch row and column, the library's own tile
attention, and the gated feed-forward layer, forward and backward, against the same block in 64 bits and its automatic gradient.  The
products in between (q | k | v and the attention's output map) are the caller's, here torch's in 32 bits."""
import math

import numpy as np
import pytest
import torch

from oracle import operators_oracle as P
from oracle import reslim_oracle as O
from paper_2505_04802_amd import binding as B
from paper_2505_04802_amd import workloads as WL

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(autouse=True)
def _float32():
    """Other modules make float64 torch's default for the whole session."""
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


def _reference(stream, delta, p, pos, freq, tiles, heads, gate, d_out):
    """Block in float64 on the leaves p; returns (stream out, last delta, gradients of everything)."""
    leaves = {n: t.double().detach().requires_grad_() for n, t in p.items()}
    s0, d0 = stream.double().requires_grad_(), delta.double().requires_grad_()
    norm = lambda s, g: s / torch.sqrt((s * s).mean(-1, keepdim=True) + EPS) * g  # noqa: E731
    s1 = s0 + d0
    qkv = (norm(s1, leaves["g1"]) @ leaves["w_qkv"].t()).view(s1.shape[0], 3 * heads, -1)
    dh, n = qkv.shape[2], freq.numel()
    axis = torch.arange(n, device=pos.device) * pos.shape[0] // n
    angle = (pos.double()[axis] * freq[:, None]).t()[torch.arange(s1.shape[0], device=pos.device) % pos.shape[1]][:, None]
    a, b = qkv[:, :2 * heads, :n], qkv[:, :2 * heads, n:2 * n]
    qk = torch.cat([a * torch.cos(angle) - b * torch.sin(angle), a * torch.sin(angle) + b * torch.cos(angle), qkv[:, :2 * heads, 2 * n:]], -1)
    outs = []
    for first, count in tiles:
        q, k, v = (t.transpose(0, 1) for t in (qk[first:first + count, :heads], qk[first:first + count, heads:], qkv[first:first + count, 2 * heads:]))
        outs.append((torch.softmax(q @ k.transpose(1, 2) / math.sqrt(dh), -1) @ v).transpose(0, 1).reshape(count, heads * dh))
    s2 = s1 + torch.cat(outs) @ leaves["w_proj"].t()
    x2 = norm(s2, leaves["g2"])
    gu = x2 @ leaves["w_in"].t() + leaves["b_in"]
    R = gu.shape[1] // 2
    y = (P.act(gu[:, :R], gate) * gu[:, R:]) @ leaves["w_out"].t() + leaves["b_out"]
    loss = ((s2 + y) * d_out.double()).sum()
    grads = torch.autograd.grad(loss, [s0, d0, *leaves.values()])
    return s2.detach(), y.detach(), dict(zip(["stream", "delta", *leaves], grads))


@pytest.mark.parametrize("dtype,tol", [(1, 2e-2), (0, 1e-5)], ids=["bf16", "f32"])
@pytest.mark.parametrize("gate", ["silu", "gelu"])
def test_block_forward_and_backward(dtype, tol, gate):
    """Tolerances are the ones of the model's own blocks: a dozen roundings of 2^-9 in a row for bf16, fp32 sums for fp32."""
    cfg = WL.ReslimConfig("gated", batch=2, in_vars=2, out_vars=2, H=36, W=44, scale=4, patch=2, embed_dim=256, heads=4, mlp_ratio=4, depth=1, tiles_y=2, tiles_x=2, halo=1,
                          dtype=dtype, seed=5)
    act = torch.bfloat16 if dtype else torch.float32
    D, heads, R = cfg.embed_dim, cfg.heads, 704
    dh, g = D // heads, torch.Generator(device="cuda").manual_seed(11)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    tile_list, gather, _, n_h = B.tiles_partition(cfg.Hp, cfg.Wp, cfg.tiles_y, cfg.tiles_x, cfg.halo)
    M = cfg.batch * n_h
    tiles = [(b * n_h + t["tok_off"], t["n_tok"]) for b in range(cfg.batch) for t in tile_list]
    at = torch.from_numpy(gather).cuda()
    pos = torch.stack([at // cfg.Wp, at % cfg.Wp]).to(torch.int32).contiguous()      # a token's patch row and column; every sample's the same
    freq = torch.from_numpy(B.reslim_rotary_frequencies(dh, 2, 100.0)[0]).cuda()
    p = {"g1": 1 + 0.1 * r(D), "w_qkv": r(3 * D, D) / 16, "w_proj": r(D, D) / 16, "g2": 1 + 0.1 * r(D), "w_in": r(2 * R, D) / 16, "b_in": 0.1 * r(2 * R), "w_out": r(D, R) / 26,
         "b_out": 0.1 * r(D)}
    p = {n: t.to(act).float() if n[0] == "w" else t for n, t in p.items()}
    stream, delta, d_out = r(M, D), r(M, D).to(act), r(M, D)
    s2_ref, y_ref, ref = _reference(stream, delta, p, pos, freq, tiles, heads, gate, d_out)
    empty = lambda *s, dtype=act: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    room = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")  # noqa: E731
    mm = lambda a, b: (a.float() @ b.float())  # noqa: E731
    w = {"w_in": p["w_in"].to(act), "b_in": p["b_in"], "w_out": p["w_out"].to(act), "b_out": p["b_out"]}
    with B.Reslim(cfg, WL.make_weights(cfg)) as model:
        # forward
        s1, x1 = torch.empty_like(stream), empty(M, D)
        B.reslim_rmsnorm_fwd(stream, p["g1"], x1, eps=EPS, delta=delta, sum_out=s1)
        qkv = mm(x1, p["w_qkv"].t()).to(act).view(M, 3 * heads, dh)
        B.reslim_rotary_fwd(qkv, qkv, pos, freq, heads=2 * heads, layout="half")
        qkv = qkv.view(cfg.batch, n_h, 3 * D)
        attn, lse = model.attention_with_lse(qkv)
        delta2 = mm(attn.view(M, D), p["w_proj"].t()).to(act)
        s2, x2 = torch.empty_like(stream), empty(M, D)
        B.reslim_rmsnorm_fwd(s1, p["g2"], x2, eps=EPS, delta=delta2, sum_out=s2)
        gu, h, y = empty(M, 2 * R), empty(M, R), empty(M, D)
        B.reslim_gated_mlp_fwd_train(x2, w, gu, h, y, room(B.reslim_gated_mlp_workspace_bytes(M, D, R, act)), gate=gate)
        # backward: d_out reaches the stream after the block and, rounded, the feed-forward layer's output
        got = {"w_in": empty(2 * R, D, dtype=torch.float32), "b_in": empty(2 * R, dtype=torch.float32), "w_out": empty(D, R, dtype=torch.float32), "b_out": empty(D, dtype=torch.float32)}
        dx2 = empty(M, D)
        B.reslim_gated_mlp_bwd(x2, gu, h, d_out.to(act), w, dx2, dict(got), room(B.reslim_gated_mlp_bwd_workspace_bytes(M, D, R, act, torch.float32)), gate=gate)
        nws = room(B.reslim_rmsnorm_bwd_workspace_bytes(M, D))
        d_s2, d_delta2, got["g2"] = d_out.clone(), empty(M, D), torch.empty_like(p["g2"])
        B.reslim_rmsnorm_bwd(s2, dx2, p["g2"], d_s2, got["g2"], nws, eps=EPS, d_sum=d_s2, d_delta=d_delta2)
        got["w_proj"] = mm(d_delta2.t(), attn.view(M, D))
        d_attn = mm(d_delta2, p["w_proj"]).to(act).view(cfg.batch, n_h, D)
        d_qkv = model.attention_bwd(qkv, attn, lse, d_attn).view(M, 3 * heads, dh)
        B.reslim_rotary_bwd(d_qkv, d_qkv, pos, freq, heads=2 * heads, layout="half")
        got["w_qkv"] = mm(d_qkv.reshape(M, 3 * D).t(), x1)
        dx1 = mm(d_qkv.reshape(M, 3 * D), p["w_qkv"]).to(act)
        d_delta, got["g1"], got["stream"] = empty(M, D), torch.empty_like(p["g1"]), torch.empty_like(stream)
        B.reslim_rmsnorm_bwd(s1, dx1, p["g1"], got["stream"], got["g1"], nws, eps=EPS, d_sum=d_s2, d_delta=d_delta)
        got["delta"] = d_delta
    for n, a, b in [("stream out", s2, s2_ref), ("feed-forward out", y, y_ref)] + [(n, t, ref[n]) for n, t in got.items()]:
        err = O.rel_l2(a.double().cpu().numpy(), b.cpu().numpy())
        print(f"  {n}: {err:.2e}", flush=True)
        assert np.isfinite(err) and err <= tol, n


def test_norm_to_eight_bits_and_the_product_that_reads_them():
    """The norm's e4m3 rows and scales go into the feed-forward layer as they are; the result is that of the rows' stated values."""
    M, D, R = 333, 512, 1344
    g = torch.Generator(device="cuda").manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    stream, delta, gamma = r(M, D), r(M, D).to(torch.bfloat16), 1 + 0.1 * r(D)
    w_in = r(2 * R, D) / math.sqrt(D)
    scale = w_in.abs().amax(1) / 448
    w = {"w_in": (w_in / scale[:, None]).to(torch.float8_e4m3fn), "in_scale": scale, "w_out": (r(D, R) / math.sqrt(R)).to(torch.bfloat16)}
    x8, xs = torch.empty(M, D, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(M, device="cuda")
    B.reslim_rmsnorm_fwd(stream, gamma, x8, eps=EPS, delta=delta, sum_out=stream, y_scale=xs)
    y = torch.empty(M, D, dtype=torch.bfloat16, device="cuda")
    B.reslim_gated_mlp_fwd(x8, w, y, torch.empty(B.reslim_gated_mlp_workspace_bytes(M, D, R, x8.dtype), dtype=torch.uint8, device="cuda"), x_scale=xs)
    want = P.gated_mlp(x8, w, "silu", torch.bfloat16, xs)
    assert P.worst(y, want["y"], want["y_bound"] * 1.01) <= 1 and P.rel2(y, want["y"]) <= P.half(torch.bfloat16)
    # and against the unrounded norm with unrounded weights: e4m3 rounds each factor of every product by up to 2^-4, a third of its square on average,
    # so the projections are off by 2^-4 sqrt(2 / 3) at most in the 2-norm, and the product of two of them by about twice that
    full = P.gated_mlp(P.rmsnorm(stream, None, gamma, EPS)[1], {"w_in": w_in, "w_out": w["w_out"]}, "silu", torch.float32)
    assert P.rel2(y, full["y"]) <= 2 * 2.0 ** -4
