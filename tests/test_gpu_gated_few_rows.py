"""The fp32 gated feed-forward layer at up to 16 rows: the kernel that streams the weights past them, for the gated product and for the output map.  Its eight
waves share the contraction's steps of 16, four of them loaded at a time: sizes with 0, 1, 4, 5, 8, 17 and 22 steps a wave, the last wave with fewer, result
features that do not end with a group of 16, and sizes on either side of where the kernel is taken."""
import math

import pytest
import torch

from oracle import operators_oracle as P
from paper_2505_04802_amd import binding as B

pytestmark = pytest.mark.gpu
F = torch.float32

# which of (gated product, output map) take the kernel: up to 16 rows, contraction (D; R) a multiple of 16
SIZES = [(1, 256, 704), (5, 80, 48), (16, 1024, 2752), (16, 2064, 592), (3, 640, 528), (8, 512, 1040), (2, 16, 2192), (11, 208, 100), (4, 100, 592), (17, 64, 96), (16, 36, 40)]
TAKEN = [(True, True)] * 7 + [(True, False), (False, True), (False, False), (False, False)]


@pytest.fixture(autouse=True)
def _float32():
    """Other modules make float64 torch's default for the whole session."""
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


@pytest.mark.parametrize("gate", ["silu", "gelu"])
@pytest.mark.parametrize("rows,D,R", SIZES)
def test_few_rows(rows, D, R, gate):
    g = torch.Generator(device="cuda").manual_seed(rows * 10007 + D * 101 + R)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    for bias in (False, True):
        x, w = r(rows, D), {"w_in": r(2 * R, D) / math.sqrt(D), "w_out": r(D, R) / math.sqrt(R)}
        if bias:
            w["b_in"], w["b_out"] = 0.3 * r(2 * R), 0.3 * r(D)
        room = torch.full((B.reslim_gated_mlp_workspace_bytes(rows, D, R, F) + 256,), 255, dtype=torch.uint8, device="cuda")
        gu, h, y, y2 = (torch.full((rows + 20, n), 7.0, device="cuda") for n in (2 * R, R, D, D))      # 20 rows behind the last stay
        B.reslim_gated_mlp_fwd_train(x, w, gu[:rows], h[:rows], y[:rows], room, gate=gate)
        B.reslim_gated_mlp_fwd(x, w, y2[:rows], room, gate=gate)
        assert torch.equal(y, y2)
        want = P.gated_mlp(x, w, gate, F)
        for n, t in (("gu", gu), ("h", h), ("y", y)):
            assert bool((t[rows:] == 7).all()), n
            over, rel = P.worst(t[:rows], want[n], want[n + "_bound"] * 1.01 + 1e-30), P.rel2(t[:rows], want[n])
            print(f"  {n}: {over:.3f} of the elementwise bound, 2-norm {rel:.2e}", flush=True)
            assert over <= 1, n
            assert rel <= 40 * P.E, n      # sums of up to 352 terms in each of 8 waves, four at a time, and a function: some 30 half steps on average


def test_a_row_does_not_depend_on_the_others():
    x = torch.randn(16, 256, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    w = {"w_in": torch.randn(2 * 704, 256, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda") / 16,
         "w_out": torch.randn(256, 704, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda") / 26}
    room = torch.empty(B.reslim_gated_mlp_workspace_bytes(16, 256, 704, F) + 256, dtype=torch.uint8, device="cuda")
    all_, one = torch.empty_like(x), torch.empty_like(x)
    B.reslim_gated_mlp_fwd(x, w, all_, room)
    for k in range(16):
        B.reslim_gated_mlp_fwd(x[k:k + 1], w, one[k:k + 1], room)
    assert torch.equal(all_, one)
    x[5, 7] = math.nan
    B.reslim_gated_mlp_fwd(x, w, one, room)
    keep = torch.arange(16, device="cuda") != 5
    assert torch.equal(one[keep], all_[keep]) and bool(torch.isnan(one[5]).all())
