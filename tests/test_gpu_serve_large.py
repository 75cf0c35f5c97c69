"""Draft verification and 8-bit rows at the sizes where a call changes its way: one launch or two, rows in parts, the last
entries of a part, copies larger than the last-level cache, extreme scales."""
import numpy as np
import pytest
import torch

import paper_2502_14317_amd as pc
from serving import quantize_rows
from test_gpu_verify_drafts import build, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,k,V", [(2, 1, 2), (2, 2, 3), (3, 1, 5), (2, 3, 16383), (3, 2, 16384), (2, 2, 16385), (3, 2, 16387),
                                   (5, 2, 33001), (256, 1, 4099), (257, 1, 4099), (300, 1, 1001), (520, 1, 2050)])
def test_verify_sizes(B, k, V):
    print("verify", B, k, V, flush=True)
    args = list(build(B, k, V, V))
    check(args)
    args[1] = None
    check(args, what="point mass")


@pytest.mark.parametrize("V", [9000, 40001])
def test_verify_edges_in_one_launch_and_in_two(V):
    draft, dp, tp, u, noise = build(8, 2, V, 5)
    draft[0, 0], draft[1, 1] = -1, V                                        # outside the vocabulary
    u[2:4] = 1.0
    dp[2:4] = tp[2:4, :2]                                                   # nothing is left of p - q
    tp[4, 0] = float("nan")
    noise[5, V // 3:V // 2] = 0.0                                           # infinite quotients: the lowest of them
    tp[6] = 0.0                                                             # no mass at all
    tp[7] = 1.0 / V; noise[7] = 1.0                                         # ties over all parts
    u[7] = 1.0; draft[7] = 0
    dp[7] = 0.5; dp[7, :, V - 2:] = 0.0                                     # only the last two entries are left
    want, count = check((draft, dp, tp, u, noise))
    assert count[0] == 0 and count[2] == 0 and want[6, 0] == -1
    assert want[7, 0] == V - 2
    draft[:, 0] = torch.tensor([0, 1, V - 1, V - 2, V // 2, 3, 4, 1024], device="cuda", dtype=torch.int32)
    check((draft, None, tp, u, noise), what="point mass")


def test_verify_huge_and_tiny_quotients():
    """Quotients over the whole range of 32 bits, subnormal ones and those beyond it among them."""
    B, V = 7, 20011
    gen = torch.Generator(device="cuda").manual_seed(2)
    tp = torch.exp2(280 * torch.rand((B, 1, V), generator=gen, device="cuda") - 152)
    noise = torch.exp2(150 * torch.rand((B, V), generator=gen, device="cuda") - 100)
    tp[1] *= 1e-30; tp[2] = 1e-45; noise[2].clamp_(min=1.0); tp[3] *= 1e30
    noise[4, ::3] = float("inf"); noise[5, 1::2] = float("nan"); noise[6] = float("inf")
    check((torch.zeros((B, 0), dtype=torch.int32, device="cuda"), None, tp, torch.zeros((B, 0), device="cuda"), noise))


@pytest.mark.parametrize("D,B,H,cap", [(128, 3, 7, 8400), (64, 4, 8, 11000)])
@pytest.mark.parametrize("ragged", [False, True], ids=["full", "ragged"])
def test_read_beyond_the_cache(D, B, H, cap, ragged):
    gen = torch.Generator(device="cuda").manual_seed(D)
    codes = torch.randint(0, 127, (2, B, H, cap, D), generator=gen, device="cuda").to(torch.uint8)
    codes |= (128 * torch.randint(0, 2, codes.shape, generator=gen, device="cuda")).to(torch.uint8)
    scales = torch.exp(4 * torch.randn((2, B, H, cap), generator=gen, device="cuda"))
    lens = torch.tensor([0, cap, cap // 3, cap - 1][:B], dtype=torch.int32, device="cuda") if ragged else None
    k, v = (torch.full((B, H, cap, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    pc.pc_kv_read_row8(codes[0], codes[1], scales[0], scales[1], lens, B, cap, H, D, k, v)
    for got, c, s in ((k, codes[0], scales[0]), (v, codes[1], scales[1])):
        want = (c.view(torch.float8_e4m3fn).float() * s[..., None]).to(torch.bfloat16)
        for b, n in enumerate(lens.tolist() if ragged else ()):
            want[b, :, n:] = 5.0
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("D", [64, 128])
def test_append_at_extreme_scales(D):
    """Rows from subnormal values to the largest: quotients by the reciprocal and by division, every code and scale."""
    gen = torch.Generator(device="cuda").manual_seed(D)
    n, H = 500, 2
    new = [torch.randn((1, n, H, D), generator=gen, device="cuda") * torch.exp2(torch.linspace(-140, 126, n, device="cuda"))[:, None, None]
           for _ in "kv"]
    new = [x.clamp(-3.3e38, 3.3e38).to(torch.bfloat16) for x in new]
    new[0][0, 7] = 0.0; new[1][0, 8, 0, 3] = float("inf"); new[0][0, 9, 1, D - 1] = float("nan")
    codes = [torch.zeros((1, H, n, D), dtype=torch.uint8, device="cuda") for _ in "kv"]
    scales = [torch.zeros((1, H, n), device="cuda") for _ in "kv"]
    pc.pc_kv_append_row8(new[0], new[1], 1, n, n, H, D, codes[0], codes[1], scales[0], scales[1], None, None)
    for x, c, s in zip(new, codes, scales):
        want, scale = quantize_rows(x[0].permute(1, 0, 2).float().cpu().numpy())
        assert np.array_equal(s[0].cpu().numpy(), scale)
        assert np.array_equal(c[0].cpu().numpy(), want)
