"""8-bit rows: pc_kv_append_row8 bit for bit against the definition in 32-bit steps (without rotation), within the
format's half step with it; pc_kv_read_row8 against code times scale; lengths, full tails, rows that are not finite."""
import numpy as np
import pytest
import torch

import paper_2502_14317_amd as pc
from serving import E4M3, f64, quantize_rows, rotate

pytestmark = pytest.mark.gpu


def alloc(B, H, cap, D, fill=170):
    codes = lambda: torch.full((B, H, cap, D), fill, dtype=torch.uint8, device="cuda")
    scales = lambda: torch.full((B, H, cap), -7.0, dtype=torch.float32, device="cuda")
    return codes(), codes(), scales(), scales()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,n,H,cap", [(1, 1, 1, 1), (3, 1, 8, 40), (2, 5, 3, 21), (1, 300, 2, 333), (70, 2, 1, 9)])
def test_append_bits(B, n, H, cap, D):
    print("append", B, n, H, cap, D, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(B + n + cap + D)
    k, v = ((torch.randn((B, n, H, D), generator=gen, device="cuda") * torch.exp(3 * torch.randn((B, n, H, 1), generator=gen, device="cuda")))
            .to(torch.bfloat16) for _ in "kv")
    k[0, 0, 0] = 0                                                          # a row of zeros
    rows = alloc(B, H, cap, D)
    len_in = torch.randint(0, cap - n + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    len_in[-1] = cap - n                                                    # ends with the segment
    len_out = torch.full((B,), -3, dtype=torch.int32, device="cuda")
    pc.pc_kv_append_row8(k, v, B, n, cap, H, D, *rows, len_in, len_out)
    assert torch.equal(len_out, len_in + n)
    for x, code, scale in ((k, rows[0], rows[2]), (v, rows[1], rows[3])):
        want_c, want_s = quantize_rows(x.float().cpu().numpy())
        got_c, got_s, lens = code.cpu().numpy(), scale.cpu().numpy(), len_in.cpu().numpy()
        for b in range(B):
            at = slice(lens[b], lens[b] + n)
            assert np.array_equal(got_c[b, :, at], want_c[b].transpose(1, 0, 2)), b
            assert np.array_equal(got_s[b, :, at], want_s[b].T), b
            rest = np.ones(cap, bool); rest[at] = False
            assert (got_c[b][:, rest] == 170).all() and (got_s[b][:, rest] == -7.0).all(), "other rows are left alone"


def test_every_magnitude_and_ties():
    """Rows over the whole range of bf16, subnormal ones included, against the definition; all finite codes come back."""
    bits = np.arange(0, 0x7f80, dtype=np.uint16)
    D = 128
    x = np.zeros((len(bits) // (D - 1) + 1, D), np.uint16)
    x[:, 1:] = np.resize(bits, x.shape[0] * (D - 1)).reshape(-1, D - 1)
    x[::2, 0] = 0x4040                                                      # 3: the largest of half the rows below
    x[1::2, 1:] |= 0x8000
    grid = (np.arange(-448 * 8, 448 * 8 + 8, 8)[:, None] / 8.0 + np.arange(D)[None] / 16.0).clip(-448, 448)
    grid[:, 0] = 448.0                                                      # scale 1: sixteenths, so ties occur
    k = torch.from_numpy(x.view(np.int16).copy()).view(torch.bfloat16).cuda().view(1, -1, 1, D)
    g = torch.from_numpy(grid).to(torch.bfloat16).cuda().view(1, -1, 1, D)
    for t in (k, g):
        n = t.shape[1]
        rows = alloc(1, 1, n, D)
        pc.pc_kv_append_row8(t.contiguous(), t.contiguous(), 1, n, n, 1, D, *rows, None, None)
        want_c, want_s = quantize_rows(t.float().cpu().numpy()[0, :, 0])
        assert np.array_equal(rows[2].cpu().numpy()[0, 0], want_s)
        got = rows[0].cpu().numpy()[0, 0]
        zero = (got & 127) == 0
        assert np.array_equal(np.where(zero, 0, got), np.where((want_c & 127) == 0, 0, want_c))
        assert torch.equal(rows[0], rows[1]) and torch.equal(rows[2], rows[3])


def test_rows_that_are_not_finite_read_back_as_nan():
    B, n, H, D = 1, 6, 2, 64
    x = torch.randn((B, n, H, D), device="cuda").to(torch.bfloat16)
    x[0, 1, 0, 7] = float("nan"); x[0, 2, 1, 63] = float("inf"); x[0, 4, 0, 0] = float("-inf")
    rows = alloc(B, H, n, D)
    pc.pc_kv_append_row8(x, x, B, n, n, H, D, *rows, None, None)
    k, v = (torch.zeros((B, H, n, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    pc.pc_kv_read_row8(*rows, None, B, n, H, D, k, v)
    bad = torch.zeros((H, n), dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[1, 2] = bad[0, 4] = True
    assert torch.isnan(k[0][bad]).all() and torch.isfinite(k[0][~bad]).all() and torch.equal(k.view(torch.int16), v.view(torch.int16))


@pytest.mark.parametrize("D", [64, 128])
def test_append_rotates(D):
    """The rotated key is rounded once: within half a step of the format, 2^-4 of the value or 2^-10 of the scale, and
    1e-6 of the row's largest for the rotation in 32 bits."""
    B, n, H, cap, base, pos0 = 3, 4, 2, 30, 5.0e5, 100
    x = torch.randn((B, n, H, D), device="cuda").to(torch.bfloat16)
    rows = alloc(B, H, cap, D)
    len_in = torch.tensor([0, 7, 26], dtype=torch.int32, device="cuda")
    pos = torch.tensor([0, 131071, 8000000], dtype=torch.int32, device="cuda")
    pc.pc_kv_append_row8(x, x, B, n, cap, H, D, *rows, len_in, None, pos=pos, pos0=pos0, rope_base=base)
    for b in range(B):
        want = rotate(f64(x[b]), int(pos[b]) + pos0 + np.arange(n), base).transpose(1, 0, 2)
        at = slice(int(len_in[b]), int(len_in[b]) + n)
        s = rows[2][b, :, at].cpu().numpy().astype(np.float64)
        top = np.abs(want).max(-1)
        assert np.all(np.abs(s - top / 448) <= 2e-6 * top / 448)
        got = E4M3[rows[0][b, :, at].cpu().numpy()] * s[..., None]
        assert np.all(np.abs(got - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * s[..., None]) + 2e-6 * top[..., None])
        plain_c, _ = quantize_rows(x[b].float().cpu().numpy())              # values are not rotated
        assert np.array_equal(rows[1][b, :, at].cpu().numpy(), plain_c.transpose(1, 0, 2))


def test_a_full_segment_drops_rows():
    B, n, H, D, cap = 4, 5, 2, 64, 8
    x = torch.randn((B, n, H, D), device="cuda").to(torch.bfloat16)
    rows = alloc(B, H, cap, D)
    len_in = torch.tensor([8, 6, -4, 99], dtype=torch.int32, device="cuda")
    len_out = torch.empty_like(len_in)
    pc.pc_kv_append_row8(x, x, B, n, cap, H, D, *rows, len_in, len_out)
    assert len_out.tolist() == [8, 8, 5, 8]
    written = (rows[2] != -7.0)[:, 0].sum(1).tolist()
    assert written == [0, 2, 5, 0]
    len_out.fill_(-1)
    pc.pc_kv_append_row8(x[:, :0].contiguous(), x[:, :0].contiguous(), B, 0, cap, H, D, *rows, len_in, len_out)
    assert len_out.tolist() == [8, 6, 0, 8]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,H,cap", [(1, 1, 1), (3, 2, 77), (5, 8, 130)])
def test_read_back(B, H, cap, D):
    gen = torch.Generator(device="cuda").manual_seed(cap)
    codes = torch.randint(0, 256, (2, B, H, cap, D), generator=gen, device="cuda").to(torch.uint8)
    scales = torch.exp(4 * torch.randn((2, B, H, cap), generator=gen, device="cuda"))
    for lens in (None, torch.randint(-1, cap + 3, (B,), generator=gen, device="cuda", dtype=torch.int32)):
        k, v = (torch.full((B, H, cap, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in "kv")
        pc.pc_kv_read_row8(codes[0], codes[1], scales[0], scales[1], lens, B, cap, H, D, k, v)
        for got, c, s in ((k, codes[0], scales[0]), (v, codes[1], scales[1])):
            want = torch.from_numpy((E4M3[c.cpu().numpy()].astype(np.float32) * s.cpu().numpy()[..., None])).to(torch.bfloat16)
            if lens is not None:
                for b, n in enumerate(lens.tolist()):
                    want[b, :, max(n, 0):] = 5.0
            got = got.cpu()
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            assert torch.equal(torch.nan_to_num(got).view(torch.int16), torch.nan_to_num(want).view(torch.int16))
