"""SharedPrefixDecoder: steps of drafted tokens over two documents, verified, rolled back and continued.  Every step's
attention against 64 bits over what the caches hold, every key that was appended within the 8-bit format of its rotated
row, the lengths after every verification."""
import numpy as np
import pytest
import torch

import paper_2502_14317_amd as pc
from paper_2502_14317_amd.layer import SharedPrefixDecoder
from serving import check_attention, f64, rotate, row_values, verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eight_bit", [False, True], ids=["16bit", "8bit"])
def test_drafted_steps(eight_bit):
    B, P, S, kt, cap, Hq, Hkv, D, base, w, k, V = 6, 2, 3, 75, 64, 8, 2, 128, 5.0e5, 7680, 3, 501
    gen = torch.Generator(device="cuda").manual_seed(7)
    mk = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    dec = SharedPrefixDecoder(B, P, S, kt, cap, Hq, Hkv, D, base, w, max_rows=k + 1, eight_bit_prefix=eight_bit)
    kc, vc, n0 = mk(P, S, Hkv, kt, D), mk(P, S, Hkv, kt, D), 9
    seg_len = torch.randint(1, kt + 1, (P, S, Hkv), generator=gen, device="cuda", dtype=torch.int32)
    dec.load(kc, vc, seg_len, 1, mk(B, n0, Hkv, D), mk(B, n0, Hkv, D))
    assert dec.len.tolist() == [n0] * B
    if eight_bit:
        back = torch.zeros_like(kc), torch.zeros_like(vc)
        pc.pc_kv_read_row8(*dec.prefix, None, P * S * Hkv, kt, 1, D, *back)
        for x, y in zip(back, (kc, vc)):
            x, y = f64(x), f64(y)
            # half a step of the code, and the result's rounding to bf16
            assert np.all(np.abs(x - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * np.abs(y).max(-1, keepdims=True) / 448) + 2.0 ** -8 * np.abs(x))
    tokens, count = torch.empty((B, k + 1), dtype=torch.int32, device="cuda"), torch.empty((B,), dtype=torch.int32, device="cuda")
    ws = pc.alloc_workspace(pc.pc_verify_drafts_workspace_bytes(B, k, V))
    seen = []
    for it in range(5):
        n = 1 if it == 2 else k + 1                                         # one step without drafts
        q, kn, vn = mk(B, n, Hq, D), mk(B, n, Hkv, D), mk(B, n, Hkv, D)
        before = dec.len.clone()
        out = dec.step(q, kn, vn)
        assert torch.equal(dec.len_new, before + n)
        c = {"B": B, "P": P, "nq": n, "Hq": Hq, "Hkv": Hkv, "D": D, "q": q, "pos": before, "pos0": w, "base": base, "own": True,
             "per_head": 1, "seg_len": seg_len, "tail_len": dec.len_new, "tail": tuple(dec.tail),
             "prefix": tuple(dec.prefix) if eight_bit else (*dec.prefix, None, None)}
        check_attention(out, dec.lse.view(-1)[:B * Hq * n].view(B, Hq, n), c, f"step {it}")
        rows = row_values(dec.tail[0], dec.tail[2])
        for b in range(B):
            at = int(before[b])
            want = rotate(f64(kn[b]), w + at + np.arange(n), base).transpose(1, 0, 2)
            top = np.abs(want).max(-1, keepdims=True)
            assert np.all(np.abs(rows[b, 0, :, at:at + n] - want) <= 2.0 ** -4 * np.abs(want) + top / 448 / 1024 + 2e-6 * top)
        if n == 1:
            dec.accept()
            continue
        logits = 2 * torch.randn((B, k + 1, V), generator=gen, device="cuda")
        target = torch.softmax(logits, -1)
        drafted = torch.softmax(logits[:, :k] + torch.randn((B, k, V), generator=gen, device="cuda"), -1)
        draft = torch.randint(0, V, (B, k), generator=gen, device="cuda", dtype=torch.int32)
        draft[:3] = drafted[:3].argmax(-1)
        u, noise = torch.rand((B, k), generator=gen, device="cuda"), torch.empty((B, V), device="cuda").exponential_(generator=gen)
        dec.verify(draft, drafted, target, u, noise, tokens, count, ws)
        want, want_count = verify(*[x.cpu().numpy() for x in (draft, drafted, target, u, noise)])
        assert np.array_equal(tokens.cpu().numpy(), want)
        assert np.array_equal(dec.len.cpu().numpy(), before.cpu().numpy() + 1 + want_count)
        seen.append(want_count)
    assert 0 < np.mean(seen) < k                                            # both kinds of steps were among them
