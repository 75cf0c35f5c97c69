"""pc_tree_attn where a sequence is said to be longer than its table, whose places end in the middle of a block of 32 keys (an odd
number of pages of 16 rows): what is not there is seen by nobody, in every body and format."""
import pytest
import torch

from test_gpu_tree_attn import NO, call
from trees import build, check_attention

pytestmark = pytest.mark.gpu

# n, H_q, H_kv, D, format: 4, 32, 32 rows a KV head (the last also through LDS where tables are wide), 64, 128 and two tiles of them
SHAPES = [(1, 4, 1, 128, "bf16"), (1, 4, 1, 64, "row8"), (8, 4, 1, 64, "row8"), (8, 4, 1, 128, "bf16"), (16, 8, 2, 128, "bf16"), (16, 4, 1, 64, "row8"),
          (32, 4, 1, 128, "bf16"), (32, 4, 1, 128, "row8"), (32, 4, 1, 64, "row8"), (40, 4, 1, 64, "bf16"), (40, 4, 1, 128, "row8")]


def first_page_is_nobodys(c):
    """Swaps page 0 of the pools with one that no table has: its rows, and in 8 bits their scales, are NaN."""
    held = set(c["table"].flatten().tolist())
    spare = next(p for p in range(c["n_pages"]) if p not in held)
    if 0 in held:
        for name in ("k", "v", "k_scale", "v_scale"):
            if c[name] is not None:
                c[name][[0, spare]] = c[name][[spare, 0]]
        c["table"][c["table"] == 0] = spare


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("pages", [1, 3, 31, 33, 131])
def test_tables_that_end_inside_a_block(pages, shape):
    n, Hq, Hkv, D, fmt = shape
    print("short tables", pages, shape, flush=True)
    c = build(2, n, Hq, Hkv, D, 16, 0, fmt, True, False, True, gain=0.3,
              lens=[16 * pages, 16 * pages])                                # logits near 0, the value that rows which are not there would have
    c["table"] = c["table"][:, :pages].contiguous()
    first_page_is_nobodys(c)
    c["len"].copy_(torch.tensor([16 * pages + n + 40, 16 * pages + n + 16]))
    out, lse, _ = call(c)
    check_attention(out, lse, c, "short tables", NO)
    c["len"].fill_(2 ** 31 - 1)                                             # the same rows are there
    far, far_lse, _ = call(c)
    assert torch.equal(far, out) and torch.equal(far_lse, lse)
