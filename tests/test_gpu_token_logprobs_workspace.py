"""pc_token_logprobs in the workspace that it asks for and not a byte more, at the borders between rows that are cut and rows that are not."""
import pytest
import torch

import paper_2502_14317_amd as pc
from test_gpu_token_logprobs import call, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab", [(1, 49152), (1, 49153), (1, 98304), (2, 98305), (5, 300001), (63, 60000), (64, 60000), (65, 60000), (64, 128256), (200, 128256)])
@pytest.mark.parametrize("n_top", [0, 64])
def test_nothing_behind_the_workspace(rows, vocab, n_top, dtype):
    print("logprobs workspace", rows, vocab, n_top, dtype, flush=True)
    logits, tokens = make(rows, vocab, dtype, 9)
    want = call(logits, tokens, n_top)[:4]
    size = pc.pc_token_logprobs_workspace_bytes(rows, vocab, n_top)
    whole = torch.full((size + (1 << 16),), 0x5a, dtype=torch.uint8, device="cuda")
    got = [torch.zeros_like(x) for x in want]
    pc.pc_token_logprobs(logits, rows, vocab, tokens, 3, n_top, got[0], got[1], got[2] if n_top else None, got[3] if n_top else None, whole[:size])
    assert (whole[size:] == 0x5a).all()
    assert all(torch.equal(x.view(torch.int32), y.view(torch.int32)) for x, y in zip(got, want))
    with pytest.raises(pc.PcError):
        pc.pc_token_logprobs(logits, rows, vocab, tokens, 3, n_top, got[0], got[1], got[2] if n_top else None, got[3] if n_top else None, whole[:255])
