"""pc_shared_attn with values of 2^119 (and of 2^-100): logits that rise a little above a row's first ones must not push its sums of
probabilities times values beyond fp32, where the result is far inside it.

Only value 0 of a query row is not 0, and value 0 of the keys says whether a key's logit is 0 or 7.5 (log2 units): blocks of 64
keys in turn, so that every longer run of keys starts low somewhere.  Scaling values by a power of two changes no rounding, so
the bounds are those of values around 1."""
import math

import pytest
import torch

from shared_bodies import CASES, build, check
from test_gpu_shared_attn_bodies import call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [119, -100])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_values_far_from_one(case, size):
    print("large values", case, size, flush=True)
    c = build(case, False, value=2.0 ** size)
    c["q"].zero_()
    c["q"][..., 0] = 7.5 * math.log(2.0) * math.sqrt(c["D"])
    for rows in (c["prefix"], c["tail"]):
        if rows:
            high = torch.arange(rows[0].shape[3], device="cuda") % 128 >= 64
            if rows[2] is None:
                rows[0][..., 0] = high.to(torch.bfloat16)
            else:
                rows[0][..., 0] = 0x38 * high.to(torch.uint8)               # 1
                rows[2].fill_(1.0)
    out, lse = call(c)
    check(out.float().cpu().numpy(), lse.cpu().numpy(), c, f"values of 2^{size}")
