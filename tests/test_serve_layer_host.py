"""SharedPrefixDecoder refuses what is not its shape before it touches the caches."""
import pytest
import torch

from paper_2502_14317_amd.layer import SharedPrefixDecoder


def make():
    return SharedPrefixDecoder(4, 2, 3, 16, 32, 8, 2, 64, 1e4, 100, max_rows=3, device="cpu")


def rows(n, B=4, Hq=8, Hkv=2, D=64):
    t = lambda H: torch.zeros((B, n, H, D), dtype=torch.bfloat16)
    return t(Hq), t(Hkv), t(Hkv)


def test_step_before_load():
    with pytest.raises(ValueError, match="load"):
        make().step(*rows(1))


@pytest.mark.parametrize("args", [rows(0), rows(4), rows(1, B=5), rows(1, Hq=4), rows(2, D=128), (rows(2)[0], *rows(1)[1:]),
                                  (*rows(1)[:2], rows(2)[2])], ids=lambda a: "-".join(str(tuple(x.shape)) for x in a))
def test_step_of_another_shape(args):
    d = make()
    d.prefix_rows = object()                                                # (as after a load)
    with pytest.raises(ValueError, match="rows of this decoder"):
        d.step(*args)
    assert not d.len_new.any()
