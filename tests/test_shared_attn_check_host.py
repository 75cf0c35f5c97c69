"""The cases that stand for the bodies of pc_shared_attn reach each of them, and the comparison that they are held to
notices mistakes, planted in a statement of the arithmetic on the CPU."""
import numpy as np
import pytest

from shared_bodies import CASES, EVERY, build, check, each_softmax, kinds, softmax_rows


def test_every_body_is_reached():
    reached = set().union(*(kinds(c) for c in CASES))
    assert EVERY - reached == set() and reached - EVERY == set()


def bf16(x):
    """Nearest bf16 value, ties to even."""
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7fff + (u >> 16 & 1)) & 0xffff0000).view(np.float32).astype(np.float64)


def emulate(c, parts, slip=1.0, lost=1.0):
    """The kernels' roundings: query rows in bf16 parts, P and the result in bf16.  slip: what a reference that moves at the
    last key leaves of the keys in front where it should leave all; lost: of the logits."""
    out, lse = np.zeros((c["B"], c["nq"], c["Hq"], c["D"])), np.full((c["B"], c["Hq"], c["nq"]), -np.inf)
    G = c["Hq"] // c["Hkv"]
    for b, g, k, v, q, seen in each_softmax(c):
        if not k.shape[0]:
            continue
        if c["pos"] is not None:
            hi = bf16(q)
            q = hi + bf16(q - hi) if parts == 2 else hi
        _, s, p, _ = softmax_rows(k, v, lost * q, seen, c["D"] ** -0.5)
        p[:, :-1] *= slip
        heads = slice(g * G, (g + 1) * G)
        out[b][:, heads] = bf16(bf16(p) @ v).reshape(c["nq"], G, -1)
        lse[b][heads] = s.reshape(c["nq"], G).T
    return out, lse


SOME = [CASES[12], CASES[16], CASES[24], CASES[34]]


@pytest.mark.parametrize("gain", [2.0, 60.0])
@pytest.mark.parametrize("rotated", [False, True])
@pytest.mark.parametrize("case", SOME, ids=lambda c: "-".join(map(str, c)))
def test_right_results_pass_and_mistakes_do_not(case, rotated, gain):
    c = build(case, rotated, gain, device="cpu")
    out, lse = emulate(c, 2)
    check(out, lse, c, "right")
    mistakes = [(0 * out, lse), (1.02 * out, lse), (out, lse + 0.05), emulate(c, 2, slip=0.9), emulate(c, 2, lost=0.99)]
    if rotated and gain > 2.0:
        mistakes.append(emulate(c, 1))                                      # the second part of the query rows is lost
    for i, wrong in enumerate(mistakes):
        with pytest.raises(AssertionError):
            check(*wrong, c, f"mistake {i}")
