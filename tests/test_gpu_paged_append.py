"""pc_kv_append_paged against its definition on the CPU: formats, page sizes, trees and chains, strides, unequal numbers of rows,
pages that are not there, offsets beyond 32 bits; what it does not write keeps every bit."""
import numpy as np
import pytest
import torch

import paper_2502_14317_amd as pc
from serving import f64
from trees import append, build

pytestmark = pytest.mark.gpu

# B, n, H_kv, D, page, rows in front (at most), format, tree, ragged, rotate
CASES = [
    (1, 1, 1, 64, 16, 0, "bf16", False, False, False),
    (2, 1, 8, 128, 16, 40, "bf16", False, False, True),
    (3, 17, 3, 64, 32, 100, "row8", True, True, True),
    (5, 64, 2, 128, 16, 50, "bf16", True, True, True),
    (4, 64, 1, 64, 64, 77, "row8", False, False, True),
    (2, 700, 4, 128, 128, 33, "bf16", False, True, True),
    (2, 333, 5, 128, 16, 9, "row8", False, True, False),
    (300, 2, 1, 64, 16, 20, "bf16", True, True, True),
]


def call(c, k_new, v_new, before, n=None):
    cache = pc.make_page_cache(c["k"], c["v"], c["table"], c["k_scale"], c["v_scale"])
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    len_out = torch.full((c["B"],), -9, dtype=torch.int32, device="cuda")
    pc.pc_kv_append_paged(k_new, v_new, c["B"], c["n"], c["Hkv"], c["D"], cache, None if before is None else i32(before), len_out, pos=c["pos"],
                          pos0=c["pos0"], rope_base=c["base"], parent=c["parent"], n_rows=c["n_rows"])
    return len_out


def make(B, n, Hkv, D, page, most, fmt, tree, ragged, rot, gain=2.0):
    c = build(B, n, Hkv, Hkv, D, page, most, fmt, tree, ragged, rot)
    gen = torch.Generator(device="cuda").manual_seed(7)
    new = [(gain * torch.randn((B, n, Hkv, D), generator=gen, device="cuda")).to(torch.bfloat16) for _ in "kv"]
    rows = [n if c["n_rows"] is None else int(c["n_rows"][b]) for b in range(B)]
    return c, new, [int(x) - r for x, r in zip(c["len"], rows)]


def check(c, new, before, got_len, what):
    want, bound, lens = append(dict(c, **c["start"]), *new, before)
    assert got_len.tolist() == lens, what
    for name, w in want.items():
        t = c[name]
        got = f64(t) if t.dtype == torch.bfloat16 else t.cpu().numpy()
        if t.dtype == torch.uint8:                                          # a code's neighbours: one bit of its magnitude apart
            same = (got & 0x80 == w & 0x80) | (got & 0x7f == 0) | (w & 0x7f == 0)
            off = np.abs((got & 0x7f).astype(int) - (w & 0x7f).astype(int))
            assert np.all((off <= bound[name]) & same), f"{what}: codes of {name}"
            assert np.mean(off) < 0.01, f"{what}: more than borders differ in {name}"
        else:
            nan = np.isnan(w)
            assert np.array_equal(nan, np.isnan(got)), f"{what}: {name}, rows written or not"
            assert np.all(np.abs(got - w)[~nan] <= bound[name][~nan]), f"{what}: {name}"


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_against_the_definition(case):
    print("append", case, flush=True)
    c, new, before = make(*case)
    c["start"] = {x: c[x].clone() for x in ("k", "v", "k_scale", "v_scale") if c[x] is not None}
    check(c, new, before, call(c, *new, before), "append")


def test_strides():
    for order in ("packed", "heads first"):
        c, new, before = make(3, 9, 4, 128, 16, 40, "bf16", True, True, True)
        c["start"] = {x: c[x].clone() for x in ("k", "v")}
        if order == "packed":
            qkv = torch.full((3, 9, 16, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
            qkv[:, :, 8:12], qkv[:, :, 12:] = new
            args = qkv[:, :, 8:12], qkv[:, :, 12:]
        else:
            args = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in new]
        check(c, new, before, call(c, *args, before), order)


def test_pages_that_are_not_there_and_no_lengths():
    c, new, before = make(3, 20, 2, 64, 16, 60, "bf16", False, False, True)
    c["table"][0, :2] = -1
    c["table"][1, 1] = c["n_pages"]
    c["table"][2, 0] = -2 ** 31
    c["table"] = c["table"][:, :1 + max(before) // 16].contiguous()          # some of the longest one's rows are behind its last page
    c["start"] = {x: c[x].clone() for x in ("k", "v")}
    check(c, new, before, call(c, *new, before), "missing pages")
    c["start"] = {x: c[x].clone() for x in ("k", "v")}
    check(c, new, [0, 0, 0], call(c, *new, None), "no lengths")


def test_rows_that_are_not_finite_and_zeros():
    c, new, before = make(1, 5, 2, 128, 16, 3, "row8", False, False, False)
    new[0][0, 0, 0, 5], new[1][0, 1, 1, 7], new[0][0, 2] = float("inf"), float("nan"), 0.0
    c["start"] = {x: c[x].clone() for x in ("k", "v", "k_scale", "v_scale")}
    check(c, new, before, call(c, *new, before), "not finite")


def test_nothing_to_append_sets_the_lengths():
    c, _, _ = make(3, 1, 2, 64, 16, 20, "bf16", False, False, False)
    c["n"] = 0
    start = c["k"].clone()
    assert call(c, None, None, [4, 0, -3]).tolist() == [4, 0, 0]
    assert torch.equal(start.view(torch.int16), c["k"].view(torch.int16))


@pytest.mark.parametrize("fmt", ["bf16", "row8"])
def test_pools_beyond_32_bits(fmt):
    c, new, before = make(2, 6, 4, 128, 128, 200, fmt, True, False, True)
    n = 2 ** 32 // (4 * 128 * 128 * (2 if fmt == "bf16" else 1)) + 40
    shift, small = n - c["n_pages"], dict(c)
    big = {x: torch.empty((n, *c[x].shape[1:]), dtype=c[x].dtype, device="cuda") for x in ("k", "v", "k_scale", "v_scale") if c[x] is not None}
    for x, t in big.items():
        t[shift:] = c[x]
    call(small, *new, before)
    call(dict(c, **big, table=torch.where(c["table"] >= 0, c["table"] + shift, -1)), *new, before)
    bits = {torch.bfloat16: torch.int16, torch.float32: torch.int32, torch.uint8: torch.uint8}
    for x, t in big.items():
        assert torch.equal(t[shift:].view(bits[t.dtype]), small[x].view(bits[t.dtype])), x


def test_graph_and_stream():
    c, new, before = make(4, 5, 2, 128, 16, 40, "row8", True, True, True)
    cache = pc.make_page_cache(c["k"], c["v"], c["table"], c["k_scale"], c["v_scale"])
    lens, out = torch.tensor(before, dtype=torch.int32, device="cuda"), torch.zeros((4,), dtype=torch.int32, device="cuda")
    run = lambda: pc.pc_kv_append_paged(*new, 4, 5, 2, 128, cache, lens, out, pos=c["pos"], pos0=c["pos0"], rope_base=c["base"],
                                        parent=c["parent"], n_rows=c["n_rows"])
    names = ("k", "v", "k_scale", "v_scale")
    start = {x: c[x].clone() for x in names}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    want = {x: c[x].clone() for x in names}
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for x in names:
            c[x].copy_(start[x])
        graph.replay()
        torch.cuda.synchronize()
        for x in names:
            assert torch.equal(c[x].view(torch.uint8), want[x].view(torch.uint8)), x


def test_tensors_of_another_gpu_are_refused():
    """(One GPU is enough: what stands for the current one's number is another.)"""
    k = torch.zeros((3, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
    cache = pc.make_page_cache(k, k.clone(), torch.zeros((2, 1), dtype=torch.int32, device="cuda"))
    for refused in (lambda: pc.binding._pages_fit(cache, 2, 1, 64, 7), lambda: pc.binding._flat(cache.tensors[2], 2, torch.int32, "table", 7),
                    lambda: pc.binding._strided(k, k.shape, torch.bfloat16, "k", 7), lambda: pc.binding._ws(k, 7)):
        with pytest.raises(ValueError, match="current GPU"):
            refused()
