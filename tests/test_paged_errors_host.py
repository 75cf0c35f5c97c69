"""Argument errors of the operators of drafted trees over a paged cache: all of them are found on the host, before any launch, and
an argument list that is right up to its workspace ends in the workspace error."""
import ctypes

import pytest
import torch

import paper_2502_14317_amd as pc
from paper_2502_14317_amd import binding
from paper_2502_14317_amd.layer import PagedTreeDecoder

LATER = ctypes.c_void_p(260)                                                # the entry behind ONE's first
ONE, ODD, TWO, TOP = ctypes.c_void_p(256), ctypes.c_void_p(264), ctypes.c_void_p(258), ctypes.c_void_p(255)       # never dereferenced
OK, NULL, SHAPE, WORKSPACE = 0, -1, -2, -3
nan, inf = float("nan"), float("inf")

PAGES = dict(k=ONE, v=ONE, k_scale=None, v_scale=None, table=ONE, n_pages=50, page=64, max_pages=9)
APPEND = dict(k_new=ONE, v_new=ONE, batch_stride=0, row_stride=0, head_stride=0, parent=None, n_rows=None, pos=None, pos0=0, rope_base=1e4,
              batch=2, n_new=3, n_kv_heads=2, head_dim=64, cache=None, len_in=None, len_out=None, stream=None)
ATTN = dict(q=ONE, batch_stride=0, row_stride=0, parent=None, n_rows=None, pos=None, pos0=0, rope_base=1e4, softmax_scale=0.0, cache=None,
            len=ONE, batch=6, n=5, n_q_heads=8, n_kv_heads=2, head_dim=128, out=ONE, lse_out=None, ws=ONE, ws_bytes=0, stream=None)
LOGPROBS = dict(logits=ONE, logits_fp32=0, row_stride=0, tokens=ONE, n_tokens=2, n_top=5, rows=7, vocab=1000, token_logprob=ONE,
                entropy=ONE, top_idx=ONE, top_logprob=ONE, ws=ONE, ws_bytes=0, stream=None)
ACCEPT = dict(tokens=ONE, parent=None, choice=ONE, choice_stride=1, n_rows=None, batch=0, n=5, cache=None, n_kv_heads=2, head_dim=64,
              len_in=ONE, len_out=None, pos=None, path=ONE, n_kept=ONE, next_token=ONE, stream=None)


def _call(fn, base, pages={}, **change):
    cache = None if pages is None else ctypes.byref(pc.pc_page_cache(*dict(PAGES, **pages).values()))
    args = dict(base, **change)
    if "cache" in args:
        args["cache"] = cache
    return getattr(pc.lib(), fn)(*args.values())


BAD_PAGES = [{"pages": {"page": x}} for x in (0, 8, 24, 100, -16, 1 << 17)] + [{"pages": {"n_pages": 0}}, {"pages": {"max_pages": 0}},
                                                                           {"pages": {"max_pages": 1 << 25}}]
BAD_MEMORY = [{"pages": {"k": ODD}}, {"pages": {"v": TWO}}, {"pages": {"table": TWO}}, {"pages": {"k_scale": TWO, "v_scale": ONE}}]
NO_MEMORY = [{"pages": {x: None}} for x in ("k", "v", "table")] + [{"pages": {"k_scale": ONE}}, {"pages": {"v_scale": ONE}}]


@pytest.mark.parametrize("fn,base,want,changes", [
    ("pc_kv_append_paged", APPEND, OK, [{"batch": 0, "k_new": None}, {"n_new": 0, "k_new": None, "pages": {"k": None}}]),
    ("pc_kv_append_paged", APPEND, NULL, [{"k_new": None}, {"v_new": None}, {"pages": None}] + NO_MEMORY),
    ("pc_kv_append_paged", APPEND, SHAPE, BAD_PAGES + BAD_MEMORY +
     [{"batch": -1}, {"batch": (1 << 20) + 1}, {"n_new": -1}, {"n_kv_heads": 0}, {"n_kv_heads": 1 << 17}, {"head_dim": 96},
      {"batch": 1 << 20, "n_new": 1 << 12}, {"parent": ONE, "n_new": 65}, {"row_stride": 4}, {"head_stride": -8}, {"batch_stride": 1 << 41},
      {"pos": ONE, "rope_base": 1.0}, {"pos": ONE, "rope_base": nan}, {"k_new": ODD}, {"v_new": TWO}, {"parent": TWO}, {"n_rows": TWO},
      {"pos": TWO}, {"len_in": TWO}, {"len_out": TWO}, {"len_in": ONE, "len_out": ONE}, {"len_in": ONE, "len_out": LATER},
      {"len_in": LATER, "len_out": ONE}]),
    ("pc_tree_attn", ATTN, WORKSPACE, [{}, {"ws": None, "ws_bytes": 1 << 40}, {"ws": ctypes.c_void_p(128), "ws_bytes": 1 << 40},
                                       {"pages": {"k_scale": ONE, "v_scale": ONE}}, {"pos": ONE, "parent": ONE, "n_rows": ONE},
                                       {"n": 64}, {"batch_stride": 1 << 20, "row_stride": 1536}]),
    ("pc_tree_attn", ATTN, NULL, [{"q": None}, {"out": None}, {"len": None}, {"pages": None}] + NO_MEMORY),
    ("pc_tree_attn", ATTN, SHAPE, BAD_PAGES + BAD_MEMORY +
     [{"batch": 0}, {"batch": (1 << 20) + 1}, {"n": 0}, {"n": 65}, {"n_q_heads": 7}, {"n_kv_heads": 0}, {"head_dim": 32}, {"n_q_heads": 1 << 21},
      {"batch": 1 << 20, "n": 64}, {"batch": 1 << 18, "pages": {"max_pages": 1 << 13}}, {"softmax_scale": -1.0}, {"softmax_scale": nan},
      {"softmax_scale": inf}, {"row_stride": 12}, {"batch_stride": -16}, {"pos": ONE, "rope_base": 0.5}, {"q": ODD}, {"out": ODD}, {"len": TWO},
      {"parent": TWO}, {"n_rows": TWO}, {"pos": TWO}, {"lse_out": TWO}]),
    ("pc_token_logprobs", LOGPROBS, OK, [{"rows": 0, "logits": None}]),
    ("pc_token_logprobs", LOGPROBS, WORKSPACE, [{}, {"ws": None, "ws_bytes": 1 << 40}, {"ws": ctypes.c_void_p(64), "ws_bytes": 1 << 40},
                                                {"logits": TWO}, {"logits_fp32": 1}, {"n_tokens": 0, "tokens": None, "token_logprob": None},
                                                {"n_top": 0, "top_idx": None, "top_logprob": None}, {"entropy": None, "top_logprob": None}]),
    ("pc_token_logprobs", LOGPROBS, NULL, [{"logits": None}, {"tokens": None}, {"token_logprob": None}, {"top_idx": None},
                                           {"n_tokens": 0, "n_top": 0, "entropy": None}]),
    ("pc_token_logprobs", LOGPROBS, SHAPE,
     [{"rows": -1}, {"rows": (1 << 21) + 1}, {"vocab": 0}, {"vocab": (1 << 24) + 1}, {"n_top": -1}, {"n_top": 65}, {"n_top": 5, "vocab": 4},
      {"logits_fp32": 2}, {"n_tokens": -1}, {"n_tokens": 65537}, {"row_stride": 999}, {"row_stride": -1}, {"row_stride": 1 << 41}, {"logits": TOP},
      {"logits": TWO, "logits_fp32": 1}, {"tokens": TWO}, {"entropy": TWO}, {"top_idx": TWO}, {"top_logprob": TWO}, {"token_logprob": TWO}]),
    ("pc_tree_accept", ACCEPT, OK, [{}, {"pages": None}, {"tokens": None, "path": None}]),
    ("pc_tree_accept", ACCEPT, NULL, [dict({x: None}, batch=3) for x in ("tokens", "choice", "path", "n_kept", "next_token", "len_in")] +
     [dict(x, batch=3) for x in NO_MEMORY]),
    ("pc_tree_accept", ACCEPT, SHAPE, [dict(x, batch=3) for x in BAD_PAGES + BAD_MEMORY] +
     [{"batch": -1}, {"batch": (1 << 20) + 1}, {"n": 0}, {"n": 65}, {"choice_stride": 0}, {"batch": 3, "n_kv_heads": 0}, {"batch": 3, "head_dim": 96},
      {"batch": 1 << 20, "n_kv_heads": 64}] + [dict({x: TWO}, batch=3) for x in ("tokens", "parent", "choice", "n_rows", "len_in", "len_out", "pos",
                                                                                  "path", "n_kept", "next_token")] +
     [dict(x, batch=3) for x in ({"len_out": ONE}, {"len_out": LATER}, {"pos": ONE}, {"pos": ODD}, {"len_out": ctypes.c_void_p(512), "pos": ctypes.c_void_p(508)})]),
])
def test_refusals(fn, base, want, changes):
    for change in changes:
        assert _call(fn, base, **change) == want, change


def test_workspaces():
    cache = lambda **c: ctypes.byref(pc.pc_page_cache(*dict(PAGES, **c).values()))
    need = pc.lib().pc_tree_attn_workspace_bytes
    small, wide = need(cache(), 6, 5, 8, 2, 128), need(cache(max_pages=900), 6, 5, 8, 2, 128)
    assert 0 < small <= wide and need(cache(), 6, 65, 8, 2, 128) == 0 and need(cache(page=20), 6, 5, 8, 2, 128) == 0 and need(None, 6, 5, 8, 2, 128) == 0
    assert need(cache(max_pages=8), 1 << 20, 1, 31, 31, 128) > 0            # more sequences and heads than a launch has workgroups
    need = pc.pc_token_logprobs_workspace_bytes
    assert need(3, 100000, 20) > 0 and need(3, 10, 11) == 0 and need(-1, 10, 1) == 0


def test_page_caches_are_checked():
    k, t = torch.zeros((5, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((3, 4), dtype=torch.int32)
    for args in ((k, k[:4], t), (k[0], k[0], t), (k.float(), k.float(), t), (k, k, t, torch.zeros(5, 2, 16), torch.zeros(5, 2, 16)),
                 (k.byte(), k.byte(), t), (k.byte(), k.byte(), t, torch.zeros(5, 2, 15), torch.zeros(5, 2, 15)), (k, k, t.long()), (k, k, t[0])):
        with pytest.raises(ValueError):
            pc.make_page_cache(*args)
    with pytest.raises(ValueError, match="GPU"):
        pc.make_page_cache(k, k, t)


def test_tensors_are_checked_before_the_library_gets_addresses():
    with pytest.raises(ValueError, match="rows"):
        binding._flat(torch.zeros(3, dtype=torch.int64), 3, torch.int32, "rows")
    with pytest.raises(ValueError, match="rows"):
        binding._flat(torch.zeros(4, dtype=torch.int32), 3, torch.int32, "rows")
    with pytest.raises(ValueError, match="GPU"):
        binding._strided(torch.zeros((2, 3)), (2, 3), torch.float32, "q")
    with pytest.raises(ValueError, match="neither"):
        pc.pc_token_logprobs(torch.zeros((2, 3), dtype=torch.float16), 2, 3, None, 0, 1, None, None, None, None, None)


def decoder(**more):
    return PagedTreeDecoder(4, 10, 16, 6, 8, 2, 64, 1e4, **dict(dict(max_rows=3, device="cpu"), **more))


def rows(n, B=4, Hq=8, Hkv=2, D=64, dtype=torch.bfloat16):
    t = lambda H: torch.zeros((B, n, H, D), dtype=dtype)
    return t(Hq), t(Hkv), t(Hkv)


@pytest.mark.parametrize("args", [rows(0), rows(4), rows(1, B=5), rows(1, Hq=4), rows(2, D=128), (rows(2)[0], *rows(1)[1:]), rows(1, dtype=torch.float32)],
                         ids=lambda a: "-".join(str(tuple(x.shape)) for x in a))
def test_steps_of_another_shape(args):
    d = decoder()
    with pytest.raises(ValueError, match="rows of this decoder"):
        d.step(*args)
    assert len(d.free) == 10


def test_trees_of_another_shape_and_sequences_that_are_not_loaded():
    d = decoder()
    for more in ({"parent": torch.zeros((4, 3), dtype=torch.int32)}, {"parent": torch.zeros((4, 2))}, {"n_rows": torch.zeros((3,), dtype=torch.int32)}):
        with pytest.raises(ValueError):
            d.step(*rows(2), **more)
    with pytest.raises(ValueError, match="not loaded"):
        d.step(*rows(2))
    with pytest.raises(ValueError, match="no step"):
        d.accept(torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2), dtype=torch.int32))


def test_loads_that_do_not_fit():
    d, mk = decoder(), lambda *s, **k: torch.zeros(s, dtype=k.get("dtype", torch.bfloat16))
    d.reserve(0, 70)
    assert len(d.free) == 5 and d.table[0].tolist() == d.pages[0] + [-1]
    for kc, more in ((mk(2, 2, 49, 64), {}), (mk(7, 2, 16, 64), {}), (mk(1, 3, 5, 64), {}), (mk(2, 5, 64), {}), (mk(1, 2, 5, 64, dtype=torch.float32), {}),
                     (mk(2, 2, 5, 64), {"seg_len": [5]}), (mk(1, 2, 5, 64), {"seg_len": [6]}), (mk(1, 2, 5, 64), {"k_tail": mk(1, 2, 64)}),
                     (mk(1, 2, 5, 64), {"k_tail": mk(1, 3, 64), "v_tail": mk(1, 3, 64)})):
        with pytest.raises(ValueError):
            d.load(1, kc, kc, 0, **more)
    with pytest.raises(ValueError):
        d.reserve(1, 97)
    with pytest.raises(ValueError):
        d.reserve(1, 81)
    assert len(d.free) == 5 and d.pages[1] is None
    d.release(0)
    assert len(d.free) == 10 and (d.table == -1).all()
