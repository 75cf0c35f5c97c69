"""Argument errors of the serving operators: all of them are found on the host, before any launch, and an argument list
that is right up to its workspace ends in the workspace error."""
import ctypes

import pytest
import torch

import paper_2502_14317_amd as pc

ONE, ODD, TWO = ctypes.c_void_p(256), ctypes.c_void_p(264), ctypes.c_void_p(258)          # never dereferenced
OK, NULL, SHAPE, WORKSPACE = 0, -1, -2, -3
nan, inf = float("nan"), float("inf")

ROWS = dict(k=ONE, v=ONE, k_scale=None, v_scale=None, seg_len=None, seg_len_per_head=0, n_seg=2, cap=64)
ATTN = dict(q=ONE, q_pos=None, pos0=0, rope_base=1e4, softmax_scale=0.0, prefix=None, tail=None, tail_own=1, batch=6, n_prefix=2,
            n_q=2, n_q_heads=8, n_kv_heads=2, head_dim=128, out=ONE, lse_out=None, ws=ONE, ws_bytes=0, stream=None)


def _rows(none=False, **change):
    return None if none else ctypes.byref(pc.pc_row_cache(*dict(ROWS, **change).values()))


def _attn(prefix={}, tail={}, **change):
    return pc.lib().pc_shared_attn(*dict(ATTN, prefix=_rows(**prefix), tail=_rows(**dict(dict(n_seg=1), **tail)), **change).values())


@pytest.mark.parametrize("want,changes", [
    (WORKSPACE, [{}, {"ws": None, "ws_bytes": 1 << 40}, {"ws": ctypes.c_void_p(128), "ws_bytes": 1 << 40}, {"prefix": {"none": True}},
                 {"tail": {"none": True}, "tail_own": 0}, {"prefix": {"k_scale": ONE, "v_scale": ONE}}, {"q_pos": ONE}]),
    (NULL, [{"q": None}, {"out": None}] + [{w: {k: None}} for w in ("prefix", "tail") for k in ("k", "v")]
     + [{"prefix": {"k_scale": ONE}}, {"tail": {"v_scale": ONE}}]),
    (SHAPE, [{"batch": 0}, {"batch": 5}, {"n_prefix": 0}, {"n_q": 0}, {"n_q_heads": 7}, {"n_kv_heads": 0}, {"head_dim": 96},
             {"batch": (1 << 20) + 2}, {"n_q": 1 << 21}, {"batch": 1 << 20, "n_q": 4}, {"tail_own": 2}, {"tail": {"none": True}},
             {"prefix": {"none": True}, "tail": {"none": True}, "tail_own": 0}, {"softmax_scale": -1.0}, {"softmax_scale": nan},
             {"softmax_scale": inf}, {"q_pos": ONE, "rope_base": 1.0}, {"q_pos": ONE, "rope_base": nan}, {"prefix": {"n_seg": -1}},
             {"prefix": {"cap": 0}}, {"prefix": {"cap": (1 << 24) + 1}}, {"prefix": {"seg_len_per_head": 2}}, {"tail": {"n_seg": 2}},
             {"prefix": {"n_seg": 1 << 20, "cap": 1 << 24}}, {"q": ODD}, {"out": ODD}, {"prefix": {"k": ODD}}, {"tail": {"v": ODD}},
             {"prefix": {"seg_len": TWO}}, {"lse_out": TWO}, {"q_pos": TWO}]),
])
def test_shared_attn(want, changes):
    for change in changes:
        assert _attn(**change) == want, change


APPEND = dict(k_new=ONE, v_new=ONE, pos=None, pos0=0, rope_base=1e4, batch=2, n_new=3, cap=8, n_kv_heads=2, head_dim=64, k8=ONE, v8=ONE,
              k_scale=ONE, v_scale=ONE, len_in=None, len_out=None, stream=None)
READ = dict(k8=ONE, v8=ONE, k_scale=ONE, v_scale=ONE, seg_len=None, batch=2, cap=8, n_kv_heads=2, head_dim=64, k=ONE, v=ONE, stream=None)
VERIFY = dict(draft=ONE, draft_len=None, draft_prob=ONE, target_prob=ONE, u=ONE, noise=ONE, batch=2, n_draft=3, vocab=100, tokens=ONE,
              n_accepted=ONE, len_in=None, len_out=None, ws=ONE, ws_bytes=0, stream=None)


def _call(fn, base, **change):
    return getattr(pc.lib(), fn)(*dict(base, **change).values())


@pytest.mark.parametrize("fn,base,want,changes", [
    ("pc_kv_append_row8", APPEND, OK, [{"batch": 0, "k_new": None}, {"n_new": 0, "k_new": None}]),
    ("pc_kv_append_row8", APPEND, NULL, [{k: None} for k in ("k_new", "v_new", "k8", "v8", "k_scale", "v_scale")]),
    ("pc_kv_append_row8", APPEND, SHAPE,
     [{"batch": -1}, {"n_new": -1}, {"cap": 0}, {"n_kv_heads": 0}, {"head_dim": 32}, {"pos": ONE, "rope_base": 0.5}, {"k_new": ODD},
      {"k8": ODD}, {"k_scale": TWO}, {"len_in": TWO}, {"len_in": ONE, "len_out": ONE}, {"batch": 1 << 20, "n_new": 1 << 20}]),
    ("pc_kv_read_row8", READ, OK, [{"batch": 0, "k": None}]),
    ("pc_kv_read_row8", READ, NULL, [{k: None} for k in ("k8", "v8", "k_scale", "v_scale", "k", "v")]),
    ("pc_kv_read_row8", READ, SHAPE, [{"batch": -1}, {"cap": 0}, {"n_kv_heads": 0}, {"head_dim": 96}, {"k": ODD}, {"v8": ODD},
                                      {"v_scale": TWO}, {"seg_len": TWO}, {"batch": 1 << 20, "cap": 1 << 24}]),
    ("pc_verify_drafts", VERIFY, WORKSPACE, [{}, {"ws": None, "ws_bytes": 1 << 40}, {"ws": ctypes.c_void_p(8), "ws_bytes": 1 << 40},
                                             {"draft_prob": None}, {"n_draft": 0, "draft": None, "u": None}]),
    ("pc_verify_drafts", VERIFY, NULL, [{k: None} for k in ("draft", "target_prob", "u", "noise", "tokens", "n_accepted")]
     + [{"len_in": ONE}, {"len_out": ONE}]),
    ("pc_verify_drafts", VERIFY, SHAPE, [{"batch": 0}, {"n_draft": -1}, {"vocab": 0}, {"vocab": (1 << 24) + 1}, {"batch": 1 << 21},
                                         {"draft": TWO}, {"u": TWO}, {"target_prob": TWO}]),
])
def test_rows_and_verification(fn, base, want, changes):
    for change in changes:
        assert _call(fn, base, **change) == want, change


def test_workspaces():
    rows = lambda **c: ctypes.byref(pc.pc_row_cache(*dict(ROWS, **c).values()))
    need = pc.lib().pc_shared_attn_workspace_bytes
    assert need(rows(cap=4096), rows(n_seg=1), 6, 2, 2, 8, 2, 128) >= 6 * 2 * 8 * 2 * (128 + 1) * 4        # two partials a row at least
    assert need(rows(), rows(n_seg=1), 6, 2, 2, 8, 2, 128) > 0
    assert need(rows(), rows(n_seg=1), 5, 2, 2, 8, 2, 128) == 0 and need(rows(cap=0), None, 6, 2, 2, 8, 2, 128) == 0
    assert pc.pc_verify_drafts_workspace_bytes(4, 3, 1000) > 0 and pc.pc_verify_drafts_workspace_bytes(0, 3, 1000) == 0


def test_row_caches_are_checked():
    k = torch.zeros((2, 1, 2, 8, 64), dtype=torch.bfloat16)
    for args in ((k, k.view(2, 2, 1, 8, 64)), (k[0], k[0]), (k.float(), k.float()), (k, k, torch.zeros(2, 1, 2, 8)),
                 (k.byte(), k.byte()), (k.byte(), k.byte(), torch.zeros(2, 1, 2, 7), torch.zeros(2, 1, 2, 7))):
        with pytest.raises(ValueError):
            pc.make_row_cache(*args)
    with pytest.raises(ValueError):
        pc.make_row_cache(k, k)                                             # not on a GPU
