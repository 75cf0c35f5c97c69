"""Host orchestration of one ParallelComp layer over the C-ABI calls (section 3.1 of the paper):
chunk-batched local attention with fused query scores -> chunk selection -> per-head token
selection -> KV compaction -> global attention of the query over the surviving KV.
All arithmetic happens inside the library's kernels; this class only owns buffers."""
import torch

from . import binding as B


class ParallelCompLayer:
    def __init__(self, n_chunks, chunk_len, query_len, n_q_heads, n_kv_heads, head_dim,
                 obs_window, rope_base, keep_chunks, keep_tokens, softmax_scale=0.0,
                 device="cuda", calibration=None):
        self.C, self.w, self.wq = n_chunks, chunk_len, query_len
        self.L = chunk_len + query_len
        self.Hq, self.Hkv, self.D = n_q_heads, n_kv_heads, head_dim
        self.kc_n, self.kt_n = keep_chunks, keep_tokens
        self.rope_base, self.scale = rope_base, softmax_scale
        self.calibration = calibration          # None or (lambda, class_lo, class_hi) of Eq. 8
        self.chunk_lens = None                  # set by chunk_prefill for ragged chunks
        self.first_len = chunk_len
        self.shape = B.make_shape(n_chunks, chunk_len, query_len, n_q_heads, n_kv_heads, head_dim,
                                  obs_window, rope_base, softmax_scale)
        dev, bf, f32, i32 = device, torch.bfloat16, torch.float32, torch.int32
        C, L, Hq, Hkv, D = self.C, self.L, self.Hq, self.Hkv, self.D
        self.o = torch.empty((C, L, Hq, D), dtype=bf, device=dev)
        self.lse = torch.empty((C, Hq, L), dtype=f32, device=dev)
        self.k_rope = torch.empty((C, L, Hkv, D), dtype=bf, device=dev)
        self.tok_score = torch.empty((C, Hkv, chunk_len), dtype=f32, device=dev)
        self.chunk_score = torch.empty((C,), dtype=f32, device=dev)
        ws = B.pc_chunk_prefill_workspace_bytes(self.shape)
        if keep_chunks > 0:
            self.chunk_idx = torch.empty((keep_chunks,), dtype=i32, device=dev)
            self.chunk_top = torch.empty((keep_chunks,), dtype=f32, device=dev)
            self.tok_idx = torch.empty((keep_chunks, Hkv, keep_tokens), dtype=i32, device=dev)
            self.tok_cnt = torch.empty((keep_chunks, Hkv), dtype=i32, device=dev)
            self.kc = torch.empty((1, keep_chunks, Hkv, keep_tokens, D), dtype=bf, device=dev)
            self.vc = torch.empty_like(self.kc)
            self.global_o = torch.empty((1, query_len, Hq, D), dtype=bf, device=dev)
            self.global_lse = torch.empty((1, Hq, query_len), dtype=f32, device=dev)
            # room for the attention call's workspace behind the prefill's
            ws = max(ws, B.pc_layer_workspace_bytes(self.shape, keep_chunks, keep_tokens))
        self.ws = B.alloc_workspace(ws, dev)

    def chunk_prefill(self, q, k, v, with_scores=True, chunk_lens=None, first_len=None):
        """Eq. 1-2 and 5-6 for all chunks: fills o, lse, k_rope, tok_score, chunk_score.
        chunk_lens [C] int32 (device): ragged chunks, see pc_chunk_prefill_attn; first_len is
        chunk_lens[0] as a host integer (where chunk 0's query rows sit; default w)."""
        self.chunk_lens = chunk_lens
        self.first_len = self.w if first_len is None else int(first_len)
        B.pc_chunk_prefill_attn(self.shape, q, k, v, self.o, self.lse, self.k_rope,
                                self.tok_score if with_scores else None,
                                self.chunk_score if with_scores else None, self.ws,
                                chunk_lens=chunk_lens)

    def evict_and_attend(self, q, v):
        """Eq. 3-4 mechanics, Eq. 7 (after Eq. 8 when calibration is set) and Eq. 9-11 on the
        results of chunk_prefill."""
        C, L, w = self.C, self.L, self.w
        B.pc_select_chunks_topk(self.chunk_score, C, self.kc_n, self.chunk_idx, self.chunk_top)
        if self.calibration is None and self.chunk_lens is None:
            B.pc_select_tokens_topk(self.tok_score, self.chunk_idx, self.kc_n, self.Hkv, w,
                                    self.kt_n, self.tok_idx)
            seg_len, per_head = None, 0
        else:
            lam, lo, hi = self.calibration if self.calibration is not None else (float("inf"), 0, 0)
            B.pc_select_tokens_calibrated(self.tok_score, self.chunk_idx, self.kc_n, self.Hkv, w,
                                          self.kt_n, lam, lo, hi, self.tok_idx, self.tok_cnt,
                                          chunk_lens=self.chunk_lens)
            seg_len, per_head = self.tok_cnt, 1
        B.pc_gather_kv(self.k_rope, v, self.chunk_idx, self.tok_idx, 1, C, L, self.kc_n, self.Hkv,
                       self.kt_n, self.D, self.kc, self.vc)
        w0 = self.first_len
        B.pc_parallel_attn(q[0, w0:w0 + self.wq], self.kc, self.vc, seg_len,
                           self.k_rope[0, w0:w0 + self.wq], v[0, w0:w0 + self.wq], 1,
                           self.wq, self.kc_n, self.kt_n, self.Hq, self.Hkv, self.D, w0,
                           self.rope_base, self.scale, self.global_o, self.global_lse, self.ws,
                           seg_len_per_head=per_head)

    def forward(self, q, k, v, chunk_lens=None, first_len=None):
        """chunk_prefill and evict_and_attend as one call; the same bits but for global_o and global_lse, whose keys
        may be cut into other parts."""
        if self.kc_n == 0:
            self.chunk_prefill(q, k, v, with_scores=True, chunk_lens=chunk_lens, first_len=first_len)
            return self.o
        self.chunk_lens = chunk_lens
        self.first_len = self.w if first_len is None else int(first_len)
        calibration = self.calibration
        if calibration is None and chunk_lens is not None:          # short chunks: counts per head, nothing evicted
            calibration = (float("inf"), 0, 0)
        B.pc_layer_forward(self.shape, q, k, v, self.first_len, self.kc_n, self.kt_n, self.o, self.lse, self.k_rope,
                           self.tok_score, self.chunk_score, self.chunk_idx, self.chunk_top, self.tok_idx, self.tok_cnt,
                           self.kc, self.vc, self.global_o, self.global_lse, self.ws, chunk_lens=chunk_lens,
                           calibration=calibration)
        return self.global_o


class StreamingParallelComp:
    """The same layer with the chunks arriving in memory-sized batches (sec. 3.1: chunks are
    encoded a batch at a time and a fixed-size priority queue keeps the best ones).  After each
    batch the queue holds the top keep_chunks of all chunks seen so far (score descending, earlier
    chunk first on ties, i.e. the offline top-k of the prefix); only the compacted KV of the chunks
    in the queue stays resident, an evicted chunk's slot is reused.  The final queue equals the
    offline selection, whatever the batch size.  The queue and its slot table live on the device
    (pc_chunk_queue_update), and the token selection and the gather of a batch's entrants are one
    launch each, driven by the device-side slot table: no host round trip between batches.  Host
    code here only owns buffers; every computation is a library call."""

    def __init__(self, n_chunks, batch_chunks, chunk_len, query_len, n_q_heads, n_kv_heads,
                 head_dim, obs_window, rope_base, keep_chunks, keep_tokens, softmax_scale=0.0,
                 device="cuda"):
        self.C, self.bc = n_chunks, min(batch_chunks, n_chunks)
        self.w, self.wq, self.L = chunk_len, query_len, chunk_len + query_len
        self.Hq, self.Hkv, self.D = n_q_heads, n_kv_heads, head_dim
        self.obs, self.rope_base, self.scale = obs_window, rope_base, softmax_scale
        self.kc_n, self.kt_n = min(keep_chunks, n_chunks), keep_tokens
        bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
        bc, L, Hq, Hkv, D = self.bc, self.L, n_q_heads, n_kv_heads, head_dim
        self.o = torch.empty((bc, L, Hq, D), dtype=bf, device=device)
        self.lse = torch.empty((bc, Hq, L), dtype=f32, device=device)
        self.k_rope = torch.empty((bc, L, Hkv, D), dtype=bf, device=device)
        self.tok_score = torch.empty((bc, Hkv, chunk_len), dtype=f32, device=device)
        self.chunk_score = torch.empty((n_chunks,), dtype=f32, device=device)     # all chunks seen
        # the device-side queue: ids in rank order, their scores and KV slots; entrants per slot
        self.queue_id = torch.full((self.kc_n,), -1, dtype=i32, device=device)
        self.queue_score = torch.zeros((self.kc_n,), dtype=f32, device=device)
        self.queue_slot = torch.zeros((self.kc_n,), dtype=i32, device=device)
        self.slot_src = torch.full((self.kc_n,), -1, dtype=i32, device=device)
        self.tok_idx = torch.empty((self.kc_n, Hkv, keep_tokens), dtype=i32, device=device)   # by slot
        self.kc = torch.empty((1, self.kc_n, Hkv, keep_tokens, D), dtype=bf, device=device)   # by slot
        self.vc = torch.empty_like(self.kc)
        self.q_query = torch.empty((query_len, Hq, D), dtype=bf, device=device)
        self.k_self = torch.empty((query_len, Hkv, D), dtype=bf, device=device)
        self.v_self = torch.empty_like(self.k_self)
        self.global_o = torch.empty((1, query_len, Hq, D), dtype=bf, device=device)
        self.global_lse = torch.empty((1, Hq, query_len), dtype=f32, device=device)
        shape = B.make_shape(bc, chunk_len, query_len, Hq, Hkv, D, obs_window, rope_base, softmax_scale)
        ws = max(B.pc_chunk_prefill_workspace_bytes(shape),
                 B.pc_parallel_attn_workspace_bytes(1, query_len, self.kc_n, keep_tokens, Hq, Hkv, D, True))
        self.ws = B.alloc_workspace(ws, device)

    def forward(self, q, k, v, after_batch=None):
        """q [C, L, H_q, D], k, v [C, L, H_kv, D] (any device-resident source; only one batch is
        touched at a time).  Returns the global attention output of the query rows.
        after_batch(first chunk id, chunks in the batch): optional callback after each batch's
        launches (tests read the queue there; it is not part of the path)."""
        self.queue_id.fill_(-1)                                  # an empty queue (plain fill)
        for c0 in range(0, self.C, self.bc):
            c1 = min(c0 + self.bc, self.C)
            nb = c1 - c0
            shape = B.make_shape(nb, self.w, self.wq, self.Hq, self.Hkv, self.D, self.obs,
                                 self.rope_base, self.scale)
            B.pc_chunk_prefill_attn(shape, q[c0:c1], k[c0:c1], v[c0:c1], self.o[:nb], self.lse[:nb],
                                    self.k_rope[:nb], self.tok_score[:nb], self.chunk_score[c0:c1],
                                    self.ws)
            if c0 == 0:              # the query rows of chunk 0 are the self segment (plain copies)
                self.q_query.copy_(q[0, self.w:]); self.k_self.copy_(self.k_rope[0, self.w:])
                self.v_self.copy_(v[0, self.w:])
            # merge the batch into the queue; then select and gather its entrants, slot by slot
            B.pc_chunk_queue_update(self.chunk_score[c0:c1], nb, c0, self.kc_n, self.queue_id,
                                    self.queue_score, self.queue_slot, self.slot_src)
            B.pc_select_tokens_topk(self.tok_score, self.slot_src, self.kc_n, self.Hkv, self.w,
                                    self.kt_n, self.tok_idx)
            B.pc_gather_kv(self.k_rope, v[c0:c1], self.slot_src, self.tok_idx, 1, nb, self.L, self.kc_n,
                           self.Hkv, self.kt_n, self.D, self.kc, self.vc)
            if after_batch is not None:
                after_batch(c0, nb)
        # every slot is filled once keep_chunks chunks have been seen (keep_chunks <= C)
        B.pc_parallel_attn(self.q_query, self.kc, self.vc, None, self.k_self, self.v_self, 1, self.wq,
                           self.kc_n, self.kt_n, self.Hq, self.Hkv, self.D, self.w, self.rope_base,
                           self.scale, self.global_o, self.global_lse, self.ws)
        return self.global_o


class DecodeCache:
    """The decoding stage (sec. 3.1, Eq. 9-11 token by token): the compressed segments of B
    sequences plus one tail segment that starts as the query block's keys / values and grows by
    one row per generated token.  Segment lengths live on the device and are advanced by
    the steps, so a run of decode steps is a run of library calls with no host round trip.
    A step = pc_decode_step: rotate and store the new token's K, V, then its query over
    [segments ; tail], itself included."""

    def __init__(self, batch, n_seg, keep_tokens, n_q_heads, n_kv_heads, head_dim, rope_base,
                 softmax_scale=0.0, device="cuda"):
        self.B, self.S, self.kt = batch, n_seg + 1, keep_tokens          # last segment = tail
        self.Hq, self.Hkv, self.D = n_q_heads, n_kv_heads, head_dim
        self.rope_base, self.scale = rope_base, softmax_scale
        bf, i32 = torch.bfloat16, torch.int32
        self.kc = torch.zeros((batch, self.S, n_kv_heads, keep_tokens, head_dim), dtype=bf, device=device)
        self.vc = torch.zeros_like(self.kc)
        self.seg_len = torch.zeros((batch, self.S), dtype=i32, device=device)
        self.out = torch.empty((batch, 1, n_q_heads, head_dim), dtype=bf, device=device)
        self.lse = torch.empty((batch, n_q_heads, 1), dtype=torch.float32, device=device)
        self.ws = B.alloc_workspace(B.pc_decode_step_workspace_bytes(
            batch, self.S, keep_tokens, n_q_heads, n_kv_heads, head_dim), device)

    def load(self, kc, vc, seg_len, k_tail, v_tail):
        """kc, vc [B, n_seg, H_kv, k_t, D] compacted segments (plain copies into the cache),
        seg_len [B, n_seg] or None (all k_t), k_tail, v_tail [B, n0, H_kv, D] rotated keys /
        values of the query block (appended through the library as already-rotated rows)."""
        n = self.S - 1
        self.kc[:, :n].copy_(kc); self.vc[:, :n].copy_(vc)
        if seg_len is None:
            self.seg_len[:, :n].fill_(self.kt)
        else:
            self.seg_len[:, :n].copy_(seg_len)
        self.seg_len[:, n].zero_()
        B.pc_kv_append(k_tail, v_tail, self.B, k_tail.shape[1], self.S, n, self.kt, self.Hkv, self.D,
                       -1, self.rope_base, self.kc, self.vc, self.seg_len)

    def step(self, q_new, k_new, v_new, pos):
        """q_new [B, 1, H_q, D], k_new, v_new [B, 1, H_kv, D] before RoPE; pos = the token's
        position (continues behind the query block).  Returns out [B, 1, H_q, D]."""
        B.pc_decode_step(q_new, k_new, v_new, self.B, self.S, self.kt, self.Hq, self.Hkv, self.D, pos,
                         self.rope_base, self.scale, self.kc, self.vc, self.seg_len, self.out, self.lse, self.ws)
        return self.out


def fp8_rows(k_t):
    """Key rows the codes of a segment occupy: whole 32-key blocks."""
    return (k_t + 31) // 32 * 32


def fp8_alloc(batch, n_seg, n_kv_heads, k_t, head_dim, device="cuda"):
    """Zeroed buffer for the K or V codes of pc_kv_quantize_fp8 / pc_parallel_attn_fp8:
    [B, S, H_kv, ceil(k_t / 32) * 32 * D] bytes (32-key blocks laid out for the matrix cores)."""
    return torch.zeros((batch, n_seg, n_kv_heads, fp8_rows(k_t) * head_dim), dtype=torch.uint8, device=device)


class DecodeCacheFp8:
    """DecodeCache with the compressed segments stored in 8 bits (E4M3 codes + one scale per
    sequence, segment and KV head, written once by pc_kv_quantize_fp8 when the cache is loaded)
    and the growing tail kept in bf16 as a one-segment cache of its own.  A step =
    pc_decode_step_fp8: append to the tail, attend over [8-bit segments ; tail]."""

    def __init__(self, batch, n_seg, keep_tokens, tail_cap, n_q_heads, n_kv_heads, head_dim, rope_base,
                 softmax_scale=0.0, device="cuda"):
        self.B, self.S, self.kt, self.cap = batch, n_seg, keep_tokens, tail_cap
        self.Hq, self.Hkv, self.D = n_q_heads, n_kv_heads, head_dim
        self.rope_base, self.scale = rope_base, softmax_scale
        bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
        self.k8 = fp8_alloc(batch, n_seg, n_kv_heads, keep_tokens, head_dim, device)
        self.v8 = fp8_alloc(batch, n_seg, n_kv_heads, keep_tokens, head_dim, device)
        self.k_scale = torch.ones((batch, n_seg, n_kv_heads), dtype=f32, device=device)
        self.v_scale = torch.ones_like(self.k_scale)
        self.seg_len = torch.zeros((batch, n_seg), dtype=i32, device=device)
        self.k_tail = torch.zeros((batch, 1, n_kv_heads, tail_cap, head_dim), dtype=bf, device=device)
        self.v_tail = torch.zeros_like(self.k_tail)
        self.tail_len = torch.zeros((batch, 1), dtype=i32, device=device)
        self.out = torch.empty((batch, 1, n_q_heads, head_dim), dtype=bf, device=device)
        self.lse = torch.empty((batch, n_q_heads, 1), dtype=f32, device=device)
        self.ws = B.alloc_workspace(B.pc_decode_step_fp8_workspace_bytes(
            batch, n_seg, keep_tokens, tail_cap, n_q_heads, n_kv_heads, head_dim), device)

    def load(self, kc, vc, seg_len, k_tail, v_tail):
        """kc, vc [B, n_seg, H_kv, k_t, D] bf16 compacted segments (quantised here), seg_len
        [B, n_seg] or None, k_tail, v_tail [B, n0, H_kv, D] rotated keys / values of the query block."""
        if seg_len is None:
            self.seg_len.fill_(self.kt)
        else:
            self.seg_len.copy_(seg_len)
        B.pc_kv_quantize_fp8(kc, vc, self.seg_len, self.B, self.S, self.kt, self.Hkv, self.D, self.k8,
                             self.v8, self.k_scale, self.v_scale)
        self.tail_len.zero_()
        B.pc_kv_append(k_tail, v_tail, self.B, k_tail.shape[1], 1, 0, self.cap, self.Hkv, self.D, -1,
                       self.rope_base, self.k_tail, self.v_tail, self.tail_len)

    def step(self, q_new, k_new, v_new, pos):
        B.pc_decode_step_fp8(q_new, k_new, v_new, self.k8, self.v8, self.k_scale, self.v_scale, self.seg_len,
                             self.k_tail, self.v_tail, self.tail_len, self.cap, self.B, self.S, self.kt, self.Hq,
                             self.Hkv, self.D, pos, self.rope_base, self.scale, self.out, self.lse, self.ws)
        return self.out


def _capturing(t):
    """Is work on t's device being recorded into a graph here?"""
    return t.is_cuda and torch.cuda.is_current_stream_capturing()


def _must_be(shape, dtype, **tensors):
    """Refuses tensors whose memory is not a whole [shape] of dtype: the library is given addresses."""
    for name, t in tensors.items():
        if t is None or t.shape != shape or t.dtype != dtype or not t.is_contiguous():
            got = t if t is None else f"{t.dtype} {tuple(t.shape)}, strides {t.stride()}"
            raise ValueError(f"{name}: {got} is not {dtype} {tuple(shape)}, contiguous")


class SharedPrefixDecoder:
    """Many answers over few compressed documents: n_prefix documents' compacted segments, each shared by batch /
    n_prefix sequences (sequence b reads document b // (batch // n_prefix)), and a tail a sequence that starts as its
    query block's keys / values and grows as tokens are generated, kept in 8-bit rows that are rounded as they are
    written.  With eight_bit_prefix the segments are kept so too.

    A step is append -> attention (-> the caller's remaining layers -> verification of drafted tokens):
      step(q, k, v)   the n rows a sequence (its last token and the drafts behind it) of this layer
      accept()        all n rows stand (no drafts), or
      verify(...)     those up to the first draft that falls stand; the others' rows are written over by the next step.
    Lengths live on the device, so a run of steps is a run of library calls with no host round trip, until the rows written
    so far could fill a tail: then a step reads the lengths, and raises if its rows would pass the capacity of one.  A step in
    a captured graph cannot: whoever replays it sees to it that the rows fit.  A graph of step and accept or verify goes on
    from replay to replay; it is captured anew where load was given other lengths of the segments."""

    def __init__(self, batch, n_prefix, n_seg, keep_tokens, tail_cap, n_q_heads, n_kv_heads, head_dim, rope_base,
                 tail_pos, max_rows=1, softmax_scale=0.0, eight_bit_prefix=False, device="cuda"):
        self.B, self.P, self.S, self.kt, self.cap = batch, n_prefix, n_seg, keep_tokens, tail_cap
        self.Hq, self.Hkv, self.D = n_q_heads, n_kv_heads, head_dim
        self.rope_base, self.scale, self.pos0, self.max_rows = rope_base, softmax_scale, tail_pos, max_rows
        i32, f32 = torch.int32, torch.float32
        rows8 = lambda *shape: [torch.zeros((*shape, head_dim), dtype=torch.uint8, device=device) for _ in "kv"] + \
            [torch.ones(shape, dtype=f32, device=device) for _ in "kv"]
        self.eight_bit_prefix = eight_bit_prefix
        seg = (n_prefix, n_seg, n_kv_heads, keep_tokens)
        if eight_bit_prefix:
            self.prefix = rows8(*seg)
        else:
            self.prefix = [torch.zeros((*seg, head_dim), dtype=torch.bfloat16, device=device) for _ in "kv"]
        self.tail = rows8(batch, 1, n_kv_heads, tail_cap)
        self.len = torch.zeros((batch,), dtype=i32, device=device)          # rows of the tails that stand
        self.len_new = torch.zeros_like(self.len)                           # with those of the step at hand
        self.rows = 0                                                       # rows of the step at hand; 0: none
        self.graph_rows = 0                                                 # of the longest step that a graph holds
        self.most = 0                                                       # no tail has more rows that stand; None: not known
        self.prefix_rows = None
        self.lse = torch.empty((batch, n_q_heads, max_rows), dtype=f32, device=device)
        self.out = torch.empty((batch, max_rows, n_q_heads, head_dim), dtype=torch.bfloat16, device=device)
        self.ws = self.tail_rows = None                                     # made with the first step

    def load(self, kc, vc, seg_len=None, seg_len_per_head=0, k_tail=None, v_tail=None):
        """kc, vc [n_prefix, n_seg, H_kv, k_t, D] bf16 compacted segments (copied, or rounded to 8-bit rows), seg_len
        int32 or None (all k_t); k_tail, v_tail [B, n0, H_kv, D] bf16 rotated keys / values of the query blocks, or None."""
        seg = (self.P, self.S, self.Hkv, self.kt, self.D)
        if self.eight_bit_prefix:
            _must_be(seg, torch.bfloat16, kc=kc, vc=vc)
        elif kc.shape != seg or vc.shape != seg:
            raise ValueError(f"kc {tuple(kc.shape)}, vc {tuple(vc.shape)}: not {seg}")
        n0 = 0
        if k_tail is not None or v_tail is not None:
            n0 = 0 if k_tail is None or k_tail.dim() != 4 else k_tail.shape[1]
            _must_be((self.B, n0, self.Hkv, self.D), torch.bfloat16, k_tail=k_tail, v_tail=v_tail)
        if n0 > self.cap:
            raise ValueError(f"the tails hold {self.cap} rows, not {n0}")
        prefix_rows = B.make_row_cache(*self.prefix, seg_len=seg_len, seg_len_per_head=seg_len_per_head)
        if self.eight_bit_prefix:                                           # a segment's head is a sequence of its own
            k8, v8, ks, vs = self.prefix
            B.pc_kv_append_row8(kc, vc, self.P * self.S * self.Hkv, self.kt, self.kt, 1, self.D, k8, v8, ks, vs, None, None)
        else:
            self.prefix[0].copy_(kc); self.prefix[1].copy_(vc)
        self.prefix_rows = prefix_rows
        self.len.zero_()
        self.rows = 0
        if self.most is not None:
            self.most = 0
        if n0 > 0:
            self._append(k_tail, v_tail, None)
            self.accept()

    def _room(self, n):
        """Refuses n rows a sequence that would pass the capacity of a tail."""
        if _capturing(self.len):
            self.most = None                                                # replays will move the lengths unseen
            self.graph_rows = max(self.graph_rows, n)
            return
        if self.most is None or self.most + n > self.cap:
            most = int(self.len.max())
            if self.most is not None:
                self.most = most
            if most + n > self.cap:
                raise ValueError(f"the tails hold {self.cap} rows: {n} more do not fit behind the {most} of the longest")

    def _append(self, k, v, pos):
        k8, v8, ks, vs = self.tail
        B.pc_kv_append_row8(k, v, self.B, k.shape[1], self.cap, self.Hkv, self.D, k8, v8, ks, vs, self.len, self.len_new,
                            pos=pos, pos0=self.pos0, rope_base=self.rope_base)
        self.rows = k.shape[1]

    def step(self, q, k, v):
        """q [B, n, H_q, D], k, v [B, n, H_kv, D] bf16 before RoPE, n <= max_rows: rows at positions tail_pos + len .. of
        their sequences.  Returns out [B, n, H_q, D] (a view of the step's buffer)."""
        n = q.shape[1]
        if self.prefix_rows is None:
            raise ValueError("load the documents first")
        if not 1 <= n <= self.max_rows or q.shape != (self.B, n, self.Hq, self.D) or k.shape != (self.B, n, self.Hkv, self.D) or \
                v.shape != k.shape:
            raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}: not up to {self.max_rows} rows of this decoder")
        for t in (q, k, v):
            if t.dtype != torch.bfloat16 or not t.is_contiguous():
                raise ValueError("q, k and v must be bfloat16 and contiguous")
        self._room(n)
        self._append(k, v, self.len)
        tail = self.tail_rows
        if tail is None:
            tail = self.tail_rows = B.make_row_cache(*self.tail, seg_len=self.len_new)
            self.ws = B.alloc_workspace(max(B.pc_shared_attn_workspace_bytes(self.prefix_rows, tail, self.B, self.P, m, self.Hq,
                                                                             self.Hkv, self.D)
                                            for m in range(1, self.max_rows + 1)), q.device)
        out = self.out.view(-1)[:q.numel()].view(q.shape)
        lse = self.lse.view(-1)[:self.B * self.Hq * n].view(self.B, self.Hq, n)
        B.pc_shared_attn(q, self.prefix_rows, tail, self.B, self.P, n, self.Hq, self.Hkv, self.D, out, lse, self.ws,
                         q_pos=self.len, pos0=self.pos0, rope_base=self.rope_base, softmax_scale=self.scale, tail_own=1)
        return out

    def accept(self):
        """Every row of the step stands."""
        self._written(1)
        # no rows more, the lengths alone: in place, since a captured step reads them where they were when it was captured
        B.pc_kv_append_row8(None, None, self.B, 0, self.cap, self.Hkv, self.D, None, None, None, None, self.len_new, self.len)
        self._stand(self.rows)

    def _written(self, n):
        """Refuses to count n rows a sequence that the step at hand, or a graph's where there is none, has not written."""
        rows = self.rows or self.graph_rows
        if n > rows:
            raise ValueError(f"{n} rows a sequence to stand, {rows} rows of the step at hand")

    def _stand(self, n):
        """The step at hand is done: up to n of its rows stand."""
        self.rows = 0
        if self.most is not None:
            self.most += n

    def verify(self, draft, draft_prob, target_prob, u, noise, tokens, n_accepted, ws, draft_len=None):
        """pc_verify_drafts; the rows of the last token and of the standing drafts stay in the tails.  No more drafts than
        rows behind the first that the step has written."""
        k, V, i32, f32 = draft.shape[1], target_prob.shape[-1], torch.int32, torch.float32
        self._written(k + 1)
        _must_be((self.B, k), i32, draft=draft)
        _must_be((self.B, k), f32, u=u)
        _must_be((self.B, k + 1, V), f32, target_prob=target_prob)
        _must_be((self.B, V), f32, noise=noise)
        _must_be((self.B, k + 1), i32, tokens=tokens)
        _must_be((self.B,), i32, n_accepted=n_accepted)
        if draft_prob is not None:
            _must_be((self.B, k, V), f32, draft_prob=draft_prob)
        if draft_len is not None:
            _must_be((self.B,), i32, draft_len=draft_len)
        B.pc_verify_drafts(draft, draft_prob, target_prob, u, noise, self.B, k, V, tokens, n_accepted, ws,
                           draft_len=draft_len, len_in=self.len, len_out=self.len)
        self._stand(k + 1)


class PagedTreeDecoder:
    """Answers of very unequal lengths out of one pool of pages, with trees of drafted tokens: a sequence's rows (its compressed
    document, its query block, its answer) lie in pages of its own, taken as it grows and given back when it ends.

      load(b, ...)    sequence b's document
      step(q, k, v, parent)   the rows of every sequence's tree of this layer (its last token at the root, drafts below): appended,
                      attended to; without a parent a chain, with one row an ordinary decoding step
      accept(tokens, choice)  the path that the target's choices follow stays, its rows move together; the next token
      release(b)      sequence b's pages are free again
    A step that has not been accepted when a sequence is loaded or released is dropped: accept() asks for the next one.

    Lengths and positions live on the device.  The host keeps a bound of each sequence's rows and reads the lengths, and how many
    rows a step has of each, only where a sequence could pass the end of its pages with all of the step's; then it takes pages for it,
    and raises if there are none, before anything is written.  A step in a captured graph takes no pages: reserve() them first,
    and see to it that the rows of the replays fit.  It is accepted in a graph, too, its own or one that is captured next and
    replayed behind it: the host does not see replays.
    Rows behind a sequence's pages are dropped, and nobody sees them."""

    def __init__(self, batch, n_pages, page, max_pages, n_q_heads, n_kv_heads, head_dim, rope_base, max_rows=1, softmax_scale=0.0,
                 eight_bit=False, device="cuda"):
        self.B, self.page, self.max_pages = batch, page, max_pages
        self.Hq, self.Hkv, self.D = n_q_heads, n_kv_heads, head_dim
        self.rope_base, self.scale, self.max_rows = rope_base, softmax_scale, max_rows
        i32, shape = torch.int32, (n_pages, n_kv_heads, page)
        kv = torch.uint8 if eight_bit else torch.bfloat16
        self.k, self.v = (torch.zeros((*shape, head_dim), dtype=kv, device=device) for _ in "kv")
        self.k_scale, self.v_scale = (torch.ones(shape, device=device) if eight_bit else None for _ in "kv")
        self.table = torch.full((batch, max_pages), -1, dtype=i32, device=device)
        self.len, self.len_new, self.pos = (torch.zeros((batch,), dtype=i32, device=device) for _ in range(3))
        self.free = list(range(n_pages - 1, -1, -1))
        self.pages = [None] * batch                                         # of a sequence; None: not loaded
        self.most = [0] * batch                                             # no sequence has more rows that stand
        self.known = True                                                   # False: graphs move the lengths unseen
        self.at_hand = None                                                 # (rows, parent, n_rows, rows at most, captured) of the step that is not accepted yet
        self.out = torch.empty((batch, max_rows, n_q_heads, head_dim), dtype=torch.bfloat16, device=device)
        self.lse = torch.empty((batch, n_q_heads, max_rows), dtype=torch.float32, device=device)
        self.path = torch.empty((batch, max_rows), dtype=i32, device=device)
        self.n_kept, self.next_token = (torch.empty((batch,), dtype=i32, device=device) for _ in range(2))
        self.cache = self.ws = None                                         # made with the first load

    def _cache(self, table):
        return B.make_page_cache(self.k, self.v, table, self.k_scale, self.v_scale)

    def _ready(self, device):
        if self.cache is not None:
            return
        if _capturing(self.len):
            raise ValueError("load a document first")
        self.cache = self._cache(self.table)
        self.ws = B.alloc_workspace(max(B.pc_tree_attn_workspace_bytes(self.cache, self.B, m, self.Hq, self.Hkv, self.D)
                                        for m in range(1, self.max_rows + 1)), device)

    def reserve(self, b, rows):
        """Pages for `rows` rows of sequence b."""
        if _capturing(self.len):
            raise ValueError("pages are taken outside of graphs")
        have, need = self.pages[b] or [], (rows + self.page - 1) // self.page
        more = need - len(have)
        if more <= 0 and self.pages[b] is not None:
            return
        if need > self.max_pages:
            raise ValueError(f"sequence {b}: {rows} rows are more than {self.max_pages} pages of {self.page}")
        if more > len(self.free):
            raise ValueError(f"sequence {b}: {more} pages more for {rows} rows, {len(self.free)} are free")
        taken = [self.free.pop() for _ in range(max(more, 0))]
        self.pages[b] = have + taken
        if taken:
            self.table[b, len(have):need].copy_(torch.tensor(taken, dtype=torch.int32))

    def release(self, b):
        """Sequence b has ended."""
        if _capturing(self.len):
            raise ValueError("a sequence ends outside of graphs")
        pages, self.at_hand = self.pages[b], None                           # (its lengths are another sequence's now)
        if pages is None:
            return
        self.free += reversed(pages)
        self.pages[b], self.most[b] = None, 0
        self.table[b].fill_(-1)
        self.len[b], self.pos[b] = 0, 0

    def load(self, b, kc, vc, pos, seg_len=None, k_tail=None, v_tail=None):
        """kc, vc [n_seg, H_kv, k_t, D] bf16: the document's compacted segments (keys rotated), as the gather leaves them, of
        seg_len[s] rows (None: k_t) each; k_tail, v_tail [n0, H_kv, D] rotated rows of the query block behind them, or None;
        pos: the position of the sequence's next row.  What sequence b held before is released; a load that is refused leaves it.
        All of a segment's heads have the same rows: one whose heads kept different numbers is not taken."""
        n_seg, _, k_t, _ = kc.shape if kc.dim() == 4 else (0, 0, 0, 0)
        if kc.shape != (n_seg, self.Hkv, k_t, self.D) or kc.shape != vc.shape or kc.dtype != torch.bfloat16 or vc.dtype != kc.dtype:
            raise ValueError(f"kc {tuple(kc.shape)}, vc {tuple(vc.shape)}: not bfloat16 [n_seg, {self.Hkv}, k_t, {self.D}]")
        lens = [k_t] * n_seg if seg_len is None else [int(x) for x in seg_len]
        if len(lens) != n_seg or any(not 0 <= x <= k_t for x in lens):
            raise ValueError(f"seg_len {lens} of {n_seg} segments of {k_t} rows")
        if (k_tail is None) != (v_tail is None):
            raise ValueError("k_tail and v_tail: both or neither")
        n0 = 0 if k_tail is None else k_tail.shape[0]
        if n0:
            _must_be((n0, self.Hkv, self.D), torch.bfloat16, k_tail=k_tail, v_tail=v_tail)
        if _capturing(self.len):
            raise ValueError("a sequence is loaded outside of graphs")
        b, pos, total = range(self.B)[b], int(pos), sum(lens) + n0
        if not -2 ** 31 <= pos < 2 ** 31:
            raise ValueError(f"position {pos} has more than 32 bits")
        self._fits(b, total)
        self._ready(self.table.device)
        to = lambda x: torch.tensor(x, dtype=torch.int32, device=self.table.device)
        parts = []                                                          # rows, sequences, rows of each, the first's places, how many are theirs
        if n_seg and k_t:                                                   # each segment a sequence of its own, behind the one before
            parts.append((kc.transpose(1, 2), vc.transpose(1, 2), n_seg, k_t, to([sum(lens[:s]) for s in range(n_seg)]), to(lens)))
        if n0:
            parts.append((k_tail[None], v_tail[None], 1, n0, to([total - n0]), to([n0])))

        def append(k, v, m, n, first, rows):
            B.pc_kv_append_paged(k, v, m, n, self.Hkv, self.D, self._cache(self.table[b].repeat(m, 1)), first, None, n_rows=rows)
        for *part, rows in parts:                                           # none of the rows: refused is what is refused, with the old document in place
            append(*part, torch.zeros_like(rows))
        self.release(b)
        self.reserve(b, total)
        for part in parts:
            append(*part)
        self.len[b], self.pos[b] = total, pos
        self.most[b] = total

    def _fits(self, b, rows):
        """Refuses a load that would not fit, before anything is released."""
        need = (rows + self.page - 1) // self.page
        if need > min(self.max_pages, len(self.free) + len(self.pages[b] or [])):
            raise ValueError(f"sequence {b}: {rows} rows need {need} pages of {self.page}, {len(self.free)} are free, {self.max_pages} a "
                             "sequence at most")

    def _room(self, n, n_rows):
        """Pages for the step's rows: n of every sequence, or min(n, n_rows[b]) of sequence b, where they are read.  Returns how many those are."""
        more = [n] * self.B
        if _capturing(self.len):
            self.known = False                                              # replays will move the lengths unseen
            return more
        short = lambda: [b for b, p in enumerate(self.pages) if p is not None and self.most[b] + more[b] > len(p) * self.page]
        if not self.known or short():
            self.most = self.len.tolist()
            if n_rows is not None:
                more[:] = [min(max(x, 0), n) for x in n_rows.tolist()]
        short = short()
        need = [(self.most[b] + more[b] + self.page - 1) // self.page for b in short]
        if any(x > self.max_pages for x in need) or sum(need) - sum(len(self.pages[b]) for b in short) > len(self.free):
            raise ValueError(f"{[more[b] for b in short]} rows more do not fit: sequences {short} of {[self.most[b] for b in short]} rows, "
                             f"{len(self.free)} pages of {self.page} are free, {self.max_pages} a sequence at most")
        for b in short:
            self.reserve(b, self.most[b] + more[b])
        return more

    def step(self, q, k, v, parent=None, n_rows=None):
        """q [B, n, H_q, D], k, v [B, n, H_kv, D] bf16 before RoPE, n <= max_rows: the nodes of every sequence's tree; parent
        [B, n] int32 or None (a chain); n_rows [B] int32: how many are a sequence's (0: it does not take part), None: all, of
        sequences that are all loaded.  Returns out [B, n, H_q, D] (a view of the step's buffer; other rows than n_rows of a sequence
        are not written)."""
        n = q.shape[1] if q.dim() == 4 else 0
        if not 1 <= n <= self.max_rows or q.shape != (self.B, n, self.Hq, self.D) or k.shape != (self.B, n, self.Hkv, self.D) or \
                v.shape != k.shape or any(t.dtype != torch.bfloat16 for t in (q, k, v)):
            raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}: not up to {self.max_rows} bfloat16 rows of this decoder")
        for name, t, shape in (("parent", parent, (self.B, n)), ("n_rows", n_rows, (self.B,))):
            if t is not None:
                _must_be(shape, torch.int32, **{name: t})
        if n_rows is None and None in self.pages:
            raise ValueError(f"sequence {self.pages.index(None)} is not loaded: say with n_rows who takes part")
        more = self._room(n, n_rows)
        self._ready(q.device)
        B.pc_kv_append_paged(k, v, self.B, n, self.Hkv, self.D, self.cache, self.len, self.len_new, pos=self.pos,
                             rope_base=self.rope_base, parent=parent, n_rows=n_rows)
        self.at_hand = None                                                 # (the rows of the step before are written over)
        out = self.out.view(-1)[:q.numel()].view(q.shape)
        lse = self.lse.view(-1)[:self.B * self.Hq * n].view(self.B, self.Hq, n)
        B.pc_tree_attn(q, self.cache, self.len_new, self.B, n, self.Hq, self.Hkv, self.D, out, lse, self.ws, parent=parent, n_rows=n_rows,
                       pos=self.pos, rope_base=self.rope_base, softmax_scale=self.scale)
        self.at_hand = (n, parent, n_rows, more, _capturing(self.len))
        return out

    def accept(self, tokens, choice, choice_stride=1):
        """pc_tree_accept of the step's trees: tokens [B, n], choice [B, n] (or [B, n, choice_stride], the first of each) int32.
        Returns path [B, n], n_kept [B], next_token [B] (views of the decoder's buffers)."""
        if self.at_hand is None:
            raise ValueError("no step at hand")
        n, parent, n_rows, more, captured = self.at_hand
        if captured != _capturing(self.len):
            raise ValueError("a step in a graph is accepted in a graph, another one outside")
        _must_be((self.B, n), torch.int32, tokens=tokens)
        path = self.path.view(-1)[:self.B * n].view(self.B, n)
        B.pc_tree_accept(tokens, parent, choice, self.B, n, path, self.n_kept, self.next_token, choice_stride=choice_stride,
                         cache=self.cache, n_kv_heads=self.Hkv, head_dim=self.D, len_in=self.len_new, len_out=self.len, pos=self.pos,
                         n_rows=n_rows)
        self.at_hand = None
        self.most = [m + x for m, x in zip(self.most, more)]
        return path, self.n_kept, self.next_token
