/*
 * parallelcomp_bench.h - measurement aids of the ParallelComp library (not part of the method's
 * boundary: nothing here computes a step of the path).  Used by the benchmark only.
 */
#ifndef PARALLELCOMP_BENCH_H
#define PARALLELCOMP_BENCH_H

#include <stddef.h>
#include <stdint.h>
#include "parallelcomp.h"   /* pc_status */

#ifdef __cplusplus
extern "C" {
#endif

/* ---- per-kernel timing (measurement aid; off by default) ------------------------------------
 * While enabled, every kernel the library launches is bracketed by a pair of HIP events recorded
 * on the stream of the call.  pc_profile_begin resets the record list (at most 4096 records are
 * kept, later launches are not recorded); pc_profile_end stops recording; pc_profile_get waits
 * for record i and returns its kernel id (pc_kernel_id) and elapsed milliseconds.
 * Not thread-safe; meant for one benchmarking thread. */
typedef enum pc_kernel_id {
  PC_KERNEL_LAYER_PREP = 0, PC_KERNEL_KV_PREPASS = 1, PC_KERNEL_FLASH = 2, PC_KERNEL_SCORES_P1 = 3,
  PC_KERNEL_SCORES_P2 = 4, PC_KERNEL_CHUNK_SCORE = 5, PC_KERNEL_SELECT_CHUNKS = 6,
  PC_KERNEL_SELECT_TOKENS = 7, PC_KERNEL_GATHER = 8, PC_KERNEL_ROPE_Q = 9, PC_KERNEL_DECODE = 10,
  PC_KERNEL_MERGE = 11, PC_KERNEL_SELF_INFO = 12, PC_KERNEL_KV_APPEND = 13,
  PC_KERNEL_SCORES_LSE = 14, PC_KERNEL_KV_QUANTIZE = 15, PC_KERNEL_DECODE_FP8 = 16,
  PC_KERNEL_PREPASS_SCORES = 17,   /* scores pass 1 fused with the K/V pre-pass */
  PC_KERNEL_CHUNK_QUEUE = 18, PC_KERNEL_FP8_IMAGES = 19, PC_KERNEL_FP8_ROWS = 20,
  PC_KERNEL_SHARED_PREFIX = 21, PC_KERNEL_SHARED_TAIL = 22, PC_KERNEL_SHARED_MERGE = 23, PC_KERNEL_ROW8_APPEND = 24,
  PC_KERNEL_ROW8_READ = 25, PC_KERNEL_VERIFY_RACE = 26, PC_KERNEL_VERIFY_PICK = 27,
  PC_KERNEL_SHARED_ALONE = 28, PC_KERNEL_VERIFY_ALONE = 29,   /* the one-launch forms */
  PC_KERNEL_PAGED_APPEND = 30, PC_KERNEL_TREE_ATTN = 31, PC_KERNEL_TREE_MERGE = 32, PC_KERNEL_LOGPROBS = 33,
  PC_KERNEL_LOGPROBS_JOIN = 34, PC_KERNEL_TREE_ACCEPT = 35,
  PC_KERNEL_COUNT = 36
} pc_kernel_id;
int         pc_profile_begin(void);
int         pc_profile_begin_kernel(int kernel_id);   /* as pc_profile_begin, but only the launches of one
                                                        kernel are bracketed (two event records per kernel
                                                        cost about 7 us of stream time each) */
int         pc_profile_end(void);
int         pc_profile_count(void);
int         pc_profile_get(int i, int* kernel_id, float* ms);
const char* pc_kernel_name(int kernel_id);

/* ---- matrix-pipe ceiling (measurement aid) ---------------------------------------------------
 * Enqueues a kernel built around independent 32x32x16 bf16 MFMAs: n_cus workgroups of 8
 * wavefronts (two per SIMD), iters x 8 MFMAs each.  mode 0: nothing but MFMAs on constant
 * operands; mode 1: the same on random operands (more bits toggle, the power-limited clock falls);
 * mode 2: random operands plus, per MFMA, one 16-byte-per-lane LDS read feeding the A operand and
 * one softmax element on the vector ALU (exponential, add, multiply), the instruction mix of a
 * flash-attention loop at 32 queries per wavefront.  scratch (device, >= n_cus * 512 * 4 bytes)
 * receives one float per lane so the work cannot be optimised away.  *flops (host) receives the
 * MFMA floating-point operations the launch performs; the caller times the launch on its stream
 * and divides.  Returns PC_ERR_NULL / PC_ERR_SHAPE (mode outside 0..2, n_cus outside 1..4096,
 * iters outside 1..2^22) / PC_ERR_WORKSPACE / PC_ERR_HIP. */
int pc_mfma_ceiling(int mode, int n_cus, int iters, float* scratch, size_t scratch_bytes,
                    double* flops, void* stream);

/* ---- copy ceiling (measurement aid) -----------------------------------------------------------
 * Enqueues a bare copy of `bytes` bytes (device pointers, 16-byte aligned, bytes a multiple of
 * 16) with 16-byte loads and stores, four in flight per thread: mode 0 ordinary, mode 1 with the
 * non-temporal hint on both sides.  The caller times it: what a read-and-write stream sustains on
 * this machine.  PC_ERR_NULL / PC_ERR_SHAPE / PC_ERR_HIP. */
int pc_copy_ceiling(int mode, const void* src, void* dst, size_t bytes, void* stream);

/* ---- how a pc_shared_attn call is done (measurement aid; host only, launches nothing) ------------
 * A side (prefix, tail): its format (0 no rows, 1 16-bit, 2 8-bit rows), the query rows a workgroup takes (16, 32, 64
 * from memory straight into registers, 256 by tiles of keys in LDS; 0 no workgroups of its own) and the parts its keys
 * are cut into.  alone: one launch for everything, both sides' workgroups with it.  tails_behind: the tails ride in the
 * prefix's launch, tail_waves wavefronts a run of a tail's keys.  Sizes and formats as pc_shared_attn; PC_ERR_SHAPE. */
typedef struct pc_shared_attn_plan_info {
  int32_t alone;
  int32_t prefix_format, prefix_rows, prefix_parts;
  int32_t tail_format, tail_rows, tail_parts, tail_waves, tails_behind;
} pc_shared_attn_plan_info;
int pc_shared_attn_plan(const pc_row_cache* prefix, const pc_row_cache* tail, int32_t batch, int32_t n_prefix,
                        int32_t n_q, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                        pc_shared_attn_plan_info* plan);

#ifdef __cplusplus
}
#endif
#endif /* PARALLELCOMP_BENCH_H */
