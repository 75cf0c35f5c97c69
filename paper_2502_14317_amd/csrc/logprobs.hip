// What the tokens of a vocabulary are worth: one pass over a row of logits x keeps, relative to a running maximum m in log2
// units, l = sum 2^(x - m) and e = sum 2^(x - m) (x - m), from which with L = log2 l
//   log2 p(v) = x_v - m - L,   entropy / ln 2 = L - e / l.
// A term of x = -inf is 0 (its factor is held above -1e4, and 2^-1e4 is 0); NaN and +inf make l NaN, and with it every number
// of the row.
// The n_top largest: the pass knows the largest logit of every thread.  With the j-th largest of those in each of F
// wavefronts, F j >= n_top, the least of the F is one that n_top logits at least reach, and few more do (20 of 128256: some 70).
// The threads whose largest reaches it, some F j, have their logits read once more, from the caches; those that reach it
// go to a list in LDS, where each counts how many are before it.  Where the list does not hold them (ties) or misses some (NaN),
// the n_top-th of the order (logit, token) is found eight bits at a time.
#include "paged.h"

#define LOGPROBS_THREADS 1024
#define LOGPROBS_WAVES (LOGPROBS_THREADS / PC_WAVE)
#define LOGPROBS_LOG2E 1.4426950408889634f
#define LOGPROBS_LN2 0.6931471805599453f

// (logit, token) as one word whose order is that of the top list: larger logit, then lower token.  0: nobody.
typedef unsigned long long top_key;
__device__ __forceinline__ top_key top_key_of(float x, int v) { return (top_key)pc_order_key(x) << 32 | (uint32_t)~v; }
__device__ __forceinline__ float top_logit(top_key k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return u == 0 ? NAN : __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int top_token(top_key k) { return (int)~(uint32_t)k; }

#define TOP_LIST 2048
struct TopLds {
  top_key key[TOP_LIST];
  int count, threads;
  uint16_t thread[LOGPROBS_THREADS];
  uint32_t wave[LOGPROBS_WAVES];
  int digits[256];
};

struct LogSum {
  float m, l, e;
  __device__ __forceinline__ void clear() { m = -INFINITY; l = 0.f; e = 0.f; }
  // relative to `to` >= m instead; where nothing but -inf has been seen l and e are 0, or NaN if a NaN has
  __device__ __forceinline__ void move(float to) {
    if (m != -INFINITY) {
      const float d = m - to, a = __builtin_amdgcn_exp2f(d);
      e = d == 0.f ? e : a * fmaf(fmaxf(d, -1e4f), l, e);
      l *= a;
    }
    m = to;
  }
  __device__ __forceinline__ void join(LogSum y) {
    const float top = fmaxf(m, y.m);
    move(top);
    y.move(top);
    l += y.l;
    e += y.e;
  }
  // returns the largest of them
  template <int N>
  __device__ __forceinline__ float add(const float (&x)[N]) {
    float most = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) most = fmaxf(most, x[i]);
    if (most * LOGPROBS_LOG2E > m) move(most * LOGPROBS_LOG2E);        // (log2 e > 0: the maximum commutes with it)
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float t = fmaf(x[i], LOGPROBS_LOG2E, -ref), p = __builtin_amdgcn_exp2f(t);
      l += p;
      e = fmaf(p, fmaxf(t, -1e4f), e);
    }
    return most;
  }
  __device__ __forceinline__ float logprob(float x) const { return (fmaf(x, LOGPROBS_LOG2E, -m) - log2f(l)) * LOGPROBS_LN2; }
  __device__ __forceinline__ float entropy() const { return (log2f(l) - e / l) * LOGPROBS_LN2; }
};

struct LogprobsArgs {
  PcLogprobs c;
  int parts;               // workgroups a row
  PcDiv parts_div;
  LogSum* sums;            // [rows, parts]
  top_key* tops;           // [rows, parts, n_top], largest first
};

// A row as 16-byte pieces between its first and last few elements, which have no whole piece; a part: a run of pieces, the
// first part with the row's head, the last one with its tail.
template <typename T>
struct LogprobsRow {
  static constexpr int VE = 16 / (int)sizeof(T);
  const T* p;
  int head, lo, hi, tail, vocab;                            // elements, pieces, pieces, first element of the tail
  bool first, last;
  __device__ __forceinline__ LogprobsRow(const PcLogprobs& c, long long row, int part, int parts) {
    p = (const T*)c.logits + row * c.row_stride;
    vocab = c.vocab;
    head = min((int)((16 - (int)((uintptr_t)p & 15)) & 15) / (int)sizeof(T), vocab);
    const int n = (vocab - head) / VE;
    tail = head + n * VE;
    lo = (int)((long long)n * part / parts); hi = (int)((long long)n * (part + 1) / parts);
    first = part == 0; last = part == parts - 1;
  }
  __device__ __forceinline__ static float value(float x) { return x; }
  __device__ __forceinline__ static float value(uint16_t x) { return bf16_bits_to_f32(x); }
  __device__ __forceinline__ static void values(u32x4 w, float (&x)[VE]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (VE == 8) { x[2 * i] = bf16_lo_to_f32(w[i]); x[2 * i + 1] = bf16_hi_to_f32(w[i]); }
      else x[i] = __uint_as_float(w[i]);
    }
  }
  __device__ __forceinline__ u32x4 piece(int i) const { return *(const u32x4*)(p + head + (long long)i * VE); }
  // f(value, token) for the element of the head or tail that is the thread's, if there is one
  template <typename F>
  __device__ __forceinline__ void edges(F f) const {
    if (first && (int)threadIdx.x < head) f(value(p[threadIdx.x]), (int)threadIdx.x);
    if (last && tail + (int)threadIdx.x < vocab && (int)threadIdx.x < VE) f(value(p[tail + threadIdx.x]), tail + (int)threadIdx.x);
  }
};

__device__ __forceinline__ top_key top_wave_max64(top_key x) {
#pragma unroll
  for (int off = PC_WAVE / 2; off > 0; off >>= 1) {
    const top_key y = __shfl_xor(x, off);
    x = y > x ? y : x;
  }
  return x;
}
template <int THREADS>
__device__ __forceinline__ top_key top_block_max(top_key x) {
  __shared__ top_key red[THREADS / PC_WAVE];
  x = top_wave_max64(x);
  __syncthreads();
  if (threadIdx.x % PC_WAVE == 0) red[threadIdx.x / PC_WAVE] = x;
  __syncthreads();
  x = red[0];
#pragma unroll
  for (int w = 1; w < THREADS / PC_WAVE; ++w) x = red[w] > x ? red[w] : x;
  return x;
}
template <int THREADS>
__device__ __forceinline__ LogSum sum_block(LogSum s) {
  __shared__ LogSum red[THREADS / PC_WAVE];
#pragma unroll
  for (int off = 1; off < PC_WAVE; off <<= 1) {
    LogSum y;
    y.m = __shfl_xor(s.m, off); y.l = __shfl_xor(s.l, off); y.e = __shfl_xor(s.e, off);
    s.join(y);                                              // (lane 0's sum is the one that counts)
  }
  __syncthreads();
  if (threadIdx.x % PC_WAVE == 0) red[threadIdx.x / PC_WAVE] = s;
  __syncthreads();
  s = red[0];
#pragma unroll
  for (int w = 1; w < THREADS / PC_WAVE; ++w) s.join(red[w]);
  return s;
}

// What a row's caller gets, from its sum and its top list (LDS or the list's keys in order)
template <typename T>
__device__ __forceinline__ void logprobs_out(const PcLogprobs& c, long long row, const LogSum& s) {
  const T* p = (const T*)c.logits + row * c.row_stride;
  for (int i = threadIdx.x; i < c.n_tokens; i += blockDim.x) {
    const int v = c.tokens[row * c.n_tokens + i];
    c.token_logprob[row * c.n_tokens + i] = v >= 0 && v < c.vocab ? s.logprob(LogprobsRow<T>::value(p[v])) : NAN;
  }
  if (threadIdx.x == 0 && c.entropy) c.entropy[row] = s.entropy();
}
__device__ __forceinline__ void logprobs_top_out(const PcLogprobs& c, long long row, const LogSum& s, int i, top_key k) {
  c.top_idx[row * c.n_top + i] = top_token(k);
  if (c.top_logprob) c.top_logprob[row * c.n_top + i] = s.logprob(top_logit(k));
}

// ------------------------------------------------------------------------------------------ the largest
// largest of the wavefront's 32-bit keys, in every lane
template <int CTRL>
__device__ __forceinline__ uint32_t top_dpp_max(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ uint32_t top_wave_max(uint32_t x) {
  x = top_dpp_max<0x111>(x);                                // row_shr: 1, 2, 4, 8: lane 15 of a row has its row's
  x = top_dpp_max<0x112>(x);
  x = top_dpp_max<0x114>(x);
  x = top_dpp_max<0x118>(x);
  return max(max((uint32_t)__builtin_amdgcn_readlane((int)x, 15), (uint32_t)__builtin_amdgcn_readlane((int)x, 31)),
             max((uint32_t)__builtin_amdgcn_readlane((int)x, 47), (uint32_t)__builtin_amdgcn_readlane((int)x, 63)));
}
// A key that at least n_top of the threads' largest reach (0: every key does); full: wavefronts all of whose threads have one
__device__ __forceinline__ uint32_t top_reach(uint32_t mine, int n_top, int full, TopLds& sm) {
  const int lane = threadIdx.x % PC_WAVE, wave = threadIdx.x / PC_WAVE;
  if (full == 0) return 0;
  uint32_t x = mine, jth = 0;
  for (int j = 0; j < n_top; j += full) {                   // (uniform)
    jth = top_wave_max(x);
    const unsigned long long has = __ballot(x == jth);
    if (lane == __ffsll((long long)has) - 1) x = 0;
  }
  if (lane == 0) sm.wave[wave] = jth;
  __syncthreads();
  uint32_t least = ~0u;
  for (int w = 0; w < full; ++w) least = min(least, sm.wave[w]);
  return least;
}
__device__ __forceinline__ void top_push(TopLds& sm, top_key k) {
  const int at = atomicAdd(&sm.count, 1);
  if (at < TOP_LIST) sm.key[at] = k;
}
// f(place, key) for the list's n_top first in order; the list has no key twice
template <int THREADS, typename F>
__device__ __forceinline__ void top_in_order(const TopLds& sm, int count, int n_top, F f) {
  for (int i = threadIdx.x; i < count; i += THREADS) {
    const top_key mine = sm.key[i];
    int before = 0;
    for (int c = 0; c < count; ++c) before += sm.key[c] > mine;
    if (before < n_top) f(before, mine);
  }
}

// f(value, token) for every element of the part
template <typename T, typename F>
__device__ __forceinline__ void logprobs_each(const LogprobsRow<T>& r, F f) {
  constexpr int VE = LogprobsRow<T>::VE;
  for (int i = r.lo + (int)threadIdx.x; i < r.hi; i += LOGPROBS_THREADS) {
    float x[VE];
    LogprobsRow<T>::values(r.piece(i), x);
#pragma unroll
    for (int e = 0; e < VE; ++e) f(x[e], r.head + i * VE + e);
  }
  r.edges(f);
}
// The part's n_top-th key, digit by digit from the top: of the keys that agree with the ones before, how many have each value
// of the next eight bits
template <typename T>
__device__ __forceinline__ top_key top_nth(const LogprobsRow<T>& r, int n_top, TopLds& sm) {
  top_key known = 0, mask = 0;
  int need = n_top;
  for (int shift = 56; shift >= 0; shift -= 8) {
    if (shift == 24) { known |= 0xff000000ull; mask |= 0xff000000ull; continue; }        // (tokens are below 2^24)
    __syncthreads();
    for (int i = threadIdx.x; i < 256; i += LOGPROBS_THREADS) sm.digits[i] = 0;
    __syncthreads();
    logprobs_each(r, [&](float x, int v) {
      const top_key k = top_key_of(x, v);
      if ((k & mask) != known) return;
      const int d = (int)(k >> shift) & 255, first = __builtin_amdgcn_readfirstlane(d);
      const unsigned long long same = __ballot(d == first);                               // (ties: one addition for all of them)
      if (d != first) atomicAdd(&sm.digits[d], 1);
      else if ((int)(threadIdx.x % PC_WAVE) == __ffsll((long long)same) - 1) atomicAdd(&sm.digits[d], __popcll(same));
    });
    __syncthreads();
    int d = 255;
    for (; d > 0 && sm.digits[d] < need; --d) need -= sm.digits[d];
    known |= (top_key)d << shift;
    mask |= 255ull << shift;
  }
  return known;
}

// The part's n_top first, in order; `largest`: of the thread's logits, but for the row's edges
template <typename T, typename F>
__device__ __forceinline__ void top_of_part(const LogprobsRow<T>& r, float largest, int n_top, TopLds& sm, F f) {
  constexpr int VE = LogprobsRow<T>::VE;
  const int n = r.hi - r.lo, all = n * VE + (r.first ? r.head : 0) + (r.last ? r.vocab - r.tail : 0);
  const int want = min(n_top, all);
  const uint32_t mine = (int)threadIdx.x < n ? pc_order_key(largest) : 0;
  if (threadIdx.x == 0) sm.count = sm.threads = 0;
  const uint32_t reach = top_reach(mine, want, min(n / PC_WAVE, LOGPROBS_WAVES), sm);
  __syncthreads();
  if ((int)threadIdx.x < n && mine >= reach) sm.thread[atomicAdd(&sm.threads, 1)] = (uint16_t)threadIdx.x;
  r.edges([&](float x, int v) { if (pc_order_key(x) >= reach) top_push(sm, top_key_of(x, v)); });
  __syncthreads();
  const int threads = sm.threads, rounds = (n + LOGPROBS_THREADS - 1) / LOGPROBS_THREADS;
  for (int j = threadIdx.x; j < threads * rounds; j += LOGPROBS_THREADS) {
    const int round = j / threads, i = r.lo + round * LOGPROBS_THREADS + sm.thread[j - round * threads];
    if (i >= r.hi) continue;
    float x[VE];
    LogprobsRow<T>::values(r.piece(i), x);
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (pc_order_key(x[e]) >= reach) top_push(sm, top_key_of(x[e], r.head + i * VE + e));
  }
  __syncthreads();
  int count = sm.count;
  if (count > TOP_LIST || count < want) {
    const top_key nth = top_nth(r, want, sm);
    __syncthreads();
    if (threadIdx.x == 0) sm.count = 0;
    __syncthreads();
    logprobs_each(r, [&](float x, int v) { if (top_key_of(x, v) >= nth) top_push(sm, top_key_of(x, v)); });
    __syncthreads();
    count = sm.count;
  }
  top_in_order<LOGPROBS_THREADS>(sm, count, n_top, f);
  for (int i = want + (int)threadIdx.x; i < n_top; i += LOGPROBS_THREADS) f(i, (top_key)0);
}

template <typename T>
__global__ __launch_bounds__(LOGPROBS_THREADS) void logprobs_rows_kernel(LogprobsArgs a) {
  constexpr int VE = LogprobsRow<T>::VE, U = 4;
  __shared__ TopLds sm;
  const int row = pc_div((int)blockIdx.x, a.parts_div), part = (int)blockIdx.x - row * a.parts;
  const LogprobsRow<T> r(a.c, row, part, a.parts);
  LogSum s;
  s.clear();
  float largest = -INFINITY;
  for (int i0 = r.lo + (int)threadIdx.x; i0 < r.hi; i0 += U * LOGPROBS_THREADS) {
    u32x4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = r.piece(min(i0 + u * LOGPROBS_THREADS, r.hi - 1));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * LOGPROBS_THREADS >= r.hi) break;
      float x[VE];
      LogprobsRow<T>::values(w[u], x);
      largest = fmaxf(largest, s.add(x));
    }
  }
  r.edges([&](float x, int) { const float one[1] = {x}; s.add(one); });
  s = sum_block<LOGPROBS_THREADS>(s);
  if (a.parts == 1) logprobs_out<T>(a.c, row, s);
  else if (threadIdx.x == 0) a.sums[blockIdx.x] = s;
  if (a.c.n_top == 0) return;
  if (a.parts == 1) top_of_part(r, largest, a.c.n_top, sm, [&](int i, top_key k) { logprobs_top_out(a.c, row, s, i, k); });
  else top_of_part(r, largest, a.c.n_top, sm, [&](int i, top_key k) { a.tops[(long long)blockIdx.x * a.c.n_top + i] = k; });
}

// A row's parts, joined.  The largest of the parts' n_top-th keys is one that n_top keys reach.
#define JOIN_THREADS 256
template <typename T>
__global__ __launch_bounds__(JOIN_THREADS) void logprobs_join_kernel(LogprobsArgs a) {
  __shared__ TopLds sm;
  const long long row = blockIdx.x;
  const int n_top = a.c.n_top;
  LogSum s;
  s.clear();
  for (int i = threadIdx.x; i < a.parts; i += JOIN_THREADS) s.join(a.sums[row * a.parts + i]);
  s = sum_block<JOIN_THREADS>(s);
  logprobs_out<T>(a.c, row, s);
  if (n_top == 0) return;
  const top_key* tops = a.tops + row * a.parts * n_top;
  top_key reach = 1;                                        // (0 is nobody)
  for (int i = threadIdx.x; i < a.parts; i += JOIN_THREADS) {
    const top_key k = tops[(long long)i * n_top + n_top - 1];
    reach = k > reach ? k : reach;
  }
  reach = top_block_max<JOIN_THREADS>(reach);
  if (threadIdx.x == 0) sm.count = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < a.parts * n_top; i += JOIN_THREADS) {
    const top_key k = tops[i];
    if (k >= reach) top_push(sm, k);
  }
  __syncthreads();
  const int count = sm.count;
  if (count <= TOP_LIST) {
    top_in_order<JOIN_THREADS>(sm, count, n_top, [&](int i, top_key k) { logprobs_top_out(a.c, row, s, i, k); });
    return;
  }
  top_key below = ~0ull;                                    // (parts whose lists end alike: one after the other)
  for (int i = 0; i < n_top; ++i) {
    top_key best = 0;
    for (int c = threadIdx.x; c < a.parts * n_top; c += JOIN_THREADS)
      if (tops[c] < below && tops[c] > best) best = tops[c];
    below = top_block_max<JOIN_THREADS>(best);
    if (threadIdx.x == 0) logprobs_top_out(a.c, row, s, i, below);
  }
}

// ---- host
static int logprobs_parts(int rows, int vocab) {
  const int parts = 512 / (rows < 1 ? 1 : rows), most = vocab / 4096;
  return parts < 1 || most < 1 ? 1 : (parts < most ? parts : most);
}
size_t pc_logprobs_ws_bytes(int rows, int vocab, int n_top) {
  const size_t n = (size_t)rows * logprobs_parts(rows, vocab);
  return pc_align_up(n * sizeof(LogSum), 256) + pc_align_up(n * n_top * sizeof(top_key), 256) + 256;
}

template <typename T>
static int launch(const LogprobsArgs& a, hipStream_t st) {
  {
    PcProfScope prof(PC_KERNEL_LOGPROBS, st);
    hipLaunchKernelGGL(logprobs_rows_kernel<T>, dim3((unsigned)(a.c.rows * a.parts)), dim3(LOGPROBS_THREADS), 0, st, a);
    PC_LAUNCH_CHECK();
  }
  if (a.parts == 1) return PC_OK;
  PcProfScope prof(PC_KERNEL_LOGPROBS_JOIN, st);
  hipLaunchKernelGGL(logprobs_join_kernel<T>, dim3((unsigned)a.c.rows), dim3(256), 0, st, a);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
int pc_launch_logprobs(const PcLogprobs& c, void* ws, hipStream_t st) {
  LogprobsArgs a;
  a.c = c;
  a.parts = logprobs_parts(c.rows, c.vocab);
  a.parts_div = pc_div_by(a.parts);
  a.sums = (LogSum*)ws;
  a.tops = (top_key*)((char*)ws + pc_align_up((size_t)c.rows * a.parts * sizeof(LogSum), 256));
  return c.fp32 ? launch<float>(a, st) : launch<uint16_t>(a, st);
}
