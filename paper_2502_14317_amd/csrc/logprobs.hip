// What the tokens of a vocabulary are worth: one pass over a row of logits x keeps, relative to a running maximum m in log2
// units, l = sum 2^(x - m) and e = sum 2^(x - m) (x - m), from which with L = log2 l
//   log2 p(v) = x_v - m - L,   entropy / ln 2 = L - e / l.
// A term of x = -inf is 0 (its factor is held above -1e4, and 2^-1e4 is 0); NaN and +inf make l NaN, and with it every number
// of the row.
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
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N]) {
    float most = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) most = fmaxf(most, x[i]);
    most *= LOGPROBS_LOG2E;                                 // (log2 e > 0: the maximum commutes with it)
    if (most > m) move(most);
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float t = fmaf(x[i], LOGPROBS_LOG2E, -ref), p = __builtin_amdgcn_exp2f(t);
      l += p;
      e = fmaf(p, fmaxf(t, -1e4f), e);
    }
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

__device__ __forceinline__ top_key top_wave_max(top_key x) {
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
  x = top_wave_max(x);
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

template <typename T>
__global__ __launch_bounds__(LOGPROBS_THREADS) void logprobs_rows_kernel(LogprobsArgs a) {
  constexpr int VE = LogprobsRow<T>::VE, U = 4;
  const int row = pc_div((int)blockIdx.x, a.parts_div), part = (int)blockIdx.x - row * a.parts;
  const LogprobsRow<T> r(a.c, row, part, a.parts);
  LogSum s;
  s.clear();
  for (int i0 = r.lo + (int)threadIdx.x; i0 < r.hi; i0 += U * LOGPROBS_THREADS) {
    u32x4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = r.piece(min(i0 + u * LOGPROBS_THREADS, r.hi - 1));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * LOGPROBS_THREADS >= r.hi) break;
      float x[VE];
      LogprobsRow<T>::values(w[u], x);
      s.add(x);
    }
  }
  r.edges([&](float x, int) { const float one[1] = {x}; s.add(one); });
  s = sum_block<LOGPROBS_THREADS>(s);
  if (a.parts == 1) logprobs_out<T>(a.c, row, s);
  else if (threadIdx.x == 0) a.sums[blockIdx.x] = s;
  // the largest, the largest below that, ..
  top_key below = ~0ull;
  for (int k = 0; k < a.c.n_top; ++k) {
    top_key best = 0;
    const auto see = [&](float x, int v) {
      const top_key key = top_key_of(x, v);
      if (key < below && key > best) best = key;
    };
    for (int i = r.lo + (int)threadIdx.x; i < r.hi; i += LOGPROBS_THREADS) {
      float x[VE];
      LogprobsRow<T>::values(r.piece(i), x);
#pragma unroll
      for (int e = 0; e < VE; ++e) see(x[e], r.head + i * VE + e);
    }
    r.edges(see);
    below = top_block_max<LOGPROBS_THREADS>(best);
    if (threadIdx.x == 0) {
      if (a.parts == 1) logprobs_top_out(a.c, row, s, k, below);
      else a.tops[(long long)blockIdx.x * a.c.n_top + k] = below;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void logprobs_join_kernel(LogprobsArgs a) {
  const long long row = blockIdx.x;
  LogSum s;
  s.clear();
  for (int i = threadIdx.x; i < a.parts; i += 256) s.join(a.sums[row * a.parts + i]);
  s = sum_block<256>(s);
  logprobs_out<T>(a.c, row, s);
  const top_key* tops = a.tops + row * a.parts * a.c.n_top;
  top_key below = ~0ull;
  for (int k = 0; k < a.c.n_top; ++k) {
    top_key best = 0;
    for (int i = threadIdx.x; i < a.parts * a.c.n_top; i += 256) {
      const top_key key = tops[i];
      if (key < below && key > best) best = key;
    }
    below = top_block_max<256>(best);
    if (threadIdx.x == 0) logprobs_top_out(a.c, row, s, k, below);
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
