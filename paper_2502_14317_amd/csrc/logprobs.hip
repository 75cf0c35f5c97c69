// What the tokens of a vocabulary are worth: one pass over a row of logits x keeps, relative to a running maximum m of them,
// l = sum exp(x - m) and e = sum exp(x - m) (x - m), from which
//   log p(v) = x_v - m - log l,   entropy = log l - e / l.
// m is a logit, and what is multiplied by log2 e for the exponential is the difference: of a logit the product is out of range for the
// lowest and largest values of either type, and from 2^30 on its rounding alone takes the exponential out of range.
// A term of x - m = -inf is 0 (where one is met its factor is held above -1e4, and exp(-1e4) is 0); NaN and +inf make l NaN, and with it every
// number of the row.
// The n_top largest: the pass knows the largest logit of every thread.  With the j-th largest of those in each of F
// wavefronts, F j >= n_top, the least of the F is one that n_top logits at least reach, and few more do (20 of 128256: some 70).
// The threads whose largest reaches it, some F j, have their logits read once more, from the caches; those that reach it
// go to a list in LDS, where each counts how many are before it.  Where the list does not hold them (ties) or misses some (NaN),
// the n_top-th of the order (logit, token) is found eight bits at a time.
#include "paged.h"

#define LOGPROBS_THREADS 512
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
  __align__(16) uint32_t wave[2 * PC_WAVE + 4];
  uint32_t reach;
  int digits[256];
};

struct LogSum {
  float m, l, e;
  __device__ __forceinline__ void clear() { m = -INFINITY; l = 0.f; e = 0.f; }
  // relative to `to` >= m instead; where nothing but -inf has been seen l and e are 0, or NaN if a NaN has
  __device__ __forceinline__ void move(float to) {
    if (m != -INFINITY) {
      const float d = m - to, a = __builtin_amdgcn_exp2f(d * LOGPROBS_LOG2E);
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
  // N logits; largest: of them.  (A wavefront whose references stay, most of them, passes by the move.)  e is left to the caller: the
  // terms' sum is returned.  HELD: their factors are held above -1e4, and what is known of l stays
  template <int N, bool HELD = false>
  __device__ __forceinline__ float add(const float (&x)[N], float largest) {
    if constexpr (!HELD) {
      if (__any(largest > m)) {
        if (largest > m) move(largest);
      }
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = x[i] - ref, p = __builtin_amdgcn_exp2f(d * LOGPROBS_LOG2E);
      if constexpr (!HELD) l += p;
      sum = fmaf(p, HELD ? fmaxf(d, -1e4f) : d, sum);
    }
    return sum;
  }
  __device__ __forceinline__ float logprob(float x) const { return (x - m) - log2f(l) * LOGPROBS_LN2; }
  __device__ __forceinline__ float entropy() const { return log2f(l) * LOGPROBS_LN2 - e / l; }
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
  __device__ __forceinline__ static u32x4 nothing() {        // a piece of -inf
    const uint32_t w = VE == 8 ? 0xff80ff80u : 0xff800000u;
    return u32x4{w, w, w, w};
  }
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
// Over the wavefront's lanes, left in the last one: rows of 16 by shifts, then row after row
template <int CTRL, int ROWS>
__device__ __forceinline__ float sum_from(float x, float none) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(none), (int)__float_as_uint(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float sum_wave_max(float x) {
  x = fmaxf(x, sum_from<0x111, 0xf>(x, -INFINITY));         // row_shr: 1, 2, 4, 8
  x = fmaxf(x, sum_from<0x112, 0xf>(x, -INFINITY));
  x = fmaxf(x, sum_from<0x114, 0xf>(x, -INFINITY));
  x = fmaxf(x, sum_from<0x118, 0xf>(x, -INFINITY));
  x = fmaxf(x, sum_from<0x142, 0xa>(x, -INFINITY));         // row_bcast: 15, 31
  return fmaxf(x, sum_from<0x143, 0xc>(x, -INFINITY));
}
__device__ __forceinline__ float sum_wave(float x) {
  x += sum_from<0x111, 0xf>(x, 0.f);
  x += sum_from<0x112, 0xf>(x, 0.f);
  x += sum_from<0x114, 0xf>(x, 0.f);
  x += sum_from<0x118, 0xf>(x, 0.f);
  x += sum_from<0x142, 0xa>(x, 0.f);
  return x + sum_from<0x143, 0xc>(x, 0.f);
}
template <int THREADS>
__device__ __forceinline__ LogSum sum_block(LogSum s) {
  __shared__ LogSum red[THREADS / PC_WAVE];
  s.move(__uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(sum_wave_max(s.m)), PC_WAVE - 1)));
  s.l = sum_wave(s.l);
  s.e = sum_wave(s.e);
  __syncthreads();
  if (threadIdx.x % PC_WAVE == PC_WAVE - 1) red[threadIdx.x / PC_WAVE] = s;
  __syncthreads();
  LogSum all;                                               // (each wavefront's relative to the largest: nothing waits for the one before)
  all.clear();
#pragma unroll
  for (int w = 0; w < THREADS / PC_WAVE; ++w) all.m = fmaxf(all.m, red[w].m);
#pragma unroll
  for (int w = 0; w < THREADS / PC_WAVE; ++w) {
    LogSum y = red[w];
    y.move(all.m);
    all.l += y.l;
    all.e += y.e;
  }
  return all;
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
// A key that at least n_top of the threads' largest reach (0: every key does): of each full wavefront's (all of its threads have
// one) j largest, which are n_top together and a few more, the n_top-th.
__device__ __forceinline__ uint32_t top_reach(uint32_t mine, int n_top, int full, TopLds& sm) {
  const int lane = threadIdx.x % PC_WAVE, wave = threadIdx.x / PC_WAVE;
  if (full == 0) return 0;
  const int most = min((n_top + full - 1) / full + 3, PC_WAVE), n = most * full;       // 128 at most
  if (wave < full) {
    uint32_t x = mine, out = 0;
    for (int j = 0; j < most; ++j) {                        // (uniform)
      const uint32_t jth = top_wave_max(x);
      const unsigned long long has = __ballot(x == jth);
      if (lane == __ffsll((long long)has) - 1) x = 0;
      if (lane == j) out = jth;
    }
    if (lane < most) sm.wave[wave * most + lane] = out;
  }
  if (threadIdx.x < 4) sm.wave[n + threadIdx.x] = 0;        // (read with the last ones)
  __syncthreads();
  if (wave == 0) {                                          // the least of those that fewer than n_top are above
    const uint32_t a = lane < n ? sm.wave[lane] : 0, b = lane + PC_WAVE < n ? sm.wave[lane + PC_WAVE] : 0;
    int above_a = 0, above_b = 0;
#pragma unroll 4
    for (int i = 0; i < n; i += 4) {
      const u32x4 x = *(const u32x4*)&sm.wave[i];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        above_a += x[u] > a;
        above_b += x[u] > b;
      }
    }
    const uint32_t in_a = lane < n && above_a < n_top ? ~a : 0, in_b = lane + PC_WAVE < n && above_b < n_top ? ~b : 0;
    const uint32_t least = ~top_wave_max(max(in_a, in_b));
    if (lane == 0) sm.reach = least;
  }
  __syncthreads();
  return sm.reach;
}
__device__ __forceinline__ void top_push(TopLds& sm, top_key k) {
  const int at = atomicAdd(&sm.count, 1);
  if (at < TOP_LIST) sm.key[at] = k;
}
// f(place, key) for the list's n_top first in order; the list has no key twice.  Eight threads a key, each with an eighth of the
// others.
template <int THREADS, typename F>
__device__ __forceinline__ void top_in_order(const TopLds& sm, int count, int n_top, F f) {
  const int eighth = threadIdx.x % 8;
  for (int i0 = 0; i0 < count; i0 += THREADS / 8) {
    const int i = i0 + (int)threadIdx.x / 8;
    const top_key mine = sm.key[min(i, count - 1)];
    int before = 0;
#pragma unroll 4
    for (int c = eighth; c < count; c += 8) before += sm.key[c] > mine;
    before += __shfl_xor(before, 1);
    before += __shfl_xor(before, 2);
    before += __shfl_xor(before, 4);
    if (i < count && eighth == 0 && before < n_top) f(before, mine);
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
  for (int j0 = threadIdx.x; j0 < threads * rounds; j0 += 2 * LOGPROBS_THREADS) {
    u32x4 w[2];
    int i[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int j = j0 + u * LOGPROBS_THREADS, round = j / threads;
      i[u] = j < threads * rounds ? r.lo + round * LOGPROBS_THREADS + sm.thread[j - round * threads] : r.hi;
      w[u] = i[u] < r.hi ? r.piece(i[u]) : LogprobsRow<T>::nothing();
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (i[u] >= r.hi) continue;
      float x[VE];
      LogprobsRow<T>::values(w[u], x);
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (pc_order_key(x[e]) >= reach) top_push(sm, top_key_of(x[e], r.head + i[u] * VE + e));
    }
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
    float x[U * VE], top = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * LOGPROBS_THREADS >= r.hi) w[u] = LogprobsRow<T>::nothing();
      float y[VE];
      LogprobsRow<T>::values(w[u], y);
#pragma unroll
      for (int e = 0; e < VE; ++e) x[u * VE + e] = y[e];
#pragma unroll
      for (int e = 0; e < VE; e += 2) top = fmaxf(fmaxf(top, x[u * VE + e]), x[u * VE + e + 1]);
    }
    float terms = s.add(x, top);
    // A logit of -inf, or worse, or a difference of that: once more, from the caches.  Pieces behind the row's end are -inf, so this is also
    // every row's last round, unless its pieces are a multiple of the round's 2048: an eighth of 128256 16-bit logits, half of 32000.
    if (__any(terms != terms)) {
      terms = 0.f;
#pragma unroll 1
      for (int i = i0; i < min(i0 + U * LOGPROBS_THREADS, r.hi); i += LOGPROBS_THREADS) {
        float y[VE];
        LogprobsRow<T>::values(r.piece(i), y);
        terms += s.template add<VE, true>(y, 0.f);
      }
    }
    s.e += terms;
    largest = fmaxf(largest, top);
  }
  r.edges([&](float x, int) {
    const float one[1] = {x};
    s.add(one, x);
    s.e += s.template add<1, true>(one, x);
  });
  s = sum_block<LOGPROBS_THREADS>(s);
  if (a.parts == 1) logprobs_out<T>(a.c, row, s);
  else if (threadIdx.x == 0) a.sums[blockIdx.x] = s;
  if (a.c.n_top == 0) return;
  top_of_part(r, largest, a.c.n_top, sm, [&](int i, top_key k) {
    if (a.parts == 1) logprobs_top_out(a.c, row, s, i, k);
    else a.tops[(long long)blockIdx.x * a.c.n_top + i] = k;
  });
}

// A row's parts, joined.  n_top keys reach the least of the parts' j-th ones, n_top <= j parts, and the largest of their n_top-th
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
  const int jth = (n_top + a.parts - 1) / a.parts;
  top_key last = 1, least = ~0ull;                          // (0 is nobody)
  for (int i = threadIdx.x; i < a.parts; i += JOIN_THREADS) {
    const top_key k = tops[(long long)i * n_top + n_top - 1], j = tops[(long long)i * n_top + jth - 1];
    last = k > last ? k : last;
    least = j < least ? j : least;
  }
  last = top_block_max<JOIN_THREADS>(last);
  least = ~top_block_max<JOIN_THREADS>(~least);
  const top_key reach = least > last ? least : last;
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
// Workgroups a row: one, in one launch, but for few rows of more than 192 KB, which are cut into about 256 parts in all, of 16 KB at
// least.  us a call, one / 256 parts in all, 5 of the largest asked for:
//   bf16 (16 x 32000) 8.7 / 12.3   (16 x 64000) 10.6 / 12.2   (64 x 64000) 10.9 / 12.9   (4 x 128256) 14.5 / 12.2   (64 x 128256) 15.6 / 14.6   (128 x 128256) 16.4 / 17.3
//   fp32 (16 x 32000) 8.4 / 11.2   (16 x 64000) 10.7 / 11.6   (64 x 64000) 12.3 / 13.2   (4 x 128256) 15.1 / 11.7   (64 x 128256) 18.3 / 16.0   (128 x 128256) 19.2 / 20.3
// (16 and 64 rows of 250 KB are cut by this and lose 1 us.)
// Threads of a workgroup, 256 / 512 / 1024: (16 x 32000 bf16, 1) 8.4 / 8.3 / 10.1, (512 x 128256 fp32, 20) 64 / 57 / 55, (2048 x 128256 bf16, 5) 104 / 100 / 109.
#define LOGPROBS_WHOLE (192 * 1024)
#define LOGPROBS_PARTS 256
#define LOGPROBS_PART 16384
static int logprobs_parts(int rows, int vocab, int fp32) {
  const long long bytes = (long long)vocab * (fp32 ? 4 : 2);
  const int parts = LOGPROBS_PARTS / (rows < 1 ? 1 : rows), most = (int)(bytes / LOGPROBS_PART);
  if (bytes <= LOGPROBS_WHOLE || parts < 4) return 1;
  return parts < most ? parts : most;
}
// Rows in one part use none: room for the 256 parts that fewer rows are cut into, or as many as they could have (of either type: 32 bits
// have as many or more)
size_t pc_logprobs_ws_bytes(int rows, int vocab, int n_top) {
  const long long bytes = (long long)vocab * 4, most = bytes > LOGPROBS_WHOLE ? rows * (bytes / LOGPROBS_PART) : 0;
  const size_t n = (size_t)(most < LOGPROBS_PARTS ? most : LOGPROBS_PARTS);
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
  a.parts = logprobs_parts(c.rows, c.vocab, c.fp32);
  a.parts_div = pc_div_by(a.parts);
  a.sums = (LogSum*)ws;                                     // (of rows in several parts)
  a.tops = (top_key*)((char*)ws + pc_align_up((size_t)c.rows * a.parts * sizeof(LogSum), 256));
  return c.fp32 ? launch<float>(a, st) : launch<uint16_t>(a, st);
}
