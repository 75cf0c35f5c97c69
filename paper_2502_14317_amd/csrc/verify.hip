// Verification of drafted tokens against the target's probabilities, from given random numbers.  Draft i of a sequence
// stands iff u_i q_i(d_i) < p_i(d_i) and all before it stand.  With a standing of n, the token that follows is drawn
// from r = max(p_a - q_a, 0) (a < n; p_a where that is zero throughout) or r = p_n (a = n) as the race
//   argmax_v r(v) / noise(v)  over r(v) > 0, the lowest v at ties,
// which r(v) / sum r wins with noise ~ Exp(1).  Nothing but a product, a difference, a correctly rounded quotient and
// comparisons, each in 32 bits and of one vocabulary entry: the answer does not depend on how the entries are dealt out.
// Bound by memory (one row of p, of noise and, after a rejection, of q), at few sequences by latency: a row is cut into
// parts, a workgroup each, whose winners a second launch compares; a short row is one workgroup's, in one launch.
#include "serve.h"

#define VERIFY_U 4                       // pieces of 4 entries of each row that a thread has in flight
#define VERIFY_PART 1024                 // entries a workgroup, at least
#define VERIFY_WORKGROUPS 512            // over all sequences, about: two a CU

// four entries at any 4-byte boundary
typedef float verify_x4 __attribute__((ext_vector_type(4), aligned(4)));

// (quotient, token) as one word whose order is that of the race: larger quotient, then lower token.  0: nobody.
typedef unsigned long long verify_key;

struct VerifyRace {
  verify_key key;
  float bar;                             // the best quotient, a little less
  __device__ __forceinline__ void clear() { key = 0; bar = 0.f; }
  // A quotient that reaches the best one has r >= best noise (1 - 2^-24): the division is for those alone.  (2^-126: a
  // product below the normal numbers; one beyond them is above every r; infinite noise times nothing yet: divided.)
  __device__ __forceinline__ void entry(float r, float noise, int v) {
    if (r > 0.f && !(r + 0x1p-126f < bar * noise)) {
      const float ratio = r / noise;
      if (ratio >= 0.f) {                // (no NaN, no noise below zero)
        const verify_key k = ((verify_key)(__float_as_uint(ratio) & 0x7fffffffu) << 32) | (uint32_t)~v;
        if (k > key) {
          key = k;
          bar = ratio * (1.f - 0x1p-20f);
        }
      }
    }
  }
};

struct VerifyArgs {
  PcVerifyCall c;
  int parts, per_part;     // workgroups a sequence, entries each (a multiple of 4)
  verify_key* race;        // [B, parts]
};

__device__ __forceinline__ int verify_drafts(const PcVerifyCall& c, int b) {
  return c.draft_len ? min(max(c.draft_len[b], 0), c.n_draft) : c.n_draft;
}

// Every workgroup finds the number of standing drafts for itself (lanes of its first wavefront take a draft each)
__device__ __forceinline__ int verify_standing(const PcVerifyCall& c, int b, int n) {
  __shared__ int first;
  if (threadIdx.x < PC_WAVE) {
    int a = n;
    for (int i0 = 0; i0 < n && a == n; i0 += PC_WAVE) {
      const int i = i0 + threadIdx.x;
      bool stands = true;
      if (i < n) {
        const long long at = (long long)b * c.n_draft + i;
        const int d = c.draft[at];
        const float u = c.u[at];
        stands = false;
        if (d >= 0 && d < c.vocab) {
          const float p = c.target_prob[((long long)b * (c.n_draft + 1) + i) * c.vocab + d];
          const float q = c.draft_prob ? c.draft_prob[at * c.vocab + d] : 1.0f;
          stands = u * q < p;
        }
      }
      const unsigned long long falls = __ballot(!stands);
      if (falls) a = i0 + __ffsll((long long)falls) - 1;
    }
    if (threadIdx.x == 0) first = a;
  }
  __syncthreads();
  return first;
}

template <int THREADS>
__device__ __forceinline__ verify_key verify_max(verify_key x) {
  __shared__ verify_key red[THREADS / PC_WAVE];
  for (int off = PC_WAVE / 2; off > 0; off >>= 1) {
    const verify_key y = __shfl_xor(x, off);
    x = y > x ? y : x;
  }
  __syncthreads();
  if (threadIdx.x % PC_WAVE == 0) red[threadIdx.x / PC_WAVE] = x;
  __syncthreads();
  for (int w = 0; w < THREADS / PC_WAVE; ++w) x = red[w] > x ? red[w] : x;
  return x;
}

// The race over entries lo .. hi - 1 of p - q (q nullptr: p without its entry `hole`)
template <int THREADS, bool HAS_Q>
__device__ __forceinline__ void verify_run(const float* p, const float* q, const float* noise, int hole, int lo, int hi, VerifyRace& race) {
  constexpr int STEP = 4 * THREADS;
  const auto left = [&](int at, float x) { return at == hole ? x - 1.0f : x; };
  for (int v = lo + 4 * (int)threadIdx.x; v + 4 <= hi; v += VERIFY_U * STEP) {
    verify_x4 x[VERIFY_U], y[VERIFY_U], e[VERIFY_U];
    int at[VERIFY_U];
#pragma unroll
    for (int k = 0; k < VERIFY_U; ++k) {
      at[k] = v + k * STEP + 4 <= hi ? v + k * STEP : v;     // (a piece that runs twice wins no more than once)
      x[k] = *(const verify_x4*)(p + at[k]);
      e[k] = *(const verify_x4*)(noise + at[k]);
      if (HAS_Q) y[k] = *(const verify_x4*)(q + at[k]);
    }
#pragma unroll
    for (int k = 0; k < VERIFY_U; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) race.entry(HAS_Q ? x[k][i] - y[k][i] : left(at[k] + i, x[k][i]), e[k][i], at[k] + i);
  }
  const int v = lo + (hi - lo) / 4 * 4 + (int)threadIdx.x;   // at most three entries are left
  if (v < hi) race.entry(HAS_Q ? p[v] - q[v] : left(v, p[v]), noise[v], v);
}

template <int THREADS>
__device__ __forceinline__ verify_key verify_part(const PcVerifyCall& c, int b, int n, int a, int lo, int hi) {
  const float* p = c.target_prob + ((long long)b * (c.n_draft + 1) + a) * c.vocab;
  const float* noise = c.noise + (long long)b * c.vocab;
  VerifyRace race;
  race.clear();
  if (a < n && c.draft_prob) {
    verify_run<THREADS, true>(p, c.draft_prob + ((long long)b * c.n_draft + a) * c.vocab, noise, -1, lo, hi, race);
  } else {
    const int hole = a < n ? c.draft[(long long)b * c.n_draft + a] : -1;
    verify_run<THREADS, false>(p, nullptr, noise, hole, lo, hi, race);
  }
  return verify_max<THREADS>(race.key);
}

// The answer, from the race's winner; where nothing was left of p - q, from a race over p
template <int THREADS>
__device__ __forceinline__ void verify_answer(const PcVerifyCall& c, int b, int n, int a, verify_key won) {
  if (won == 0 && a < n) {
    VerifyRace race;
    race.clear();
    verify_run<THREADS, false>(c.target_prob + ((long long)b * (c.n_draft + 1) + a) * c.vocab, nullptr, c.noise + (long long)b * c.vocab,
                               -1, 0, c.vocab, race);
    won = verify_max<THREADS>(race.key);
  }
  const int token = won ? (int)~(uint32_t)won : -1;
  for (int i = threadIdx.x; i <= c.n_draft; i += THREADS)
    c.tokens[(long long)b * (c.n_draft + 1) + i] = i < a ? c.draft[(long long)b * c.n_draft + i] : (i == a ? token : -1);
  if (threadIdx.x == 0) {
    c.count[b] = a;
    if (c.len_out) c.len_out[b] = c.len_in[b] + 1 + a;
  }
}

__global__ __launch_bounds__(256) void verify_race_kernel(VerifyArgs x) {
  const int b = blockIdx.x / x.parts, part = blockIdx.x % x.parts;
  const int n = verify_drafts(x.c, b), a = verify_standing(x.c, b, n);
  const verify_key won = verify_part<256>(x.c, b, n, a, part * x.per_part, min(x.c.vocab, (part + 1) * x.per_part));
  if (threadIdx.x == 0) x.race[blockIdx.x] = won;
}

__global__ __launch_bounds__(256) void verify_pick_kernel(VerifyArgs x) {
  const int b = blockIdx.x;
  verify_key won = 0;
  for (int i = threadIdx.x; i < x.parts; i += 256) {
    const verify_key y = x.race[(long long)b * x.parts + i];
    won = y > won ? y : won;
  }
  const int n = verify_drafts(x.c, b), a = verify_standing(x.c, b, n);
  verify_answer<256>(x.c, b, n, a, verify_max<256>(won));
}

__global__ __launch_bounds__(1024) void verify_alone_kernel(VerifyArgs x) {
  const int b = blockIdx.x;
  const int n = verify_drafts(x.c, b), a = verify_standing(x.c, b, n);
  verify_answer<1024>(x.c, b, n, a, verify_part<1024>(x.c, b, n, a, 0, x.c.vocab));
}

// One workgroup of 16 wavefronts a sequence, in one launch, where each has a CU to itself and at most 16384 entries.  us a
// call, (sequences x entries) one launch / two:
//   (8 x 16000) 8.5 / 10.3    (8 x 24000) 11.1 / 10.7   (8 x 128256) 24.8 / 10.4   (96 x 16000) 9.3 / 10.2
//   (256 x 16000) 12.0 / 13.5 (256 x 32000) 18.4 / 18.7 (300 x 16000) 18.0 / 16.9  (400 x 4000) 15.5 / 10.3
static bool verify_alone(int batch, int vocab) { return batch <= 256 && vocab <= 16384; }
// Two launches otherwise.  With 512 / 1024 workgroups: (24 x 64000) 10.2 / 10.8, (64 x 128256) 20.6 / 21.9, (400 x 128256)
// 92 / 106.
static int verify_parts(int batch, int vocab) {
  const int parts = VERIFY_WORKGROUPS / batch, most = vocab / VERIFY_PART;
  return parts < 1 || most < 1 ? 1 : (parts < most ? parts : most);
}
size_t pc_verify_ws_bytes(int batch, int vocab) { return (size_t)batch * verify_parts(batch, vocab) * sizeof(verify_key); }

int pc_launch_verify(const PcVerifyCall& c, void* ws, hipStream_t st) {
  VerifyArgs x;
  x.c = c; x.race = (verify_key*)ws;
  x.parts = verify_parts(c.batch, c.vocab);
  x.per_part = ((c.vocab + x.parts - 1) / x.parts + 3) / 4 * 4;
  if (verify_alone(c.batch, c.vocab)) {
    PcProfScope prof(PC_KERNEL_VERIFY_ALONE, st);
    hipLaunchKernelGGL(verify_alone_kernel, dim3((unsigned)c.batch), dim3(1024), 0, st, x);
    PC_LAUNCH_CHECK();
    return PC_OK;
  }
  {
    PcProfScope prof(PC_KERNEL_VERIFY_RACE, st);
    hipLaunchKernelGGL(verify_race_kernel, dim3((unsigned)(c.batch * x.parts)), dim3(256), 0, st, x);
    PC_LAUNCH_CHECK();
  }
  PcProfScope prof(PC_KERNEL_VERIFY_PICK, st);
  hipLaunchKernelGGL(verify_pick_kernel, dim3((unsigned)c.batch), dim3(256), 0, st, x);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
