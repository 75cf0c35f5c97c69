// Verification of drafted tokens against the target's probabilities, from given random numbers.  Draft i of a sequence
// stands iff u_i q_i(d_i) < p_i(d_i) and all before it stand.  With a standing of n, the token that follows is drawn
// from r = max(p_a - q_a, 0) (a < n; p_a where that is zero throughout) or r = p_n (a = n) as the race
//   argmax_v r(v) / noise(v)  over r(v) > 0, the lowest v at ties,
// which r(v) / sum r wins with noise ~ Exp(1).  Nothing but a product, a difference, a correctly rounded quotient and
// comparisons, each in 32 bits and of one vocabulary entry: the answer does not depend on how the entries are dealt out.
// Bound by memory (one row of p, of noise and, after a rejection, of q), and at few sequences by two launches' latency:
// a row is cut into parts, one workgroup each, whose winners a second launch compares.
#include "serve.h"

#define VERIFY_THREADS 256

// (ratio, index) as one word whose order is that of the race: larger ratio, then lower index.  0: nobody.
typedef unsigned long long verify_key;
__device__ __forceinline__ verify_key verify_make(float ratio, int v) {
  return ((verify_key)__float_as_uint(ratio) << 32) | (uint32_t)~v;
}
__device__ __forceinline__ void verify_entry(float r, float noise, int v, verify_key& best) {
  if (!(r > 0.f)) return;
  const float ratio = r / noise;
  if (!(ratio >= 0.f)) return;                               // a NaN, or a noise below zero
  const verify_key k = verify_make(ratio, v);
  best = k > best ? k : best;
}

struct VerifyArgs {
  PcVerifyCall c;
  int parts, per_part;     // workgroups a sequence, entries each
  verify_key* race;        // [B, parts, 2]: the residual's winner, the target row's
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
        stands = false;
        if (d >= 0 && d < c.vocab) {
          const float p = c.target_prob[((long long)b * (c.n_draft + 1) + i) * c.vocab + d];
          const float q = c.draft_prob ? c.draft_prob[at * c.vocab + d] : 1.0f;
          stands = c.u[at] * q < p;
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

__device__ __forceinline__ verify_key verify_max(verify_key x, verify_key* red) {
  for (int off = PC_WAVE / 2; off > 0; off >>= 1) {
    const verify_key y = __shfl_xor(x, off);
    x = y > x ? y : x;
  }
  if (threadIdx.x % PC_WAVE == 0) red[threadIdx.x / PC_WAVE] = x;
  __syncthreads();
  for (int w = 0; w < VERIFY_THREADS / PC_WAVE; ++w) x = red[w] > x ? red[w] : x;
  __syncthreads();
  return x;
}

__global__ __launch_bounds__(VERIFY_THREADS) void verify_race_kernel(VerifyArgs x) {
  __shared__ verify_key red[VERIFY_THREADS / PC_WAVE];
  const PcVerifyCall& c = x.c;
  const int b = blockIdx.x / x.parts, part = blockIdx.x % x.parts;
  const int n = verify_drafts(c, b), a = verify_standing(c, b, n);
  const float* p = c.target_prob + ((long long)b * (c.n_draft + 1) + a) * c.vocab;
  const float* q = a < n && c.draft_prob ? c.draft_prob + ((long long)b * c.n_draft + a) * c.vocab : nullptr;
  const int hole = a < n && !c.draft_prob ? c.draft[(long long)b * c.n_draft + a] : -1;
  const float* noise = c.noise + (long long)b * c.vocab;
  verify_key rest = 0, whole = 0;
  const int hi = min(c.vocab, (part + 1) * x.per_part);
  for (int v = part * x.per_part + threadIdx.x; v < hi; v += VERIFY_THREADS) {
    const float pv = p[v], e = noise[v];
    const float qv = q ? q[v] : (v == hole ? 1.0f : 0.0f);
    verify_entry(pv - qv, e, v, rest);
    verify_entry(pv, e, v, whole);
  }
  rest = verify_max(rest, red);
  whole = verify_max(whole, red);
  if (threadIdx.x == 0) {
    verify_key* dst = x.race + 2LL * blockIdx.x;
    dst[0] = rest; dst[1] = whole;
  }
}

__global__ __launch_bounds__(PC_WAVE) void verify_pick_kernel(VerifyArgs x) {
  const PcVerifyCall& c = x.c;
  const int b = blockIdx.x;
  const int n = verify_drafts(c, b), a = verify_standing(c, b, n);
  verify_key rest = 0, whole = 0;
  for (int i = threadIdx.x; i < x.parts; i += PC_WAVE) {
    const verify_key* src = x.race + 2 * ((long long)b * x.parts + i);
    rest = src[0] > rest ? src[0] : rest;
    whole = src[1] > whole ? src[1] : whole;
  }
  for (int off = PC_WAVE / 2; off > 0; off >>= 1) {
    const verify_key y = __shfl_xor(rest, off), z = __shfl_xor(whole, off);
    rest = y > rest ? y : rest;
    whole = z > whole ? z : whole;
  }
  const verify_key won = rest ? rest : whole;
  const int token = won ? (int)~(uint32_t)won : -1;
  for (int i = threadIdx.x; i <= c.n_draft; i += PC_WAVE)
    c.tokens[(long long)b * (c.n_draft + 1) + i] = i < a ? c.draft[(long long)b * c.n_draft + i] : (i == a ? token : -1);
  if (threadIdx.x == 0) {
    c.count[b] = a;
    if (c.len_out) c.len_out[b] = c.len_in[b] + 1 + a;
  }
}

static int verify_parts(int batch, int vocab) {
  int parts = 512 / batch, most = (vocab + 1023) / 1024;
  parts = parts < 1 ? 1 : parts;
  return parts < most ? parts : most;
}
size_t pc_verify_ws_bytes(int batch, int vocab) { return (size_t)batch * verify_parts(batch, vocab) * 2 * sizeof(verify_key); }

int pc_launch_verify(const PcVerifyCall& c, void* ws, hipStream_t st) {
  VerifyArgs x;
  x.c = c; x.race = (verify_key*)ws;
  x.parts = verify_parts(c.batch, c.vocab);
  x.per_part = (c.vocab + x.parts - 1) / x.parts;
  {
    PcProfScope prof(PC_KERNEL_VERIFY_RACE, st);
    hipLaunchKernelGGL(verify_race_kernel, dim3((unsigned)(c.batch * x.parts)), dim3(VERIFY_THREADS), 0, st, x);
    PC_LAUNCH_CHECK();
  }
  PcProfScope prof(PC_KERNEL_VERIFY_PICK, st);
  hipLaunchKernelGGL(verify_pick_kernel, dim3((unsigned)c.batch), dim3(PC_WAVE), 0, st, x);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
