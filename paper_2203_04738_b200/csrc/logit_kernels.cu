// Operators over rows of logits: log probabilities of given tokens with entropy and top alternatives, their gradient, and
// distillation from a teacher's top logits.
#include <math.h>

#include "elem.cuh"

namespace mg {
namespace {

constexpr int kMaxTop = 128, kMaxTeacher = 1024;
constexpr int kRowThreads = 256, kRowWarps = kRowThreads / 32;

// sum of v over the block, the same bits in every thread
__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < kRowWarps; ++w) s += red[w];
  return s;
}
__device__ __forceinline__ float block_max(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = red[0];
#pragma unroll
  for (int w = 1; w < kRowWarps; ++w) s = fmaxf(s, red[w]);
  return s;
}

// Order of the alternatives as one whole number: the value's bits so that they rise with the value (-0 as +0, NaN below -inf), then the
// token, lower ones first.  Every key of a row is different and above zero.
__device__ __forceinline__ unsigned long long top_key(float x, int v) {
  x += 0.f;
  const int b = __float_as_int(x);
  const unsigned u = x != x ? 0u : (unsigned)(b < 0 ? b ^ 0x7fffffff : b) ^ 0x80000000u;
  return ((unsigned long long)u << 32) | (unsigned)(0xffffffffu - (unsigned)v);
}

struct LogprobArgs {
  int N, V, top; i64 ld;
  const int32_t* tokens; float *logprob, *entropy, *lse, *top_logprob; int32_t* top_id;
};

template <class T>
__global__ void __launch_bounds__(kRowThreads) logprob_kernel(const T* __restrict__ logits, const LogprobArgs a) {
  __shared__ float red[kRowWarps];
  __shared__ unsigned long long best[kRowWarps];
  const int r = blockIdx.x;
  const T* x = logits + (i64)r * a.ld;
  float m = -INFINITY;
  for (int v = threadIdx.x; v < a.V; v += kRowThreads) m = fmaxf(m, to_f32(x[v]));
  m = block_max(m, red);
  const float m0 = m == -INFINITY ? 0.f : m;
  float s = 0.f, w = 0.f;
  for (int v = threadIdx.x; v < a.V; v += kRowThreads) {
    const float d = to_f32(x[v]) - m0, e = expf(d);
    s += e;
    w += e == 0.f ? 0.f : e * d;
  }
  s = block_sum(s, red);
  w = block_sum(w, red);
  // (log probabilities are (x - max) - log sum: x - lse would lose the second part where the row lies far from zero)
  const float lse = s == 0.f ? -INFINITY : m0 + logf(s);
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[r] = lse;
    if (a.entropy) a.entropy[r] = s == 0.f ? 0.f : logf(s) - w / s;
    if (a.tokens) {
      const int t = a.tokens[r];
      const float y = t >= 0 && t < a.V ? to_f32(x[t]) : 0.f;
      a.logprob[r] = t >= 0 && t < a.V ? (s == 0.f ? -INFINITY : (y - m0) - logf(s)) : 0.f;
    }
  }
  unsigned long long last = ~0ull;
  for (int k = 0; k < a.top; ++k) {
    unsigned long long mine = 0;
    for (int v = threadIdx.x; v < a.V; v += kRowThreads) {
      const unsigned long long q = top_key(to_f32(x[v]), v);
      if (q < last && q > mine) mine = q;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long q = __shfl_xor_sync(0xffffffffu, mine, o);
      mine = q > mine ? q : mine;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) best[threadIdx.x >> 5] = mine;
    __syncthreads();
    last = best[0];
    for (int q = 1; q < kRowWarps; ++q) last = best[q] > last ? best[q] : last;
    if (threadIdx.x == 0) {
      const int v = (int)(0xffffffffu - (unsigned)last);
      a.top_id[(i64)r * a.top + k] = v;
      a.top_logprob[(i64)r * a.top + k] = s == 0.f ? -INFINITY : (to_f32(x[v]) - m0) - logf(s);
    }
  }
}

struct LogprobGradArgs {
  int N, V; i64 ld, dld;
  const int32_t* tokens; const float *lse, *entropy, *dlogprob, *dentropy;
};

template <class T>
__global__ void __launch_bounds__(kRowThreads) logprob_back_kernel(const T* logits, T* dlogits, const LogprobGradArgs a) {
  const int r = blockIdx.x;
  const T* x = logits + (i64)r * a.ld;
  T* d = dlogits + (i64)r * a.dld;
  const int tok = a.tokens ? a.tokens[r] : -1;
  const bool has = tok >= 0 && tok < a.V;
  const float gl = has ? a.dlogprob[r] : 0.f, ge = a.dentropy ? a.dentropy[r] : 0.f, ent = a.dentropy ? a.entropy[r] : 0.f, lse = a.lse[r];
  for (int v = threadIdx.x; v < a.V; v += kRowThreads) {
    const float logp = to_f32(x[v]) - lse, p = lse == -INFINITY ? 0.f : expf(logp);
    float g = p == 0.f ? 0.f : -p * (gl + ge * (logp + ent));
    if (v == tok && lse != -INFINITY) g += gl;
    d[v] = from_f32<T>(g);
  }
}

struct DistillArgs {
  int N, V, K; i64 ld, dld; float tau;
  const int32_t* top_id; const float *top_logit, *weight; float* row_loss;
};

template <class T>
__global__ void __launch_bounds__(kRowThreads) distill_kernel(const T* logits, T* dlogits, const DistillArgs a) {
  __shared__ float red[kRowWarps];
  __shared__ float prob[kMaxTeacher];
  __shared__ int id[kMaxTeacher];
  __shared__ float logit[kMaxTeacher];
  const int r = blockIdx.x;
  const T* x = logits + (i64)r * a.ld;
  T* d = dlogits + (i64)r * a.dld;
  const float inv = 1.0f / a.tau;
  // the teacher
  float ym = -INFINITY, present = 0.f;
  for (int k = threadIdx.x; k < a.K; k += kRowThreads) {
    const int v = a.top_id[(i64)r * a.K + k];
    const bool in = v >= 0 && v < a.V;
    const float y = in ? a.top_logit[(i64)r * a.K + k] * inv : -INFINITY;
    id[k] = in ? v : -1;
    prob[k] = y;
    logit[k] = in ? to_f32(x[v]) * inv : -INFINITY;
    ym = fmaxf(ym, y);
    if (y != -INFINITY) present = 1.f;
  }
  present = block_sum(present, red);
  const float w = a.weight ? a.weight[r] : 1.0f / (float)a.N;
  ym = block_max(ym, red);
  if (ym == -INFINITY) ym = 0.f;
  float mass = 0.f;
  for (int k = threadIdx.x; k < a.K; k += kRowThreads) mass += expf(prob[k] - ym);
  mass = block_sum(mass, red);
  // the student
  float m = -INFINITY;
  for (int v = threadIdx.x; v < a.V; v += kRowThreads) m = fmaxf(m, to_f32(x[v]) * inv);
  m = block_max(m, red);
  if (m == -INFINITY) m = 0.f;
  float s = 0.f;
  for (int v = threadIdx.x; v < a.V; v += kRowThreads) s += expf(to_f32(x[v]) * inv - m);
  s = block_sum(s, red);
  const float logs = logf(s), logmass = logf(mass);
  float loss = 0.f;
  for (int k = threadIdx.x; k < a.K; k += kRowThreads) {
    const float logp = (prob[k] - ym) - logmass, p = expf(logp), z = logit[k];
    const float logq = z == -INFINITY ? -INFINITY : (z - m) - logs;
    loss += p == 0.f ? 0.f : p * (logp - logq);
    prob[k] = p;
  }
  loss = block_sum(loss, red);
  if (threadIdx.x == 0) a.row_loss[r] = present != 0.f ? a.tau * a.tau * loss : 0.f;
  const float scale = w * a.tau;
  const bool none = present == 0.f || w == 0.f;
  for (int v = threadIdx.x; v < a.V; v += kRowThreads) {
    const float e = expf(to_f32(x[v]) * inv - m);
    float q = s == 0.f ? 0.f : e / s;
    for (int k = 0; k < a.K; ++k)
      if (id[k] == v) q -= prob[k];
    d[v] = from_f32<T>(none ? 0.f : scale * q);
  }
}

__global__ void __launch_bounds__(1024) distill_loss_kernel(int N, const float* __restrict__ row_loss, const float* __restrict__ weight, float* __restrict__ loss) {
  __shared__ float part[32];
  float s = 0.f;
  for (int r = threadIdx.x; r < N; r += 1024) {
    const float w = weight ? weight[r] : 1.0f / (float)N;
    s += w == 0.f ? 0.f : w * row_loss[r];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x < 32) {
    s = part[threadIdx.x];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (threadIdx.x == 0) *loss = s;
  }
}

int check_logits(int N, int V, int dtype, const void* logits, i64 ld) {
  if (N < 0 || V <= 0 || !elem_known(dtype)) return MGRIT_INVALID_ARG;
  if (N == 0) return MGRIT_OK;
  return !logits || !elem_aligned(logits, dtype) || (N > 1 && ld < V) ? MGRIT_INVALID_ARG : MGRIT_OK;
}
int launched() { return cudaGetLastError() == cudaSuccess ? MGRIT_OK : MGRIT_CUDA_ERROR; }

}  // namespace
}  // namespace mg

extern "C" {

int token_logprobs(int32_t N, int32_t V, int32_t dtype, const void* logits, int64_t ld, const int32_t* tokens, int32_t top,
                   float* logprob, float* entropy, float* lse, float* top_logprob, int32_t* top_id, mgrit_stream_t stream) {
  using namespace mg;
  int rc = check_logits(N, V, dtype, logits, ld);
  if (rc != MGRIT_OK) return rc;
  if (top < 0 || top > V || (top > 0 && N > 0 && (!top_logprob || !top_id)) || (tokens && !logprob)) return MGRIT_INVALID_ARG;
  if (!aligned4(tokens) || !aligned4(logprob) || !aligned4(entropy) || !aligned4(lse) || !aligned4(top_logprob) || !aligned4(top_id)) return MGRIT_INVALID_ARG;
  if (top > kMaxTop) return MGRIT_UNSUPPORTED;
  if (N == 0) return MGRIT_OK;
  const LogprobArgs a{N, V, top, ld, tokens, logprob, entropy, lse, top_logprob, top_id};
  with_elem(dtype, [&](auto tag) {
    using T = decltype(tag);
    logprob_kernel<T><<<N, kRowThreads, 0, (cudaStream_t)stream>>>(static_cast<const T*>(logits), a);
  });
  count_launch();
  return launched();
}

int token_logprobs_backward(int32_t N, int32_t V, int32_t dtype, const void* logits, int64_t ld, const int32_t* tokens,
                            const float* lse, const float* entropy, const float* dlogprob, const float* dentropy, void* dlogits,
                            int64_t dld, mgrit_stream_t stream) {
  using namespace mg;
  int rc = check_logits(N, V, dtype, logits, ld);
  if (rc == MGRIT_OK) rc = check_logits(N, V, dtype, dlogits, dld);
  if (rc != MGRIT_OK) return rc;
  if (!aligned4(tokens) || !aligned4(lse) || !aligned4(entropy) || !aligned4(dlogprob) || !aligned4(dentropy)) return MGRIT_INVALID_ARG;
  if (N == 0) return MGRIT_OK;
  if (!lse || !tokens != !dlogprob || !entropy != !dentropy || (!tokens && !entropy)) return MGRIT_INVALID_ARG;
  if (dlogits == logits && dld != ld && N > 1) return MGRIT_INVALID_ARG;
  const LogprobGradArgs a{N, V, ld, dld, tokens, lse, entropy, dlogprob, dentropy};
  with_elem(dtype, [&](auto tag) {
    using T = decltype(tag);
    logprob_back_kernel<T><<<N, kRowThreads, 0, (cudaStream_t)stream>>>(static_cast<const T*>(logits), static_cast<T*>(dlogits), a);
  });
  count_launch();
  return launched();
}

int distill_topk_fwd_bwd(int32_t N, int32_t V, int32_t K, int32_t dtype, float tau, const void* logits, int64_t ld,
                         const int32_t* top_id, const float* top_logit, const float* weight, float* loss, float* row_loss,
                         void* dlogits, int64_t dld, mgrit_stream_t stream) {
  using namespace mg;
  int rc = check_logits(N, V, dtype, logits, ld);
  if (rc == MGRIT_OK) rc = check_logits(N, V, dtype, dlogits, dld);
  if (rc != MGRIT_OK) return rc;
  if (K < 1 || !(tau > 0.f) || tau > 3.0e38f || 1.0f / tau > 3.0e38f || !loss || !aligned4(loss)) return MGRIT_INVALID_ARG;
  if (K > kMaxTeacher) return MGRIT_UNSUPPORTED;
  cudaStream_t s = (cudaStream_t)stream;
  if (N > 0) {
    if (!top_id || !top_logit || !row_loss || (dlogits == logits && dld != ld && N > 1)) return MGRIT_INVALID_ARG;
    if (!aligned4(top_id) || !aligned4(top_logit) || !aligned4(weight) || !aligned4(row_loss)) return MGRIT_INVALID_ARG;
    const DistillArgs a{N, V, K, ld, dld, tau, top_id, top_logit, weight, row_loss};
    with_elem(dtype, [&](auto tag) {
      using T = decltype(tag);
      distill_kernel<T><<<N, kRowThreads, 0, s>>>(static_cast<const T*>(logits), static_cast<T*>(dlogits), a);
    });
    count_launch();
  }
  distill_loss_kernel<<<1, 1024, 0, s>>>(N, row_loss, weight, loss);
  count_launch();
  return launched();
}

}  // extern "C"
