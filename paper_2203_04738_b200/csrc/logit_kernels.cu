// Operators over rows of logits: log probabilities of given tokens with entropy and top alternatives, their gradient, and
// distillation from a teacher's top logits.
//
// All are bound by HBM (a row is read once, gradients are written once) with one or two exponentials an element, which take up to three
// quarters of that time (16 a cycle and SM).  Rows of up to 16 x kThreads x kVecs vectors are held in registers:
//  * short rows (V <= 1024): a group of 8 or 32 lanes has a row;
//  * longer ones: a block, or a cluster of up to 16 blocks that share a row and meet through distributed shared memory.  A thread
//    loads all of its 16-byte vectors at once, the next row's while it works on one, so that the largest logit, the sums, the top alternatives and the gradient are all
//    formed without reading a row again, and without the rescaling that running sums need.  Few rows are split over more blocks than
//    they need, so that a single token's row of 131072 is read by 16 SMs;
//  * rows beyond that: a block per row in several passes (only their first one from HBM, the others mostly from L2).
// Rows may start anywhere: vectors are aligned in memory, the first and the last one of a row are read element by element.
#include <cooperative_groups.h>
#include <math.h>

#include "elem.cuh"

namespace cg = cooperative_groups;

namespace mg {
namespace {

constexpr int kMaxTop = 128, kMaxTeacher = 1024;
constexpr int kVecs = 16;                      // 16-byte vectors of a thread
constexpr int kMaxCluster = 16;
constexpr int kShortRow = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float max_nan(float a, float b) { float y; asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b)); return y; }

// Order of the alternatives as one whole number: the value's bits so that they rise with the value (-0 as +0, NaN below -inf), then the
// token, lower ones first.  Every key of a row is different and above zero.
__device__ __forceinline__ unsigned value_key(float x) {
  x += 0.f;
  const int b = __float_as_int(x);
  return x != x ? 0u : (unsigned)(b < 0 ? b ^ 0x7fffffff : b) ^ 0x80000000u;
}
__device__ __forceinline__ unsigned long long top_key(float x, int v) { return ((unsigned long long)value_key(x) << 32) | (unsigned)(0xffffffffu - (unsigned)v); }
__device__ __forceinline__ float key_value(unsigned k) { const unsigned u = k ^ 0x80000000u; return k == 0u ? __int_as_float(0x7fc00000) : __uint_as_float((int)u < 0 ? u ^ 0x7fffffffu : u); }
__device__ __forceinline__ int key_token(unsigned long long k) { return (int)(0xffffffffu - (unsigned)k); }

// ---- vectors of 16 bytes ---------------------------------------------------------------------------------------------------------

template <class T> struct V16 {
  static constexpr int E = 16 / sizeof(T);     // elements
  uint4 w;
  __device__ __forceinline__ float get(int i) const { return to_f32(reinterpret_cast<const T*>(&w)[i]); }
  __device__ __forceinline__ void set(int i, float v) { reinterpret_cast<T*>(&w)[i] = from_f32<T>(v); }
  __device__ __forceinline__ T& raw(int i) { return reinterpret_cast<T*>(&w)[i]; }
  // elements 2 i and 2 i + 1
  __device__ __forceinline__ F<2> pair(int i) const {
    const unsigned* u = reinterpret_cast<const unsigned*>(&w);
    if constexpr (sizeof(T) == 4) {
      return F<2>{{__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1])}};
    } else {
      const float2 f = unpack2(u[i], T{});
      return F<2>{{f.x, f.y}};
    }
  }
  __device__ __forceinline__ void set_pair(int i, const F<2>& f) {
    unsigned* u = reinterpret_cast<unsigned*>(&w);
    if constexpr (sizeof(T) == 4) {
      u[2 * i] = __float_as_uint(f.x[0]);
      u[2 * i + 1] = __float_as_uint(f.x[1]);
    } else {
      u[i] = pack2(f.x[0], f.x[1], T{});
    }
  }
};
// the largest element, NaN where there is one (two 16-bit values an instruction)
__device__ __forceinline__ unsigned max2(unsigned a, unsigned b, __nv_bfloat16) { unsigned y; asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b)); return y; }
__device__ __forceinline__ unsigned max2(unsigned a, unsigned b, __half) { unsigned y; asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b)); return y; }
template <class T> __device__ __forceinline__ float max_of(const V16<T>& v) {
  if constexpr (sizeof(T) == 4) {
    return max_nan(max_nan(v.get(0), v.get(1)), max_nan(v.get(2), v.get(3)));
  } else {
    V16<T> m;
    m.w.x = max2(max2(v.w.x, v.w.y, T{}), max2(v.w.z, v.w.w, T{}), T{});
    return max_nan(m.get(0), m.get(1));
  }
}

// A row's place in memory: `skip` elements lie between the 16-byte word in which it starts and its first element
template <class T> struct RowAt {
  T* base;                                     // that word
  int skip, vecs;                              // vectors that hold some of the row
  __device__ __forceinline__ RowAt(T* row, int V) {
    skip = (int)(((uintptr_t)row & 15u) / sizeof(T));
    base = row - skip;
    vecs = (int)(((i64)V + skip + V16<T>::E - 1) / V16<T>::E);
  }
};
template <class T> __device__ __forceinline__ V16<T> load_vec(const T* row, const RowAt<const T>& at, int i, int V) {
  constexpr int E = V16<T>::E;
  V16<T> v;
  if (i > 0 && i + 1 < at.vecs) {
    v.w = __ldcs(reinterpret_cast<const uint4*>(at.base) + i);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int k = i * E + e - at.skip;
      v.raw(e) = k >= 0 && k < V ? row[k] : from_f32<T>(-INFINITY);
    }
  }
  return v;
}

// A block's share of a row on its way to registers: a thread copies its vectors to its own places in shared memory, asynchronously, while the
// row before is worked on, and reads them back itself, so nobody waits for anybody.  Vectors at a row's ends are copied whole where the
// bytes around the row belong to the array (they are replaced by -inf when read back), and element by element where they do not.
template <class T, int NT> struct Stage {
  static constexpr int E = V16<T>::E;
  const T *first, *end;                        // the array
  i64 ld;
  int V, cluster, rank;
  uint4* mine;                                 // the thread's places, NT apart
  __device__ __forceinline__ int share(const RowAt<const T>& at) const { return (at.vecs + cluster - 1) / cluster; }
  __device__ __forceinline__ void bring(i64 r) const {
    const T* row = first + r * ld;
    const RowAt<const T> at(row, V);
    const int per = share(at), lo = rank * per, n = max(0, min(at.vecs - lo, per));
    const T* p = at.base + (i64)(lo + (int)threadIdx.x) * E;
    const unsigned to = (unsigned)__cvta_generic_to_shared(mine);
    // all but the array's own ends, where a vector would reach outside
    const bool cut_head = lo == 0 && at.base < first, cut_tail = n > 0 && at.base + (i64)(lo + n) * E > end;
    const int left = n - (cut_tail ? 1 : 0) - (int)threadIdx.x;
#pragma unroll
    for (int q = 0; q < kVecs; ++q)
      if (q * NT < left && !(q == 0 && cut_head && threadIdx.x == 0))
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + q * (NT * 16)), "l"(p + q * (NT * E)) : "memory");
    if (cut_head || cut_tail) {
#pragma unroll 1
      for (int q = 0; q < kVecs; ++q) {
        const int i = q * NT + (int)threadIdx.x;
        if ((cut_head && i == 0) || (cut_tail && i == n - 1)) {
#pragma unroll 1
          for (int e = 0; e < E; ++e) {
            const T* from = p + (i64)q * (NT * E) + e;
            if (from >= first && from < end) reinterpret_cast<T*>(mine + q * NT)[e] = *from;
          }
        }
      }
    }
  }
  // -> the number of the block's vectors, and where they start in the row
  __device__ __forceinline__ int take(i64 r, V16<T> (&x)[kVecs], int& lo) const {
    const RowAt<const T> at(first + r * ld, V);
    const int per = share(at);
    lo = rank * per;
    const int n = max(0, min(at.vecs - lo, per));
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (lo == 0 && threadIdx.x == 0)
#pragma unroll 1
      for (int e = 0; e < at.skip; ++e) reinterpret_cast<T*>(mine)[e] = from_f32<T>(-INFINITY);
    const int last = at.vecs - 1 - lo;         // the row's last vector, counted from the block's first
    if (last >= 0 && last < n && last % NT == (int)threadIdx.x)
#pragma unroll 1
      for (int e = V + at.skip - (at.vecs - 1) * E; e < E; ++e) reinterpret_cast<T*>(mine + last / NT * NT)[e] = from_f32<T>(-INFINITY);
#pragma unroll
    for (int q = 0; q < kVecs; ++q)
      if (q * NT < n - (int)threadIdx.x) x[q].w = mine[q * NT];
    return n;
  }
};
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// ---- reductions over a block -----------------------------------------------------------------------------------------------------

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// what the warps of a block have left, one value each: every warp puts them together for itself
template <int NW> __device__ __forceinline__ float all_max(const float* v) { const int l = threadIdx.x & 31; return warp_max(l < NW ? v[l] : -INFINITY); }
template <int NW> __device__ __forceinline__ float all_sum(const float* v) { const int l = threadIdx.x & 31; return warp_sum(l < NW ? v[l] : 0.f); }

// Statistics of some of a row's logits: the largest, m; s = sum 2^((x - m) log2 e); w = sum of the same terms times their exponents.
// A part without any logit above -inf has m = -inf and s = 0.
struct Stats { float m, s, w; };
__device__ __forceinline__ float ref_of(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ Stats joined(const Stats& a, const Stats& b) {
  const float m = max_nan(a.m, b.m), r = ref_of(m);
  const float da = (a.m - r) * kLog2e, db = (b.m - r) * kLog2e, fa = ex2(da), fb = ex2(db);
  Stats o;
  o.m = m;
  o.s = a.s * fa + b.s * fb;
  o.w = (fa == 0.f ? 0.f : fa * fmaf(a.s, da, a.w)) + (fb == 0.f ? 0.f : fb * fmaf(b.s, db, b.w));      // (da may be -inf)
  return o;
}
// log s of a row, NaN where the row holds a NaN or +inf
__device__ __forceinline__ float log_sum(const Stats& t) { return t.m != t.m || t.m == INFINITY ? __int_as_float(0x7fc00000) : logf(t.s); }

struct LogprobArgs {
  int N, V, top; i64 ld;
  const int32_t* tokens; float *logprob, *entropy, *lse, *top_logprob; int32_t* top_id;
};
// log probability of a logit of the row (x - max, then - log of the sum: x - lse would lose the second part where the row lies far from zero)
__device__ __forceinline__ float logprob_of(float x, const Stats& t, float ls) { return t.m == -INFINITY ? -INFINITY : (x - t.m) - ls; }
template <class T> __device__ __forceinline__ void write_row(const LogprobArgs& a, const T* x, int r, const Stats& t) {
  const float ls = log_sum(t);
  if (a.lse) a.lse[r] = t.m == -INFINITY ? -INFINITY : t.m + ls;
  if (a.entropy) a.entropy[r] = t.m == -INFINITY ? 0.f : ls - kLn2 * (t.w / t.s);
  if (a.tokens) {
    const int v = a.tokens[r];
    a.logprob[r] = v >= 0 && v < a.V ? logprob_of(to_f32(x[v]), t, ls) : 0.f;
  }
}

// ---- log probabilities: rows in the registers of a block or a cluster --------------------------------------------------------------

constexpr int kList = 2048;                    // candidates that a block holds: its own, or those of a cluster
static_assert(kList >= kMaxCluster * kMaxTop, "the lists of a whole cluster");

// Writes the `top` largest of n keys, in order, to out(rank, key): each key counts those above it.
template <int NT, class Out> __device__ __forceinline__ void by_rank(const unsigned long long* list, int n, int top, Out&& out) {
  for (int i = threadIdx.x; i < n; i += NT) {
    const unsigned long long k = list[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) rank += list[j] > k;
    if (rank < top) out(rank, k);
  }
}

// The top alternatives: a warp's lanes have the largest logit each of their own share, and the warp's j-th largest of these, j = top /
// warps rounded up, is a bound: at least j of its logits reach it.  So at least `top` logits reach the lowest of the warps' bounds, and
// those that do are few (some hundred of 32768 random ones for top = 20); they are put in order by counting.  Where ties or a NaN
// make them many, the largest is taken out `top` times instead.
template <class T, int NT>
__global__ void __launch_bounds__(NT, 512 / NT) logprob_kernel(const T* __restrict__ logits, const LogprobArgs a, int cluster) {
  constexpr int E = V16<T>::E, NW = NT / 32;
  extern __shared__ uint4 staged[];
  __shared__ unsigned long long list[kList];
  __shared__ unsigned long long best[2][kMaxTop];
  __shared__ float wmax[NW], wbound[NW], wsum[NW], wdot[NW];
  __shared__ Stats part[2];
  __shared__ int count[2];
  const int rank = blockIdx.x % cluster, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, step = gridDim.x / cluster;
  pdl_wait();
  pdl_trigger();
  const Stage<T, NT> stage{logits, logits + ((i64)(a.N - 1) * a.ld + a.V), a.ld, a.V, cluster, rank, staged + threadIdx.x};
  int r = blockIdx.x / cluster;
  if (r < a.N) stage.bring(r);
  copies_issued();
  if (threadIdx.x < 2) count[threadIdx.x] = 0;
  for (int buf = 0; r < a.N; r += step, buf ^= 1) {
    V16<T> x[kVecs];
    int lo;
    const int n = stage.take(r, x, lo);        // the block's vectors
    if (r + step < a.N) stage.bring(r + step);
    copies_issued();
    const T* row = logits + (i64)r * a.ld;
    const RowAt<const T> at(row, a.V);
    float m = -INFINITY;
#pragma unroll
    for (int q = 0; q < kVecs; ++q)
      if (q * NT + threadIdx.x < n) m = max_nan(m, max_of(x[q]));
    const float mine = m;
    m = warp_max(m);
    if (lane == 0) wmax[warp] = m;
    if (a.top > 0) {
      // the warp's j-th largest of its lanes' largest logits; warps without logits have no say
      const int warps = max(1, min(NW, (n + 31) / 32)), j = (a.top + warps - 1) / warps;
      unsigned k = value_key(mine), b = 0u;
      for (int i = 0; i < min(j, 32); ++i) {
        b = __reduce_max_sync(0xffffffffu, k);
        const unsigned who = __ballot_sync(0xffffffffu, k == b);
        if (lane == __ffs(who) - 1) k = 0u;
      }
      if (j > 32) b = 0u;
      if (lane == 0) wbound[warp] = warp * 32 < n ? (b == 0u ? INFINITY : -key_value(b)) : -INFINITY;
    }
    __syncthreads();
    m = all_max<NW>(wmax);
    // sums: exponents stop at -150, where the terms are zero (a term of -inf would make 0 x inf of its product)
    const float m0 = ref_of(m);
    F<2> s = F<2>::all(0.f), w = F<2>::all(0.f);
    const F<2> from = F<2>::all(-m0), scale = F<2>::all(kLog2e);
#pragma unroll
    for (int q = 0; q < kVecs; ++q) {
      if (q * NT + threadIdx.x < n) {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          const F<2> t = each((x[q].pair(e) + from) * scale, [](float v, int) { return fmaxf(v, -150.f); });
          const F<2> y = each(t, [](float v, int) { return ex2(v); });
          s = s + y;
          w = fma_(y, t, w);
        }
      }
    }
    const float s1 = warp_sum(s.x[0] + s.x[1]), w1 = warp_sum(w.x[0] + w.x[1]);
    if (lane == 0) { wsum[warp] = s1; wdot[warp] = w1; }
    if (threadIdx.x == 0) count[buf ^ 1] = 0;
    if (a.top > 0) {
      const float bound = -all_max<NW>(wbound);      // (they are kept with their signs turned)
      if (mine >= bound) {
#pragma unroll
        for (int q = 0; q < kVecs; ++q) {
          if (q * NT + threadIdx.x < n && max_of(x[q]) >= bound) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const int v = (lo + q * NT + (int)threadIdx.x) * E + e - at.skip;
              if (x[q].get(e) >= bound && v >= 0 && v < a.V) {
                const int place = atomicAdd(&count[buf], 1);
                if (place < kList) list[place] = top_key(x[q].get(e), v);
              }
            }
          }
        }
      }
    }
    __syncthreads();
    Stats t{m, 0.f, 0.f};
    t.s = all_sum<NW>(wsum);
    t.w = all_sum<NW>(wdot);
    if (m == -INFINITY) t.s = t.w = 0.f;
    const auto answer = [&](int k, unsigned long long key, const Stats& t, float ls) {
      a.top_id[(i64)r * a.top + k] = key_token(key);
      a.top_logprob[(i64)r * a.top + k] = logprob_of(key_value((unsigned)(key >> 32)), t, ls);
    };
    const float ls = log_sum(t);
    if (threadIdx.x == 0) {
      if (cluster == 1) write_row(a, row, r, t);
      else part[buf] = t;
    }
    const auto own = [&](int c) {              // how many alternatives block c of the cluster can have
      const int per = (at.vecs + cluster - 1) / cluster, l = c * per, h = min(at.vecs, l + per);
      return min(a.top, max(0, min(a.V, h * E - at.skip) - max(0, l * E - at.skip)));
    };
    if (a.top > 0) {
      const int have = own(rank), found = count[buf];
      const auto keep = [&](int k, unsigned long long key) {
        if (cluster == 1) answer(k, key, t, ls);
        else best[buf][k] = key;
      };
      if (m == m && found <= kList) {
        by_rank<NT>(list, found, have, keep);
      } else {
        unsigned long long last = ~0ull;
        for (int k = 0; k < have; ++k) {
          unsigned long long high = 0;
#pragma unroll
          for (int q = 0; q < kVecs; ++q) {
            if (q * NT + threadIdx.x < n) {
#pragma unroll
              for (int e = 0; e < E; ++e) {
                const int v = (lo + q * NT + (int)threadIdx.x) * E + e - at.skip;
                const unsigned long long key = top_key(x[q].get(e), v);
                if (v >= 0 && v < a.V && key < last && key > high) high = key;
              }
            }
          }
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) {
            const unsigned long long other = __shfl_xor_sync(0xffffffffu, high, o);
            high = other > high ? other : high;
          }
          __syncthreads();
          if (lane == 0) list[warp] = high;
          __syncthreads();
          last = list[0];
#pragma unroll
          for (int q = 1; q < NW; ++q) last = list[q] > last ? list[q] : last;
          if (threadIdx.x == 0) keep(k, last);
        }
      }
    }
    if (cluster > 1) {
      // the first block joins what the others have found, while they go on to the next row
      cg::cluster_group all = cg::this_cluster();
      all.sync();
      if (rank == 0) {
        // a lane fetches a block's statistics, a thread one alternative: one trip to the other blocks, not one for each
        t = lane < cluster ? *all.map_shared_rank(&part[buf], lane) : Stats{-INFINITY, 0.f, 0.f};
#pragma unroll
        for (int o = kMaxCluster / 2; o > 0; o >>= 1) {
          const Stats b{__shfl_down_sync(0xffffffffu, t.m, o), __shfl_down_sync(0xffffffffu, t.s, o), __shfl_down_sync(0xffffffffu, t.w, o)};
          t = joined(t, b);
        }
        t = Stats{__shfl_sync(0xffffffffu, t.m, 0), __shfl_sync(0xffffffffu, t.s, 0), __shfl_sync(0xffffffffu, t.w, 0)};
        // (places without an alternative hold zero, below every key)
        const int total = cluster * a.top;
        for (int k = threadIdx.x; k < total; k += NT) {
          const int c = k / a.top;
          list[k] = k - c * a.top < own(c) ? all.map_shared_rank(best[buf], c)[k - c * a.top] : 0ull;
        }
        __syncthreads();
        if (threadIdx.x == 0) write_row(a, row, r, t);
        const float ls = log_sum(t);
        by_rank<NT>(list, total, a.top, [&](int k, unsigned long long key) { answer(k, key, t, ls); });
      }
    }
  }
  if (cluster > 1) cg::this_cluster().sync();  // nobody leaves while its shared memory may be read
}

// ---- log probabilities of short rows -----------------------------------------------------------------------------------------------

// G lanes have a row, PER logits each
template <int G> __device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o, G);
  return v;
}
template <int G> __device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o, G));
  return v;
}
constexpr int kShortThreads = 256;

template <class T, int G, int PER>
__global__ void __launch_bounds__(kShortThreads) logprob_short_kernel(const T* __restrict__ logits, const LogprobArgs a) {
  const int l = threadIdx.x % G;
  pdl_wait();
  pdl_trigger();
  const i64 r_ = ((i64)blockIdx.x * kShortThreads + threadIdx.x) / G;
  const bool live = r_ < a.N;
  const int r = live ? (int)r_ : a.N - 1;      // (the last group's lanes go along)
  const T* row = logits + (i64)r * a.ld;
  float x[PER];
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < PER; ++i) x[i] = i * G + l < a.V ? to_f32(row[i * G + l]) : -INFINITY;
#pragma unroll
  for (int i = 0; i < PER; ++i) m = max_nan(m, x[i]);
  m = group_max<G>(m);
  const float m0 = ref_of(m);
  Stats t{m, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const float e = fmaxf((x[i] - m0) * kLog2e, -150.f), y = ex2(e);
    t.s += y;
    t.w = fmaf(y, e, t.w);
  }
  t.s = group_sum<G>(t.s);
  t.w = group_sum<G>(t.w);
  if (m == -INFINITY) t.s = t.w = 0.f;
  if (l == 0 && live) write_row(a, row, r, t);
  if (a.top == 0) return;
  // the largest key, `top` times; a lane knows the largest of its own and looks for the next one when it is taken
  const float ls = log_sum(t);
  unsigned long long last = ~0ull;
  for (int k = 0; k < a.top; ++k) {
    unsigned long long high = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const unsigned long long key = top_key(x[i], i * G + l);
      if (i * G + l < a.V && key < last && key > high) high = key;
    }
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(0xffffffffu, high, o, G);
      high = other > high ? other : high;
    }
    last = high;
    if (l == 0 && live) {
      a.top_id[(i64)r * a.top + k] = key_token(last);
      a.top_logprob[(i64)r * a.top + k] = logprob_of(key_value((unsigned)(last >> 32)), t, ls);
    }
  }
}

// ---- log probabilities of rows beyond a cluster's registers -------------------------------------------------------------------------

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
  for (int o = 16; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = red[0];
#pragma unroll
  for (int w = 1; w < kRowWarps; ++w) s = max_nan(s, red[w]);
  return s;
}

template <class T>
__global__ void __launch_bounds__(kRowThreads) logprob_wide_kernel(const T* __restrict__ logits, const LogprobArgs a) {
  __shared__ float red[kRowWarps];
  __shared__ unsigned long long best[kRowWarps];
  const int r = blockIdx.x;
  pdl_wait();
  pdl_trigger();
  const T* x = logits + (i64)r * a.ld;
  float m = -INFINITY;
  for (int v = threadIdx.x; v < a.V; v += kRowThreads) m = max_nan(m, to_f32(x[v]));
  m = block_max(m, red);
  const float m0 = ref_of(m);
  Stats t{m, 0.f, 0.f};
  for (int v = threadIdx.x; v < a.V; v += kRowThreads) {
    const float e = fmaxf((to_f32(x[v]) - m0) * kLog2e, -150.f), y = ex2(e);
    t.s += y;
    t.w = fmaf(y, e, t.w);
  }
  t.s = block_sum(t.s, red);
  t.w = block_sum(t.w, red);
  if (m == -INFINITY) t.s = t.w = 0.f;
  if (threadIdx.x == 0) write_row(a, x, r, t);
  const float ls = log_sum(t);
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
      const int v = key_token(last);
      a.top_id[(i64)r * a.top + k] = v;
      a.top_logprob[(i64)r * a.top + k] = logprob_of(to_f32(x[v]), t, ls);
    }
  }
}

// ---- gradient of log probabilities and entropies -----------------------------------------------------------------------------------

struct LogprobGradArgs {
  int N, V; i64 ld, dld;
  const int32_t* tokens; const float *lse, *entropy, *dlogprob, *dentropy;
};
constexpr int kGradThreads = 256, kGradVecs = 4;

// Statistics are given, so every element is on its own: a block has a part of a row, all of its loads in flight at once.
template <class T>
__global__ void __launch_bounds__(kGradThreads) logprob_back_kernel(const T* logits, T* dlogits, const LogprobGradArgs a, int parts) {
  constexpr int E = V16<T>::E;
  const int r = blockIdx.x / parts, lo = (blockIdx.x - r * parts) * (kGradThreads * kGradVecs);
  pdl_wait();
  pdl_trigger();
  const T* row = logits + (i64)r * a.ld;
  T* out = dlogits + (i64)r * a.dld;
  const RowAt<const T> at(row, a.V);
  const RowAt<T> to(out, a.V);
  V16<T> x[kGradVecs];
#pragma unroll
  for (int q = 0; q < kGradVecs; ++q) {
    const int i = lo + q * kGradThreads + threadIdx.x;
    if (i < at.vecs) x[q] = load_vec<T>(row, at, i, a.V);
  }
  const int tok = a.tokens ? a.tokens[r] : -1;
  const bool has = tok >= 0 && tok < a.V;
  const float gl = has ? a.dlogprob[r] : 0.f, ge = a.dentropy ? a.dentropy[r] : 0.f, ent = a.dentropy ? a.entropy[r] : 0.f, lse = a.lse[r];
  const bool dead = lse == -INFINITY;
  const float c0 = fmaf(ge, ent, gl);          // gradient: -p (gl + ge (log p + ent)), and gl at the token
#pragma unroll
  for (int q = 0; q < kGradVecs; ++q) {
    const int i = lo + q * kGradThreads + threadIdx.x;
    if (i < at.vecs) {
      V16<T> y;
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
        const F<2> logp = x[q].pair(e) + F<2>::all(-lse);
        const F<2> p = each(logp * F<2>::all(kLog2e), [](float v, int) { return ex2(v); });
        F<2> g = fma_(logp, F<2>::all(-ge), F<2>::all(-c0)) * p;
        y.set_pair(e, each(g, [&](float v, int k) { return p.x[k] == 0.f ? 0.f : v; }));
      }
      if (dead) y.w = make_uint4(0u, 0u, 0u, 0u);
      if (has && !dead && tok + at.skip >= i * E && tok + at.skip < i * E + E) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (i * E + e - at.skip == tok) {
            const float logp = x[q].get(e) - lse, p = ex2(logp * kLog2e);
            y.set(e, (p == 0.f ? 0.f : -p * fmaf(ge, logp, c0)) + gl);
          }
      }
      if (i > 0 && i + 1 < at.vecs && to.skip == at.skip) {
        *(reinterpret_cast<uint4*>(to.base) + i) = y.w;
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int v = i * E + e - at.skip;
          if (v >= 0 && v < a.V) out[v] = y.raw(e);
        }
      }
    }
  }
}

// ---- distillation --------------------------------------------------------------------------------------------------------------------

struct DistillArgs {
  int N, V, K; i64 ld, dld; float tau;
  const int32_t* top_id; const float *top_logit, *weight; float *row_loss, *loss;
};
// The student's side of one row: q = 2^((x - m) c) / s with c = log2(e) / tau
struct Student { float m, s; };

// A block, or a cluster, has a row in its registers (see above).  The gradient of the whole row is scale q; the places of the teacher's
// alternatives are written once more, by the first of those that name the same token, after the block has written the rest.
template <class T, int NT>
__global__ void __launch_bounds__(NT, 512 / NT) distill_kernel(const T* logits, T* dlogits, const DistillArgs a, int cluster) {
  constexpr int E = V16<T>::E, NW = NT / 32;
  extern __shared__ uint4 staged[];
  __shared__ float prob[2][kMaxTeacher];       // teacher: logit / tau, then probability (rows in turn: a slow warp may still read the last one's)
  __shared__ float gap[2][kMaxTeacher];        // student's logit
  __shared__ int id[2][kMaxTeacher];
  __shared__ float wm[NW], wy[NW], wany[NW], wsum[NW], wmass[NW], wloss[NW];
  __shared__ Student part[2];
  const int rank = blockIdx.x % cluster, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, step = gridDim.x / cluster;
  pdl_wait();
  pdl_trigger();
  const Stage<T, NT> stage{logits, logits + ((i64)(a.N - 1) * a.ld + a.V), a.ld, a.V, cluster, rank, staged + threadIdx.x};
  const float inv = 1.0f / a.tau, c = kLog2e * inv, uniform = 1.0f / (float)a.N;
  int r = blockIdx.x / cluster;
  if (r < a.N) stage.bring(r);
  copies_issued();
  // The thread's first alternative is fetched ahead: its token and logit two rows, the student's logit of that token one row.
  struct Teacher { int v; float y, z; };
  const bool teaches = warp * 32 < a.K;        // (the other warps have no alternatives)
  const auto named = [&](int row, int k) {
    Teacher t{-1, -INFINITY, -INFINITY};
    if (row < a.N && k < a.K) {
      t.v = a.top_id[(i64)row * a.K + k];
      t.y = a.top_logit[(i64)row * a.K + k];
    }
    return t;
  };
  const auto look_up = [&](Teacher& t, int row) {
    if (t.v >= 0 && t.v < a.V) t.z = to_f32(logits[(i64)row * a.ld + t.v]);
    else t.v = -1;
  };
  const auto weight_of = [&](int row) { return a.weight ? a.weight[min(row, a.N - 1)] : uniform; };
  Teacher now{-1, -INFINITY, -INFINITY}, soon = now;
  if (teaches) {
    now = named(r, threadIdx.x);
    look_up(now, r);
    soon = named(r + step, threadIdx.x);
  }
  float next_weight = weight_of(r);
  // Elements of vectors that the row only has a part of, written one by one by the last warp: lanes 0.. those of its first vector, lanes
  // 16.. those of its last one; the logits are fetched a row ahead.
  const auto edge_of = [&](int row) {
    if (warp != NW - 1 || row >= a.N || (lane & 15) >= E) return -1;
    const RowAt<const T> at(logits + (i64)row * a.ld, a.V);
    const int per = stage.share(at), e = lane & 15, v = (lane < 16 ? 0 : (at.vecs - 1) * E) + e - at.skip;
    if (v < 0 || v >= a.V) return -1;
    const bool partial = lane < 16 ? at.skip > 0 : at.vecs * E > a.V + at.skip;
    const int owner = (lane < 16 ? 0 : at.vecs - 1) / per;
    return partial && owner == rank ? v : -1;
  };
  int edge = edge_of(r);
  float edge_logit = edge >= 0 ? to_f32(logits[(i64)r * a.ld + edge]) : 0.f;
  for (int buf = 0; r < a.N; r += step, buf ^= 1) {
    const T* row = logits + (i64)r * a.ld;
    T* out = dlogits + (i64)r * a.dld;
    const float weight = next_weight;
    next_weight = weight_of(r + step);
    float ym = -INFINITY;
    bool any = false;
    if (teaches) {
      for (int k = threadIdx.x; k < a.K; k += NT) {
        Teacher t = now;
        if (k >= NT) {
          t = named(r, k);
          look_up(t, r);
        }
        const float y = t.v >= 0 ? t.y * inv : -INFINITY;
        id[buf][k] = t.v;
        prob[buf][k] = y;
        gap[buf][k] = t.v >= 0 ? t.z : -INFINITY;
        ym = fmaxf(ym, y);                     // (a NaN shows in the sum)
        any = any || y != -INFINITY;
      }
      now = soon;
      look_up(now, r + step);
      soon = named(r + 2 * step, threadIdx.x);
      ym = warp_max(ym);
      any = __any_sync(0xffffffffu, any);
    }
    V16<T> x[kVecs];
    int lo;
    const int n = stage.take(r, x, lo);
    if (r + step < a.N) stage.bring(r + step);
    copies_issued();
    const RowAt<const T> at(row, a.V);
    const RowAt<T> to(out, a.V);
    float m = -INFINITY;
#pragma unroll
    for (int q = 0; q < kVecs; ++q)
      if (q * NT + threadIdx.x < n) m = max_nan(m, max_of(x[q]));
    m = warp_max(m);
    if (lane == 0) { wm[warp] = m; wy[warp] = ym; wany[warp] = any ? 1.f : 0.f; }
    __syncthreads();
    m = all_max<NW>(wm);
    ym = all_max<NW>(wy);
    const float present = all_max<NW>(wany);
    const float m0 = ref_of(m), y0 = ref_of(ym);
    const F<2> scale = F<2>::all(c);
    F<2> sum = F<2>::all(0.f);
    float mass = 0.f;
#pragma unroll
    for (int q = 0; q < kVecs; ++q) {
      if (q * NT + threadIdx.x < n) {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) sum = sum + each((x[q].pair(e) + F<2>::all(-m0)) * scale, [](float v, int) { return ex2(v); });
      }
    }
    if (teaches) {
      for (int k = threadIdx.x; k < a.K; k += NT) mass += ex2((prob[buf][k] - y0) * kLog2e);
      mass = warp_sum(mass);
    }
    float s = warp_sum(sum.x[0] + sum.x[1]);
    if (lane == 0) { wsum[warp] = s; wmass[warp] = mass; }
    __syncthreads();
    s = all_sum<NW>(wsum);
    float M = m0;
    if (cluster > 1) {
      cg::cluster_group all = cg::this_cluster();
      if (threadIdx.x == 0) part[buf] = Student{m, s};
      all.sync();                              // (also: every block has read what it needs before the first gradient is written)
      const Student b = lane < cluster ? *all.map_shared_rank(&part[buf], lane) : Student{-INFINITY, 0.f};      // (one trip for all)
      M = ref_of(warp_max(b.m));
      s = warp_sum(b.s == 0.f ? 0.f : b.s * ex2((b.m - M) * c));
    }
    const float gain = weight * a.tau;
    float loss = 0.f;
    if (teaches) {
      const float ls = logf(s), lmass = logf(all_sum<NW>(wmass));
      for (int k = threadIdx.x; k < a.K; k += NT) {
        const float logp = (prob[buf][k] - y0) - lmass, p = ex2(logp * kLog2e), z = gap[buf][k];
        const float logq = z == -INFINITY ? -INFINITY : (z - M) * inv - ls;
        loss += p == 0.f ? 0.f : p * (logp - logq);
        prob[buf][k] = p;
      }
      loss = warp_sum(loss);
    }
    if (lane == 0) wloss[warp] = loss;
    const bool none = present == 0.f || weight == 0.f;
    const F<2> f = F<2>::all(s == 0.f ? 0.f : gain / s), from = F<2>::all(-M);
    const int whole_from = lo == 0 && at.skip > 0 ? 1 : 0;      // vectors that are the row's alone
    const int left = n - (lo + n == at.vecs && at.vecs * E > a.V + at.skip ? 1 : 0) - (int)threadIdx.x;
    if (to.skip == at.skip) {
      uint4* dst = reinterpret_cast<uint4*>(to.base) + lo + threadIdx.x;
      if (!none) {
#pragma unroll
        for (int q = 0; q < kVecs; ++q) {
          if (q * NT < left && !(q == 0 && (int)threadIdx.x < whole_from)) {
            V16<T> y;
#pragma unroll
            for (int e = 0; e < E / 2; ++e) y.set_pair(e, each((x[q].pair(e) + from) * scale, [](float v, int) { return ex2(v); }) * f);
            __stcs(dst + q * NT, y.w);
          }
        }
      } else {
#pragma unroll 1
        for (int q = 0; q < kVecs; ++q)
          if (q * NT < left && !(q == 0 && (int)threadIdx.x < whole_from)) __stcs(dst + q * NT, make_uint4(0u, 0u, 0u, 0u));
      }
    } else {                                   // rows of the two arrays start at different places of a vector
#pragma unroll
      for (int q = 0; q < kVecs; ++q) {
        if (q * NT < left && !(q == 0 && (int)threadIdx.x < whole_from)) {
          T* dst = out + (i64)(lo + q * NT + (int)threadIdx.x) * E - at.skip;
#pragma unroll
          for (int e = 0; e < E; ++e) dst[e] = from_f32<T>(none ? 0.f : ex2((x[q].get(e) - M) * c) * f.x[0]);
        }
      }
    }
    if (warp == NW - 1) {
      if (edge >= 0) out[edge] = from_f32<T>(none ? 0.f : ex2((edge_logit - M) * c) * f.x[0]);
      edge = edge_of(r + step);
      edge_logit = edge >= 0 ? to_f32(logits[(i64)(r + step) * a.ld + edge]) : 0.f;
    }
    __syncthreads();
    if (rank == 0 && warp == NW - 1) {
      const float t = all_sum<NW>(wloss);
      if (lane == 0) a.row_loss[r] = present != 0.f ? a.tau * a.tau * t : 0.f;
    }
    if (!none && teaches) {
      const int begin = lo * E - at.skip, stop = (lo + n) * E - at.skip;      // the block's own tokens
      for (int k0 = warp * 32; k0 < a.K; k0 += NT) {
        const int k = k0 + lane, v = k < a.K ? id[buf][k] : -1;
        float p = k < a.K ? prob[buf][k] : 0.f;
        bool first = true;
        const int namesakes = __popc(__match_any_sync(0xffffffffu, v));      // (every lane takes part)
        if (a.K > 32 || __any_sync(0xffffffffu, v >= 0 && namesakes > 1)) {
          // the same token may be named twice: its first place adds all of them up, in their order
          p = 0.f;
#pragma unroll 4
          for (int j = 0; j < a.K; ++j) {
            const bool same = id[buf][j] == v;
            first = first && !(same && j < k);
            p += same ? prob[buf][j] : 0.f;
          }
        }
        if (v >= 0 && v >= begin && v < stop && first) {
          const float q = s == 0.f ? 0.f : ex2((gap[buf][k] - M) * c) / s;
          out[v] = from_f32<T>(gain * (q - p));
        }
      }
    }
  }
  if (cluster > 1) cg::this_cluster().sync();  // nobody leaves while its shared memory may be read
}

// Short rows: G lanes have a row, PER logits each; the teacher's probabilities of each token meet in shared memory, in the order of the
// alternatives.
template <class T, int G, int PER>
__global__ void __launch_bounds__(kShortThreads) distill_short_kernel(const T* logits, T* dlogits, const DistillArgs a) {
  constexpr int ROWS = kShortThreads / G;
  __shared__ float target[ROWS][G * PER];
  __shared__ float part[ROWS];
  const int l = threadIdx.x % G, g = threadIdx.x / G;
  pdl_wait();
  pdl_trigger();
  const i64 r_ = (i64)blockIdx.x * ROWS + g;
  const bool live = r_ < a.N;
  const int r = live ? (int)r_ : a.N - 1;
  const T* row = logits + (i64)r * a.ld;
  T* out = dlogits + (i64)r * a.dld;
  const float inv = 1.0f / a.tau, c = kLog2e * inv;
  const float weight = a.weight ? a.weight[r] : 1.0f / (float)a.N;
  const int32_t* ids = a.top_id + (i64)r * a.K;
  const float* ys = a.top_logit + (i64)r * a.K;
  float x[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) x[i] = i * G + l < a.V ? to_f32(row[i * G + l]) : -INFINITY;
  float m = -INFINITY, s = 0.f, ym = -INFINITY, mass = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) { m = max_nan(m, x[i]); target[g][i * G + l] = 0.f; }
  m = group_max<G>(m);
  const float M = ref_of(m);
#pragma unroll
  for (int i = 0; i < PER; ++i) s += ex2((x[i] - M) * c);
  s = group_sum<G>(s);
  const auto teacher = [&](int k) {
    const int v = k < a.K ? ids[k] : -1;
    return v >= 0 && v < a.V ? ys[k] * inv : -INFINITY;
  };
  float any = 0.f;
  for (int k = l; k < a.K; k += G) {
    const float y = teacher(k);
    ym = fmaxf(ym, y);
    if (y != -INFINITY) any = 1.f;
  }
  ym = group_max<G>(ym);
  any = group_max<G>(any);
  const float y0 = ref_of(ym);
  for (int k = l; k < a.K; k += G) mass += ex2((teacher(k) - y0) * kLog2e);
  mass = group_sum<G>(mass);
  const float ls = logf(s), lmass = logf(mass);
  float loss = 0.f;
  __syncwarp();
  for (int k0 = 0; k0 < a.K; k0 += G) {
    const int k = k0 + l, v = k < a.K ? ids[k] : -1;
    const bool in = v >= 0 && v < a.V;
    float p = 0.f;
    if (in) {
      const float logp = (ys[k] * inv - y0) - lmass, z = to_f32(row[v]);
      const float logq = z == -INFINITY ? -INFINITY : (z - M) * inv - ls;
      p = ex2(logp * kLog2e);
      loss += p == 0.f ? 0.f : p * (logp - logq);
    }
    for (int j = 0; j < G; ++j) {              // (the lane that owns a token adds to it)
      const int w = __shfl_sync(0xffffffffu, in ? v : -1, j, G);
      const float pw = __shfl_sync(0xffffffffu, p, j, G);
      if (w >= 0 && w % G == l) target[g][w] += pw;
    }
  }
  loss = group_sum<G>(loss);
  loss = any != 0.f ? a.tau * a.tau * loss : 0.f;
  if (l == 0 && live) a.row_loss[r] = loss;
  const bool none = any == 0.f || weight == 0.f;
  const float scale = weight * a.tau, f = s == 0.f ? 0.f : 1.0f / s;
  __syncwarp();                                // every lane of the row has read it
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const float q = s == 0.f ? 0.f : ex2((x[i] - M) * c) * f;
    if (live && i * G + l < a.V) out[i * G + l] = from_f32<T>(none ? 0.f : scale * (q - target[g][i * G + l]));
  }
  if (gridDim.x == 1) {                        // the only block also adds the rows' losses up
    if (l == 0) part[g] = live && weight != 0.f ? weight * loss : 0.f;
    __syncthreads();
    if (threadIdx.x < 32) {
      float t = threadIdx.x < ROWS ? part[threadIdx.x] : 0.f;
      t = warp_sum(t);
      if (threadIdx.x == 0) *a.loss = t;
    }
  }
}

// rows beyond a cluster's registers
template <class T>
__global__ void __launch_bounds__(kRowThreads) distill_wide_kernel(const T* logits, T* dlogits, const DistillArgs a) {
  __shared__ float red[kRowWarps];
  __shared__ float prob[kMaxTeacher];
  __shared__ int id[kMaxTeacher];
  __shared__ float logit[kMaxTeacher];
  const int r = blockIdx.x;
  const T* x = logits + (i64)r * a.ld;
  T* d = dlogits + (i64)r * a.dld;
  const float inv = 1.0f / a.tau;
  pdl_wait();
  pdl_trigger();
  // the teacher
  float ym = -INFINITY, present = 0.f;
  for (int k = threadIdx.x; k < a.K; k += kRowThreads) {
    const int v = a.top_id[(i64)r * a.K + k];
    const bool in = v >= 0 && v < a.V;
    const float y = in ? a.top_logit[(i64)r * a.K + k] * inv : -INFINITY;
    id[k] = in ? v : -1;
    prob[k] = y;
    logit[k] = in ? to_f32(x[v]) * inv : -INFINITY;
    ym = fmaxf(ym, y);      // (a NaN shows in the sum)
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
  for (int v = threadIdx.x; v < a.V; v += kRowThreads) m = max_nan(m, to_f32(x[v]) * inv);
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
    const float q = s == 0.f ? 0.f : expf(to_f32(x[v]) * inv - m) / s;
    d[v] = from_f32<T>(none ? 0.f : scale * q);
  }
  __syncthreads();
  for (int k = threadIdx.x; k < a.K && !none; k += kRowThreads) {
    const int v = id[k];
    if (v < 0) continue;
    float p = 0.f;
    bool again = false;
    for (int j = 0; j < a.K; ++j) {
      if (id[j] != v) continue;
      again = again || j < k;
      p += prob[j];
    }
    if (!again) d[v] = from_f32<T>(scale * ((s == 0.f ? 0.f : expf(logit[k] - m) / s) - p));
  }
}

__global__ void __launch_bounds__(1024) distill_loss_kernel(int N, const float* __restrict__ row_loss, const float* __restrict__ weight, float* __restrict__ loss) {
  __shared__ float part[32];
  pdl_wait();
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
int launched(cudaError_t e) {
  count_launch();
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? MGRIT_OK : MGRIT_CUDA_ERROR;
}

// Blocks that share a row of `vecs` vectors, and their threads.  The fewest that hold it, 64 threads where they suffice; where that leaves
// SMs without work, more of them, down to two vectors a thread (8 rows of 131072 in bf16: 21 us on 32 blocks, 9 on 128).  0: too long.
struct Split { int cluster, threads; };
Split split_of(int N, i64 vecs) {
  if (vecs > (i64)kMaxCluster * 512 * kVecs) return {0, 0};
  if (vecs <= 64 * kVecs && (i64)N * ((vecs + 255) / 256) >= 296) return {1, 64};
  int c = 1;
  const int threads = vecs <= 256 * kVecs ? 256 : 512;
  while ((vecs + c - 1) / c > threads * kVecs) c *= 2;
  while (c < kMaxCluster && (i64)N * c < 148 && vecs / (2 * c) >= 1024) c *= 2;
  return {c, (vecs + c - 1) / c <= 256 * kVecs ? 256 : 512};
}
// Blocks stay for several rows, each with the next one on its way.
template <class K, class T, class... Args> cudaError_t launch_rows(K kern, int N, Split sp, cudaStream_t s, int (&known)[kMaxDevices], const T* x, Args&&... args) {
  const int dev = current_device_slot(), smem = kVecs * sp.threads * 16;
  if (dev < 0) return cudaErrorInvalidDevice;
  if (!known[dev]) {
    int per_sm = 0, sms = 0;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, sp.threads, smem);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess || per_sm * sms == 0) return e != cudaSuccess ? e : cudaErrorInvalidConfiguration;
    known[dev] = per_sm * sms;
  }
  const int most = known[dev] / sp.cluster, groups = N < most ? N : most;
  return launch_pdl_cluster(kern, sp.cluster, dim3((unsigned)(groups * sp.cluster)), dim3(sp.threads), (size_t)smem, s, x, static_cast<Args&&>(args)..., sp.cluster);
}
// vectors of a row; one more where rows start inside a vector
i64 vecs_of(int V, int dtype, const void* p, i64 ld) {
  const i64 es = (i64)elem_size(dtype);
  return (V * es + 15) / 16 + ((((uintptr_t)p | (uintptr_t)(ld * es)) & 15u) ? 1 : 0);
}

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
  cudaError_t e = cudaSuccess;
  const LogprobArgs a{N, V, top, ld, tokens, logprob, entropy, lse, top_logprob, top_id};
  with_elem(dtype, [&](auto tag) {
    using T = decltype(tag);
    const T* x = static_cast<const T*>(logits);
    cudaStream_t s = (cudaStream_t)stream;
    const Split sp = split_of(N, vecs_of(V, dtype, logits, ld));
    static int known[3][kMaxDevices];          // resident blocks of the three kernels, by device
    const auto few = [&](auto kern, int lanes) { e = launch_pdl(kern, dim3((unsigned)(((i64)N * lanes + kShortThreads - 1) / kShortThreads)), dim3(kShortThreads), 0, s, x, a); };
    if (V <= 64) few(logprob_short_kernel<T, 8, 8>, 8);
    else if (V <= 256) few(logprob_short_kernel<T, 32, 8>, 32);
    else if (V <= kShortRow) few(logprob_short_kernel<T, 32, 32>, 32);
    else if (sp.cluster == 0) e = launch_pdl(logprob_wide_kernel<T>, dim3(N), dim3(kRowThreads), 0, s, x, a);
    else if (sp.threads == 64) e = launch_rows(logprob_kernel<T, 64>, N, sp, s, known[0], x, a);
    else if (sp.threads == 256) e = launch_rows(logprob_kernel<T, 256>, N, sp, s, known[1], x, a);
    else e = launch_rows(logprob_kernel<T, 512>, N, sp, s, known[2], x, a);
  });
  return launched(e);
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
  const i64 parts = (vecs_of(V, dtype, logits, ld) + kGradThreads * kGradVecs - 1) / (kGradThreads * kGradVecs);
  if (N * parts >= INT32_MAX) return MGRIT_UNSUPPORTED;
  cudaError_t e = cudaSuccess;
  const LogprobGradArgs a{N, V, ld, dld, tokens, lse, entropy, dlogprob, dentropy};
  with_elem(dtype, [&](auto tag) {
    using T = decltype(tag);
    e = launch_pdl(logprob_back_kernel<T>, dim3((unsigned)(N * parts)), dim3(kGradThreads), 0, (cudaStream_t)stream, static_cast<const T*>(logits), static_cast<T*>(dlogits), a,
                   (int)parts);
  });
  return launched(e);
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
    const DistillArgs a{N, V, K, ld, dld, tau, top_id, top_logit, weight, row_loss, loss};
    cudaError_t e = cudaSuccess;
    bool added = false;
    with_elem(dtype, [&](auto tag) {
      using T = decltype(tag);
      const T* x = static_cast<const T*>(logits);
      T* d = static_cast<T*>(dlogits);
      const Split sp = split_of(N, vecs_of(V, dtype, logits, ld));
      static int known[3][kMaxDevices];        // resident blocks of the three kernels, by device
      const auto few = [&](auto kern, int lanes) {
        const i64 blocks = ((i64)N * lanes + kShortThreads - 1) / kShortThreads;
        added = blocks == 1;
        e = launch_pdl(kern, dim3((unsigned)blocks), dim3(kShortThreads), 0, s, x, d, a);
      };
      if (V <= 64) few(distill_short_kernel<T, 8, 8>, 8);
      else if (V <= 256) few(distill_short_kernel<T, 32, 8>, 32);
      else if (V <= kShortRow) few(distill_short_kernel<T, 32, 32>, 32);
      else if (sp.cluster == 0) e = launch_pdl(distill_wide_kernel<T>, dim3(N), dim3(kRowThreads), 0, s, x, d, a);
      else if (sp.threads == 64) e = launch_rows(distill_kernel<T, 64>, N, sp, s, known[0], x, d, a);
    else if (sp.threads == 256) e = launch_rows(distill_kernel<T, 256>, N, sp, s, known[1], x, d, a);
      else e = launch_rows(distill_kernel<T, 512>, N, sp, s, known[2], x, d, a);
    });
    rc = launched(e);
    if (rc != MGRIT_OK || added) return rc;
  }
  return launched(launch_pdl(distill_loss_kernel, dim3(1), dim3(1024), 0, s, N, (const float*)row_loss, weight, loss));
}

}  // extern "C"
