// Operators over rows of logits: log probabilities of given tokens with entropy and top alternatives, their gradient, and
// distillation from a teacher's top logits.
//
// All are bound by HBM (a row is read once, gradients are written once) with one or two exponentials an element, which take up to three
// quarters of that time (16 a cycle and SM).
//  * short rows (V <= 64): eight lanes have a row, in registers;
//  * many rows of up to some KB: a warp has a row, and no two warps wait for each other (65536 rows of 1100 logits in bf16: distillation
//    98 us, bytes 46; with a block to a row it is bound by the blocks' starts and meetings, some 3 ns a row: 484);
//  * other rows: a block, or a cluster of up to 16 that meet through distributed shared memory.  The first
//    pass streams the row once with a reference for the exponents that only moves when it has to; what is looked at twice (the gradient's
//    pass, the vectors that hold a top alternative) comes from L2, where the rows in work have room.  Small blocks and no state but the
//    sums: holding a row in registers or shared memory instead took 138 us for distillation of 4096 x 32768 in bf16 (bytes: 82), bound
//    by the length and the latency of its code with 16 warps on an SM.  Few rows are split further, so that one token's row of 131072 is
//    read by 16 SMs.
// Rows may start anywhere: whole 16-byte vectors that are the row's alone are moved as such, the few elements around them one by one.
#include <cooperative_groups.h>
#include <math.h>

#include "elem.cuh"

namespace cg = cooperative_groups;

namespace mg {
namespace {

constexpr int kMaxTop = 128, kMaxTeacher = 1024;
constexpr int kRow = 256, kBatch = 4;          // threads of a block, 16-byte vectors of a thread at a time
constexpr int kBlocks = 5;                     // on an SM: registers are kept to that (4: 115 us for distillation of 4096 x 32768 bf16; 5: 110)
constexpr int kMaxCluster = 16;
constexpr int kShortRow = 64;
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

// A block's or a warp's part of a row: n whole vectors from `first`, element v0 of the row on; and at most one of the row's other elements
// for each of the threads l < 16 (in front of the row's first whole vector, behind its last one)
template <class T> struct Part {
  static constexpr int E = V16<T>::E;
  i64 n; int v0, edge;
  const uint4* first;
  __device__ __forceinline__ Part(const T* row, int V, int cluster, int rank, int l) {
    const int skip = (int)((16u - ((uintptr_t)row & 15u)) & 15u) / (int)sizeof(T), head = min(skip, V), vecs = (V - head) / E;
    const int per = (vecs + cluster - 1) / cluster, lo = min(vecs, rank * per);
    n = min(vecs - lo, per);
    v0 = head + lo * E;
    first = reinterpret_cast<const uint4*>(row + v0);
    const int tail = V - head - vecs * E;
    edge = -1;
    if (l < 8 && rank == 0 && l < head) edge = l;
    if (l >= 8 && l < 16 && rank == cluster - 1 && l - 8 < tail) edge = head + vecs * E + l - 8;
  }
};
// how many elements block `rank` of the cluster has
template <class T> __device__ __forceinline__ int elements_of(const T* row, int V, int cluster, int rank) {
  constexpr int E = V16<T>::E;
  const int skip = (int)((16u - ((uintptr_t)row & 15u)) & 15u) / (int)sizeof(T), head = min(skip, V), vecs = (V - head) / E;
  const int per = (vecs + cluster - 1) / cluster, lo = min(vecs, rank * per);
  return min(vecs - lo, per) * E + (rank == 0 ? head : 0) + (rank == cluster - 1 ? V - head - vecs * E : 0);
}

// What a thread has seen of a row: the largest logit, m; s = sum 2^((x - r) c) and w, the same terms times their exponents, for a reference r that
// follows the largest logit only when that has left it far behind (the terms stay below 2^16; what the sums lose by it is 16 roundings).
struct Seen {
  float m = -INFINITY, r = -3.4028235e38f;
  F<2> s = F<2>::all(0.f), w = F<2>::all(0.f);
  __device__ __forceinline__ void follow(float top, float c) {
    m = max_nan(m, top);
    if ((top - r) * c > 16.f) {                // (the first time: r is the lowest value there is)
      const float d = (r - top) * c, f = ex2(d);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        w.x[i] = f == 0.f ? 0.f : f * fmaf(s.x[i], d, w.x[i]);
        s.x[i] *= f;
      }
      r = top;
    }
  }
  // W: with w.  Exponents stop at -150 there, where the terms are zero (a term of -inf would make 0 x inf of its product).
  template <bool W> __device__ __forceinline__ void add(const F<2>& x, float c) {
    F<2> t = (x + F<2>::all(-r)) * F<2>::all(c);
    if (W) t = each(t, [](float v, int) { return fmaxf(v, -150.f); });
    const F<2> y = each(t, [](float v, int) { return ex2(v); });
    s = s + y;
    if (W) w = fma_(y, t, w);
  }
};
template <bool W, class T> __device__ __forceinline__ void see_edge(Seen& t, float x, float c) {
  t.follow(x, c);
  t.add<W>(F<2>{{x, -INFINITY}}, c);
}

// The thread's vectors first + i, i = l, l + G, .. < n of a row, a batch of loads in flight at a time: sums, and the largest logits of the
// thread's best batch (which starts at `where`) and of the others.
struct Best { float high = -INFINITY, others = -INFINITY; int where = -1; };
template <int G, bool W, bool TOP, class T> __device__ __forceinline__ void see_vectors(const Part<T>& p, int l, float c, Seen& t, Best& b) {
  for (int i = l; i < p.n; i += G * kBatch) {
    V16<T> x[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (i + q * G < p.n) x[q].w = p.first[i + q * G];
    float m = -INFINITY;
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (i + q * G < p.n) m = max_nan(m, max_of(x[q]));
    t.follow(m, c);
    if (TOP) {
      if (m > b.high) { b.others = b.high; b.high = m; b.where = i; }
      else b.others = fmaxf(b.others, m);
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      if (i + q * G < p.n) {
#pragma unroll
        for (int e = 0; e < V16<T>::E / 2; ++e) t.add<W>(x[q].pair(e), c);
      }
    }
  }
}
// The thread's logits from `least` on, to offer(logit, token): as a rule those of its best batch are all
template <int G, class T, class Offer> __device__ __forceinline__ void offer_vectors(const Part<T>& p, int l, const Best& b, float least, Offer&& offer) {
  if (!(b.high >= least)) return;
  const bool all = b.others >= least;
  for (int i = all ? l : b.where; i < p.n; i += G * kBatch) {
    V16<T> x[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (i + q * G < p.n) x[q].w = p.first[i + q * G];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      if (i + q * G < p.n && max_of(x[q]) >= least) {
#pragma unroll
        for (int e = 0; e < V16<T>::E; ++e)
          if (x[q].get(e) >= least) offer(x[q].get(e), p.v0 + (i + q * G) * V16<T>::E + e);
      }
    }
    if (!all) break;
  }
}

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

// ---- log probabilities of longer rows --------------------------------------------------------------------------------------------

constexpr int kList = 2048;                    // candidates that a block holds: its own, or those of a cluster
constexpr int kRanked = 512;                   // of its own as many are put in order by counting (2 us); more are ties, and taken out one by one
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

// The top alternatives: every warp names the j largest of its threads' largest logits, j = top / warps rounded up; the top-th largest of all that
// are named is a bound that at least `top` logits reach (more than 32 names: the lowest of them).  Only threads whose largest logit reaches it look at
// their logits again, as a rule at one batch of them, since a thread knows the largest logit of its best batch and of all the others.  What
// they find, little more than `top`, is put in order by counting.  Where ties or a NaN make it much, the largest is taken out `top` times.
template <class T, bool TOP>
__global__ void __launch_bounds__(kRow, kBlocks) logprob_kernel(const T* __restrict__ logits, const LogprobArgs a, int cluster) {
  constexpr int E = V16<T>::E, NW = kRow / 32;
  __shared__ unsigned long long list[TOP ? kList : 1];
  __shared__ unsigned long long best[TOP ? kMaxTop : 1];
  __shared__ float wmax[NW], wsum[NW], wdot[NW];
  __shared__ unsigned named[TOP ? kMaxTop + 32 * NW : 1];
  __shared__ Stats part;
  __shared__ int count;
  const int r = blockIdx.x / cluster, rank = blockIdx.x - r * cluster, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  pdl_trigger();
  const T* row = logits + (i64)r * a.ld;
  const Part<T> p(row, a.V, cluster, rank, threadIdx.x);
  if (threadIdx.x == 0) count = 0;
  const float edge = p.edge >= 0 ? to_f32(row[p.edge]) : -INFINITY;
  Seen t;
  Best mine;
  see_vectors<kRow, true, TOP>(p, threadIdx.x, kLog2e, t, mine);
  if (p.edge >= 0) see_edge<true, T>(t, edge, kLog2e);
  float m = warp_max(t.m);
  if (lane == 0) wmax[warp] = m;
  // (warps without vectors have nothing to name)
  const int warps = max(1, min(NW, (int)((p.n + 31) / 32))), j = TOP ? (a.top + warps - 1) / warps : 0;
  if (TOP && warp < warps) {
    unsigned k = value_key(t.m), b = 0u;
    for (int i = 0; i < min(j, 32); ++i) {
      b = __reduce_max_sync(0xffffffffu, k);
      const unsigned who = __ballot_sync(0xffffffffu, k == b);
      if (lane == __ffs(who) - 1) k = 0u;
      if (lane == 0) named[warp * min(j, 32) + i] = b;
    }
  }
  __syncthreads();
  m = all_max<NW>(wmax);
  const float m0 = ref_of(m), d = (t.r - m0) * kLog2e, f = ex2(d);
  const float s1 = warp_sum((t.s.x[0] + t.s.x[1]) * f), w1 = warp_sum(f == 0.f ? 0.f : f * (fmaf(t.s.x[0], d, t.w.x[0]) + fmaf(t.s.x[1], d, t.w.x[1])));
  if (lane == 0) { wsum[warp] = s1; wdot[warp] = w1; }
  if (TOP) {
    unsigned bound = 0u;
    if (warps * j <= 32) {
      const unsigned theirs = lane < warps * j ? named[lane] : 0u;
      int above = 0;
#pragma unroll 8
      for (int i = 0; i < 32; ++i) {
        const unsigned o = __shfl_sync(0xffffffffu, theirs, i);
        above += o > theirs || (o == theirs && i < lane);
      }
      bound = __shfl_sync(0xffffffffu, theirs, __ffs(__ballot_sync(0xffffffffu, above == a.top - 1)) - 1);
    } else if (j <= 32) {
      bound = 0xffffffffu;
      for (int i = lane; i < warps * j; i += 32) bound = min(bound, named[i]);
      bound = __reduce_min_sync(0xffffffffu, bound);
    }
    const float least = bound == 0u ? -INFINITY : key_value(bound);
    const auto offer = [&](float x, int v) {
      const int place = atomicAdd(&count, 1);
      if (place < kRanked) list[place] = top_key(x, v);
    };
    if (p.edge >= 0 && edge >= least) offer(edge, p.edge);
    offer_vectors<kRow>(p, threadIdx.x, mine, least, offer);
  }
  __syncthreads();
  Stats all{m, all_sum<NW>(wsum), all_sum<NW>(wdot)};
  if (m == -INFINITY) all.s = all.w = 0.f;
  const auto answer = [&](int k, unsigned long long key, const Stats& t, float ls) {
    a.top_id[(i64)r * a.top + k] = key_token(key);
    a.top_logprob[(i64)r * a.top + k] = logprob_of(key_value((unsigned)(key >> 32)), t, ls);
  };
  const float ls = log_sum(all);
  if (threadIdx.x == 0) {
    if (cluster == 1) write_row(a, row, r, all);
    else part = all;
  }
  if (TOP) {
    const int have = min(a.top, elements_of(row, a.V, cluster, rank)), found = count;
    const auto keep = [&](int k, unsigned long long key) {
      if (cluster == 1) answer(k, key, all, ls);
      else best[k] = key;
    };
    if (m == m && found <= kRanked) {
      by_rank<kRow>(list, found, have, keep);
    } else {
      unsigned long long last = ~0ull;
      for (int k = 0; k < have; ++k) {
        unsigned long long top = 0;
        const auto look = [&](float x, int v) {
          const unsigned long long key = top_key(x, v);
          if (key < last && key > top) top = key;
        };
        if (p.edge >= 0) look(edge, p.edge);
        for (int i = threadIdx.x; i < p.n; i += kRow) {
          V16<T> x;
          x.w = __ldg(p.first + i);
#pragma unroll
          for (int e = 0; e < E; ++e) look(x.get(e), p.v0 + i * E + e);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          const unsigned long long other = __shfl_xor_sync(0xffffffffu, top, o);
          top = other > top ? other : top;
        }
        __syncthreads();
        if (lane == 0) list[warp] = top;
        __syncthreads();
        last = list[0];
#pragma unroll
        for (int q = 1; q < NW; ++q) last = list[q] > last ? list[q] : last;
        if (threadIdx.x == 0) keep(k, last);
      }
    }
  }
  if (cluster == 1) return;
  // the first block joins what the others have found: a lane fetches a block's statistics, a thread one alternative
  cg::cluster_group blocks = cg::this_cluster();
  blocks.sync();
  if (rank == 0) {
    all = lane < cluster ? *blocks.map_shared_rank(&part, lane) : Stats{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int o = kMaxCluster / 2; o > 0; o >>= 1) {
      const Stats b{__shfl_down_sync(0xffffffffu, all.m, o), __shfl_down_sync(0xffffffffu, all.s, o), __shfl_down_sync(0xffffffffu, all.w, o)};
      all = joined(all, b);
    }
    all = Stats{__shfl_sync(0xffffffffu, all.m, 0), __shfl_sync(0xffffffffu, all.s, 0), __shfl_sync(0xffffffffu, all.w, 0)};
    if (threadIdx.x == 0) write_row(a, row, r, all);
    if (TOP) {
      // each block's own are in order: at least `top` of all reach the lowest of the blocks' j-th ones
      const int j = (a.top + cluster - 1) / cluster;
      unsigned long long least = ~0ull;
      if (lane < cluster) least = j <= elements_of(row, a.V, cluster, lane) ? blocks.map_shared_rank(best, lane)[j - 1] : 0ull;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long other = __shfl_xor_sync(0xffffffffu, least, o);
        least = other < least ? other : least;
      }
      if (threadIdx.x == 0) count = 0;
      __syncthreads();
      for (int k = threadIdx.x; k < cluster * a.top; k += kRow) {
        const int c = k / a.top;
        if (k - c * a.top < elements_of(row, a.V, cluster, c)) {
          const unsigned long long key = blocks.map_shared_rank(best, c)[k - c * a.top];
          if (key >= least) list[atomicAdd(&count, 1)] = key;
        }
      }
      __syncthreads();
      const float ls = log_sum(all);
      by_rank<kRow>(list, count, a.top, [&](int k, unsigned long long key) { answer(k, key, all, ls); });
    }
  }
  blocks.sync();                               // nobody leaves while its shared memory may be read
}

// ---- log probabilities: a warp has a row ---------------------------------------------------------------------------------------------

constexpr int kWarpRows = 8;                   // rows of a block
constexpr int kWarpList = 128;                 // candidates of a row
constexpr int kWarpTop = 32;                   // alternatives that 32 lanes' largest logits can bound

template <class T, bool TOP>
__global__ void __launch_bounds__(kWarpRows * 32, kBlocks) logprob_warp_kernel(const T* __restrict__ logits, const LogprobArgs a) {
  constexpr int E = V16<T>::E;
  __shared__ unsigned long long lists[TOP ? kWarpRows : 1][kWarpList];
  __shared__ int counts[kWarpRows];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  pdl_trigger();
  const i64 r_ = (i64)blockIdx.x * kWarpRows + warp;
  if (r_ >= a.N) return;                       // (whole warps: nothing below waits for another)
  const int r = (int)r_;
  const T* row = logits + (i64)r * a.ld;
  const Part<T> p(row, a.V, 1, 0, lane);
  const float edge = p.edge >= 0 ? to_f32(row[p.edge]) : -INFINITY;
  Seen t;
  Best mine;
  see_vectors<32, true, TOP>(p, lane, kLog2e, t, mine);
  if (p.edge >= 0) see_edge<true, T>(t, edge, kLog2e);
  const float m = warp_max(t.m), m0 = ref_of(m), d = (t.r - m0) * kLog2e, f = ex2(d);
  Stats all{m, warp_sum((t.s.x[0] + t.s.x[1]) * f), warp_sum(f == 0.f ? 0.f : f * (fmaf(t.s.x[0], d, t.w.x[0]) + fmaf(t.s.x[1], d, t.w.x[1])))};
  if (m == -INFINITY) all.s = all.w = 0.f;
  if (lane == 0) write_row(a, row, r, all);
  if (!TOP) return;
  // the top-th largest of the lanes' largest logits: at least `top` logits reach it
  unsigned k = value_key(t.m), bound = 0u;
  for (int i = 0; i < a.top; ++i) {
    bound = __reduce_max_sync(0xffffffffu, k);
    const unsigned who = __ballot_sync(0xffffffffu, k == bound);
    if (lane == __ffs(who) - 1) k = 0u;
  }
  const float least = bound == 0u ? -INFINITY : key_value(bound), ls = log_sum(all);
  unsigned long long* list = lists[TOP ? warp : 0];
  if (lane == 0) counts[warp] = 0;
  __syncwarp();
  const auto offer = [&](float x, int v) {
    const int place = atomicAdd(&counts[warp], 1);
    if (place < kWarpList) list[place] = top_key(x, v);
  };
  if (p.edge >= 0 && edge >= least) offer(edge, p.edge);
  offer_vectors<32>(p, lane, mine, least, offer);
  __syncwarp();
  const auto answer = [&](int i, unsigned long long key) {
    a.top_id[(i64)r * a.top + i] = key_token(key);
    a.top_logprob[(i64)r * a.top + i] = logprob_of(key_value((unsigned)(key >> 32)), all, ls);
  };
  const int found = counts[warp];
  if (m == m && found <= kWarpList) {
    for (int i = lane; i < found; i += 32) {
      const unsigned long long key = list[i];
      int rank = 0;
#pragma unroll 4
      for (int q = 0; q < found; ++q) rank += list[q] > key;
      if (rank < a.top) answer(rank, key);
    }
    return;
  }
  unsigned long long last = ~0ull;             // many are equal, or there is a NaN
  for (int i = 0; i < a.top; ++i) {
    unsigned long long top = 0;
    const auto look = [&](float x, int v) {
      const unsigned long long key = top_key(x, v);
      if (key < last && key > top) top = key;
    };
    if (p.edge >= 0) look(edge, p.edge);
    for (int q = lane; q < p.n; q += 32) {
      V16<T> x;
      x.w = p.first[q];
#pragma unroll
      for (int e = 0; e < E; ++e) look(x.get(e), p.v0 + q * E + e);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(0xffffffffu, top, o);
      top = other > top ? other : top;
    }
    last = top;
    if (lane == 0) answer(i, last);
  }
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
  // the largest one, `top` times: its value's key (0: taken, or no logit), then the lowest token that has it
  const float ls = log_sum(t);
  unsigned key[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) key[i] = i * G + l < a.V ? value_key(x[i]) + 1u : 0u;
  for (int k = 0; k < a.top; ++k) {
    unsigned high = 0u, v = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < PER; ++i) high = max(high, key[i]);
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) high = max(high, __shfl_xor_sync(0xffffffffu, high, o, G));
#pragma unroll
    for (int i = PER - 1; i >= 0; --i) v = key[i] == high ? (unsigned)(i * G + l) : v;
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v = min(v, __shfl_xor_sync(0xffffffffu, v, o, G));
#pragma unroll
    for (int i = 0; i < PER; ++i) key[i] = v == (unsigned)(i * G + l) ? 0u : key[i];
    if (l == 0 && live) {
      a.top_id[(i64)r * a.top + k] = (int)v;
      a.top_logprob[(i64)r * a.top + k] = logprob_of(key_value(high - 1u), t, ls);
    }
  }
}

// ---- gradient of log probabilities and entropies -----------------------------------------------------------------------------------

struct LogprobGradArgs {
  int N, V; i64 ld, dld;
  const int32_t* tokens; const float *lse, *entropy, *dlogprob, *dentropy;
};

// one row's gradient, element by element: -p (gl + ge (log p + entropy)), and gl at the token
struct RowGrad {
  int tok; bool dead;
  float gl, ge, lse, c0;
  __device__ __forceinline__ RowGrad(const LogprobGradArgs& a, int r) {
    tok = a.tokens ? a.tokens[r] : -1;
    if (tok >= a.V) tok = -1;
    gl = tok >= 0 ? a.dlogprob[r] : 0.f;
    ge = a.dentropy ? a.dentropy[r] : 0.f;
    c0 = fmaf(ge, a.dentropy ? a.entropy[r] : 0.f, gl);
    lse = a.lse[r];
    dead = lse == -INFINITY;
  }
  __device__ __forceinline__ float one(float v, int at) const {
    const float logp = v - lse, q = ex2(logp * kLog2e), g = q == 0.f ? 0.f : -q * fmaf(ge, logp, c0);
    return dead ? 0.f : at == tok ? g + gl : g;
  }
  template <class T> __device__ __forceinline__ void vector(const V16<T>& x, int v, const T* row, T* out) const {
    constexpr int E = V16<T>::E;
    V16<T> y;
#pragma unroll
    for (int e = 0; e < E / 2; ++e) {
      const F<2> logp = x.pair(e) + F<2>::all(-lse);
      const F<2> pr = each(logp * F<2>::all(kLog2e), [](float v, int) { return ex2(v); });
      const F<2> g = fma_(logp, F<2>::all(-ge), F<2>::all(-c0)) * pr;
      y.set_pair(e, each(g, [&](float v, int k) { return pr.x[k] == 0.f ? 0.f : v; }));
    }
    if (dead) y.w = make_uint4(0u, 0u, 0u, 0u);
    if ((unsigned)(tok - v) < (unsigned)E) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (v + e == tok) y.set(e, one(x.get(e), tok));
    }
    if ((((uintptr_t)row ^ (uintptr_t)out) & 15u) == 0) {
      __stcs(reinterpret_cast<uint4*>(out + v), y.w);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) out[v + e] = y.raw(e);
    }
  }
};
// Statistics are given, so every element is on its own: a block has a part of a row, all of its loads in flight at once.
template <class T>
__global__ void __launch_bounds__(kRow) logprob_back_kernel(const T* logits, T* dlogits, const LogprobGradArgs a, int parts) {
  constexpr int E = V16<T>::E;
  const int r = blockIdx.x / parts, rank = blockIdx.x - r * parts;
  pdl_wait();
  pdl_trigger();
  const T* row = logits + (i64)r * a.ld;
  T* out = dlogits + (i64)r * a.dld;
  const Part<T> p(row, a.V, parts, rank, threadIdx.x);
  V16<T> x[kBatch];
#pragma unroll
  for (int q = 0; q < kBatch; ++q)
    if ((int)threadIdx.x + q * kRow < p.n) x[q].w = __ldcs(p.first + threadIdx.x + q * kRow);
  const float edge = p.edge >= 0 ? to_f32(row[p.edge]) : 0.f;
  const RowGrad g(a, r);
#pragma unroll
  for (int q = 0; q < kBatch; ++q) {
    const int i = (int)threadIdx.x + q * kRow;
    if (i < p.n) g.vector(x[q], p.v0 + i * E, row, out);
  }
  if (p.edge >= 0) out[p.edge] = from_f32<T>(g.one(edge, p.edge));
}

// the same, a warp to a row
template <class T>
__global__ void __launch_bounds__(kRow) logprob_back_warp_kernel(const T* logits, T* dlogits, const LogprobGradArgs a) {
  constexpr int E = V16<T>::E;
  const int lane = threadIdx.x & 31;
  pdl_wait();
  pdl_trigger();
  const i64 r_ = (i64)blockIdx.x * (kRow / 32) + (threadIdx.x >> 5);
  if (r_ >= a.N) return;
  const int r = (int)r_;
  const T* row = logits + (i64)r * a.ld;
  T* out = dlogits + (i64)r * a.dld;
  const Part<T> p(row, a.V, 1, 0, lane);
  const float edge = p.edge >= 0 ? to_f32(row[p.edge]) : 0.f;
  const RowGrad g(a, r);
  for (int i = lane; i < p.n; i += 32 * kBatch) {
    V16<T> x[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (i + q * 32 < p.n) x[q].w = __ldcs(p.first + i + q * 32);
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (i + q * 32 < p.n) g.vector(x[q], p.v0 + (i + q * 32) * E, row, out);
  }
  if (p.edge >= 0) out[p.edge] = from_f32<T>(g.one(edge, p.edge));
}

// ---- distillation --------------------------------------------------------------------------------------------------------------------

struct DistillArgs {
  int N, V, K; i64 ld, dld; float tau;
  const int32_t* top_id; const float *top_logit, *weight; float *row_loss, *loss;
};
// The student's side of one row: q = 2^((x - m) c) / s with c = log2(e) / tau
struct Student { float m, s; };                // (differences first, then / tau: a logit / tau alone may leave the range, and loses digits)

// f 2^((x - M) c) of the thread's vectors
template <int G, class T> __device__ __forceinline__ void write_scaled(const Part<T>& p, int l, uint4* out, float M, float c, float f) {
  for (int i = l; i < p.n; i += G * kBatch) {
    V16<T> x[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (i + q * G < p.n) x[q].w = __ldcs(p.first + i + q * G);
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      if (i + q * G < p.n) {
        V16<T> y;
#pragma unroll
        for (int e = 0; e < V16<T>::E / 2; ++e)
          y.set_pair(e, each((x[q].pair(e) + F<2>::all(-M)) * F<2>::all(c), [](float v, int) { return ex2(v); }) * F<2>::all(f));
        __stcs(out + i + q * G, y.w);
      }
    }
  }
}

// Two passes over a row, the second from L2.  The gradient of the whole row is scale q; the places of the teacher's alternatives are written
// once more, by the first of those that name the same token, after the block has written the rest.
template <class T>
__global__ void __launch_bounds__(kRow, kBlocks) distill_kernel(const T* logits, T* dlogits, const DistillArgs a, int cluster) {
  constexpr int E = V16<T>::E, NW = kRow / 32;
  extern __shared__ float teacher[];           // [K] logit, then probability; [K] the student's logit; [K] token
  float *prob = teacher, *gap = prob + a.K;
  int* id = reinterpret_cast<int*>(gap + a.K);
  __shared__ float wm[NW], wy[NW], wany[NW], wsum[NW], wmass[NW], wloss[NW];
  __shared__ Student part;
  const int r = blockIdx.x / cluster, rank = blockIdx.x - r * cluster, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  pdl_trigger();
  const T* row = logits + (i64)r * a.ld;
  T* out = dlogits + (i64)r * a.dld;
  const Part<T> p(row, a.V, cluster, rank, threadIdx.x);
  const float inv = 1.0f / a.tau, c = kLog2e * inv;
  const float edge = p.edge >= 0 ? to_f32(row[p.edge]) : -INFINITY;
  const float weight = a.weight ? a.weight[r] : 1.0f / (float)a.N;
  const bool teaches = warp * 32 < a.K;        // (the other warps have no alternatives)
  for (int k = threadIdx.x; k < a.K; k += kRow) {
    const int v = a.top_id[(i64)r * a.K + k];
    const bool in = v >= 0 && v < a.V;
    id[k] = in ? v : -1;
    prob[k] = in ? a.top_logit[(i64)r * a.K + k] : -INFINITY;
  }
  Seen t;
  Best unused;
  see_vectors<kRow, false, false>(p, threadIdx.x, c, t, unused);
  if (p.edge >= 0) see_edge<false, T>(t, edge, c);
  float ym = -INFINITY;
  bool any = false;
  for (int k = threadIdx.x; k < a.K; k += kRow) {
    gap[k] = id[k] >= 0 ? to_f32(row[id[k]]) : -INFINITY;
    ym = fmaxf(ym, prob[k]);                   // (a NaN shows in the sum)
    any = any || prob[k] != -INFINITY;
  }
  float m = warp_max(t.m);
  ym = warp_max(ym);
  any = __any_sync(0xffffffffu, any);
  if (lane == 0) { wm[warp] = m; wy[warp] = ym; wany[warp] = any ? 1.f : 0.f; }
  __syncthreads();
  m = all_max<NW>(wm);
  ym = all_max<NW>(wy);
  const float present = all_max<NW>(wany);
  const float m0 = ref_of(m), y0 = ref_of(ym);
  float s = warp_sum((t.s.x[0] + t.s.x[1]) * ex2((t.r - m0) * c)), mass = 0.f;
  if (teaches) {
    for (int k = threadIdx.x; k < a.K; k += kRow) mass += ex2((prob[k] - y0) * c);
    mass = warp_sum(mass);
  }
  if (lane == 0) { wsum[warp] = s; wmass[warp] = mass; }
  __syncthreads();
  s = all_sum<NW>(wsum);
  if (m == -INFINITY) s = 0.f;
  if (m != m || m == INFINITY) s = __int_as_float(0x7fc00000);
  float M = m0;
  if (cluster > 1) {
    cg::cluster_group blocks = cg::this_cluster();
    if (threadIdx.x == 0) part = Student{m, s};
    blocks.sync();                             // (also: every block has read what it needs before the first gradient is written)
    const Student b = lane < cluster ? *blocks.map_shared_rank(&part, lane) : Student{-INFINITY, 0.f};
    M = ref_of(warp_max(b.m));
    s = warp_sum(b.s == 0.f ? 0.f : b.s * ex2((b.m - M) * c));
    blocks.barrier_arrive();                   // (waited for at the end: nobody leaves while its shared memory may be read)
  }
  const float gain = weight * a.tau;
  float loss = 0.f;
  if (teaches) {
    const float ls = logf(s), lmass = logf(all_sum<NW>(wmass));
    for (int k = threadIdx.x; k < a.K; k += kRow) {
      const float logp = (prob[k] - y0) * inv - lmass, pr = ex2(logp * kLog2e), z = gap[k];
      const float logq = z == -INFINITY ? -INFINITY : (z - M) * inv - ls;
      loss += pr == 0.f ? 0.f : pr * (logp - logq);
      prob[k] = pr;
    }
    loss = warp_sum(loss);
  }
  if (lane == 0) wloss[warp] = loss;
  const bool none = present == 0.f || weight == 0.f;
  const float f = s == 0.f ? 0.f : gain / s;
  const auto one = [&](float v) { return none ? 0.f : ex2((v - M) * c) * f; };
  const bool same = (((uintptr_t)row ^ (uintptr_t)out) & 15u) == 0;
  if (same && !none) {
    write_scaled<kRow>(p, threadIdx.x, reinterpret_cast<uint4*>(out + p.v0), M, c, f);
  } else {                                     // a row of zeros, or rows that start at different places of a vector
    for (int i = threadIdx.x; i < p.n; i += kRow) {
      V16<T> x;
      x.w = __ldcs(p.first + i);
#pragma unroll
      for (int e = 0; e < E; ++e) out[p.v0 + i * E + e] = from_f32<T>(one(x.get(e)));
    }
  }
  if (p.edge >= 0) out[p.edge] = from_f32<T>(one(edge));
  __syncthreads();
  if (rank == 0 && warp == NW - 1) {
    loss = all_sum<NW>(wloss);
    if (lane == 0) a.row_loss[r] = present != 0.f ? a.tau * (a.tau * loss) : 0.f;
  }
  if (!none && teaches) {
    const int begin = p.v0, stop = p.v0 + (int)p.n * E;      // the block's whole vectors
    for (int k0 = warp * 32; k0 < a.K; k0 += kRow) {
      const int k = k0 + lane, v = k < a.K ? id[k] : -1;
      float pr = k < a.K ? prob[k] : 0.f;
      bool first = true;
      const int namesakes = __popc(__match_any_sync(0xffffffffu, v));      // (every lane takes part)
      if (a.K > 32 || __any_sync(0xffffffffu, v >= 0 && namesakes > 1)) {
        // the same token may be named twice: its first place adds all of them up, in their order
        pr = 0.f;
#pragma unroll 4
        for (int j = 0; j < a.K; ++j) {
          const bool twin = id[j] == v;
          first = first && !(twin && j < k);
          pr += twin ? prob[j] : 0.f;
        }
      }
      const bool own = (v >= begin && v < stop) || (v >= 0 && rank == 0 && v < begin) || (rank == cluster - 1 && v >= stop);
      if (v >= 0 && own && first) {
        const float q = s == 0.f ? 0.f : ex2((gap[k] - M) * c) / s;
        out[v] = from_f32<T>(gain * (q - pr));
      }
    }
  }
  if (cluster > 1) cg::this_cluster().barrier_wait();
}

// The same, a warp to a row.  The alternatives of each row lie in shared memory (K <= kWarpTeacher).
constexpr int kWarpTeacher = 128;
template <class T>
__global__ void __launch_bounds__(kWarpRows * 32, kBlocks) distill_warp_kernel(const T* logits, T* dlogits, const DistillArgs a) {
  constexpr int E = V16<T>::E;
  extern __shared__ float teacher[];           // for each row: [K] probability, [K] the student's logit, [K] token
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float *prob = teacher + warp * 3 * a.K, *gap = prob + a.K;
  int* id = reinterpret_cast<int*>(gap + a.K);
  pdl_wait();
  pdl_trigger();
  const i64 r_ = (i64)blockIdx.x * kWarpRows + warp;
  if (r_ >= a.N) return;                       // (whole warps: nothing below waits for another)
  const int r = (int)r_;
  const T* row = logits + (i64)r * a.ld;
  T* out = dlogits + (i64)r * a.dld;
  const Part<T> p(row, a.V, 1, 0, lane);
  const float inv = 1.0f / a.tau, c = kLog2e * inv;
  const float edge = p.edge >= 0 ? to_f32(row[p.edge]) : -INFINITY;
  const float weight = a.weight ? a.weight[r] : 1.0f / (float)a.N;
  float ym = -INFINITY;
  bool any = false;
  for (int k = lane; k < a.K; k += 32) {
    const int v = a.top_id[(i64)r * a.K + k];
    const bool in = v >= 0 && v < a.V;
    const float y = in ? a.top_logit[(i64)r * a.K + k] : -INFINITY;
    id[k] = in ? v : -1;
    prob[k] = y;
    gap[k] = in ? to_f32(row[v]) : -INFINITY;
    ym = fmaxf(ym, y);                         // (a NaN shows in the sum)
    any = any || y != -INFINITY;
  }
  Seen t;
  Best unused;
  see_vectors<32, false, false>(p, lane, c, t, unused);
  if (p.edge >= 0) see_edge<false, T>(t, edge, c);
  const float m = warp_max(t.m), M = ref_of(m);
  float s = warp_sum((t.s.x[0] + t.s.x[1]) * ex2((t.r - M) * c)), mass = 0.f;
  if (m == -INFINITY) s = 0.f;
  if (m != m || m == INFINITY) s = __int_as_float(0x7fc00000);
  ym = warp_max(ym);
  any = __any_sync(0xffffffffu, any);
  const float y0 = ref_of(ym);
  for (int k = lane; k < a.K; k += 32) mass += ex2((prob[k] - y0) * c);
  mass = warp_sum(mass);
  const float ls = logf(s), lmass = logf(mass), gain = weight * a.tau;
  float loss = 0.f;
  for (int k = lane; k < a.K; k += 32) {
    const float logp = (prob[k] - y0) * inv - lmass, pr = ex2(logp * kLog2e), z = gap[k];
    const float logq = z == -INFINITY ? -INFINITY : (z - M) * inv - ls;
    loss += pr == 0.f ? 0.f : pr * (logp - logq);
    prob[k] = pr;
  }
  loss = warp_sum(loss);
  if (lane == 0) a.row_loss[r] = any ? a.tau * (a.tau * loss) : 0.f;
  const bool none = !any || weight == 0.f;
  const float f = s == 0.f ? 0.f : gain / s;
  const auto one = [&](float v) { return none ? 0.f : ex2((v - M) * c) * f; };
  if ((((uintptr_t)row ^ (uintptr_t)out) & 15u) == 0 && !none) {
    write_scaled<32>(p, lane, reinterpret_cast<uint4*>(out + p.v0), M, c, f);
  } else {
    for (int i = lane; i < p.n; i += 32) {
      V16<T> x;
      x.w = __ldcs(p.first + i);
#pragma unroll
      for (int e = 0; e < E; ++e) out[p.v0 + i * E + e] = from_f32<T>(one(x.get(e)));
    }
  }
  if (p.edge >= 0) out[p.edge] = from_f32<T>(one(edge));
  __syncwarp();                                // the places of the alternatives are written once more
  for (int k = lane; k < a.K && !none; k += 32) {
    const int v = id[k];
    if (v < 0) continue;
    float pr = 0.f;
    bool first = true;
#pragma unroll 4
    for (int j = 0; j < a.K; ++j) {
      const bool twin = id[j] == v;
      first = first && !(twin && j < k);
      pr += twin ? prob[j] : 0.f;
    }
    if (first) out[v] = from_f32<T>(gain * ((s == 0.f ? 0.f : ex2((gap[k] - M) * c) / s) - pr));
  }
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
    return v >= 0 && v < a.V ? ys[k] : -INFINITY;
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
  for (int k = l; k < a.K; k += G) mass += ex2((teacher(k) - y0) * c);
  mass = group_sum<G>(mass);
  const float ls = logf(s), lmass = logf(mass);
  float loss = 0.f;
  __syncwarp();
  for (int k0 = 0; k0 < a.K; k0 += G) {
    const int k = k0 + l, v = k < a.K ? ids[k] : -1;
    const bool in = v >= 0 && v < a.V;
    float p = 0.f;
    if (in) {
      const float logp = (ys[k] - y0) * inv - lmass, z = to_f32(row[v]);
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
  loss = any != 0.f ? a.tau * (a.tau * loss) : 0.f;
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

// Blocks that share a row: more than one where rows alone leave SMs without work, down to 8 KB each, and for a row that is read twice, one for
// each 128 KB of it.  (The second reading comes from L2 in whole for 4096 rows of 64 KB, 48 MB of them in work in 740 blocks; for 1000 rows of
// 512 KB on clusters of four, 95 MB in work, a third of it comes from DRAM again.)
int blocks_of(int N, i64 bytes, bool twice) {
  int c = 1;
  while (twice && c < kMaxCluster && bytes > c * (i64)131072) c *= 2;
  while (c < kMaxCluster && (i64)N * c < 296 && bytes >= 2 * c * (i64)8192) c *= 2;
  return c;
}
// A warp to a row, of up to `most` bytes, where there are rows for eight warps on every one of 148 multiprocessors; or the row is so short that a block
// finds less than half a vector for each of its threads.  (us, a warp : a block to a row.  32768 rows of 4001 logits of 16 bits: 73 : 273
// with the best five, gradient 91 : 109, distillation 111 : 276.  16384 rows of 8000: 65 : 160, 92 : 79, 115 : 164.  8192 rows of 8000 of 32
// bits: 60 : 88, 92 : 79, 141 : 116.  600 rows of 8000 of 16 bits: 12 : 10, 13 : 6, 14 : 10.)
bool warp_rows(int N, i64 bytes, i64 most) { return bytes <= 2048 || (bytes <= most && N >= 8 * 148 * (bytes > 16384 ? 2 : 1)); }

template <class... KArgs, class... Args>
cudaError_t launch_rows(void (*kern)(KArgs...), int N, int cluster, size_t smem, cudaStream_t s, Args&&... args) {
  if (cluster > 8) {                           // more than the portable size
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl_cluster(kern, cluster, dim3((unsigned)N * (unsigned)cluster), dim3(kRow), smem, s, static_cast<Args&&>(args)..., cluster);
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
  if (top > kMaxTop || N > INT32_MAX / kMaxCluster) return MGRIT_UNSUPPORTED;
  if (N == 0) return MGRIT_OK;
  cudaError_t e = cudaSuccess;
  const LogprobArgs a{N, V, top, ld, tokens, logprob, entropy, lse, top_logprob, top_id};
  with_elem(dtype, [&](auto tag) {
    using T = decltype(tag);
    const T* x = static_cast<const T*>(logits);
    cudaStream_t s = (cudaStream_t)stream;
    const int c = blocks_of(N, (i64)V * (i64)sizeof(T), false);
    const auto few = [&](auto kern, int lanes) { e = launch_pdl(kern, dim3((unsigned)(((i64)N * lanes + kShortThreads - 1) / kShortThreads)), dim3(kShortThreads), 0, s, x, a); };
    const auto warps = [&](auto kern) { e = launch_pdl(kern, dim3((unsigned)(((i64)N + kWarpRows - 1) / kWarpRows)), dim3(kWarpRows * 32), 0, s, x, a); };
    if (V <= kShortRow) few(logprob_short_kernel<T, 8, 8>, 8);
    else if (top <= kWarpTop && warp_rows(N, (i64)V * (i64)sizeof(T), 32768)) { if (top > 0) warps(logprob_warp_kernel<T, true>); else warps(logprob_warp_kernel<T, false>); }
    else if (top > 0) e = launch_rows(logprob_kernel<T, true>, N, c, 0, s, x, a);
    else e = launch_rows(logprob_kernel<T, false>, N, c, 0, s, x, a);
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
  const i64 parts = ((i64)V * (i64)elem_size(dtype) / 16 + kRow * kBatch - 1) / (kRow * kBatch) + (V * (i64)elem_size(dtype) < 16);
  if (N * parts >= INT32_MAX) return MGRIT_UNSUPPORTED;
  cudaError_t e = cudaSuccess;
  const LogprobGradArgs a{N, V, ld, dld, tokens, lse, entropy, dlogprob, dentropy};
  with_elem(dtype, [&](auto tag) {
    using T = decltype(tag);
    if (warp_rows(N, (i64)V * (i64)sizeof(T), 8192))
      e = launch_pdl(logprob_back_warp_kernel<T>, dim3((unsigned)(((i64)N + kRow / 32 - 1) / (kRow / 32))), dim3(kRow), 0, (cudaStream_t)stream, static_cast<const T*>(logits),
                     static_cast<T*>(dlogits), a);
    else
      e = launch_pdl(logprob_back_kernel<T>, dim3((unsigned)(N * parts)), dim3(kRow), 0, (cudaStream_t)stream, static_cast<const T*>(logits), static_cast<T*>(dlogits), a,
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
  if (K < 1 || !(tau > 0.f) || tau > 3.0e38f || kLog2e / tau > 3.4e38f || !loss || !aligned4(loss)) return MGRIT_INVALID_ARG;
  if (K > kMaxTeacher || N > INT32_MAX / kMaxCluster) return MGRIT_UNSUPPORTED;
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
      const int c = blocks_of(N, (i64)V * (i64)sizeof(T), true);
      const auto few = [&](auto kern, int lanes) {
        const i64 blocks = ((i64)N * lanes + kShortThreads - 1) / kShortThreads;
        added = blocks == 1;
        e = launch_pdl(kern, dim3((unsigned)blocks), dim3(kShortThreads), 0, s, x, d, a);
      };
      if (V <= kShortRow) few(distill_short_kernel<T, 8, 8>, 8);
      else if (K <= kWarpTeacher && warp_rows(N, (i64)V * (i64)sizeof(T), 16384))
        e = launch_pdl(distill_warp_kernel<T>, dim3((unsigned)(((i64)N + kWarpRows - 1) / kWarpRows)), dim3(kWarpRows * 32), (size_t)kWarpRows * K * 12, s, x, d, a);
      else e = launch_rows(distill_kernel<T>, N, c, (size_t)K * 12, s, x, d, a);
    });
    rc = launched(e);
    if (rc != MGRIT_OK || added) return rc;
  }
  return launched(launch_pdl(distill_loss_kernel, dim3(1), dim3(1024), 0, s, N, (const float*)row_loss, weight, loss));
}

}  // extern "C"
