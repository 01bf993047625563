// Gated linear recurrence h_t = a_t h_{t-1} + b_t, forward and backward.
//
// Every column (b, unit) is a recurrence of its own, so a column is a chain of T dependent multiply-adds over data that is read once:
// bound by HBM as long as enough of the time axis is in flight at once.  Two kernels:
//
//  * scan_short_kernel, T <= kShort: a thread walks its columns.  One step of generation is this kernel: a launch and a trip to memory.
//  * scan_tile_kernel: the time axis is cut into tiles of kSteps x kWarps steps and 32 x VC columns.  A thread holds kSteps steps of VC
//    columns in registers from the only time they are read to the time the results are written.  It reduces them to one pair
//    (A, B): h_out = A h_in + B; the pairs of a tile's warps meet in shared memory, those of the tiles in the workspace.  A tile
//    publishes its pair as soon as it has it; the state in front of a tile is the last published state before it, carried
//    through the pairs of the tiles in between (decoupled look-back), and is published in turn.  Tiles are handed out by a counter,
//    earlier times first, so whatever a tile waits for has been started before it, and the wait ends; it is bounded all the same.
//    The state is carried through the pairs one after the other, by the operation that the tiles themselves would have used, so that the
//    bits do not depend on how far a tile had to look back.
//
// Backward is the same scan from the last step to the first: mu_t = a_t (seed_t + mu_{t+1}).
#include "elem.cuh"

namespace mg {
namespace {

__device__ int g_scan_status = 0;              // 1: a look-back's wait ran out
int* g_scan_status_ptrs[kMaxDevices] = {nullptr};

struct ScanRows { char* p; i64 ts, bs; };      // strides in elements
struct ScanArgs {
  int T, B, H;
  float dt;
  ScanRows gate, cand, h, seed, dgate, dcand, reset;
  const float* h0; const int32_t* lengths; float* hT;
  const float* dhT; float* dh0;
  // tiles: nk along time, nc along the columns
  int nk, nc;
  unsigned* ticket; int* flags; float2* pairs; float* states; int* status;
};

constexpr int kShort = 8;                      // steps that one thread walks
constexpr int kShortThreads = 128;
constexpr int kSteps = 8, kWarps = 8, kTileSteps = kSteps * kWarps;
constexpr int kLook = 4;                       // flags that a lane looks at: 128 tiles back
constexpr uint64_t kWaitNs = 2000000000ull;    // bound of a look-back's wait
constexpr float kMaxDt = 1e18f;

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float rcp(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float rcp_exact(float x) { const float y = rcp(x); return fmaf(fmaf(-x, y, 1.0f), y, y); }      // one Newton step
__device__ __forceinline__ float min_nan(float a, float b) { float y; asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b)); return y; }

// a, b and, for the derivatives, z, 1 - z, n and r (implicit: 1 / (1 + dt z), classic: 1) of one element.
// With E = e^-g and F = e^2c:  z = 1 / (1 + E), n = (F - 1) / (F + 1), 1 / (1 + dt z) = (1 + E) / (1 + E + dt); 1 - z = E z and
// 1 - dt z = ((1 - dt) + E) z lose nothing where z is near 1.  Small candidates take the first terms of the tangent's series, since F - 1
// would lose their digits (|c| < 0.1: the term left out is 5e-8 of the value).  E stops at e^40 (z = 4e-18) and F at e^20 (n = 1).
// 16-bit types: both quotients from one reciprocal, since four of these operations an element take as long as its bytes (16 a cycle
// and SM: 67 M elements in 65 us, the bytes in 61); what that costs is two roundings of fp32.
struct Coef { float a, b, z, omz, n, r; };
template <int CELL, bool FAST> __device__ __forceinline__ Coef coefficients(float g, float c, float dt) {
  Coef o;
  if (CELL == MGRIT_SCAN_COEFFICIENTS) { o.a = g; o.b = c; o.z = o.omz = o.n = o.r = 0.f; return o; }
  const float E = ex2(min_nan(-g, 40.0f) * 1.44269504f), F = ex2(min_nan(c, 10.0f) * 2.88539008f);
  const float P = CELL == MGRIT_CELL_CLASSIC ? 1.0f + E : (1.0f + E) + dt, Q = 1.0f + F;
  float ip, iq;
  if (FAST) {
    const float R = rcp(P * Q);
    ip = Q * R;
    iq = P * R;
  } else {
    ip = rcp_exact(P);
    iq = rcp_exact(Q);
  }
  const float c2 = c * c;
  o.n = fabsf(c) < 0.1f ? c * fmaf(c2, fmaf(c2, 0.13333334f, -0.33333334f), 1.0f) : (F - 1.0f) * iq;
  if (CELL == MGRIT_CELL_CLASSIC) {
    o.z = ip;
    o.omz = E * ip;
    o.r = 1.0f;
    o.a = ((1.0f - dt) + E) * ip;
    o.b = dt * ip * o.n;
  } else {
    o.r = o.a = (1.0f + E) * ip;
    o.b = dt * ip * o.n;                       // dt z r = dt / (1 + E + dt)
    o.z = FAST ? rcp(1.0f + E) : rcp_exact(1.0f + E);
    o.omz = E * o.z;
  }
  return o;
}

// d(gate), d(cand) of a step whose state has the derivative 1
template <int CELL> __device__ __forceinline__ void slopes(const Coef& k, float hp, float dt, float& wg, float& wc) {
  if (CELL == MGRIT_SCAN_COEFFICIENTS) { wg = hp; wc = 1.0f; return; }
  const float s = dt * k.z * k.r;
  wg = s * k.r * (k.n - hp) * k.omz;
  wc = s * (1.0f - k.n) * (1.0f + k.n);
}

// VC consecutive elements of a row
template <class T, int VC> struct Vec;
template <class T> struct Vec<T, 1> { T x; __device__ __forceinline__ float get(int) const { return to_f32(x); } __device__ __forceinline__ void set(int, float v) { x = from_f32<T>(v); } };
template <> struct alignas(8) Vec<float, 2> { float x, y; __device__ __forceinline__ float get(int i) const { return i ? y : x; } __device__ __forceinline__ void set(int i, float v) { (i ? y : x) = v; } };
template <> struct alignas(4) Vec<__nv_bfloat16, 2> {
  __nv_bfloat162 v;
  __device__ __forceinline__ float get(int i) const { return i ? __high2float(v) : __low2float(v); }
  __device__ __forceinline__ void set(int i, float f) { (i ? v.y : v.x) = __float2bfloat16_rn(f); }
};
template <> struct alignas(4) Vec<__half, 2> {
  __half2 v;
  __device__ __forceinline__ float get(int i) const { return i ? __high2float(v) : __low2float(v); }
  __device__ __forceinline__ void set(int i, float f) { (i ? v.y : v.x) = __float2half_rn(f); }
};
template <class T, int VC> __device__ __forceinline__ Vec<T, VC> load(const T* p) { return *reinterpret_cast<const Vec<T, VC>*>(p); }
template <class T, int VC> __device__ __forceinline__ void store(T* p, const Vec<T, VC>& v) { *reinterpret_cast<Vec<T, VC>*>(p) = v; }
template <class T, int VC> __device__ __forceinline__ Vec<T, VC> zeros() {
  Vec<T, VC> v;
#pragma unroll
  for (int i = 0; i < VC; ++i) v.set(i, 0.f);
  return v;
}

// What a thread knows of its columns: first column, sequence, addresses of step 0
template <class T> struct Column {
  i64 col; int b, u, len;
  bool live;
  __device__ __forceinline__ Column(const ScanArgs& a, i64 c) : col(c) {
    live = c < (i64)a.B * a.H;
    b = live ? (int)(c / a.H) : 0;
    u = live ? (int)(c - (i64)b * a.H) : 0;
    len = !live ? 0 : a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  }
  __device__ __forceinline__ T* at(const ScanRows& r, int t) const { return reinterpret_cast<T*>(r.p) + (i64)t * r.ts + (i64)b * r.bs + u; }
  __device__ __forceinline__ bool fresh(const ScanArgs& a, int t) const {
    return a.reset.p && reinterpret_cast<const uint8_t*>(a.reset.p)[(i64)t * a.reset.ts + (i64)b * a.reset.bs] != 0;
  }
};

template <class T, int CELL, int VC, bool BACK>
__global__ void __launch_bounds__(kShortThreads) scan_short_kernel(const ScanArgs a) {
  constexpr bool FAST = sizeof(T) == 2;
  const Column<T> q(a, ((i64)blockIdx.x * kShortThreads + threadIdx.x) * VC);
  if (!q.live) return;
  const float* first = BACK ? a.dhT : a.h0;
  float h[VC];
#pragma unroll
  for (int v = 0; v < VC; ++v) h[v] = first ? first[q.col + v] : 0.f;
  for (int i = 0; i < a.T; ++i) {
    const int t = BACK ? a.T - 1 - i : i;
    if (t >= q.len) {
      if (BACK) {
        store<T, VC>(q.at(a.dgate, t), zeros<T, VC>());
        store<T, VC>(q.at(a.dcand, t), zeros<T, VC>());
      } else {
        store<T, VC>(q.at(a.h, t), zeros<T, VC>());
      }
      continue;
    }
    const bool fresh = q.fresh(a, t);
    const Vec<T, VC> g = load<T, VC>(q.at(a.gate, t)), c = load<T, VC>(q.at(a.cand, t));
    if (BACK) {
      Vec<T, VC> hv = zeros<T, VC>(), sd = zeros<T, VC>(), dg, dc;
      if (t > 0 && !fresh) hv = load<T, VC>(q.at(a.h, t - 1));
      if (a.seed.p) sd = load<T, VC>(q.at(a.seed, t));
#pragma unroll
      for (int v = 0; v < VC; ++v) {
        const Coef k = coefficients<CELL, FAST>(g.get(v), c.get(v), a.dt);
        const float hp = t == 0 && !fresh && a.h0 ? a.h0[q.col + v] : hv.get(v), lam = h[v] + sd.get(v);
        float wg, wc;
        slopes<CELL>(k, hp, a.dt, wg, wc);
        dg.set(v, lam * wg);
        dc.set(v, lam * wc);
        h[v] = fresh ? 0.f : k.a * lam;
      }
      store<T, VC>(q.at(a.dgate, t), dg);
      store<T, VC>(q.at(a.dcand, t), dc);
    } else {
      Vec<T, VC> out;
#pragma unroll
      for (int v = 0; v < VC; ++v) {
        const Coef k = coefficients<CELL, FAST>(g.get(v), c.get(v), a.dt);
        h[v] = fresh ? k.b : fmaf(k.a, h[v], k.b);
        out.set(v, h[v]);
      }
      store<T, VC>(q.at(a.h, t), out);
    }
  }
  float* last = BACK ? a.dh0 : a.hT;
  if (last) {
#pragma unroll
    for (int v = 0; v < VC; ++v) last[q.col + v] = h[v];
  }
}

__device__ __forceinline__ int ld_acquire(const int* p) { int v; asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory"); return v; }
__device__ __forceinline__ void st_release(int* p, int v) { asm volatile("st.release.gpu.global.s32 [%0], %1;" :: "l"(p), "r"(v) : "memory"); }
__device__ __forceinline__ uint64_t now_ns() { uint64_t t; asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t)); return t; }

// h through the pair p.  A = 0 cuts what came before off, whatever it was (a reset sets it; 0 x NaN would not be 0).
__device__ __forceinline__ float through(float2 p, float h) { return p.x == 0.f ? p.y : fmaf(p.x, h, p.y); }

// The state in front of tile k of column tile c, for the warp's columns: waits until a state and all pairs after it have been published.
template <int VC> __device__ __forceinline__ void look_back(const ScanArgs& a, int k, int c, int lane, float (&h)[VC]) {
  int from = -1;                               // the tile whose state is taken
  uint64_t t0 = 0;
  for (unsigned round = 0; from < 0; ++round) {
    int last = k - 1;                          // tiles last, last - 1, ... of this look
#pragma unroll 1
    for (int w = 0; w < kLook && last >= 0; ++w, last -= 32) {
      const int f = last - lane >= 0 ? ld_acquire(a.flags + (i64)(last - lane) * a.nc + c) : 0;
      const unsigned state = __ballot_sync(0xffffffffu, f == 2), none = __ballot_sync(0xffffffffu, f == 0);
      const int s = state ? __ffs(state) - 1 : 32, n = none ? __ffs(none) - 1 : 32;
      if (s < n) { from = last - s; break; }
      if (n < 32) break;                       // a tile in between has not published anything yet
    }
    if (from < 0 && (round & 31u) == 31u) {
      int stop = 0;
      if (lane == 0) {
        const uint64_t t = now_ns();
        if (t0 == 0) t0 = t;
        stop = *(volatile int*)a.status != 0;
        if (!stop && t - t0 > kWaitNs) { atomicExch(a.status, 1); stop = 1; }
      }
      if (__shfl_sync(0xffffffffu, stop, 0)) {
#pragma unroll
        for (int v = 0; v < VC; ++v) h[v] = __int_as_float(0x7fc00000);      // the results are void, and look it
        return;
      }
    }
  }
  __syncwarp();                                // what one lane acquired is ordered in front of every lane's loads
  const i64 row = (i64)a.nc * (32 * VC), col = (i64)c * (32 * VC) + lane * VC;
#pragma unroll
  for (int v = 0; v < VC; ++v) h[v] = __ldcg(a.states + from * row + col + v);
  const float2* p = a.pairs + (from + 1) * row + col;
#pragma unroll 4
  for (int j = from + 1; j < k; ++j, p += row) {
#pragma unroll
    for (int v = 0; v < VC; ++v) h[v] = through(__ldcg(p + v), h[v]);
  }
}

template <class T, int CELL, int VC, bool BACK>
__global__ void __launch_bounds__(kWarps * 32) scan_tile_kernel(const ScanArgs a) {
  constexpr bool FAST = sizeof(T) == 2;
  constexpr int S = kSteps, CT = 32 * VC;
  __shared__ float2 pair[kWarps][CT];
  __shared__ float front[CT];
  __shared__ unsigned tile_s;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned tile = blockIdx.x;
  if (a.nk > 1) {
    if (threadIdx.x == 0) tile_s = atomicAdd(a.ticket, 1u);
    __syncthreads();
    tile = tile_s;
  }
  const int k = (int)(tile / (unsigned)a.nc), c = (int)(tile - (unsigned)k * (unsigned)a.nc);
  const Column<T> q(a, (i64)c * CT + lane * VC);
  const int i0 = k * kTileSteps + warp * S;    // the thread's first step, counted from the scan's start
  const auto time_of = [&](int i) { return BACK ? a.T - 1 - i : i; };

  // the thread's steps: read once, kept as coefficients (and what the gradients need)
  float ca[S][VC], cb[S][VC], wg[BACK ? S : 1][VC], wc[BACK ? S : 1][VC];      // cb: b, backward: the seed
  unsigned inside = 0, fresh = 0;
  {
    Vec<T, VC> g[S], n[S], hv[BACK ? S : 1], sd[BACK ? S : 1];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int t = time_of(i0 + s);
      const bool in = t >= 0 && t < q.len;
      g[s] = n[s] = zeros<T, VC>();
      if (BACK) hv[BACK ? s : 0] = sd[BACK ? s : 0] = zeros<T, VC>();
      if (in) {
        inside |= 1u << s;
        g[s] = load<T, VC>(q.at(a.gate, t));
        n[s] = load<T, VC>(q.at(a.cand, t));
        if (BACK) {
          if (t > 0) hv[BACK ? s : 0] = load<T, VC>(q.at(a.h, t - 1));
          if (a.seed.p) sd[BACK ? s : 0] = load<T, VC>(q.at(a.seed, t));
        }
      }
    }
    if (a.reset.p) {
#pragma unroll
      for (int s = 0; s < S; ++s)
        if ((inside >> s & 1u) && q.fresh(a, time_of(i0 + s))) fresh |= 1u << s;
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const bool in = inside >> s & 1u, fr = fresh >> s & 1u;
#pragma unroll
      for (int v = 0; v < VC; ++v) {
        const Coef o = coefficients<CELL, FAST>(g[s].get(v), n[s].get(v), a.dt);
        ca[s][v] = !in ? 1.f : fr ? 0.f : o.a;
        if (BACK) {
          float hp = hv[BACK ? s : 0].get(v);
          if (time_of(i0 + s) == 0) hp = in && a.h0 ? a.h0[q.col + v] : 0.f;
          if (fr) hp = 0.f;
          cb[s][v] = sd[BACK ? s : 0].get(v);
          slopes<CELL>(o, hp, a.dt, wg[BACK ? s : 0][v], wc[BACK ? s : 0][v]);
        } else {
          cb[s][v] = in ? o.b : 0.f;
        }
      }
    }
  }
  // one step of the scan: forward h -> a h + b, backward mu -> a (mu + seed)
  const auto step = [&](int s, int v, float h) {
    if (fresh >> s & 1u) return BACK ? 0.f : cb[s][v];
    return BACK ? ca[s][v] * (h + cb[s][v]) : fmaf(ca[s][v], h, cb[s][v]);
  };
#pragma unroll
  for (int v = 0; v < VC; ++v) {
    float A = 1.f, h = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      A = (fresh >> s & 1u) ? 0.f : ca[s][v] * A;
      h = step(s, v, h);
    }
    pair[warp][lane * VC + v] = make_float2(A, h);
  }
  __syncthreads();

  if (warp == 0) {
    float2 whole[VC];
    float h[VC];
#pragma unroll
    for (int v = 0; v < VC; ++v) {
      whole[v] = pair[0][lane * VC + v];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) {
        const float2 p = pair[w][lane * VC + v];
        whole[v] = make_float2(p.x == 0.f ? 0.f : p.x * whole[v].x, through(p, whole[v].y));
      }
    }
    const bool more = k + 1 < a.nk;
    const i64 at = ((i64)k * a.nc + c) * CT + lane * VC;
    int* flag = a.flags + (i64)k * a.nc + c;
    if (k == 0) {
      const float* first = BACK ? a.dhT : a.h0;
#pragma unroll
      for (int v = 0; v < VC; ++v) h[v] = q.live && first ? first[q.col + v] : 0.f;
    } else {
      if (more) {
#pragma unroll
        for (int v = 0; v < VC; ++v) __stcg(a.pairs + at + v, whole[v]);
        __syncwarp();
        if (lane == 0) { __threadfence(); st_release(flag, 1); }
      }
      look_back<VC>(a, k, c, lane, h);
    }
    if (more) {
#pragma unroll
      for (int v = 0; v < VC; ++v) __stcg(a.states + at + v, through(whole[v], h[v]));
      __syncwarp();
      if (lane == 0) { __threadfence(); st_release(flag, 2); }
    }
#pragma unroll
    for (int v = 0; v < VC; ++v) front[lane * VC + v] = h[v];
  }
  __syncthreads();

  float h[VC];
#pragma unroll
  for (int v = 0; v < VC; ++v) {
    h[v] = front[lane * VC + v];
    for (int w = 0; w < warp; ++w) h[v] = through(pair[w][lane * VC + v], h[v]);
  }
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int t = time_of(i0 + s);
    const bool in = inside >> s & 1u, write = q.live && t >= 0 && t < a.T;
    Vec<T, VC> x = zeros<T, VC>(), y = zeros<T, VC>();
#pragma unroll
    for (int v = 0; v < VC; ++v) {
      if (BACK) {
        const float lam = h[v] + cb[s][v];
        if (in) {
          x.set(v, lam * wg[BACK ? s : 0][v]);
          y.set(v, lam * wc[BACK ? s : 0][v]);
        }
      }
      h[v] = step(s, v, h[v]);
      if (!BACK && in) x.set(v, h[v]);
    }
    if (write) {
      store<T, VC>(q.at(BACK ? a.dgate : a.h, t), x);
      if (BACK) store<T, VC>(q.at(a.dcand, t), y);
    }
  }
  float* last = BACK ? a.dh0 : a.hT;
  if (last && k + 1 == a.nk && warp == kWarps - 1 && q.live) {
#pragma unroll
    for (int v = 0; v < VC; ++v) last[q.col + v] = h[v];
  }
}

// ---- arguments ---------------------------------------------------------------------------------------------------------------

bool scan_sizes_served(int T, int B, int H) { return T >= 0 && B >= 0 && H > 0 && (i64)B * H < ((i64)1 << 31) && T < INT32_MAX - 1024; }
// rows of H elements that never overlap: one of the two strides steps over all that the other one covers
bool rows_apart(const mgrit_rows& r, int T, int B, int H) {
  if (T <= 1 && B <= 1) return true;
  const i64 ts = r.t_stride < 0 ? -r.t_stride : r.t_stride, bs = r.b_stride < 0 ? -r.b_stride : r.b_stride;
  if (T <= 1) return bs >= H;
  if (B <= 1) return ts >= H;
  return (bs >= H && ts / bs >= B - 1 && ts - bs * (B - 1) >= H) || (ts >= H && bs / ts >= T - 1 && bs - ts * (T - 1) >= H);
}

ScanRows rows_of(const mgrit_rows& r) { return ScanRows{static_cast<char*>(r.data), r.t_stride, r.b_stride}; }

int check_scan(const gated_scan_args* x, bool back, ScanArgs& a) {
  if (!x || x->T < 0 || x->B < 0 || x->H <= 0 || x->cell < 0 || x->cell > MGRIT_SCAN_COEFFICIENTS || !elem_known(x->dtype)) return MGRIT_INVALID_ARG;
  if (!(x->dt >= 0.f && x->dt <= kMaxDt)) return MGRIT_INVALID_ARG;
  if (!scan_sizes_served(x->T, x->B, x->H)) return MGRIT_UNSUPPORTED;
  a = ScanArgs{};
  a.T = x->T; a.B = x->B; a.H = x->H; a.dt = x->dt;
  a.h0 = x->h0; a.lengths = x->lengths;
  if (!aligned4(x->h0) || !aligned4(x->lengths)) return MGRIT_INVALID_ARG;
  if (back) {
    a.dhT = x->dhT; a.dh0 = x->dh0;
    if (!aligned4(x->dhT) || !aligned4(x->dh0)) return MGRIT_INVALID_ARG;
  } else {
    a.hT = x->hT;
    if (!aligned4(x->hT)) return MGRIT_INVALID_ARG;
  }
  if (x->T == 0 || x->B == 0) return MGRIT_OK;
  if (!x->gate.data || !x->cand.data || !x->h.data) return MGRIT_INVALID_ARG;
  a.gate = rows_of(x->gate); a.cand = rows_of(x->cand); a.h = rows_of(x->h); a.reset = rows_of(x->reset);
  bool ok = elem_aligned(a.gate.p, x->dtype) && elem_aligned(a.cand.p, x->dtype) && elem_aligned(a.h.p, x->dtype);
  if (back) {
    if (!x->dgate.data || !x->dcand.data || (!x->dh_seed.data && !x->dhT)) return MGRIT_INVALID_ARG;
    a.seed = rows_of(x->dh_seed); a.dgate = rows_of(x->dgate); a.dcand = rows_of(x->dcand);
    ok = ok && elem_aligned(a.seed.p, x->dtype) && elem_aligned(a.dgate.p, x->dtype) && elem_aligned(a.dcand.p, x->dtype) &&
         rows_apart(x->dgate, x->T, x->B, x->H) && rows_apart(x->dcand, x->T, x->B, x->H);
  } else {
    ok = ok && rows_apart(x->h, x->T, x->B, x->H);
  }
  return ok ? MGRIT_OK : MGRIT_INVALID_ARG;
}

// nothing to step over: the last state is the first one (hT may be h0), its derivative likewise
int copy_state(float* dst, const float* src, size_t n, cudaStream_t s) {
  if (!dst || n == 0 || dst == src) return MGRIT_OK;
  const cudaError_t e = src ? cudaMemcpyAsync(dst, src, n * sizeof(float), cudaMemcpyDeviceToDevice, s) : cudaMemsetAsync(dst, 0, n * sizeof(float), s);
  return e == cudaSuccess ? MGRIT_OK : MGRIT_CUDA_ERROR;
}

// Workspace: counter | flags | pairs | states, for the narrower of the column tiles (which has more flags and as many values)
struct ScanSpace { size_t flags, pairs, states, total; };
ScanSpace scan_space(int T, i64 cols) {
  const size_t up = 255, nk = ((size_t)T + kTileSteps - 1) / kTileSteps, padded = ((size_t)cols + 63) / 64 * 64;
  ScanSpace s;
  s.flags = 256;
  s.pairs = (s.flags + nk * (padded / 32) * sizeof(int) + up) & ~up;
  s.states = s.pairs + nk * padded * sizeof(float2);
  s.total = (s.states + nk * padded * sizeof(float) + up) & ~up;
  return s;
}

int* scan_status_ptr() {
  const int dev = current_device_slot();
  if (dev < 0) return nullptr;
  if (!g_scan_status_ptrs[dev]) {
    int* p = nullptr;
    if (cudaGetSymbolAddress((void**)&p, g_scan_status) != cudaSuccess || !p) { cudaGetLastError(); return nullptr; }
    g_scan_status_ptrs[dev] = p;
  }
  return g_scan_status_ptrs[dev];
}

// two columns a thread where rows allow it: H even, all strides even and all addresses on pairs
bool pairs_of_columns(const ScanArgs& a, int dtype) {
  const uintptr_t mask = 2 * elem_size(dtype) - 1;
  const auto fits = [&](const ScanRows& r) { return !r.p || (((uintptr_t)r.p & mask) == 0 && r.ts % 2 == 0 && r.bs % 2 == 0); };
  return a.H % 2 == 0 && fits(a.gate) && fits(a.cand) && fits(a.h) && fits(a.seed) && fits(a.dgate) && fits(a.dcand);
}

template <class T, int CELL, int VC, bool BACK> cudaError_t launch_scan(const ScanArgs& a, cudaStream_t s) {
  const i64 cols = (i64)a.B * a.H;
  if (a.T <= kShort) {
    scan_short_kernel<T, CELL, VC, BACK><<<(unsigned)((cols / VC + kShortThreads - 1) / kShortThreads), kShortThreads, 0, s>>>(a);
  } else {
    scan_tile_kernel<T, CELL, VC, BACK><<<(unsigned)a.nk * (unsigned)a.nc, kWarps * 32, 0, s>>>(a);
  }
  count_launch();
  return cudaGetLastError();
}
template <class T, int CELL> cudaError_t launch_scan(const ScanArgs& a, int vc, bool back, cudaStream_t s) {
  if (vc == 2) return back ? launch_scan<T, CELL, 2, true>(a, s) : launch_scan<T, CELL, 2, false>(a, s);
  return back ? launch_scan<T, CELL, 1, true>(a, s) : launch_scan<T, CELL, 1, false>(a, s);
}

int run_scan(const gated_scan_args* x, bool back, void* ws, size_t ws_bytes, cudaStream_t s) {
  ScanArgs a;
  const int rc = check_scan(x, back, a);
  if (rc != MGRIT_OK) return rc;
  if (a.T == 0 || a.B == 0) return back ? copy_state(a.dh0, a.dhT, (size_t)a.B * a.H, s) : copy_state(a.hT, a.h0, (size_t)a.B * a.H, s);
  const int vc = pairs_of_columns(a, x->dtype) ? 2 : 1;
  const i64 cols = (i64)a.B * a.H, nc = (cols + 32 * vc - 1) / (32 * vc), nk = ((i64)a.T + kTileSteps - 1) / kTileSteps;
  if (nk * nc >= INT32_MAX) return MGRIT_UNSUPPORTED;
  a.nk = (int)nk; a.nc = (int)nc;
  if (nk > 1) {
    const ScanSpace sp = scan_space(a.T, cols);
    if (!ws || ((uintptr_t)ws & 255u)) return MGRIT_INVALID_ARG;
    if (ws_bytes < sp.total) return MGRIT_WORKSPACE_TOO_SMALL;
    char* w = static_cast<char*>(ws);
    a.ticket = reinterpret_cast<unsigned*>(w);
    a.flags = reinterpret_cast<int*>(w + sp.flags);
    a.pairs = reinterpret_cast<float2*>(w + sp.pairs);
    a.states = reinterpret_cast<float*>(w + sp.states);
    a.status = scan_status_ptr();
    if (!a.status || cudaMemsetAsync(ws, 0, sp.flags + (size_t)(nk * nc) * sizeof(int), s) != cudaSuccess) { cudaGetLastError(); return MGRIT_CUDA_ERROR; }
  }
  cudaError_t e = cudaSuccess;
  with_elem(x->dtype, [&](auto tag) {
    using T = decltype(tag);
    e = x->cell == MGRIT_CELL_CLASSIC ? launch_scan<T, MGRIT_CELL_CLASSIC>(a, vc, back, s)
      : x->cell == MGRIT_CELL_IMPLICIT ? launch_scan<T, MGRIT_CELL_IMPLICIT>(a, vc, back, s) : launch_scan<T, MGRIT_SCAN_COEFFICIENTS>(a, vc, back, s);
  });
  return e == cudaSuccess ? MGRIT_OK : MGRIT_CUDA_ERROR;
}

}  // namespace

int scan_device_status() {
  const int dev = current_device_slot();
  if (dev < 0) return -1;
  if (!g_scan_status_ptrs[dev]) return 0;      // no scan over several tiles has run on this device
  int v = 0;
  return cudaMemcpy(&v, g_scan_status_ptrs[dev], sizeof(int), cudaMemcpyDeviceToHost) == cudaSuccess ? v : -1;
}
int scan_clear_device_status() {
  const int dev = current_device_slot();
  if (dev < 0) return -1;
  if (!g_scan_status_ptrs[dev]) return 0;
  return cudaMemset(g_scan_status_ptrs[dev], 0, sizeof(int)) == cudaSuccess ? 0 : -1;
}

}  // namespace mg

extern "C" {

size_t gated_scan_workspace_bytes(int32_t T, int32_t B, int32_t H) {
  if (!mg::scan_sizes_served(T, B, H) || T <= mg::kTileSteps || B == 0) return 0;
  return mg::scan_space(T, (mg::i64)B * H).total;
}

int gated_scan_forward(const gated_scan_args* args, void* ws, size_t ws_bytes, mgrit_stream_t stream) {
  return mg::run_scan(args, false, ws, ws_bytes, (cudaStream_t)stream);
}

int gated_scan_backward(const gated_scan_args* args, void* ws, size_t ws_bytes, mgrit_stream_t stream) {
  return mg::run_scan(args, true, ws, ws_bytes, (cudaStream_t)stream);
}

}  // extern "C"
