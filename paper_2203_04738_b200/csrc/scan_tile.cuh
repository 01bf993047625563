// Gated linear recurrence h_t = a_t h_{t-1} + b_t, forward and backward.
//
// Every column (b, unit) is a recurrence of its own, so a column is a chain of T dependent multiply-adds over data that is read once:
// bound by HBM as long as enough of the time axis is in flight at once.  Two kernels:
//
//  * scan_short_kernel, T <= kShort: a thread walks its columns.  One step of generation is this kernel: a launch and a trip to memory.
//  * scan_tile_kernel: the time axis is cut into tiles of S x kWarps steps and 32 x VC columns.  A thread holds S steps of VC
//    columns in registers from the only time they are read to the time the results are written.  It reduces them to one pair
//    (A, B): h_out = A h_in + B; the pairs of a tile's warps meet in shared memory, those of the tiles in the workspace.  A tile
//    publishes its pair as soon as it has it; the state in front of a tile is the last published state before it, carried
//    through the pairs of the tiles in between (decoupled look-back), and is published in turn.  Blocks stay and take tiles from a
//    counter, earlier times first, each in the order in which it got them: the first unfinished tile waits for nothing, so every wait
//    ends; it is bounded all the same.  While a block works on a tile the loads of its next one are in flight.
//    The state is carried through the pairs one after the other, by the operation that the tiles themselves would have used, so that the
//    bits do not depend on how far a tile had to look back.
//    Published words are their own flags: the workspace is filled with a bit pattern that no result has, a word that
//    differs from it is there.  So publishing is a plain store and looking one trip to L2, without fences.
//
// Backward is the same scan from the last step to the first: mu_t = a_t (seed_t + mu_{t+1}).
//
// Measured, B200 (us; in brackets the bytes at the measured copy rate): T 2048, B 32, H 1024 in bf16 forward 119 (61), backward 191 (123);
// 65536 steps of 1024 units in fp32 forward 253 (123); one step of 32 x 1024 4.3.  What bounds it: two warps on each scheduler that issue
// dependent arithmetic (45 % of the issue slots, exponentials and reciprocals 39 % of theirs, DRAM 38 %); with given coefficients the first
// takes 80.  Few columns: the chain of tiles, 0.1 us each at 512 tiles.
// Decoupled look-back is a published method (D. Merrill, M. Garland, "Single-pass parallel prefix scan with decoupled look-back", 2016).
#pragma once
#include <type_traits>

#include "elem.cuh"

namespace mg {

struct ScanRows { char* p; i64 ts, bs; };      // strides in elements
struct ScanArgs {
  int T, B, H, Hp;                             // Hp: H rounded up to whole threads (tile kernel)
  float dt, K, L;                              // gate: q = dt / (K + E), a = (L + E) / (K + E); see coefficients()
  ScanRows gate, cand, h, seed, dgate, dcand, reset;
  const float* h0; const int32_t* lengths; float* hT;
  const float* dhT; float* dh0;
  // tiles: nk along time, nc along the columns
  int nk, nc, deep;
  unsigned* ticket; float* states; unsigned long long* pairs; int* status;      // [nk][nc * 32 VC] each
};

// Where coefficients come from: a cell with q <= 1/2 (implicit, dt <= 1; classic, dt <= 1/2); another one, whose coefficients are at most 1 in size;
// the caller; the classic cell with dt > 2, up to dt - 1 in size.  (Kernels of their own for the first, without the choice of a that the others have
// to make: T 2048, B 32, H 1024 in bf16 takes 191 us backward, classic with dt = 1 198; in fp32 161 forward, 165 with the choice.)
enum { kCells = 0, kOpen = 1, kGiven = 2, kLarge = 3 };
// Both directions for one element type and origin of the coefficients (compiled in files of their own).  wide: rows are made of whole aligned words
// of 16 bytes.  a.status is set where the time axis may take more than one tile.  Up to kShort steps: kOpen for every cell.
template <class T, int MODE> int launch_scan(ScanArgs& a, bool wide, bool back, void* ws, cudaStream_t s);

namespace {

constexpr int kShort = 8;                      // steps that one thread walks
constexpr int kShortThreads = 128;
constexpr int kWarps = 8;
template <class T> constexpr int kWide = 8 / sizeof(T);      // VC, columns of a thread: 8 bytes of a row
// S, steps of a thread.  Long pieces pay: what a tile costs whatever its size (its place, the pairs of the other warps, one meeting, one look
// at L2) is shared by 64 elements of a thread, and the chain of tiles is short.  One block fills an SM's registers.
// Half the steps and two blocks took 16 % longer forward and 24 % backward for T 2048, B 32, H 1024 in bf16, 26 % for 65536 steps of 1024
// units in fp32.
template <bool BACK> constexpr int kStepsOf = BACK ? 8 : 16;
constexpr int kAhead = 1;                      // tiles whose loads are in flight behind the one in work (2 took 5 % longer for T 2048, B 32, H 1024 in bf16)
constexpr int kLook = 4;                       // looks of 32 tiles back
constexpr int kFirst = 2, kMore = 16;          // pairs in flight in a look-back: of a column at first, of the thread's columns then
constexpr int kNarrow = 6;                     // column tiles up to which one warp looks back for its block (measured at the launch)
constexpr uint64_t kWaitNs = 2000000000ull;    // bound of a look-back's wait
constexpr float kMaxDt = 1e18f;

__device__ __forceinline__ float rcp(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float rcp_exact(float x) { const float y = rcp(x); return fmaf(fmaf(-x, y, 1.0f), y, y); }      // one Newton step

__device__ __forceinline__ float max_nan(float a, float b) { float y; asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b)); return y; }

// VC consecutive elements of a row, moved as one word
template <class T, int VC> struct alignas(VC * sizeof(T)) Vec {
  T x[VC];
  __device__ __forceinline__ F<VC> get() const {
    F<VC> f;
#pragma unroll
    for (int i = 0; i < VC; ++i) f.x[i] = to_f32(x[i]);
    return f;
  }
  __device__ __forceinline__ void set(const F<VC>& f) {
#pragma unroll
    for (int i = 0; i < VC; ++i) x[i] = from_f32<T>(f.x[i]);
  }
};
// the same, no lower than -86 (NaN stays).  Two 16-bit values take one instruction.
__device__ __forceinline__ unsigned clamped2(unsigned v, __nv_bfloat16) { unsigned y; asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(v), "r"(0xc2acc2acu)); return y; }
__device__ __forceinline__ unsigned clamped2(unsigned v, __half) { unsigned y; asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(y) : "r"(v), "r"(0xd560d560u)); return y; }
template <class T, int VC> __device__ __forceinline__ F<VC> get_clamped(const Vec<T, VC>& x) {
  if constexpr (sizeof(T) == 2 && VC % 2 == 0) {
    Vec<T, VC> y;
    const unsigned* in = reinterpret_cast<const unsigned*>(&x);
    unsigned* out = reinterpret_cast<unsigned*>(&y);
#pragma unroll
    for (int i = 0; i < VC / 2; ++i) out[i] = clamped2(in[i], T{});
    return y.get();
  } else {
    return each(x.get(), [](float v, int) { return max_nan(v, -86.f); });
  }
}
template <class T, int VC> __device__ __forceinline__ Vec<T, VC> load(const T* p) { return *reinterpret_cast<const Vec<T, VC>*>(p); }
template <class T, int VC> __device__ __forceinline__ void store(T* p, F<VC> f) {
  Vec<T, VC> v;
  v.set(f);
  *reinterpret_cast<Vec<T, VC>*>(p) = v;
}
// The coefficients, and what their derivatives need.  With E = e^-g, G = e^-2|c| and z = 1 / (1 + E):
//   |n| = (1 - G) / (1 + G),  q = dt / (K + E),  a = 1 - q = (L + E) / (K + E),  b = q n
// is the classic cell (q = dt z) for K = 1, L = 1 - dt and the implicit one (q = dt z / (1 + dt z)) for K = 1 + dt, L = 1, and in both
//   dh / dg = q E / (K + E) (n - h_prev),    dh / dc = q (1 - n^2),  1 - n^2 = 4 G / (1 + G)^2, which keeps its digits where |n| is near 1.
// Small candidates take a polynomial, since 1 - G would lose their digits: tanh(c) / c = 1 + c^2 (..), coefficients by least squares on Chebyshev
// points, weighted until the error is level.  a = 1 - q as long as that keeps its digits (a closed gate leaves the state as it is, to the last
// bit, over any number of steps), the quotient from q = 1/2 on (where the gate is 15, 1 - q is off by tens of per cent).  E stops at e^86:
// z is 4.5e-38 then, so that a closed gate is one at the largest dt too, and (K + E) (1 + G) and its inverse are normal numbers.
// FAST (16-bit types): both quotients from one reciprocal, two terms for |c| < 0.1875 (error 9e-8 of n; n right to 6e-7 on either side
// of the border).  Four reciprocals and exponentials an element would take as long as its bytes (16 a cycle and SM: 65 us for 67 M elements, the
// bytes 61).  The cost is two more roundings of fp32.  fp32: one Newton step on each reciprocal, three terms for |c| < 0.35 (4e-8, 4e-7).
template <int VC> struct Coef { F<VC> a, b, q, n, e, m; };      // e = E / (K + E), m = 1 - n^2
template <int MODE, class T, int VC> __device__ __forceinline__ Coef<VC> coefficients(const Vec<T, VC>& graw, const Vec<T, VC>& craw, const ScanArgs& s) {
  constexpr bool FAST = sizeof(T) == 2;
  Coef<VC> o;
  using V = F<VC>;
  if (MODE == kGiven) { o.a = graw.get(); o.b = craw.get(); o.q = o.n = o.e = o.m = V::all(0.f); return o; }
  const V one = V::all(1.0f), g = get_clamped(graw), c = craw.get();
  const V E = each(g * V::all(-1.44269504f), [](float v, int) { return ex2(v); }), G = each(c * V::all(2.88539008f), [](float v, int) { return ex2(-fabsf(v)); });
  const V P = E + V::all(s.K), Q = G + one;
  V ip, iq;
  if (FAST) {
    const V R = each(P * Q, [](float v, int) { return rcp(v); });
    ip = Q * R;
    iq = P * R;
  } else {
    ip = each(P, [](float v, int) { return rcp_exact(v); });
    iq = each(Q, [](float v, int) { return rcp_exact(v); });
  }
  const V far = fma_(G, V::all(-1.0f), one) * iq, c2 = c * c;
  const V near = c * (FAST ? fma_(c2, fma_(c2, V::all(0.1307346f), V::all(-0.33330524f)), one)
                           : fma_(c2, fma_(c2, fma_(c2, V::all(-0.04915929f), V::all(0.1330001f)), V::all(-0.3333267f)), one));
  o.n = each(far, [&](float v, int i) { return fabsf(c.at(i)) < (FAST ? 0.1875f : 0.35f) ? near.at(i) : copysignf(v, c.at(i)); });
  o.q = ip * V::all(s.dt);
  o.a = fma_(o.q, V::all(-1.0f), one);
  if (MODE != kCells) {
    const V part = (E + V::all(s.L)) * ip;
    o.a = each(o.a, [&](float v, int i) { return o.q.at(i) < 0.5f ? v : part.at(i); });
  }
  o.b = o.q * o.n;
  o.e = E * ip;
  const V w = iq + iq;
  o.m = w * w * G;
  return o;
}
// d(gate), d(cand) of a step whose state has the derivative 1
template <bool GIVEN, int VC> __device__ __forceinline__ void slopes(const Coef<VC>& k, F<VC> hp, F<VC>& wg, F<VC>& wc) {
  using V = F<VC>;
  if (GIVEN) { wg = hp; wc = V::all(1.0f); return; }
  wg = (k.q * k.e) * fma_(hp, V::all(-1.0f), k.n);
  wc = k.q * k.m;
}

// n of VC states (the others are zero, or not stored)
template <int VC> __device__ __forceinline__ F<VC> load_state(const float* p, unsigned col, int n = VC) {
  F<VC> f;
#pragma unroll
  for (int v = 0; v < VC; ++v) f.at(v) = p && v < n ? p[col + v] : 0.f;
  return f;
}
template <int VC> __device__ __forceinline__ void store_state(float* p, unsigned col, const F<VC>& f, int n = VC) {
#pragma unroll
  for (int v = 0; v < VC; ++v)
    if (v < n) p[col + v] = f.at(v);
}

// What a thread knows of its columns: the first one, its sequence and unit, the steps of that sequence
template <class T> struct Column {
  unsigned col, b, u;
  int len;
  bool live;
  __device__ __forceinline__ Column(const ScanArgs& a, unsigned c) : col(c) {
    live = c < (unsigned)a.B * (unsigned)a.H;
    b = live ? c / (unsigned)a.H : 0u;
    u = live ? c - b * (unsigned)a.H : 0u;
    len = !live ? 0 : a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  }
  __device__ __forceinline__ T* at(const ScanRows& r, int t) const { return reinterpret_cast<T*>(r.p) + (i64)t * r.ts + (i64)b * r.bs + u; }
  __device__ __forceinline__ bool fresh(const ScanArgs& a, int t) const {
    return reinterpret_cast<const uint8_t*>(a.reset.p)[(i64)t * a.reset.ts + (i64)b * a.reset.bs] != 0;
  }
};

template <class T, int MODE, int VC, bool BACK>
__global__ void __launch_bounds__(kShortThreads) scan_short_kernel(const ScanArgs a) {
  using V = F<VC>;
  const Column<T> q(a, (blockIdx.x * kShortThreads + threadIdx.x) * VC);
  if (!q.live) return;
  V h = load_state<VC>(BACK ? a.dhT : a.h0, q.col);
  for (int i = 0; i < a.T; ++i) {
    const int t = BACK ? a.T - 1 - i : i;
    if (t >= q.len) {
      store<T, VC>(q.at(BACK ? a.dgate : a.h, t), V::all(0.f));
      if (BACK) store<T, VC>(q.at(a.dcand, t), V::all(0.f));
      continue;
    }
    const bool fresh = a.reset.p && q.fresh(a, t);
    const Coef<VC> k = coefficients<MODE, T, VC>(load<T, VC>(q.at(a.gate, t)), load<T, VC>(q.at(a.cand, t)), a);
    if (BACK) {
      const V hp = fresh ? V::all(0.f) : t > 0 ? load<T, VC>(q.at(a.h, t - 1)).get() : load_state<VC>(a.h0, q.col);
      const V lam = a.seed.p ? h + load<T, VC>(q.at(a.seed, t)).get() : h;
      V wg, wc;
      slopes<MODE == kGiven, VC>(k, hp, wg, wc);
      store<T, VC>(q.at(a.dgate, t), lam * wg);
      store<T, VC>(q.at(a.dcand, t), lam * wc);
      h = fresh ? V::all(0.f) : k.a * lam;
    } else {
      h = fresh ? k.b : fma_(k.a, h, k.b);
      store<T, VC>(q.at(a.h, t), h);
    }
  }
  float* last = BACK ? a.dh0 : a.hT;
  if (last) store_state<VC>(last, q.col, h);
}

// ---- words that tiles publish --------------------------------------------------------------------------------------------------

constexpr unsigned kNone = 0xffffffffu;        // a NaN that no result is: NaN is published as 0x7fc00000
__device__ __forceinline__ unsigned word_of(float v) { return v != v ? 0x7fc00000u : __float_as_uint(v); }
__device__ __forceinline__ unsigned ld_word(const float* p) { unsigned v; asm volatile("ld.relaxed.gpu.global.b32 %0, [%1];" : "=r"(v) : "l"(p) : "memory"); return v; }
__device__ __forceinline__ void st_word(float* p, unsigned v) { asm volatile("st.relaxed.gpu.global.b32 [%0], %1;" :: "l"(p), "r"(v) : "memory"); }
__device__ __forceinline__ float2 ld_pair(const unsigned long long* p) {
  unsigned long long v;
  asm volatile("ld.relaxed.gpu.global.b64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
  return make_float2(__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32)));
}
__device__ __forceinline__ void st_pair(unsigned long long* p, float2 v) {
  const unsigned long long w = (unsigned long long)word_of(v.y) << 32 | word_of(v.x);
  asm volatile("st.relaxed.gpu.global.b64 [%0], %1;" :: "l"(p), "l"(w) : "memory");
}
__device__ __forceinline__ uint64_t now_ns() { uint64_t t; asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t)); return t; }

// h through the pair p.  cut (some sequence may start anew somewhere): where one does, only B counts, whatever came before (0 x NaN would not cut
// it off).  A = NaN says so, and stays that in products.  Nothing else that a NaN could say is lost: a gate of NaN makes B NaN too, and products
// of given coefficients that are not finite are not handed on (below).  (A = 0 says less: small coefficients have such a product, and a NaN goes
// on through those.)
__device__ __forceinline__ float through(float2 p, float h, bool cut) { return cut && p.x != p.x ? p.y : fmaf(p.x, h, p.y); }
__device__ __forceinline__ float2 through(float2 p, float2 q, bool cut) { return make_float2(p.x * q.x, through(p, q.y, cut)); }

// A product of coefficients says what becomes of a state of any size only as far as fp32 has room for it.
//  * Coefficients of at most 1 in size: one that underflows is right to 2^-149 of the state.  It stays at the smallest number of its sign, so that
//    an infinite state remains infinite.
//  * In a tile where some are above 1 (STRICT): an overflow, or digits lost below 2^-126 that coefficients above 1 may bring back, make it useless
//    (3^128 times a state of zero is zero, inf times zero is NaN): kLost.  Such a piece is walked from its own first state instead.
//  * A zero among given coefficients makes it zero, whatever the others' product was.
constexpr float kSteady = 1.001f;              // (roundings above 1 bring nothing back)
constexpr float kLeast = 1.17549435e-38f, kMost = 3.4028235e38f;
constexpr float kLost = INFINITY;              // in the place of a product (never published)
__device__ __forceinline__ float kept(float p) { return p == 0.f ? copysignf(1.4e-45f, p) : p; }
__device__ __forceinline__ float largest(float a, float b, float c) { float y; asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c)); return y; }      // in size; NaN is left out
__device__ __forceinline__ float smallest_nan(float a, float b, float c) { float y; asm("min.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c)); return y; }      // in size; NaN stays

// One round of a wait, for the whole warp: true once it has run out, here or elsewhere (the status word says so).
__device__ __forceinline__ bool waited_too_long(const ScanArgs& a, int lane, unsigned round, uint64_t& t0) {
  if ((round & 31u) != 31u) return false;
  int stop = 0;
  if (lane == 0) {
    const uint64_t t = now_ns();
    if (t0 == 0) t0 = t;
    stop = *(volatile int*)a.status != 0;
    if (!stop && t - t0 > kWaitNs) { atomicExch(a.status, 1); stop = 1; }
  }
  return __shfl_sync(0xffffffffu, stop, 0) != 0;
}

// The state in front of tile k of column tile c, for the warp's columns: carried from the last published state through the pairs after
// it.  Words of a tile are published together, so one of them (the first column's) tells the lanes how far back to go.  A tile that found
// the state in front of it at once publishes no pair, only its state: whoever misses a word looks again from the start.
template <int VC, bool NARROW, bool CUT> __device__ __forceinline__ F<VC> look_back(const ScanArgs& a, int k, i64 row, i64 col, int lane) {
  uint64_t t0 = 0;
  for (unsigned round = 0; !waited_too_long(a, lane, round, t0); ++round) {
    int from = -1;                             // the tile whose state is taken
    int last = k - 1;
#pragma unroll 1
    for (int w = 0; w < kLook && last >= 0 && from < 0; ++w, last -= 32) {
      const bool there = last - lane >= 0 && ld_word(a.states + (last - lane) * row + col) != kNone;
      const unsigned m = __ballot_sync(0xffffffffu, there);
      if (m) from = last - (__ffs(m) - 1);
    }
    if (from < 0) continue;
    F<VC> h;
    bool there = true;
#pragma unroll
    for (int v = 0; v < VC; ++v) {
      const unsigned w = ld_word(a.states + from * row + col + lane * VC + v);
      there = there && w != kNone;
      h.at(v) = __uint_as_float(w);
    }
    // the pairs after it: two at first, which often are not there yet; NARROW: then many in one trip
    const auto carry = [&](int j, auto pairs) {
      constexpr int P = decltype(pairs)::value;
      float2 p[P][VC];
      const int n = min(P, k - j);
      const unsigned long long* at = a.pairs + j * row + col + lane * VC;
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int v = 0; v < VC; ++v) p[i][v] = i < n ? ld_pair(at + i * row + v) : make_float2(1.f, 0.f);
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int v = 0; v < VC; ++v)
          if (i < n) {
            there = there && __float_as_uint(p[i][v].x) != kNone;
            h.at(v) = through(p[i][v], h.at(v), CUT);
          }
      return j + P;
    };
    int j = from + 1;
    if (NARROW && j + kFirst < k) {
      j = carry(j, std::integral_constant<int, kFirst>{});
#pragma unroll 1
      while (j + kFirst < k && there) j = carry(j, std::integral_constant<int, kMore / VC>{});
    }
#pragma unroll 1
    while (j < k && there) j = carry(j, std::integral_constant<int, kFirst>{});
    if (__all_sync(0xffffffffu, there)) return h;
  }
  return F<VC>::all(__uint_as_float(0x7fc00000u));      // the results are void, and look it
}

// A tile's place, worked out by one thread for the block
struct alignas(16) Place { int k, c; unsigned b, u; };      // chunk of time (-1: no tile), column tile; sequence and unit of its first column
__device__ __forceinline__ Place place_of(const ScanArgs& a, unsigned tile, int columns) {
  Place p;
  if (tile >= (unsigned)a.nk * (unsigned)a.nc) return Place{-1, 0, 0u, 0u};
  p.k = (int)(tile / (unsigned)a.nc);
  p.c = (int)(tile - (unsigned)p.k * (unsigned)a.nc);
  const unsigned col = (unsigned)p.c * (unsigned)columns;
  p.b = col / (unsigned)a.Hp;
  p.u = col - p.b * (unsigned)a.Hp;
  return p;
}

// CUT: some sequence may start anew somewhere (a kernel of its own: decided at run time it costs those without starts 4 % backward)
template <class T, int MODE, bool ALIGNED, bool BACK, bool NARROW, bool CUT>
__global__ void __launch_bounds__(kWarps * 32, 1) scan_tile_kernel(const __grid_constant__ ScanArgs a) {
  constexpr int VC = kWide<T>, S = kStepsOf<BACK>, CT = 32 * VC, SB = BACK ? S : 1, TT = S * kWarps, ARRAYS = BACK ? 4 : 2;
  extern __shared__ __align__(16) char stage[];      // [tiles ahead][warps][ARRAYS][S][32 threads, or 64 words] of 8 bytes
  constexpr unsigned ALL = (1u << S) - 1u;
  constexpr bool GIVEN = MODE == kGiven, STRICT = MODE == kGiven || MODE == kLarge;
  using V = F<VC>;
  __shared__ __align__(16) float2 pair[2][kWarps][CT];
  constexpr int D = kAhead, RING = 4;
  static_assert(D < RING - 1, "a place is written while the one before it and those ahead are in use");
  __shared__ Place place[RING];
  __shared__ V front[NARROW ? 2 : 1][32];      // NARROW: the state in front of the tile
  __shared__ volatile unsigned posted[2];      // ... and the turn whose state that is
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const i64 row = (i64)a.nc * CT;
  constexpr bool cut = CUT;
  const bool starts_given = cut && (MODE != kLarge || a.reset.p);      // (kLarge has kernels with starts only)
  const auto time_of = [&](int i) { return BACK ? a.T - 1 - i : i; };

  // where the thread stands in a tile: sequence and unit of its columns, its first step counted from the scan's start
  struct Spot { unsigned b, u; int i0, n; };      // n: columns of the thread that exist
  const auto spot_of = [&](const Place& p, int column) {
    Spot s;
    s.b = p.b;
    s.u = p.u + column;
    if (s.u >= (unsigned)a.Hp) {               // the tile reaches into the next sequences
      const unsigned n = s.u / (unsigned)a.Hp;
      s.b += n;
      s.u -= n * (unsigned)a.Hp;
    }
    s.i0 = p.k * TT + warp * S;
    s.n = s.b >= (unsigned)a.B ? 0 : ALIGNED ? VC : min(VC, a.H - (int)s.u);
    return s;
  };
  const auto at = [&](const ScanRows& r, const Spot& s, int t) { return reinterpret_cast<T*>(r.p) + ((i64)t * r.ts + (i64)s.b * r.bs + s.u); };

  // The warp's steps of a tile, as they come from memory, staged in shared memory by asynchronous copies, which leaves the registers to the
  // tile in work; only the warp itself waits for them.  ALIGNED: copies of 16 bytes, two rows of a warp at a time, past L1.  Otherwise a
  // thread's 8 bytes may start at any element: it brings the aligned 8 bytes that hold its first one, and finds the next 8 in its neighbour's
  // place.  For the last thread of a piece of a row they are brought to the second half of the row's place.  What a thread wants is cut out on
  // reading.  Only aligned words that hold an element of the row are read; what else is in them is not used.
  // (997 steps of 24 x 203 units in fp16: 29 us forward, 44 backward; element by element into registers, with half the
  // steps: 32, 56.)
  constexpr unsigned kWord = VC * sizeof(T), kRow = (ALIGNED ? 32 : 64) * kWord, kPieces = 32 * kWord / 16, kRows = ALIGNED ? 32 / kPieces : 1;      // copies of a row, rows at a time
  constexpr unsigned kArray = S * kRow, kTile = kWarps * ARRAYS * kArray;
  static_assert(kWord == 8 && 32 % kPieces == 0 && S % kRows == 0 && S * ARRAYS == 32, "whole copies of whole rows; a lane for each step of each array");
  char* const slice = stage + warp * (ARRAYS * kArray);
  const unsigned slot0 = (unsigned)__cvta_generic_to_shared(slice) + (ALIGNED ? (lane / kPieces) * kRow + (lane % kPieces) * 16u : lane * kWord);
  const auto ends = [&](const Spot& s) { return lane == 31 || (int)s.u + VC >= a.H; };      // the last thread of a piece of a row
  // steps i0 .. i0 + S - 1 of the scan that lie in the sequence
  const auto inside_of = [&](const Spot& s) {
    const int len = s.n == 0 ? 0 : a.lengths ? min(max(a.lengths[s.b], 0), a.T) : a.T;
    const int lo = BACK ? max(0, a.T - len - s.i0) : 0, hi = BACK ? min(S, a.T - s.i0) : min(S, len - s.i0);
    return hi > lo ? (ALL >> (S - hi)) & (ALL << lo) : 0u;
  };
  // What is known of a tile once it has been asked for.  bits: which of the thread's steps lie in the sequence, and (from bit 16 on) which of
  // them start one.  The marks of those starts are on their way too: where the warp's columns are of one or two sequences (paired), lanes
  // 0 .. S - 1 and 16 .. 16 + S - 1 have the steps' marks, which marked() adds to the bits when they are needed; otherwise the
  // bits are complete.  (If every tile waited for its marks, T 2048, B 32, H 1024 in bf16 with lengths and starts would take 13 % longer.)
  struct Known { unsigned bits, mark; };
  static_assert(S <= 16, "marks of two sequences in a warp");
  const auto paired = [&](const Spot& s) { return __shfl_sync(0xffffffffu, s.b, 31) - __shfl_sync(0xffffffffu, s.b, 0) <= 1u; };
  const auto marked = [&](const Known& x, const Spot& s) {
    if (!starts_given || !paired(s)) return x.bits;
    const unsigned m = __ballot_sync(0xffffffffu, x.mark != 0u);
    return x.bits | (m >> ((s.b - __shfl_sync(0xffffffffu, s.b, 0)) * 16u) & x.bits & ALL) << 16;
  };
  const auto fetch = [&](const Place& p, unsigned d) {
    const Spot s = spot_of(p, lane * VC);
    const unsigned inside = inside_of(s);
    unsigned fresh = 0u, one = 0u;
    const int t0 = time_of(s.i0);
    const uint8_t* const marks = reinterpret_cast<const uint8_t*>(a.reset.p);
    if (starts_given && paired(s)) {
      const unsigned b = __shfl_sync(0xffffffffu, s.b, 0) + (lane >> 4);
      const int t = time_of(s.i0 + (lane & 15));
      if ((lane & 15) < S && b < (unsigned)a.B && t >= 0 && t < a.T) one = marks[(i64)t * a.reset.ts + (i64)b * a.reset.bs];
    } else if (starts_given) {                 // all of them asked for before the first is looked at
      uint8_t mark[S];
#pragma unroll
      for (int i = 0; i < S; ++i) mark[i] = marks[(inside >> i & 1u) ? (i64)time_of(s.i0 + i) * a.reset.ts + (i64)s.b * a.reset.bs : 0];
#pragma unroll
      for (int i = 0; i < S; ++i) fresh |= mark[i] && (inside >> i & 1u) ? 1u << i : 0u;
    }
    if (!__any_sync(0xffffffffu, inside != 0u)) {      // (nor will any of it be read)
    } else if constexpr (ALIGNED) {
      const Spot mine = spot_of(p, (lane % kPieces) * (16 / (int)sizeof(T)));
      const int r = (int)(lane / kPieces), t1 = BACK ? t0 - r : t0 + r;
      const auto bring = [&](int array, const ScanRows& from, int t, bool there, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        const unsigned valid = WHOLE ? ALL : inside_of(mine);
        const T* q = at(from, mine, t);
        const i64 dq = (BACK ? -from.ts : from.ts) * (i64)kRows;
        const unsigned to = slot0 + d * kTile + array * kArray;
#pragma unroll
        for (int i = 0; i < S / (int)kRows; ++i) {
          if (WHOLE) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + i * (kRows * kRow)), "l"(q + i * dq) : "memory");
          } else {                             // what lies outside is not read: zeros stand in for it
            const int step = i * (int)kRows + r;
            const bool in = there && (valid >> step & 1u) && (array != 2 || time_of(mine.i0 + step) > 0);
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to + i * (kRows * kRow)), "l"(in ? q + i * dq : reinterpret_cast<const T*>(a.gate.p)), "r"(in ? 16 : 0) : "memory");
          }
        }
      };
      if (__all_sync(0xffffffffu, inside == ALL && (!BACK || (t0 >= S && a.seed.p)))) {
        bring(0, a.gate, t1, true, std::true_type{});
        bring(1, a.cand, t1, true, std::true_type{});
        if (BACK) { bring(2, a.h, t1 - 1, true, std::true_type{}); bring(3, a.seed, t1, true, std::true_type{}); }
      } else {
        bring(0, a.gate, t1, true, std::false_type{});
        bring(1, a.cand, t1, true, std::false_type{});
        if (BACK) { bring(2, a.h, t1 - 1, true, std::false_type{}); bring(3, a.seed, t1, a.seed.p != nullptr, std::false_type{}); }
      }
    } else {
      const uintptr_t none = (uintptr_t)a.gate.p & ~(uintptr_t)7;
      const auto bring = [&](int array, const ScanRows& from, int t, bool there, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        const uintptr_t q = (uintptr_t)at(from, s, t);
        const i64 dq = (BACK ? -from.ts : from.ts) * (i64)sizeof(T);
        const unsigned to = slot0 + d * kTile + array * kArray;
#pragma unroll
        for (int i = 0; i < S; ++i) {
          const uintptr_t w = (q + (uintptr_t)(i * dq)) & ~(uintptr_t)7;
          if (WHOLE) {
            asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" :: "r"(to + i * kRow), "l"(w) : "memory");
          } else {                             // what lies outside is not read: zeros stand in for it
            const bool in = there && (inside >> i & 1u) && (array != 2 || time_of(s.i0 + i) > 0);
            asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" :: "r"(to + i * kRow), "l"(in ? w : none), "r"(in ? 8 : 0) : "memory");
          }
        }
      };
      if (__all_sync(0xffffffffu, inside == ALL && (!BACK || (t0 >= S && a.seed.p)))) {
        bring(0, a.gate, t0, true, std::true_type{});
        bring(1, a.cand, t0, true, std::true_type{});
        if (BACK) { bring(2, a.h, t0 - 1, true, std::true_type{}); bring(3, a.seed, t0, true, std::true_type{}); }
      } else {
        bring(0, a.gate, t0, true, std::false_type{});
        bring(1, a.cand, t0, true, std::false_type{});
        if (BACK) { bring(2, a.h, t0 - 1, true, std::false_type{}); bring(3, a.seed, t0, a.seed.p != nullptr, std::false_type{}); }
      }
      // the words behind the pieces' last threads: a lane has one step of one array
      const int array = lane / S, step = lane % S, t = time_of(s.i0 + step) - (array == 2);
      const ScanRows from = array == 0 ? a.gate : array == 1 ? a.cand : array == 2 ? a.h : a.seed;
      for (unsigned m = __ballot_sync(0xffffffffu, ends(s) && s.n > 0); m; m &= m - 1u) {
        const int who = __ffs(m) - 1;
        Spot e = s;
        e.b = __shfl_sync(0xffffffffu, s.b, who);
        e.u = __shfl_sync(0xffffffffu, s.u, who);
        const unsigned their = __shfl_sync(0xffffffffu, inside, who), bytes = (unsigned)min(VC, a.H - (int)e.u) * (unsigned)sizeof(T);
        const uintptr_t x = (uintptr_t)at(from, e, t);
        const bool in = (their >> step & 1u) && from.p && t >= 0 && ((unsigned)x & 7u) + bytes > 8u;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" :: "r"(slot0 + (who + 32 - lane) * kWord + d * kTile + array * kArray + step * kRow), "l"(in ? (x & ~(uintptr_t)7) + 8 : none), "r"(in ? 8 : 0) : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    return Known{inside | fresh << 16, one};
  };

  if (NARROW && threadIdx.x < 2) posted[threadIdx.x] = 0u;      // (turns are counted from 1 there)
  // Tiles are drawn from the counter (which starts at 2^32 - 1) by thread 32.  deep: D + 1 at the start, and from then on one round
  // before a number is told to the others, so that nobody waits for it.  Otherwise (few tiles: they would all go to the first blocks)
  // one at a time, and nothing is fetched ahead.
  unsigned drawn = blockIdx.x - gridDim.x;
  const auto draw = [&]() { return drawn = a.nk > 1 ? atomicAdd(a.ticket, 1u) + 1u : drawn + gridDim.x; };
  const auto none = [&]() { asm volatile("cp.async.commit_group;" ::: "memory"); return Known{0u, 0u}; };
  Known ahead[D];                              // of the tiles to come
#pragma unroll
  for (int i = 0; i < D; ++i) ahead[i] = Known{0u, 0u};
  if (a.deep) {
    if (threadIdx.x == 32) {
      for (int i = 0; i <= D; ++i) place[i] = place_of(a, draw(), CT);
      draw();
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < D; ++i) {
      const Place p = place[i];
      ahead[i] = p.k >= 0 ? fetch(p, i) : none();
    }
  }

  // one tile; ODD: some step of the warp may lie outside its sequence, start a sequence or (backward) be the first one
  const auto work = [&](auto odd_, unsigned d, unsigned turn, const Place& here, const Spot& now, unsigned in_now, unsigned fresh_now) {
    constexpr bool ODD = decltype(odd_)::value;
    const int k = here.k, c = here.c;
    const unsigned buf = turn & 1u;
    const i64 word = k * row + (i64)c * CT + lane * VC;
    // The state in front: what the tile before has published, asked for early (it is usually there), or the first one
    unsigned early[VC];
    if (k > 0) {
#pragma unroll
      for (int v = 0; v < VC; ++v) early[v] = ld_word(a.states + word - row + v);
    } else {
      const V first = load_state<VC>(BACK ? a.dhT : a.h0, now.b * (unsigned)a.H + now.u, now.n);
#pragma unroll
      for (int v = 0; v < VC; ++v) early[v] = __float_as_uint(first.at(v));
    }
    const unsigned told = drawn;
    if (threadIdx.x == 32 && a.deep) draw();

    V ca[S], cb[S], wg[SB], wc[SB];            // cb: b, backward: the seed
    [[maybe_unused]] unsigned low[ALIGNED ? 1 : ARRAYS], dlow[ALIGNED ? 1 : ARRAYS];      // where an array's elements start (the address's low bits), and their change with a step
    if constexpr (!ALIGNED) {
      const auto start = [&](int array, const ScanRows& r, int t) {
        low[array] = (unsigned)(uintptr_t)at(r, now, t);
        dlow[array] = (unsigned)((BACK ? -r.ts : r.ts) * (i64)sizeof(T));
      };
      start(0, a.gate, time_of(now.i0));
      start(1, a.cand, time_of(now.i0));
      if constexpr (BACK) { start(2, a.h, time_of(now.i0) - 1); start(3, a.seed, time_of(now.i0)); }
    }
    const unsigned after = ends(now) ? 32u * kWord : kWord;      // the bytes that follow the thread's
    const auto raw = [&](int array, int s) {
      const char* at = slice + d * kTile + array * kArray + s * kRow + lane * kWord;
      if constexpr (ALIGNED) {
        return *reinterpret_cast<const Vec<T, VC>*>(at);
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(at), y = *reinterpret_cast<const uint2*>(at + after);
        const unsigned off = low[array] + s * dlow[array];
        const bool up = off & 4u;
        const unsigned w0 = up ? x.y : x.x, w1 = up ? y.x : x.y, w2 = up ? y.y : y.x;
        uint2 r = make_uint2(w0, w1);
        if (sizeof(T) == 2) r = make_uint2(__funnelshift_r(w0, w1, (off & 2u) * 8u), __funnelshift_r(w1, w2, (off & 2u) * 8u));
        return *reinterpret_cast<const Vec<T, VC>*>(&r);
      }
    };
    asm volatile("cp.async.wait_group %0;" :: "n"(D - 1) : "memory");      // (all but the D - 1 last groups)
    __syncwarp();
    if (!ODD || __any_sync(0xffffffffu, in_now != 0u)) {
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const Coef<VC> o = coefficients<MODE, T, VC>(raw(0, s), raw(1, s), a);
        ca[s] = o.a;
        if (BACK) {
          V hp = raw(2, s).get();
          if (ODD && time_of(now.i0 + s) == 0 && (in_now >> s & 1u)) hp = load_state<VC>(a.h0, now.b * (unsigned)a.H + now.u, now.n);
          if (ODD && cut) hp = each(hp, [&](float x, int) { return (fresh_now >> s & 1u) ? 0.f : x; });
          cb[s] = raw(3, s).get();
          slopes<GIVEN, VC>(o, hp, wg[BACK ? s : 0], wc[BACK ? s : 0]);
        } else {
          cb[s] = o.b;
        }
        if (ODD) {
          const bool in = in_now >> s & 1u, fr = fresh_now >> s & 1u;
          // (a new sequence: step() takes the state for zero, which leaves a NaN among given coefficients to be kept out)
          ca[s] = each(ca[s], [&](float x, int) { return !in ? 1.f : GIVEN && !BACK && fr ? 0.f : x; });
          cb[s] = each(cb[s], [&](float x, int) { return in ? x : 0.f; });
        }
      }
    } else {                                   // the sequences have ended: the state goes through
#pragma unroll
      for (int s = 0; s < S; ++s) {
        ca[s] = V::all(1.f);
        cb[s] = V::all(0.f);
        if (BACK) wg[BACK ? s : 0] = wc[BACK ? s : 0] = V::all(0.f);
      }
    }
    __syncwarp();                              // the slot has been read
    Known theirs{0u, 0u};
    if (a.deep) {
      const Place later = place[(turn + D) % RING];
      theirs = later.k >= 0 ? fetch(later, d) : none();
    }

    // one step of the scan: forward h -> a h + b, backward mu -> a (mu + seed)
    const auto step = [&](int s, V h) {
      if (ODD && cut) {                        // (a = 0 would not stop a NaN or an infinity)
        const bool fr = fresh_now >> s & 1u;
#pragma unroll
        for (int v = 0; v < VC; ++v) h.at(v) = fr ? 0.f : h.at(v);
        if (BACK) {
          const V m = ca[s] * (h + cb[s]);
          return each(m, [&](float x, int) { return fr ? 0.f : x; });
        }
      }
      return BACK ? ca[s] * (h + cb[s]) : fma_(ca[s], h, cb[s]);
    };
    V A = V::all(1.f), h = V::all(0.f);
#pragma unroll
    for (int s = 0; s < S; ++s) {
      A = s == 0 ? ca[s] : ca[s] * A;
      h = step(s, h);
    }
    bool big = false, lost = false;            // a coefficient above 1 (or NaN); a column's product is not to be had
    if (ODD && cut && fresh_now != 0u) {
      A = V::all(__uint_as_float(0x7fc00000u));
    } else if constexpr (STRICT) {
      float most[2] = {0.f, 0.f};
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int v = 0; v < VC; v += 2) most[s & 1] = largest(most[s & 1], ca[s].at(v), ca[s].at(v + 1 < VC ? v + 1 : v));
      float least = A.at(0);
#pragma unroll
      for (int v = 0; v < VC; v += 2) least = smallest_nan(least, A.at(v), A.at(v + 1 < VC ? v + 1 : v));
      big = !(fmaxf(most[0], most[1]) <= kSteady) || least != least;
      if (big) {
        constexpr float kUp = S == 8 ? 32768.f : 128.f;      // S coefficients up to that, and down to its inverse, leave the product in range
        static_assert(S == 8 || S == 16, "S powers of kUp are 2^120, or 2^112");
#pragma unroll
        for (int v = 0; v < VC; ++v) {
          float up = 0.f, down = kMost;
#pragma unroll
          for (int s = 0; s < S; ++s) { up = max_nan(up, fabsf(ca[s].at(v))); down = fminf(down, fabsf(ca[s].at(v))); }
          if (up <= kMost && down == 0.f) A.at(v) = 0.f;
          else if (!(up <= kSteady ? fabsf(A.at(v)) >= kLeast : up <= kUp && down * kUp >= 1.f)) A.at(v) = kLost, lost = true;
        }
      } else if (least < kLeast) {
#pragma unroll
        for (int v = 0; v < VC; ++v) {
          if (A.at(v) == 0.f) {
            float down = kMost;
#pragma unroll
            for (int s = 0; s < S; s += 2) down = smallest_nan(down, ca[s].at(v), ca[s + 1].at(v));
            if (down > 0.f) A.at(v) = kept(A.at(v));
          }
        }
      }
    } else {
      A = each(A, [](float x, int) { return kept(x); });
    }
#pragma unroll
    for (int v = 0; v < VC; ++v) pair[buf][warp][lane * VC + v] = make_float2(A.at(v), h.at(v));
    if (threadIdx.x == 32 && a.deep) place[(turn + D + 1) % RING] = place_of(a, told, CT);
    if (k == 0) {
      // The last tile may write its result over the first state (hT = h0), long after, but in another block, to which only the states that are
      // published lead.  So every warp has its first state before the block meets, not just asked for it: what it does next depends on the values.
      bool bad = false;
#pragma unroll
      for (int v = 0; v < VC; ++v) bad = bad || __uint_as_float(early[v]) != __uint_as_float(early[v]);
      if (__any_sync(0xffffffffu, bad)) {
#pragma unroll
        for (int v = 0; v < VC; ++v) early[v] = word_of(__uint_as_float(early[v]));
      }
    }
    // The only meeting of the block's warps, as a rule: the arrays are used in turn.  grows: a coefficient of the tile is above 1, so that pieces that
    // underflow are of no use either; walk: some piece has to be walked.
    bool grows = false, walk = false;
    if constexpr (STRICT) {
      grows = __syncthreads_or(big);
      if (grows) {
        if (!big) {
#pragma unroll
          for (int v = 0; v < VC; ++v) {
            if (fabsf(A.at(v)) < kLeast && A.at(v) != 0.f) {
              pair[buf][warp][lane * VC + v].x = A.at(v) = kLost;
              lost = true;
            }
          }
        }
        walk = __syncthreads_or(lost);
      }
    } else {
      __syncthreads();
    }

    // every warp carries the state in front of the tile through the pairs of the warps before it; the last one speaks for the tile
    const bool speaker = warp == kWarps - 1 && k + 1 < a.nk;
    float2 whole[VC];
    const auto join = [&](bool cuts) {
#pragma unroll
      for (int v = 0; v < VC; ++v) whole[v] = pair[buf][0][lane * VC + v];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) {
#pragma unroll
        for (int v = 0; v < VC; ++v) whole[v] = through(pair[buf][w][lane * VC + v], whole[v], cuts);
      }
#pragma unroll
      for (int v = 0; v < VC; ++v) {
        float& p = whole[v].x;
        if (!STRICT) {
          p = kept(p);
        } else if (grows || p == 0.f) {
          float up = 0.f, down = kMost;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            const float x = pair[buf][w][lane * VC + v].x;
            up = largest(up, x, x);
            down = smallest_nan(down, x, x);
          }
          if (down == 0.f) {                   // (all of them are finite)
            p = 0.f;
          } else if (up <= kSteady) {
            p = kept(p);
          } else if (down == down && !(up <= 32768.f && down * 32768.f >= 1.f)) {
            float q = 1.f;
            bool out = false;
#pragma unroll 1
            for (int w = 0; w < kWarps; ++w) {
              q *= pair[buf][w][lane * VC + v].x;
              out = out || !(fabsf(q) >= kLeast && fabsf(q) <= kMost);
            }
            if (out) p = kLost;
          }
        }
      }
    };
    // what the tile makes of the state in front of it; without a product: piece by piece
    const auto tell = [&](const V& first, bool cuts) {
#pragma unroll
      for (int v = 0; v < VC; ++v) {
        float x = through(whole[v], first.at(v), cuts);
        if (STRICT && whole[v].x == kLost) {
          x = first.at(v);
#pragma unroll 1
          for (int w = 0; w < kWarps; ++w) x = through(pair[buf][w][lane * VC + v], x, cuts);
        }
        st_word(a.states + word + v, word_of(x));
      }
    };
    if (speaker && !walk) join(cut);
#pragma unroll
    for (int v = 0; v < VC; ++v) h.at(v) = __uint_as_float(early[v]);
    if (k > 0) {
      bool known = true;
#pragma unroll
      for (int v = 0; v < VC; ++v) known = known && early[v] != kNone;
      if (!__all_sync(0xffffffffu, known)) {
        if (speaker && !walk) {                // (a pair that does not come is waited for until the state behind it is there)
#pragma unroll
          for (int v = 0; v < VC; ++v)
            if (!STRICT || whole[v].x != kLost) st_pair(a.pairs + word + v, whole[v]);
        }
        if (!NARROW || warp == kWarps - 1) {
          h = look_back<VC, NARROW, CUT>(a, k, row, (i64)c * CT, lane);
        } else {                               // the last warp asks L2 for all of them
          // (every lane looks for itself, a bounded number of times; then the warp meets, and stays or leaves as one)
          uint64_t t0 = 0;
          bool there;
          do {
            unsigned round = 0;
#pragma unroll 1
            while (posted[buf] != turn + 1u && ++round < 4096u) {}
            __syncwarp();
            there = __any_sync(0xffffffffu, round < 4096u);
          } while (!there && !waited_too_long(a, lane, 31u, t0));
          __syncwarp();
          __threadfence_block();
          h = there ? front[buf][lane] : V::all(__uint_as_float(0x7fc00000u));      // (run out: the results are void, and look it)
        }
      }
      if (NARROW && warp == kWarps - 1) {       // (whether it had to look back or not: the others asked a moment earlier)
        front[buf][lane] = h;
        __syncwarp();
        __threadfence_block();
        if (lane == 0) posted[buf] = turn + 1u;
      }
    }
    if (!walk) {
      if (speaker) tell(h, cut);
#pragma unroll
      for (int w = 0; w < kWarps - 1; ++w) {
#pragma unroll
        for (int v = 0; v < VC; ++v) {
          const float2 p = pair[buf][w][lane * VC + v];
          if (w < warp) h.at(v) = through(p, h.at(v), cut);
        }
      }
    } else {
      // One warp after the other: a column's piece without a product is walked, and what comes out of it takes the place of its pair.  Other
      // columns go by their pairs as ever, so that their bits do not depend on their neighbours.
      const V first = h;
#pragma unroll 1
      for (int w = 0; w < kWarps; ++w) {
        if (w == warp && lost) {
          V x = h;
#pragma unroll
          for (int s = 0; s < S; ++s) x = step(s, x);
#pragma unroll
          for (int v = 0; v < VC; ++v)
            if (A.at(v) == kLost) pair[buf][w][lane * VC + v] = make_float2(__uint_as_float(0x7fc00000u), x.at(v));
        }
        __syncthreads();
        if (w < warp) {
#pragma unroll
          for (int v = 0; v < VC; ++v) h.at(v) = through(pair[buf][w][lane * VC + v], h.at(v), true);
        }
      }
      if (speaker) {
        join(true);
        tell(first, true);
      }
    }
    T *po = at(BACK ? a.dgate : a.h, now, time_of(now.i0)), *pw = BACK ? at(a.dcand, now, time_of(now.i0)) : nullptr;
    const i64 dout = BACK ? -a.dgate.ts : a.h.ts;
    const auto put = [&](T* p, const V& x) {
      if constexpr (ALIGNED) {
        store<T, VC>(p, x);
      } else {
#pragma unroll
        for (int v = 0; v < VC; ++v)
          if (v < now.n) p[v] = from_f32<T>(x.at(v));
      }
    };
#pragma unroll
    for (int s = 0; s < S; ++s) {
      V x, y;
      if (BACK) {
        const V lam = h + cb[s];
        x = lam * wg[BACK ? s : 0];
        y = lam * wc[BACK ? s : 0];
      }
      h = step(s, h);
      if (!BACK) x = h;
      bool write = true;
      if (ODD) {
        const int t = time_of(now.i0 + s);
        write = now.n > 0 && t >= 0 && t < a.T;
        const bool in = in_now >> s & 1u;
        x = each(x, [&](float v, int) { return in ? v : 0.f; });
        if (BACK) y = each(y, [&](float v, int) { return in ? v : 0.f; });
      }
      if (write) {
        put(po + s * dout, x);
        if (BACK) put(pw - s * a.dcand.ts, y);
      }
    }
    float* last = BACK ? a.dh0 : a.hT;
    if (last && k + 1 == a.nk && warp == kWarps - 1) store_state<VC>(last, now.b * (unsigned)a.H + now.u, h, now.n);
    return theirs;
  };
  for (unsigned turn = 0, d = 0;; ++turn, d = d + 1 == D ? 0 : d + 1) {
    if (!a.deep) {
      if (threadIdx.x == 32) place[turn % RING] = place_of(a, draw(), CT);
      __syncthreads();
    }
    const Place here = place[turn % RING];
    if (here.k < 0) break;
    const Spot now = spot_of(here, lane * VC);
    if (!a.deep) {
      ahead[0] = fetch(here, d);
#pragma unroll
      for (int i = 1; i < D; ++i) none();
    }
    const unsigned bits = marked(ahead[0], now);
    // (CUT: one body for all warps.  With two, half of the time went into fetching instructions: 188 us forward, 301 backward for T 2048, B 32, H 1024
    // in bf16 with lengths and starts, 138 and 230 with one.)
    Known theirs;
    if (!CUT && __all_sync(0xffffffffu, bits == ALL && !(BACK && time_of(now.i0 + S - 1) <= 0)))
      theirs = work(std::false_type{}, d, turn, here, now, bits & 0xffffu, bits >> 16);
    else
      theirs = work(std::true_type{}, d, turn, here, now, bits & 0xffffu, bits >> 16);
#pragma unroll
    for (int i = 0; i + 1 < D; ++i) ahead[i] = ahead[i + 1];
    ahead[D - 1] = theirs;
  }
}

constexpr int kWidest = 32 * 4;
// Workspace: counter | states | pairs, filled with kNone.  Columns are padded to the wider column tile, time to the shorter (backward) tile.
constexpr int kLeastSteps = kStepsOf<true> * kWarps;
struct ScanSpace { size_t states, pairs, total; };
ScanSpace scan_space(i64 nk, i64 padded) {
  ScanSpace s;
  s.states = 256;
  s.pairs = s.states + (((size_t)nk * padded * sizeof(float) + 255) & ~(size_t)255);
  s.total = s.pairs + (((size_t)nk * padded * sizeof(float2) + 255) & ~(size_t)255);
  return s;
}

// blocks of a kernel that fit the device at once, asked once for each kernel and device
template <class K> int resident_blocks(K kern, int threads, int smem, int (&known)[kMaxDevices]) {
  const int dev = current_device_slot();
  if (dev < 0) return 0;
  if (!known[dev]) {
    int per_sm = 0, sms = 0;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, threads, smem) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return 0;
    known[dev] = per_sm * sms;
  }
  return known[dev];
}

template <class T, int MODE, bool ALIGNED, bool BACK> int launch_kernels(ScanArgs& a, void* ws, cudaStream_t s) {
  constexpr int VC = kWide<T>;
  if (a.T <= kShort) {
    if constexpr (MODE == kOpen || MODE == kGiven) {
      constexpr int VS = ALIGNED ? VC : 1;
      const i64 cols = (i64)a.B * a.H;
      scan_short_kernel<T, MODE, VS, BACK><<<(unsigned)((cols / VS + kShortThreads - 1) / kShortThreads), kShortThreads, 0, s>>>(a);
    }
  } else {
    constexpr int steps = kStepsOf<BACK> * kWarps, wide = 32 * VC;
    a.Hp = (a.H + VC - 1) / VC * VC;
    const i64 cols = (i64)a.B * a.Hp;
    if (cols >= ((i64)1 << 31)) return MGRIT_UNSUPPORTED;
    const i64 nc = (cols + wide - 1) / wide, nk = ((i64)a.T + steps - 1) / steps;
    if (nk * nc >= INT32_MAX) return MGRIT_UNSUPPORTED;
    a.nk = (int)nk; a.nc = (int)nc;
    if (nk > 1) {
      const ScanSpace sp = scan_space(nk, nc * wide);
      char* w = static_cast<char*>(ws);
      a.ticket = reinterpret_cast<unsigned*>(w);
      a.states = reinterpret_cast<float*>(w + sp.states);
      a.pairs = reinterpret_cast<unsigned long long*>(w + sp.pairs);
      if (!a.status || cudaMemsetAsync(ws, 0xff, sp.total, s) != cudaSuccess) { cudaGetLastError(); return MGRIT_CUDA_ERROR; }
    }
    // Few column tiles: every tile looks far back, and the blocks' warps in each other's way.  One warp then asks for all of them, for many
    // pairs at a time.  With more column tiles a state is usually there, and warps that look for themselves are ahead.  16384 steps, us, one warp :
    // every warp, for 1, 2, 4, 5, 6, 8 and 12 column tiles: bf16 forward 31 : 57, 32 : 53, 38 : 53, 45 : 60, 50 : 60, 63 : 69, 84 : 82, backward
    // 48 : 90, 52 : 90, 72 : 105, 80 : 108, 90 : 115, 104 : 118, 139 : 141; fp32 forward 19 : 31, 21 : 32, 30 : 35, 35 : 39, 39 : 40, 50 : 48,
    // 68 : 60, backward 29 : 53, 35 : 54, 51 : 63, 61 : 68, 71 : 71, 88 : 82, 119 : 103.
    constexpr int smem = kAhead * (BACK ? 4 : 2) * kStepsOf<BACK> * kWarps * (ALIGNED ? 32 : 64) * 8;
    const auto run = [&](auto kern, int (&known)[kMaxDevices]) {
      const int most = resident_blocks(kern, kWarps * 32, smem, known);
      if (most <= 0) { cudaGetLastError(); return false; }
      // every block gets four tiles or more: enough that the first ones to run may take several at once
      a.deep = nk * nc >= 4 * (i64)most;
      kern<<<(unsigned)(nk * nc < most ? nk * nc : most), kWarps * 32, smem, s>>>(a);
      return true;
    };
    static int known[4][kMaxDevices];
    bool ok;
    if constexpr (MODE == kLarge)
      ok = run(scan_tile_kernel<T, MODE, ALIGNED, BACK, false, true>, known[0]);
    else
      ok = nc <= kNarrow ? a.reset.p ? run(scan_tile_kernel<T, MODE, ALIGNED, BACK, true, true>, known[0]) : run(scan_tile_kernel<T, MODE, ALIGNED, BACK, true, false>, known[1])
                         : a.reset.p ? run(scan_tile_kernel<T, MODE, ALIGNED, BACK, false, true>, known[2]) : run(scan_tile_kernel<T, MODE, ALIGNED, BACK, false, false>, known[3]);
    if (!ok) return MGRIT_CUDA_ERROR;
  }
  count_launch();
  return cudaGetLastError() == cudaSuccess ? MGRIT_OK : MGRIT_CUDA_ERROR;
}

}  // namespace

template <class T, int MODE> int launch_scan(ScanArgs& a, bool wide, bool back, void* ws, cudaStream_t s) {
  // (states of the classic cell with dt > 2 grow without bound wherever its gates are open: one kernel for whatever is left)
  if constexpr (MODE != kLarge)
    if (wide) return back ? launch_kernels<T, MODE, true, true>(a, ws, s) : launch_kernels<T, MODE, true, false>(a, ws, s);
  return back ? launch_kernels<T, MODE, false, true>(a, ws, s) : launch_kernels<T, MODE, false, false>(a, ws, s);
}

}  // namespace mg
