// Gated linear recurrence h_t = a_t h_{t-1} + b_t, forward and backward.
#include "elem.cuh"

namespace mg {
namespace {

struct ScanRows { char* p; i64 ts, bs; };      // strides in elements
struct ScanArgs {
  int T, B, H;
  float dt;
  ScanRows gate, cand, h, seed, dgate, dcand, reset;
  const float* h0; const int32_t* lengths; float* hT;
  const float* dhT; float* dh0;
};

constexpr int kScanThreads = 256;

// a, b and, for the derivatives, z, n and r (implicit: 1 / (1 + dt z), classic: 1) of one element.
// With E = e^-g and F = e^2c:  z = 1 / (1 + E), n = (F - 1) / (F + 1), 1 / (1 + dt z) = (1 + E) / (1 + E + dt).
// 1 - dt z is formed as ((1 - dt) + E) z, which loses nothing where z is near 1.
struct Coef { float a, b, z, n, r; };
template <int CELL> __device__ __forceinline__ Coef coefficients(float g, float c, float dt) {
  Coef o;
  if (CELL == MGRIT_SCAN_COEFFICIENTS) { o.a = g; o.b = c; o.z = o.n = o.r = 0.f; return o; }
  const float E = __expf(-g);
  o.n = tanhf(c);
  o.z = 1.0f / (1.0f + E);
  if (CELL == MGRIT_CELL_CLASSIC) {
    o.r = 1.0f;
    o.a = E < 1e30f ? ((1.0f - dt) + E) * o.z : 1.0f;
    if (E != E) o.a = E;
  } else {
    o.r = 1.0f / (1.0f + dt * o.z);
    o.a = o.r;
  }
  o.b = dt * o.z * o.n * o.r;
  return o;
}

// One thread per column (b, unit), one step after the other.
template <class T, int CELL>
__global__ void __launch_bounds__(kScanThreads) scan_fwd_kernel(const ScanArgs a) {
  const i64 col = (i64)blockIdx.x * kScanThreads + threadIdx.x;
  if (col >= (i64)a.B * a.H) return;
  const int b = (int)(col / a.H), u = (int)(col % a.H);
  const int len = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const T* gate = reinterpret_cast<const T*>(a.gate.p) + b * a.gate.bs + u;
  const T* cand = reinterpret_cast<const T*>(a.cand.p) + b * a.cand.bs + u;
  T* out = reinterpret_cast<T*>(a.h.p) + b * a.h.bs + u;
  const uint8_t* reset = a.reset.p ? reinterpret_cast<const uint8_t*>(a.reset.p) + b * a.reset.bs : nullptr;
  float h = a.h0 ? a.h0[col] : 0.f;
  for (int t = 0; t < len; ++t) {
    const Coef k = coefficients<CELL>(to_f32(gate[t * a.gate.ts]), to_f32(cand[t * a.cand.ts]), a.dt);
    h = reset && reset[t * a.reset.ts] ? k.b : fmaf(k.a, h, k.b);
    out[t * a.h.ts] = from_f32<T>(h);
  }
  for (int t = len; t < a.T; ++t) out[t * a.h.ts] = from_f32<T>(0.f);
  if (a.hT) a.hT[col] = h;
}

template <class T, int CELL>
__global__ void __launch_bounds__(kScanThreads) scan_bwd_kernel(const ScanArgs a) {
  const i64 col = (i64)blockIdx.x * kScanThreads + threadIdx.x;
  if (col >= (i64)a.B * a.H) return;
  const int b = (int)(col / a.H), u = (int)(col % a.H);
  const int len = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const T* gate = reinterpret_cast<const T*>(a.gate.p) + b * a.gate.bs + u;
  const T* cand = reinterpret_cast<const T*>(a.cand.p) + b * a.cand.bs + u;
  const T* h = reinterpret_cast<const T*>(a.h.p) + b * a.h.bs + u;
  const T* seed = a.seed.p ? reinterpret_cast<const T*>(a.seed.p) + b * a.seed.bs + u : nullptr;
  T* dgate = reinterpret_cast<T*>(a.dgate.p) + b * a.dgate.bs + u;
  T* dcand = reinterpret_cast<T*>(a.dcand.p) + b * a.dcand.bs + u;
  const uint8_t* reset = a.reset.p ? reinterpret_cast<const uint8_t*>(a.reset.p) + b * a.reset.bs : nullptr;
  for (int t = len; t < a.T; ++t) {
    dgate[t * a.dgate.ts] = from_f32<T>(0.f);
    dcand[t * a.dcand.ts] = from_f32<T>(0.f);
  }
  float mu = a.dhT ? a.dhT[col] : 0.f;
  for (int t = len - 1; t >= 0; --t) {
    const Coef k = coefficients<CELL>(to_f32(gate[t * a.gate.ts]), to_f32(cand[t * a.cand.ts]), a.dt);
    const bool fresh = reset && reset[t * a.reset.ts];
    const float hp = fresh ? 0.f : t > 0 ? to_f32(h[(t - 1) * a.h.ts]) : a.h0 ? a.h0[col] : 0.f;
    const float lam = mu + (seed ? to_f32(seed[t * a.seed.ts]) : 0.f);
    float dg, dc;
    if (CELL == MGRIT_SCAN_COEFFICIENTS) { dg = lam * hp; dc = lam; }
    else {
      dg = lam * (a.dt * k.r * k.r) * (k.n - hp) * (k.z * (1.f - k.z));
      dc = lam * (a.dt * k.z * k.r) * (1.f - k.n * k.n);
    }
    dgate[t * a.dgate.ts] = from_f32<T>(dg);
    dcand[t * a.dcand.ts] = from_f32<T>(dc);
    mu = fresh ? 0.f : k.a * lam;
  }
  if (a.dh0) a.dh0[col] = mu;
}

// ---- arguments ---------------------------------------------------------------------------------------------------------------

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
  if (!(x->dt >= 0.f) || x->dt > 3.0e38f) return MGRIT_INVALID_ARG;
  if ((i64)x->B * x->H >= ((i64)1 << 31) || x->T >= INT32_MAX - 1024) return MGRIT_UNSUPPORTED;
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

template <class T, int CELL> void launch_scan(const ScanArgs& a, bool back, cudaStream_t s) {
  const unsigned grid = (unsigned)(((i64)a.B * a.H + kScanThreads - 1) / kScanThreads);
  if (back) scan_bwd_kernel<T, CELL><<<grid, kScanThreads, 0, s>>>(a);
  else scan_fwd_kernel<T, CELL><<<grid, kScanThreads, 0, s>>>(a);
  count_launch();
}

int run_scan(const gated_scan_args* x, bool back, void* ws, size_t ws_bytes, cudaStream_t s) {
  ScanArgs a;
  const int rc = check_scan(x, back, a);
  if (rc != MGRIT_OK) return rc;
  if (a.T == 0 || a.B == 0) return back ? copy_state(a.dh0, a.dhT, (size_t)a.B * a.H, s) : copy_state(a.hT, a.h0, (size_t)a.B * a.H, s);
  with_elem(x->dtype, [&](auto tag) {
    using T = decltype(tag);
    if (x->cell == MGRIT_CELL_CLASSIC) launch_scan<T, MGRIT_CELL_CLASSIC>(a, back, s);
    else if (x->cell == MGRIT_CELL_IMPLICIT) launch_scan<T, MGRIT_CELL_IMPLICIT>(a, back, s);
    else launch_scan<T, MGRIT_SCAN_COEFFICIENTS>(a, back, s);
  });
  return cudaGetLastError() == cudaSuccess ? MGRIT_OK : MGRIT_CUDA_ERROR;
}

}  // namespace
}  // namespace mg

extern "C" {

size_t gated_scan_workspace_bytes(int32_t T, int32_t B, int32_t H) {
  (void)T; (void)B; (void)H;
  return 0;
}

int gated_scan_forward(const gated_scan_args* args, void* ws, size_t ws_bytes, mgrit_stream_t stream) {
  return mg::run_scan(args, false, ws, ws_bytes, (cudaStream_t)stream);
}

int gated_scan_backward(const gated_scan_args* args, void* ws, size_t ws_bytes, mgrit_stream_t stream) {
  return mg::run_scan(args, true, ws, ws_bytes, (cudaStream_t)stream);
}

}  // extern "C"
