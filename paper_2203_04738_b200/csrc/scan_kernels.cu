// Gated linear recurrence: arguments, workspace, status word and entry points.  The kernels are in scan_tile.cuh, compiled for one element type
// and one origin of the coefficients at a time.
#include "scan_tile.cuh"

namespace mg {

extern template int launch_scan<float, kCells>(ScanArgs&, bool, bool, void*, cudaStream_t);
extern template int launch_scan<float, kOpen>(ScanArgs&, bool, bool, void*, cudaStream_t);
extern template int launch_scan<float, kGiven>(ScanArgs&, bool, bool, void*, cudaStream_t);
extern template int launch_scan<float, kLarge>(ScanArgs&, bool, bool, void*, cudaStream_t);
extern template int launch_scan<__nv_bfloat16, kCells>(ScanArgs&, bool, bool, void*, cudaStream_t);
extern template int launch_scan<__nv_bfloat16, kOpen>(ScanArgs&, bool, bool, void*, cudaStream_t);
extern template int launch_scan<__nv_bfloat16, kGiven>(ScanArgs&, bool, bool, void*, cudaStream_t);
extern template int launch_scan<__nv_bfloat16, kLarge>(ScanArgs&, bool, bool, void*, cudaStream_t);
extern template int launch_scan<__half, kCells>(ScanArgs&, bool, bool, void*, cudaStream_t);
extern template int launch_scan<__half, kOpen>(ScanArgs&, bool, bool, void*, cudaStream_t);
extern template int launch_scan<__half, kGiven>(ScanArgs&, bool, bool, void*, cudaStream_t);
extern template int launch_scan<__half, kLarge>(ScanArgs&, bool, bool, void*, cudaStream_t);

namespace {

__device__ int g_scan_status = 0;              // 1: a look-back's wait ran out
int* g_scan_status_ptrs[kMaxDevices] = {nullptr};

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

// (the stride of an axis with one place says nothing)
ScanRows rows_of(const mgrit_rows& r, const gated_scan_args* x) { return ScanRows{static_cast<char*>(r.data), x->T > 1 ? r.t_stride : 0, x->B > 1 ? r.b_stride : 0}; }

int check_scan(const gated_scan_args* x, bool back, ScanArgs& a) {
  if (!x || x->T < 0 || x->B < 0 || x->H <= 0 || x->cell < 0 || x->cell > MGRIT_SCAN_COEFFICIENTS || !elem_known(x->dtype)) return MGRIT_INVALID_ARG;
  if (!(x->dt >= 0.f && x->dt <= kMaxDt)) return MGRIT_INVALID_ARG;
  if (!scan_sizes_served(x->T, x->B, x->H)) return MGRIT_UNSUPPORTED;
  a = ScanArgs{};
  a.T = x->T; a.B = x->B; a.H = x->H; a.dt = x->dt;
  a.K = x->cell == MGRIT_CELL_IMPLICIT ? 1.0f + x->dt : 1.0f;
  a.L = x->cell == MGRIT_CELL_IMPLICIT ? 1.0f : 1.0f - x->dt;
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
  a.gate = rows_of(x->gate, x); a.cand = rows_of(x->cand, x); a.h = rows_of(x->h, x); a.reset = rows_of(x->reset, x);
  bool ok = elem_aligned(a.gate.p, x->dtype) && elem_aligned(a.cand.p, x->dtype) && elem_aligned(a.h.p, x->dtype);
  if (back) {
    if (!x->dgate.data || !x->dcand.data || (!x->dh_seed.data && !x->dhT)) return MGRIT_INVALID_ARG;
    a.seed = rows_of(x->dh_seed, x); a.dgate = rows_of(x->dgate, x); a.dcand = rows_of(x->dcand, x);
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

size_t scan_workspace(int T, int B, int H) {
  if (!scan_sizes_served(T, B, H) || T <= kLeastSteps || B == 0) return 0;
  return scan_space(((i64)T + kLeastSteps - 1) / kLeastSteps, ((i64)B * ((H + 3) / 4 * 4) + kWidest - 1) / kWidest * kWidest).total;
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

// several columns a thread and asynchronous copies where rows allow it: units and strides whole words of 16 bytes, all addresses on such words
bool wide_columns(const ScanArgs& a, int dtype) {
  const int n = 16 / (int)elem_size(dtype);
  const auto fits = [&](const ScanRows& r) { return !r.p || (((uintptr_t)r.p & 15u) == 0 && r.ts % n == 0 && r.bs % n == 0); };
  return a.H % n == 0 && fits(a.gate) && fits(a.cand) && fits(a.h) && fits(a.seed) && fits(a.dgate) && fits(a.dcand);
}

int run_scan(const gated_scan_args* x, bool back, void* ws, size_t ws_bytes, cudaStream_t s) {
  ScanArgs a;
  int rc = check_scan(x, back, a);
  if (rc != MGRIT_OK) return rc;
  if (a.T == 0 || a.B == 0) return back ? copy_state(a.dh0, a.dhT, (size_t)a.B * a.H, s) : copy_state(a.hT, a.h0, (size_t)a.B * a.H, s);
  const size_t need = scan_workspace(a.T, a.B, a.H);
  if (need > 0 && (!ws || ((uintptr_t)ws & 255u))) return MGRIT_INVALID_ARG;
  if (ws_bytes < need) return MGRIT_WORKSPACE_TOO_SMALL;
  const bool wide = wide_columns(a, x->dtype);
  const bool implicit = x->cell == MGRIT_CELL_IMPLICIT, walked = a.T <= kShort;
  const int mode = x->cell == MGRIT_SCAN_COEFFICIENTS ? kGiven : !walked && x->dt <= (implicit ? 1.0f : 0.5f) ? kCells
                   : !walked && !implicit && x->dt > 2.0f ? kLarge : kOpen;
  if (need > 0 && !(a.status = scan_status_ptr())) return MGRIT_CUDA_ERROR;
  with_elem(x->dtype, [&](auto tag) {
    using T = decltype(tag);
    rc = mode == kCells   ? launch_scan<T, kCells>(a, wide, back, ws, s)
         : mode == kOpen  ? launch_scan<T, kOpen>(a, wide, back, ws, s)
         : mode == kGiven ? launch_scan<T, kGiven>(a, wide, back, ws, s)
                          : launch_scan<T, kLarge>(a, wide, back, ws, s);
  });
  return rc;
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

size_t gated_scan_workspace_bytes(int32_t T, int32_t B, int32_t H) { return mg::scan_workspace(T, B, H); }

int gated_scan_forward(const gated_scan_args* args, void* ws, size_t ws_bytes, mgrit_stream_t stream) {
  return mg::run_scan(args, false, ws, ws_bytes, (cudaStream_t)stream);
}

int gated_scan_backward(const gated_scan_args* args, void* ws, size_t ws_bytes, mgrit_stream_t stream) {
  return mg::run_scan(args, true, ws, ws_bytes, (cudaStream_t)stream);
}

}  // extern "C"
