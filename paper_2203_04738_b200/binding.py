"""Thin ctypes binding of the C ABI in include/mgrit_gru.h: argument marshalling only.

Tensors are torch CUDA tensors (fp32, contiguous); outputs and the workspace are allocated with
torch; work is enqueued on torch's current stream.  Every step of the path runs in the
library's kernels -- if the library has not been built, importing this module raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmgrit_gru.so")
if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2203_04738_b200.build` "
                      "(there is no CPU or PyTorch fallback)")
lib = ctypes.CDLL(LIB_PATH)

OK = 0
CELL_CLASSIC, CELL_IMPLICIT = 0, 1
RELAX_F, RELAX_FCF, RELAX_FCFCF = 0, 1, 2
OPERANDS_FP32, OPERANDS_TF32, OPERANDS_BF16, OPERANDS_TF32_1PASS = 0, 1, 2, 3
FLAG_SKIP_DUPLICATE_FRELAX, FLAG_F_CYCLE, FLAG_RAGGED_T, FLAG_GI_CARRIES_COPIES, FLAG_GI_F32_UNUSED = 1, 2, 4, 8, 16
FLAG_H_LEADS_WITH_H0 = 32
SCAN_COEFFICIENTS = 2                      # `cell` of the gated scan: gate and candidate are the coefficients themselves
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


class Cfg(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("T", "B", "I", "H", "cf", "levels", "iters", "cell", "relax_fine", "relax_coarse", "operands", "flags")] + \
               [("dt", ctypes.c_float)]


class _Params(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("W_ih", "W_hh", "b_ih", "b_hh")]


class _Grads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("dW_ih", "dW_hh", "db_ih", "db_hh")]


_vp, _sz, _i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
lib.mgrit_gru_workspace_bytes.argtypes = [ctypes.POINTER(Cfg), ctypes.POINTER(_sz), ctypes.POINTER(_sz)]
lib.mgrit_gru_gi_bytes.argtypes = [ctypes.POINTER(Cfg)]
lib.mgrit_gru_gi_bytes.restype = _sz
lib.gru_input_projection.argtypes = [ctypes.POINTER(Cfg), ctypes.POINTER(_Params), _vp, _vp, _vp, _sz, _vp]
lib.mgrit_gru_forward.argtypes = [ctypes.POINTER(Cfg), ctypes.POINTER(_Params), _vp, _vp, _vp, _vp,
                                  ctypes.POINTER(ctypes.c_float), _vp, _sz, _vp]
lib.gru_serial_forward.argtypes = [ctypes.POINTER(Cfg), ctypes.POINTER(_Params), _vp, _vp, _vp, _vp, _vp, _sz, _vp]
lib.mgrit_gru_adjoint.argtypes = [ctypes.POINTER(Cfg), ctypes.POINTER(_Params), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                  ctypes.POINTER(_Grads), ctypes.POINTER(ctypes.c_float), _vp, _sz, _vp]
lib.gru_serial_backward.argtypes = [ctypes.POINTER(Cfg), ctypes.POINTER(_Params), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                    ctypes.POINTER(_Grads), _vp, _sz, _vp]
lib.mgrit_gru_stack_workspace_bytes.argtypes = [ctypes.POINTER(Cfg), _i32, ctypes.POINTER(_sz), ctypes.POINTER(_sz)]
lib.mgrit_gru_stack_forward.argtypes = [ctypes.POINTER(Cfg), _i32, ctypes.POINTER(_Params), _vp, _vp, _vp, _vp,
                                        ctypes.POINTER(ctypes.c_float), _vp, _sz, _vp]
lib.mgrit_gru_stack_adjoint.argtypes = [ctypes.POINTER(Cfg), _i32, ctypes.POINTER(_Params), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                        ctypes.POINTER(_Grads), ctypes.POINTER(ctypes.c_float), _vp, _sz, _vp]
lib.mgrit_lstm_workspace_bytes.argtypes = [ctypes.POINTER(Cfg), ctypes.POINTER(_sz), ctypes.POINTER(_sz)]
lib.mgrit_lstm_forward.argtypes = [ctypes.POINTER(Cfg), ctypes.POINTER(_Params), _vp, _vp, _vp, _vp, ctypes.POINTER(ctypes.c_float), _vp, _sz, _vp]
lib.mgrit_lstm_adjoint.argtypes = [ctypes.POINTER(Cfg), ctypes.POINTER(_Params), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                   ctypes.POINTER(_Grads), ctypes.POINTER(ctypes.c_float), _vp, _sz, _vp]
lib.gru_step_rows.argtypes = [ctypes.POINTER(Cfg), ctypes.POINTER(_Params), _i32, ctypes.c_float, _vp, _vp, _vp, _vp]
lib.gru_adjoint_step_rows.argtypes = [ctypes.POINTER(Cfg), ctypes.POINTER(_Params), _i32, ctypes.c_float, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
lib.xent_head_workspace_bytes.argtypes = [_i32, _i32]
lib.xent_head_workspace_bytes.restype = _sz
lib.xent_head_fwd_bwd.argtypes = [_i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
lib.xent_head_fwd_bwd_noalloc.argtypes = [_i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
lib.sgd_update.argtypes = [_vp, _vp, _sz, ctypes.c_float, _vp]
lib.adam_update.argtypes = [_vp, _vp, _vp, _vp, _sz, ctypes.c_float, ctypes.c_float, ctypes.c_float, ctypes.c_float, _i32, _vp]
lib.gated_scan_workspace_bytes.argtypes = [_i32, _i32, _i32]
lib.gated_scan_workspace_bytes.restype = _sz
lib.gated_scan_forward.argtypes = [ctypes.c_char_p, _vp, _sz, _vp]
lib.gated_scan_backward.argtypes = [ctypes.c_char_p, _vp, _sz, _vp]
lib.token_logprobs.argtypes = [_i32, _i32, _i32, _vp, ctypes.c_int64, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp]
lib.token_logprobs_backward.argtypes = [_i32, _i32, _i32, _vp, ctypes.c_int64, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_int64, _vp]
lib.distill_topk_fwd_bwd.argtypes = [_i32, _i32, _i32, _i32, ctypes.c_float, _vp, ctypes.c_int64, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_int64, _vp]
lib.mgrit_gru_selftest_bounded_wait.argtypes = [_i32, _vp]
lib.mgrit_gru_last_device_status.restype = ctypes.c_int
lib.mgrit_gru_clear_device_status.restype = ctypes.c_int
lib.mgrit_gru_kernel_launches.restype = ctypes.c_ulonglong
lib.mgrit_gru_profile_enable.argtypes = [ctypes.c_int]
lib.mgrit_gru_profile_read.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_ulonglong),
                                       ctypes.POINTER(ctypes.c_double)]
lib.mgrit_gru_profile_records.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double),
                                          ctypes.POINTER(ctypes.c_int32), _sz, ctypes.POINTER(_sz)]
lib.mgrit_gru_strerror.argtypes = [ctypes.c_int]
lib.mgrit_gru_strerror.restype = ctypes.c_char_p


class MgritError(RuntimeError):
    def __init__(self, code):
        self.code = code
        super().__init__(f"mgrit_gru error {code}: {lib.mgrit_gru_strerror(code).decode()}")


def _check(rc):
    if rc != OK:
        raise MgritError(rc)


def make_cfg(T, B, I, H, cf=4, levels=2, iters=2, cell=CELL_IMPLICIT, relax_fine=RELAX_F, relax_coarse=RELAX_FCF,
             operands=OPERANDS_FP32, flags=0, dt=1.0) -> Cfg:
    return Cfg(T, B, I, H, cf, levels, iters, cell, relax_fine, relax_coarse, operands, flags, dt)


def _ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "CUDA contiguous tensor required"
    return ctypes.c_void_p(t.data_ptr())


def _f32(t):
    assert t is None or t.dtype == torch.float32
    return _ptr(t)


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _params(p):
    return _Params(*[p[n].data_ptr() for n in ("W_ih", "W_hh", "b_ih", "b_hh")])


def workspace_bytes(cfg: Cfg):
    f, a = _sz(0), _sz(0)
    _check(lib.mgrit_gru_workspace_bytes(ctypes.byref(cfg), ctypes.byref(f), ctypes.byref(a)))
    return f.value, a.value


def alloc_gi(cfg: Cfg, device) -> torch.Tensor:
    """The gi buffer for cfg as a flat fp32 tensor: gi[T,B,3H] first, then (with FLAG_GI_CARRIES_COPIES) room for the
    bf16 copies that travel from the forward call to the adjoint call.  `gi_view(cfg, buf)` is the projection itself."""
    nbytes = lib.mgrit_gru_gi_bytes(ctypes.byref(cfg))
    if nbytes == 0:
        raise MgritError(-1)
    return torch.empty((nbytes + 3) // 4, dtype=torch.float32, device=device)


def gi_view(cfg: Cfg, buf: torch.Tensor) -> torch.Tensor:
    return buf[: cfg.T * cfg.B * 3 * cfg.H].view(cfg.T, cfg.B, 3 * cfg.H)


def _ws(nbytes, ws, dev):
    if ws is None or ws.numel() < nbytes:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    return ws


def gru_input_projection(cfg, p, x, gi=None, ws=None):
    gi = torch.empty(cfg.T, cfg.B, 3 * cfg.H, device=x.device) if gi is None else gi
    ws = _ws(workspace_bytes(cfg)[0], ws, x.device)
    _check(lib.gru_input_projection(ctypes.byref(cfg), ctypes.byref(_params(p)), _f32(x), _f32(gi), _ptr(ws), ws.numel(), _stream()))
    return gi


def _h_array(cfg, h, dev):
    """The state array of a forward call and the number of leading slots that are not part of h[T,B,H]."""
    lead = 1 if cfg.flags & FLAG_H_LEADS_WITH_H0 else 0
    if h is None:
        h = torch.empty(cfg.T + lead, cfg.B, cfg.H, device=dev)
    assert h.shape[0] == cfg.T + lead and h.is_contiguous()
    return h, lead


def mgrit_gru_forward(cfg, p, x, h0, want_resnorm=False, gi=None, h=None, ws=None):
    """-> (h[T,B,H], gi[T,B,3H], resnorm list or None).  With FLAG_H_LEADS_WITH_H0 the array passed as `h` (or allocated
    here) has T + 1 slots, slot 0 receives h_0, and the returned h is the view of its slots 1..T."""
    dev = x.device
    gi = alloc_gi(cfg, dev) if gi is None else gi       # (a flat buffer when the copies flag is set, else viewed as [T,B,3H])
    if gi.dim() == 1 and not (cfg.flags & FLAG_GI_CARRIES_COPIES):
        gi = gi_view(cfg, gi)
    h, lead = _h_array(cfg, h, dev)
    ws = _ws(workspace_bytes(cfg)[0], ws, dev)
    rn = (ctypes.c_float * max(cfg.iters, 1))() if want_resnorm else None
    _check(lib.mgrit_gru_forward(ctypes.byref(cfg), ctypes.byref(_params(p)), _f32(x), _f32(h0), _f32(gi), _f32(h), rn,
                                 _ptr(ws), ws.numel(), _stream()))
    return h[lead:], gi, (list(rn)[:cfg.iters] if want_resnorm else None)


def gru_serial_forward(cfg, p, x, h0, gi=None, h=None, ws=None):
    dev = x.device
    gi = torch.empty(cfg.T, cfg.B, 3 * cfg.H, device=dev) if gi is None else gi
    h, lead = _h_array(cfg, h, dev)
    ws = _ws(workspace_bytes(cfg)[0], ws, dev)
    _check(lib.gru_serial_forward(ctypes.byref(cfg), ctypes.byref(_params(p)), _f32(x), _f32(h0), _f32(gi), _f32(h),
                                  _ptr(ws), ws.numel(), _stream()))
    return h[lead:], gi


@dataclass
class AdjointResult:
    dh: torch.Tensor | None
    dh0: torch.Tensor
    dx: torch.Tensor | None
    dW_ih: torch.Tensor
    dW_hh: torch.Tensor
    db_ih: torch.Tensor
    db_hh: torch.Tensor
    resnorm: list | None = None


def _adjoint(fn, serial, cfg, p, x, h0, gi, h, dh_seed, dhT, want_dx, want_resnorm, ws, out, want_dh=True):
    dev = x.device
    o = out or AdjointResult(
        dh=torch.empty(cfg.T, cfg.B, cfg.H, device=dev) if want_dh else None, dh0=torch.empty(cfg.B, cfg.H, device=dev),
        dx=torch.empty(cfg.T, cfg.B, cfg.I, device=dev) if want_dx else None,
        dW_ih=torch.empty(3 * cfg.H, cfg.I, device=dev), dW_hh=torch.empty(3 * cfg.H, cfg.H, device=dev),
        db_ih=torch.empty(3 * cfg.H, device=dev), db_hh=torch.empty(3 * cfg.H, device=dev))
    ws = _ws(workspace_bytes(cfg)[1], ws, dev)
    g = _Grads(o.dW_ih.data_ptr(), o.dW_hh.data_ptr(), o.db_ih.data_ptr(), o.db_hh.data_ptr())
    args = [ctypes.byref(cfg), ctypes.byref(_params(p)), _f32(x), _f32(h0), _f32(gi), _f32(h), _f32(dh_seed), _f32(dhT),
            _f32(o.dh), _f32(o.dh0), _f32(o.dx), ctypes.byref(g)]
    if not serial:
        rn = (ctypes.c_float * max(cfg.iters, 1))() if want_resnorm else None
        args.append(rn)
    args += [_ptr(ws), ws.numel(), _stream()]
    _check(fn(*args))
    if not serial and want_resnorm:
        o.resnorm = list(rn)[:cfg.iters]
    return o


def mgrit_gru_adjoint(cfg, p, x, h0, gi, h, dh_seed=None, dhT=None, want_dx=True, want_resnorm=False, ws=None, out=None,
                      want_dh=True):
    return _adjoint(lib.mgrit_gru_adjoint, False, cfg, p, x, h0, gi, h, dh_seed, dhT, want_dx, want_resnorm, ws, out, want_dh)


def gru_serial_backward(cfg, p, x, h0, gi, h, dh_seed=None, dhT=None, want_dx=True, ws=None, out=None, want_dh=True):
    return _adjoint(lib.gru_serial_backward, True, cfg, p, x, h0, gi, h, dh_seed, dhT, want_dx, False, ws, out, want_dh)


def gru_step_rows(cfg, p, gamma, gi_rows, u_prev, out=None):
    """out[n,B,H] = Phi_gamma(gi_rows[n,B,3H], u_prev[n,B,H]): one cell evaluation for n*B independent rows (fp32 engine)."""
    n = u_prev.shape[0]
    out = torch.empty_like(u_prev) if out is None else out
    _check(lib.gru_step_rows(ctypes.byref(cfg), ctypes.byref(_params(p)), n, float(gamma), _f32(gi_rows), _f32(u_prev), _f32(out),
                             _stream()))
    return out


def gru_adjoint_step_rows(cfg, p, gamma, gi_rows, h_lin, mu, out=None, ws=None):
    """out[n,B,H] = (dPhi_gamma/dh at (gi_rows, h_lin))^T mu: the adjoint of gru_step_rows, row by row."""
    n = mu.shape[0]
    out = torch.empty_like(mu) if out is None else out
    ws = _ws(5 * n * cfg.B * cfg.H * 4 + 5 * 256, ws, mu.device)
    _check(lib.gru_adjoint_step_rows(ctypes.byref(cfg), ctypes.byref(_params(p)), n, float(gamma), _f32(gi_rows), _f32(h_lin),
                                     _f32(mu), _f32(out), _ptr(ws), ws.numel(), _stream()))
    return out


def stack_workspace_bytes(cfg: Cfg, n_layers: int):
    f, a = _sz(0), _sz(0)
    _check(lib.mgrit_gru_stack_workspace_bytes(ctypes.byref(cfg), n_layers, ctypes.byref(f), ctypes.byref(a)))
    return f.value, a.value


def _param_array(layers):
    arr = (_Params * len(layers))()
    for k, p in enumerate(layers):
        arr[k] = _params(p)
    return arr


def mgrit_gru_stack_forward(cfg, layers, x, h0, want_resnorm=False, ws=None):
    """All layers in one state, one MGRIT cycle for the stack.  layers: list of parameter dicts; h0[n_layers,B,H].
    -> (h[T,n_layers,B,H], gi0[T,B,3H], resnorm list or None)"""
    dev, nl = x.device, len(layers)
    gi0 = torch.empty(cfg.T, cfg.B, 3 * cfg.H, device=dev)
    h = torch.empty(cfg.T, nl, cfg.B, cfg.H, device=dev)
    ws = _ws(stack_workspace_bytes(cfg, nl)[0], ws, dev)
    rn = (ctypes.c_float * max(cfg.iters, 1))() if want_resnorm else None
    _check(lib.mgrit_gru_stack_forward(ctypes.byref(cfg), nl, _param_array(layers), _f32(x), _f32(h0), _f32(gi0), _f32(h), rn,
                                       _ptr(ws), ws.numel(), _stream()))
    return h, gi0, (list(rn)[:cfg.iters] if want_resnorm else None)


def mgrit_gru_stack_adjoint(cfg, layers, x, h0, gi0, h, dh_seed=None, dhT=None, want_dx=True, want_dh=True, want_resnorm=False, ws=None):
    """-> (dh[T,n_layers,B,H] or None, dh0[n_layers,B,H], dx or None, list of per-layer AdjointResult (gradients only), resnorm)"""
    dev, nl = x.device, len(layers)
    dh = torch.empty(cfg.T, nl, cfg.B, cfg.H, device=dev) if want_dh else None
    dh0 = torch.empty(nl, cfg.B, cfg.H, device=dev)
    dx = torch.empty(cfg.T, cfg.B, cfg.I, device=dev) if want_dx else None
    outs, garr = [], (_Grads * nl)()
    for k in range(nl):
        Ik = cfg.I if k == 0 else cfg.H
        o = AdjointResult(dh=None, dh0=None, dx=None, dW_ih=torch.empty(3 * cfg.H, Ik, device=dev), dW_hh=torch.empty(3 * cfg.H, cfg.H, device=dev),
                          db_ih=torch.empty(3 * cfg.H, device=dev), db_hh=torch.empty(3 * cfg.H, device=dev))
        garr[k] = _Grads(o.dW_ih.data_ptr(), o.dW_hh.data_ptr(), o.db_ih.data_ptr(), o.db_hh.data_ptr())
        outs.append(o)
    ws = _ws(stack_workspace_bytes(cfg, nl)[1], ws, dev)
    rn = (ctypes.c_float * max(cfg.iters, 1))() if want_resnorm else None
    _check(lib.mgrit_gru_stack_adjoint(ctypes.byref(cfg), nl, _param_array(layers), _f32(x), _f32(h0), _f32(gi0), _f32(h), _f32(dh_seed),
                                       _f32(dhT), _f32(dh), _f32(dh0), _f32(dx), garr, rn, _ptr(ws), ws.numel(), _stream()))
    return dh, dh0, dx, outs, (list(rn)[:cfg.iters] if want_resnorm else None)


def lstm_workspace_bytes(cfg: Cfg):
    f, a = _sz(0), _sz(0)
    _check(lib.mgrit_lstm_workspace_bytes(ctypes.byref(cfg), ctypes.byref(f), ctypes.byref(a)))
    return f.value, a.value


def mgrit_lstm_forward(cfg, p, x, u0, want_resnorm=False, ws=None):
    """Implicit LSTM by MGRIT.  p: dict W_ih[4H,I], W_hh[4H,H], b_ih, b_hh; u0[2,B,H] = (c_0, h_0).
    -> (u[T,2,B,H], gi[T,B,4H], resnorm list or None)"""
    dev = x.device
    gi = torch.empty(cfg.T, cfg.B, 4 * cfg.H, device=dev)
    u = torch.empty(cfg.T, 2, cfg.B, cfg.H, device=dev)
    ws = _ws(lstm_workspace_bytes(cfg)[0], ws, dev)
    rn = (ctypes.c_float * max(cfg.iters, 1))() if want_resnorm else None
    _check(lib.mgrit_lstm_forward(ctypes.byref(cfg), ctypes.byref(_params(p)), _f32(x), _f32(u0), _f32(gi), _f32(u), rn, _ptr(ws),
                                  ws.numel(), _stream()))
    return u, gi, (list(rn)[:cfg.iters] if want_resnorm else None)


def mgrit_lstm_adjoint(cfg, p, x, u0, gi, u, du_seed=None, dhT=None, want_dx=True, want_du=True, want_resnorm=False, ws=None):
    """-> (du[T,2,B,H] or None, du0[2,B,H], AdjointResult with dx and the 4H-row gradients, resnorm)"""
    dev = x.device
    du = torch.empty(cfg.T, 2, cfg.B, cfg.H, device=dev) if want_du else None
    du0 = torch.empty(2, cfg.B, cfg.H, device=dev)
    o = AdjointResult(dh=None, dh0=None, dx=torch.empty(cfg.T, cfg.B, cfg.I, device=dev) if want_dx else None,
                      dW_ih=torch.empty(4 * cfg.H, cfg.I, device=dev), dW_hh=torch.empty(4 * cfg.H, cfg.H, device=dev),
                      db_ih=torch.empty(4 * cfg.H, device=dev), db_hh=torch.empty(4 * cfg.H, device=dev))
    g = _Grads(o.dW_ih.data_ptr(), o.dW_hh.data_ptr(), o.db_ih.data_ptr(), o.db_hh.data_ptr())
    ws = _ws(lstm_workspace_bytes(cfg)[1], ws, dev)
    rn = (ctypes.c_float * max(cfg.iters, 1))() if want_resnorm else None
    _check(lib.mgrit_lstm_adjoint(ctypes.byref(cfg), ctypes.byref(_params(p)), _f32(x), _f32(u0), _f32(gi), _f32(u), _f32(du_seed),
                                  _f32(dhT), _f32(du), _f32(du0), _f32(o.dx), ctypes.byref(g), rn, _ptr(ws), ws.numel(), _stream()))
    return du, du0, o, (list(rn)[:cfg.iters] if want_resnorm else None)


def xent_head_fwd_bwd(hT, Wc, bc, labels, ws=None):
    """-> (loss[1], dhT[B,H], dWc[C,H], dbc[C]) device tensors"""
    B, H = hT.shape
    C = Wc.shape[0]
    dev = hT.device
    assert labels.dtype == torch.int32
    loss = torch.empty(1, device=dev)
    dhT, dWc, dbc = torch.empty(B, H, device=dev), torch.empty(C, H, device=dev), torch.empty(C, device=dev)
    ws = _ws(lib.xent_head_workspace_bytes(B, C), ws, dev)
    _check(lib.xent_head_fwd_bwd(B, H, C, _f32(hT), _f32(Wc), _f32(bc), _ptr(labels), _f32(loss), _f32(dhT), _f32(dWc),
                                 _f32(dbc), _ptr(ws), ws.numel(), _stream()))
    return loss, dhT, dWc, dbc


def xent_head_fwd_bwd_noalloc(hT, Wc, bc, labels, out=None):
    """Loss head for callers that must not allocate device memory inside the call: the library's built-in
    scratch replaces the workspace (B*C <= 65536).  `out` = (loss[1], dhT[B,H], dWc[C,H], dbc[C]) preallocated
    by the caller; when omitted this convenience wrapper allocates the four outputs with torch before the call.
    Calls share one scratch array: do not overlap them on the GPU."""
    B, H = hT.shape
    C = Wc.shape[0]
    dev = hT.device
    assert labels.dtype == torch.int32
    if out is None:
        out = (torch.empty(1, device=dev), torch.empty(B, H, device=dev), torch.empty(C, H, device=dev), torch.empty(C, device=dev))
    loss, dhT, dWc, dbc = out
    _check(lib.xent_head_fwd_bwd_noalloc(B, H, C, _f32(hT), _f32(Wc), _f32(bc), _ptr(labels), _f32(loss), _f32(dhT), _f32(dWc),
                                         _f32(dbc), _stream()))
    return loss, dhT, dWc, dbc


# ---- linear recurrences, token probabilities, distillation: arrays of fp32, bf16 or fp16, any strides with contiguous rows ----------

def _require(ok, what, *args):
    if not ok:
        raise ValueError(what.format(*args))


def _int32(*sizes):
    """Sizes as they are, refused beyond 32 bits (ctypes would cut them off)."""
    for n in sizes:
        if not -2 ** 31 <= n < 2 ** 31:
            raise ValueError(f"a size of {n}: at most 2^31 - 1")
    return sizes


def _dtype(t):
    code = _DTYPES.get(t.dtype)
    _require(code is not None, "fp32, bf16 or fp16 required, got {}", t.dtype)
    return code


# the current stream's handle and the current device without the objects around them (7 us of a call that takes 12)
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_device_now = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _run(dev, fn, *args):
    """fn(*args, stream) on the current stream of `dev`, whatever device is current."""
    if _device_now() == dev.index:
        rc = fn(*args, _stream_of(dev.index))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _stream_of(dev.index))
    if rc != OK:
        raise MgritError(rc)


def _like(t, dev, shape, dtype, name):
    """Address of a contiguous array of that device, shape and type (0: not given)."""
    if t is None:
        return 0
    if not (t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.device == dev):
        raise ValueError(f"{name}: contiguous {dtype} array of shape {tuple(shape)} on {dev} required")
    return t.data_ptr()


def _strided(t, shape, dtype, dev, name):
    """(address, stride of t, stride of b) of an array of that shape, type and device with contiguous units."""
    if t is None:
        return 0, 0, 0
    if t.shape == shape and t.dtype is dtype and t.device == dev:
        st, sb, su = t.stride()
        if su == 1 or shape[2] == 1:
            return t.data_ptr(), st, sb
    raise ValueError(f"{name}: {dtype} array of shape {tuple(shape)} on {dev} with contiguous units required")


_SCAN_ARGS = struct.Struct("@5if" + 3 * "Pqq" + "Pqq" + "PPP" + "Pqq" + "P" + 2 * "Pqq" + "P")      # gated_scan_args
_scan_ws_bytes = functools.lru_cache(maxsize=4096)(lib.gated_scan_workspace_bytes)      # (of the sizes alone)


def _scan_head(gate, cand, h, reset, lengths, h0, cell, dt, shape, dev):
    """The fields of gated_scan_args that both calls have; h: its (address, strides)."""
    t = gate.dtype
    if reset is None:
        r = (0, 0, 0)
    else:
        _require(reset.dtype in (torch.uint8, torch.bool) and reset.shape == shape[:2] and reset.device == dev, "reset: uint8 or bool array [T,B] on {} required", dev)
        r = (reset.data_ptr(), *reset.stride())
    return (*shape, cell, _dtype(gate), dt, *_strided(gate, shape, t, dev, "gate"), *_strided(cand, shape, t, dev, "cand"), *h, *r,
            0 if h0 is None else _like(h0, dev, shape[1:], torch.float32, "h0"), 0 if lengths is None else _like(lengths, dev, shape[1:2], torch.int32, "lengths"))


def _scan_pack(*fields):
    try:
        return _SCAN_ARGS.pack(*fields)
    except struct.error as e:
        raise ValueError(f"a size or cell out of range: {e}") from None


def _scan_call(fn, packed, shape, ws, dev):
    n = _scan_ws_bytes(*shape)
    if n == 0:
        return _run(dev, fn, packed, None, 0)
    if ws is None or ws.numel() < n:
        ws = torch.empty(n, dtype=torch.uint8, device=dev)
    _require(ws.device == dev and ws.dtype == torch.uint8 and ws.is_contiguous(), "ws: contiguous uint8 array on {} required", dev)
    _run(dev, fn, packed, ws.data_ptr(), ws.numel())


def gated_scan_forward(gate, cand, h0=None, cell=CELL_IMPLICIT, dt=1.0, lengths=None, reset=None, h=None, hT=None, ws=None):
    """Gated linear recurrence h_t = a_t h_{t-1} + b_t over gate[T,B,H] and cand[T,B,H] (fp32, bf16 or fp16; any strides with contiguous
    units, so time-major or batch-major arrays and halves of one projection serve) -> (h[T,B,H] of the same type, hT[B,H] fp32).
    cell: CELL_CLASSIC, CELL_IMPLICIT (a, b from sigmoid(gate) and tanh(cand)) or SCAN_COEFFICIENTS (a = gate, b = cand).
    h0[B,H] fp32; lengths[B] int32; reset[T,B] uint8 or bool: the sequence starts anew there.  hT may be h0: one call with T = 1 is a step
    of generation that updates the state in place.  Behind a sequence's end h is zero and hT keeps the state."""
    _require(gate.dim() == 3 and gate.is_cuda, "gate: CUDA array [T,B,H] required")
    shape, dev = gate.shape, gate.device
    if h is None:
        h = gate.new_empty(shape)
        rows = (h.data_ptr(), shape[1] * shape[2], shape[2])
    else:
        rows = _strided(h, shape, gate.dtype, dev, "h")
    if hT is None:
        hT = gate.new_empty(shape[1:], dtype=torch.float32)
        last = hT.data_ptr()
    else:
        last = _like(hT, dev, shape[1:], torch.float32, "hT")
    packed = _scan_pack(*_scan_head(gate, cand, rows, reset, lengths, h0, cell, dt, shape, dev), last, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    _scan_call(lib.gated_scan_forward, packed, shape, ws, dev)
    return h, hT


def gated_scan_backward(gate, cand, h, h0=None, dh_seed=None, dhT=None, cell=CELL_IMPLICIT, dt=1.0, lengths=None, reset=None, dgate=None,
                        dcand=None, dh0=None, ws=None):
    """Gradients of gated_scan_forward at its states h, given dh_seed[T,B,H] (w.r.t. every h_t) and / or dhT[B,H] (w.r.t. hT)
    -> (dgate, dcand, dh0[B,H] fp32)."""
    _require(gate.dim() == 3 and gate.is_cuda, "gate: CUDA array [T,B,H] required")
    shape, dev, t = gate.shape, gate.device, gate.dtype
    dgate = gate.new_empty(shape) if dgate is None else dgate
    dcand = gate.new_empty(shape) if dcand is None else dcand
    dh0 = gate.new_empty(shape[1:], dtype=torch.float32) if dh0 is None else dh0
    packed = _scan_pack(*_scan_head(gate, cand, _strided(h, shape, t, dev, "h"), reset, lengths, h0, cell, dt, shape, dev), 0,
                             *_strided(dh_seed, shape, t, dev, "dh_seed"), _like(dhT, dev, shape[1:], torch.float32, "dhT"),
                             *_strided(dgate, shape, t, dev, "dgate"), *_strided(dcand, shape, t, dev, "dcand"), _like(dh0, dev, shape[1:], torch.float32, "dh0"))
    _scan_call(lib.gated_scan_backward, packed, shape, ws, dev)
    return dgate, dcand, dh0


@dataclass
class TokenLogprobs:
    logprob: torch.Tensor | None
    entropy: torch.Tensor
    lse: torch.Tensor
    top_logprob: torch.Tensor | None
    top_id: torch.Tensor | None


def _logit_rows(t, name, like=None):
    """(address, elements from row to row) of a matrix of logits with contiguous rows."""
    if t.dim() != 2 or not t.is_cuda or (like is not None and not (t.shape == like.shape and t.dtype is like.dtype and t.device == like.device)):
        raise ValueError(f"{name}: CUDA matrix [N,V] required" + ("" if like is None else ", of the logits' shape, type and device"))
    ld, one = t.stride()
    _require(one == 1 or t.shape[1] == 1, "{}: the elements of a row must be contiguous", name)
    return t.data_ptr(), ld


def token_logprobs(logits, tokens=None, top=0, out=None):
    """Log probabilities of tokens[N] (int32) under the rows of logits[N,V] (fp32, bf16 or fp16), the entropy and the log of the sum of
    exponentials of each row, and its `top` most probable tokens (equal logits: the lower token first; top <= 128)
    -> TokenLogprobs of fp32 arrays (top_id int32).  `out`: a TokenLogprobs of an earlier call of the same sizes, to be overwritten."""
    p, ld = _logit_rows(logits, "logits")
    shape, dev, f32 = logits.shape, logits.device, torch.float32
    N, V, top = _int32(*shape, top)
    if out is None:
        each, ent, lse = logits.new_empty((3, N), dtype=f32).unbind()
        out = TokenLogprobs(None if tokens is None else each, ent, lse, logits.new_empty((N, top), dtype=f32) if top > 0 else None,
                            logits.new_empty((N, top), dtype=torch.int32) if top > 0 else None)
        q = each.data_ptr()
        to = (q if tokens is not None else 0, q + 4 * N, q + 8 * N, out.top_logprob.data_ptr() if top > 0 else 0, out.top_id.data_ptr() if top > 0 else 0)
    else:
        rows = shape[:1]
        to = (_like(out.logprob, dev, rows, f32, "logprob"), _like(out.entropy, dev, rows, f32, "entropy"), _like(out.lse, dev, rows, f32, "lse"),
              _like(out.top_logprob, dev, (N, top), f32, "top_logprob"), _like(out.top_id, dev, (N, top), torch.int32, "top_id"))
    _run(dev, lib.token_logprobs, N, V, _dtype(logits), p, ld, 0 if tokens is None else _like(tokens, dev, shape[:1], torch.int32, "tokens"), top, *to)
    return out


def token_logprobs_backward(logits, tokens, lse, entropy=None, dlogprob=None, dentropy=None, dlogits=None):
    """Gradient w.r.t. the logits, given those w.r.t. the tokens' log probabilities and / or the entropies and the statistics that the
    forward call returned.  dlogits may be the logits themselves (in place).  -> dlogits[N,V]"""
    p, ld = _logit_rows(logits, "logits")
    (N, V), dev, f32 = _int32(*logits.shape), logits.device, torch.float32
    rows = logits.shape[:1]
    dlogits = logits.new_empty((N, V)) if dlogits is None else dlogits
    d, dld = _logit_rows(dlogits, "dlogits", logits)
    _run(dev, lib.token_logprobs_backward, N, V, _dtype(logits), p, ld, _like(tokens, dev, rows, torch.int32, "tokens") if dlogprob is not None else 0,
         _like(lse, dev, rows, f32, "lse"), _like(entropy, dev, rows, f32, "entropy") if dentropy is not None else 0,
         _like(dlogprob, dev, rows, f32, "dlogprob"), _like(dentropy, dev, rows, f32, "dentropy"), d, dld)
    return dlogits


def distill_topk_fwd_bwd(logits, top_id, top_logit, weight=None, temperature=1.0, dlogits=None, loss=None, row_loss=None):
    """Distillation of the rows of logits[N,V] from a teacher's top_id[N,K] (int32) and top_logit[N,K] (logits or log probabilities, as
    token_logprobs returns them): -> (loss[1], row_loss[N], dlogits[N,V]).  weight[N]: of the rows (the mean without it).
    dlogits may be the logits themselves (in place)."""
    p, ld = _logit_rows(logits, "logits")
    _require(top_id.dim() == 2, "top_id: matrix [N,K] required")
    (N, V, K), dev, f32 = _int32(*logits.shape, top_id.shape[1]), logits.device, torch.float32
    rows = logits.shape[:1]
    if dlogits is None:
        dlogits = logits.new_empty((N, V))
        d, dld = dlogits.data_ptr(), V
    else:
        d, dld = _logit_rows(dlogits, "dlogits", logits)
    # (one array for both: loss first)
    if loss is None and row_loss is None:
        loss, row_loss = logits.new_empty(N + 1, dtype=f32).split_with_sizes((1, N))
        one = loss.data_ptr()
        each = one + 4
    else:
        loss = logits.new_empty(1, dtype=f32) if loss is None else loss
        row_loss = logits.new_empty(rows, dtype=f32) if row_loss is None else row_loss
        one, each = _like(loss, dev, (1,), f32, "loss"), _like(row_loss, dev, rows, f32, "row_loss")
    _run(dev, lib.distill_topk_fwd_bwd, N, V, K, _dtype(logits), temperature, p, ld, _like(top_id, dev, (N, K), torch.int32, "top_id"),
         _like(top_logit, dev, (N, K), f32, "top_logit"), _like(weight, dev, rows, f32, "weight"), one, each, d, dld)
    return loss, row_loss, dlogits


def sgd_update(p, g, lr):
    _check(lib.sgd_update(_f32(p), _f32(g), p.numel(), ctypes.c_float(lr), _stream()))
    return p


def adam_update(p, g, m, v, lr, step, beta1=0.9, beta2=0.999, eps=1e-8):
    _check(lib.adam_update(_f32(p), _f32(g), _f32(m), _f32(v), p.numel(), ctypes.c_float(lr), ctypes.c_float(beta1),
                           ctypes.c_float(beta2), ctypes.c_float(eps), int(step), _stream()))
    return p


def last_device_status() -> int:
    return lib.mgrit_gru_last_device_status()


def clear_device_status() -> None:
    _check(lib.mgrit_gru_clear_device_status())


def selftest_bounded_wait(limit_ms: int = 20) -> None:
    """Launch the library's wait self-test: a bounded wait that runs out and records MGRIT_DEVICE_TIMEOUT."""
    _check(lib.mgrit_gru_selftest_bounded_wait(limit_ms, _stream()))


def kernel_launches() -> int:
    return int(lib.mgrit_gru_kernel_launches())


KERNEL_CLASSES = ("input_projection", "forward_step", "adjoint_linearise", "adjoint_step", "gradient_gemms",
                  "forward_serial_chain", "adjoint_serial_chain")


def profile_enable(on: bool) -> None:
    _check(lib.mgrit_gru_profile_enable(1 if on else 0))


def profile_records():
    """-> list of (class name, ms, flops) per recorded launch, in launch order."""
    n = _sz(0)
    _check(lib.mgrit_gru_profile_records(None, None, None, 0, ctypes.byref(n)))
    cap = n.value
    ms, fl, kc = (ctypes.c_double * cap)(), (ctypes.c_double * cap)(), (ctypes.c_int32 * cap)()
    _check(lib.mgrit_gru_profile_records(ms, fl, kc, cap, ctypes.byref(n)))
    return [(KERNEL_CLASSES[kc[i]], ms[i], fl[i]) for i in range(cap)]


def profile_read():
    """-> {class name: (total ms, launches, algorithmic flops)} for the launches recorded since profile_enable(True)."""
    out = {}
    for i, name in enumerate(KERNEL_CLASSES):
        ms, n, fl = ctypes.c_double(0), ctypes.c_ulonglong(0), ctypes.c_double(0)
        _check(lib.mgrit_gru_profile_read(i, ctypes.byref(ms), ctypes.byref(n), ctypes.byref(fl)))
        out[name] = (ms.value, int(n.value), fl.value)
    return out
