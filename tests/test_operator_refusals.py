"""What the operators over given arrays refuse, answered on the host before any device is touched: the C ABI by its error codes, the
binding by ValueError.  The addresses passed here are never read."""
import ctypes

import pytest
import torch

P = 1 << 20            # an aligned address that nothing reads
INVALID, UNSUPPORTED, SMALL, CUDA = -1, -4, -3, -5


@pytest.fixture(scope="module")
def L():
    from paper_2203_04738_b200.build import build
    build()
    from paper_2203_04738_b200 import binding
    return binding


FIELDS = ("T", "B", "H", "cell", "dtype", "dt", "gate", "gts", "gbs", "cand", "cts", "cbs", "h", "hts", "hbs", "reset", "rts", "rbs", "h0", "lengths", "hT", "seed", "sts",
          "sbs", "dhT", "dgate", "dgts", "dgbs", "dcand", "dcts", "dcbs", "dh0")


def scan_args(L, **kw):
    T, B, H = kw.get("T", 10), kw.get("B", 2), kw.get("H", 16)
    v = dict(T=T, B=B, H=H, cell=1, dtype=0, dt=1.0, reset=0, rts=0, rbs=0, h0=P, lengths=0, hT=P, seed=P, dhT=P, dgate=P, dcand=P, dh0=P, gate=P, cand=P, h=P)
    v.update({k + e: s for k in ("g", "c", "h", "s", "dg", "dc") for e, s in (("ts", B * H), ("bs", H))})
    v.update(kw)
    return L._SCAN_ARGS.pack(*[v[f] for f in FIELDS])


BAD_SCAN = [(dict(T=-1), INVALID), (dict(B=-1), INVALID), (dict(H=0), INVALID), (dict(cell=3), INVALID), (dict(cell=-1), INVALID), (dict(dtype=3), INVALID),
            (dict(dt=-1.0), INVALID), (dict(dt=float("nan")), INVALID), (dict(dt=float("inf")), INVALID), (dict(gate=0), INVALID), (dict(cand=0), INVALID),
            (dict(h=0), INVALID), (dict(gate=P + 2), INVALID), (dict(dtype=1, cand=P + 1), INVALID), (dict(h0=P + 2), INVALID), (dict(lengths=P + 1), INVALID),
            (dict(B=1 << 20, H=1 << 11), UNSUPPORTED), (dict(T=2 ** 31 - 1), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", BAD_SCAN)
def test_scan_refusals(L, kw, code):
    for fn in (L.lib.gated_scan_forward, L.lib.gated_scan_backward):
        assert fn(scan_args(L, **kw), P, 1 << 40, None) == code, kw


def test_scan_refusals_of_one_direction(L):
    fwd, bwd = (lambda **kw: L.lib.gated_scan_forward(scan_args(L, **kw), P, 1 << 40, None)), (lambda **kw: L.lib.gated_scan_backward(scan_args(L, **kw), P, 1 << 40, None))
    assert fwd(hT=P + 2) == INVALID
    for ts, bs in ((0, 16), (32, 0), (32, 15), (31, 16), (16, 32), (16, 159)):         # rows of the output would overlap
        assert fwd(hts=ts, hbs=bs) == INVALID and bwd(dgts=ts, dgbs=bs) == INVALID and bwd(dcts=ts, dcbs=bs) == INVALID
    assert bwd(seed=0, dhT=0) == INVALID and bwd(dgate=0) == INVALID and bwd(dcand=0) == INVALID
    assert bwd(seed=P + 1) == INVALID and bwd(dhT=P + 1) == INVALID and bwd(dh0=P + 2) == INVALID and bwd(dgate=P + 3) == INVALID
    assert L.lib.gated_scan_forward(None, P, 1 << 40, None) == INVALID and L.lib.gated_scan_backward(None, P, 1 << 40, None) == INVALID


def test_scan_workspace_is_checked(L):
    n = L.lib.gated_scan_workspace_bytes(100000, 2, 16)
    a = scan_args(L, T=100000, h=P)
    if n > 0:
        assert L.lib.gated_scan_forward(a, P, n - 1, None) == SMALL and L.lib.gated_scan_backward(a, P, n - 1, None) == SMALL
        assert L.lib.gated_scan_forward(a, 0, n, None) == INVALID and L.lib.gated_scan_forward(a, P + 4, n, None) == INVALID
    assert L.lib.gated_scan_workspace_bytes(1, 32, 1024) == 0
    assert L.lib.gated_scan_workspace_bytes(-1, 32, 1024) == 0 and L.lib.gated_scan_workspace_bytes(10, 0, 4) == 0
    assert L.lib.gated_scan_workspace_bytes(2 ** 31 - 1, 1, 4) == 0


def logprob(L, **kw):
    v = dict(N=4, V=100, dtype=0, logits=P, ld=100, tokens=P, top=5, logprob=P, entropy=P, lse=P, tl=P, ti=P)
    v.update(kw)
    return L.lib.token_logprobs(*v.values(), None)


def logprob_back(L, **kw):
    v = dict(N=4, V=100, dtype=0, logits=P, ld=100, tokens=P, lse=P, entropy=P, dl=P, de=P, d=2 * P, dld=100)
    v.update(kw)
    return L.lib.token_logprobs_backward(*v.values(), None)


def distill(L, **kw):
    v = dict(N=4, V=100, K=5, dtype=0, tau=1.0, logits=P, ld=100, ids=P, y=P, w=P, loss=P, row=P, d=2 * P, dld=100)
    v.update(kw)
    return L.lib.distill_topk_fwd_bwd(*v.values(), None)


@pytest.mark.parametrize("call", [logprob, logprob_back, distill])
def test_row_refusals(L, call):
    for kw in (dict(N=-1), dict(V=0), dict(V=-3), dict(dtype=-1), dict(dtype=3), dict(logits=0), dict(logits=P + 2), dict(dtype=2, logits=P + 1), dict(ld=99), dict(ld=-100)):
        assert call(L, **kw) == INVALID, kw


def test_logprob_refusals(L):
    for kw in (dict(top=-1), dict(top=101), dict(tl=0), dict(ti=0), dict(logprob=0), dict(tokens=P + 2), dict(lse=P + 1), dict(entropy=P + 2), dict(ti=P + 3)):
        assert logprob(L, **kw) == INVALID, kw
    assert logprob(L, V=1000, ld=1000, top=129) == UNSUPPORTED
    assert logprob(L, N=0, logits=0, tokens=0, logprob=0, tl=0, ti=0) == 0
    for kw in (dict(lse=0), dict(tokens=0), dict(dl=0), dict(entropy=0), dict(de=0), dict(tokens=0, dl=0, entropy=0, de=0), dict(d=0), dict(d=P + 1), dict(dld=99),
               dict(d=P, ld=100, dld=101), dict(lse=P + 2)):
        assert logprob_back(L, **kw) == INVALID, kw
    assert logprob_back(L, N=0, logits=0, d=0) == 0


def test_distill_refusals(L):
    for kw in (dict(K=0), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")), dict(tau=float("inf")), dict(tau=1e-39), dict(ids=0), dict(y=0), dict(loss=0), dict(row=0),
               dict(d=0), dict(dld=50), dict(d=P, dld=101), dict(ids=P + 2), dict(y=P + 1), dict(w=P + 2), dict(loss=P + 2), dict(row=P + 3)):
        assert distill(L, **kw) == INVALID, kw
    assert distill(L, K=1025) == UNSUPPORTED


def test_the_binding_refuses_arrays_that_it_cannot_pass_on(L):
    x = torch.zeros(3, 2, 8)
    for fn in (lambda: L.gated_scan_forward(x, x), lambda: L.gated_scan_backward(x, x, x, dh_seed=x), lambda: L.token_logprobs(x[0]),
               lambda: L.token_logprobs_backward(x[0], None, x[0, :, 0]), lambda: L.distill_topk_fwd_bwd(x[0], x[0].int(), x[0]), lambda: L.gated_scan_forward(x[0], x[0])):
        with pytest.raises(ValueError):
            fn()


def test_a_sound_call_without_a_device_is_an_error_not_a_crash(L):
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    assert logprob(L) == CUDA and logprob_back(L) == CUDA and distill(L) == CUDA
    assert L.lib.gated_scan_forward(scan_args(L), P, 1 << 30, None) == CUDA


def test_distill_refuses_temperatures_whose_inverse_is_out_of_range(L):
    for tau in (4e-39, 1e-44, 3.2e38):
        assert distill(L, tau=tau) == INVALID, tau


def test_scan_refuses_columns_by_their_padded_width(L):
    """More than 8 steps are taken by whole threads of columns, 4 of a 16-bit type or 2 of fp32."""
    for kw in (dict(T=9, B=1 << 29, H=1, dtype=1), dict(T=9, B=1 << 29, H=3, dtype=2), dict(T=64, B=1 << 30, H=1, dtype=0), dict(T=9, B=(1 << 27) + 1, H=13, dtype=1)):
        for fn in (L.lib.gated_scan_forward, L.lib.gated_scan_backward):
            assert fn(scan_args(L, **kw), P, 1 << 62, None) == UNSUPPORTED, kw


def test_gradients_of_more_pieces_than_a_grid_has_blocks_are_refused(L):
    assert logprob_back(L, N=(1 << 27) - 1, V=1 << 20, ld=1 << 20, dld=1 << 20) == UNSUPPORTED
