"""The gated linear recurrence where its coefficients, states and cells leave the middle of their range: products that underflow or overflow,
states that are not finite, saturated gates and candidates, large dt."""
import numpy as np
import pytest
import torch

from tests import operator_refs as R

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def dev(a, t=F32):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(t)


def same_places(x, y):
    """NaN and infinities in the same places."""
    return torch.equal(x.isnan(), y.isnan()) and torch.equal(x.isposinf(), y.isposinf()) and torch.equal(x.isneginf(), y.isneginf())


# one column tile and many, rows at any address, sequences that share a warp
SHAPES = [(400, 1, 40), (400, 3, 33), (300, 40, 256), (700, 24, 17)]


@pytest.mark.parametrize("T,B,H", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("cell,strong", [(R.CLASSIC, 3.0), (R.CLASSIC, 0.0), (R.IMPLICIT, 8.0), (R.GIVEN, 0.01), (R.GIVEN, 0.0)])
def test_what_is_not_finite_stays_in_its_sequence_where_coefficients_are_small(T, B, H, dtype, cell, strong):
    """Steps that forget nearly everything do not forget a NaN or an infinity: it reaches the sequence's last (backward: first) step, whether or
    not a mark says that some other step starts a sequence, and no other column or sequence.  (Implicit cell: dt = 8, a = 1 / 9.)"""
    from paper_2203_04738_b200 import binding as L
    rng = np.random.default_rng(T + H)
    dt = 8.0 if cell == R.IMPLICIT else 1.0
    gate = dev(np.full((T, B, H), strong), dtype)
    cand, h0, dhT = dev(np.clip(rng.standard_normal((T, B, H)), -3, 3), dtype), dev(rng.standard_normal((B, H))), dev(rng.standard_normal((B, H)))
    seed = dev(rng.standard_normal((T, B, H)), dtype)
    col, step = (B - 1, H // 2), 20
    kw = dict(h0=h0, cell=cell, dt=dt)
    other = torch.ones(B, H, dtype=torch.bool, device="cuda")
    other[col] = False
    for bad in (float("nan"), float("inf")):
        x = cand.clone()
        if cell == R.GIVEN or bad != bad:
            x[step][col] = bad
        else:                                  # (a cell's candidate of +inf is a candidate of 1)
            continue
        s = seed.clone()
        s[T - 1 - step][col] = bad
        h, _ = L.gated_scan_forward(gate, cand, **kw)
        for at in (None, T - 40):              # no start, and one far behind the NaN (backward: in front of it)
            reset = torch.zeros(T, B, dtype=torch.uint8, device="cuda")
            back = torch.zeros(T, B, dtype=torch.uint8, device="cuda")
            if at is not None:
                reset[at] = 1
                back[T - at] = 1
            first, last = (at or T), (T - at if at else 0)
            clean, got = (L.gated_scan_forward(gate, v, reset=reset, **kw) for v in (cand, x))
            assert not torch.isfinite(got[0][(slice(step, first), *col)]).any(), "forward"
            assert torch.equal(got[0][:, other], clean[0][:, other]) and torch.equal(got[1][other], clean[1][other])
            assert torch.equal(got[0][:step], clean[0][:step]) and torch.equal(got[0][first:], clean[0][first:])
            assert torch.isfinite(got[1][col]).item() == (at is not None)
            clean, got = (L.gated_scan_backward(gate, cand, h, dh_seed=v, dhT=dhT, reset=back, **kw) for v in (seed, s))
            assert not torch.isfinite(got[1][(slice(last, T - step), *col)]).any(), "backward"
            for p, q in zip(got[:2], clean[:2]):
                assert torch.equal(p[:, other], q[:, other]) and torch.equal(p[:last], q[:last]) and torch.equal(p[T - step:], q[T - step:])
            assert torch.equal(got[2][other], clean[2][other]) and torch.isfinite(got[2][col]).item() == (at is not None)
        # an array of marks without a start: the same places (values may differ by a rounding, which a fused multiply-add saves in one kernel)
        none = torch.zeros(T, B, dtype=torch.uint8, device="cuda")
        for p, q in zip(L.gated_scan_forward(gate, x, reset=none, **kw), L.gated_scan_forward(gate, x, **kw)):
            assert same_places(p, q)
        for p, q in zip(L.gated_scan_backward(gate, cand, h, dh_seed=s, dhT=dhT, reset=none, **kw), L.gated_scan_backward(gate, cand, h, dh_seed=s, dhT=dhT, **kw)):
            assert same_places(p, q)
