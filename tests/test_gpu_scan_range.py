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


def growing(name, T, B, H, rng):
    """Coefficients whose products leave fp32's range while no state does -> a[T,B,H], b[T,B,H], h0[B,H]."""
    one = np.ones((T, B, H))
    a, b, h0 = 0.9 * one, np.zeros((T, B, H)), np.zeros((B, H))
    if name == "nothing grows":                # zero states, until the last steps
        a, b[-5:] = 3.0 * one, rng.standard_normal((5, B, H))
    elif name == "growth, then a zero":        # the product overflows, then a zero cuts
        a = 3.0 * one
        a[T // 2] = 0.0
        a[T // 2 + 1:] = 0.5
        b[T // 2:] = rng.standard_normal((T - T // 2, B, H))
    elif name == "up and down":                # 2^200 within ten steps, and back
        a = np.where((np.arange(T) // 10 % 2 == 0)[:, None, None], 2.0 ** 20, 2.0 ** -20) * one
        h0 = 2.0 ** -100 * rng.standard_normal((B, H))
    elif name == "down and up":
        a = np.where((np.arange(T) // 10 % 2 == 0)[:, None, None], 2.0 ** -20, 2.0 ** 20) * one
        h0 = 2.0 ** 100 * rng.standard_normal((B, H))
    elif name == "slow growth":                # 1.25^T over several tiles, signs of both kinds
        a = 1.25 * np.where(rng.random((T, B, H)) < 0.5, -1.0, 1.0)
        h0 = 2.0 ** (-0.32 * T) * rng.standard_normal((B, H))
    elif name == "an infinite state":          # decays do not make it finite
        a = np.where(rng.random((T, B, H)) < 0.5, -0.05, 0.05)
        b = rng.standard_normal((T, B, H))
        h0 = np.where(rng.random((B, H)) < 0.3, np.inf, rng.standard_normal((B, H)))
    return a, b, h0


@pytest.mark.parametrize("name", ["nothing grows", "growth, then a zero", "up and down", "down and up", "slow growth", "an infinite state"])
@pytest.mark.parametrize("T,B,H", [(150, 1, 8), (300, 2, 33), (300, 9, 128), (260, 5, 27)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products_that_leave_the_range_where_no_state_does(name, T, B, H, dtype):
    """Forward and backward against 64 bits, with all columns of that kind and with some among ordinary ones, whose bits stay what they are."""
    from paper_2203_04738_b200 import binding as L
    rng = np.random.default_rng(T * H)
    a, b, h0 = growing(name, T, B, H, rng)
    plain = (0.5 + 0.4 * rng.random((T, B, H)), rng.standard_normal((T, B, H)), rng.standard_normal((B, H)))
    some = rng.random((B, H)) < 0.1
    ordinary = torch.from_numpy(~some).cuda()
    hs = dev(rng.standard_normal((T, B, H)), dtype)
    reset = dev((rng.random((T, B)) < 0.01).astype(np.uint8), torch.uint8)
    lengths = dev(rng.integers(T // 2, T + 1, B).astype(np.int32), torch.int32)
    bits = {}
    for kind in ("plain", "all", "some"):
        pick = lambda x, y: {"plain": y, "all": x, "some": np.where(some, x, y)}[kind]
        ga, cb, s0 = dev(pick(a, plain[0]), dtype), dev(pick(b, plain[1]), dtype), dev(pick(h0, plain[2]))
        for rs, ln in ((None, None), (torch.zeros_like(reset), None), (reset, lengths)):
            kw = dict(cell=R.GIVEN, reset=rs, lengths=ln)
            # every sequence the other way round for the backward pass: the derivative meets the coefficients in the order of the forward pass
            gr, sd = ga.flip(0), cb.flip(0)
            for i in range(B if ln is not None else 0):
                k = int(ln[i])
                gr[:k, i], sd[:k, i] = ga[:k, i].flip(0), cb[:k, i].flip(0)
            n = lambda t: None if t is None else t.cpu().numpy()
            h, hT = L.gated_scan_forward(ga, cb, h0=s0, **kw)
            ref, refT, bound, boundT = R.scan_forward(R.to64(ga), R.to64(cb), R.to64(s0), R.GIVEN, 1.0, n(ln), n(rs))
            R.check(h, ref, np.nan_to_num(bound) + R.rounding(np.nan_to_num(ref, posinf=0, neginf=0), dtype), f"{kind} h")
            R.check(hT, refT, np.nan_to_num(boundT), f"{kind} hT")
            g = L.gated_scan_backward(gr, cb, hs, h0=s0 * 0 if name != "an infinite state" else None, dh_seed=sd, dhT=s0, **kw)
            refs, bounds = R.scan_backward(R.to64(gr), R.to64(cb), R.to64(hs), np.zeros((B, H)), R.to64(sd), R.to64(s0), R.GIVEN, 1.0, n(ln), n(rs))
            for what, got, r, bd in zip(("dgate", "dcand", "dh0"), g, refs, bounds):
                R.check(got, r, np.nan_to_num(bd) + (0 if what == "dh0" else R.rounding(np.nan_to_num(r, posinf=0, neginf=0), dtype)), f"{kind} {what}")
            out = [h, hT[None], g[0], g[1], g[2][None]]
            key = (rs is None, ln is None)
            if kind == "plain":
                bits[key] = out
            elif kind == "some":
                assert all(torch.equal(p[:, ordinary], q[:, ordinary]) for p, q in zip(out, bits[key]))
    assert L.last_device_status() == 0


def test_a_long_chain_of_growth_and_decay():
    """Every tile of a long sequence has columns without a product that can be handed on: states go from tile to tile."""
    from paper_2203_04738_b200 import binding as L
    T, B, H = 20000, 1, 20
    rng = np.random.default_rng(1)
    a, b, h0 = growing("up and down", T, B, H, rng)
    a[:, :, 1::2] = 0.9
    b[:, :, 1::2] = rng.standard_normal((T, 1, H // 2))
    ga, cb, s0 = dev(a), dev(b), dev(h0)
    ref, refT, bound, boundT = R.scan_forward(a, R.to64(cb), R.to64(s0), R.GIVEN, 1.0)
    first = None
    for _ in range(5):
        h, hT = L.gated_scan_forward(ga, cb, h0=s0, cell=R.GIVEN)
        R.check(h, ref, bound, "h")
        R.check(hT, refT, boundT, "hT")
        assert first is None or torch.equal(h, first)
        first = h


@pytest.mark.parametrize("T,B,H", [(150, 1, 8), (300, 2, 33), (300, 9, 128), (2000, 1, 27)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_the_classic_cell_beyond_two(T, B, H, dtype):
    """dt = 16: coefficients down to -15 while gates are open, over two thirds of the steps without a state to grow; then closed ones, which open
    now and then."""
    from paper_2203_04738_b200 import binding as L
    rng = np.random.default_rng(T)
    n = 2 * T // 3
    gate, cand = rng.uniform(-6, -4, (T, B, H)), np.clip(rng.standard_normal((T, B, H)), -2, 2)
    gate[rng.random((T, B, H)) < 1 / T] = 2.0
    gate[:n], cand[:n] = 4.0, 0.0
    zero = torch.zeros(B, H, device="cuda")
    reset = dev((rng.random((T, B)) < 0.01).astype(np.uint8), torch.uint8)
    lengths = dev(rng.integers(n + 10, T + 1, B).astype(np.int32), torch.int32)
    g, c = dev(gate, dtype), dev(cand, dtype)
    hs = dev(rng.standard_normal((T, B, H)), dtype)
    for rs, ln in ((None, None), (reset, None), (None, lengths), (reset, lengths)):
        m = lambda t: None if t is None else t.cpu().numpy()
        kw = dict(cell=R.CLASSIC, dt=16.0, reset=rs, lengths=ln)
        h, hT = L.gated_scan_forward(g, c, h0=zero, **kw)
        ref, refT, bound, boundT = R.scan_forward(R.to64(g), R.to64(c), R.to64(zero), R.CLASSIC, 16.0, m(ln), m(rs))
        R.check(h, ref, bound + R.rounding(ref, dtype), "h")
        R.check(hT, refT, boundT, "hT")
        # the other way round, without a derivative until the closed gates
        gr, sd = g.flip(0), dev(np.where(np.arange(T)[:, None, None] < T - n, rng.standard_normal((T, B, H)), 0), dtype)
        got = L.gated_scan_backward(gr, c, hs, dh_seed=sd, **kw)
        refs, bounds = R.scan_backward(R.to64(gr), R.to64(c), R.to64(hs), np.zeros((B, H)), R.to64(sd), None, R.CLASSIC, 16.0, m(ln), m(rs))
        for what, x, r, bd in zip(("dgate", "dcand", "dh0"), got, refs, bounds):
            R.check(x, r, bd + (0 if what == "dh0" else R.rounding(r, dtype)), what)
    assert L.last_device_status() == 0
