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


# Saturated cells.  With E = e^-g the exponential's argument is rounded twice (2 u |g|) and it is off by two units in the last place itself (4 u):
# E is off by (4 + 2.4 |g|) u of itself; a = (L + E) / (K + E) by that and 12 u for its sums, the reciprocal and the products, all in terms of
# (|L| + E) / (K + E), which is a itself where 1 - dt is not negative; q = dt / (K + E) the same.  n by 64 u of itself.  1 - n^2 =
# 4 G / (1 + G)^2 with G = e^-2|c| by (8 + 9.6 |c|) u and 8 u of itself.
U = R.U


def cell64(g, c, cell, dt):
    K, L = (1 + dt, 1.0) if cell == R.IMPLICIT else (1.0, 1 - dt)
    E, G = np.exp(-g), np.exp(-2 * np.abs(c))
    a, pa, q, e = (L + E) / (K + E), (abs(L) + E) / (K + E), dt / (K + E), E / (K + E)
    n, m = np.tanh(c), 4 * G / (1 + G) ** 2
    kg, kc = (16 + 2.4 * np.abs(g)) * U, (16 + 9.6 * np.abs(c)) * U
    return a, pa * kg, q, q * n, np.abs(q * n) * (kg + 64 * U), n, e, m, kg, kc


def check_saturated(T, B, H, dtype, cell, dt, gates, cands, seed, seeds=False, h0=1.0):
    from paper_2203_04738_b200 import binding as L
    rng = np.random.default_rng(seed)
    g, c = dev(rng.uniform(*gates, (T, B, H)), dtype), dev(rng.uniform(*cands, (T, B, H)), dtype)
    s0, dT, sd = dev(h0 * rng.standard_normal((B, H))), dev(rng.standard_normal((B, H))), dev(rng.standard_normal((T, B, H)), dtype) if seeds else None
    h, hT = L.gated_scan_forward(g, c, h0=s0, cell=cell, dt=dt)
    a, da, q, b, db, n, e, m, kg, kc = cell64(R.to64(g), R.to64(c), cell, float(np.float32(dt)))
    tiny = 2.0 ** -120                     # (products and exponentials below the normal numbers)
    s = R.to64(s0)
    S, err = np.abs(s), np.zeros((B, H))
    ref, bound = np.zeros((T, B, H)), np.zeros((T, B, H))
    for t in range(T):
        err = np.abs(a[t]) * err + da[t] * (S + err) + db[t]
        s, S = a[t] * s + b[t], np.abs(a[t]) * S + np.abs(b[t])
        err += 2 * U * S + tiny
        ref[t], bound[t] = s, err + 32 * U * S
    R.check(h, ref, bound + R.rounding(ref, dtype), "h")
    R.check(hT, ref[-1], bound[-1], "hT")
    got = L.gated_scan_backward(g, c, h, h0=s0, dh_seed=sd, dhT=dT, cell=cell, dt=dt)
    prev = np.concatenate((R.to64(s0)[None], R.to64(h)[:-1]))
    mu = R.to64(dT)
    S, err = np.abs(mu), np.zeros((B, H))
    dg, dc, bg, bc = (np.zeros((T, B, H)) for _ in range(4))
    for t in range(T - 1, -1, -1):
        lam = mu + (0 if sd is None else R.to64(sd)[t])
        S = S + (0 if sd is None else np.abs(R.to64(sd)[t]))
        el = err + 34 * U * S
        dg[t], dc[t] = lam * q[t] * e[t] * (n[t] - prev[t]), lam * q[t] * m[t]
        bg[t] = q[t] * e[t] * (el * np.abs(n[t] - prev[t]) + (2 * kg[t] + 64 * U) * S * (np.abs(n[t]) + np.abs(prev[t]))) + tiny
        bc[t] = q[t] * m[t] * (el + (kg[t] + kc[t] + 8 * U) * S) + tiny
        err = np.abs(a[t]) * el + da[t] * (S + el)
        mu, S = a[t] * lam, np.abs(a[t]) * S
        err += 2 * U * S + tiny
    for what, x, r, bd in zip(("dgate", "dcand", "dh0"), got, (dg, dc, mu), (bg, bc, err)):
        R.check(x, r, bd + (0 if what == "dh0" else R.rounding(r, dtype)), what)
    assert L.last_device_status() == 0


RANGE = [(1, 3, 64), (3, 2, 33), (40, 2, 130), (300, 3, 33), (300, 5, 128)]
CELL_DT = [(R.CLASSIC, 0.5), (R.CLASSIC, 1.0), (R.IMPLICIT, 1.0), (R.IMPLICIT, 4.0), (R.IMPLICIT, 64.0), (R.IMPLICIT, 1e4)]


@pytest.mark.parametrize("T,B,H", RANGE)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("cell,dt", CELL_DT[:3])
def test_saturated_candidates_keep_the_digits_of_their_slope(T, B, H, dtype, cell, dt):
    check_saturated(T, B, H, dtype, cell, dt, (-6, 1), (-30, 30), seed=T + H)
    check_saturated(T, B, H, dtype, cell, dt, (-6, 1), (-30, 30), seed=T, seeds=True)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_infinite_candidates_are_candidates_of_one(dtype):
    from paper_2203_04738_b200 import binding as L
    T, B, H = 200, 2, 24
    rng = np.random.default_rng(2)
    gate, h0 = dev(rng.standard_normal((T, B, H)), dtype), dev(rng.standard_normal((B, H)))
    sign = dev(np.where(rng.random((T, B, H)) < 0.5, -1.0, 1.0), dtype)
    for cell in (R.CLASSIC, R.IMPLICIT):
        far, near = (L.gated_scan_forward(gate, sign * x, h0=h0, cell=cell) for x in (float("inf"), 60.0))
        assert torch.equal(far[0], near[0]) and torch.equal(far[1], near[1])
        g = L.gated_scan_backward(gate, sign * float("inf"), far[0], h0=h0, dhT=h0, cell=cell)
        assert not g[1].any() and torch.isfinite(g[0]).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T", [1, 20])
def test_candidates_of_every_size(T, dtype):
    """tanh itself, by b = n of one step (a gate of 100 leaves nothing else).  G = e^-2|c| is off by (4 + 4.8 |c|) u of itself, which 1 - G takes over
    with its full size: at the border to the polynomial by 11 u of n in 16-bit types (|c| = 0.1875), by 6 u in fp32 (0.35).  The reciprocal and the
    other roundings add 6 and 4 u, the reciprocal of the gate 4 u and 1 u, the last products 2 u.  The polynomial: 2 u and three roundings."""
    from paper_2203_04738_b200 import binding as L
    c = np.concatenate([s * np.geomspace(1e-4, 20, 20000) for s in (1, -1)]).reshape(1, 5, 8000)
    cand = dev(np.repeat(c, T, 0), dtype)
    n = np.tanh(R.to64(cand)[-1])
    _, hT = L.gated_scan_forward(torch.full_like(cand, 100.0), cand, cell=R.CLASSIC)
    err = np.abs(R.to64(hT) - n) / np.abs(n)
    assert err.max() <= (13 if dtype == F32 else 23) * U, err.max() / U


@pytest.mark.parametrize("T,B,H", RANGE)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("cell,dt", CELL_DT + [(R.IMPLICIT, 1e8)])
def test_open_gates_keep_the_digits_of_what_they_leave(T, B, H, dtype, cell, dt):
    """a is small where a gate is open or dt is large, and right to its own last digits: with the last state's derivative alone, every gradient is a
    product of such coefficients."""
    check_saturated(T, B, H, dtype, cell, dt, (-6, 30), (-30, 30), seed=T + H)
    check_saturated(T, B, H, dtype, cell, dt, (6, 30), (-3, 3), seed=T, seeds=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_open_gates_of_steps_beyond_one(dtype):
    """dt > 1 turns the classic cell's coefficient negative: a few steps of growing states, or dt = 2, whose coefficients are at most 1 in size."""
    for T, dt in ((1, 64.0), (1, 1e4), (4, 64.0), (8, 4.0), (16, 2.0), (150, 2.0)):
        check_saturated(T, 3, 40, dtype, R.CLASSIC, dt, (-6, 30), (-3, 3), seed=T)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_closed_gates_leave_a_state_as_it_is(dtype):
    """z = e^-35 = 6e-16: a is 1, not a product of roundings near 1, over 20000 steps."""
    from paper_2203_04738_b200 import binding as L
    rng = np.random.default_rng(0)
    h0 = dev(rng.uniform(0.5, 2.0, (1, 40)))
    cand = dev(rng.standard_normal((20000, 1, 40)), dtype)
    for cell in (R.CLASSIC, R.IMPLICIT):
        h, hT = L.gated_scan_forward(torch.full_like(cand, -35.0), cand, h0=h0, cell=cell)
        assert torch.equal(hT, h0)
        assert torch.equal(L.gated_scan_backward(torch.full_like(cand, -35.0), cand, h, h0=h0, dhT=h0, cell=cell)[2], h0)


@pytest.mark.parametrize("T,B,H", RANGE)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("cell,dt", CELL_DT + [(R.IMPLICIT, 1e12), (R.IMPLICIT, 1e18)])
def test_closed_gates_stay_closed_at_any_dt(T, B, H, dtype, cell, dt):
    check_saturated(T, B, H, dtype, cell, dt, (-84, -30), (-30, 30), seed=T + H, h0=1e-6)
    check_saturated(T, B, H, dtype, cell, dt, (-84, 30), (-30, 30), seed=T, seeds=True)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T", [1, 300])
def test_a_gate_of_minus_infinity_keeps_the_state(T, dtype):
    """z counts as e^-86 at least, 4.5e-38: even dt = 1e18 moves a state by no more than 4.5e-20 a step.  A gate of +inf is one of z = 1."""
    from paper_2203_04738_b200 import binding as L
    rng = np.random.default_rng(0)
    h0, inf = dev(rng.uniform(0.5, 2.0, (2, 40))), float("inf")
    cand = dev(rng.standard_normal((T, 2, 40)), dtype)
    for cell in (R.CLASSIC, R.IMPLICIT):
        for dt in (1.0, 1e18):
            h, hT = L.gated_scan_forward(torch.full_like(cand, -inf), cand, h0=h0, cell=cell, dt=dt)
            assert torch.equal(hT, h0)
            g = L.gated_scan_backward(torch.full_like(cand, -inf), cand, h, h0=h0, dhT=h0, cell=cell, dt=dt)
            assert torch.equal(g[2], h0) and g[1].abs().max().item() <= 1e-18
        for a, b in zip(L.gated_scan_forward(torch.full_like(cand, inf), cand, h0=h0, cell=cell), L.gated_scan_forward(torch.full_like(cand, 120.0), cand, h0=h0, cell=cell)):
            assert torch.equal(a, b) and torch.isfinite(a).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("cell,dt", [(R.CLASSIC, 0.5), (R.CLASSIC, 1.0), (R.IMPLICIT, 1.0), (R.IMPLICIT, 8.0), (R.GIVEN, 1.0)])
@pytest.mark.parametrize("T,B,H", [(7, 3, 40), (150, 2, 24), (520, 6, 33), (700, 3, 512)])
def test_scattered_values_that_are_not_finite(T, B, H, cell, dt, dtype):
    """NaN in every input, infinities among states and derivatives: they reach what the definition says they reach, whatever starts and ends around
    them, and everything else is right."""
    from paper_2203_04738_b200 import binding as L
    nan, inf = float("nan"), float("inf")
    for seed, (lengths, reset) in enumerate(((False, False), (True, False), (False, True), (True, True))):
        rng = np.random.default_rng(100 * seed + T)

        def made(x, values, share):
            x = np.clip(x, -4, 4)
            for v in values:
                x = np.where(rng.random(x.shape) < share / len(values), v, x)
            return x

        few = 3 / (T * B * H) if T * B * H > 3000 else 0.003
        gate = made(rng.standard_normal((T, B, H)) - (0 if cell == R.GIVEN else 1), (nan,), few)
        if cell == R.GIVEN:
            gate = gate / 5
        arrays = dict(g=dev(gate, dtype), c=dev(made(rng.standard_normal((T, B, H)), (nan,), few), dtype), h0=dev(made(rng.standard_normal((B, H)), (nan, inf, -inf), 0.1)),
                      hs=dev(made(rng.standard_normal((T, B, H)), (nan,), few), dtype), sd=dev(made(rng.standard_normal((T, B, H)), (nan, inf, -inf), 3 * few), dtype),
                      dT=dev(made(rng.standard_normal((B, H)), (nan, inf, -inf), 0.1)))
        ln = rng.integers(0, T + 1, B).astype(np.int32) if lengths else None
        rs = (rng.random((T, B)) < 4 / T).astype(np.uint8) if reset else None
        kw = dict(cell=cell, dt=dt, lengths=None if ln is None else dev(ln, torch.int32), reset=None if rs is None else dev(rs, torch.uint8))
        n = {k: R.to64(v) for k, v in arrays.items()}
        clean = lambda x: np.nan_to_num(x, nan=0, posinf=0, neginf=0)
        h, hT = L.gated_scan_forward(arrays["g"], arrays["c"], h0=arrays["h0"], **kw)
        with np.errstate(invalid="ignore", over="ignore"):
            ref, refT, bound, boundT = R.scan_forward(n["g"], n["c"], n["h0"], cell, dt, ln, rs)
            # (a candidate of NaN in a 16-bit type reaches the steps before it in the backward pass, as a gate of NaN does)
            g64 = np.where(np.isnan(n["c"]), nan, n["g"]) if dtype != F32 and cell != R.GIVEN else n["g"]
            refs, bounds = R.scan_backward(g64, n["c"], n["hs"], n["h0"], n["sd"], n["dT"], cell, dt, ln, rs)
        R.check(h, ref, clean(bound) + R.rounding(clean(ref), dtype), "h")
        R.check(hT, refT, clean(boundT), "hT")
        got = L.gated_scan_backward(arrays["g"], arrays["c"], arrays["hs"], h0=arrays["h0"], dh_seed=arrays["sd"], dhT=arrays["dT"], **kw)
        for what, x, r, bd in zip(("dgate", "dcand", "dh0"), got, refs, bounds):
            R.check(x, r, clean(bd) + (0 if what == "dh0" else R.rounding(clean(r), dtype)), what)
    assert L.last_device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,B,H,batch_major", [(90, 2, 24, False), (150, 3, 33, True), (520, 2, 64, False), (700, 2, 520, False), (700, 5, 121, True)])
@pytest.mark.parametrize("span", [3, 20, 60])
def test_coefficients_of_any_size_between_bounded_states(span, T, B, H, batch_major, dtype):
    """States that jump between levels 2^-span .. 2^span at every step, by coefficients of up to 2^(2 span) in size, some of them zero."""
    from paper_2203_04738_b200 import binding as L
    for seed, (lengths, reset) in enumerate(((False, False), (True, False), (False, True), (True, True))):
        rng = np.random.default_rng(10 * T + seed)
        level = rng.integers(-span, span + 1, (T + 1, B, H)).astype(np.float64)
        a = 2.0 ** (level[1:] - level[:-1]) * np.where(rng.random((T, B, H)) < 0.5, -1, 1) * (rng.random((T, B, H)) > 0.01)
        arr = (lambda x: x.transpose(0, 1)) if batch_major else (lambda x: x)
        lay = lambda x: arr(dev(x.swapaxes(0, 1) if batch_major else x, dtype))
        n = lambda *s: rng.standard_normal(s)
        g, c, hs, sd = lay(a), lay(2.0 ** level[1:] * n(T, B, H)), lay(2.0 ** level[1:] * n(T, B, H)), lay(2.0 ** -level[1:] * n(T, B, H))
        h0 = dev(2.0 ** level[0] * n(B, H))
        ln = rng.integers(0, T + 1, B).astype(np.int32) if lengths else None
        rs = (rng.random((T, B)) < 4 / T).astype(np.uint8) if reset else None
        end = np.full(B, T) if ln is None else ln
        dT = dev(2.0 ** -np.take_along_axis(level, end[None, :, None], 0)[0] * n(B, H))
        kw = dict(cell=R.GIVEN, h0=h0, lengths=None if ln is None else dev(ln, torch.int32), reset=None if rs is None else dev(rs, torch.uint8))
        h, hT = L.gated_scan_forward(g, c, **kw)
        m = [R.to64(x) for x in (g, c, hs, h0, sd, dT)]
        ref, refT, bound, boundT = R.scan_forward(m[0], m[1], m[3], R.GIVEN, 1.0, ln, rs)
        R.check(h, ref, bound + R.rounding(ref, dtype), "h")
        R.check(hT, refT, boundT, "hT")
        got = L.gated_scan_backward(g, c, hs, dh_seed=sd, dhT=dT, **kw)
        refs, bounds = R.scan_backward(*m, R.GIVEN, 1.0, ln, rs)
        for what, x, r, bd in zip(("dgate", "dcand", "dh0"), got, refs, bounds):
            R.check(x, r, bd + (0 if what == "dh0" else R.rounding(r, dtype)), what)
    assert L.last_device_status() == 0
