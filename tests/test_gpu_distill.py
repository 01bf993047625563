"""Distillation from a teacher's top logits (distill_topk_fwd_bwd) against 64 bits: types, widths, absent and repeated alternatives,
weights, masked logits, in place."""
import numpy as np
import pytest
import torch

from tests import operator_refs as R
from tests.test_gpu_token_logprobs import BF16, DTYPES, F16, F32, ints, rows

pytestmark = pytest.mark.gpu


def teacher(N, V, K, seed, repeats=False):
    rng = np.random.default_rng(seed)
    ids = np.stack([rng.choice(V, K, replace=repeats or K > V) for _ in range(N)])
    return ids, np.sort(3 * rng.standard_normal((N, K)), axis=1)[:, ::-1].astype(np.float32).copy()


def check_distill(x, ids, y, w, tau, name="", **kw):
    from paper_2203_04738_b200 import binding as L
    f = lambda a: None if a is None else torch.from_numpy(np.asarray(a, dtype=np.float32)).cuda()
    before = R.to64(x)
    loss, row, d = L.distill_topk_fwd_bwd(x, ints(ids), f(y), weight=f(w), temperature=tau, **kw)
    (rl, rr, rd), (bl, br, bd) = R.distill(before, ids, np.asarray(y, dtype=np.float64), None if w is None else np.asarray(w, np.float32).astype(np.float64), tau)
    R.check(row, rr, br + 2 * R.U * np.nan_to_num(np.abs(rr), posinf=0), name + " row_loss")
    R.check(d, rd, bd + R.rounding(np.nan_to_num(rd), d.dtype), name + " dlogits")
    R.check(loss, np.array([rl]), bl + 4 * R.U * abs(np.nan_to_num(rl)), name + " loss")
    return loss, row, d


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 2, 31, 51, 64, 400, 1024, 1025, 2048, 5000, 8192, 16385, 32768, 32771, 70001, 131072, 140001])
def test_widths(V, dtype):
    for i, (N, K, ld, off, tau) in enumerate(((1, 1, None, 0, 1.0), (6, 8, V + 5, 1, 2.0), (11, 64, None, 0, 0.7))):
        K = min(V, K)
        ids, y = teacher(N, V, K, V + i)
        w = None if i == 0 else np.random.default_rng(i).random(N)
        check_distill(rows(N, V, dtype, V + i, ld=ld, offset=off), ids, y, w, tau, f"{N}x{V}")


@pytest.mark.parametrize("N,V,K", [(300, 51, 8), (2000, 300, 3), (333, 5000, 40), (310, 33000, 16), (3, 300000, 20), (2, 1100000, 5)])
def test_many_rows_and_very_wide_ones(N, V, K):
    for dtype in (F32, BF16):
        ids, y = teacher(N, V, K, N)
        check_distill(rows(N, V, dtype, N), ids, y, None, 2.0, f"{N}x{V}")


@pytest.mark.parametrize("V", [51, 3000, 40000])
@pytest.mark.parametrize("K", [1, 33, 257, 1024])
def test_numbers_of_alternatives(V, K):
    ids, y = teacher(4, V, K, K, repeats=True)
    check_distill(rows(4, V, F32, K), ids, y, [1.0, 0.5, 0.25, 2.0], 1.0, f"{V} {K}")


@pytest.mark.parametrize("V", [40, 2500, 50000])
def test_absent_repeated_and_masked(V):
    inf, nan = float("inf"), float("nan")
    for dtype in DTYPES:
        N, K = 14, 6
        ids, y = teacher(N, V, K, V)
        x = rows(N, V, dtype, V).clone()
        w = np.full(N, 0.3, np.float32)
        ids[0] = -1                                       # no alternative at all
        ids[1, 2:] = V                                    # two of them
        ids[2] = ids[2, 0]                                # the same one six times
        ids[3, 3] = ids[3, 0]
        y[4, 1:] = -inf                                   # one probability
        y[5] = -inf                                       # none
        x[6, 0] = -inf                                    # a token that cannot occur, not the teacher's ...
        x[6, ids[6]] = 0.5
        x[7, ids[7, 2]] = -inf                            # ... and one of the teacher's: infinite loss, finite gradient
        x[8] = -inf                                       # nothing left of the student
        x[9, V // 2] = nan
        y[10, 1] = nan
        y[11, 0] = inf
        x[12, 1] = nan                                    # without weight
        w[12] = 0
        ids[13, 1], y[13, 1] = -7, nan                    # NaN in an absent place
        check_distill(x, ids, y, w, 2.0, str(dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V,K,ld", [(1190, 1025, 16, None), (1201, 1100, 128, 1103), (1184, 4003, 129, None), (1184, 4003, 7, 4008), (1187, 150, 33, None), (1183, 4003, 7, None)])
def test_many_rows_of_middling_width(N, V, K, ld, dtype):
    inf, nan = float("inf"), float("nan")
    ids, y = teacher(N, V, K, V)
    x = rows(N, V, dtype, V, ld=ld, offset=0 if ld is None else 1)
    w = np.random.default_rng(K).random(N).astype(np.float32)
    ids[0] = -1
    ids[1, 2:] = V
    ids[2] = ids[2, 0]
    ids[3, 3] = ids[3, 0]
    y[4, 1:] = -inf
    y[5] = -inf
    x[8] = -inf
    x[9] = torch.finfo(dtype).min
    x[10, V // 2] = nan
    y[11, 1] = nan
    w[12] = 0
    x[13, ids[13, 0]] = -inf
    w[8:12] = w[13] = 0                                # (their losses are not finite)
    ref = check_distill(x, ids, y, w, 2.0)[2]
    out = torch.full((N, V + 2), 9.0, dtype=dtype, device="cuda")
    check_distill(x, ids, y, w, 2.0, dlogits=out[:, 1:V + 1])
    assert torch.equal(out[:, 1:V + 1], ref) and (out[:, 0] == 9).all() and (out[:, V + 1] == 9).all()
    check_distill(x, ids, y, w, 2.0, dlogits=x)
    assert torch.equal(x, ref)


def test_in_place_and_inside_wider_rows():
    for dtype, V in ((F32, 51), (BF16, 4001), (F16, 33001)):
        ids, y = teacher(5, V, 7, 1)
        x = rows(5, V, dtype, 2, ld=V + 9, offset=3)
        ref = check_distill(x, ids, y, None, 1.0)[2]
        out = torch.full((5, V + 4), 9.0, dtype=dtype, device="cuda")
        check_distill(x, ids, y, None, 1.0, dlogits=out[:, 1:V + 1])
        assert torch.equal(out[:, 1:V + 1], ref) and (out[:, 0] == 9).all() and (out[:, V + 1:] == 9).all()
        check_distill(x, ids, y, None, 1.0, dlogits=x)
        assert torch.equal(x, ref)


def test_no_rows():
    from paper_2203_04738_b200 import binding as L
    loss, row, d = L.distill_topk_fwd_bwd(torch.empty(0, 9, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, device="cuda"))
    assert float(loss) == 0 and row.shape == (0,) and d.shape == (0, 9)


def test_offsets_past_32_bits():
    N, V = 3, 40001
    ld = (1 << 31) + 77
    buf = torch.zeros(2 * ld + V, dtype=BF16, device="cuda")
    x = torch.as_strided(buf, (N, V), (ld, 1))
    x.copy_(rows(N, V, BF16, 3))
    ids, y = teacher(N, V, 9, 4)
    check_distill(x, ids, y, None, 1.0, dlogits=x)
    del buf, x
    torch.cuda.empty_cache()


def test_gradient_against_differences():
    from paper_2203_04738_b200 import binding as L
    rng = np.random.default_rng(0)
    N, V, K, tau = 6, 80, 5, 1.5
    x = rows(N, V, F32, 8)
    ids, y = teacher(N, V, K, 3)
    w = rng.random(N).astype(np.float32)
    t = lambda a: torch.from_numpy(a).cuda()
    _, _, d = L.distill_topk_fwd_bwd(x, ints(ids), t(y), weight=t(w), temperature=tau)
    got, x64, eps = R.to64(d), R.to64(x), 1e-5
    loss = lambda z: R.distill(z, ids, y.astype(np.float64), w.astype(np.float64), tau)[0][0]
    for _ in range(5):
        v = rng.standard_normal(x64.shape)
        num = (loss(x64 + eps * v) - loss(x64 - eps * v)) / (2 * eps)
        assert abs(num - (got * v).sum()) <= (400 * R.U + 1e-8) * (np.abs(got * v).sum() + w.sum())


def test_results_repeat_and_replay():
    from paper_2203_04738_b200 import binding as L
    for N, V in ((3, 131072), (40, 33000), (500, 60)):
        x = rows(N, V, BF16, N)
        ids, y = teacher(N, V, 8, 1)
        ids, y = ints(ids), torch.from_numpy(y).cuda()
        first = L.distill_topk_fwd_bwd(x, ids, y)
        out = [torch.empty_like(t) for t in first]
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            L.distill_topk_fwd_bwd(x, ids, y, loss=out[0], row_loss=out[1], dlogits=out[2])
        for _ in range(5):
            for o in out:
                o.zero_()
            g.replay()
            assert all(torch.equal(a, b) for a, b in zip(out, first))


@pytest.mark.parametrize("V", [40, 300, 2500, 50000])
@pytest.mark.parametrize("tau", [5e-39, 1e-38, 1e-30, 1e-3, 1e3, 1e18, 1e30])
def test_temperatures_of_any_size(V, tau):
    """A teacher's or student's distances are divided by tau, not their logits: a small tau names one token, a large one leaves the uniform
    distribution."""
    from paper_2203_04738_b200 import binding as L
    for N in (5, 1300):
        if N * V > 3e6:
            continue
        rng = np.random.default_rng(V)
        K = 6
        ids, y = teacher(N, V, K, V)
        y += 100.0
        x = rows(N, V, F32, V).clone()
        ids[:, 0] = x.argmax(1).cpu().numpy()         # (the teacher's best is the student's)
        w = np.full(N, 1.0, np.float32)
        f = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float32)).cuda()
        loss, row, d = L.distill_topk_fwd_bwd(x, ints(ids), f(y), weight=f(w), temperature=tau)
        t = float(np.float32(tau))
        x64, y64 = R.to64(x), y.astype(np.float64)
        q, p = np.exp(np.maximum((x64 - x64.max(1, keepdims=True)) / t, -1e4)), np.exp(np.maximum((y64 - y64.max(1, keepdims=True)) / t, -1e4))
        q, p = q / q.sum(1, keepdims=True), p / p.sum(1, keepdims=True)
        for r in range(N):
            np.add.at(q[r], ids[r], -p[r])
        assert torch.isfinite(d).all() and not row.isnan().any() and not loss.isnan().any()
        if tau <= 1e18:                                   # (tau^2 times log(V / K) leaves fp32 beyond)
            assert torch.isfinite(row).all() and (torch.isfinite(loss).all() or row.double().sum() > 3.4e38)      # (1300 rows of 2e36: 2.5e39)
        # differences are exact to u of themselves, their exponents count to 150 at most: 2 (2 + 2.2 * 104) u and the sum's 40 u, of at most one each
        far = np.abs(R.to64(d) / t - q)
        assert far.max() <= 512 * R.U, far.max()
        if tau <= 1e-30:
            assert not row.any()
