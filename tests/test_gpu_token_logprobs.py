"""Log probabilities of tokens with entropy and top alternatives (token_logprobs) and their gradient, against 64 bits: types, widths
around a warp's, a block's and a cluster's share of a row, odd rows and strides, masked vocabularies, ties, NaN."""
import numpy as np
import pytest
import torch

from tests import operator_refs as R

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DTYPES = [F32, BF16, F16]


def rows(N, V, dtype, seed, scale=2.5, ld=None, offset=0):
    """[N,V] view of rows `ld` apart that start `offset` elements into their buffer"""
    rng = np.random.default_rng(seed)
    ld = ld or V
    x = torch.from_numpy((scale * rng.standard_normal((N, V))).astype(np.float32)).cuda().to(dtype)
    buf = torch.full((N * ld + offset + V,), float("nan"), dtype=dtype, device="cuda")
    v = buf[offset:offset + N * ld].view(N, ld)[:, :V]
    v.copy_(x)
    return v


def ints(a):
    return torch.from_numpy(np.asarray(a).astype(np.int32)).cuda()


def check_rows(x, tokens, top, name=""):
    from paper_2203_04738_b200 import binding as L
    r = L.token_logprobs(x, ints(tokens), top=top)
    w = R.logprobs(R.to64(x), np.asarray(tokens), top)
    R.check(r.lse, w["lse"], w["b_lse"], name + " lse")
    R.check(r.logprob, w["logprob"], w["b_logprob"], name + " logprob")
    R.check(r.entropy, w["entropy"], w["b_entropy"], name + " entropy")
    if top:
        assert np.array_equal(r.top_id.cpu().numpy(), w["top_id"]), name + " ids"
        R.check(r.top_logprob, w["top_logprob"], w["b_top"], name + " top_logprob")
    return r


WIDTHS = [1, 2, 7, 31, 32, 33, 51, 64, 100, 255, 256, 257, 400, 1000, 1023, 1024, 1025, 2047, 2048, 2049, 4096, 5000, 8191, 8193, 16384, 16391, 32768, 32769, 50001,
          65537, 131072, 140003]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", WIDTHS)
def test_widths(V, dtype):
    rng = np.random.default_rng(V)
    for N, top, ld, off in ((1, min(V, 20), None, 0), (5, min(V, 128), V + 3, 1), (37 if V < 20000 else 9, min(V, 5), None, 0)):
        x = rows(N, V, dtype, V + N, ld=ld, offset=off)
        tok = rng.integers(0, V, N)
        tok[0] = V - 1
        check_rows(x, tok, top, f"{N}x{V}")


@pytest.mark.parametrize("N,V", [(1, 300000), (3, 262145), (2, 1100000)])
def test_very_wide_rows(N, V):
    for dtype in (BF16, F32):
        check_rows(rows(N, V, dtype, V, ld=V + 1), np.arange(N) * 1000, 64, f"{V}")


@pytest.mark.parametrize("N,V", [(300, 51), (3000, 400), (700, 6000), (400, 33001)])
def test_many_rows(N, V):
    for dtype in DTYPES:
        check_rows(rows(N, V, dtype, N), np.random.default_rng(N).integers(-1, V + 1, N), 5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V,ld,top", [(1190, 1025, None, 20), (1201, 1100, 1103, 32), (1187, 2047, 2050, 31), (1184, 4003, None, 5), (1184, 4096, 4104, 33), (2373, 8001, None, 7),
                                        (1300, 150, None, 20), (1300, 263, 270, 32), (1183, 4003, None, 32)])
def test_many_rows_of_middling_width(N, V, ld, top, dtype):
    """Values, alternatives and gradients, with masked rows, ties and NaN among the others."""
    from paper_2203_04738_b200 import binding as L
    x = rows(N, V, dtype, V, ld=ld, offset=0 if ld is None else 1)
    inf = float("inf")
    x[0] = -inf
    x[1] = -inf
    x[1, V // 2] = 2.0
    x[9, 1::2] = -inf
    x[10] = torch.finfo(dtype).min
    x[11, V // 3] = float("nan")
    x[12, V - 1] = inf
    x[13, ::2] = 4.0                                   # equal ones
    x[14, :120] = 4.0
    x[15] = 0.5
    x[16, :130] = 4.0
    x[N - 1, V - 1] = 9.0
    tok = np.random.default_rng(N).integers(-1, V + 1, N)
    r = check_rows(x, tok, top)
    rng = np.random.default_rng(V)
    dl, de = [torch.from_numpy(rng.standard_normal(N).astype(np.float32)).cuda() for _ in range(2)]
    d = L.token_logprobs_backward(x, ints(tok), r.lse, r.entropy, dlogprob=dl, dentropy=de)
    ref, bound = R.logprobs_backward(R.to64(x), tok, R.to64(r.lse), R.to64(r.entropy), R.to64(dl), R.to64(de))
    R.check(d, ref, bound + R.rounding(ref, dtype), "gradient")
    out = torch.full((N, V + 2), 5.0, dtype=dtype, device="cuda")
    L.token_logprobs_backward(x, ints(tok), r.lse, r.entropy, dlogprob=dl, dentropy=de, dlogits=out[:, 1:V + 1])
    assert torch.equal(out[:, 1:V + 1].nan_to_num(7.0), d.nan_to_num(7.0)) and (out[:, 0] == 5).all() and (out[:, V + 1] == 5).all()


@pytest.mark.parametrize("V", [9, 51, 700, 3000, 20000, 70000])
def test_ties_go_to_the_lower_token(V):
    rng = np.random.default_rng(V)
    for dtype in DTYPES:
        x = torch.empty(6, V, device="cuda", dtype=dtype)
        x[0] = 1.5                                                              # one value in the whole row
        x[1] = torch.from_numpy(rng.integers(0, 2, V).astype(np.float32)).cuda()      # two values
        x[2] = torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.0, -0.0)        # zeros of both signs are equal
        x[3] = torch.arange(V, device="cuda") // 7                             # rising: every next element is better
        x[4] = -(torch.arange(V, device="cuda") // 5)
        x[5] = torch.from_numpy(rng.integers(-3, 4, V).astype(np.float32)).cuda()
        if dtype != F32:
            x[3], x[4] = x[3] % 64, x[4] % 64
        for top in (1, min(V, 20), min(V, 128)):
            check_rows(x, [0, 1, 2, V - 1, 4, 5], top, f"{dtype} {top}")


@pytest.mark.parametrize("V,equal", [(3000, 400), (3000, 600), (40000, 511), (40000, 520), (131072, 30000)])
def test_many_equal_best_logits(V, equal):
    """As many equal candidates as are put in order by counting, and more."""
    for dtype in (F32, BF16):
        x = torch.full((3, V), -1.0, dtype=dtype, device="cuda")
        for r in range(3):
            x[r, torch.randperm(V, device="cuda")[:equal]] = 4.0
            x[r, V // 2 + r] = 6.0
        for top in (1, 20, 128):
            check_rows(x, [0, V // 2, V - 1], top, f"{dtype} {top}")


@pytest.mark.parametrize("V", [40, 1500, 9000, 66000])
def test_masked_vocabularies_infinities_and_nan(V):
    for dtype in DTYPES:
        x = rows(10, V, dtype, V).clone()
        inf = float("inf")
        x[0] = -inf                                    # nothing is left
        x[1] = -inf
        x[1, V // 2] = 2.0                             # one token is left
        x[2, 1::2] = -inf
        x[3] = torch.finfo(dtype).min                  # the type's lowest value everywhere: equal, so a uniform distribution
        x[4, : V - 3] = torch.finfo(dtype).min         # ... as a mask
        x[5, V // 3] = float("nan")
        x[6, V - 1] = inf
        x[7] = float("nan")
        x[8, V - 2:] = -inf
        x[9, 0] = torch.finfo(dtype).max
        check_rows(x, [3, V // 2, 1, 0, V - 1, 0, V - 1, 1, V - 1, 0], min(V, 30), str(dtype))


def test_parts_of_the_answer():
    from paper_2203_04738_b200 import binding as L
    x = rows(4, 500, F32, 1)
    r = L.token_logprobs(x)
    assert r.logprob is None and r.top_id is None
    full = L.token_logprobs(x, ints([0, -1, 500, 499]), top=3)
    assert torch.equal(full.lse, r.lse) and torch.equal(full.entropy, r.entropy) and full.logprob[1] == 0 and full.logprob[2] == 0
    again = L.token_logprobs(x, ints([0, -1, 500, 499]), top=3, out=full)
    assert again is full
    r = L.token_logprobs(torch.empty(0, 7, device="cuda"), ints([]), top=2)
    assert r.logprob.shape == (0,) and r.top_id.shape == (0, 2)


def test_offsets_past_32_bits():
    from paper_2203_04738_b200 import binding as L
    N, V = 3, 40001
    ld = (1 << 31) + 77
    buf = torch.zeros(2 * ld + V, dtype=BF16, device="cuda")
    x = torch.as_strided(buf, (N, V), (ld, 1))
    x.copy_(rows(N, V, BF16, 3))
    r = check_rows(x, [5, 6, 40000], 20)
    d = L.token_logprobs_backward(x, ints([5, 6, 40000]), r.lse, dlogprob=torch.ones(N, device="cuda"))
    ref, bound = R.logprobs_backward(R.to64(x), np.array([5, 6, 40000]), R.to64(r.lse), None, np.ones(N), None)
    R.check(d, ref, bound + R.rounding(ref, BF16), "gradient")
    del buf, x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V,ld", [(1, 1, None), (3, 5, 9), (70, 51, None), (4, 1024, None), (5, 4097, 4100), (2, 32768, None), (3, 70001, 70003), (400, 300, None)])
def test_gradient(N, V, ld, dtype):
    from paper_2203_04738_b200 import binding as L
    rng = np.random.default_rng(V + N)
    x = rows(N, V, dtype, V, ld=ld, offset=1)
    tok = rng.integers(-1, V + 1, N)
    tok[0] = V - 1
    f = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()
    dl, de = f(rng.standard_normal(N)), f(rng.standard_normal(N))
    r = L.token_logprobs(x, ints(tok))
    for use_l, use_e in ((True, True), (True, False), (False, True)):
        a, b = dl if use_l else None, de if use_e else None
        d = L.token_logprobs_backward(x, ints(tok), r.lse, r.entropy, dlogprob=a, dentropy=b)
        ref, bound = R.logprobs_backward(R.to64(x), tok, R.to64(r.lse), R.to64(r.entropy), R.to64(a), R.to64(b))
        R.check(d, ref, bound + R.rounding(ref, dtype), f"{use_l} {use_e}")
    y = x.clone(memory_format=torch.preserve_format) if ld is None else x
    L.token_logprobs_backward(y, ints(tok), r.lse, r.entropy, dentropy=de, dlogits=y)          # in place
    assert torch.equal(y, d)


def test_gradient_of_masked_rows():
    from paper_2203_04738_b200 import binding as L
    for V in (30, 5000):
        x = rows(4, V, F32, V).clone()
        x[0] = -float("inf")
        x[1, 1:] = -float("inf")
        x[2, ::2] = -float("inf")
        x[3, 3] = float("nan")
        tok = np.array([1, 0, 1, 2])
        r = L.token_logprobs(x, ints(tok))
        one = torch.ones(4, device="cuda")
        d = L.token_logprobs_backward(x, ints(tok), r.lse, r.entropy, dlogprob=one, dentropy=one)
        ref, bound = R.logprobs_backward(R.to64(x), tok, R.to64(r.lse), R.to64(r.entropy), np.ones(4), np.ones(4))
        R.check(d, ref, bound, str(V))
        assert not d[0].any()


def test_gradient_against_differences():
    from paper_2203_04738_b200 import binding as L
    rng = np.random.default_rng(0)
    N, V = 5, 90
    x = rows(N, V, F32, 8)
    tok = rng.integers(0, V, N)
    dl, de = rng.standard_normal(N), rng.standard_normal(N)
    f = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()
    r = L.token_logprobs(x, ints(tok))
    got = R.to64(L.token_logprobs_backward(x, ints(tok), r.lse, r.entropy, dlogprob=f(dl), dentropy=f(de)))
    dl, de = R.to64(f(dl)), R.to64(f(de))

    def loss(z):
        w = R.logprobs(z, tok, 0)
        return (dl * w["logprob"]).sum() + (de * w["entropy"]).sum()

    x64, eps = R.to64(x), 1e-5
    for _ in range(5):
        v = rng.standard_normal(x64.shape)
        num = (loss(x64 + eps * v) - loss(x64 - eps * v)) / (2 * eps)
        # differences: 1e-10 of third derivatives; the gradient: some hundred roundings of fp32 at worst
        assert abs(num - (got * v).sum()) <= (400 * R.U + 1e-8) * (np.abs(got * v).sum() + np.abs(dl).sum() + np.abs(de).sum())


def test_results_repeat_and_replay():
    from paper_2203_04738_b200 import binding as L
    for N, V in ((3, 131072), (40, 33000), (500, 60)):
        x = rows(N, V, BF16, N)
        tok = ints(np.arange(N) % V)
        first = L.token_logprobs(x, tok, top=10)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        out = L.token_logprobs(x, tok, top=10)
        with torch.cuda.graph(g):
            L.token_logprobs(x, tok, top=10, out=out)
        for _ in range(5):
            out.lse.zero_(), out.top_id.zero_()
            g.replay()
            for a, b in zip((out.logprob, out.entropy, out.lse, out.top_logprob, out.top_id), (first.logprob, first.entropy, first.lse, first.top_logprob, first.top_id)):
                assert torch.equal(a, b)
