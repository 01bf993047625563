"""The gated linear recurrence (gated_scan_forward / gated_scan_backward) against its definition in 64 bits, one step after the other:
types, cells, layouts, padded and packed batches, sizes around a thread's, a warp's and a tile's share of the time axis."""
import numpy as np
import pytest
import torch

from tests import operator_refs as R

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def make(T, B, H, dtype, cell, lengths, reset, batch_major, seed):
    rng = np.random.default_rng(seed)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).cuda().to(t)
    rows = (B, T) if batch_major else (T, B)
    arr = (lambda x: x.transpose(0, 1)) if batch_major else (lambda x: x)
    proj = np.clip(rng.standard_normal((*rows, 2 * H)), -4, 4)
    proj[..., :H] = 1 / (1 + np.exp(-proj[..., :H] - 2)) if cell == R.GIVEN else proj[..., :H] - 2
    proj = dev(proj, dtype)
    d = dict(gate=arr(proj[..., :H]), cand=arr(proj[..., H:]), h0=dev(rng.standard_normal((B, H)), F32),
             seed=arr(dev(rng.standard_normal((*rows, H)), dtype)), dhT=dev(rng.standard_normal((B, H)), F32), lengths=None, reset=None)
    if lengths:
        n = rng.integers(0, T + 1, B)
        n[rng.integers(0, B)] = T
        if B > 1:
            n[(np.argmax(n) + 1) % B] = 0
        d["lengths"] = dev(n.astype(np.int32), torch.int32)
    if reset:
        d["reset"] = arr(dev((rng.random(rows) < min(0.5, 4 / T)).astype(np.uint8), torch.uint8))
    return d


def check_both(T, B, H, dtype, cell, dt=1.0, lengths=False, reset=False, batch_major=False, seed=0, h0=True, seeds=True, dhT=True):
    from paper_2203_04738_b200 import binding as L
    d = make(T, B, H, dtype, cell, lengths, reset, batch_major, seed)
    kw = dict(h0=d["h0"] if h0 else None, cell=cell, dt=dt, lengths=d["lengths"], reset=d["reset"])
    h, hT = L.gated_scan_forward(d["gate"], d["cand"], **kw)
    n64 = {k: R.to64(v) for k, v in d.items()}
    ln = None if d["lengths"] is None else d["lengths"].cpu().numpy()
    args = (n64["gate"], n64["cand"])
    ref, refT, bound, boundT = R.scan_forward(*args, n64["h0"] if h0 else None, cell, dt, ln, n64["reset"])
    R.check(h, ref, bound + R.rounding(ref, dtype), "h")
    R.check(hT, refT, boundT, "hT")
    assert h.dtype == dtype and hT.dtype == F32
    g = L.gated_scan_backward(d["gate"], d["cand"], h, dh_seed=d["seed"] if seeds else None, dhT=d["dhT"] if dhT else None, **kw)
    refs, bounds = R.scan_backward(*args, R.to64(h), n64["h0"] if h0 else None, n64["seed"] if seeds else None, n64["dhT"] if dhT else None, cell, dt, ln,
                                   n64["reset"])
    for name, got, r, bd in zip(("dgate", "dcand", "dh0"), g, refs, bounds):
        R.check(got, r, bd + (0 if name == "dh0" else R.rounding(r, dtype)), name)
    assert L.last_device_status() == 0


SIZES = [(1, 1, 1), (1, 3, 8), (2, 2, 5), (3, 1, 64), (7, 1, 33), (8, 2, 32), (9, 3, 30), (16, 4, 64), (17, 3, 31), (31, 2, 96), (33, 5, 7), (63, 2, 65),
         (64, 2, 64), (65, 1, 66), (127, 2, 40), (128, 3, 64), (129, 1, 130), (255, 2, 16), (257, 2, 34), (300, 5, 34), (513, 3, 62), (1000, 2, 16), (2049, 1, 130)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_scan_against_64_bits(i, dtype):
    T, B, H = SIZES[i]
    for cell in (R.CLASSIC, R.IMPLICIT, R.GIVEN):
        k = i + cell + (0 if dtype == F32 else 1)
        check_both(T, B, H, dtype, cell, dt=(1.0, 0.5, 1.0, 0.125)[k % 4], lengths=k % 2 == 1, reset=(k // 2) % 2 == 1, batch_major=k % 3 == 0, seed=31 * i + cell)


@pytest.mark.parametrize("T,B,H,batch_major", [(20000, 1, 8, False), (16384, 2, 33, True), (9000, 1, 200, False), (4100, 3, 70, True)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_sequences(T, B, H, batch_major, dtype):
    check_both(T, B, H, dtype, R.IMPLICIT, reset=T == 9000, lengths=B == 3, batch_major=batch_major, seed=T)


def test_many_columns():
    check_both(70, 40, 900, BF16, R.IMPLICIT, seed=1)
    check_both(2, 3, 70001, F16, R.GIVEN, seed=2)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,B,H,lengths,reset", [(997, 24, 203, True, True), (1000, 100, 63, True, True), (1000, 60, 129, False, True), (300, 300, 17, True, True), (1500, 7, 1001, True, False),
                                                 (640, 64, 200, True, True), (700, 40, 202, False, False)])
def test_many_tiles_of_odd_rows(T, B, H, lengths, reset, dtype):
    """Rows at any address, tiles of one, two and more sequences, sequences that start and end anywhere, all blocks with several tiles."""
    check_both(T, B, H, dtype, R.IMPLICIT, lengths=lengths, reset=reset, batch_major=H == 203, seed=H)


@pytest.mark.parametrize("h0,seeds,dhT", [(False, True, True), (True, False, True), (False, True, False)])
def test_absent_arrays(h0, seeds, dhT):
    check_both(150, 2, 24, F32, R.CLASSIC, h0=h0, seeds=seeds, dhT=dhT, seed=5)
    check_both(1, 2, 24, BF16, R.IMPLICIT, h0=h0, seeds=seeds, dhT=dhT, seed=6)


def test_gradient_against_differences():
    """The kernel's own gradient against central differences of its definition (64 bits), summed over the sequence."""
    from paper_2203_04738_b200 import binding as L
    T, B, H = 40, 2, 6
    for cell in (R.CLASSIC, R.IMPLICIT, R.GIVEN):
        d = make(T, B, H, F32, cell, True, True, False, 9)
        g64, c64, h64 = (R.to64(d[k]) for k in ("gate", "cand", "h0"))
        ln, rs, sd, dT = d["lengths"].cpu().numpy(), R.to64(d["reset"]), R.to64(d["seed"]), R.to64(d["dhT"])
        live = np.arange(T)[:, None, None] < ln[None, :, None]

        def loss(g, c, h0):
            h, hT, _, _ = R.scan_forward(g, c, h0, cell, 1.0, ln, rs)
            return np.where(live, h * sd, 0).sum() + (hT * dT).sum()

        h, _ = L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"], cell=cell, lengths=d["lengths"], reset=d["reset"])
        got = [R.to64(x) for x in L.gated_scan_backward(d["gate"], d["cand"], h, h0=d["h0"], dh_seed=d["seed"], dhT=d["dhT"], cell=cell, lengths=d["lengths"], reset=d["reset"])]
        rng, eps = np.random.default_rng(4), 1e-5
        for _ in range(6):
            v = [rng.standard_normal(x.shape) for x in (g64, c64, h64)]
            num = (loss(g64 + eps * v[0], c64 + eps * v[1], h64 + eps * v[2]) - loss(g64 - eps * v[0], c64 - eps * v[1], h64 - eps * v[2])) / (2 * eps)
            ana = sum((x * y).sum() for x, y in zip(got, v))
            # differences: eps^2 of the third derivative (1e-10 of it); the gradients: fp32 over 40 steps, KC u each, by their sizes
            size = sum(np.abs(x * y).sum() for x, y in zip(got, v))
            assert abs(num - ana) <= (40 * R.KC * R.U + 1e-8) * size


def test_nothing_is_read_behind_a_sequences_end():
    """NaN and infinities in padded places change nothing, and what is written there is zero."""
    from paper_2203_04738_b200 import binding as L
    T, B, H = 200, 4, 48
    for dtype in (F32, BF16):
        d = make(T, B, H, dtype, R.IMPLICIT, False, True, False, 3)
        lengths = torch.tensor([0, 1, 77, 200], dtype=torch.int32, device="cuda")
        pad = torch.arange(T, device="cuda")[:, None] >= lengths
        outs = []
        for junk in (0.0, float("nan"), float("inf")):
            x = {k: d[k].clone() for k in ("gate", "cand", "seed")}
            for v in x.values():
                v[pad] = junk
            rs = torch.where(pad, int(junk != 0.0), d["reset"].int()).to(torch.uint8)
            h, hT = L.gated_scan_forward(x["gate"], x["cand"], h0=d["h0"], lengths=lengths, reset=rs)
            hh = h.clone()
            g = L.gated_scan_backward(x["gate"], x["cand"], hh, h0=d["h0"], dh_seed=x["seed"], dhT=d["dhT"], lengths=lengths, reset=rs)
            outs.append([h, hT, *g])
            assert not h[pad].any() and not g[0][pad].any() and not g[1][pad].any()
            assert torch.equal(hT[0], d["h0"][0]) and torch.equal(g[2][0], d["dhT"][0])
        for o in outs[1:]:
            assert all(torch.equal(x, y) for x, y in zip(o, outs[0]))


def test_lengths_outside_the_array_count_as_its_ends():
    from paper_2203_04738_b200 import binding as L
    d = make(70, 3, 16, F32, R.CLASSIC, False, False, False, 3)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    a = L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"], cell=R.CLASSIC, lengths=i32(-5, 1000, 2 ** 31 - 1))
    b = L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"], cell=R.CLASSIC, lengths=i32(0, 70, 70))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_a_new_sequence_hides_what_came_before_it():
    """A NaN or an infinity in one document reaches the steps up to its end and none of the next one's, in either direction."""
    from paper_2203_04738_b200 import binding as L
    T, B, H, cut = 300, 1, 40, 171
    d = make(T, B, H, F32, R.GIVEN, False, False, False, 8)
    reset = torch.zeros(T, B, dtype=torch.uint8, device="cuda")
    reset[cut] = 1
    clean, _ = L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"], cell=R.GIVEN, reset=reset)
    for bad in (float("nan"), float("inf")):
        for where in ("gate", "cand"):
            x = {k: d[k].clone() for k in ("gate", "cand")}
            x[where][20] = bad
            h, hT = L.gated_scan_forward(x["gate"], x["cand"], h0=d["h0"], cell=R.GIVEN, reset=reset)
            assert torch.equal(h[cut:], clean[cut:]) and torch.equal(h[:20], clean[:20]) and not torch.isfinite(h[20:cut]).any()
        sd = d["seed"].clone()
        sd[250] = bad
        kw = dict(h0=d["h0"], dhT=d["dhT"], cell=R.GIVEN, reset=reset)
        g, g0 = (L.gated_scan_backward(d["gate"], d["cand"], clean, dh_seed=s, **kw) for s in (sd, d["seed"]))
        assert torch.equal(g[1][:cut], g0[1][:cut]) and torch.equal(g[2], g0[2]) and not torch.isfinite(g[1][cut:251]).any()


def test_no_steps_and_no_sequences():
    from paper_2203_04738_b200 import binding as L
    e = torch.empty(0, 3, 8, device="cuda")
    h0, dT = torch.randn(3, 8, device="cuda"), torch.randn(3, 8, device="cuda")
    h, hT = L.gated_scan_forward(e, e, h0=h0)
    assert h.shape == (0, 3, 8) and torch.equal(hT, h0)
    assert not L.gated_scan_forward(e, e)[1].any()
    assert torch.equal(L.gated_scan_backward(e, e, e, h0=h0, dhT=dT)[2], dT)
    e = torch.empty(5, 0, 8, device="cuda")
    assert L.gated_scan_forward(e, e)[1].shape == (0, 8) and L.gated_scan_backward(e, e, e, dhT=torch.empty(0, 8, device="cuda"))[2].shape == (0, 8)


def test_steps_of_generation_update_the_state_in_place():
    from paper_2203_04738_b200 import binding as L
    T, B, H = 150, 5, 72
    d = make(T, B, H, BF16, R.IMPLICIT, False, False, False, 12)
    whole, hT = L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"])
    state = d["h0"].clone()
    steps = [L.gated_scan_forward(d["gate"][t:t + 1], d["cand"][t:t + 1], h0=state, hT=state)[0] for t in range(T)]
    ref, refT, bound, boundT = R.scan_forward(R.to64(d["gate"]), R.to64(d["cand"]), R.to64(d["h0"]), R.IMPLICIT, 1.0)
    R.check(torch.cat(steps), ref, bound + R.rounding(ref, BF16), "steps")
    R.check(state, refT, boundT, "state")
    # ... and a chunk of a prompt after another, the state handed on in place
    state = d["h0"].clone()
    for lo, hi in ((0, 1), (1, 100), (100, 150)):
        L.gated_scan_forward(d["gate"][lo:hi], d["cand"][lo:hi], h0=state, hT=state)
    R.check(state, refT, boundT, "chunks")


@pytest.mark.parametrize("T,B,H,dtype", [(1, 64, 1024, BF16), (9, 64, 1024, BF16), (60, 64, 1024, F32), (128, 40, 999, F16), (129, 64, 1024, BF16), (700, 16, 512, BF16)])
def test_the_last_state_may_replace_the_first_one(T, B, H, dtype):
    """hT = h0 for one tile and several along time: every reader of the first state comes before its writer."""
    from paper_2203_04738_b200 import binding as L
    d = make(T, B, H, dtype, R.IMPLICIT, False, False, False, T)
    want, last = L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"])
    for _ in range(30):
        state = d["h0"].clone()
        h, hT = L.gated_scan_forward(d["gate"], d["cand"], h0=state, hT=state)
        assert hT is state and torch.equal(state, last) and torch.equal(h, want)


def test_two_calls_at_once_that_fill_the_device():
    """Each of them wants every SM: blocks of both run side by side, and neither waits for one of its own that has not started."""
    from paper_2203_04738_b200 import binding as L
    ds = [make(2500, 8, 1024, BF16, R.IMPLICIT, False, False, s == 2, s) for s in (1, 2)]
    want = [L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"]) for d in ds]
    gwant = [L.gated_scan_backward(d["gate"], d["cand"], w[0], h0=d["h0"], dh_seed=d["seed"]) for d, w in zip(ds, want)]
    streams = [torch.cuda.Stream() for _ in ds]
    for _ in range(6):
        got = []
        for s, d, w in zip(streams, ds, want):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append([*L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"]), *L.gated_scan_backward(d["gate"], d["cand"], w[0], h0=d["h0"], dh_seed=d["seed"])])
        torch.cuda.synchronize()
        for o, w, g in zip(got, want, gwant):
            assert all(torch.equal(x, y) for x, y in zip(o, [*w, *g]))
    assert L.last_device_status() == 0


def test_strides_of_single_places_say_nothing():
    from paper_2203_04738_b200 import binding as L
    d = make(50, 1, 64, F32, R.IMPLICIT, False, False, False, 4)
    want, last = L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"])
    odd = lambda x: torch.as_strided(x, x.shape, (x.stride(0), 3, 1))
    h, hT = L.gated_scan_forward(odd(d["gate"].contiguous()), odd(d["cand"].contiguous()), h0=d["h0"])
    assert torch.equal(h, want) and torch.equal(hT, last)


def test_strides_past_32_bits():
    """Rows of a larger array whose offsets in elements pass 2^32: nothing else of the array is touched."""
    from paper_2203_04738_b200 import binding as L
    T, H, step = 200, 64, 22_000_003
    big = torch.zeros(T * step + H, dtype=BF16, device="cuda")
    view = big[: T * step].view(T, 1, step)[:, :, 5:5 + H]
    d = make(T, 1, H, BF16, R.IMPLICIT, False, False, False, 2)
    view.copy_(d["gate"])
    ref, refT, bound, boundT = R.scan_forward(R.to64(d["gate"]), R.to64(d["cand"]), R.to64(d["h0"]), R.IMPLICIT, 1.0)
    h, hT = L.gated_scan_forward(view, d["cand"], h0=d["h0"])
    R.check(h, ref, bound + R.rounding(ref, BF16), "h")
    view.zero_()
    L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"], h=view)
    R.check(view, ref, bound + R.rounding(ref, BF16), "h in the large array")
    view.zero_()
    assert not big.any()
    del big, view
    torch.cuda.empty_cache()


def test_broadcast_inputs_and_outputs_inside_wider_rows():
    from paper_2203_04738_b200 import binding as L
    T, B, H = 140, 3, 20
    d = make(T, B, H, F16, R.IMPLICIT, False, True, False, 21)
    gate, seed = d["gate"][:, :1].expand(T, B, H), d["seed"][:1].expand(T, B, H)
    wide = torch.full((T, B, 3 * H + 1), 7.0, dtype=F16, device="cuda")
    h, dg, dc = wide[..., :H], wide[..., H:2 * H], wide[..., 2 * H + 1:]
    kw = dict(h0=d["h0"], reset=d["reset"].bool())
    _, hT = L.gated_scan_forward(gate, d["cand"], h=h, **kw)
    args = (R.to64(gate), R.to64(d["cand"]))
    ref, refT, bound, boundT = R.scan_forward(*args, R.to64(d["h0"]), R.IMPLICIT, 1.0, None, R.to64(d["reset"]))
    R.check(h, ref, bound + R.rounding(ref, F16), "h")
    R.check(hT, refT, boundT, "hT")
    L.gated_scan_backward(gate, d["cand"], h, dh_seed=seed, dgate=dg, dcand=dc, **kw)
    refs, bounds = R.scan_backward(*args, R.to64(h), R.to64(d["h0"]), R.to64(seed), None, R.IMPLICIT, 1.0, None, R.to64(d["reset"]))
    R.check(dg, refs[0], bounds[0] + R.rounding(refs[0], F16), "dgate")
    R.check(dc, refs[1], bounds[1] + R.rounding(refs[1], F16), "dcand")
    assert (wide[..., 2 * H] == 7.0).all()


def test_results_repeat_bit_for_bit():
    from paper_2203_04738_b200 import binding as L
    d = make(8192, 2, 100, F32, R.IMPLICIT, False, True, False, 5)
    first = L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"], reset=d["reset"])
    gfirst = L.gated_scan_backward(d["gate"], d["cand"], first[0], h0=d["h0"], dh_seed=d["seed"], dhT=d["dhT"], reset=d["reset"])
    for _ in range(20):
        again = L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"], reset=d["reset"])
        assert all(torch.equal(a, b) for a, b in zip(again, first))
        again = L.gated_scan_backward(d["gate"], d["cand"], first[0], h0=d["h0"], dh_seed=d["seed"], dhT=d["dhT"], reset=d["reset"])
        assert all(torch.equal(a, b) for a, b in zip(again, gfirst))


def test_graphs_that_share_a_workspace_and_calls_on_two_streams():
    from paper_2203_04738_b200 import binding as L
    T, B, H = 3000, 2, 64
    ds = [make(T, B, H, BF16, R.IMPLICIT, False, False, False, s) for s in (1, 2)]
    want = [L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"]) for d in ds]
    n = max(L.lib.gated_scan_workspace_bytes(T, B, H), 1)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")      # (whatever it held before)
    outs = [(torch.empty(T, B, H, dtype=BF16, device="cuda"), torch.empty(B, H, device="cuda")) for _ in ds]
    graphs = []
    for d, o in zip(ds, outs):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"], h=o[0], hT=o[1], ws=ws)
        graphs.append(g)
    for _ in range(3):                                               # one after the other, on one stream
        for o in outs:
            o[0].zero_(), o[1].zero_()
        for g in graphs + graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])
    # two calls at once, each with a workspace of its own
    streams = [torch.cuda.Stream() for _ in ds]
    for _ in range(5):
        got = []
        for s, d in zip(streams, ds):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(L.gated_scan_forward(d["gate"], d["cand"], h0=d["h0"]))
        torch.cuda.synchronize()
        for o, w in zip(got, want):
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])
    assert L.last_device_status() == 0
