"""The gated scan where its tiles wait for one another most: one to six column tiles (up to four of them, one warp looks back for its block and the
others wait for that warp), long sequences, and a device that other kernels share."""
import numpy as np
import pytest
import torch

from tests import operator_refs as R
from tests.test_gpu_gated_scan import BF16, F16, F32, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,H", [(F32, 20), (F32, 64), (F32, 130), (F32, 256), (F32, 300), (BF16, 50), (BF16, 128), (BF16, 250), (F16, 512), (F16, 700)])
def test_few_column_tiles_beside_other_work(dtype, H):
    from paper_2203_04738_b200 import binding as L
    T = 6000
    d = make(T, 1, H, dtype, R.IMPLICIT, False, False, False, H)
    kw = dict(h0=d["h0"])
    ref, refT, bound, boundT = R.scan_forward(R.to64(d["gate"]), R.to64(d["cand"]), R.to64(d["h0"]), R.IMPLICIT, 1.0)
    want = L.gated_scan_forward(d["gate"], d["cand"], **kw)
    R.check(want[0], ref, bound + R.rounding(ref, dtype), "h")
    R.check(want[1], refT, boundT, "hT")
    gwant = L.gated_scan_backward(d["gate"], d["cand"], want[0], dh_seed=d["seed"], dhT=d["dhT"], **kw)
    torch.cuda.synchronize()
    side, x = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda", dtype=BF16)
    for i in range(12):
        with torch.cuda.stream(side):
            for _ in range(i % 4):                 # blocks of the scan start late, or beside others
                x @ x
        got = L.gated_scan_forward(d["gate"], d["cand"], **kw)
        ggot = L.gated_scan_backward(d["gate"], d["cand"], want[0], dh_seed=d["seed"], dhT=d["dhT"], **kw)
        assert all(torch.equal(p, q) for p, q in zip((*got, *ggot), (*want, *gwant)))
    torch.cuda.synchronize()
    assert L.last_device_status() == 0


@pytest.mark.parametrize("T,B,H,dtype", [(129, 60, 1024, BF16), (140, 3, 1000, F32), (257, 8, 130, F16), (3000, 1, 64, F32)])
@pytest.mark.parametrize("back", [False, True])
def test_states_in_place_over_several_tiles(T, B, H, dtype, back):
    """The last tile writes over the first state, which warps of other blocks have read: with NaN and infinities among the states, forward (hT = h0,
    which the header allows) and, chunk after chunk, as generation does it."""
    from paper_2203_04738_b200 import binding as L
    d = make(T, B, H, dtype, R.IMPLICIT, False, False, False, T)
    h0 = d["h0"].clone()
    h0.view(-1)[::7], h0.view(-1)[3::11] = float("nan"), float("inf")
    h0.view(torch.int32).view(-1)[5::13] = -1              # (the NaN that stands for a word not yet there)
    d["h0"] = h0
    if back:
        want = L.gated_scan_backward(d["gate"], d["cand"], d["seed"], h0=d["h0"], dh_seed=d["seed"], dhT=h0)
        assert torch.equal(want[2].isnan(), h0.isnan()) and torch.equal(want[2].isinf(), h0.isinf())
        return
    want, last = L.gated_scan_forward(d["gate"], d["cand"], h0=h0)
    assert torch.equal(last.isnan(), h0.isnan()) and torch.equal(last.isinf(), h0.isinf())
    clean = ~(h0.isnan() | h0.isinf())
    for _ in range(20):
        state = h0.clone()
        h, hT = L.gated_scan_forward(d["gate"], d["cand"], h0=state, hT=state)
        assert torch.equal(state[clean], last[clean]) and torch.equal(h[:, clean], want[:, clean]) and torch.equal(state.isnan(), last.isnan())
