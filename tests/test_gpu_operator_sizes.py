"""Sizes past 32 bits of the operators over given arrays: refused before anything is allocated or launched (arrays repeat one row, so that they need no
memory)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_rows_and_alternatives_past_32_bits_are_refused():
    from paper_2203_04738_b200 import binding as L
    x = torch.zeros(1, 4, device="cuda")
    i32 = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = torch.cuda.memory_allocated()
    for n in (2 ** 32 + 1, 2 ** 31):
        many = x.expand(n, 4)
        with pytest.raises(ValueError):
            L.token_logprobs(many)
        with pytest.raises(ValueError):
            L.token_logprobs_backward(many, i32.expand(n), x[:, 0].expand(n), dlogprob=x[:, 0].expand(n))
        with pytest.raises(ValueError):
            L.distill_topk_fwd_bwd(many, i32.expand(n, 1), x[:, :1].expand(n, 1))
        with pytest.raises(ValueError):
            L.token_logprobs(x, top=n)
    assert torch.cuda.memory_allocated() == before


def test_scans_past_32_bits_are_refused():
    from paper_2203_04738_b200 import binding as L
    x, out = torch.zeros(1, 1, 4, device="cuda"), torch.zeros(1, 1, 4, device="cuda")
    long = x.expand(2 ** 31, 1, 4)
    for dt in (1e40, 1e30):                    # (the library's own refusal)
        with pytest.raises(L.MgritError):
            L.gated_scan_forward(x, x, dt=dt)
    with pytest.raises(ValueError):
        L.gated_scan_forward(x, x, cell=2 ** 31)
    with pytest.raises(ValueError):
        L.gated_scan_forward(long, long, h=long, hT=out[0])
