"""The operators as a program uses them together: a teacher answers with its top alternatives (token_logprobs), a student with a linear
recurrence (gated_scan) learns from them (distill_topk_fwd_bwd), and then generates one token at a time; against 64 bits throughout."""
import numpy as np
import pytest
import torch

from tests import operator_refs as R

pytestmark = pytest.mark.gpu


class Student(torch.nn.Module):
    """projection -> linear recurrence -> softmax head, in 64-bit torch: the arithmetic of the gated scan step by step"""

    def __init__(self, I, H, V, seed):
        super().__init__()
        g = torch.Generator().manual_seed(seed)
        u = lambda *s: torch.nn.Parameter((torch.rand(*s, generator=g, dtype=torch.float64) * 2 - 1) / s[-1] ** 0.5)
        self.W, self.b, self.Wc, self.bc = u(2 * H, I), u(1, 2 * H), u(V, H), u(1, V)

    def forward(self, x, h0, cell, lengths):
        gi = x @ self.W.T + self.b
        H = self.W.shape[0] // 2
        z, n = torch.sigmoid(gi[..., :H]), torch.tanh(gi[..., H:])
        r = 1 / (1 + z) if cell == R.IMPLICIT else torch.ones_like(z)
        a, b = (r if cell == R.IMPLICIT else 1 - z), z * n * r
        hs, h = [], h0
        for t in range(x.shape[0]):
            live = (t < lengths)[:, None]
            h = torch.where(live, a[t] * h + b[t], h)
            hs.append(torch.where(live, h, torch.zeros_like(h)))
        return torch.stack(hs) @ self.Wc.T + self.bc, h


def test_a_student_learns_from_a_teachers_alternatives_and_generates():
    from paper_2203_04738_b200 import binding as L
    T, B, I, H, V, K, tau = 70, 4, 24, 40, 130, 9, 2.0
    rng = np.random.default_rng(11)
    x = torch.from_numpy(rng.standard_normal((T, B, I)))
    lengths = torch.tensor([70, 1, 0, 33])
    live = torch.arange(T)[:, None] < lengths
    # fp32 copies of all parameters and inputs are exact: the 64-bit side starts from the rounded values
    m = Student(I, H, V, 5)
    with torch.no_grad():
        for p in m.parameters():
            p.copy_(p.float())
    x = x.float().double()
    h0 = torch.from_numpy(rng.standard_normal((B, H))).float().double()
    dev = lambda t: t.detach().float().cuda().contiguous()
    W, b, Wc, bc, xd, hd, ld = dev(m.W), dev(m.b), dev(m.Wc), dev(m.bc), dev(x), dev(h0), lengths.int().cuda()

    for cell in (R.CLASSIC, R.IMPLICIT):
        # the teacher answers
        t_logits = torch.from_numpy(3 * rng.standard_normal((T * B, V))).float().cuda()
        answer = L.token_logprobs(t_logits, top=K)
        # the student: forward, loss, backward; rows behind a sequence's end have weight zero
        gi = xd @ W.T + b
        h, hT = L.gated_scan_forward(gi[..., :H], gi[..., H:], h0=hd, cell=cell, lengths=ld)
        logits = h.reshape(T * B, H) @ Wc.T + bc
        w = (live.float() / live.sum()).reshape(-1).cuda()
        loss, _, dlogits = L.distill_topk_fwd_bwd(logits, answer.top_id, answer.top_logprob, weight=w, temperature=tau, dlogits=logits)
        dWc, dbc, dh = dlogits.T @ h.reshape(T * B, H), dlogits.sum(0), (dlogits @ Wc).view(T, B, H)
        dgi = torch.empty_like(gi)
        _, _, dh0 = L.gated_scan_backward(gi[..., :H], gi[..., H:], h, h0=hd, dh_seed=dh, cell=cell, lengths=ld, dgate=dgi[..., :H], dcand=dgi[..., H:])
        dW, db = dgi.view(T * B, 2 * H).T @ xd.view(T * B, I), dgi.sum((0, 1))
        # ... and in 64 bits
        m.zero_grad()
        hz = h0.clone().requires_grad_(True)
        z, hT64 = m(x, hz, cell, lengths)
        q = torch.log_softmax(z.reshape(T * B, V) / tau, 1)
        tl = torch.log_softmax(t_logits.double().cpu(), 1)
        best = tl.topk(K, dim=1)
        p = torch.log_softmax(best.values / tau, 1)
        rows = tau ** 2 * (p.exp() * (p - q.gather(1, best.indices))).sum(1)
        want = (rows * w.double().cpu()).sum()
        want.backward()
        assert torch.equal(answer.top_id.cpu().long(), best.indices)
        # products of up to 280 terms in fp32 (torch's, without tf32) and a recurrence of 70 steps: 1e-4 of each array's norm
        assert abs(float(loss) - float(want.detach())) < 1e-4 * float(want.detach())
        near = lambda got, ref: torch.linalg.norm(got.double().cpu() - ref) <= 1e-4 * torch.linalg.norm(ref)
        assert near(hT, hT64.detach())
        for got, ref in ((dWc, m.Wc.grad), (dbc, m.bc.grad[0]), (dW, m.W.grad), (db, m.b.grad[0]), (dh0, hz.grad)):
            assert near(got, ref)

        # one token at a time from the state after the prompt: the same log probabilities as in one piece
        more = torch.from_numpy(rng.standard_normal((6, B, I))).float()
        gi = torch.cat((gi, more.cuda() @ W.T + b))
        state = hT.clone()
        for t in range(6):
            g = gi[T + t:T + t + 1]
            step, _ = L.gated_scan_forward(g[..., :H], g[..., H:], h0=state, cell=cell, hT=state)
            out = L.token_logprobs(step[0] @ Wc.T + bc, torch.arange(B, dtype=torch.int32, device="cuda"), top=3)
        whole, last = L.gated_scan_forward(gi[T:, :, :H], gi[T:, :, H:], h0=hT, cell=cell)
        assert near(state, last.double().cpu())
        z = (R.to64(whole[-1]) @ R.to64(Wc).T + R.to64(bc))
        ref = R.logprobs(z, np.arange(B), 3)
        # logits of 40 terms in fp32: 40 u of their size at worst, twice
        assert np.abs(R.to64(out.logprob) - ref["logprob"]).max() < 1e-4 and np.array_equal(out.top_id.cpu().numpy(), ref["top_id"])


def test_a_gated_student_of_an_mgrit_teacher():
    """The library's own path in front: the head of a GRU that MGRIT solved gives the alternatives."""
    from paper_2203_04738_b200 import binding as L
    T, B, I, H, V = 64, 4, 16, 32, 50
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g)
    p = {"W_ih": n(3 * H, I) / 4, "W_hh": n(3 * H, H) / 6, "b_ih": n(3 * H), "b_hh": n(3 * H)}
    x, h0, Wc = n(T, B, I), torch.zeros(B, H, device="cuda"), n(V, H)
    states, _, _ = L.mgrit_gru_forward(L.make_cfg(T, B, I, H), p, x, h0)
    logits = states.reshape(T * B, H) @ Wc.T
    tok = torch.randint(0, V, (T * B,), device="cuda", generator=g).int()
    r = L.token_logprobs(logits, tok, top=8)
    ref = R.logprobs(R.to64(logits), tok.cpu().numpy(), 8)
    R.check(r.logprob, ref["logprob"], ref["b_logprob"])
    assert np.array_equal(r.top_id.cpu().numpy(), ref["top_id"])
    loss, row, d = L.distill_topk_fwd_bwd(logits.bfloat16(), r.top_id, r.top_logprob)
    # a model that is its own teacher, up to the tail and the rounding to bf16: the loss is - log of the alternatives' mass, and a little
    mass = np.exp(ref["top_logprob"]).sum(1)
    x16 = R.to64(logits.bfloat16())
    (rl, rr, rd), (bl, br, bd) = R.distill(x16, r.top_id.cpu().numpy(), R.to64(r.top_logprob), None, 1.0)
    R.check(row, rr, br)
    R.check(d, rd, bd + R.rounding(rd, torch.bfloat16))
    # rounding moves a logit by at most 2^-8 of it, and the divergence by no more than twice that
    assert np.abs(rr + np.log(mass)).max() <= 2 * 2 ** -8 * np.abs(x16).max()
