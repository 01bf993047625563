"""Operators over logits and long sequences, as cases that can be timed and compared.

Three operators, each in every direction that it has:

  scan      the gated linear recurrence h_t = a_t h_{t-1} + b_t, whose coefficients come from two pre-activations (gate and
            candidate) by the library's classic or implicit cell without its recurrent matrix, or are given: forward and
            backward, packed sequences (`reset`), ragged batches (`lengths`), time-major and batch-major arrays.
  logprob   log probabilities of given tokens with the entropy of their distribution and its top alternatives; its backward pass.
  distill   distillation from a teacher's top logits: loss, and gradient with respect to the student's logits, in one call.

`own` selects who computes: the library through its binding, or a plain form in elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
CELLS = {"classic": 0, "implicit": 1, "given": 2}


def _scan(back, T, B, H, dtype, cell="implicit", dt=1.0, lengths=False, reset=False, batch_major=False, **name):
    return dict(op="scan", back=back, T=T, B=B, H=H, dtype=dtype, cell=cell, dt=dt, lengths=lengths, reset=reset, batch_major=batch_major, **name)


def _logprob(back, N, V, K, dtype, **name):
    return dict(op="logprob", back=back, N=N, V=V, K=K, dtype=dtype, **name)


def _distill(N, V, K, dtype, tau, weight=False, **name):
    return dict(op="distill", N=N, V=V, K=K, dtype=dtype, tau=tau, weight=weight, **name)


def listed():
    return [
        # one token for each of 32 running sequences: the recurrent state is all that serving keeps; latency
        _scan(False, 1, 32, 1024, "bf16", name="scan_token"),
        # the layer of the default training shape, forward and backward
        _scan(False, 2048, 32, 1024, "bf16", name="scan_train"),
        _scan(True, 2048, 32, 1024, "bf16", name="scan_back_train"),
        # one very long sequence in fp32: few columns, all the parallelism is in time
        _scan(False, 65536, 1, 1024, "f32", cell="classic", name="scan_one_long"),
        # a padded batch of packed documents, batch-major, odd length and odd width
        _scan(True, 997, 24, 203, "f16", lengths=True, reset=True, batch_major=True, name="scan_back_ragged"),
        # the answer's log probability and 20 alternatives for eight sequences that decode; latency over a wide vocabulary
        _logprob(False, 8, 131072, 20, "bf16", name="logprob_token"),
        # scoring a prompt of 2048 tokens over an odd vocabulary (rows that start at odd addresses)
        _logprob(False, 2048, 50001, 5, "f16", name="logprob_prompt"),
        # per-step outputs of a small classifier over the default training shape: many short rows
        _logprob(False, 65536, 51, 5, "f32", name="logprob_classes"),
        # the gradient of a policy's log probabilities and entropies
        _logprob(True, 4096, 32768, 0, "bf16", name="logprob_back"),
        # the classifier of the default training shape learns from a teacher's eight top classes
        _distill(32, 51, 8, "f32", 2.0, name="distill_classes"),
        # a batch of tokens against 32 stored alternatives of a teacher
        _distill(4096, 32768, 32, "bf16", 1.0, weight=True, name="distill_vocab"),
        # a wide, odd vocabulary in fp32
        _distill(1000, 131071, 64, "f32", 2.0, name="distill_wide"),
    ]


def draw(rng):
    lg = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    op = rng.choice(["scan", "scan", "logprob", "logprob", "distill"])
    if op == "scan":
        while True:
            T, B, H = lg(1, 65536), lg(1, 64), lg(8, 4096)
            if rng.random() < 0.6:
                H = max(8, H // 8 * 8)
            if T * B * H <= (1 << 25 if dtype == "f32" else 1 << 26):
                break
        return _scan(rng.random() < 0.5, T, B, H, dtype, cell=rng.choice(["implicit", "classic", "given"]), dt=rng.choice([1.0, 0.5, 1.0]),
                     lengths=rng.random() < 0.3, reset=rng.random() < 0.3, batch_major=rng.random() < 0.4)
    while True:
        N, V = lg(1, 65536), lg(8, 150000)
        if rng.random() < 0.5:
            V = max(8, V // 8 * 8)
        if N * V <= (1 << 26 if dtype == "f32" else 1 << 27):
            break
    if op == "logprob":
        back = rng.random() < 0.4
        return _logprob(back, N, V, 0 if back else min(V, rng.choice([0, 1, 5, 20, 64])), dtype)
    return _distill(N, V, min(V, lg(1, 128)), dtype, rng.choice([1.0, 2.0, 0.7]), weight=rng.random() < 0.5)


def _lengths(case):
    """Lengths of a padded batch, from an empty sequence to a full one (their sum is known before the inputs are made)."""
    T, B = case["T"], case["B"]
    return [T if B == 1 else round(T * i / (B - 1)) for i in range(B)]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)
    s = {"case": case}
    if case["op"] == "scan":
        T, B, H = case["T"], case["B"], case["H"]
        arrange = (lambda x: x.transpose(0, 1)) if case["batch_major"] else (lambda x: x)
        rows = (B, T) if case["batch_major"] else (T, B)
        proj = normal(*rows, 2 * H)              # one projection holds both pre-activations, side by side
        if case["cell"] == "given":              # decays between 0 and 1, most of them near 1
            proj[..., :H] = torch.sigmoid(proj[..., :H] + 2.0)
        else:                                    # gates that open now and then
            proj[..., :H] -= 2.0
        proj = proj.to(t)
        s.update(gate=arrange(proj[..., :H]), cand=arrange(proj[..., H:]), h0=0.5 * normal(B, H), lengths=None, reset=None)
        if case["lengths"]:
            order = torch.randperm(B, device="cuda", generator=g)
            s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")[order]
        if case["reset"]:                        # documents of 64 steps on average
            s["reset"] = arrange((torch.rand(*rows, device="cuda", generator=g) < 1 / 64).to(torch.uint8))
        if case["back"]:
            # states of the kind that the recurrence visits; the backward pass is linearised at the states that it is given
            s["h"] = arrange(torch.tanh(0.5 * normal(*rows, H)).to(t))
            if case["lengths"]:
                s["h"].mul_((torch.arange(T, device="cuda")[:, None] < s["lengths"]).to(t)[:, :, None])
            s["dh_seed"], s["dhT"] = arrange(normal(*rows, H).to(t)), normal(B, H)
        return s
    N, V, K = case["N"], case["V"], case["K"]
    logits = torch.empty(N, V, device="cuda", dtype=t)
    step = max(1, (1 << 26) // V)
    for i in range(0, N, step):                  # (by parts: the values are made in fp32)
        logits[i:i + step] = 2.5 * normal(min(step, N - i), V)
    s["logits"] = logits
    if case["op"] == "logprob":
        s["tokens"] = torch.randint(0, V, (N,), device="cuda", generator=g).to(torch.int32)
        if case["back"]:
            s["dlogprob"], s["dentropy"] = normal(N), 0.01 * normal(N)
            # what the forward pass left: statistics of each row
            s["lse"], s["entropy"] = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
            for i in range(0, N, step):
                x = logits[i:i + step].double()
                lse = torch.logsumexp(x, 1)
                s["lse"][i:i + step] = lse
                s["entropy"][i:i + step] = lse - (torch.exp(x - lse[:, None]) * x).sum(1)
        return s
    # the teacher's alternatives: different tokens of a row, in falling order; the student has risen there already
    start = torch.randint(0, V, (N, 1), device="cuda", generator=g)
    jump = max(1, V // K)
    s["top_id"] = ((start + jump * torch.arange(K, device="cuda")) % V).to(torch.int32)
    s["top_logit"] = 3.0 * normal(N, K).sort(dim=1, descending=True).values
    logits.scatter_add_(1, s["top_id"].long(), (s["top_logit"] + 4.0).to(t))
    s["weight"] = torch.rand(N, device="cuda", generator=g) / N if case["weight"] else None
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------------------

def _coefficients(case, gate, cand):
    """a_t, b_t and what their derivatives need: gate value z and candidate n."""
    if case["cell"] == "given":
        return gate, cand, None, None
    z, n = torch.sigmoid(gate), torch.tanh(cand)
    q = case["dt"] * z
    return (1 - q, q * n, z, n) if case["cell"] == "classic" else (1 / (1 + q), q * n / (1 + q), z, n)


def _valid(s):
    """[T,B,1]: whether a step belongs to its sequence; None where all do."""
    if s["lengths"] is None:
        return None
    return (torch.arange(s["case"]["T"], device="cuda")[:, None] < s["lengths"])[:, :, None]


def _scan_in_time(a, b):
    """h_t = a_t h_{t-1} + b_t from h = 0 along the first axis, in log2(T) passes over the arrays."""
    d = 1
    while d < a.shape[0]:
        b = torch.cat((b[:d], b[d:] + a[d:] * b[:-d]))
        a = torch.cat((a[:d], a[d:] * a[:-d]))
        d *= 2
    return b


def _plain_scan(s):
    case = s["case"]
    a, b, _, _ = _coefficients(case, s["gate"].float(), s["cand"].float())
    if s["reset"] is not None:
        a = torch.where(s["reset"][:, :, None] != 0, 0.0, a)
    valid = _valid(s)
    if valid is not None:
        a, b = torch.where(valid, a, 1.0), torch.where(valid, b, 0.0)
    b = torch.cat((a[:1] * s["h0"] + b[:1], b[1:]))
    h = _scan_in_time(a, b)
    hT = h[-1]
    if valid is not None:
        h = torch.where(valid, h, 0.0)
    return h.to(s["gate"].dtype), hT.clone()


def _plain_scan_back(s):
    case = s["case"]
    gate, cand = s["gate"].float(), s["cand"].float()
    a, _, z, n = _coefficients(case, gate, cand)
    prev = torch.cat((s["h0"][None], s["h"][:-1].float()))
    seed = s["dh_seed"].float()
    carry = a
    if s["reset"] is not None:
        fresh = s["reset"][:, :, None] != 0
        carry, prev = torch.where(fresh, 0.0, a), torch.where(fresh, 0.0, prev)
    valid = _valid(s)
    if valid is not None:
        carry, seed = torch.where(valid, carry, 1.0), torch.where(valid, seed, 0.0)
    # lambda_t = seed_t + carry_{t+1} lambda_{t+1}, from the last step to the first
    seed = torch.cat((seed[:-1], seed[-1:] + s["dhT"]))
    ahead = torch.cat((torch.zeros_like(carry[:1]), carry[1:].flip(0)))
    lam = _scan_in_time(ahead, seed.flip(0)).flip(0)
    dh0 = carry[0] * lam[0]
    if case["cell"] == "given":
        dgate, dcand = lam * prev, lam
    else:
        q = case["dt"] * z
        r = 1.0 if case["cell"] == "classic" else 1 / (1 + q)
        dgate = lam * case["dt"] * r * r * (n - prev) * z * (1 - z)
        dcand = lam * q * r * (1 - n * n)
    if valid is not None:
        dgate, dcand = torch.where(valid, dgate, 0.0), torch.where(valid, dcand, 0.0)
    t = s["gate"].dtype
    return dgate.to(t), dcand.to(t), dh0


def _plain_logprob(s):
    K, x = s["case"]["K"], s["logits"].float()
    top = x.amax(1, keepdim=True)
    d = x - top
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    logprob = x.gather(1, s["tokens"].long()[:, None]) - lse
    entropy = torch.log(total) - (e * d).sum(1, keepdim=True) / total
    out = [logprob[:, 0], entropy[:, 0], lse[:, 0]]
    if K > 0:
        # keys that fall with the value and, among equal values, with the index: every key is unique
        bits = (x + 0.0).view(torch.int32)
        bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = bits * (1 << 32) + ((1 << 32) - 1 - torch.arange(x.shape[1], device="cuda"))
        top_id = (1 << 32) - 1 - (key.topk(K, dim=1).values & ((1 << 32) - 1))
        out += [x.gather(1, top_id) - lse, top_id.to(torch.int32)]
    return out


def _plain_logprob_back(s):
    x = s["logits"].float()
    logp = x - s["lse"][:, None]
    p = torch.exp(logp)
    d = -p * (s["dlogprob"][:, None] + s["dentropy"][:, None] * (logp + s["entropy"][:, None]))
    d.scatter_add_(1, s["tokens"].long()[:, None], s["dlogprob"][:, None])
    return d.to(s["logits"].dtype)


def _plain_distill(s):
    case = s["case"]
    tau, ids = case["tau"], s["top_id"].long()
    x = s["logits"].float() / tau
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    y = s["top_logit"] / tau
    y = y - y.amax(1, keepdim=True)
    f = torch.exp(y)
    mass = f.sum(1, keepdim=True)
    p = f / mass
    row_loss = tau * tau * (p * (y - torch.log(mass) - (x.gather(1, ids) - top - torch.log(total)))).sum(1)
    w = s["weight"] if s["weight"] is not None else torch.full_like(row_loss, 1 / case["N"])
    d = e / total
    d.scatter_add_(1, ids, -p)
    return (w * row_loss).sum().reshape(1), row_loss, (d * (tau * w)[:, None]).to(s["logits"].dtype)


# ---- the library ---------------------------------------------------------------------------------------------------------------

def _own_run(s):
    from paper_2203_04738_b200 import binding as L
    case = s["case"]
    if case["op"] == "scan":
        kw = dict(h0=s["h0"], cell=CELLS[case["cell"]], dt=case["dt"], lengths=s["lengths"], reset=s["reset"])
        if case["back"]:
            return L.gated_scan_backward(s["gate"], s["cand"], s["h"], dh_seed=s["dh_seed"], dhT=s["dhT"], **kw)
        return L.gated_scan_forward(s["gate"], s["cand"], **kw)
    if case["op"] == "logprob":
        if case["back"]:
            return L.token_logprobs_backward(s["logits"], s["tokens"], s["lse"], s["entropy"], dlogprob=s["dlogprob"], dentropy=s["dentropy"])
        r = L.token_logprobs(s["logits"], s["tokens"], top=case["K"])
        return [r.logprob, r.entropy, r.lse] + ([r.top_logprob, r.top_id] if case["K"] > 0 else [])
    return L.distill_topk_fwd_bwd(s["logits"], s["top_id"], s["top_logit"], weight=s["weight"], temperature=case["tau"])


def run(state):
    if own:
        return _own_run(state)
    case = state["case"]
    if case["op"] == "scan":
        return _plain_scan_back(state) if case["back"] else _plain_scan(state)
    if case["op"] == "logprob":
        return _plain_logprob_back(state) if case["back"] else _plain_logprob(state)
    return _plain_distill(state)


def work(case):
    b = SIZE[case["dtype"]]
    if case["op"] == "scan":
        T, B, H = case["T"], case["B"], case["H"]
        rows = sum(_lengths(case)) if case["lengths"] else T * B       # steps whose inputs are read
        # forward: gate and candidate, the states, first and last state; backward: gate, candidate, states, seeds, two gradients
        state = 4 * B * H
        by = rows * H * b * (4 if case["back"] else 2) + T * B * H * b * (2 if case["back"] else 1) + state * (3 if case["back"] else 2)
        by += (rows if case["reset"] else 0) + (4 * B if case["lengths"] else 0)
        return {"bytes": by, "flops": rows * H * (4 if case["cell"] == "given" else 20 if case["back"] else 12)}
    N, V, K = case["N"], case["V"], case["K"]
    if case["op"] == "logprob":
        if case["back"]:
            return {"bytes": 2 * N * V * b + 20 * N, "flops": 6 * N * V}
        return {"bytes": N * V * b + N * (16 + 8 * K), "flops": 6 * N * V}
    return {"bytes": 2 * N * V * b + N * (8 * K + (8 if case["weight"] else 4)), "flops": 7 * N * V}


def exact(case, seed):
    """The definitions in 64 bits: the recurrences one step after the other, the rest row by row from the normalised distributions."""
    s = prepare(case, seed)
    D = torch.float64
    if case["op"] == "scan":
        T, B, H = case["T"], case["B"], case["H"]
        g, c = s["gate"].to(D), s["cand"].to(D)
        if case["cell"] == "given":
            a, b = g, c
        else:
            z, n = 1 / (1 + torch.exp(-g)), torch.tanh(c)
            den = 1 + case["dt"] * z if case["cell"] == "implicit" else torch.ones_like(z)
            a = 1 / den if case["cell"] == "implicit" else 1 - case["dt"] * z
            b = case["dt"] * z * n / den
        keep = torch.ones(T, B, 1, dtype=D, device="cuda") if s["reset"] is None else (s["reset"] == 0).to(D)[:, :, None]
        inside = torch.ones(T, B, 1, dtype=torch.bool, device="cuda")
        if s["lengths"] is not None:
            inside = (torch.arange(T, device="cuda")[:, None] < s["lengths"][None, :])[:, :, None]
        h0 = s["h0"].to(D)
        if not case["back"]:
            h, out = h0, torch.zeros(T, B, H, dtype=D, device="cuda")
            for t in range(T):
                h = torch.where(inside[t], a[t] * keep[t] * h + b[t], h)
                out[t] = torch.where(inside[t], h, torch.zeros_like(h))
            return [out, h]
        given, seeds, mu = s["h"].to(D), s["dh_seed"].to(D), s["dhT"].to(D)
        dg, dc = torch.zeros(T, B, H, dtype=D, device="cuda"), torch.zeros(T, B, H, dtype=D, device="cuda")
        for t in range(T - 1, -1, -1):
            lam = torch.where(inside[t], mu + seeds[t], torch.zeros_like(mu))
            hp = (h0 if t == 0 else given[t - 1]) * keep[t]
            if case["cell"] == "given":
                dg[t], dc[t] = lam * hp, lam
            else:
                # derivatives of a hp + b through the gate: both are functions of q = dt z
                slope = case["dt"] * z[t] * (1 - z[t])
                dg[t] = lam * slope * (n[t] - hp) / den[t] ** 2
                dc[t] = lam * case["dt"] * z[t] / den[t] * (1 - n[t] ** 2)
            mu = torch.where(inside[t], a[t] * keep[t] * (mu + seeds[t]), mu)
        return [dg, dc, mu]
    N, V, K = case["N"], case["V"], case["K"]
    logits, rows = s["logits"], max(1, (1 << 25) // V)
    parts = []
    for i in range(0, N, rows):
        x = logits[i:i + rows].to(D)
        if case["op"] == "logprob":
            tok = s["tokens"][i:i + rows].long()[:, None]
            logq = torch.log_softmax(x, 1)
            q = torch.exp(logq)
            if case["back"]:
                one = torch.zeros_like(x).scatter_(1, tok, 1.0)
                ent = s["entropy"][i:i + rows].to(D)[:, None]
                logp = x - s["lse"][i:i + rows].to(D)[:, None]
                p = torch.exp(logp)
                parts.append([s["dlogprob"][i:i + rows].to(D)[:, None] * (one - p) - s["dentropy"][i:i + rows].to(D)[:, None] * p * (logp + ent)])
            else:
                row = [logq.gather(1, tok)[:, 0], -(q * logq).sum(1), torch.logsumexp(x, 1)]
                if K > 0:
                    first = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :K]      # ties: the lower index first
                    row += [logq.gather(1, first), first]
                parts.append(row)
        else:
            tau, ids = case["tau"], s["top_id"][i:i + rows].long()
            logq = torch.log_softmax(x / tau, 1)
            logp = torch.log_softmax(s["top_logit"][i:i + rows].to(D) / tau, 1)
            p = torch.exp(logp)
            w = s["weight"][i:i + rows].to(D) if case["weight"] else torch.full((x.shape[0],), 1 / N, dtype=D, device="cuda")
            loss = tau ** 2 * (p * (logp - logq.gather(1, ids))).sum(1)
            target = torch.zeros_like(x).scatter_add_(1, ids, p)
            parts.append([(w * loss), loss, tau * w[:, None] * (torch.exp(logq) - target)])
    out = [torch.cat([p[k] for p in parts]) for k in range(len(parts[0]))]
    if case["op"] == "distill":
        out[0] = out[0].sum().reshape(1)
    return out[0] if case["op"] == "logprob" and case["back"] else out
