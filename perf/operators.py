"""The scoring and distillation operators: the cases they are measured on, their plain form and their 64-bit value.

Four operators around the LM head of a policy (a = hidden W^T, z = kappa a, softmax over the vocabulary):

scores        log-probability of a given token, entropy and the k most likely alternatives of every row, from hidden
              states and the head weight;
scores_grad   the same without alternatives, then the gradients of a loss on the log-probabilities and entropies to
              the hidden states and the head weight;
logits        the first operator for a caller that holds the logits (a decoding step that is about to sample);
distill       distillation from a teacher's top logits: loss per token and in total, and its gradients to the hidden
              states and the head weight.

Where `own` is false, `run` computes them with elementary torch operations in 32 bits.  Where it is true it makes the
calls of paper_2507_19766_b200.  The inputs of the operators that return token ids have eight-bit mantissas (a head
and activations dequantised from eight bits), so that every logit is the same number whatever the order of its sum and
the ids are defined; ties go to the lowest id.
"""
import math

import torch

own = False

BF16, F16, F32 = "bf16", "f16", "f32"
_DTYPE = {BF16: torch.bfloat16, F16: torch.float16, F32: torch.float32}
_DEV = "cuda"


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token of one sequence scored against a 151936-entry head: the whole weight is read for it
        dict(name="scores one token", op="scores", dtype=BF16, T=1, H=2048, V=151936, k=20, kappa=1.0),
        # a float32 head of test size: 512 packed tokens
        dict(name="scores float32", op="scores", dtype=F32, T=512, H=256, V=4096, k=5, kappa=1.0),
        # packed sequences of ragged lengths on a mid-sized head
        dict(name="scores ragged batch", op="scores", dtype=BF16, T=1537, H=1024, V=32768, k=8, kappa=1.0),
        # a teacher or reference model scoring half a segment, with the alternatives a student is trained on
        dict(name="scores half segment", op="scores", dtype=BF16, T=8192, H=2048, V=151936, k=32, kappa=1.0),
        # gradients of a user's loss on log-probabilities and entropies: float32 head of test size
        dict(name="scores_grad float32", op="scores_grad", dtype=F32, T=512, H=256, V=4096, kappa=1.0),
        # the same for a micro-batch of a policy update with an entropy bonus
        dict(name="scores_grad micro-batch", op="scores_grad", dtype=BF16, T=2011, H=2048, V=151936, kappa=1.0),
        # one decoding step of a single sequence whose sampler holds float32 logits
        dict(name="logits one row", op="logits", dtype=F32, T=1, V=151936, pad=0, k=20, kappa=1.0, masked=0.0),
        # a decoding step of a batch; rows padded to a longer stride, half of them under a grammar's mask
        dict(name="logits decoding batch", op="logits", dtype=F16, T=257, V=32003, pad=61, k=20, kappa=1.25, masked=0.5),
        # the log-probabilities of a prompt
        dict(name="logits prompt", op="logits", dtype=BF16, T=4096, V=151936, pad=0, k=8, kappa=1.0, masked=0.0),
        # distillation step, float32 head of test size, the teacher's remainder as one bucket
        dict(name="distill float32", op="distill", dtype=F32, T=512, H=256, V=4096, k=16, kappa=1.0, mode="tail"),
        # distillation step on ragged packed sequences, teacher lists renormalised
        dict(name="distill ragged batch", op="distill", dtype=BF16, T=1537, H=1024, V=32768, k=20, kappa=1.0, mode="renorm"),
        # distillation step of half a segment on the 151936-entry head
        dict(name="distill half segment", op="distill", dtype=BF16, T=8192, H=2048, V=151936, k=32, kappa=1.0, mode="tail"),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["scores", "scores", "scores_grad", "logits", "distill"])
    kappa = rng.choice([1.0, 1.0, 0.5, 1.25])
    if op == "logits":
        dtype = rng.choice([BF16, F16, F32])
        V = _between(rng, 300, 151936)
        T = _between(rng, 1, 4096)
        T = max(1, min(T, 4096 * 151936 // V // (2 if dtype == F32 else 1)))
        return dict(op=op, dtype=dtype, T=T, V=V, pad=rng.choice([0, rng.randrange(1, 64)]), k=rng.randrange(0, 33),
                    kappa=kappa, masked=rng.choice([0.0, 0.0, 0.3]))
    if rng.random() < 0.25:
        dtype, H, V, T = F32, 8 * _between(rng, 8, 32), _between(rng, 300, 4096), _between(rng, 1, 512)
    else:
        dtype, H, V, T = BF16, 8 * _between(rng, 16, 256), _between(rng, 1000, 151936), _between(rng, 1, 8192)
        T = max(1, min(T, (2011 if op == "scores_grad" else 8192) * 2048 * 151936 // (H * V)))
    case = dict(op=op, dtype=dtype, T=T, H=H, V=V, kappa=kappa)
    if op == "scores":
        case["k"] = rng.randrange(0, 33)
    if op == "distill":
        case["k"] = rng.randrange(1, 49)
        case["mode"] = rng.choice(["raw", "renorm", "tail"])
    return case


# ------------------------------------------------------------------------------------------------ inputs
def _eight_bit(x, step):
    """x rounded to whole multiples of `step` between -127 and 127."""
    return torch.clamp(torch.round(x / step), -127, 127) * step


def _head_inputs(case, g, eight_bit):
    T, H, V = case["T"], case["H"], case["V"]
    W = torch.randn(V, H, generator=g, device=_DEV)
    hidden = torch.randn(T, H, generator=g, device=_DEV)
    # the token of a row; in four rows of ten the row is sharply peaked on it, as trained policies are
    targets = torch.randint(0, V, (T,), generator=g, device=_DEV, dtype=torch.int32)
    peaked = torch.rand(T, generator=g, device=_DEV) < 0.4
    height = 8.0 + 12.0 * torch.rand(T, generator=g, device=_DEV)
    rows = W[targets.long()]
    hidden += (peaked * height * 64.0 / H)[:, None] * rows
    W *= 1.0 / 64.0
    if eight_bit:
        # weights of up to 127 steps of 2^-11, activations of up to 127 steps of 2^-5
        W, hidden = _eight_bit(W, 2.0 ** -11), _eight_bit(hidden, 2.0 ** -5)
    dt = _DTYPE[case["dtype"]]
    return hidden.to(dt), W.to(dt), targets


def _teacher_lists(case, g, targets):
    """Top-k lists of a teacher: distinct ids by falling log-probability; one row in sixteen has a shorter list,
    padded with -1, and one in thirty-two an empty one."""
    T, V, k = case["T"], case["V"], case["k"]
    gaps = torch.randint(1, max(2, (V - 1) // k), (T, k), generator=g, device=_DEV)
    gaps[:, 0] = 0
    ids = (targets.long()[:, None] + gaps.cumsum(1)) % V
    order = torch.rand(T, k, generator=g, device=_DEV)
    order[:, 0] = torch.where(torch.rand(T, generator=g, device=_DEV) < 0.7, -1.0, order[:, 0])
    ids = ids.gather(1, order.argsort(1))
    scale = 0.5 + 3.0 * torch.rand(T, 1, generator=g, device=_DEV)
    logits = (scale * torch.randn(T, k, generator=g, device=_DEV)).sort(1, descending=True).values
    mass = 0.7 + 0.2999 * torch.rand(T, 1, generator=g, device=_DEV)
    logp = torch.log_softmax(logits, 1) + mass.log()
    length = torch.full((T, 1), k, device=_DEV)
    u = torch.rand(T, 1, generator=g, device=_DEV)
    length = torch.where(u < 3 / 32, torch.clamp(length // 2, min=1), length)
    length = torch.where(u < 1 / 32, torch.zeros_like(length), length)
    beyond = torch.arange(k, device=_DEV)[None, :] >= length
    ids = ids.masked_fill(beyond, -1)
    logp = logp.masked_fill(beyond, -math.inf)
    weights = (torch.rand(T, generator=g, device=_DEV) < 0.9).float()      # some tokens are not trained on
    return ids.to(torch.int32).contiguous(), logp.float().contiguous(), weights


def prepare(case, seed):
    g = torch.Generator(device=_DEV).manual_seed(int(seed))
    state = dict(case=dict(case))
    if case["op"] == "logits":
        T, V = case["T"], case["V"]
        x = torch.empty(T, V + case["pad"], device=_DEV, dtype=_DTYPE[case["dtype"]])
        logits = x[:, :V]
        for t0 in range(0, T, 512):
            n = min(512, T - t0)
            z = 2.5 * torch.randn(n, V, generator=g, device=_DEV)
            z += 6.0 * torch.rand(n, 1, generator=g, device=_DEV) * (z > 6.0)
            if case["masked"] > 0:
                under = torch.rand(n, 1, generator=g, device=_DEV) < case["masked"]
                few = torch.rand(n, 1, generator=g, device=_DEV) < 0.25          # a grammar that leaves a handful
                keep = torch.where(few, 6.0 / V, 0.2)
                z = z.masked_fill(under & (torch.rand(n, V, generator=g, device=_DEV) >= keep), -math.inf)
            logits[t0:t0 + n] = z.to(logits.dtype)
        # the sampled token is one that the mask leaves, where it leaves any
        noise = torch.rand(T, 64, generator=g, device=_DEV)
        at = torch.randint(0, V, (T, 64), generator=g, device=_DEV)
        noise = torch.where(torch.isinf(logits.gather(1, at)), -1.0, noise)
        best = logits.argmax(1)
        sampled = at.gather(1, noise.argmax(1, keepdim=True))[:, 0]
        state["targets"] = torch.where(noise.amax(1) < 0, best, sampled).to(torch.int32)
        state["logits"] = logits
        return state
    hidden, W, targets = _head_inputs(case, g, eight_bit=case["op"] == "scores")
    state.update(hidden=hidden, W=W, targets=targets)
    T = case["T"]
    if case["op"] == "scores_grad":
        state["d_logp"] = torch.randn(T, generator=g, device=_DEV) / T
        state["d_entropy"] = 0.3 * torch.randn(T, generator=g, device=_DEV) / T
    if case["op"] == "distill":
        state["teacher_ids"], state["teacher_logp"], state["weights"] = _teacher_lists(case, g, targets)
    return state


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_top(a, k):
    """ids of the k largest of each row of a, ties to the lowest id."""
    V = a.shape[1]
    bits = (a + 0.0).view(torch.int32)
    rank = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).to(torch.int64)
    key = (rank << 32) | (V - torch.arange(V, device=a.device))
    return torch.topk(key, k, dim=1).indices


def _softmax_parts(z):
    """z - max, its exponential, and the sum of that in 64 bits: next to probability one the others are what counts."""
    m = z.amax(1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    t = z - m
    e = t.exp()
    return m, t, e, e.sum(1, keepdim=True, dtype=torch.float64)


def _plain_entropy(t, e, s):
    # p log p of an entry that the mask removed is zero
    return s.log() - torch.where(e > 0, e * t, torch.zeros_like(e)).sum(1, keepdim=True, dtype=torch.float64) / s


def _plain_scores(a, kappa, targets, k):
    m, t, e, s = _softmax_parts(a * kappa)
    lse = m + s.log()
    # a row whose mask leaves nothing: no token has a probability, and there is nothing to be uncertain about
    nothing = torch.isneginf(lse)
    logp = (t.gather(1, targets.long()[:, None]) - s.log()).masked_fill(nothing, -math.inf)
    out = dict(logp=logp[:, 0].float(), entropy=_plain_entropy(t, e, s).masked_fill(nothing, 0.0)[:, 0].float(),
               lse=lse[:, 0].float())
    if k:
        ids = _plain_top(a, k)
        out["top_ids"] = ids.to(torch.int32)
        out["top_logp"] = (t.gather(1, ids) - s.log()).masked_fill(nothing, -math.inf).float()
    return out


def _plain_scores_grad(state):
    c = state["case"]
    h, w, y = state["hidden"].float(), state["W"].float(), state["targets"].long()
    _, t, e, s = _softmax_parts((h @ w.t()) * c["kappa"])
    entropy = _plain_entropy(t, e, s)
    logp_all = t - s.log().float()
    p = e / s.float()
    g, ge = state["d_logp"][:, None], state["d_entropy"][:, None]
    dz = -p * (g + ge * (logp_all + entropy.float()))
    at_y = (t.gather(1, y[:, None]) - s.log())
    # at the token itself 1 - p, which 32 bits lose where p is near one
    dz.scatter_(1, y[:, None], (-torch.expm1(at_y) * g - at_y.exp() * ge * (at_y + entropy)).float())
    dz *= c["kappa"]
    return dict(logp=at_y[:, 0].float(), entropy=entropy[:, 0].float(),
                d_hidden=(dz @ w).to(state["hidden"].dtype), d_W=(dz.t() @ h).to(state["W"].dtype))


def _plain_distill(state):
    c = state["case"]
    kappa, mode = c["kappa"], c["mode"]
    h, w = state["hidden"].float(), state["W"].float()
    _, t, e, s = _softmax_parts((h @ w.t()) * kappa)
    on = state["teacher_ids"] >= 0
    ids = state["teacher_ids"].long().clamp(min=0)
    logq = state["teacher_logp"].double()
    if mode == "renorm":
        top = logq.amax(1, keepdim=True)
        logq = logq - torch.where(torch.isinf(top), torch.zeros_like(top), top)
        logq = logq - logq.exp().sum(1, keepdim=True).log()
    logq = torch.where(on, logq, -math.inf)
    q = logq.exp()
    Q = q.sum(1, keepdim=True)
    logp = t.gather(1, ids) - s.log()
    kl = torch.where(q > 0, q * (logq - logp), torch.zeros_like(q)).sum(1, keepdim=True)
    p = (e / s.float()) * torch.ones_like(e).scatter_add_(1, ids, torch.where(on, -1.0, 0.0))     # zero on the list
    c_on = c_off = Q
    if mode == "tail":
        rest_p = p.sum(1, keepdim=True, dtype=torch.float64)
        rest_q = (1.0 - Q).clamp(min=0.0)
        some = rest_q > 0
        kl = kl + torch.where(some, rest_q * (rest_q.log() - rest_p.log()), torch.zeros_like(rest_q))
        c_on, c_off = torch.ones_like(Q), torch.where(some, 1.0 - rest_q / rest_p, torch.ones_like(Q))
    # a token whose list is empty has nothing to learn from
    some_list = on.any(1, keepdim=True)
    kl = torch.where(some_list, kl, torch.zeros_like(kl))
    scale = state["weights"].double()[:, None] * some_list / c["T"]
    dz = p * (kappa * scale * c_off).float()
    dz.scatter_add_(1, ids, torch.where(on, kappa * scale * (c_on * logp.exp() - q), torch.zeros_like(q)).float())
    loss = (state["weights"].double() * kl[:, 0]).sum() / c["T"]
    return dict(loss=loss.float(), kl=kl[:, 0].float(), d_hidden=(dz @ w).to(state["hidden"].dtype),
                d_W=(dz.t() @ h).to(state["W"].dtype))


def _plain(state):
    c = state["case"]
    if c["op"] == "scores":
        return _plain_scores(state["hidden"].float() @ state["W"].float().t(), c["kappa"], state["targets"], c["k"])
    if c["op"] == "logits":
        return _plain_scores(state["logits"].float(), c["kappa"], state["targets"], c["k"])
    return _plain_scores_grad(state) if c["op"] == "scores_grad" else _plain_distill(state)


# ------------------------------------------------------------------------------------------------ the framework's calls
def _own(state):
    import paper_2507_19766_b200 as U
    c = state["case"]
    if c["op"] == "logits":
        o = U.logits_scores(state["logits"], state["targets"], top_k=c["k"], inv_temperature=c["kappa"])
        return _scores_dict(o, c["k"])
    more = dict(dw_dtype=c["dtype"]) if c["op"] != "scores" else dict(top_k=c["k"])
    if c["op"] == "distill":
        more.update(top_k=c["k"], distill_mode=c["mode"])
    p = U.HeadParams(T=c["T"], H=c["H"], V=c["V"], dtype=c["dtype"], inv_temperature=c["kappa"], **more)
    h, w = state["hidden"], state["W"]
    if c["op"] == "scores":
        return _scores_dict(U.token_scores(p, h, w, state["targets"]), c["k"])
    workspace = U.alloc_head_workspace(p, h.device)
    if c["op"] == "scores_grad":
        o = U.token_scores(p, h, w, state["targets"], workspace=workspace)
        d_hidden, d_W = U.token_scores_bwd(p, h, w, state["targets"], o, state["d_logp"], state["d_entropy"],
                                           workspace=workspace)
        return dict(logp=o.logp, entropy=o.entropy, d_hidden=d_hidden, d_W=d_W)
    o = U.distill_fwd(p, h, w, state["teacher_ids"], state["teacher_logp"], state["weights"], workspace=workspace)
    d_hidden, d_W = U.distill_bwd(p, h, w, state["teacher_ids"], o, workspace=workspace)
    return dict(loss=o.loss[0], kl=o.kl, d_hidden=d_hidden, d_W=d_W)


def _scores_dict(o, k):
    out = dict(logp=o.logp, entropy=o.entropy, lse=o.lse)
    if k:
        out["top_ids"], out["top_logp"] = o.top_ids, o.top_logp
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ work and 64-bit values
def work(case):
    T, V = case["T"], case["V"]
    size = {BF16: 2, F16: 2, F32: 4}[case["dtype"]]
    k = case.get("k", 0)
    if case["op"] == "logits":
        return dict(bytes=T * V * size + T * (16 + 8 * k), flops=6.0 * T * V)
    H = case["H"]
    operands = size * (T + V) * H
    if case["op"] == "scores":
        return dict(bytes=operands + T * (16 + 8 * k), flops=2.0 * T * H * V)
    return dict(bytes=2 * operands + T * (16 + 8 * k), flops=6.0 * T * H * V)


def _rows(T, V):
    """Row ranges whose 64-bit logits take about a gigabyte."""
    n = max(1, min(T, 2 ** 27 // V))
    return [(t, min(T, t + n)) for t in range(0, T, n)]


def _exact_scores(logits_of, targets, T, V, kappa, k):
    parts = []
    for a, b in _rows(T, V):
        z = logits_of(a, b) * kappa
        logp_all = torch.log_softmax(z, 1)
        logp = logp_all.gather(1, targets[a:b].long()[:, None])[:, 0]
        entropy, nothing = torch.special.entr(logp_all.exp()).sum(1), torch.isneginf(z).all(1)
        part = dict(logp=logp.masked_fill(nothing, -math.inf), entropy=entropy.masked_fill(nothing, 0.0), lse=torch.logsumexp(z, 1))
        if k:
            part["top_logp"] = torch.topk(logp_all, k, 1).values.masked_fill(nothing[:, None], -math.inf)
        parts.append(part)
    out = {n: torch.cat([q[n] for q in parts]) for n in parts[0]}
    if k:
        out["top_ids"] = None       # whole numbers: the two sides are compared with each other
    return out


def _exact_grad(case, state, loss_of):
    """Sum over row ranges of the outputs of loss_of(z, a, b) -> (loss, values) and of the loss's gradients."""
    T, V = case["T"], case["V"]
    W = state["W"].double()
    d_W, d_h, total, values = torch.zeros_like(W), [], 0.0, []
    for a, b in _rows(T, V):
        h = state["hidden"][a:b].double()
        z = ((h @ W.t()) * case["kappa"]).requires_grad_(True)
        loss, got = loss_of(z, a, b)
        (dz,) = torch.autograd.grad(loss, z)
        dz = dz * case["kappa"]
        d_h.append(dz @ W)
        d_W += dz.t() @ h
        total = total + loss.detach()
        values.append({n: v.detach() for n, v in got.items()})
        del z, dz, loss, got
    out = {n: torch.cat([v[n] for v in values]) for n in values[0]}
    return total, dict(out, d_hidden=torch.cat(d_h), d_W=d_W)


def exact(case, seed):
    state = prepare(case, seed)
    T, V, kappa, k = case["T"], case["V"], case["kappa"], case.get("k", 0)
    if case["op"] == "logits":
        return _exact_scores(lambda a, b: state["logits"][a:b].double(), state["targets"], T, V, kappa, k)
    if case["op"] == "scores":
        W = state["W"].double()
        return _exact_scores(lambda a, b: state["hidden"][a:b].double() @ W.t(), state["targets"], T, V, kappa, k)
    if case["op"] == "scores_grad":
        def loss_of(z, a, b):
            logp_all = torch.log_softmax(z, 1)
            logp = logp_all.gather(1, state["targets"][a:b].long()[:, None])[:, 0]
            entropy = -(logp_all.exp() * logp_all).sum(1)
            loss = (state["d_logp"][a:b].double() * logp + state["d_entropy"][a:b].double() * entropy).sum()
            return loss, dict(logp=logp, entropy=entropy)
        return _exact_grad(case, state, loss_of)[1]

    def distill_loss(z, a, b):
        logp_all = torch.log_softmax(z, 1)
        ids, l = state["teacher_ids"][a:b].long(), state["teacher_logp"][a:b].double()
        listed_ids = ids >= 0
        safe = torch.where(listed_ids, l, torch.full_like(l, -1e4))
        logq = torch.log_softmax(safe, 1) if case["mode"] == "renorm" else safe
        q = torch.where(listed_ids, logq.exp(), torch.zeros_like(l))
        kl = (q * (logq - logp_all.gather(1, ids.clamp(min=0)))).sum(1)
        if case["mode"] == "tail":
            hit = torch.zeros_like(z, dtype=torch.bool)
            hit[torch.arange(b - a, device=z.device)[:, None].expand_as(ids)[listed_ids], ids[listed_ids]] = True
            rest_logp = torch.logsumexp(logp_all.masked_fill(hit, -math.inf), 1)
            rest_q = 1.0 - q.sum(1)
            kl = kl + torch.where(rest_q > 0, rest_q * (rest_q.clamp(min=1e-300).log() - rest_logp), torch.zeros_like(rest_q))
        kl = torch.where(listed_ids.any(1), kl, torch.zeros_like(kl))
        return (state["weights"][a:b].double() * kl).sum() / T, dict(kl=kl)

    total, out = _exact_grad(case, state, distill_loss)
    return dict(out, loss=total)
