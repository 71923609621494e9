"""Plain 64-bit forms of the scoring and distillation operators for the tests, and bounds for what the kernels'
arithmetic may add.

Bounds.  A rounding to a type is off by at most eps/2 relative (bf16 2^-8, float32 2^-24).  A logit is a sum of H
products in float32: its error is at most H 2^-23 sum_h |h W| kappa (one rounding or truncation per addition), E
below.  lse and the log-prob of an entry carry E each; ex2 and the float32 sums of positive terms add about 2^-20
relative to a sum, i.e. 2^-20 absolute to its logarithm; values are rounded to float32 at the end.
"""
import math

import torch


def logits64(hidden, W, kappa):
    return kappa * (hidden.double() @ W.double().t())


def logit_error(hidden, W, kappa):
    """E [T]: bound of the error of a row's logits."""
    H = hidden.shape[1]
    return kappa * H * 2.0 ** -23 * (hidden.double().abs() @ W.double().abs().t()).amax(1)


def scores64(z, targets=None, k=0):
    """From z = kappa a [T, V] in float64: dict of logp, entropy, lse, top_ids, top_logp.  A row of -inf only has
    lse = logp = -inf and entropy 0; ids by (value falling, id rising), NaN never chosen."""
    T, V = z.shape
    m = z.amax(1, keepdim=True)
    m = torch.where(torch.isinf(m) & (m < 0), torch.zeros_like(m), m)
    ln_s = torch.logsumexp(z - m, 1)             # beside a maximum of -10^38 the sum's logarithm would be lost
    lse = m[:, 0] + ln_s
    nothing = torch.isneginf(lse)
    logp_all = torch.where(nothing[:, None], torch.full_like(z, -math.inf), z - m - ln_s[:, None])
    p = logp_all.exp()
    ent = -(torch.where(p > 0, p * logp_all, torch.where(torch.isnan(p), p, torch.zeros_like(p)))).sum(1)
    out = dict(lse=lse, entropy=ent, logp_all=logp_all)
    if targets is not None:
        out["logp"] = logp_all.gather(1, targets.long()[:, None])[:, 0]
    if k:
        # stable: equal values keep the order of their ids
        order = torch.sort(torch.where(torch.isnan(z), torch.full_like(z, -math.inf), z), dim=1, descending=True, stable=True).indices
        out["top_ids"] = order[:, :k].to(torch.int32)
        out["top_logp"] = logp_all.gather(1, order[:, :k])
    return out


def scores_dz64(z, targets, kappa, d_logp, d_entropy):
    """(dz, size): the gradient to the logits a, and the sum of the magnitudes of its terms."""
    s = scores64(z, targets)
    logp, H = s["logp_all"], s["entropy"][:, None]
    p = logp.exp()
    dz = torch.zeros_like(z)
    size = torch.zeros_like(z)
    if d_logp is not None:
        g = d_logp.double()[:, None]
        hot = torch.zeros_like(z).scatter_(1, targets.long()[:, None], 1.0)
        dz += g * (hot - p)
        size += g.abs() * (hot + p)
    if d_entropy is not None:
        e = d_entropy.double()[:, None]
        dz -= e * p * (logp + H)
        size += e.abs() * p * (logp.abs() + H)
    return kappa * dz, kappa * size


def distill64(z, ids, teacher, weights, mode, kappa=1.0, teacher_kappa=1.0, N=None):
    """dict of loss, kl [T], dz [T, V] (to the logits a) and size (magnitude of its terms).  Ids outside [0, V) are
    no entries; an id listed twice is two entries."""
    T, V = z.shape
    N = N or T
    kl, dz, size = torch.zeros(T, dtype=torch.float64), torch.zeros(T, V, dtype=torch.float64), torch.zeros(T, V, dtype=torch.float64)
    z, ids, teacher = z.cpu(), ids.cpu().long(), teacher.cpu().double()
    w = torch.ones(T, dtype=torch.float64) if weights is None else weights.cpu().double()
    for t in range(T):
        ok = (ids[t] >= 0) & (ids[t] < V)
        if not bool(ok.any()):
            continue
        i, l = ids[t][ok], teacher[t][ok]
        if mode == "renorm":
            l = torch.log_softmax(l * teacher_kappa, 0)
        q = l.exp()
        logp = torch.log_softmax(z[t], 0)
        p = logp.exp()
        on = torch.zeros(V, dtype=torch.bool)
        on[i] = True
        kl[t] = torch.where(q > 0, q * (l - logp[i]), torch.zeros_like(q)).sum()
        Q = q.sum()
        d = -torch.zeros(V, dtype=torch.float64).index_add_(0, i, q)
        if mode == "tail":
            rest_q = (1.0 - Q).clamp(min=0.0)
            if rest_q > 0:
                rest_logp = torch.logsumexp(logp[~on], 0)
                kl[t] += rest_q * (rest_q.log() - rest_logp)
                d = d + torch.where(on, p, p * (1.0 - rest_q / rest_logp.exp()))
            else:
                d = d + p
            sz = d.abs() + torch.where(on, p, p * (1.0 + (rest_q / rest_logp.exp() if rest_q > 0 else 0.0)))
        else:
            d = d + Q * p
            sz = d.abs() + Q * p
        if w[t] != 0:
            dz[t] = kappa * w[t] / N * d
            size[t] = kappa * abs(w[t]) / N * (sz + torch.zeros(V, dtype=torch.float64).index_add_(0, i, q))
    loss = (torch.where(w != 0, w * kl, torch.zeros_like(kl))).sum() / N
    return dict(loss=loss, kl=kl, dz=dz, size=size)


def check_grads(d_hidden, d_W, dz, size, hidden, W, E, tensor_path, dw_dtype, d_W_before=None):
    """Both gradients against dz W and dz^T hidden, element by element.  A term of dz is relatively off by the error
    of its log-prob (2 E + 2^-19: twice a logit's error, ex2, the saved float32 numbers) and on the tensor path by
    the rounding of dz to bf16; the products are added in float32 (one rounding per addition)."""
    dz, size, h, w = dz.cpu(), size.cpu(), hidden.double().cpu(), W.double().cpu()
    T, V = dz.shape
    rel = (2.0 * E.cpu()[:, None] + 2.0 ** -19) * size + (2.0 ** -8 if tensor_path else 2.0 ** -23) * dz.abs()
    half = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}

    def close(got, want, slack, what):
        got = got.double().cpu()
        bound = slack * (1 + 2.0 ** -8) + half[what[1]] * want.abs() + 1e-30
        bad = (got - want).abs() > bound
        assert not bool(bad.any()), (what, float(((got - want).abs() / bound).max()))

    close(d_hidden, dz @ w, rel @ w.abs() + V * 2.0 ** -23 * (dz.abs() @ w.abs()), ("d_hidden", d_hidden.dtype))
    want = dz.t() @ h
    slack = rel.t() @ h.abs() + T * 2.0 ** -23 * (dz.abs().t() @ h.abs())
    if d_W_before is not None:
        want = want + d_W_before.double().cpu()
    close(d_W, want, slack, ("d_W", d_W.dtype))


def check_low_temperature(out, z, targets, k):
    """Scores of exact logits at a large scale, where only lse may round like the logits themselves.  A difference to the
    maximum is exact but for the scale's rounding and its own (2^-23 relative); sums of positive terms and their
    logarithm add 2^-20."""
    ref = scores64(z, targets, k)

    def close(got, want, what):
        err = (got.double() - want).abs()
        assert bool((err <= 2.0 ** -19 + 2.0 ** -21 * want.abs()).all()), (what, float(err.max()))
    close(out.logp, ref["logp"], "logp")
    close(out.top_logp, ref["top_logp"], "top_logp")
    spread = (ref["logp_all"].exp() * (ref["logp_all"] + ref["entropy"][:, None]).abs()).sum(1)
    err = (out.entropy.double() - ref["entropy"]).abs()
    assert bool((err <= (2.0 ** -19 + 2.0 ** -21 * ref["entropy"]) * (2 + spread)).all()), ("entropy", float(err.max()))
    assert torch.equal(out.top_ids.cpu(), ref["top_ids"].cpu())
    assert bool(((out.lse.double() - ref["lse"]).abs() <= 2.0 ** -23 * ref["lse"].abs()).all())
