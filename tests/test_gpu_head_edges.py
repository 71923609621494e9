"""Edges of token scoring and distillation: teacher lists that hold more or all of the probability, NaN weights beside
alternatives, rows whose gradients are zero, vocabularies of millions, the planes of float32 operands one by one."""
import math

import pytest
import torch

import paper_2507_19766_b200 as U
from paper_2507_19766_b200 import binding as B
from tests import head_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
PATHS = [("bf16", "auto"), ("bf16", "simt"), ("f32", "simt"), ("f32", "tensor")]


def operands(T, H, V, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    W, hidden = torch.randn(V, H, generator=g) / 8, torch.randn(T, H, generator=g)
    targets = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    return hidden.to(DT[dtype]).to(DEV), W.to(DT[dtype]).to(DEV), targets.to(DEV)


# ------------------------------------------------------------------------------------------------ teacher lists
def tail_loss(z, ids, teacher, weights, N):
    """Mode tail in 64 bits: (loss, kl [T]).  The remainder 1 - sum q is an event of its own where there is one and the
    student has entries for it."""
    kl = []
    for t in range(z.shape[0]):
        ok = ids[t] >= 0
        i, l = ids[t][ok], teacher[t][ok]
        logp = torch.log_softmax(z[t], 0)
        q = l.exp()
        k = (q * (l - logp[i])).sum()
        off = torch.ones(z.shape[1], dtype=torch.bool)
        off[i] = False
        rest = 1.0 - q.sum()
        if bool(off.any()) and float(rest) > 0:
            k = k + rest * (rest.log() - torch.logsumexp(logp[off], 0))
        kl.append(k)
    kl = torch.stack(kl)
    return (weights * kl).sum() / N, kl


def check_tail(p, hidden, W, ids, teacher, weights, tensor_path):
    """Loss and gradients against the loss above and its derivative by autograd."""
    ws = U.alloc_head_workspace(p, DEV)
    out = U.distill_fwd(p, hidden, W, ids, teacher, weights, workspace=ws)
    d_h, d_W = U.distill_bwd(p, hidden, W, ids, out, workspace=ws)
    assert B.check_status(ws) == B.OK
    kappa = p.inv_temperature
    z = R.logits64(hidden, W, kappa).cpu().requires_grad_(True)
    i, l, w = ids.cpu().long(), teacher.cpu().double(), weights.cpu().double()
    loss, kl = tail_loss(z, i, l, w, p.T)
    (dz,) = torch.autograd.grad(loss, z)
    Q = torch.where(i >= 0, l.exp(), torch.zeros_like(l)).sum(1)
    mass = Q.clamp(min=1.0)                        # what the log-probs of a row are weighted with
    E = R.logit_error(hidden, W, kappa).cpu()
    tol = (2 * E + 2.0 ** -19 + 2.0 ** -22 * z.detach().abs().amax(1)) * mass
    kl, loss = kl.detach(), loss.detach()
    assert bool(((out.kl.double().cpu() - kl).abs() <= 2 * tol + 2.0 ** -23 * kl.abs()).all()), (out.kl.cpu() - kl).abs().max()
    slack = float(((2 * tol + 2.0 ** -23 * kl.abs()) * w).sum() / p.T + 2.0 ** -23 * loss.abs())
    assert abs(float(out.loss[0]) - float(loss)) <= slack
    # the terms of dz: the list's mass times p, q on the list, the remainder's share of p off it
    prob = torch.softmax(z.detach(), 1)
    on = torch.zeros_like(prob).scatter_add_(1, i.clamp(min=0), (i >= 0).double()) > 0
    q = torch.zeros_like(prob).scatter_add_(1, i.clamp(min=0), torch.where(i >= 0, l.exp(), torch.zeros_like(l)))
    rest_p = torch.where(on, torch.zeros_like(prob), prob).sum(1)
    share = torch.where(rest_p > 0, (1 - Q).clamp(min=0.0) / rest_p, torch.zeros_like(Q))
    size = mass[:, None] * prob + torch.where(on, q, prob * share[:, None])
    R.check_grads(d_h, d_W, kappa * dz, kappa * w[:, None] / p.T * size, hidden, W, E + 2.0 ** -20, tensor_path, p.dw_dtype)
    return out, d_h, d_W


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("T,H,V,K", [(20, 64, 700, 6), (130, 64, 1200, 9)])
def test_lists_above_one(dtype, path, T, H, V, K):
    """Mode tail, lists whose probabilities add up to more than one (log-probs stored in few bits, or of no distribution):
    nothing is left for the remainder, and the gradient is that of the loss."""
    hidden, W, _ = operands(T, H, V, dtype, seed=T)
    g = torch.Generator().manual_seed(K)
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]).to(torch.int32)
    total = torch.tensor([0.8, 1.003, 1.05, 1.3, 2.5]).repeat(T)[:T]
    teacher = torch.log_softmax(torch.randn(T, K, generator=g), 1) + total.log()[:, None]
    weights = (torch.rand(T, generator=g) < 0.9).float()
    p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=K, distill_mode="tail", kernel_path=path, inv_temperature=0.9)
    check_tail(p, hidden, W, ids.to(DEV), teacher.to(DEV), weights.to(DEV), dtype == "bf16" and path != "simt")


@pytest.mark.parametrize("path", ["simt", "tensor"])
def test_lists_above_one_against_differences(path):
    """The returned loss moves along a direction of (hidden, W) as its gradients say, sum q = 1.3."""
    T, H, V, K = 24, 32, 300, 5
    hidden, W, _ = operands(T, H, V, "f32", seed=3)
    g = torch.Generator().manual_seed(4)
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)])
    teacher = torch.log_softmax(torch.randn(T, K, generator=g), 1) + math.log(1.3)
    p = U.HeadParams(T=T, H=H, V=V, dtype="f32", top_k=K, distill_mode="tail", kernel_path=path)
    dev_ids = ids.to(torch.int32).to(DEV)
    out = U.distill_fwd(p, hidden, W, dev_ids, teacher.to(DEV))
    d_h, d_W = (x.double().cpu() for x in U.distill_bwd(p, hidden, W, dev_ids, out))
    h, w = hidden.double().cpu(), W.double().cpu()
    dh, dw = torch.randn(T, H, generator=g).double(), torch.randn(V, H, generator=g).double() / 8
    eps = 1e-5
    loss = lambda s: float(tail_loss((h + s * dh) @ (w + s * dw).t(), ids, teacher.double(), torch.ones(T).double(), T)[0])
    got, size = float((d_h * dh).sum() + (d_W * dw).sum()), float((d_h * dh).abs().sum() + (d_W * dw).abs().sum())
    # float32 gradients (a few 10^-6 of the sum of magnitudes), the difference's own eps^2
    assert abs(got - (loss(eps) - loss(-eps)) / (2 * eps)) <= 1e-5 * size


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("T,V", [(20, 40), (20, 128), (130, 96), (70, 1)])
def test_lists_of_the_whole_vocabulary(dtype, path, T, V):
    """Mode tail, lists that hold every id and add up to a little less than one (a softmax stored in float32), to a tenth less,
    or to more: the student has no entry for a remainder, and the loss is that of the list."""
    hidden, W, _ = operands(T, 64, V, dtype, seed=T + V)
    g = torch.Generator().manual_seed(V)
    ids = torch.stack([torch.randperm(V, generator=g) for _ in range(T)]).to(torch.int32).to(DEV)
    total = torch.tensor([1 - 1e-6, 0.9, 1.1]).double().repeat(T)[:T]
    teacher = (torch.log_softmax(torch.randn(T, V, generator=g).double(), 1) + total.log()[:, None]).float().to(DEV)
    p = U.HeadParams(T=T, H=64, V=V, dtype=dtype, top_k=V, distill_mode="tail", kernel_path=path)
    out, d_h, d_W = check_tail(p, hidden, W, ids, teacher, torch.ones(T, device=DEV), dtype == "bf16" and path != "simt")
    assert bool(torch.isfinite(out.loss).all()) and bool(torch.isfinite(out.kl).all())


# ------------------------------------------------------------------------------------------------ alternatives
def test_nan_columns_beside_alternatives():
    """Eight adjacent NaN rows of W in every stretch of 128 columns, and one logit per stretch far above the others: the NaN
    columns stand for no entry, so the alternatives are those of the path that looks at every logit."""
    T, H, V, k = 70, 64, 2560, 32
    g = torch.Generator().manual_seed(12)
    hidden, W = torch.randint(1, 3, (T, H), generator=g).float(), torch.randint(-3, 4, (V, H), generator=g).float() / 8
    W[5::128] = 2.0                                          # far above: 2 sum h, against noise of 0.25 sqrt(H) h
    for first in range(120, V, 128):
        W[first:first + 8] = float("nan")
    for dtype in ("bf16", "f32"):
        h, w = hidden.to(DT[dtype]).to(DEV), W.to(DT[dtype]).to(DEV)
        ids = [U.token_scores(U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=k, kernel_path=path), h, w).top_ids.cpu()
               for path in ("tensor", "simt")]
        ref = R.scores64(R.logits64(h, w, 1.0), None, k)     # all sums are exact
        assert torch.equal(ids[1], ref["top_ids"].cpu())
        assert torch.equal(ids[0], ref["top_ids"].cpu())


# ------------------------------------------------------------------------------------------------ failure reports
@pytest.mark.parametrize("T,V", [(1, 200_000), (3, 5000), (700, 20_000)])
def test_rows_report_a_wait_that_ran_out(T, V):
    """The row kernel with copies that are never issued: its waits give up after their limit, the kernel returns, the status
    word says so, and no number is made of what shared memory happened to hold."""
    logits = torch.randn(T, V, generator=torch.Generator(device=DEV).manual_seed(V), device=DEV)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    U.logits_scores(logits, top_k=8)                         # leaves numbers in shared memory
    out = U.head.selftest_logits_wait(logits, 8, ws, 100_000)
    assert B.check_status(ws) == -5
    assert bool(torch.isnan(out.lse).all())
    assert bool((out.top_ids == -1).all()) and bool(torch.isnan(out.top_logp).all())
    for bad in (10, 10 ** 12):
        with pytest.raises(U.UlorlError):
            U.head.selftest_logits_wait(logits, 8, ws, bad)
    again = U.logits_scores(logits, top_k=8)                 # and the next call is an ordinary one
    assert torch.equal(again.top_logp, U.logits_scores(logits, top_k=8).top_logp) and bool(torch.isfinite(again.lse).all())


# ------------------------------------------------------------------------------------------------ sizes
@pytest.mark.parametrize("dtype,V", [("bf16", 64 * 65535 + 1), ("f32", 128 * 65535 + 1)])
def test_vocabulary_of_millions_on_cuda_cores(dtype, V):
    """More tiles of d_W than one dimension of a grid other than the first takes."""
    T, H = 2, 8
    g = torch.Generator(device=DEV).manual_seed(1)
    hidden, W = torch.randn(T, H, generator=g, device=DEV).to(DT[dtype]), torch.randn(V, H, generator=g, device=DEV).to(DT[dtype])
    targets = torch.tensor([3, V - 1], dtype=torch.int32, device=DEV)
    p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, kernel_path="simt")
    out = U.token_scores(p, hidden, W, targets)
    d = torch.tensor([1.0, -2.0], device=DEV)
    d_h, d_W = U.token_scores_bwd(p, hidden, W, targets, out, d, None)
    dz, size = R.scores_dz64(R.logits64(hidden, W, 1.0), targets, 1.0, d, None)
    R.check_grads(d_h, d_W, dz, size, hidden, W, R.logit_error(hidden, W, 1.0) * 2, False, "f32")


# ------------------------------------------------------------------------------------------------ gradients of scores
@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("which", ["both", "logp", "entropy"])
def test_rows_without_gradients_add_nothing(dtype, path, which):
    """Padding rows with finite hidden states whose logits overflow: scores of NaN, gradients of zero, and nothing of them in
    d_hidden and d_W."""
    T, H, V = 70, 64, 500
    hidden, W, targets = operands(T, H, V, dtype, seed=6)
    pad = torch.arange(T, device=DEV) % 5 == 2
    hidden[pad] = 3e38 if dtype == "bf16" else 1e38
    W[::3] = 4.0
    p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, kernel_path=path)
    out = U.token_scores(p, hidden, W, targets)
    assert bool(torch.isnan(out.logp[pad]).any()) and bool(torch.isnan(out.entropy[pad]).all()) and bool(torch.isfinite(out.logp[~pad]).all())
    g = torch.Generator().manual_seed(7)
    d_logp, d_ent = (torch.randn(T, generator=g).to(DEV).masked_fill(pad, 0.0) for _ in range(2))
    d_logp, d_ent = d_logp if which != "entropy" else None, d_ent if which != "logp" else None
    d_h, d_W = U.token_scores_bwd(p, hidden, W, targets, out, d_logp, d_ent)
    assert not bool(d_h[pad].any())
    # the same without the rows
    q = U.HeadParams(T=int((~pad).sum()), H=H, V=V, dtype=dtype, kernel_path=path)
    h, y = hidden[~pad].contiguous(), targets[~pad].contiguous()
    dz, size = R.scores_dz64(R.logits64(h, W, 1.0), y, 1.0, None if d_logp is None else d_logp[~pad], None if d_ent is None else d_ent[~pad])
    R.check_grads(d_h[~pad], d_W, dz, size, h, W, R.logit_error(h, W, 1.0) * (2 + math.log(V)), dtype == "bf16" and path != "simt", "f32")
    assert q.T < T


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("mode", ["raw", "renorm", "tail"])
def test_tokens_that_are_not_trained_on_add_nothing(dtype, path, mode):
    """Padding rows with finite hidden states whose logits overflow, of weight zero or with an empty list."""
    T, H, V, K = 70, 64, 500, 6
    hidden, W, _ = operands(T, H, V, dtype, seed=8)
    W[::3] = 4.0
    g = torch.Generator().manual_seed(9)
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]).to(torch.int32).to(DEV)
    teacher = (torch.log_softmax(torch.randn(T, K, generator=g), 1) - 0.2).to(DEV)
    weights = torch.ones(T, device=DEV)
    light, empty = torch.arange(T, device=DEV) % 5 == 2, torch.arange(T, device=DEV) % 7 == 3
    weights[light] = 0.0
    ids[empty] = -1
    p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=K, distill_mode=mode, kernel_path=path)

    def step():
        out = U.distill_fwd(p, hidden, W, ids, teacher, weights)
        return (out.loss, *U.distill_bwd(p, hidden, W, ids, out))
    want = step()
    hidden[light | empty] = 3e38 if dtype == "bf16" else 1e38
    got = step()
    assert not bool(got[1][light | empty].any())
    assert bool(torch.isfinite(got[0]).all()) and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("level", [40.0, 640.0, 5600.0])
def test_dz_of_large_logits_keeps_its_scale(level):
    """bf16 operands, logits of `level` plus fractions: dz, read back through hidden states of one 1 each, rounds the exact
    values to bf16, with no common factor of a row beside the rounding."""
    T, H, V = 40, 48, 40000
    g = torch.Generator().manual_seed(int(level))
    W, hidden = torch.zeros(V, H), torch.zeros(T, H)
    hidden[:, :2] = 1.0
    hidden[torch.arange(T), 8 + torch.arange(T)] = 1.0
    W[:, 0] = level
    W[:, 1] = torch.randint(0, 8, (V,), generator=g).float() * 2.0 ** -11       # sums are exact: multiples of 2^-11 below 2^13
    W[:, 8:] = torch.randint(0, 256, (V, H - 8), generator=g).float() * 2.0 ** -8
    targets = torch.randint(0, V, (T,), generator=g, dtype=torch.int32).to(DEV)
    h, w = hidden.to(torch.bfloat16).to(DEV), W.to(torch.bfloat16).to(DEV)
    p = U.HeadParams(T=T, H=H, V=V)
    out = U.token_scores(p, h, w, targets)
    d_logp = (torch.rand(T, generator=g) + 0.5).to(DEV)
    _, d_W = U.token_scores_bwd(p, h, w, targets, out, d_logp, None)
    got = d_W[:, 8:].t().double()                            # [T, V]: dz times one
    dz, _ = R.scores_dz64(R.logits64(h, w, 1.0), targets, 1.0, d_logp, None)
    # A value is relatively off by less than 2^-16 before its rounding: exponents of up to 17 that are rounded (2^-20) after the
    # logarithm of the sum (2^-19 with its own rounding), ex2 2^-22, and, where the row's constant is one number, two roundings of
    # a number below 128 (2^-17 ln 2).  Rounding to bf16 keeps the order, so a row's sum lies between those of the two ends.
    eps = 2.0 ** -16
    off = torch.ones_like(dz).scatter_(1, targets.long()[:, None], 0.0)         # the target's column is set on its own
    low, high = (((dz * s).float().to(torch.bfloat16).double() * off).sum(1) for s in (1 + eps, 1 - eps))
    total = (got * off).sum(1)
    assert bool((total >= low).all()) and bool((total <= high).all()), float(((total - (low + high) / 2) / total).abs().max())


# ------------------------------------------------------------------------------------------------ planes of float32 operands
def planes(x):
    out = []
    for _ in range(3):
        out.append(x.float().to(torch.bfloat16).double())
        x = x.double() - out[-1]
    return out


def without(x, y, product):
    """x y as five of the six products of their planes."""
    a, b = planes(x), planes(y)
    return sum(a[i] * b[j] for i, j in ((0, 2), (2, 0), (1, 1), (0, 1), (1, 0), (0, 0)) if (i, j) != product)


@pytest.mark.parametrize("single", ["hidden", "W"])
def test_each_product_of_planes_counts(single):
    """Contractions of one product of two float32 numbers each, where every one of the six products of planes shows: with
    hidden diagonal the logits and d_W are that, with W diagonal the logits and d_hidden."""
    n = 40
    g = torch.Generator().manual_seed(5)
    full, diag = 0.25 + 0.25 * torch.rand(n, n, generator=g), 1.0 + torch.rand(n, generator=g)
    hidden, W = (torch.diag(diag), full) if single == "hidden" else (full, torch.diag(diag))
    hidden, W = hidden.to(DEV), W.to(DEV)
    targets = torch.randint(0, n, (n,), generator=g, dtype=torch.int32).to(DEV)
    d_logp = (torch.rand(n, generator=g) + 0.5).to(DEV)
    p = U.HeadParams(T=n, H=n, V=n, dtype="f32", kernel_path="tensor")
    out = U.token_scores(p, hidden, W, targets)
    d_h, d_W = U.token_scores_bwd(p, hidden, W, targets, out, d_logp, None)
    z = R.logits64(hidden, W, 1.0)
    dz, _ = R.scores_dz64(z, targets, 1.0, d_logp, None)
    far = lambda got, want: float(((got - want).abs() / want.abs()).max())
    # a logit: the last sum cut off by at most 2^-23, the products left out 2 * 2^-24; twice that, for the small sums too
    tol = 2.0 ** -21
    if single == "hidden":
        x, y = hidden.diag()[:, None].cpu(), W.t().cpu()                        # z[t, v] = hidden[t, t] W[v, t]
    else:
        x, y = hidden.cpu(), W.diag()[None, :].cpu()                            # z[t, v] = hidden[t, v] W[v, v]
    assert far(out.norm[:, 0].double(), z.amax(1)) <= tol
    # dz: logits below 1 off by 2^-22 each, ln of the sum (3.7) and its product with log2 e to 2^-22 each with their roundings,
    # an exponent of up to 6 rounded, ex2 2^-22, the sum 2^-22: below 3.5 * 2^-21; then a product as above
    grad = 2.0 ** -19
    if single == "hidden":
        a, b, got = dz.t().cpu(), hidden.diag()[None, :].cpu(), d_W             # d_W[v, h] = dz[h, v] hidden[h, h]
    else:
        a, b, got = dz.cpu(), W.diag()[None, :].cpu(), d_h                      # d_hidden[t, h] = dz[t, h] W[h, h]
    b = b.double().expand_as(a)
    assert far(got.double().cpu(), a * b) <= grad
    # and each of the products is more than that
    for product in ((0, 2), (2, 0), (1, 1), (0, 1), (1, 0)):
        assert far(without(x.double(), y.double(), product).amax(1), (x.double() * y.double()).amax(1)) > tol, product
        assert far(without(a, b, product), a * b) > grad, product


# ------------------------------------------------------------------------------------------------ paths
@pytest.mark.parametrize("T,H,V", [(8, 336, 2993), (100, 64, 900), (60, 128, 4000), (1, 256, 5000)])
@pytest.mark.parametrize("path", ["auto", "simt", "tensor", "simt-tensor", "tensor-simt"])
def test_entropy_gradients_of_peaked_rows(T, H, V, path):
    """float32 operands, gradients of the entropy alone, rows that are sharply peaked: a gradient of 10^-8 is not lost beside
    the difference of the logits of two paths, whichever the two calls take (auto: by the sizes, each for itself)."""
    hidden, W, targets = operands(T, H, V, "f32", seed=T + V)
    g = torch.Generator().manual_seed(3)
    rows = torch.arange(T) % 3 != 1
    hidden[rows] += (W[targets.long()] * (64.0 * 24 / H))[rows]
    d_ent = torch.randn(T, generator=g).to(DEV)
    p, q = (U.HeadParams(T=T, H=H, V=V, dtype="f32", kernel_path=x) for x in (path.split("-")[0], path.split("-")[-1]))
    out = U.token_scores(p, hidden, W, targets)
    d_h, d_W = U.token_scores_bwd(q, hidden, W, None, out, None, d_ent)
    z = R.logits64(hidden, W, 1.0)
    dz, size = R.scores_dz64(z, targets, 1.0, None, d_ent)
    assert float(R.scores64(z, targets)["entropy"].min()) < 1e-5
    R.check_grads(d_h, d_W, dz, size, hidden, W, R.logit_error(hidden, W, 1.0) * (2 + math.log(V)), False, "f32")


# ------------------------------------------------------------------------------------------------ many calls
@pytest.mark.parametrize("T,V,k,dtype", [(4909, 60244, 31, torch.float32), (4096, 60001, 8, torch.bfloat16), (149, 400_000, 4, torch.float16)])
def test_long_rows_are_read_once_and_whole(T, V, k, dtype):
    """Rows of many batches, more blocks than the GPU runs at once: every call sees the same numbers, bit for bit."""
    z = torch.randn(T, V, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(dtype)
    y = torch.zeros(T, dtype=torch.int32, device=DEV)
    first = U.logits_scores(z, y, top_k=k)
    values = torch.sort(z, dim=1, descending=True).values[:, :k] if T * V < 3e8 else torch.topk(z, k, dim=1).values
    assert torch.equal(z.gather(1, first.top_ids.long()), values)
    for _ in range(100):
        out = U.logits_scores(z, y, top_k=k)
        for name in ("lse", "logp", "entropy", "top_ids", "top_logp"):
            assert torch.equal(getattr(out, name), getattr(first, name)), name
