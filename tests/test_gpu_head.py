"""Token scores, their gradients and distillation on the LM head against plain 64-bit forms."""
import math

import pytest
import torch

import paper_2507_19766_b200 as U
from paper_2507_19766_b200 import binding as B
from tests import head_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def operands(T, H, V, dtype, seed, spread=1.0, grid=False):
    g = torch.Generator().manual_seed(seed)
    W = torch.randn(V, H, generator=g) / 8
    hidden = spread * torch.randn(T, H, generator=g)
    targets = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    if T > 2:                                     # peaked rows: probability next to one at the target
        n = T // 3
        hidden[:n] += W[targets[:n].long()] * (64.0 * 24 / H)
    if grid:                                      # every sum exact: logits are the same in any order of addition
        W, hidden = torch.clamp(torch.round(W * 16), -8, 8) / 16, torch.clamp(torch.round(hidden * 4), -12, 12) / 4
    return hidden.to(DT[dtype]).to(DEV), W.to(DT[dtype]).to(DEV), targets.to(DEV)


def close(got, want, bound, what):
    got, want = got.double().cpu(), want.double().cpu()
    bound = (bound if torch.is_tensor(bound) else torch.tensor(bound)).double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(torch.isinf(got), torch.isinf(want)) and bool((got == want)[torch.isinf(want)].all()), what
    d = torch.where(torch.isfinite(want), (got - want).abs(), torch.zeros_like(want))
    assert bool((d <= bound).all()), (what, float((d / bound).max()))


def check_scores(out, hidden, W, targets, k, kappa, exact_ids):
    z = R.logits64(hidden, W, kappa)
    ref = R.scores64(z, targets, k)
    E = R.logit_error(hidden, W, kappa)
    mag = z.abs().amax(1)
    tol = 2 * E + 2.0 ** -20 + 2.0 ** -22 * mag           # two logits, a sum's logarithm, roundings of z and lse
    close(out.lse, ref["lse"], tol, "lse")
    if targets is not None:
        close(out.logp, ref["logp"], tol, "logp")
    # |dH| <= sum p |dlogp| (1 + |log p + H|): the derivative of the entropy to the logits
    spread = (ref["logp_all"].exp() * (ref["logp_all"] + ref["entropy"][:, None]).abs()).sum(1)
    close(out.entropy, ref["entropy"], tol * (1 + spread) + 2.0 ** -20 * (1 + ref["entropy"]), "entropy")
    if k:
        close(out.top_logp, ref["top_logp"], tol[:, None], "top_logp")
        if exact_ids:
            assert torch.equal(out.top_ids.cpu(), ref["top_ids"].cpu())
        else:                                             # near ties may swap: each id's own value stands at its place
            ids = out.top_ids.long()
            assert bool(((ids >= 0) & (ids < W.shape[0])).all())
            close(ref["logp_all"].gather(1, ids), ref["top_logp"], 2 * tol[:, None], "values at the ids")
            assert all(len(set(r)) == k for r in ids.cpu().tolist())


# sizes: one token, tile edges of 128 / 256 rows and 256 columns, a vocabulary of one entry, of less than a chunk
SIZES = [(1, 64, 1000, 5), (16, 72, 20001, 3), (17, 128, 2500, 20), (33, 64, 40003, 32), (64, 200, 3000, 8), (65, 200, 3000, 8), (3, 8, 1, 1), (2, 8, 7, 7), (5, 72, 31, 8), (127, 64, 255, 9), (129, 136, 257, 32),
         (300, 256, 4099, 20), (257, 512, 2048, 0), (700, 64, 20000, 32)]


@pytest.mark.parametrize("T,H,V,k", SIZES)
@pytest.mark.parametrize("dtype,path", [("bf16", "auto"), ("bf16", "simt"), ("f32", "simt"), ("f32", "tensor")])
@pytest.mark.parametrize("grid", [True, False])
def test_token_scores(T, H, V, k, dtype, path, grid):
    kappa = 1.0 if grid else 0.85
    hidden, W, targets = operands(T, H, V, dtype, seed=T + H + V, grid=grid)
    p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=k, inv_temperature=kappa, kernel_path=path)
    ws = U.alloc_head_workspace(p, DEV, backward=False)
    out = U.token_scores(p, hidden, W, targets, workspace=ws)
    assert B.check_status(ws) == B.OK
    check_scores(out, hidden, W, targets, k, kappa, exact_ids=grid)
    # without targets: the same entropy and alternatives, no log-prob
    bare = U.token_scores(p, hidden, W)
    assert bare.logp is None and torch.equal(bare.entropy, out.entropy) and torch.equal(bare.lse, out.lse)
    if k:
        assert torch.equal(bare.top_ids, out.top_ids) and torch.equal(bare.top_logp, out.top_logp)


def test_ties_go_to_the_lowest_id():
    """Logits of a handful of values: whole runs of equal entries cross tiles and splits."""
    g = torch.Generator().manual_seed(5)
    T, H, V, k = 130, 16, 3001, 32
    hidden = torch.randint(-1, 2, (T, H), generator=g).float()
    hidden[0] = 0                                            # every logit equal
    W = torch.randint(-1, 2, (V, H), generator=g).float()
    for dtype, path in (("bf16", "auto"), ("bf16", "simt"), ("f32", "simt"), ("f32", "tensor")):
        h, w = hidden.to(DT[dtype]).to(DEV), W.to(DT[dtype]).to(DEV)
        p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=k, kernel_path=path)
        out = U.token_scores(p, h, w)
        ref = R.scores64(R.logits64(h, w, 1.0), None, k)
        assert torch.equal(out.top_ids.cpu(), ref["top_ids"].cpu())
        assert out.top_ids[0].tolist() == list(range(k))
        assert abs(float(out.entropy[0]) - math.log(V)) <= 2.0 ** -19


def test_peaked_rows_keep_their_digits():
    """1 - p of 10^-6: the log-prob and the entropy keep a relative precision that the difference of a logit and
    lse in float32 does not have."""
    T, H, V = 64, 64, 1024
    W = torch.zeros(V, H)
    W[torch.arange(V), torch.arange(V) % H] = 1.0            # h picks one logit per coordinate: sums are exact
    hidden = torch.zeros(T, H)
    hidden[torch.arange(T), torch.arange(T)] = 1.0
    W[:64] *= torch.linspace(10, 24, 64).to(torch.bfloat16).float()[:, None]
    for dtype, path in (("bf16", "auto"), ("f32", "simt"), ("f32", "tensor")):
        h, w = hidden.to(DT[dtype]).to(DEV), W.to(DT[dtype]).to(DEV)
        targets = torch.arange(T, dtype=torch.int32, device=DEV)
        p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, kernel_path=path)
        out = U.token_scores(p, h, w, targets)
        ref = R.scores64(R.logits64(h, w, 1.0), targets)
        # a term e^(z - max): ex2 2^-22, its argument 2 roundings of about 35 (in units of log2); their sum a few more
        rel = 2.0 ** -22 + 2 * 35 * math.log(2) * 2.0 ** -24 + 20 * 2.0 ** -24
        close(out.logp, ref["logp"], rel * ref["logp"].abs(), "logp")
        close(out.entropy, ref["entropy"], 2 * rel * ref["entropy"].abs() + rel * ref["logp"].abs(), "entropy")


def test_bad_target_is_reported_and_clamped():
    T, H, V = 40, 64, 500
    for dtype in ("bf16", "f32"):
        hidden, W, targets = operands(T, H, V, dtype, seed=3)
        bad = targets.clone()
        bad[3], bad[17] = V, -5
        p = U.HeadParams(T=T, H=H, V=V, dtype=dtype)
        ws = U.alloc_head_workspace(p, DEV)
        out = U.token_scores(p, hidden, W, bad, workspace=ws)
        assert B.check_status(ws) == -6
        U.token_scores_bwd(p, hidden, W, bad, out, out.logp, workspace=ws)
        assert B.check_status(ws) == -6                       # the finding outlives the backward call
        ok = bad.clamp(0, V - 1)
        again = U.token_scores(p, hidden, W, ok, workspace=ws)
        assert B.check_status(ws) == B.OK
        assert torch.equal(out.logp, again.logp)


def test_nan_hidden_row_stays_in_its_row():
    T, H, V, k = 20, 64, 700, 4
    for dtype in ("bf16", "f32"):
        hidden, W, targets = operands(T, H, V, dtype, seed=4)
        clean = U.token_scores(U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=k), hidden, W, targets)
        hidden[7, 3] = float("nan")
        out = U.token_scores(U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=k), hidden, W, targets)
        assert bool(torch.isnan(out.logp[7])) and bool(torch.isnan(out.entropy[7])) and out.top_ids[7].tolist() == [-1] * k
        keep = torch.arange(T, device=DEV) != 7
        for name in ("logp", "entropy", "lse", "top_ids", "top_logp"):
            assert torch.equal(getattr(out, name)[keep], getattr(clean, name)[keep]), name


# ------------------------------------------------------------------------------------------------ gradients of scores
@pytest.mark.parametrize("T,H,V", [(1, 64, 1000), (2, 8, 5), (129, 136, 257), (300, 256, 4099), (1000, 520, 700)])
@pytest.mark.parametrize("dtype,path,dw", [("bf16", "auto", "bf16"), ("bf16", "auto", "f32"), ("bf16", "simt", "f32"), ("f32", "simt", "f32"),
                                           ("f32", "tensor", "f32"), ("f32", "tensor", "bf16")])
@pytest.mark.parametrize("which", ["both", "logp", "entropy"])
def test_token_scores_gradients(T, H, V, dtype, path, dw, which):
    kappa = 0.8
    hidden, W, targets = operands(T, H, V, dtype, seed=T + V)
    g = torch.Generator().manual_seed(T)
    d_logp = torch.randn(T, generator=g).to(DEV) if which != "entropy" else None
    d_ent = torch.randn(T, generator=g).to(DEV) if which != "logp" else None
    if T > 4:                                     # rows that a loss leaves out
        for d in (d_logp, d_ent):
            if d is not None:
                d[2:4] = 0
    p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, inv_temperature=kappa, kernel_path=path, dw_dtype=dw)
    ws = U.alloc_head_workspace(p, DEV)
    out = U.token_scores(p, hidden, W, targets, workspace=ws)
    d_h, d_W = U.token_scores_bwd(p, hidden, W, targets if d_logp is not None else None, out, d_logp, d_ent, workspace=ws)
    assert B.check_status(ws) == B.OK
    dz, size = R.scores_dz64(R.logits64(hidden, W, kappa), targets, kappa, d_logp, d_ent)
    R.check_grads(d_h, d_W, dz, size, hidden, W, R.logit_error(hidden, W, kappa) * (2 + math.log(V)),
                  dtype == "bf16" and path != "simt", dw)
    if T > 4:
        assert not bool(d_h[2:4].any())


@pytest.mark.parametrize("dtype,dw,path", [("bf16", "f32", "auto"), ("bf16", "bf16", "auto"), ("f32", "f32", "simt"), ("f32", "f32", "tensor"),
                                           ("f32", "bf16", "tensor")])
def test_gradients_by_panels_and_accumulated(dtype, dw, path):
    """Several token panels, d_W added into, against one panel: the same sums."""
    T, H, V = 700, 64, 900
    hidden, W, targets = operands(T, H, V, dtype, seed=9)
    g = torch.Generator().manual_seed(1)
    d_logp = torch.randn(T, generator=g).to(DEV)
    before = torch.randn(V, H, generator=g).to(DEV).to(DT[dw])
    dz, size = R.scores_dz64(R.logits64(hidden, W, 1.0), targets, 1.0, d_logp, None)
    for kw in (dict(bwd_panel_tokens=256), dict(dw_accumulate=True), dict(bwd_panel_tokens=512, dw_accumulate=True)):
        p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, dw_dtype=dw, kernel_path=path, **kw)
        out = U.token_scores(p, hidden, W, targets)
        d_W = before.clone() if kw.get("dw_accumulate") else torch.full((V, H), 7.0, device=DEV, dtype=DT[dw])
        d_h, d_W = U.token_scores_bwd(p, hidden, W, targets, out, d_logp, None, d_W=d_W)
        R.check_grads(d_h, d_W, dz, size, hidden, W, R.logit_error(hidden, W, 1.0) * 8, dtype == "bf16", dw,
                      before if kw.get("dw_accumulate") else None)


@pytest.mark.parametrize("path", ["simt", "tensor"])
def test_score_gradients_against_differences(path):
    """float32 head: the loss moves along a direction of (hidden, W) as the gradients say."""
    T, H, V, kappa = 24, 32, 300, 0.9
    hidden, W, targets = operands(T, H, V, "f32", seed=21)
    g = torch.Generator().manual_seed(2)
    d_logp, d_ent = torch.randn(T, generator=g).to(DEV), torch.randn(T, generator=g).to(DEV)
    p = U.HeadParams(T=T, H=H, V=V, dtype="f32", inv_temperature=kappa, kernel_path=path)
    out = U.token_scores(p, hidden, W, targets)
    d_h, d_W = U.token_scores_bwd(p, hidden, W, targets, out, d_logp, d_ent)

    def loss(h, w):
        s = R.scores64(kappa * (h @ w.t()), targets)
        return float((d_logp.double() * s["logp"] + d_ent.double() * s["entropy"]).sum())
    dh, dw = torch.randn(T, H, generator=g).double().to(DEV), torch.randn(V, H, generator=g).double().to(DEV) / 8
    eps = 1e-5
    slope = (loss(hidden.double() + eps * dh, W.double() + eps * dw) - loss(hidden.double() - eps * dh, W.double() - eps * dw)) / (2 * eps)
    got = float((d_h.double() * dh).sum() + (d_W.double() * dw).sum())
    # float32 gradients (a few 10^-6 of the sum of magnitudes), the difference's own eps^2
    size = float((d_h.double() * dh).abs().sum() + (d_W.double() * dw).abs().sum())
    assert abs(got - slope) <= 1e-5 * size


# ------------------------------------------------------------------------------------------------ distillation
def teacher_lists(T, V, K, seed, ragged=True):
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]).to(torch.int32)
    logp = torch.log_softmax(2 * torch.randn(T, K, generator=g), 1) + torch.log(0.6 + 0.3999 * torch.rand(T, 1, generator=g))
    if ragged and T > 6:
        ids[1, K // 2:] = -1                       # a shorter list
        ids[2, :] = -1                             # none
        logp[3, 0] = -math.inf                     # an entry without probability
        ids[4, 0], logp[4, 0] = -1, float("nan")   # padding may hold anything
    return ids.to(DEV), logp.to(DEV)


def check_distill(p, hidden, W, ids, teacher, weights, tensor_path, grad_loss=None):
    ws = U.alloc_head_workspace(p, DEV)
    out = U.distill_fwd(p, hidden, W, ids, teacher, weights, workspace=ws)
    gl = None if grad_loss is None else torch.tensor([grad_loss], device=DEV)
    d_h, d_W = U.distill_bwd(p, hidden, W, ids, out, grad_loss=gl, workspace=ws)
    kappa = p.inv_temperature
    z = R.logits64(hidden, W, kappa)
    ref = R.distill64(z, ids, teacher, weights, p.distill_mode, kappa, p.teacher_inv_temperature, p.norm_tokens or None)
    E = R.logit_error(hidden, W, kappa).cpu()
    # every log-prob is off by 2 E + 2^-20 + roundings of numbers up to |z|; the weights q and 1 - Q add up to at most
    # one (renorm: one)
    tol = 2 * E + 2.0 ** -19 + 2.0 ** -22 * z.abs().amax(1).cpu()
    close(out.kl, ref["kl"], 2 * tol + 2.0 ** -23 * ref["kl"].abs(), "kl")
    w = torch.ones(p.T) if weights is None else weights.cpu()
    N = p.norm_tokens or p.T
    close(out.loss, ref["loss"][None], ((2 * tol + 2.0 ** -23 * ref["kl"].abs()) * w.abs()).sum() / N + 2.0 ** -23 * ref["loss"].abs(), "loss")
    s = abs(grad_loss) if grad_loss is not None else 1.0
    R.check_grads(d_h, d_W, (grad_loss or 1.0) * ref["dz"], s * ref["size"], hidden, W, E + 2.0 ** -20, tensor_path, p.dw_dtype)
    return out, d_h, d_W, ws


DISTILL_SIZES = [(1, 64, 1000, 5), (20, 64, 3001, 7), (40, 136, 2000, 33), (64, 64, 500, 4), (16, 72, 20001, 3), (17, 128, 2500, 20), (33, 64, 40003, 32), (64, 200, 3000, 8), (65, 200, 3000, 8), (3, 8, 5, 5), (9, 16, 40, 1), (129, 136, 257, 32), (300, 256, 4099, 20), (70, 64, 700, 128)]


@pytest.mark.parametrize("T,H,V,K", DISTILL_SIZES)
@pytest.mark.parametrize("mode", ["raw", "renorm", "tail"])
@pytest.mark.parametrize("dtype,path,dw", [("bf16", "auto", "bf16"), ("bf16", "simt", "f32"), ("f32", "simt", "f32"), ("f32", "tensor", "f32")])
def test_distillation(T, H, V, K, mode, dtype, path, dw):
    hidden, W, _ = operands(T, H, V, dtype, seed=T + K)
    ids, teacher = teacher_lists(T, V, K, seed=V)
    if K == V and mode == "tail":                  # nothing is left for the remainder: the lists are made complete
        teacher = torch.log_softmax(teacher, 1).clamp(min=-30.0)
        teacher[:, 0] = torch.where(teacher.double().exp().sum(1) < 1, teacher[:, 0] + 1e-3, teacher[:, 0])
    weights = (torch.rand(T, generator=torch.Generator().manual_seed(K)) < 0.8).float().to(DEV) if T > 3 else None
    p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=K, inv_temperature=0.9, kernel_path=path, dw_dtype=dw,
                     distill_mode=mode, teacher_inv_temperature=0.7 if mode == "renorm" else 1.0)
    out, d_h, _, ws = check_distill(p, hidden, W, ids, teacher, weights, dtype == "bf16" and path != "simt")
    assert B.check_status(ws) == B.OK
    if weights is not None:
        assert not bool(d_h[weights == 0].any())
        if T > 6:
            assert float(out.kl[2]) == 0.0 and not bool(d_h[2].any())


@pytest.mark.parametrize("dtype,path", [("bf16", "auto"), ("f32", "simt"), ("f32", "tensor")])
def test_ids_listed_twice_and_out_of_range(dtype, path):
    T, H, V, K = 12, 64, 600, 8
    hidden, W, _ = operands(T, H, V, dtype, seed=77)
    ids, teacher = teacher_lists(T, V, K, seed=5, ragged=False)
    ids[0, 5] = ids[0, 1]
    ids[1, :] = 17
    ids[2, 2], ids[2, 6] = ids[2, 0], ids[2, 0]
    for mode in ("raw", "renorm", "tail"):
        p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=K, distill_mode=mode, kernel_path=path)
        *_, ws = check_distill(p, hidden, W, ids, teacher, None, dtype == "bf16", grad_loss=-2.5)
        assert B.check_status(ws) == B.OK
    bad = ids.clone()
    bad[5, 3], bad[6, 0] = V, -7
    p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=K, distill_mode="raw", norm_tokens=100, kernel_path=path)
    ws = U.alloc_head_workspace(p, DEV)
    U.distill_fwd(p, hidden, W, bad, teacher, workspace=ws)
    assert B.check_status(ws) == -6
    check_distill(p, hidden, W, bad, teacher, None, dtype == "bf16")


@pytest.mark.parametrize("mode", ["raw", "renorm", "tail"])
def test_distillation_against_differences(mode):
    T, H, V, K = 20, 32, 200, 6
    hidden, W, _ = operands(T, H, V, "f32", seed=8)
    ids, teacher = teacher_lists(T, V, K, seed=9)
    p = U.HeadParams(T=T, H=H, V=V, dtype="f32", top_k=K, distill_mode=mode)
    out = U.distill_fwd(p, hidden, W, ids, teacher)
    d_h, d_W = U.distill_bwd(p, hidden, W, ids, out)
    g = torch.Generator().manual_seed(2)
    dh, dw = torch.randn(T, H, generator=g).double().to(DEV), torch.randn(V, H, generator=g).double().to(DEV) / 8
    loss = lambda h, w: float(R.distill64(h @ w.t(), ids, teacher, None, mode)["loss"])
    eps = 1e-5
    slope = (loss(hidden.double() + eps * dh, W.double() + eps * dw) - loss(hidden.double() - eps * dh, W.double() - eps * dw)) / (2 * eps)
    got = float((d_h.double() * dh).sum() + (d_W.double() * dw).sum())
    size = float((d_h.double() * dh).abs().sum() + (d_W.double() * dw).abs().sum())
    assert abs(got - slope) <= 1e-5 * size


@pytest.mark.parametrize("kappa", [0.35, 0.7, 1.0, 1.1, 1.9])
def test_lists_of_whole_chunks(kappa):
    """Lists that hold every column of the first chunks of a sweep, of its last one, or of the vocabulary."""
    for V, K, first in ((600, 64, 0), (257, 33, 224), (96, 96, 0)):
        T = 70
        hidden, W, _ = operands(T, 64, V, "bf16", seed=V)
        g = torch.Generator().manual_seed(K)
        ids = torch.stack([first + torch.randperm(K, generator=g) for _ in range(T)]).to(torch.int32).to(DEV)
        logp = (torch.log_softmax(torch.randn(T, K, generator=g), 1) - 0.1).to(DEV)
        mode = "raw" if K == V else "tail"
        p = U.HeadParams(T=T, H=64, V=V, top_k=K, distill_mode=mode, inv_temperature=kappa)
        check_distill(p, hidden, W, ids, logp, None, True)


def test_overconfident_student_keeps_the_remainder():
    """Mode tail, a student that gives the list all but 10^-7: the remainder's log-prob is not a difference of ones."""
    T, H, V, K = 6, 64, 2048, 4
    W = torch.zeros(V, H)
    W[torch.arange(V), torch.arange(V) % H] = 1.0
    W[:4] *= torch.tensor([22.0, 21.0, 20.0, 23.0])[:, None]
    hidden = torch.zeros(T, H)
    hidden[:, :4] = 1.0
    ids = torch.arange(4, dtype=torch.int32).repeat(T, 1).to(DEV)
    teacher = torch.log(torch.tensor([0.4, 0.3, 0.1, 0.1])).repeat(T, 1).to(DEV)
    for dtype in ("bf16", "f32"):
        h, w = hidden.to(DT[dtype]).to(DEV), W.to(DT[dtype]).to(DEV)
        p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=K, distill_mode="tail")
        check_distill(p, h, w, ids, teacher, None, dtype == "bf16")


def test_student_that_leaves_nothing_off_the_list():
    """Mode tail, a student whose list outweighs the rest by e^200: the rest's probability underflows in float32, its
    logarithm and the gradient's share of it do not."""
    T, H, V, K = 5, 64, 600, 3
    W = torch.zeros(V, H)
    W[torch.arange(V), torch.arange(V) % H] = 1.0
    W[:3] *= torch.tensor([200.0, 201.0, 199.0])[:, None]
    hidden = torch.zeros(T, H)
    hidden[:, :3] = 1.0
    ids = torch.arange(3, dtype=torch.int32).repeat(T, 1).to(DEV)
    teacher = torch.log(torch.tensor([0.5, 0.3, 0.1])).repeat(T, 1).to(DEV)
    for dtype in ("bf16", "f32"):
        for mode in ("raw", "tail"):
            p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=K, distill_mode=mode)
            out, d_h, d_W, _ = check_distill(p, hidden.to(DT[dtype]).to(DEV), W.to(DT[dtype]).to(DEV), ids, teacher, None, dtype == "bf16")
            assert bool(torch.isfinite(d_h).all()) and bool(torch.isfinite(d_W).all()) and bool(torch.isfinite(out.kl).all())


@pytest.mark.parametrize("dtype,path", [("f32", "simt"), ("bf16", "simt")])
def test_forward_by_panels(dtype, path):
    """The CUDA-core path's forward passes by panels of tokens: the same results as in one."""
    T, H, V, k = 700, 64, 900, 6
    hidden, W, targets = operands(T, H, V, dtype, seed=19)
    ids, teacher = teacher_lists(T, V, k, seed=20)
    one = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=k, kernel_path=path, distill_mode="tail")
    many = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=k, kernel_path=path, distill_mode="tail", bwd_panel_tokens=200)
    a, b = (U.token_scores(p, hidden, W, targets) for p in (one, many))
    c, d = (U.distill_fwd(p, hidden, W, ids, teacher) for p in (one, many))
    for x, y in ((a, b), (c, d)):
        for name, v in vars(x).items():
            assert torch.equal(v, getattr(y, name)), name


@pytest.mark.parametrize("T,V,H,path", [(20, 1000, 64, "simt"), (300, 20000, 256, "tensor")])
def test_float32_path_goes_by_the_sizes(T, V, H, path):
    """What AUTO takes for float32 operands is one of the two paths, bit for bit and with its workspace; a forward of one fits a backward of the other."""
    hidden, W, targets = operands(T, H, V, "f32", seed=T)
    outs = []
    for way in ("auto", path):
        p = U.HeadParams(T=T, H=H, V=V, dtype="f32", top_k=4, kernel_path=way)
        assert way == path or U.head_workspace_bytes(p, False) == U.head_workspace_bytes(U.HeadParams(**{**vars(p), "kernel_path": path}), False)
        outs.append(U.token_scores(p, hidden, W, targets))
    for name, v in vars(outs[0]).items():
        assert torch.equal(v, getattr(outs[1], name)), name
    # a forward of one path and a backward of the other belong together
    d = torch.randn(T, generator=torch.Generator().manual_seed(1)).to(DEV)
    z = R.logits64(hidden, W, 1.0)
    dz, size = R.scores_dz64(z, targets, 1.0, d, None)
    for fwd, bwd in (("simt", "tensor"), ("tensor", "simt")):
        a, b = (U.HeadParams(T=T, H=H, V=V, dtype="f32", kernel_path=x) for x in (fwd, bwd))
        s = U.token_scores(a, hidden, W, targets)
        R.check_grads(*U.token_scores_bwd(b, hidden, W, targets, s, d, None), dz, size, hidden, W, 2 * R.logit_error(hidden, W, 1.0), False, "f32")


def test_float32_planes_keep_their_digits():
    """float32 operands on the tensor cores: long contractions (several panels of tokens, several parts of the
    vocabulary) against 64 bits, relative to the whole; bf16 operands would be 10^-3 off, two planes 10^-5."""
    T, H, V, k = 2500, 264, 6001, 8
    hidden, W, targets = operands(T, H, V, "f32", seed=91)
    ids, teacher = teacher_lists(T, V, k, seed=92)
    g = torch.Generator().manual_seed(93)
    d_logp = torch.randn(T, generator=g).to(DEV)
    z = R.logits64(hidden, W, 1.0)
    dz, _ = R.scores_dz64(z, targets, 1.0, d_logp, None)
    ref = R.scores64(z, targets, k)
    p = U.HeadParams(T=T, H=H, V=V, dtype="f32", top_k=k, distill_mode="tail", kernel_path="tensor")
    out = U.token_scores(p, hidden, W, targets)
    d_h, d_W = U.token_scores_bwd(p, hidden, W, targets, out, d_logp, None)
    # a sum of n terms in float32: n/2 additions, each rounded or cut off by at most 2^-23, mostly one way
    far = lambda got, want: float((got.double() - want).norm() / want.norm())
    assert far(out.logp, ref["logp"]) <= H * 2.0 ** -24 and far(out.lse, ref["lse"]) <= H * 2.0 ** -24
    slack = 4 * H * 2.0 ** -24                     # p is off by the error of its logit, about |z| = 4 times that
    assert far(d_h, dz @ W.double()) <= slack + 2048 * 2.0 ** -24 and far(d_W, dz.t() @ hidden.double()) <= slack + 2048 * 2.0 ** -24
    q = U.HeadParams(**{**vars(p), "kernel_path": "simt"})
    a, b = (U.distill_fwd(x, hidden, W, ids, teacher) for x in (p, q))
    (ah, aw), (bh, bw) = U.distill_bwd(p, hidden, W, ids, a), U.distill_bwd(q, hidden, W, ids, b)
    assert far(a.kl, b.kl.double()) <= H * 2.0 ** -23
    assert far(ah, bh.double()) <= 2 * (slack + 2048 * 2.0 ** -24) and far(aw, bw.double()) <= 2 * (slack + 2048 * 2.0 ** -24)
    print("f32 planes: logp %.1e d_h %.1e d_W %.1e" % (far(out.logp, ref["logp"]), far(d_h, dz @ W.double()), far(d_W, dz.t() @ hidden.double())))


# ------------------------------------------------------------------------------------------------ together
def test_teacher_scores_feed_a_student():
    """A teacher scores a batch, a student is trained on its alternatives: with the teacher's own head and hidden
    states the loss is that of the truncation alone and the listed gradients vanish."""
    T, H, V, k = 200, 128, 3000, 16
    hidden, W, targets = operands(T, H, V, "bf16", seed=31)
    p = U.HeadParams(T=T, H=H, V=V, top_k=k, distill_mode="tail", dw_dtype="bf16")
    ws = U.alloc_head_workspace(p, DEV)
    s = U.token_scores(p, hidden, W, targets, workspace=ws)
    d = U.distill_fwd(p, hidden, W, s.top_ids, s.top_logp, workspace=ws)
    # student = teacher: KL of equal distributions; every term is a difference of log-probs off by 2^-19 + 2^-22 |z|
    tol = 2.0 ** -18 + 2.0 ** -20 * float(R.logits64(hidden, W, 1.0).abs().max())
    assert float(d.kl.abs().max()) <= tol and abs(float(d.loss)) <= tol
    assert float(d.entry_grad.abs().max()) <= tol / T
    other, *_ = operands(T, H, V, "bf16", seed=32)
    check_distill(p, other, W, s.top_ids, s.top_logp, None, True)
    # the log-probs are those that the policy loss takes: ratio one, nothing clipped
    lp = B.Params(T=T, H=H, V=V, num_seqs=1, mpt_mode="off")
    offsets = torch.tensor([0, T], dtype=torch.int32, device=DEV)
    adv = torch.ones(1, device=DEV)
    f = B.token_loss_fwd(lp, hidden, W, targets, s.logp, None, adv, offsets)
    assert float((f.logp - s.logp).abs().max()) <= tol and f.stats_host()["n_clip_high"] == 0
    assert abs(float(f.loss[0]) + 1.0) <= 2 * tol


def test_logits_and_head_agree():
    T, H, V, k = 64, 64, 5000, 12
    hidden, W, targets = operands(T, H, V, "bf16", seed=41, grid=True)
    head = U.token_scores(U.HeadParams(T=T, H=H, V=V, top_k=k, inv_temperature=0.7), hidden, W, targets)
    z = (hidden.double() @ W.double().t()).float()
    row = U.logits_scores(z, targets, top_k=k, inv_temperature=0.7)
    assert torch.equal(head.top_ids, row.top_ids)
    for name in ("logp", "lse", "entropy", "top_logp"):
        assert float((getattr(head, name) - getattr(row, name)).abs().max()) <= 2.0 ** -17


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_step_on_a_side_stream(dtype):
    """Forward and backward of both operators captured into one graph and replayed on other inputs; two graphs that
    share a workspace, replayed one after the other."""
    T, H, V, k = 130, 64, 1500, 6
    p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=k, distill_mode="tail", dw_dtype=dtype)
    sets = []
    for seed in (1, 2):
        h, w, y = operands(T, H, V, dtype, seed)
        sets.append((h, w, y, *teacher_lists(T, V, k, seed)))
    ws = U.alloc_head_workspace(p, DEV)

    def step(h, w, y, ids, l):
        s = U.token_scores(p, h, w, y, workspace=ws)
        g1 = U.token_scores_bwd(p, h, w, y, s, s.logp, s.entropy, workspace=ws)
        d = U.distill_fwd(p, h, w, ids, l, workspace=ws)
        g2 = U.distill_bwd(p, h, w, ids, d, workspace=ws)
        r = U.logits_scores(w.view(-1)[: H * (V // 2)].view(H, V // 2), top_k=k)
        return [s.logp, s.entropy, s.top_ids, s.top_logp, *g1, d.loss, d.kl, *g2, r.entropy, r.top_ids]
    want = [[x.clone() for x in step(*a)] for a in sets]
    static = [x.clone() for x in sets[0]]
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*static)
        side.synchronize()
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                outs.append(step(*static))
            graphs.append(graph)
        for n in (1, 0, 1):
            for dst, src in zip(static, sets[n]):
                dst.copy_(src)
            for graph in graphs:
                graph.replay()
            side.synchronize()
            for got in outs:
                assert all(torch.equal(a, b) for a, b in zip(got, want[n]))
    del graphs


@pytest.mark.parametrize("T,dtype,path", [(20, "bf16", "auto"), (300, "bf16", "auto"), (300, "f32", "simt"), (300, "f32", "tensor")])
def test_low_temperature_keeps_its_digits(T, dtype, path):
    """Exact logits of half a million, scaled, that differ by tenths: scores, alternatives and gradients."""
    H, V, k, kappa = 64, 3001, 8, 2.0 ** 13
    g = torch.Generator().manual_seed(61)
    W = torch.zeros(V, H)
    W[:, 0] = 40.0
    W[:, 1:9] = torch.randint(0, 4, (V, 8), generator=g).float() * 2.0 ** -14
    hidden = torch.zeros(T, H)
    hidden[:, 0] = 1.0
    hidden[torch.arange(T), 1 + torch.arange(T) % 8] = 1.0
    h, w = hidden.to(DT[dtype]).to(DEV), W.to(DT[dtype]).to(DEV)
    targets = torch.randint(0, V, (T,), generator=g, dtype=torch.int32).to(DEV)
    p = U.HeadParams(T=T, H=H, V=V, dtype=dtype, top_k=k, inv_temperature=kappa, kernel_path=path)
    out = U.token_scores(p, h, w, targets)
    z = R.logits64(h, w, kappa)
    R.check_low_temperature(out, z, targets, k)
    for d_logp, d_ent in ((torch.randn(T, generator=g).to(DEV), None), (None, torch.randn(T, generator=g).to(DEV))):
        d_h, d_W = U.token_scores_bwd(p, h, w, targets, out, d_logp, d_ent)
        dz, size = R.scores_dz64(z, targets, kappa, d_logp, d_ent)
        # the entropy's dz carries the errors of log p and of the entropy, 2^-18 each beside terms of their size
        R.check_grads(d_h, d_W, dz, size, h, w, torch.full((T,), 2.0 ** -18), dtype == "bf16", "f32")
    # the student's own list: no loss, and lists that leave the maximum out keep the scale of the rest
    ids = out.top_ids.clone()
    d = U.distill_fwd(p, h, w, ids, torch.full((T, k), math.log(1.0 / (2 * k)), device=DEV))
    ref = R.distill64(z, ids, torch.full((T, k), math.log(1.0 / (2 * k))), None, "raw", kappa)
    err = (d.kl.double().cpu() - ref["kl"]).abs()
    assert bool((err <= 2.0 ** -19 + 2.0 ** -20 * ref["kl"].abs()).all()), float(err.max())


def test_two_streams_at_once():
    """Calls that overlap on two streams, each with its own workspace, give what they give alone."""
    sets = []
    for seed, (T, V, k) in ((71, (900, 9001, 20)), (72, (40, 30001, 8))):
        p = U.HeadParams(T=T, H=256, V=V, top_k=k, distill_mode="tail")
        sets.append((p, operands(T, 256, V, "bf16", seed), teacher_lists(T, V, k, seed), U.alloc_head_workspace(p, DEV), torch.cuda.Stream()))

    def calls(p, ops, lists, ws):
        s = U.token_scores(p, *ops, workspace=ws)
        g = U.token_scores_bwd(p, *ops, s, s.logp, None, workspace=ws)
        d = U.distill_fwd(p, *ops[:2], *lists, workspace=ws)
        return [s.logp, s.entropy, s.top_ids, *g, d.loss, *U.distill_bwd(p, *ops[:2], lists[0], d, workspace=ws)]
    want = [calls(*a[:4]) for a in sets]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for a in sets:
            with torch.cuda.stream(a[4]):
                got.append(calls(*a[:4]))
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert all(torch.equal(b, c) for b, c in zip(x, y))


def test_status_of_a_workspace_for_backward_calls():
    """A workspace that has seen no forward call reads as clean."""
    T, H, V = 70, 64, 500
    hidden, W, targets = operands(T, H, V, "bf16", seed=81)
    p = U.HeadParams(T=T, H=H, V=V)
    torch.full((U.head_workspace_bytes(p),), 255, dtype=torch.uint8, device=DEV)         # dirty bytes for the allocator to hand out
    out = U.token_scores(p, hidden, W, targets)
    ws = U.alloc_head_workspace(p, DEV)
    U.token_scores_bwd(p, hidden, W, targets, out, out.logp, workspace=ws)
    assert B.check_status(ws) == B.OK


def test_results_do_not_depend_on_the_run():
    T, H, V, k = 700, 256, 9001, 20
    hidden, W, targets = operands(T, H, V, "bf16", seed=51)
    ids, teacher = teacher_lists(T, V, k, seed=52)
    p = U.HeadParams(T=T, H=H, V=V, top_k=k, distill_mode="tail", dw_dtype="bf16")
    first = None
    for _ in range(3):
        s = U.token_scores(p, hidden, W, targets)
        d = U.distill_fwd(p, hidden, W, ids, teacher)
        got = [s.logp, s.entropy, s.top_ids, s.top_logp, *U.token_scores_bwd(p, hidden, W, targets, s, s.logp, s.entropy),
               d.loss, d.kl, *U.distill_bwd(p, hidden, W, ids, d)]
        assert first is None or all(torch.equal(a, b) for a, b in zip(got, first))
        first = [x.clone() for x in got]


def test_empty_batch():
    for dtype in ("bf16", "f32"):
        p = U.HeadParams(T=0, H=64, V=100, dtype=dtype, top_k=3)
        h, w = torch.empty(0, 64, dtype=DT[dtype], device=DEV), torch.ones(100, 64, dtype=DT[dtype], device=DEV)
        y, none = torch.empty(0, dtype=torch.int32, device=DEV), torch.empty(0, device=DEV)
        s = U.token_scores(p, h, w, y)
        assert s.logp.numel() == 0 and tuple(s.top_ids.shape) == (0, 3)
        _, d_W = U.token_scores_bwd(p, h, w, y, s, none, None)
        assert not bool(d_W.any())
        ids, l = torch.empty(0, 3, dtype=torch.int32, device=DEV), torch.empty(0, 3, device=DEV)
        d = U.distill_fwd(p, h, w, ids, l)
        assert float(d.loss[0]) == 0.0
        assert not bool(U.distill_bwd(p, h, w, ids, d)[1].any())
        assert U.logits_scores(torch.empty(0, 50, device=DEV), y, top_k=2).lse.numel() == 0


def test_rows_behind_the_outputs_are_left_alone():
    """Outputs that are parts of larger tensors: nothing outside them changes."""
    T, H, V, k = 129, 64, 777, 5
    hidden, W, targets = operands(T, H, V, "bf16", seed=61)
    p = U.HeadParams(T=T, H=H, V=V, top_k=k, dw_dtype="bf16")
    big = {n: torch.full(s, 123, dtype=t, device=DEV) for n, s, t in (
        ("vec", (5 * T + 64,), torch.float32), ("ids", (T * k + 64,), torch.int32), ("tl", (T * k + 64,), torch.float32),
        ("dh", (T + 8, H), torch.bfloat16), ("dw", (V + 8, H), torch.bfloat16))}
    v = big["vec"]
    out = U.head.ScoresOut(v[2 * T:3 * T], v[3 * T:4 * T], v[4 * T:5 * T], v[:2 * T].view(T, 2), big["ids"][:T * k].view(T, k),
                           big["tl"][:T * k].view(T, k))
    n = U.head_workspace_bytes(p)
    ws = torch.full((n + 4096,), 77, dtype=torch.uint8, device=DEV)
    U.token_scores(p, hidden, W, targets, out=out, workspace=ws[:n])
    U.token_scores_bwd(p, hidden, W, targets, out, out.logp, out.entropy, big["dh"][:T], big["dw"][:V], workspace=ws[:n])
    torch.cuda.synchronize()
    assert bool((v[5 * T:] == 123).all()) and bool((big["ids"][T * k:] == 123).all()) and bool((big["tl"][T * k:] == 123).all())
    assert bool((big["dh"][T:] == 123).all()) and bool((big["dw"][V:] == 123).all()) and bool((ws[n:] == 77).all())
    check_scores(out, hidden, W, targets, k, 1.0, exact_ids=False)
