"""Scores from given logits against a plain 64-bit form: types, strides, masks, ties, NaN."""
import math

import pytest
import torch

import paper_2507_19766_b200 as U
from tests import head_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def check(logits, targets, k, kappa=1.0):
    out = U.logits_scores(logits, targets, top_k=k, inv_temperature=kappa)
    z = kappa * logits.double()
    ref = R.scores64(z, targets, k)
    mag = torch.where(torch.isfinite(z), z.abs(), torch.zeros_like(z)).amax(1)
    # z - max in float32 (two roundings of numbers up to twice |z|), ex2, a sum of positive terms; lse is rounded too
    tol = (2.0 ** -20 + 2.0 ** -21 * mag).cpu()

    def close(got, want, bound, what):
        got, want = got.double().cpu(), want.double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)), what
        assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)]), what
        d = torch.where(torch.isfinite(want), (got - want).abs(), torch.zeros_like(want))
        assert bool((d <= bound).all()), (what, float((d / bound).max()))
    close(out.lse, ref["lse"], tol, "lse")
    if targets is not None:
        close(out.logp, ref["logp"], tol, "logp")
    spread = torch.where(ref["logp_all"] > -math.inf, ref["logp_all"].exp() * (ref["logp_all"] + ref["entropy"][:, None]).abs(),
                         torch.zeros_like(z)).sum(1).cpu()
    close(out.entropy, ref["entropy"], tol * (1 + spread) + 2.0 ** -20 * (1 + ref["entropy"].cpu()), "entropy")
    if k:
        nan_rows = torch.isnan(ref["lse"])
        assert torch.equal(out.top_ids[~nan_rows].cpu(), ref["top_ids"][~nan_rows].cpu())
        close(out.top_logp[~nan_rows], ref["top_logp"][~nan_rows], tol[~nan_rows.cpu()][:, None], "top_logp")
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,k", [(1, 1, 1), (3, 5, 5), (2, 31, 0), (7, 257, 32), (5, 1000, 20), (40, 4099, 8), (3, 32003, 32),
                                   (2, 151936, 20), (1, 300000, 32), (600, 513, 1)])
def test_types_sizes_strides(dtype, T, V, k):
    g = torch.Generator(device=DEV).manual_seed(V + T)
    for pad, shift in ((0, 0), (7, 0), (64, 3)):             # contiguous; odd row stride; rows off every 16-byte boundary
        flat = torch.full((T * (V + pad) + shift,), float("nan"), device=DEV, dtype=dtype)   # padding may hold anything
        logits = flat[shift:].view(T, V + pad)[:, :V]
        logits.copy_(3 * torch.randn(T, V, generator=g, device=DEV))
        targets = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
        check(logits, targets, k, kappa=1.0 if pad else 0.7)


@pytest.mark.parametrize("dtype", TYPES)
def test_masks(dtype):
    """-inf and the type's lowest value as masks, rows that keep a few entries, one, or none."""
    V, k = 5003, 20
    g = torch.Generator(device=DEV).manual_seed(7)
    z = (3 * torch.randn(8, V, generator=g, device=DEV)).to(dtype)
    low = torch.finfo(dtype).min
    z[0, torch.rand(V, generator=g, device=DEV) < 0.5] = -math.inf
    z[1, :] = -math.inf                                       # nothing left
    z[2, :] = -math.inf
    z[2, 4001] = 1.5                                          # one entry left
    z[3, 6:] = -math.inf                                      # six left, fewer than asked for
    z[4, torch.rand(V, generator=g, device=DEV) < 0.9] = low
    z[5, :] = low                                             # uniform over lowest values
    z[6, :] = low
    z[6, 17] = -math.inf
    z[6, 3000] = 0.0
    targets = torch.tensor([3, 9, 4001, 100, 5, 6, 3000, 7], dtype=torch.int32, device=DEV)
    out = check(z, targets, k)
    assert float(out.lse[1]) == -math.inf and float(out.entropy[1]) == 0.0 and float(out.logp[1]) == -math.inf
    assert out.top_ids[1].tolist() == list(range(k))
    assert float(out.logp[2]) == 0.0 and float(out.entropy[2]) == 0.0
    assert float(out.logp[3]) == -math.inf and sorted(out.top_ids[3].tolist()[:6]) == list(range(6))
    assert out.top_ids[3].tolist()[6:] == list(range(6, 20))
    assert out.top_ids[5].tolist() == list(range(k))
    check(z[:, :1], torch.zeros(8, dtype=torch.int32, device=DEV), 1)


@pytest.mark.parametrize("dtype", TYPES)
def test_nan_and_infinite_entries(dtype):
    V, k = 900, 4
    g = torch.Generator(device=DEV).manual_seed(8)
    z = torch.randn(6, V, generator=g, device=DEV).to(dtype)
    z[1, 5] = float("nan")
    z[2, 5] = math.inf
    z[3, :] = float("nan")
    z[4, 0], z[4, 1:] = float("nan"), -math.inf
    targets = torch.full((6,), 5, dtype=torch.int32, device=DEV)
    out = U.logits_scores(z, targets, top_k=k)
    for row in (1, 2, 3, 4):
        assert bool(torch.isnan(out.logp[row])) and bool(torch.isnan(out.entropy[row])), row
    for row in (0, 5):
        ref = R.scores64(z[row:row + 1].double(), targets[:1], k)
        assert torch.equal(out.top_ids[row:row + 1].cpu(), ref["top_ids"].cpu())
    # NaN is never an alternative, +inf is the first one
    assert 5 not in out.top_ids[1].tolist() and out.top_ids[2].tolist()[0] == 5
    assert out.top_ids[3].tolist() == [-1] * k and bool(torch.isnan(out.top_logp[3]).all())
    assert out.top_ids[4].tolist() == [1, 2, 3, 4]
    # a target outside the vocabulary has no log-prob
    out = U.logits_scores(z, torch.tensor([-1, 0, 0, 0, 0, V], dtype=torch.int32, device=DEV))
    assert bool(torch.isnan(out.logp[0])) and bool(torch.isnan(out.logp[5]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [700, 40001])
def test_ties_and_sorted_rows(dtype, V):
    """Rows of one value, of a few, rising, falling, with the large entries side by side or in one lane's places."""
    k = 32
    z = torch.zeros(9, V, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(9)
    z[1] = torch.randint(0, 3, (V,), generator=g, device=DEV).float()
    z[2] = torch.arange(V, device=DEV) / 64.0
    z[3] = -torch.arange(V, device=DEV) / 64.0
    z[4, V // 2:V // 2 + 400] = 5.0 + torch.rand(min(400, V - V // 2), generator=g, device=DEV)
    step = 2048 if dtype != torch.float32 else 1024           # places that one lane of the block reads
    z[5, 5::step] = 9.0
    z[5, 6::step] = torch.linspace(9, 20, z[5, 6::step].numel(), device=DEV)
    z[6] = torch.where(torch.arange(V, device=DEV) % 2 == 0, -0.0, 0.0)     # equal values of either sign
    z[7, -3:] = 1.0
    for lane in range(8):
        z[8, 8 * lane::step] = torch.arange(z[8, 8 * lane::step].numel(), device=DEV) / 8.0 + 1
    check(z.to(dtype), None, k)
    check(z[:, 3:].to(dtype), None, 1)


def test_many_entries_above_the_bound():
    """One lane holds hundreds of the largest entries and the other lanes next to nothing: more candidates than the
    block's list holds."""
    V, k = 4_000_000, 20
    z = torch.zeros(2, V, device=DEV)
    lanes = torch.arange(V, device=DEV) // 4 % 256
    z[0] = torch.where(lanes < 19, torch.rand(V, device=DEV) + 1, z[0])
    check(z, None, k)


def test_long_offsets():
    """Rows that start beyond 2^31 elements and 2^32 bytes."""
    V, ld, T = 1000, 600_000_003, 5
    flat = torch.empty(ld * (T - 1) + V, dtype=torch.bfloat16, device=DEV)
    z = flat.as_strided((T, V), (ld, 1))
    z.copy_(torch.randn(T, V, device=DEV))
    check(z, torch.arange(T, dtype=torch.int32, device=DEV), 8)


@pytest.mark.parametrize("kappa", [1e-6, 1e6])
def test_extreme_temperatures(kappa):
    """Masked entries have no probability at either end, and the row is uniform or greedy."""
    V, k = 3001, 8
    g = torch.Generator(device=DEV).manual_seed(11)
    for dtype in TYPES:
        z = torch.randn(4, V, generator=g, device=DEV).to(dtype)
        z[:, ::3] = -math.inf
        z[2] = -math.inf
        z[2, 5] = 1.0
        targets = torch.tensor([1, 3, 5, 4], dtype=torch.int32, device=DEV)
        out = check(z, targets, k, kappa=kappa)
        if kappa < 1:
            assert abs(float(out.entropy[0]) - math.log(V - (V + 2) // 3)) <= 2.0 ** -19
        assert float(out.entropy[2]) == 0.0 and float(out.logp[2]) == 0.0


def test_low_temperature_keeps_its_digits():
    """Scaled logits of 4 million that differ by tenths: what the scaled maximum loses to rounding is put back."""
    V, k, kappa = 5001, 12, 1e5
    g = torch.Generator().manual_seed(12)
    for T in (1, 7, 400):
        z = (40.0 + torch.randint(0, 12, (T, V), generator=g).double() * 2.0 ** -18).float().to(DEV)
        targets = torch.randint(0, V, (T,), generator=g, dtype=torch.int32).to(DEV)
        out = U.logits_scores(z, targets, top_k=k, inv_temperature=kappa)
        R.check_low_temperature(out, float(torch.tensor(kappa)) * z.double(), targets, k)
