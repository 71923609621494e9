"""What the scoring and distillation calls refuse, on the host: no launch, no device needed."""
import ctypes

import pytest
import torch

import paper_2507_19766_b200 as U
from paper_2507_19766_b200 import binding as B


@pytest.fixture(scope="module")
def lib():
    from paper_2507_19766_b200 import build
    build.build()
    return B.load_library()


def params(**kw):
    return U.HeadParams(**{**dict(T=8, H=64, V=100, top_k=4), **kw})


def test_struct_size_matches_header(lib):
    assert ctypes.sizeof(B.CHeadParams) == 56


@pytest.mark.parametrize("kw", [dict(T=-1), dict(H=0), dict(V=0), dict(H=60), dict(top_k=-1), dict(top_k=129), dict(inv_temperature=0.0),
                                dict(inv_temperature=float("nan")), dict(inv_temperature=float("inf")), dict(inv_temperature=2e6), dict(inv_temperature=5e-7),
                                dict(T=2 ** 30 + 1), dict(V=2 ** 31 - 1), dict(T=2 ** 32 + 8), dict(kernel_path="tensor_1cta"),
                                dict(dtype="f32", kernel_path="tensor", H=2 ** 29 + 8), dict(norm_tokens=-1), dict(bwd_panel_tokens=-1),
                                dict(teacher_inv_temperature=0.5), dict(distill_mode="tail", teacher_inv_temperature=2.0),
                                dict(distill_mode="renorm", teacher_inv_temperature=0.0)])
def test_invalid_parameters(lib, kw):
    with pytest.raises(U.UlorlError):
        U.head_workspace_bytes(params(**kw))


def test_unknown_names(lib):
    for kw in (dict(dtype="f16"), dict(dw_dtype="f8"), dict(distill_mode="reverse"), dict(kernel_path="cpu")):
        with pytest.raises(U.UlorlError):
            U.head_workspace_bytes(params(**kw))


def test_workspace_sizes(lib):
    """Scoring needs no dz panel; a bf16 d_W from one panel needs no float32 copy of itself."""
    big = dict(T=8192, H=2048, V=151936)
    fwd = U.head_workspace_bytes(params(**big, top_k=32), backward=False)
    bwd = U.head_workspace_bytes(params(**big, top_k=32, dw_dtype="bf16"))
    assert fwd < 128 << 20
    assert 8192 * 151936 * 2 <= bwd <= 8192 * 151936 * 2 + (64 << 20)
    more = U.head_workspace_bytes(params(**big, top_k=32, dw_dtype="bf16", dw_accumulate=True))
    assert more - bwd >= 151936 * 2048 * 4
    one = U.head_workspace_bytes(params(T=1, H=2048, V=151936, top_k=20), backward=False)
    assert one < 1 << 20


def call(lib, name, cp, ptrs, n):
    return getattr(lib, name)(ctypes.byref(cp), *ptrs, *([None] * (n - len(ptrs))), None, 0, None)


def test_missing_pointers_and_small_workspaces(lib):
    cp = params().to_c()
    fake = ctypes.c_void_p(1 << 20)                                    # never followed: the checks come first
    INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
    assert call(lib, "ulorl_token_scores", cp, [], 9) == INVALID       # top_k = 4 without its outputs
    s = lambda ws, n, ids=fake, tl=fake, norm=None, h=fake: lib.ulorl_token_scores(
        ctypes.byref(cp), h, fake, fake, fake, None, None, norm, ids, tl, ws, n, None)
    assert s(None, 0) == INVALID
    assert s(fake, 0) == WORKSPACE
    assert s(fake, 0, ids=None) == INVALID
    assert s(fake, 0, norm=ctypes.c_void_p((1 << 20) + 4)) == UNSUPPORTED
    assert s(fake, 0, h=ctypes.c_void_p((1 << 20) + 2)) == UNSUPPORTED
    # log-probs without targets
    assert lib.ulorl_token_scores(ctypes.byref(cp), fake, fake, None, fake, None, None, None, fake, fake, fake, 0, None) == INVALID
    assert call(lib, "ulorl_token_scores_bwd", cp, [fake] * 6, 10) == INVALID          # neither gradient
    assert call(lib, "ulorl_distill_fwd", cp, [fake] * 5, 11) == INVALID               # no loss
    assert call(lib, "ulorl_distill_bwd", cp, [fake] * 6, 9) == INVALID
    k0 = params(top_k=0).to_c()
    assert call(lib, "ulorl_distill_fwd", k0, [fake] * 11, 11) == INVALID              # a list of no entries
    many = params(top_k=33).to_c()
    assert call(lib, "ulorl_token_scores", many, [fake] * 9, 9) == UNSUPPORTED
    more = params(V=3).to_c()
    assert call(lib, "ulorl_token_scores", more, [fake] * 9, 9) == INVALID             # top_k > V


def test_logits_refusals(lib):
    fake = ctypes.c_void_p(1 << 20)
    f = lambda dtype=0, T=4, V=10, ld=10, k=2, kappa=1.0, logits=fake, targets=fake, ids=fake, logp=fake: lib.ulorl_logits_scores(
        logits, dtype, T, V, ld, k, kappa, targets, logp, None, None, ids, ids, None)
    assert f(dtype=3) == -2 and f(k=33, V=50, ld=50) == -2
    assert f(kappa=2e6) == -2 and f(kappa=5e-7) == -2 and f(V=2 ** 31 - 1, ld=2 ** 31) == -2 and f(T=2 ** 30 + 1) == -2
    for kw in (dict(T=-1), dict(V=0), dict(ld=9), dict(k=-1), dict(k=11), dict(kappa=0.0), dict(kappa=float("nan")), dict(logits=None),
               dict(targets=None), dict(ids=None), dict(k=0), dict(logits=ctypes.c_void_p((1 << 20) + 2))):
        assert f(**kw) == -1, kw
    assert f(T=0, ids=None) == 0


def test_python_side_refusals(lib):
    h, w = torch.zeros(8, 64, dtype=torch.bfloat16), torch.zeros(100, 64, dtype=torch.bfloat16)
    with pytest.raises(U.UlorlError, match="CUDA"):
        U.token_scores(params(), h, w)
    with pytest.raises(U.UlorlError, match="CUDA"):
        U.logits_scores(torch.zeros(2, 5))
    with pytest.raises(U.UlorlError, match="CUDA"):
        U.distill_fwd(params(), h, w, None, None)
    with pytest.raises(U.UlorlError, match="sizes"):                   # would be 8 in the 32 bits of the C side
        U.HeadParams(T=2 ** 32 + 8, H=64, V=100).to_c()
