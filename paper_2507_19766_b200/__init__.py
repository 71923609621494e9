"""B200-native fused UloRL token-loss path (LM head + log-softmax + entropy + SAIS/POIS ratio +
MPT mask + clipped token-normalised loss, forward and backward) behind a C ABI, with token scores and
distillation from a teacher's top logits on the same head.

`binding` wraps libulorl.so (hand-written CUDA for sm_100a); `head` the scoring and distillation calls; `dp` is the
host logic of the data-parallel step (rank launch, sharding, the collectives); `segments` the bookkeeping of the
segment rollout.  Importing the package does not load the library; the first call does and raises if it is missing.
"""
from . import binding, dp, head  # noqa: F401
from .binding import (Params, UlorlError, alloc_fwd_outputs, alloc_workspace, check_status, launch_count,  # noqa: F401
                      token_loss_bwd, token_loss_decide, token_loss_fwd, workspace_bytes)
from .head import (HeadParams, alloc_head_workspace, distill_bwd, distill_fwd, head_workspace_bytes,  # noqa: F401
                   logits_scores, token_scores, token_scores_bwd)
