"""MI355X-native receiver-side bounded-loss gradient aggregation (DBLP), and the two ends of a worker's
training step that makes the gradients.

Thin Python binding over the C-ABI library libdblp_agg.so (hand-written HIP
kernels for gfx950).  Argument marshalling only: every step of the path runs
in the library's kernels.  There is no CPU fallback; a missing library is an
error.
"""
from .binding import (Aggregator, ClrController, DblpError, lib, policy_linear, policy_three_level,  # noqa: F401
                      policy_two_level, sumsq_static)
from .worker import (Drop, dropout, embed, embed_grad, embed_grad_workspace, logits_workspace, policy_loss,  # noqa: F401
                     token_logprobs)
