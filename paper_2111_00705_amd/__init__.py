"""MI355X (gfx950) library for communication-compressed distributed AMSGrad (error feedback and CD-Adam), and
operators of language-model training that write parameter gradients into the optimiser's rows.

The work is in csrc/ (hand-written HIP kernels behind the C ABI of
include/comp_ams.h and include/comp_ams_operators.h); this package only builds and binds it.
"""
from .binding import (BLOCKSIGN, EDEVICE, EINVAL, ENOMEM, ESTATE, EXPORTS, METHOD_CD, METHOD_EF, METHOD_NAIVE, METHOD_NONE, OK, RANDK, TOPK, CompAms,
                      CompAmsError, lib, probe_copy, probe_update)
from .operators import (distill, distill_backward, distill_grad, layer_norm, layer_norm_backward, rel_bias_bounds, rel_bias_softmax,
                        rel_bias_softmax_backward, token_logprobs)

__all__ = ["CompAms", "CompAmsError", "lib", "probe_copy", "probe_update", "TOPK", "BLOCKSIGN", "RANDK", "METHOD_EF", "METHOD_CD", "METHOD_NAIVE", "METHOD_NONE", "EXPORTS",
           "OK", "EINVAL", "ENOMEM", "EDEVICE", "ESTATE", "layer_norm", "layer_norm_backward", "rel_bias_bounds", "rel_bias_softmax",
           "rel_bias_softmax_backward", "token_logprobs", "distill", "distill_backward", "distill_grad"]
