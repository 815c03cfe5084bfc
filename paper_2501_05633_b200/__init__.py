"""B200-native RegTop-k sparsification step (arXiv 2501.05633, Algorithm 2) behind a C ABI.

`binding` marshals torch tensors into the C calls of include/regtopk.h; every step of the method runs
in the CUDA library (csrc/regtopk.cu).  `synth` holds the seeded synthetic input generators; it
contains none of the method's arithmetic.  `training` marshals into the calls of include/regtopk_train.h: the
operators of a backward pass that fills the sparsifier's accumulator rows (csrc/dropout_norm.cu, csrc/grouped_matmul.cu).
`experts` does so for include/regtopk_experts.h: routing, moving tokens, activations kept in 8 bits and the root-mean-square norm of
an expert sublayer (csrc/route.cu, csrc/move_tokens.cu, csrc/activation.cu, csrc/rms_norm.cu).
"""
from .binding import RegTopK, RegTopKError, aggregate_pairs_static, build, load_library, library_path  # noqa: F401
from .training import dropout, grouped_matmul, grouped_matmul_dw, layer_norm, layer_norm_backward, training_status  # noqa: F401
from .experts import (Rows8, activation, activation_backward, join_tokens, join_tokens_backward, pack8, rms_norm,  # noqa: F401
                      rms_norm_backward, route, route_backward, sort_tokens, spread_tokens, unpack8)
