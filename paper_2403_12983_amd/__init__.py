"""MI355X-native OSSCAR layer solver: thin ctypes binding over libosscar.so (hand-written HIP, gfx950)."""
from .binding import (OSSCAR_ACT_GELU, OSSCAR_ACT_GELU_TANH, OSSCAR_ACT_RELU, OSSCAR_ACT_SILU, OSSCAR_BF16, OSSCAR_F32, OSSCAR_I8, OSSCAR_INIT_GIVEN, OSSCAR_INIT_MAGNITUDE, OSSCAR_SEARCH_ALWAYS_ACCEPT,
                      OSSCAR_SEARCH_EAGER, OSSCAR_SEARCH_EXACT_IN, OSSCAR_SEARCH_IMPATIENT, OSSCAR_SEARCH_IMPATIENT_LATER, OSSCAR_SEARCH_LAUNCH_PER_SWAP, OSSCAR_SEARCH_NO_LOOKAHEAD, OsscarError, Solver, lib_path, load_library, osscar_gram_static, EXPORTED_SYMBOLS)
from .layer_ops import (LogProbs, osscar_gated_backward, osscar_gated_forward, osscar_int_product, osscar_int_rows, osscar_int_weights,
                        osscar_logprobs, osscar_logprobs_backward)

__all__ = ["Solver", "OsscarError", "osscar_gram_static", "load_library", "lib_path", "EXPORTED_SYMBOLS", "OSSCAR_F32", "OSSCAR_BF16",
           "OSSCAR_INIT_MAGNITUDE", "OSSCAR_INIT_GIVEN", "OSSCAR_SEARCH_ALWAYS_ACCEPT", "OSSCAR_SEARCH_EAGER", "OSSCAR_SEARCH_NO_LOOKAHEAD", "OSSCAR_SEARCH_EXACT_IN",
           "OSSCAR_I8", "OSSCAR_ACT_SILU", "OSSCAR_ACT_GELU", "OSSCAR_ACT_GELU_TANH", "OSSCAR_ACT_RELU", "LogProbs",
           "osscar_gated_forward", "osscar_gated_backward", "osscar_int_weights", "osscar_int_rows", "osscar_int_product",
           "osscar_logprobs", "osscar_logprobs_backward",
           "OSSCAR_SEARCH_LAUNCH_PER_SWAP", "OSSCAR_SEARCH_IMPATIENT", "OSSCAR_SEARCH_IMPATIENT_LATER"]
