"""S2O causal prefill attention, and the key/value cache's operators behind it, for AMD MI355X (gfx950): hand-written HIP kernels behind a
C ABI (include/s2o.h, libs2o.so) plus this thin ctypes binding.  Importing the package does
not load the library; the first call does, and fails loudly if it has not been built."""
from .binding import (Evicted, Plan, S2ODecodeParams, S2OError, S2OEvictParams, S2OParams, S2OWeightsParams,  # noqa: F401
                      load_library, make_decode_params, make_evict_params, make_params, make_weights_params, s2o_attention,
                      s2o_attention_local, s2o_attention_prefix, s2o_attention_sizes, s2o_decode, s2o_decode_sizes, s2o_evict,
                      s2o_evict_sizes, s2o_key_weights, s2o_key_weights_sizes, s2o_plan, s2o_plan_sizes)
