"""MI355X-native NSA speculative-verification attention (the hot path of SSV, arxiv 2605.19893).

The product is the HIP library behind include/ssv_nsa.h and include/ssv_round.h; this package is its thin Python binding.
"""
from .binding import (SSV_BF16, SSV_F32, SSV_REFRESH, SSV_REFRESH_SHARED, SSV_REUSE, SsvCmpParams, SsvCommitParams, SsvError,  # noqa: F401
                      SsvNsaParams, SsvNsaPlan, SsvPrefixParams, SsvSampleParams, load_library, make_cmp_params, make_commit_params,
                      make_params, make_prefix_params, make_sample_params, ssv_accept, ssv_commit, ssv_nsa_compress,
                      ssv_nsa_plan_query, ssv_nsa_supported, ssv_nsa_verify, ssv_nsa_verify_static, ssv_nsa_workspace_bytes,
                      ssv_prefix_verify, ssv_prefix_workspace_bytes, ssv_sample, ssv_sample_workspace_bytes)
