"""MI355X-native rank-order search: cost models over batches of rank orders (ring, halving-doubling, BCube,
double binary tree), multi-start 2-opt and pair-swap descents, integer simulated annealing, cost matrix from probes; the parts of a
learned policy over orders that matrix products do not cover (embedding, gated recurrence, norm, policy and preference losses, and for
sampling products in 8 bits and shaped logits).

Thin binding over the C ABI in include/cc.h; the computation lives in csrc/*.hip."""
from .binding import (CC_COST_MAX, CC_MAX_N, CC_MOVES_2OPT, CC_MOVES_FLIP, CC_MOVES_OROPT, CC_RING_MAX, CC_RING_MAX_DIRECTED, CC_RING_SUM,  # noqa: F401
                      CC_RING_SUM_DIRECTED, EXPORTS, LIB_PATH, OBJECTIVES, CCError, SearchBuffers, cc_2opt_search,
                      cc_2opt_search_ex, cc_2opt_search_noalloc, cc_2opt_workspace_bytes, cc_bcube_cost_batch, cc_bcube_cost_batch_weighted,
                      cc_best_of_restarts, cc_cost_matrix_from_probes, cc_dbt_cost_batch, cc_init_tours, cc_local_search, cc_local_search_ex,
                      cc_rd_batch_workspace_bytes, cc_rd_cost_batch, cc_rd_swap_search, cc_rd_swap_search_ex, cc_ring_cost_batch,
                      cc_ring_cost_batch_u16, cc_ring_cost_batch_u8, cc_sa_rd_search, cc_sa_rd_search_ex, cc_sa_search, cc_sa_search_ex,
                      cc_status_string, cc_validate_matrix, cc_version, lib)
from .order_model import (CC_MEAN_ORDERS, CC_MEAN_TOKENS, CC_SCAN_CHUNK, PolicyLoss, PreferenceLoss, RmsNorm, cc_embed,  # noqa: F401
                          cc_embed_backward, cc_embed_workspace_bytes, cc_gated_scan, cc_gated_scan_backward,
                          cc_gated_scan_workspace_bytes, cc_policy_loss, cc_preference_loss, cc_product_i8, cc_product_i8_workspace_bytes,
                          cc_quantize_rows, cc_rms_norm, cc_rms_norm_backward, cc_rms_norm_workspace_bytes, cc_shape_logits,
                          cc_shape_logits_backward, cc_token_logprob, cc_token_logprob_backward, cc_token_workspace_bytes)
