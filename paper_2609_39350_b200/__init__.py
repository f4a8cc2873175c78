"""B200-native planner hot path of HAPMoE: a thin ctypes binding over libhap.so.

Every step of the path (layer costs, candidate decode, pipeline dynamic program, argmin)
runs in the CUDA kernels of the library; this package only marshals arguments.  PyTorch is
used for device memory and streams.  There is no CPU fallback: if the library is missing
or no CUDA device is present, the calls raise.
"""
from .binding import (HapError, HapProblem, hap_problem_create, hap_enumerate, hap_get_pconfs, hap_decode,  # noqa: F401
                      hap_eval_layer_costs, hap_eval_layer_costs_f64, hap_pipeline_dp, hap_pipeline_dp_f64, hap_search_best,
                      hap_search_range_f64,
                      hap_search_range, hap_argmin, hap_argmin_static, hap_joint_bottleneck, hap_count_cells, hap_get_timings, hap_launches_per_pass, hap_eval_appendix_b, hap_simulate_1f1b, hap_release_cached_memory, hap_self_check, hap_problem_save, hap_problem_load, hap_problem_dims, hap_problem_destroy, load_library, EXPORTS, INF, COEF,
                      NCOEF, MAX_PP, OPT_NO_MAPTAB, OPT_REFINE, OPT_EXACT, OPT_UNIFORM, OPT_NO_TRIE, OPT_NO_FUSE, OPT_COUNT_SPLITS,
                      OPT_HETERO_DISPATCH)
from .operators import (EXPERT_FORWARD, EXPERT_GRAD_INPUT, EXPERT_GRAD_WEIGHT, HapAdamWTensors, hap_expert_matmul,  # noqa: F401,E402
                        hap_expert_gated, hap_expert_gated_backward, hap_linear_cross_entropy_workspace, hap_linear_cross_entropy,
                        hap_linear_cross_entropy_backward, hap_adamw_tensors, hap_adamw_step, hap_adamw_state, hap_operator_status,
                        hap_measure_workspace, hap_measure_profile)
from .tokens import (SOFTMAX, SIGMOID, HapRouting, hap_routing, hap_route, hap_route_backward, hap_expert_order_workspace, hap_expert_order,  # noqa: F401,E402
                     hap_expert_dispatch, hap_expert_combine, hap_expert_combine_backward, hap_embedding, hap_embedding_backward_workspace,
                     hap_embedding_backward, hap_layer_norm, hap_layer_norm_backward_workspace, hap_layer_norm_backward, hap_measure_tokens_workspace,
                     hap_measure_tokens)
