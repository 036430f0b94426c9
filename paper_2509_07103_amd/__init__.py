"""MI355X-native lmKAN layer: Python names mirror the C ABI of include/lmkan.h."""
from .binding import (LMKAN_BF16, LMKAN_F16, LMKAN_F32, LMKAN_FLAG_ACCUMULATE_GRAD_COEF, LMKAN_FLAG_WORKSPACE_HAS_RECORDS,
                      LMKAN_LAYOUT_PACKED, LMKAN_LAYOUT_PAPER, LMKAN_MAX_GRID, LMKAN_PACK_TILE, LMKAN_LINEAR_RELU, LMKAN_MAX_ORTHO_STEPS,
                      LMKAN_STATIC_SCRATCH_BYTES, QUINTIC_SCHEDULE,
                      Conv2d, LayerDesc, LinearDesc, LmkanError, MatrixDesc, MuonParams, lib, lmkan_backward, lmkan_conv2d_backward,
                      lmkan_conv2d_forward, lmkan_conv2d_rows, lmkan_forward, lmkan_forward_static, lmkan_grid,
                      lmkan_fold, lmkan_hessian_reg,
                      lmkan_locate, lmkan_microbench, MICROBENCH, lmkan_pack, lmkan_time_next_kernel, lmkan_packed_bytes, lmkan_status_string,
                      lmkan_version, lmkan_workspace_bytes,
                      lmkan_orthogonalize, lmkan_orthogonalize_workspace_bytes, lmkan_muon_step, lmkan_quantize_rows,
                      lmkan_linear_i8, lmkan_linear_i8_workspace_bytes,
                      LMKAN_CHECKPOINT_BLOCK, LMKAN_LINEAR_ACCUMULATE, LMKAN_MAX_ADAPTER_RANK, LMKAN_MAX_ADAPTERS,
                      LMKAN_NORM_ACCUMULATE, AdapterDesc, NormDesc, lmkan_adapters_add, lmkan_adapters_workspace_bytes,
                      lmkan_checkpoint_exps_bytes, lmkan_checkpoint_rows, lmkan_layer_norm, lmkan_layer_norm_backward,
                      lmkan_layer_norm_backward_workspace_bytes, lmkan_linear_grad, lmkan_linear_grad_workspace_bytes,
                      lmkan_restore_rows)

__all__ = [n for n in dir() if n.startswith(("lmkan_", "LMKAN_", "Layer", "Lmkan", "Conv2d", "lib", "MICROBENCH",
                                            "Linear", "Matrix", "Muon", "QUINTIC", "Norm", "Adapter"))]
