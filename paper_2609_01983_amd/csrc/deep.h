// Launches of the operators of deep GCNs, between the entry points (api.hip) and the kernels.
#pragma once

#include "internal.h"

namespace dgc {

// ---- norms around a block (norm.hip): arguments as dualgcn_norm_residual and its backward pass
// take them, checked
constexpr int kMaxNormWidth = 8192;
int launch_norm_residual(const dualgcn_norm &p, const void *R, const void *B, void *Rn, void *Z, int32_t n,
                         int32_t F, hipStream_t stream);
size_t norm_backward_workspace_bytes(int32_t n, int32_t F);
int launch_norm_backward(const dualgcn_norm &p, const void *Rn, const void *B, const void *dZ, const void *dRn,
                         void *dR, void *dB, const dualgcn_norm_grads &g, int32_t n, int32_t F, void *workspace,
                         hipStream_t stream);

// ---- distillation (distill.hip): arguments as dualgcn_distill_xent takes them, checked
size_t distill_workspace_bytes(int32_t n, int32_t C);
int launch_distill(const void *Y, bool y_bf16, const int32_t *ids, const void *teacher, bool t_bf16,
                   const int32_t *labels, int32_t n, int32_t C, int32_t K, float T, float soft, float hard, void *G,
                   bool g_bf16, float *loss, void *workspace, hipStream_t stream);

// ---- the update phase in 8 bits (fp8.hip): arguments as the entry points take them, checked
constexpr int kFp8Block = DUALGCN_FP8_BLOCK;
int launch_quantize(const void *X, bool bf16, int32_t n, int32_t F, void *Q, float *scales, hipStream_t stream);
int launch_quantize_weight(const float *W, int32_t rows, int32_t cols, bool transpose, void *Q, float *scales,
                           hipStream_t stream);
int launch_update_fp8(const void *X, const float *sx, const void *W, const float *sw, void *T, bool out_bf16,
                      int32_t n, int32_t F_in, int32_t F_out, hipStream_t stream);

}  // namespace dgc
