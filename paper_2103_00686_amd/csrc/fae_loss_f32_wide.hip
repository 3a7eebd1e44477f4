// Softmax cross entropy: the kernels for f32 rows as two fp16 numbers each.
#define LOSS_KERNELS
#include "fae_loss.h"

void loss_launch_f32_wide(fae_ctx *ctx, int mode, const loss_args &a) { loss_launch<LOSS_F32_WIDE>(ctx, mode, a); }
