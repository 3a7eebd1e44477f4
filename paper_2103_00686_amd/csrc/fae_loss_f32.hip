// Softmax cross entropy: the kernels for f32 rows as three bf16 numbers each.
#define LOSS_KERNELS
#include "fae_loss.h"

void loss_launch_f32(fae_ctx *ctx, int mode, const loss_args &a) { loss_launch<LOSS_F32>(ctx, mode, a); }
