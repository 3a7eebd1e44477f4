// Softmax cross entropy: the kernels for f32 rows.
#define LOSS_KERNELS
#include "fae_loss.h"

void loss_launch_f32(fae_ctx *ctx, int mode, const loss_args &a) { loss_launch<float>(ctx, mode, a); }
