// Softmax cross entropy: the kernels for f16 rows.
#define LOSS_KERNELS
#include "fae_loss.h"

void loss_launch_f16(fae_ctx *ctx, int mode, const loss_args &a) { loss_launch<LOSS_F16>(ctx, mode, a); }
