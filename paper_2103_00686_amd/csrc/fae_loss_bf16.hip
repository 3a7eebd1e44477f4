// Softmax cross entropy: the kernels for bf16 rows.
#define LOSS_KERNELS
#include "fae_loss.h"

void loss_launch_bf16(fae_ctx *ctx, int mode, const loss_args &a) { loss_launch<LOSS_BF16>(ctx, mode, a); }
