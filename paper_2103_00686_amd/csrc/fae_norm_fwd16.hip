// Layer norm's forward of bf16 and fp16 rows.
#include "fae_norm.h"

void norm_fwd16_by_type(fae_ctx *ctx, const fae_norm *n, const NormShape &s, const NormArgs &a)
{
    if (n->x_type == FAE_BF16)
        norm_by_width<false, fae_bf16, fae_bf16>(ctx, s, a);
    else
        norm_by_width<false, fae_f16, fae_f16>(ctx, s, a);
}
