// Layer norm's forward of fp32 rows.
#include "fae_norm.h"

void norm_fwd_by_type(fae_ctx *ctx, const fae_norm *n, const NormShape &s, const NormArgs &a)
{
    if (n->y_type == FAE_F32)
        norm_by_width<false, float, float>(ctx, s, a);
    else if (n->y_type == FAE_BF16)
        norm_by_width<false, float, fae_bf16>(ctx, s, a);
    else
        norm_by_width<false, float, fae_f16>(ctx, s, a);
}
