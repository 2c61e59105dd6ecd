/* include/eager_model.h in a C99 translation unit: every entry point with its declared type, the layout of
 * the structures, and the calls that need no GPU.  Compiled, linked and run by tests/test_model_host.py. */
#include "eager_model.h"

#include <stddef.h>

typedef char check_heads[sizeof(eager_heads) == 24 ? 1 : -1];
typedef char check_packed[(sizeof(eager_packed) == 32 && offsetof(eager_packed, cu_seqlens) == 24) ? 1 : -1];
typedef char check_rotation[(sizeof(eager_rotation) == 32 && offsetof(eager_rotation, table_rows) == 24) ? 1 : -1];
typedef char check_projection[(sizeof(eager_projection) == 32 && offsetof(eager_projection, x_stride) == 16) ? 1 : -1];

int (*const p_norm)(int, const eager_packed *, const eager_heads *, const eager_heads *, const void *, const void *,
                    const eager_rotation *, float, const eager_heads *, const eager_heads *, void *) = eager_qk_norm_rope;
int (*const p_norm_backward)(int, const eager_packed *, const eager_heads *, const eager_heads *, const eager_heads *,
                             const eager_heads *, const void *, const void *, const eager_rotation *, float,
                             const eager_heads *, const eager_heads *, void *, void *, void *, int64_t, void *) =
    eager_qk_norm_rope_backward;
int (*const p_attention)(int, const eager_packed *, const eager_heads *, const eager_heads *, const eager_heads *, float,
                         const eager_heads *, float *, void *) = eager_attention;
int (*const p_attention_backward)(int, const eager_packed *, const eager_heads *, const eager_heads *, const eager_heads *,
                                  const eager_heads *, const float *, const eager_heads *, float, const eager_heads *,
                                  const eager_heads *, const eager_heads *, void *, int64_t, void *) = eager_attention_backward;
int (*const p_loss)(int, const eager_projection *, const void *, const void *, const int64_t *, float *, float *, void *,
                    int64_t, void *) = eager_cross_entropy;
int (*const p_loss_backward)(int, const eager_projection *, const void *, const void *, const int64_t *, const float *,
                             const float *, void *, void *, void *, int64_t, void *) = eager_cross_entropy_backward;

int main(void)
{
    const int32_t *cu = (const int32_t *)(uintptr_t)4096;
    eager_packed shape = {100, 4, 2, 64, 3, 0};
    eager_projection projection = {100, 64, 1000, 64, 64};
    int64_t bytes = 0;
    if (eager_attention_workspace_bytes(EAGER_BF16, &shape, &bytes) != EAGER_OK || bytes < 2 * 4 * 100 * 4) return 1;
    if (eager_qk_norm_rope_workspace_bytes(EAGER_F32, &shape, &bytes) != EAGER_OK || bytes < 2 * 64 * 4) return 2;
    if (eager_cross_entropy_workspace_bytes(EAGER_F32, &projection, 0, &bytes) != EAGER_OK || bytes <= 0) return 3;
    if (eager_cross_entropy_workspace_bytes(EAGER_F32, &projection, 1, &bytes) != EAGER_OK || bytes < 100 * 1000 * 4) return 4;
    shape.cu_seqlens = cu;
    if (eager_attention(EAGER_BF16, &shape, 0, 0, 0, 1.0f, 0, 0, 0) != EAGER_EINVAL) return 5;
    return 0;
}
