/* The norms, rotations and distillation of include/eager_model.h in a C99 translation unit: declared types, layouts, and
 * the calls that need no GPU.  Compiled, linked and run by tests/test_hidden_host.py. */
#include "eager_model.h"

#include <stddef.h>

typedef char check_rows[sizeof(eager_rows) == 16 ? 1 : -1];
typedef char check_angles[(sizeof(eager_angles) == 64 && offsetof(eager_angles, base) == 16 && offsetof(eager_angles, magnitude) == 56) ? 1 : -1];
typedef char check_teacher[(sizeof(eager_teacher) == 24 && offsetof(eager_teacher, temperature) == 20) ? 1 : -1];

int (*const p_norm)(int, int64_t, int32_t, const eager_rows *, const eager_rows *, const void *, const void *, float,
                    const eager_rows *, const eager_rows *, float *, void *) = eager_layer_norm;
int (*const p_norm_backward)(int, int64_t, int32_t, const eager_rows *, const eager_rows *, const eager_rows *, const void *,
                             const float *, const eager_rows *, void *, void *, void *, int64_t, void *) = eager_layer_norm_backward;
int (*const p_table)(const eager_angles *, float *, float *, void *) = eager_rotary_table;
int (*const p_rotary)(int, const eager_packed *, const eager_heads *, const eager_heads *, const eager_rotation *, int32_t, int,
                      const eager_heads *, const eager_heads *, void *) = eager_rotary;
int (*const p_rotary_backward)(int, const eager_packed *, const eager_heads *, const eager_heads *, const eager_rotation *,
                               int32_t, int, const eager_heads *, const eager_heads *, void *) = eager_rotary_backward;
int (*const p_taught)(int, const eager_projection *, const void *, const void *, const eager_teacher *, float *, float *,
                      float *, void *, int64_t, void *) = eager_distillation;
int (*const p_taught_backward)(int, const eager_projection *, const void *, const void *, const eager_teacher *,
                               const float *, const float *, const float *, void *, void *, void *, int64_t, void *) =
    eager_distillation_backward;

int main(void)
{
    eager_projection projection = {100, 64, 1000, 64, 64};
    eager_angles angles = {0, 64, EAGER_ANGLES_PLAIN, 10000.0, 0.0, 0.0, 0.0, 0.0, 1.0};
    int64_t bytes = 0, more = 0;
    if (eager_layer_norm_workspace_bytes(EAGER_BF16, 1000, 1024, &bytes) != EAGER_OK || bytes < 2 * 1024 * 4) return 1;
    if (eager_distillation_workspace_bytes(EAGER_F32, &projection, 16, 1, &more) != EAGER_OK ||
        eager_cross_entropy_workspace_bytes(EAGER_F32, &projection, 1, &bytes) != EAGER_OK || more < bytes + 800) return 2;
    if (eager_rotary_table(&angles, 0, 0, 0) != EAGER_OK) return 3;             /* a table of no positions */
    angles.part = 12;
    if (eager_rotary_table(&angles, 0, 0, 0) != EAGER_EINVAL) return 4;
    if (eager_rotary(EAGER_F32, 0, 0, 0, 0, 8, EAGER_ROTARY_HALVES, 0, 0, 0) != EAGER_EINVAL) return 5;
    return 0;
}
