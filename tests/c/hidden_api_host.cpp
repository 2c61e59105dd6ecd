// The host side of layer norm, rotation and distillation (eager_model_api.cpp) compiled WITHOUT the kernels, the launchers
// replaced by recorders: what each call hands over, under AddressSanitizer and UndefinedBehaviorSanitizer on the CPU.
// Built and run by tests/test_hidden_host.py.
#include "../../include/eager_model.h"
#include "../../paper_1908_04207_amd/csrc/eager_model.h"
#include "../../paper_1908_04207_amd/csrc/eager_model_rules.h"

#include <cmath>
#include <cstdio>
#include <cstdlib>

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); std::exit(1); } } while (0)

static int launches;
static hipError_t answer = hipSuccess;
static bool last_bf16, last_interleaved;
static eager::LayerNormArgs norm;
static eager::RotaryArgs rotary;
static eager::TableArgs table;
static eager::CrossEntropyArgs loss;

namespace eager {
hipError_t launch_norm_rope(const NormRopeArgs &, bool, hipStream_t) { std::abort(); }
hipError_t launch_norm_rope_backward(const NormRopeArgs &, bool, hipStream_t) { std::abort(); }
hipError_t launch_attention(const AttentionArgs &, bool, hipStream_t) { std::abort(); }
hipError_t launch_attention_backward(const AttentionArgs &, bool, hipStream_t) { std::abort(); }
hipError_t launch_cross_entropy(const CrossEntropyArgs &a, bool b, hipStream_t) { loss = a, last_bf16 = b, ++launches; return answer; }
hipError_t launch_cross_entropy_backward(const CrossEntropyArgs &a, bool b, hipStream_t) { loss = a, last_bf16 = b, ++launches; return answer; }
hipError_t launch_layer_norm(const LayerNormArgs &a, bool b, hipStream_t) { norm = a, last_bf16 = b, ++launches; return answer; }
hipError_t launch_layer_norm_backward(const LayerNormArgs &a, bool b, hipStream_t) { norm = a, last_bf16 = b, ++launches; return answer; }
hipError_t launch_rotary(const RotaryArgs &a, bool b, bool i, hipStream_t) { rotary = a, last_bf16 = b, last_interleaved = i, ++launches; return answer; }
hipError_t launch_rotary_table(const TableArgs &a, hipStream_t) { table = a, ++launches; return answer; }
}  // namespace eager

// addresses that nothing reads
static void *at(int n) { return reinterpret_cast<void *>(static_cast<uintptr_t>(0x10000 * (n + 1))); }
static float *floats(int n) { return static_cast<float *>(at(n)); }

static void layer_norms()
{
    const eager_rows x = {at(0), 512}, r = {at(1), 520}, s = {at(2), 528}, y = {at(3), 536}, d = {at(4), 544};
    CHECK(eager_layer_norm(EAGER_BF16, 40, 512, &x, &r, at(5), at(6), 0.25f, &s, &y, floats(7), nullptr) == EAGER_OK);
    CHECK(launches == 1 && last_bf16 && norm.x.data == at(0) && norm.residual.stride == 520 && norm.sum.data == at(2) &&
          norm.y.stride == 536 && norm.w == at(5) && norm.b == at(6) && norm.stats == at(7) && norm.rows == 40 && norm.width == 512 &&
          norm.eps == 0.25f && norm.inv_width == 1.0f / 512);
    CHECK(eager_layer_norm(EAGER_F32, 40, 512, &x, nullptr, at(5), nullptr, 0.0f, nullptr, &x, floats(7), nullptr) == EAGER_OK);
    CHECK(!last_bf16 && !norm.residual.data && !norm.sum.data && !norm.b && norm.y.data == at(0));
    // in an input's place: either output, either input; a lone row may have any stride
    CHECK(eager_layer_norm(EAGER_F32, 40, 512, &x, &r, at(5), nullptr, 0.0f, &r, &x, floats(7), nullptr) == EAGER_OK);
    const eager_rows other = {at(0), 1024};
    CHECK(eager_layer_norm(EAGER_F32, 40, 512, &x, &r, at(5), nullptr, 0.0f, &s, &other, floats(7), nullptr) == EAGER_EINVAL);
    CHECK(eager_layer_norm(EAGER_F32, 1, 512, &x, &r, at(5), nullptr, 0.0f, &s, &other, floats(7), nullptr) == EAGER_OK);
    int64_t bytes = -1;
    CHECK(eager_layer_norm_workspace_bytes(EAGER_F32, 4000, 512, &bytes) == EAGER_OK && bytes == 256 * 2 * 512 * 4);
    launches = 0;
    CHECK(eager_layer_norm_backward(EAGER_F32, 4000, 512, &y, &r, &s, at(5), floats(7), &d, at(8), nullptr, at(9), bytes, nullptr) == EAGER_OK);
    CHECK(launches == 1 && norm.x.data == at(2) && norm.residual.data == at(1) && norm.sum.data == at(4) && norm.y.data == at(3) &&
          norm.dw == at(8) && !norm.db && norm.partials == at(9) && norm.blocks == 256 && norm.rows == 4000);
    CHECK(eager_layer_norm_backward(EAGER_F32, 4000, 512, &y, &r, &s, at(5), floats(7), &d, at(8), nullptr, at(9), bytes - 1, nullptr) == EAGER_EINVAL);
    CHECK(eager_layer_norm_workspace_bytes(EAGER_F32, 30, 512, &bytes) == EAGER_OK && bytes == 0);
    CHECK(eager_layer_norm_backward(EAGER_F32, 30, 512, &y, nullptr, &s, at(5), floats(7), &y, nullptr, at(8), nullptr, 0, nullptr) == EAGER_OK);
    CHECK(norm.blocks == 1 && !norm.residual.data && !norm.dw && norm.db == at(8));
    // no rows: the sums over them are still asked for
    CHECK(eager_layer_norm_backward(EAGER_F32, 0, 512, &y, nullptr, &s, at(5), nullptr, &y, at(8), at(8), nullptr, 0, nullptr) == EAGER_OK && norm.blocks == 0);
    answer = hipErrorLaunchFailure;
    CHECK(eager_layer_norm(EAGER_F32, 1, 512, &x, nullptr, at(5), nullptr, 0.0f, nullptr, &y, floats(7), nullptr) == EAGER_EDEVICE);
    answer = hipSuccess;
}

static void rotations()
{
    const eager_packed shape = {100, 6, 3, 64, 0, nullptr};
    const eager_heads q = {at(0), 1024, 64}, k = {at(1), 1024, 64}, yq = {at(2), 384, 64}, yk = {at(3), 192, 64};
    const eager_rotation rot = {floats(4), floats(5), static_cast<int32_t *>(at(6)), 50};
    CHECK(eager_rotary(EAGER_BF16, &shape, &q, &k, &rot, 48, EAGER_ROTARY_INTERLEAVED, &yq, &yk, nullptr) == EAGER_OK);
    CHECK(last_bf16 && last_interleaved && rotary.half == 24 && rotary.sign == 1.0f && rotary.moved[0] == 64 && rotary.moved[1] == 64 &&
          rotary.heads[0] == 6 && rotary.heads[1] == 3 && rotary.tokens == 100 && rotary.table_rows == 50 && rotary.x[1].data == at(1) &&
          rotary.y[0].row == 384);
    for (int i = 0; i < 2; ++i) CHECK(rotary.groups[i] * eager::kTurnedHeads >= rotary.heads[i] && (rotary.groups[i] - 1) * eager::kTurnedHeads < rotary.heads[i]);
    // in place: what is not turned is not moved, array by array
    CHECK(eager_rotary_backward(EAGER_F32, &shape, &q, &k, &rot, 48, EAGER_ROTARY_HALVES, &q, &yk, nullptr) == EAGER_OK);
    CHECK(!last_bf16 && !last_interleaved && rotary.sign == -1.0f && rotary.moved[0] == 48 && rotary.moved[1] == 64);
    const eager_heads wide = {at(0), 2048, 64}, far = {at(0), 1024, 128};
    CHECK(eager_rotary(EAGER_F32, &shape, &q, &k, &rot, 48, EAGER_ROTARY_HALVES, &wide, &yk, nullptr) == EAGER_EINVAL);
    CHECK(eager_rotary(EAGER_F32, &shape, &q, &k, &rot, 48, EAGER_ROTARY_HALVES, &far, &yk, nullptr) == EAGER_EINVAL);
    const eager_packed one = {1, 1, 1, 64, 0, nullptr};
    CHECK(eager_rotary(EAGER_F32, &one, &far, &k, &rot, 48, EAGER_ROTARY_HALVES, &wide, &yk, nullptr) == EAGER_OK);
}

static void tables()
{
    const long double pi = 3.14159265358979323846264338327950288L;
    for (int scaling = EAGER_ANGLES_PLAIN; scaling <= EAGER_ANGLES_PARTS; ++scaling)
        for (int part : {8, 24, 64, 128}) {
            const eager_angles t = {1000, part, scaling, 20000.0, 12.0, 300.0, 2.0, 20.0, 0.75};
            CHECK(eager_rotary_table(&t, floats(0), floats(1), nullptr) == EAGER_OK);
            CHECK(table.half == part / 2 && table.positions == 1000 && table.magnitude == 0.75 && table.cos_table == floats(0) && table.sin_table == floats(1));
            for (int i = 0; i < part / 2; ++i) {
                long double base = 20000.0L, f;
                if (scaling == EAGER_ANGLES_BASE) base *= powl(12.0L, static_cast<long double>(part) / (part - 2));
                f = powl(base, -2.0L * i / part);
                if (scaling == EAGER_ANGLES_LINEAR) f /= 12;
                if (scaling == EAGER_ANGLES_PARTS) {
                    const long double turns = 300 * f / (2 * pi), keep = turns >= 20 ? 1 : turns <= 2 ? 0 : (turns - 2) / 18;
                    f = keep * f + (1 - keep) * f / 12;
                }
                CHECK(fabsl(table.quarters[i] - f * 2 / pi) <= 4e-15L * f);
            }
        }
}

static void teachers()
{
    const eager_projection shape = {70, 64, 999, 64, 72};
    const eager_teacher t = {static_cast<int64_t *>(at(0)), floats(1), 17, 3.0f};
    int64_t forward = 0, backward = 0;
    CHECK(eager_distillation_workspace_bytes(EAGER_BF16, &shape, 17, 0, &forward) == EAGER_OK);
    CHECK(eager_distillation_workspace_bytes(EAGER_BF16, &shape, 17, 1, &backward) == EAGER_OK);
    launches = 0;
    CHECK(eager_distillation(EAGER_BF16, &shape, at(2), at(3), &t, floats(4), floats(5), floats(6), at(7), forward, nullptr) == EAGER_OK);
    CHECK(launches == 1 && last_bf16 && loss.teacher.index == at(0) && loss.teacher.logits == at(1) && loss.teacher.entries == 17 &&
          loss.teacher.temperature == 3.0f && loss.teacher.picked == at(6) && loss.loss == at(4) && loss.lse == at(5) && !loss.target &&
          loss.workspace == at(7) && loss.rows == 70 && loss.vocab == 999 && loss.w_stride == 72);
    CHECK(eager_distillation_backward(EAGER_BF16, &shape, at(2), at(3), &t, floats(4), floats(5), floats(6), at(8), nullptr, at(7), backward, nullptr) == EAGER_OK);
    CHECK(launches == 2 && loss.lse == at(4) && loss.teacher.picked == at(5) && loss.dloss == at(6) && loss.dx == at(8) && !loss.dw && !loss.loss);
    // the cross entropy has no teacher
    CHECK(eager_cross_entropy_workspace_bytes(EAGER_BF16, &shape, 0, &forward) == EAGER_OK);
    CHECK(eager_cross_entropy(EAGER_BF16, &shape, at(2), at(3), static_cast<int64_t *>(at(0)), floats(4), floats(5), at(7), forward, nullptr) == EAGER_OK);
    CHECK(loss.target == at(0) && !loss.teacher.index);
}

int main()
{
    layer_norms();
    rotations();
    tables();
    teachers();
    std::puts("ok");
    return 0;
}
