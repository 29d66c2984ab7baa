/*
 * A plain C11 user of include/comp_ams_operators.h: proves that the header is C, and drives the host-side validation of its calls - the
 * part that answers before any device call - so that it can run under AddressSanitizer / UBSan on a machine without a GPU.
 * Returns 0 when every call answered as the header says.
 */
#include "comp_ams_operators.h"

#include <math.h>
#include <stdio.h>
#include <string.h>

#define EXPECT(call, want)                                                            \
    do {                                                                              \
        int got__ = (call);                                                           \
        if (got__ != (want)) {                                                        \
            printf("%s: got %d, expected %d\n", #call, got__, (int)(want));           \
            ++failures;                                                               \
        }                                                                             \
    } while (0)

int main(void)
{
    int failures = 0;
    static float buf[64];
    static int32_t ints[64];
    static int64_t longs[64];
    uint64_t bytes = 0;
    const int32_t bounds[3] = {-1, 0, 4}, bad[3] = {0, 0, 1};
    const int64_t st3[3] = {16, 16, 4}, st9[9] = {16, 16, 4, 16, 16, 4, 16, 16, 4};

    EXPECT(comp_ams_layer_norm(NULL, NULL, NULL, buf, buf, buf, 1, 4, 4, 4, 1e-5f, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_layer_norm(buf, NULL, NULL, buf, NULL, buf, 1, 4, 4, 4, 1e-5f, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_layer_norm(buf, NULL, NULL, buf, buf, buf, 2, 4, 3, 4, 1e-5f, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_layer_norm(buf, NULL, NULL, buf, buf, buf, INT64_MAX, 4, INT64_MAX, 4, 1e-5f, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_layer_norm(buf, NULL, NULL, buf, buf, buf, 2, 4, INT64_MAX, 4, 1e-5f, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_layer_norm(buf, NULL, NULL, buf, buf, buf, 0, 4, 4, 4, 1e-5f, COMP_AMS_BF16, NULL), COMP_AMS_OK);
    EXPECT(comp_ams_layer_norm_work_bytes(1024, 768, 8, &bytes), COMP_AMS_OK);
    EXPECT(bytes > 0 ? 0 : 1, 0);
    EXPECT(comp_ams_layer_norm_work_bytes(INT64_MAX, 768, 8, &bytes), COMP_AMS_EINVAL);
    EXPECT(comp_ams_layer_norm_work_bytes(7, 768, 2, &bytes), COMP_AMS_EINVAL);
    EXPECT(comp_ams_layer_norm_backward(buf, buf, NULL, buf, buf, buf, buf, buf, 4, 4, 4, 4, 4, 2, 4, COMP_AMS_F32, COMP_AMS_F16, NULL, 0, NULL),
           COMP_AMS_EINVAL);
    EXPECT(comp_ams_layer_norm_backward(buf, buf, NULL, buf, buf, buf, buf, buf, 4, 4, 4, 4, 4, 2, INT64_MAX, COMP_AMS_F32, COMP_AMS_F16, buf, 1 << 20, NULL),
           COMP_AMS_EINVAL);

    EXPECT(comp_ams_rel_bias_softmax(buf, buf, buf, bad, 4, NULL, 1, 1, 4, 4, st3, st3, 0, 1.f, 0, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_rel_bias_softmax(buf, buf, buf, bounds, 4, NULL, INT64_MAX, 1, 4, 4, st3, st3, 0, 1.f, 0, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_rel_bias_softmax(buf, buf, buf, bounds, 4, NULL, 1, 1, 4, 4, st3, st3, INT64_MIN, 1.f, 0, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_rel_bias_softmax(buf, buf, buf, bounds, 4, NULL, 1, 1, 4, 4, st3, st3, 0, NAN, 0, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_rel_bias_softmax(buf, buf, buf, bounds, 4, NULL, 1, 0, 4, 4, st3, st3, 0, 1.f, 0, COMP_AMS_F32, NULL), COMP_AMS_OK);
    EXPECT(comp_ams_rel_bias_softmax(NULL, buf, buf, bounds, 4, NULL, 1, 1, 4, 4, st3, st3, 0, 1.f, 0, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_rel_bias_work_bytes(1, 1, 4, 4, 4, COMP_AMS_F32, &bytes), COMP_AMS_OK);
    EXPECT(comp_ams_rel_bias_softmax_backward(buf, buf, buf, buf, bounds, 4, NULL, 1, 1, 4, 4, st9, 0, 1.f, 0, 1, 4, COMP_AMS_F32, COMP_AMS_F32, buf, 0,
                                              NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_rel_bias_softmax_backward(buf, buf, buf, buf, bounds, 4, NULL, 3, 1, 4, 4, st9, 0, 1.f, 0, 2, 4, COMP_AMS_F32, COMP_AMS_F32, buf,
                                              1 << 20, NULL), COMP_AMS_EINVAL);

    EXPECT(comp_ams_token_logprobs(buf, buf, ints, buf, buf, NULL, 2, 8, 8, 2, COMP_AMS_F32, NULL, 0, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_token_logprobs(buf, buf, ints, buf, buf, longs, 2, 8, 8, 9, COMP_AMS_F32, NULL, 0, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_token_logprobs(buf, buf, ints, buf, buf, longs, 0, 8, 8, 2, COMP_AMS_F32, NULL, 0, NULL), COMP_AMS_OK);
    EXPECT(comp_ams_token_logprobs_work_bytes(INT64_MAX, 8, 2, COMP_AMS_F32, &bytes), COMP_AMS_EINVAL);
    EXPECT(comp_ams_token_logprobs_work_bytes((int64_t)1 << 30, 400000, 128, COMP_AMS_F32, &bytes), COMP_AMS_OK);

    EXPECT(comp_ams_distill(buf, buf, buf, ints, buf, 2, 8, 8, 0, 1.f, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_distill(buf, buf, buf, ints, buf, 2, 8, 8, 2, -1.f, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_distill(buf, buf, buf, ints, buf, 0, 8, 8, 2, 1.f, COMP_AMS_F16, NULL), COMP_AMS_OK);
    EXPECT(comp_ams_distill_backward(buf, NULL, buf, buf, ints, buf, 2, 8, 8, 8, 2, 1.f, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_distill_grad(buf, NULL, buf, buf, ints, buf, 2, 8, 8, 8, 2, 1.f, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(strlen(comp_ams_operators_last_error()) > 0 ? 0 : 1, 0);

    printf("operators validation: %d failures\n", failures);
    return failures != 0;
}
