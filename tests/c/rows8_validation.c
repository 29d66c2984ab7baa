/*
 * A plain C11 user of include/comp_ams_rows8.h: proves that the header is C, and drives the host-side validation of its calls - the part
 * that answers before any device call - so that it can run under AddressSanitizer / UBSan on a machine without a GPU.
 * Returns 0 when every call answered as the header says.
 */
#include "comp_ams_rows8.h"

#include <math.h>
#include <stdio.h>

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
    static int8_t bytes8[64];
    uint64_t bytes = 0;
    const int64_t far = INT64_MAX;

    EXPECT(comp_ams_quantize_rows(bytes8, buf, buf, far, 4, 4, 4, 0, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_quantize_rows(bytes8, buf, buf, 2, 4, far, 4, 0, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_quantize_rows(NULL, NULL, NULL, 0, 4, 4, 4, 1, COMP_AMS_F16, NULL), COMP_AMS_OK);
    EXPECT(comp_ams_restore_rows(buf, bytes8, buf, 2, far, 4, 4, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_restore_rows(NULL, NULL, buf, 5, 0, 0, 0, COMP_AMS_F32, NULL), COMP_AMS_OK);
    EXPECT(comp_ams_rms_norm(buf, NULL, NULL, buf, NULL, buf, 2, 4, 4, 4, far, 4, 1e-5f, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_rms_norm(buf, NULL, NULL, buf, NULL, buf, far, 4, 4, 4, far, 4, 1e-5f, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_rms_norm(buf, NULL, NULL, buf, NULL, buf, 1, 4, 4, 4, 4, 4, NAN, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_rms_norm(NULL, NULL, NULL, NULL, NULL, buf, 0, 4, 4, 4, 4, 4, 0.f, COMP_AMS_BF16, NULL), COMP_AMS_OK);
    EXPECT(comp_ams_rms_norm_q8(bytes8, NULL, NULL, NULL, buf, NULL, buf, 2, 4, 4, 4, 4, 4, 1e-5f, 0, COMP_AMS_F32, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_rms_norm_backward(buf, buf, buf, buf, NULL, buf, buf, NULL, 4, 4, 4, 4, 4, 4, 3, 4, COMP_AMS_F32, COMP_AMS_F32, buf, 256, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_rms_norm_backward(buf, buf, buf, buf, NULL, buf, buf, NULL, 4, 4, 4, 4, 4, 4, 2, far, COMP_AMS_F32, COMP_AMS_F32, buf, 256, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_rms_norm_work_bytes(1024, 768, 8, &bytes), COMP_AMS_OK);
    EXPECT(bytes > 0 ? 0 : 1, 0);
    EXPECT(comp_ams_rms_norm_work_bytes(far, 768, 8, &bytes), COMP_AMS_EINVAL);
    EXPECT(comp_ams_linear_q8(buf, bytes8, buf, bytes8, buf, NULL, 2, 4, 3, 3, far, 4, COMP_AMS_F32, NULL, 0, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_linear_q8(buf, bytes8, buf, bytes8, buf, NULL, far, 4, far, 3, 4, 4, COMP_AMS_F32, NULL, 0, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_linear_q8(NULL, NULL, NULL, bytes8, buf, NULL, 0, 4, 3, 3, 4, 4, COMP_AMS_F32, NULL, 0, NULL), COMP_AMS_OK);
    EXPECT(comp_ams_linear_q8_work_bytes(2147483647, 131071, 2147483647, 0, 0, &bytes), COMP_AMS_EINVAL);
    EXPECT(comp_ams_linear_q8_work_bytes(0, 0, 0, 0, 0, &bytes), COMP_AMS_OK);
    EXPECT(comp_ams_linear_q8_work_bytes(100, 131071, 100, 0, 1, &bytes), COMP_AMS_OK);
    EXPECT(comp_ams_linear_weight_grad(buf, buf, buf, bytes8, buf, 4, 4, 3, far, 4, 2, 16, 0, 0, COMP_AMS_F32, COMP_AMS_F32, buf, 256, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_linear_weight_grad(buf, buf, buf, bytes8, buf, 4, far, far, 4, 4, 2, 16, 0, 0, COMP_AMS_F32, COMP_AMS_F32, buf, 256, NULL), COMP_AMS_EINVAL);
    EXPECT(comp_ams_linear_weight_grad_work_bytes(0, 0, 0, 1, 0, COMP_AMS_F32, 1, &bytes), COMP_AMS_OK);
    EXPECT(comp_ams_linear_weight_grad_work_bytes((int64_t)1 << 40, 1 << 20, 1 << 19, 65535, 0, COMP_AMS_F32, 0, &bytes), COMP_AMS_EINVAL);
    EXPECT(comp_ams_linear_weight_grad_work_bytes(65535, 1 << 23, 1 << 23, 65535, 0, COMP_AMS_F32, 0, &bytes), COMP_AMS_EINVAL);
    EXPECT(comp_ams_linear_weight_grad_work_bytes((1 << 29) - 1, 1 << 23, 1 << 23, 1, 0, COMP_AMS_F32, 0, &bytes), COMP_AMS_OK);
    EXPECT(comp_ams_operators_last_error()[0] ? 0 : 1, 0);

    printf("rows8 validation: %d failures\n", failures);
    return failures != 0;
}
