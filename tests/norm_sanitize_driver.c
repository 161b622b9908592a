/* Host path of layer norm and dropout under the sanitizers: validation and workspace sizing over extreme sizes. Nothing is launched. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "../include/dlconv.h"

int main(void)
{
    int bad = 0, n = 0;
    static const int64_t rows[] = {0, 1, 2, 63, 64, 65, 4099, 6912, 110592, 1769472, (int64_t)1 << 25, ((int64_t)1 << 46) / 1048576 - 1};
    static const int32_t chans[] = {1, 2, 7, 8, 9, 48, 77, 256, 304, 1024, 2048, 2056, 8192, 16384, 16392, 1048576};
    for (unsigned i = 0; i < sizeof rows / sizeof *rows; ++i)
        for (unsigned j = 0; j < sizeof chans / sizeof *chans; ++j) {
            size_t bytes = 0;
            const dl_status s = dl_layer_norm_bwd_workspace_bytes(rows[i], chans[j], &bytes);
            const int fits = rows[i] < ((int64_t)1 << 46) / chans[j];
            bad += s != (fits ? DL_OK : DL_ERR_SHAPE) || (fits && bytes < 8u * (size_t)chans[j]);
            ++n;
        }
    size_t bytes;
    bad += dl_layer_norm_bwd_workspace_bytes(INT64_MAX, 2, &bytes) != DL_ERR_SHAPE;
    bad += dl_layer_norm_bwd_workspace_bytes(INT64_MIN, 2, &bytes) != DL_ERR_SHAPE;
    bad += dl_layer_norm_bwd_workspace_bytes(1, INT32_MIN, &bytes) != DL_ERR_SHAPE;
    bad += dl_layer_norm_bwd_workspace_bytes(1, INT32_MAX, &bytes) != DL_ERR_SHAPE;
    void *p16 = (void *)16, *p32 = (void *)32;
    float *f = (float *)16;
    dl_dropout d = {0.1f, UINT64_MAX, UINT64_MAX, NULL};
    bad += dropout_fwd(p16, NULL, &d, DL_F16, INT64_MAX, p16, NULL) != DL_ERR_SHAPE;
    bad += dropout_bwd(p16, &d, DL_F32, INT64_MIN, p16, NULL) != DL_ERR_SHAPE;
    bad += layer_norm_fwd(p16, f, f, DL_BF16, INT64_MAX, INT32_MAX, 1e-5f, p16, f, f, NULL) != DL_ERR_SHAPE;
    bad += layer_norm_bwd(p16, p16, f, f, f, DL_F16, 4, 8, p16, f, f, NULL, 0, NULL) != DL_ERR_WORKSPACE;
    d.p = nanf("");
    bad += dropout_add_layer_norm_fwd(p16, p16, &d, f, f, DL_F16, 4, 8, 0.f, p16, p32, f, f, NULL) != DL_ERR_VALUE;
    d.p = INFINITY;
    bad += dropout_add_layer_norm_bwd(p16, p16, p16, &d, f, f, f, DL_F16, 4, 8, p16, p32, f, f, p16, 1 << 20, NULL) != DL_ERR_VALUE;
    d.p = 1.f;
    bad += dropout_fwd(NULL, NULL, &d, DL_F16, 0, NULL, NULL) != DL_OK;
    printf("norm host path: %d sizes, %d wrong status codes\n", n, bad);
    return bad != 0;
}
