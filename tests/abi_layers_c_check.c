/* Test helper (not part of the product): a plain C99 program that includes cser_layers.h, takes the address of every entry
 * point and makes calls that need no GPU.  Built and run by tests/test_layers_abi.py. */
#include <stdio.h>
#include <string.h>
#include "cser_layers.h"

int main(void) {
    typedef void (*fn_t)(void);
    const fn_t fns[] = {
        (fn_t)cser_drop_create, (fn_t)cser_drop_apply, (fn_t)cser_drop_grad, (fn_t)cser_drop_destroy, (fn_t)cser_drop_launch_count,
        (fn_t)cser_norm_create, (fn_t)cser_norm_apply, (fn_t)cser_norm_grad, (fn_t)cser_norm_destroy, (fn_t)cser_norm_launch_count,
    };
    cser_rows rows;
    cser_pixels pixels;
    cser_norm_inputs in;
    size_t i;
    for (i = 0; i < sizeof(fns) / sizeof(fns[0]); ++i)
        if (!fns[i]) return 1;
    memset(&rows, 0, sizeof(rows));
    memset(&pixels, 0, sizeof(pixels));
    memset(&in, 0, sizeof(in));
    /* invalid arguments are rejected before any CUDA call */
    if (cser_drop_create(1, 1, 1, 1.0, 0, 1, 0, CSER_TYPE_BF16) != NULL) return 2;
    if (strstr(cser_last_error(), "p must be") == NULL) return 3;
    if (cser_drop_create(1, 1, 1, 0.5, 0, 0, 0, CSER_TYPE_BF16) != NULL) return 4;
    if (cser_drop_create(1, 1, 1, 0.5, 0, 1, 0, 3) != NULL) return 5;
    if (cser_drop_apply(NULL, 1, 0, NULL, &rows, NULL, 0, NULL, &rows, NULL) != CSER_ERR_INVALID) return 6;
    if (cser_drop_grad(NULL, 1, 0, NULL, &rows, &rows, NULL, 0, NULL) != CSER_ERR_INVALID) return 7;
    if (cser_norm_create(1, 1, 8, 3, CSER_ACT_RELU, 1e-5f, CSER_TYPE_F16, NULL) != NULL) return 8;
    if (strstr(cser_last_error(), "multiple of groups") == NULL) return 9;
    if (cser_norm_create(1, 1, 8, 2, 3, 1e-5f, CSER_TYPE_F16, NULL) != NULL) return 10;
    if (cser_norm_apply(NULL, &in, &pixels, NULL, NULL) != CSER_ERR_INVALID) return 11;
    if (cser_norm_grad(NULL, &in, NULL, &pixels, &pixels, NULL, 0, NULL, 0, NULL) != CSER_ERR_INVALID) return 12;
    if (cser_drop_launch_count(NULL) != 0 || cser_norm_launch_count(NULL) != 0) return 13;
    cser_drop_destroy(NULL);
    cser_norm_destroy(NULL);
    printf("c abi ok: %u entry points\n", (unsigned)(sizeof(fns) / sizeof(fns[0])));
    return 0;
}
