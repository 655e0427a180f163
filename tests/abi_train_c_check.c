/* Test helper (not part of the product): a plain C99 program that includes cser_train.h, takes the address of every entry
 * point and makes calls that need no GPU.  Built and run by tests/test_train_abi.py. */
#include <stdio.h>
#include <string.h>
#include "cser_train.h"

int main(void) {
    typedef void (*fn_t)(void);
    const fn_t fns[] = {
        (fn_t)cser_orth_create, (fn_t)cser_orth_apply, (fn_t)cser_orth_destroy, (fn_t)cser_orth_debug_stall_next,
        (fn_t)cser_orth_launch_count, (fn_t)cser_xent_create, (fn_t)cser_xent_loss, (fn_t)cser_xent_grad,
        (fn_t)cser_xent_destroy, (fn_t)cser_xent_launch_count,
    };
    const int64_t zero = 0, four = 4, five = 5;
    cser_xent_inputs in;
    size_t i;
    for (i = 0; i < sizeof(fns) / sizeof(fns[0]); ++i)
        if (!fns[i]) return 1;
    memset(&in, 0, sizeof(in));
    /* invalid arguments are rejected before any CUDA call */
    if (cser_orth_create(1, 19, 1, &zero, &four, &five, NULL, NULL, 5, CSER_TYPE_F32, CSER_TYPE_F32) != NULL) return 2;
    if (strstr(cser_last_error(), "outside the vector") == NULL) return 3;
    if (cser_orth_create(1, 20, 1, &zero, &four, &five, &four, NULL, 5, CSER_TYPE_F32, CSER_TYPE_F32) != NULL) return 4;
    if (cser_orth_create(1, 20, 1, &zero, &four, &five, NULL, NULL, 5, CSER_TYPE_F32, 3) != NULL) return 5;
    if (cser_orth_apply(NULL, NULL, NULL, 0.0f, NULL, NULL) != CSER_ERR_INVALID) return 6;
    if (cser_xent_create(1, 8, 30, 16, CSER_TYPE_F32, 0) != NULL) return 7;
    if (strstr(cser_last_error(), "type") == NULL) return 8;
    if (cser_xent_loss(NULL, &in, NULL, NULL, NULL) != CSER_ERR_INVALID) return 9;
    if (cser_xent_grad(NULL, &in, NULL, NULL, NULL, NULL, 0, NULL) != CSER_ERR_INVALID) return 10;
    if (cser_orth_launch_count(NULL) != 0 || cser_xent_launch_count(NULL) != 0) return 11;
    cser_orth_destroy(NULL);
    cser_xent_destroy(NULL);
    printf("c abi ok: %u entry points\n", (unsigned)(sizeof(fns) / sizeof(fns[0])));
    return 0;
}
