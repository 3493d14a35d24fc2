/* A C99 consumer of the head's and the adapters' part of the public header:
 * reports the layout of its structs and makes only calls that fail before
 * touching a device. */
#include <stddef.h>
#include <stdio.h>

#include "esopt.h"

#define F(T, f) printf(" " #f " %zu", offsetof(T, f))

int main(void) {
    printf("es_head_score_t %zu", sizeof(es_head_score_t));
    F(es_head_score_t, x); F(es_head_score_t, weight); F(es_head_score_t, x_stride);
    F(es_head_score_t, w_stride); F(es_head_score_t, ids); F(es_head_score_t, teacher);
    F(es_head_score_t, loss); F(es_head_score_t, logp); F(es_head_score_t, lse);
    F(es_head_score_t, status); F(es_head_score_t, workspace); F(es_head_score_t, workspace_bytes);
    F(es_head_score_t, rows); F(es_head_score_t, vocab); F(es_head_score_t, hidden);
    F(es_head_score_t, entries); F(es_head_score_t, scale); F(es_head_score_t, reserved);
    printf("\nes_head_gradient_t %zu", sizeof(es_head_gradient_t));
    F(es_head_gradient_t, x); F(es_head_gradient_t, weight); F(es_head_gradient_t, x_stride);
    F(es_head_gradient_t, w_stride); F(es_head_gradient_t, ids); F(es_head_gradient_t, teacher);
    F(es_head_gradient_t, logp); F(es_head_gradient_t, lse); F(es_head_gradient_t, grad);
    F(es_head_gradient_t, d_x); F(es_head_gradient_t, d_weight); F(es_head_gradient_t, dx_stride);
    F(es_head_gradient_t, dw_stride); F(es_head_gradient_t, status); F(es_head_gradient_t, workspace);
    F(es_head_gradient_t, workspace_bytes); F(es_head_gradient_t, rows); F(es_head_gradient_t, vocab);
    F(es_head_gradient_t, hidden); F(es_head_gradient_t, entries); F(es_head_gradient_t, scale);
    F(es_head_gradient_t, reserved);
    printf("\nes_adapt_t %zu", sizeof(es_adapt_t));
    F(es_adapt_t, x); F(es_adapt_t, weight); F(es_adapt_t, out); F(es_adapt_t, x_stride);
    F(es_adapt_t, w_stride); F(es_adapt_t, out_stride); F(es_adapt_t, a); F(es_adapt_t, b);
    F(es_adapt_t, scales); F(es_adapt_t, index); F(es_adapt_t, status); F(es_adapt_t, workspace);
    F(es_adapt_t, workspace_bytes); F(es_adapt_t, rows); F(es_adapt_t, inner); F(es_adapt_t, outer);
    F(es_adapt_t, members); F(es_adapt_t, rank); F(es_adapt_t, reserved);
    printf("\nvalues %u %u\n", ES_HEAD_BAD_ID, ES_ADAPT_BAD_INDEX);
    printf("score_null %d\n", es_head_score(NULL, NULL));
    printf("gradient_null %d\n", es_head_gradient(NULL, NULL));
    printf("adapt_null %d\n", es_adapt_project(NULL, NULL));
    printf("bytes_null %d\n", (int)(es_head_score_bytes(NULL) + es_head_gradient_bytes(NULL) +
                                    es_adapt_bytes(NULL)));
    return 0;
}
