/* A C99 consumer of the cache's part of the public header: reports the layout
 * of its structs and makes only calls that fail before touching a device. */
#include <stddef.h>
#include <stdio.h>

#include "esopt.h"

#define F(T, f) printf(" " #f " %zu", offsetof(T, f))

int main(void) {
    printf("es_kv_desc_t %zu", sizeof(es_kv_desc_t));
    F(es_kv_desc_t, k_pages); F(es_kv_desc_t, v_pages); F(es_kv_desc_t, k_scales);
    F(es_kv_desc_t, v_scales); F(es_kv_desc_t, n_pages); F(es_kv_desc_t, page);
    F(es_kv_desc_t, kv_heads); F(es_kv_desc_t, head_dim); F(es_kv_desc_t, format);
    F(es_kv_desc_t, reserved);
    printf("\nes_kv_append_t %zu", sizeof(es_kv_append_t));
    F(es_kv_append_t, q); F(es_kv_append_t, k); F(es_kv_append_t, v); F(es_kv_append_t, q_out);
    F(es_kv_append_t, q_stride); F(es_kv_append_t, k_stride); F(es_kv_append_t, v_stride);
    F(es_kv_append_t, q_out_stride); F(es_kv_append_t, q_gain); F(es_kv_append_t, k_gain);
    F(es_kv_append_t, rope); F(es_kv_append_t, positions); F(es_kv_append_t, slots);
    F(es_kv_append_t, status); F(es_kv_append_t, tokens); F(es_kv_append_t, q_heads);
    F(es_kv_append_t, rot); F(es_kv_append_t, rope_rows); F(es_kv_append_t, eps);
    F(es_kv_append_t, flags);
    printf("\nes_kv_attend_t %zu", sizeof(es_kv_attend_t));
    F(es_kv_attend_t, q); F(es_kv_attend_t, out); F(es_kv_attend_t, q_stride);
    F(es_kv_attend_t, out_stride); F(es_kv_attend_t, tables); F(es_kv_attend_t, lengths);
    F(es_kv_attend_t, starts); F(es_kv_attend_t, first); F(es_kv_attend_t, limit);
    F(es_kv_attend_t, slopes); F(es_kv_attend_t, status); F(es_kv_attend_t, rows);
    F(es_kv_attend_t, n_seqs); F(es_kv_attend_t, table_stride); F(es_kv_attend_t, q_heads);
    F(es_kv_attend_t, max_rows); F(es_kv_attend_t, max_length); F(es_kv_attend_t, scale);
    F(es_kv_attend_t, cap);
    printf("\nvalues %u %u %u %u %u %u %u %u\n", ES_KV_INT8, ES_KV_E4M3, ES_KV_BF16, ES_KV_ADJACENT,
           ES_KV_BAD_SLOT, ES_KV_BAD_POSITION, ES_KV_BAD_PAGE, ES_KV_BAD_LENGTH);
    es_kv_t* kv = NULL;
    printf("create_null %d\n", es_kv_create(NULL, &kv));
    printf("attend_null %d\n", es_kv_attend(NULL, NULL, NULL));
    printf("destroy_null %d\n", es_kv_destroy(NULL));
    return 0;
}
