/*
 * The structs of the calls for sequences that share blocks as a C11 caller sees them, one "key value" pair per line; and the answers of
 * the host-only call.  Needs no GPU.
 */
#include <stddef.h>
#include <stdio.h>
#include <string.h>

#include "amoeba.h"

#define SIZE(T) printf("sizeof." #T " %zu\n", sizeof(T))
#define OFF(T, f) printf("offsetof." #T "." #f " %zu\n", offsetof(T, f))

int main(void) {
    SIZE(amoeba_prefixes);
    OFF(amoeba_prefixes, d_group_starts); OFF(amoeba_prefixes, d_prefix_lens); OFF(amoeba_prefixes, num_groups);
    OFF(amoeba_prefixes, max_group_rows); OFF(amoeba_prefixes, always); OFF(amoeba_prefixes, reserved);
    SIZE(amoeba_table_step);
    OFF(amoeba_table_step, d_block_table); OFF(amoeba_table_step, d_block_refs); OFF(amoeba_table_step, d_seq_lens);
    OFF(amoeba_table_step, d_new_lens); OFF(amoeba_table_step, d_parents); OFF(amoeba_table_step, d_shared_lens);
    OFF(amoeba_table_step, d_lens_out); OFF(amoeba_table_step, d_q_starts); OFF(amoeba_table_step, d_first_positions);
    OFF(amoeba_table_step, d_positions); OFF(amoeba_table_step, d_slots); OFF(amoeba_table_step, d_pairs);
    OFF(amoeba_table_step, d_num_pairs); OFF(amoeba_table_step, d_free_count); OFF(amoeba_table_step, num_seqs);
    OFF(amoeba_table_step, max_blocks_per_seq); OFF(amoeba_table_step, num_rows); OFF(amoeba_table_step, pairs_cap);
    amoeba_layout l;
    memset(&l, 0, sizeof l);
    l.model.num_layers = 2; l.model.hidden = 512; l.model.num_q_heads = 16; l.model.num_kv_heads = 8;
    l.model.head_dim = 128; l.model.intermediate = 1792; l.model.elem_bytes = 2;
    l.tp = 2; l.block_tokens = 16; l.num_blocks = 10;
    amoeba_batch b;
    memset(&b, 0, sizeof b);
    b.num_seqs = 3; b.max_blocks_per_seq = 4; b.num_rows = 3; b.max_q_len = 1;
    amoeba_prefixes x;
    memset(&x, 0, sizeof x);
    x.num_groups = 2; x.max_group_rows = 2;
    int64_t n = 0;
    printf("ws %d\n", (int)amoeba_attend_shared_workspace_bytes(&l, &b, &x, &n));
    printf("ws_bytes %lld\n", (long long)n);
    x.num_groups = -1;
    printf("ws_groups %d\n", (int)amoeba_attend_shared_workspace_bytes(&l, &b, &x, &n));
    return 0;
}
