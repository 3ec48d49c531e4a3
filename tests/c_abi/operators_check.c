/*
 * The structs of the serving operators as a C11 caller sees them, one "key value" pair per line; and the answers of the
 * host-only calls.  Needs no GPU.
 */
#include <stddef.h>
#include <stdio.h>
#include <string.h>

#include "amoeba.h"

#define SIZE(T) printf("sizeof." #T " %zu\n", sizeof(T))
#define OFF(T, f) printf("offsetof." #T "." #f " %zu\n", offsetof(T, f))

int main(void) {
    SIZE(amoeba_batch);
    OFF(amoeba_batch, d_block_table); OFF(amoeba_batch, d_seq_lens); OFF(amoeba_batch, d_q_starts);
    OFF(amoeba_batch, num_seqs); OFF(amoeba_batch, max_blocks_per_seq); OFF(amoeba_batch, num_rows);
    OFF(amoeba_batch, max_q_len);
    SIZE(amoeba_rotation);
    OFF(amoeba_rotation, d_q_norm); OFF(amoeba_rotation, d_k_norm); OFF(amoeba_rotation, d_inv_freq);
    OFF(amoeba_rotation, d_positions); OFF(amoeba_rotation, norm_eps); OFF(amoeba_rotation, rot_dim);
    OFF(amoeba_rotation, interleaved); OFF(amoeba_rotation, reserved);
    amoeba_layout l;
    memset(&l, 0, sizeof l);
    l.model.num_layers = 2; l.model.hidden = 512; l.model.num_q_heads = 16; l.model.num_kv_heads = 8;
    l.model.head_dim = 128; l.model.intermediate = 1792; l.model.elem_bytes = 2;
    l.tp = 2; l.block_tokens = 16; l.num_blocks = 10;
    amoeba_batch b;
    memset(&b, 0, sizeof b);
    b.num_seqs = 3; b.max_blocks_per_seq = 4; b.num_rows = 3; b.max_q_len = 1;
    int64_t n = 0;
    printf("attend_ws %d\n", (int)amoeba_attend_workspace_bytes(&l, &b, &n));
    printf("attend_ws_bytes %lld\n", (long long)n);
    printf("evict_ws %d\n", (int)amoeba_evict_workspace_bytes(&l, 2, 3, 100, &n));
    printf("evict_ws_bytes %lld\n", (long long)n);
    printf("evict_ws_budget %d\n", (int)amoeba_evict_workspace_bytes(&l, 2, 3, 0, &n));
    return 0;
}
