// Attention of few query rows a sequence over quantised pools.
#pragma once
#include "laps_internal.h"

// Of the attention over 4-bit and 8-bit pools.
constexpr int LAPS_KVQ_MAX_PAGES = 1 << 26;       // of a page table's row: positions stay below 2^30
constexpr long LAPS_KVQ_MAX_SEQ_HEADS = 1 << 20;   // sequences times query heads: its grid

struct RowsAttn {
    const bf16_t* q;
    bf16_t* out;
    const unsigned char *k_pool, *v_pool;
    const int *cu, *seq_len, *prefix_len, *page_table;   // seq_len may be NULL
    int n_seq, n_tokens, max_pages, n_pool_pages, n_q, n_kv, hd;
    int bits;   // of a value of the pools, 4 or 8
};
struct RowsPlan {
    int row_tiles;    // 16-row tiles of a block
    int row_blocks;   // blocks of rows that workgroups of their own walk, a sequence and kv head
    int more_rows;    // as many times that, the last ones first in the launch
    int parts;        // most parts of a sequence's keys
    int min_parts;    // as many at least, where there are keys for them
};
// Which of the two kernels a launch shape takes: this one, or the blocks of 128 or 256 rows of the bf16 pools' attention.
bool laps_attn_takes_rows(int n_seq, int n_tokens, int n_q, int n_kv);
RowsPlan laps_attn_rows_plan(int bits, int n_seq, int n_tokens, int n_q, int n_kv, int max_pages);
size_t laps_attn_rows_bytes(const RowsPlan& p, int n_tokens, int n_q, int hd);   // partial results of the parts
int laps_launch_attn_rows(const RowsAttn& a, const RowsPlan& p, float* partial, hipStream_t s);
