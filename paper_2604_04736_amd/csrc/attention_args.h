// What attention.hip hands to the kernels of attention.h, one source file for each type of elements.
#ifndef HOT_ATTENTION_ARGS_H
#define HOT_ATTENTION_ARGS_H

#include <hip/hip_runtime.h>

#include "hot.h"

namespace hot_detail {

struct AttentionArgs {
    int queries, keys, batch, heads, kv_heads, per, width;         // per: query heads to a key head
    int tables, entries, buckets, codes, groups, causal, table_type; // entries: of the batch, to a table
    int pack;                          // heads side by side in a tile's rows (forward)
    int shape, splits, tiles_q;
    int chunk;                         // entries that a workgroup takes one after the other (dq)
    int by_head;                       // splits are of the heads that read a key head (times runs of their queries), not of queries alone (dk and dv)
    int first_query;
    long items, all_rows, bounds_count;                            // all_rows: batch x heads x queries
    float scale, plain_scale;          // times log2 e, and as it is
    hot_pitch p_q, p_k, p_v, p_o, p_go, p_gq, p_gk, p_gv;
    const void *q, *k, *v, *table, *grad_o;
    const int32_t *query_code, *key_code, *query_groups, *key_groups;
    const int4 *query_range, *key_range;
    const int2 *bucket;
    void *o, *rest, *grad_q, *grad_k, *grad_v, *grad_table;
    float *stats;                      // [all_rows, 2]: the largest z in units of log 2, and log2 of the sum
    float *bias;                       // [tables, heads, codes], in units of log 2
    float *part_o, *part_ml;           // [splits, all_rows, width], [splits, all_rows, 2]
    float *part_k, *part_v;            // [splits, batch, kv_heads, keys, width]
    int4 *query_spans, *key_spans;     // [groups, 64s of queries or keys]
    float *d;                          // [all_rows]
    float *parts;                      // [items of dq, buckets]
    unsigned *bounds;                  // [batch, heads] and [batch, kv_heads]
};

template <class T> __attribute__((visibility("hidden"))) void attention_begin(const AttentionArgs &a, hipStream_t s);
template <class T> __attribute__((visibility("hidden"))) void attention_forward(const AttentionArgs &a, hipStream_t s);
template <class T> __attribute__((visibility("hidden"))) void attention_prepare(const AttentionArgs &a, hipStream_t s);
template <class T> __attribute__((visibility("hidden"))) void attention_keys(const AttentionArgs &a, hipStream_t s);
template <class T> __attribute__((visibility("hidden"))) void attention_queries(const AttentionArgs &a, hipStream_t s);

}  // namespace hot_detail

#endif  // HOT_ATTENTION_ARGS_H
