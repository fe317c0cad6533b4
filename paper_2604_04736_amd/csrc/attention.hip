// libhot: attention with a learned relative position bias by buckets, forward and backward (the kernels are in attention.h).
//
// Forward: the table is spread over differences of codes (one small launch), then one launch over tiles of queries, which joins a second one where there are too
// few tiles to fill the compute units and the keys are split.  Backward: D of every query, dk and dv from tiles of keys, dq and the table's sums
// from tiles of queries, both of which form z again (seven products where five would do if one kernel added to another's results, whose order would
// then be left to chance), and the table's gradient from the workgroups' sums.
#include <hip/hip_runtime.h>

#include "hot.h"
#include "vec.h"
#include "element.h"
#include "attention_args.h"

namespace {

using hot_detail::AttentionArgs;

bool aligned8(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

constexpr long kMostRows = 0x7FFFFFFFL;

bool attention_ok(const hot_attention_desc *d)
{
    if (!d || d->queries < 0 || d->keys < 0 || d->batch < 0 || d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads || d->width < HOT_ATTENTION_LEAST_WIDTH ||
        d->width > HOT_ATTENTION_MOST_WIDTH || d->groups < 0 || !known_type(d->dtype) || !(d->scale >= -1.0e30 && d->scale <= 1.0e30))
        return false;
    // (65535: the last dimension of a grid)
    if (d->tables < 0 || d->tables > 65535 || d->heads > 65535) return false;
    if (d->queries >= kMostRows || d->keys >= kMostRows) return false;
    const double entries = (double)d->batch * (double)d->heads;
    if (entries * (double)d->queries >= (double)kMostRows || entries * (double)d->keys >= (double)kMostRows || entries >= (double)kMostRows) return false;
    if (d->tables) {
        if (d->batch % d->tables || d->buckets < 1 || d->buckets > HOT_ATTENTION_MOST_BUCKETS || d->codes < 1 || d->codes > HOT_ATTENTION_MOST_CODES ||
            d->first_query < 0 || (d->table_dtype != d->dtype && d->table_dtype != HOT_F32) || (double)d->tables * d->heads * (double)d->codes >= 1.0e12)
            return false;
    }
    for (const hot_pitch *p : {&d->q, &d->k, &d->v, &d->o, &d->grad_o, &d->grad_q, &d->grad_k, &d->grad_v})
        if (p->batch < 0 || p->head < 0 || p->row < 0) return false;
    return true;
}

// How the forward call cuts its work: shape 0 a wave with sixteen rows and 32 keys at a time, 1 and 2 four waves with sixteen or 32 rows each and 64 keys
struct Cut {
    int pack, shape, splits, tiles;
    long items;
};

Cut forward_cut(const hot_attention_desc &d)
{
    Cut c;
    const int per = d.heads / d.kv_heads;
    // heads of one key head side by side in a tile where one head's queries do not fill it: its keys are then read once for all
    c.pack = d.queries * per <= 64 ? per : 1;
    const long rows = d.queries * c.pack;
    c.shape = rows <= 16 ? 0 : (rows <= 64 ? 1 : 2);
    const int tile = c.shape == 0 ? 16 : (c.shape == 1 ? 64 : 128), keys = c.shape == 0 ? 32 : 64;
    c.tiles = (int)((rows + tile - 1) / tile);
    c.items = (long)d.batch * (d.heads / c.pack) * c.tiles;
    // workgroups for every place there is, but at least four tiles of keys to each
    const long places = c.shape == 0 ? 2048 : 512, tiles_k = (d.keys + keys - 1) / keys;
    long splits = c.items ? places / c.items : 1;
    if (splits > tiles_k / 4) splits = tiles_k / 4;
    if (splits > 128) splits = 128;
    c.splits = splits < 2 ? 1 : (int)splits;
    c.items *= c.splits;
    return c;
}

struct BackwardCut {
    int shape, tiles, chunk, splits, by_head;
    long items;
};

BackwardCut queries_cut(const hot_attention_desc &d)
{
    BackwardCut c = {};
    c.shape = d.queries <= 64 ? 1 : 2;
    const int tile = c.shape == 1 ? 64 : 128;
    c.tiles = (int)((d.queries + tile - 1) / tile);
    const long entries = d.tables ? d.batch / d.tables : d.batch, sets = d.tables ? d.tables : 1;
    // at most about 8192 rows of sums for the table
    const long all = (long)d.batch * d.heads * c.tiles;
    c.chunk = (int)(all / 8192 + 1);
    if (c.chunk > entries) c.chunk = entries < 1 ? 1 : (int)entries;
    c.items = sets * ((entries + c.chunk - 1) / c.chunk) * d.heads * c.tiles;
    long splits = c.items ? 512 / c.items : 1;
    const long most = (d.keys + 63) / 64 / 4;
    splits = splits < most ? splits : most;
    c.splits = splits < 2 ? 1 : (int)splits;
    c.items *= c.splits;
    return c;
}

BackwardCut keys_cut(const hot_attention_desc &d)
{
    BackwardCut c = {};
    const int tile = 64, per = d.heads / d.kv_heads;
    c.tiles = (int)((d.keys + tile - 1) / tile);
    c.items = (long)d.batch * d.kv_heads * c.tiles;
    // few workgroups, whose work is of unequal length where order counts: heads of a key head apart, then runs of queries
    const long want = c.items ? 1024 / c.items : 1, tiles_q = (d.queries + 63) / 64;
    c.splits = 1;
    if (want > 1) {
        c.by_head = per > 1;
        long runs = c.by_head ? want / per : want;
        runs = runs < tiles_q / 4 ? runs : tiles_q / 4;
        c.splits = (int)((runs < 1 ? 1 : runs) * (c.by_head ? per : 1));
    }
    c.items *= c.splits;
    return c;
}

long up16(long bytes) { return (bytes + 15) & ~15L; }

struct Room {
    long query_spans, key_spans, part_o, part_ml, d, bounds, parts, part_k, part_v, all;
};

Room room_of(const hot_attention_desc &d, bool backward)
{
    Room r = {};
    long at = 0;
    const auto take = [&](long bytes) {
        const long here = at;
        at += up16(bytes);
        return here;
    };
    const long rows = (long)d.batch * d.heads * d.queries;
    take(d.tables ? (long)d.tables * d.heads * d.codes * 4 : 0);
    r.query_spans = take((long)d.groups * ((d.queries + 63) / 64) * 8);
    r.key_spans = take((long)d.groups * ((d.keys + 63) / 64) * 8);
    if (!backward) {
        const long splits = forward_cut(d).splits;
        r.part_o = take(splits > 1 ? splits * rows * d.width * 4 : 0);
        r.part_ml = take(splits > 1 ? splits * rows * 8 : 0);
    } else {
        const BackwardCut q = queries_cut(d), k = keys_cut(d);
        r.d = take(rows * 4);
        r.bounds = take((long)d.batch * (d.heads + d.kv_heads) * 4);
        r.parts = take(d.tables ? q.items * d.buckets * 4 : 0);
        r.part_o = take(q.splits > 1 ? q.splits * rows * d.width * 4 : 0);
        const long part = k.splits > 1 ? (long)k.splits * d.batch * d.kv_heads * d.keys * d.width * 4 : 0;
        r.part_k = take(part);
        r.part_v = take(part);
    }
    r.all = at;
    return r;
}

AttentionArgs args_of(const hot_attention_desc &d)
{
    AttentionArgs a = {};
    a.queries = (int)d.queries;
    a.keys = (int)d.keys;
    a.batch = d.batch;
    a.heads = d.heads;
    a.kv_heads = d.kv_heads;
    a.per = d.heads / d.kv_heads;
    a.width = d.width;
    a.tables = d.tables;
    a.entries = d.tables ? d.batch / d.tables : d.batch;
    a.buckets = d.buckets;
    a.codes = d.codes;
    a.groups = d.groups;
    a.causal = d.causal != 0;
    a.first_query = d.first_query;
    a.table_type = d.table_dtype;
    a.pack = a.splits = a.chunk = 1;
    a.all_rows = (long)d.batch * d.heads * d.queries;
    a.scale = (float)(d.scale * 1.4426950408889634);
    a.plain_scale = (float)d.scale;
    a.p_q = d.q;
    a.p_k = d.k;
    a.p_v = d.v;
    a.p_o = d.o;
    a.p_go = d.grad_o;
    a.p_gq = d.grad_q;
    a.p_gk = d.grad_k;
    a.p_gv = d.grad_v;
    return a;
}

// The arrays that both calls read; false if one is missing or off its grid
bool give(AttentionArgs &a, const hot_attention_desc &d, const Room &r, char *ws, const void *q, const void *k, const void *v, const void *table, const int32_t *query_code,
          const int32_t *key_code, const int32_t *query_range, const int32_t *key_range, const int32_t *bucket, const int32_t *query_groups, const int32_t *key_groups)
{
    if (a.all_rows && (!q || !on_element(q, d.dtype))) return false;
    if (d.keys && d.batch && (!k || !v || !on_element(k, d.dtype) || !on_element(v, d.dtype))) return false;
    if (d.tables && (!table || !query_code || !key_code || !query_range || !key_range || !bucket || !on_element(table, d.table_dtype) || !aligned4(query_code) ||
                     !aligned4(key_code) || !aligned8(query_range) || !aligned8(key_range) || !aligned8(bucket)))
        return false;
    if (d.groups && (!query_groups || !key_groups || !aligned4(query_groups) || !aligned4(key_groups))) return false;
    a.q = q;
    a.k = k;
    a.v = v;
    a.table = table;
    a.query_code = query_code ? query_code + d.first_query : nullptr;
    a.key_code = key_code;
    a.query_range = reinterpret_cast<const int2 *>(query_range);
    a.key_range = reinterpret_cast<const int2 *>(key_range);
    a.bucket = reinterpret_cast<const int2 *>(bucket);
    a.query_groups = query_groups;
    a.key_groups = key_groups;
    a.bias = reinterpret_cast<float *>(ws);
    a.query_spans = reinterpret_cast<int2 *>(ws + r.query_spans);
    a.key_spans = reinterpret_cast<int2 *>(ws + r.key_spans);
    a.part_o = reinterpret_cast<float *>(ws + r.part_o);
    return true;
}

#define HOT_BY_TYPE(CALL, a)                                               \
    do {                                                                   \
        if (desc->dtype == HOT_F32) hot_detail::CALL<float>(a, s);         \
        else if (desc->dtype == HOT_BF16) hot_detail::CALL<__bf16>(a, s);  \
        else hot_detail::CALL<_Float16>(a, s);                             \
    } while (0)

}  // namespace

extern "C" {

int64_t hot_attention_workspace_bytes(const hot_attention_desc *desc, int which)
{
    if (!attention_ok(desc) || which < 0 || which > 1) return HOT_EINVAL;
    const long n = room_of(*desc, which == 1).all;
    return n < 16 ? 16 : n;
}

int hot_attention_forward(const hot_attention_desc *desc, const void *q, const void *k, const void *v, const void *table, const int32_t *query_code,
                          const int32_t *key_code, const int32_t *query_range, const int32_t *key_range, const int32_t *bucket, const int32_t *query_groups, const int32_t *key_groups, void *o,
                          void *rest, float *stats, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (!attention_ok(desc)) return HOT_EINVAL;
    AttentionArgs a = args_of(*desc);
    char *const ws = static_cast<char *>(workspace);
    const Room r = room_of(*desc, false);
    if (!give(a, *desc, r, ws, q, k, v, table, query_code, key_code, query_range, key_range, bucket, query_groups, key_groups)) return HOT_EINVAL;
    if (a.all_rows == 0) return HOT_OK;
    if (!o || !on_element(o, desc->dtype) || !on_element(rest, desc->dtype) || (rest && desc->dtype == HOT_F32) || !aligned4(stats) ||
        (r.all && (!workspace || !aligned16(workspace) || workspace_bytes < r.all)))
        return HOT_EINVAL;
    const Cut c = forward_cut(*desc);
    a.pack = c.pack;
    a.shape = c.shape;
    a.splits = c.splits;
    a.tiles_q = c.tiles;
    a.items = c.items;
    a.o = o;
    a.rest = rest;
    a.stats = stats;
    a.part_ml = reinterpret_cast<float *>(ws + r.part_ml);
    hipStream_t s = static_cast<hipStream_t>(stream);
    HOT_BY_TYPE(attention_begin, a);
    HOT_BY_TYPE(attention_forward, a);
    return hot_detail::note_hip(hipGetLastError());
}

int hot_attention_backward(const hot_attention_desc *desc, const void *q, const void *k, const void *v, const void *table, const int32_t *query_code,
                           const int32_t *key_code, const int32_t *query_range, const int32_t *key_range, const int32_t *bucket, const int32_t *query_groups, const int32_t *key_groups, const void *o,
                           const void *rest, const float *stats, const void *grad_o, void *grad_q, void *grad_k, void *grad_v, void *grad_table, void *workspace,
                           int64_t workspace_bytes, void *stream)
{
    if (!attention_ok(desc)) return HOT_EINVAL;
    AttentionArgs a = args_of(*desc);
    char *const ws = static_cast<char *>(workspace);
    const Room r = room_of(*desc, true);
    if (!give(a, *desc, r, ws, q, k, v, table, query_code, key_code, query_range, key_range, bucket, query_groups, key_groups)) return HOT_EINVAL;
    const int t = desc->dtype;
    if (!on_element(grad_q, t) || !on_element(grad_k, t) || !on_element(grad_v, t) || !on_element(grad_table, desc->table_dtype) || (grad_table && !desc->tables) ||
        (r.all && (!workspace || !aligned16(workspace) || workspace_bytes < r.all)))
        return HOT_EINVAL;
    if (a.all_rows && (!o || !stats || !grad_o || !on_element(o, t) || !on_element(rest, t) || (rest && t == HOT_F32) || !aligned4(stats) || !on_element(grad_o, t)))
        return HOT_EINVAL;
    a.o = const_cast<void *>(o);
    a.rest = const_cast<void *>(rest);
    a.stats = const_cast<float *>(stats);
    a.grad_o = grad_o;
    a.grad_q = grad_q;
    a.grad_k = grad_k;
    a.grad_v = grad_v;
    a.grad_table = grad_table;
    a.d = reinterpret_cast<float *>(ws + r.d);
    a.bounds = reinterpret_cast<unsigned *>(ws + r.bounds);
    a.parts = reinterpret_cast<float *>(ws + r.parts);
    a.part_k = reinterpret_cast<float *>(ws + r.part_k);
    a.part_v = reinterpret_cast<float *>(ws + r.part_v);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (a.all_rows) {
        a.bounds_count = t == HOT_F16 ? (long)desc->batch * (desc->heads + desc->kv_heads) : 0;
        HOT_BY_TYPE(attention_begin, a);
        HOT_BY_TYPE(attention_prepare, a);
    }
    if ((grad_k || grad_v) && desc->keys && desc->batch) {
        const BackwardCut c = keys_cut(*desc);
        a.tiles_k = c.tiles;
        a.splits = c.splits;
        a.by_head = c.by_head;
        a.items = c.items;
        HOT_BY_TYPE(attention_keys, a);
    }
    if ((grad_q && a.all_rows) || grad_table) {
        const BackwardCut c = queries_cut(*desc);
        a.shape = c.shape;
        a.tiles_q = c.tiles;
        a.chunk = c.chunk;
        a.splits = c.splits;
        a.items = c.items;
        HOT_BY_TYPE(attention_queries, a);
    }
    return hot_detail::note_hip(hipGetLastError());
}

}  // extern "C"
