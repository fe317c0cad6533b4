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
#include "fragment.h"

namespace {

// Rows of `width` elements as rows of `wide`, a multiple of eight, with zeros behind; those of negative groups are zeros.  [batch, heads, tokens, wide]
template <class T>
__global__ void __launch_bounds__(256)
hot_attention_pack_kernel(const T *__restrict__ from, T *__restrict__ to, hot_pitch p, long rows, int heads, int tokens, int width, int wide, const int32_t *groups, int group_rows)
{
    const int pieces = wide / 8;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < rows * pieces; i += (long)gridDim.x * 256) {
        const long row = i / pieces;
        const int c = (int)(i % pieces), t = (int)(row % tokens), h = (int)(row / tokens % heads), b = (int)(row / tokens / heads);
        const bool there = !group_rows || groups[(long)(b % group_rows) * tokens + t] >= 0;
        *reinterpret_cast<V8<T> *>(to + row * wide + c * 8) = eight(from + b * p.batch + h * p.head + t * p.row, c * 8, width, there);
    }
}

void pack_rows(const void *from, void *to, const hot_pitch &p, int batch, int heads, int tokens, int width, int wide, int bytes, const int32_t *groups, int group_rows, hipStream_t s)
{
    const long rows = (long)batch * heads * tokens, blocks = (rows * (wide / 8) + 255) / 256;
    if (!rows) return;
    const unsigned n = (unsigned)(blocks < 8192 ? blocks : 8192);
    if (bytes == 2) hot_attention_pack_kernel<_Float16><<<n, 256, 0, s>>>(static_cast<const _Float16 *>(from), static_cast<_Float16 *>(to), p, rows, heads, tokens, width, wide, groups, group_rows);
    else hot_attention_pack_kernel<float><<<n, 256, 0, s>>>(static_cast<const float *>(from), static_cast<float *>(to), p, rows, heads, tokens, width, wide, groups, group_rows);
}

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
    if (d->queries > HOT_ATTENTION_MOST_TOKENS || d->keys > HOT_ATTENTION_MOST_TOKENS) return false;
    const double entries = (double)d->batch * (double)d->heads;
    if (entries * (double)d->queries >= (double)kMostRows || entries * (double)d->keys >= (double)kMostRows || entries >= (double)kMostRows) return false;
    if (d->tables) {
        if (d->batch % d->tables || d->buckets < 1 || d->buckets > HOT_ATTENTION_MOST_BUCKETS || d->codes < 1 || d->codes > HOT_ATTENTION_MOST_CODES ||
            d->first_query < 0 || d->first_query + d->queries > kMostRows || (d->table_dtype != d->dtype && d->table_dtype != HOT_F32) || (double)d->tables * d->heads * (double)d->codes >= 1.0e12)
            return false;
    }
    for (const hot_pitch *p : {&d->q, &d->k, &d->v, &d->o, &d->grad_o, &d->grad_q, &d->grad_k, &d->grad_v})
        if (p->batch < 0 || p->head < 0 || p->row < 0) return false;
    return true;
}

// How the forward call cuts its work: shape 0 a wave with sixteen rows and 32 keys at a time, 1 and 2 tiles of 64 and 128 rows and 64 keys
struct Cut {
    int pack, shape, splits, tiles;
    long items;
};

// Whether tiles of 128 rows leave some of the two places of 256 compute units empty.  Tiles of 64 are then better, though each of them reads all keys (two texts' rows of 3001 tokens x 8
// heads x 80 packed, 384 tiles: forward 74 -> 67 us, dq 124 -> 104; 768 entries and heads of 65 tokens, 768 tiles, the other way: dq 39 -> 47).
bool few(long sets, long rows) { return sets * ((rows + 127) / 128) < 512; }

Cut forward_cut(const hot_attention_desc &d)
{
    Cut c;
    const int per = d.heads / d.kv_heads;
    // heads of one key head side by side in a tile where one head's queries do not fill it: its keys are then read once for all
    c.pack = d.queries * per <= 64 ? per : 1;
    const long rows = d.queries * c.pack;
    c.shape = rows <= 16 ? 0 : (rows <= 64 || few((long)d.batch * (d.heads / c.pack), rows) ? 1 : 2);
    const int tile = c.shape == 0 ? 16 : (c.shape == 1 ? 64 : 128), keys = c.shape == 0 ? 32 : 64;
    c.tiles = (int)((rows + tile - 1) / tile);
    c.items = (long)d.batch * (d.heads / c.pack) * c.tiles;
    // workgroups for every place there is (a wave each: eight to a unit; 64 splits of 16384 keys instead of 32 gained nothing), but at least four tiles of keys to each
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
    c.shape = d.queries <= 64 || few((long)d.batch * d.heads, d.queries) ? 1 : 2;
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

// Whether a tensor's rows have to be copied before they can go to LDS: 16-bit elements off the 4-byte grid, or 64 rows that 31 bits cannot span
bool copied(const hot_attention_desc &d, const hot_pitch &p)
{
    const long bytes = type_bytes(d.dtype);
    return (bytes == 2 && (d.loose || (d.width | p.batch | p.head | p.row) % 2)) || p.row >= (1L << 31) / 64 / bytes - d.width;
}

long packed_width(const hot_attention_desc &d) { return (d.width + 7) / 8 * 8; }

struct Room {
    long pack_q, pack_k, pack_v, pack_go;        // negative: as they lie
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
    r.query_spans = take((long)d.groups * ((d.queries + 63) / 64) * 16);
    r.key_spans = take((long)d.groups * ((d.keys + 63) / 64) * 16);
    const auto pack = [&](const hot_pitch &p, long heads, long tokens) { return copied(d, p) ? take(d.batch * heads * tokens * packed_width(d) * type_bytes(d.dtype)) : -1L; };
    r.pack_k = pack(d.k, d.kv_heads, d.keys);
    r.pack_v = pack(d.v, d.kv_heads, d.keys);
    r.pack_q = backward ? pack(d.q, d.heads, d.queries) : -1L;
    r.pack_go = backward ? pack(d.grad_o, d.heads, d.queries) : -1L;
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
                     !aligned4(key_code) || !aligned16(query_range) || !aligned16(key_range) || !aligned8(bucket)))
        return false;
    // (groups of no tokens need no array: that of an empty tensor is null)
    if (d.groups && ((d.queries && !query_groups) || (d.keys && !key_groups) || !aligned4(query_groups) || !aligned4(key_groups))) return false;
    a.q = q;
    a.k = k;
    a.v = v;
    a.table = table;
    a.query_code = query_code ? query_code + d.first_query : nullptr;
    a.key_code = key_code;
    a.query_range = reinterpret_cast<const int4 *>(query_range);
    a.key_range = reinterpret_cast<const int4 *>(key_range);
    a.bucket = reinterpret_cast<const int2 *>(bucket);
    a.query_groups = query_groups;
    a.key_groups = key_groups;
    a.bias = reinterpret_cast<float *>(ws);
    a.query_spans = reinterpret_cast<int4 *>(ws + r.query_spans);
    a.key_spans = reinterpret_cast<int4 *>(ws + r.key_spans);
    a.part_o = reinterpret_cast<float *>(ws + r.part_o);
    return true;
}

// The tensors that go to LDS: copied, or as they lie.  False if one is off the grid that the description promises.
bool place(AttentionArgs &a, const hot_attention_desc &d, const Room &r, char *ws, bool backward, hipStream_t s)
{
    struct Part {
        const void **at;
        hot_pitch *pitch;
        long room;
        int heads, tokens;
        const int32_t *groups;
    } parts[4] = {{&a.k, &a.p_k, r.pack_k, a.kv_heads, a.keys, a.key_groups},
                  {&a.v, &a.p_v, r.pack_v, a.kv_heads, a.keys, a.key_groups},
                  {&a.q, &a.p_q, r.pack_q, a.heads, a.queries, a.query_groups},
                  {&a.grad_o, &a.p_go, r.pack_go, a.heads, a.queries, a.query_groups}};
    for (int i = 0; i < (backward ? 4 : 2); ++i) {
        const Part &p = parts[i];
        if (p.room < 0 && !aligned4(*p.at)) return false;
    }
    for (int i = 0; i < (backward ? 4 : 2); ++i) {
        Part &p = parts[i];
        if (p.room < 0) continue;
        const long w = packed_width(d);
        pack_rows(*p.at, ws + p.room, *p.pitch, a.batch, p.heads, p.tokens, a.width, (int)w, type_bytes(d.dtype), p.groups, a.groups, s);
        *p.at = ws + p.room;
        *p.pitch = hot_pitch{p.heads * p.tokens * w, p.tokens * w, w};
    }
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
    if (!place(a, *desc, r, ws, false, s)) return HOT_EINVAL;
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
    if (!place(a, *desc, r, ws, true, s)) return HOT_EINVAL;
    if (a.all_rows) {
        a.bounds_count = t == HOT_F16 ? (long)desc->batch * (desc->heads + desc->kv_heads) : 0;
        HOT_BY_TYPE(attention_begin, a);
        HOT_BY_TYPE(attention_prepare, a);
    }
    if ((grad_k || grad_v) && desc->keys && desc->batch) {
        const BackwardCut c = keys_cut(*desc);
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
