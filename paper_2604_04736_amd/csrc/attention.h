// Kernels of attention.hip for one type of elements (attention_f32.hip, attention_bf16.hip, attention_f16.hip).
//
//   z_ij = scale q_i . k_j + bias(i, j),   m_i = max_j z_ij,   l_i = sum_j exp(z_ij - m_i),   p_ij = exp(z_ij - m_i) / l_i,   o_i = sum_j p_ij v_j
//   dv_j = sum_i p_ij do_i,   dz_ij = p_ij (do_i . v_j - D_i),  D_i = do_i . o_i,   dq_i = scale sum_j dz_ij k_j,   dk_j = scale sum_i dz_ij q_i,
//   dtable[b, h] = sum of dz over the pairs of head h whose bucket is b
//
// One pass over the keys with running m and l; z is in registers alone, forward and backward.  Everything is in units of log 2: scale and the bias are
// multiplied by log2 e once, so an element costs one fused multiply-add, a subtraction and the hardware's 2^x.
// A lane holds one query's results (one key's in the kernel of dk and dv), see fragment.h: maxima and sums are additions within lanes and two shuffles, and p and
// dz are operands of the next product where they are.  Those operands have 16 bits: two pieces of each, since one rounding of p or dz does not average
// out where few keys count or where keys have a common mean (dz adds up to zero over a row, its roundings do not).
// D is formed from o and what o's rounding left over, for the same reason.
// fp16's pieces end at 2^-24: p is held times 2^14, dz in units of a bound on it, 2 max |do_i| max |v_j| of the head.
#ifndef HOT_ATTENTION_H
#define HOT_ATTENTION_H

#include <hip/hip_runtime.h>

#include "attention_args.h"
#include "element.h"
#include "fragment.h"

namespace {

using hot_detail::AttentionArgs;
using hot_detail::kBins;

constexpr float kNone = -__builtin_inff();
template <class T>
constexpr float kShift = __is_same(T, _Float16) ? 14.0f : 0.0f;

__device__ __forceinline__ float two_to(float x) { return __builtin_amdgcn_exp2f(x); }

// Workgroups go to the eight dies in turn; each die gets a run of items, so that those which read the same keys share its L2.
__device__ __forceinline__ long item_of(long id, long items)
{
    const long per = (items + 7) / 8, item = id % 8 * per + id / 8;
    return id / 8 < per && item < items ? item : -1;
}

// The pieces of a tile of rows that a thread takes from memory to LDS: sixteen bytes each
template <class T, int DP, int ROWS, int THREADS>
struct Fetch {
    typedef Piece<T> P;
    static constexpr int kPerRow = DP / P::N, kAll = ROWS * kPerRow, kEach = (kAll + THREADS - 1) / THREADS;
    typename P::V v[kEach];

    // rows first .. of `base` (pitch `row`), zeros where `there` says no
    template <class There>
    __device__ __forceinline__ void ask(const T *base, long row, int first, int width, There there)
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int c = (int)threadIdx.x + i * THREADS, r = c / kPerRow, at = c % kPerRow * P::N;
            v[i] = (typename P::V)((T)0.0f);
            if ((kAll % THREADS == 0 || c < kAll) && there(first + r)) v[i] = P::take(base + (long)(first + r) * row, at, width);
        }
    }
    __device__ __forceinline__ void put(char *tile) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int c = (int)threadIdx.x + i * THREADS, r = c / kPerRow, at = c % kPerRow * P::N;
            if (kAll % THREADS == 0 || c < kAll) *reinterpret_cast<typename P::V *>(tile + r * Rows<T, DP>::kPitch + at * (int)sizeof(T)) = v[i];
        }
    }
};

// Smallest and largest of the values that threads offer, to all of them.  `room`: two words.
__device__ __forceinline__ void range_of(int value, bool offers, int *room, int &low, int &high)
{
    if (threadIdx.x == 0) {
        room[0] = 0x7FFFFFFF;
        room[1] = -0x7FFFFFFF;
    }
    __syncthreads();
    if (offers) {
        atomicMin(room, value);
        atomicMax(room + 1, value);
    }
    __syncthreads();
    low = room[0];
    high = room[1];
}

// ---------------------------------------------------------------------------------
// The table as a vector over differences of codes, in units of log 2; what a type's lowest value would overflow to stays finite, so that it is no mask.
// And zeros for the bounds of fp16 (see above).
__global__ void __launch_bounds__(256)
hot_attention_begin_kernel(AttentionArgs a)
{
    const long n = (long)a.tables * a.heads * a.codes;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) {
        const int code = (int)(i % a.codes), h = (int)(i / a.codes % a.heads), t = (int)(i / a.codes / a.heads);
        const unsigned b = (unsigned)a.bucket[code], last = (unsigned)a.buckets - 1u;
        const long at = ((long)t * a.buckets + (b < last ? b : last)) * a.heads + h;
        const float v = a.table_type == HOT_F32 ? static_cast<const float *>(a.table)[at]
                                                : (a.table_type == HOT_BF16 ? (float)static_cast<const __bf16 *>(a.table)[at] : (float)static_cast<const _Float16 *>(a.table)[at]);
        float u = v * 1.4426950408889634f;
        if (__builtin_isfinite(v)) u = u > 3.4028234e38f ? 3.4028234e38f : (u < -3.4028234e38f ? -3.4028234e38f : u);
        a.bias[i] = u;
    }
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < a.bounds_count; i += (long)gridDim.x * 256) a.bounds[i] = 0u;
}

// A query's place: of the rows of a tile, which hold queries of `pack` heads side by side
struct Query {
    int i, h, code, group, last;       // last: the last key that it may see, by order alone
    bool there;
};

__device__ __forceinline__ Query query_of(const AttentionArgs &a, int b, int unit, int row)
{
    Query q;
    q.there = row < a.queries * a.pack;
    q.i = q.there ? row / a.pack : 0;
    q.h = unit * a.pack + (a.pack > 1 ? row - row / a.pack * a.pack : 0);
    if (!q.there) q.h = unit * a.pack;
    q.code = a.tables ? a.query_code[q.i] : 0;
    q.group = a.groups ? a.query_groups[(long)(b % a.groups) * a.queries + q.i] : 0;
    if (q.group < 0) q.there = false;
    if (!q.there) q.group = -3;            // (that of no key)
    q.last = !q.there ? -1 : (a.causal ? q.i + a.keys - a.queries : a.keys - 1);
    return q;
}

// ---------------------------------------------------------------------------------
template <class T, int DP, int QB, int WAVES, int KT>
__global__ void __launch_bounds__(64 * WAVES)
hot_attention_forward_kernel(AttentionArgs a)
{
    constexpr int THREADS = 64 * WAVES, KS = DP / 32, DB = DP / 16, KB = KT / 16, TILE = WAVES * QB * 16;
    typedef Rows<T, DP> R;
    __shared__ __attribute__((aligned(16))) char k_tile[KT * R::kPitch];
    __shared__ __attribute__((aligned(16))) char v_tile[KT * R::kPitch];
    __shared__ __attribute__((aligned(16))) int codes[KT], groups[KT];
    __shared__ int room[2];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
    const int units = a.heads / a.pack, rows = a.queries * a.pack;

    for (long id = blockIdx.x; id < ((a.items + 7) & ~7L); id += gridDim.x) {
        long item = item_of(id, a.items);
        if (item < 0) continue;
        const int split = (int)(item % a.splits);
        item /= a.splits;
        const int tile_q = a.tiles_q - 1 - (int)(item % a.tiles_q);
        item /= a.tiles_q;
        const int unit = (int)(item % units), b = (int)(item / units);
        const int kvh = unit * a.pack / a.per, table = a.tables ? b / a.entries : 0;
        const T *const q = static_cast<const T *>(a.q) + b * a.p_q.batch;
        const T *const k = static_cast<const T *>(a.k) + b * a.p_k.batch + kvh * a.p_k.head;
        const T *const v = static_cast<const T *>(a.v) + b * a.p_v.batch + kvh * a.p_v.head;
        const int *const kg = a.groups ? a.key_groups + (long)(b % a.groups) * a.keys : nullptr;

        Query at[QB];
        V8<T> qf[QB][KS];
        const float *bias[QB];
        int lowest = 0x7FFFFFFF, highest = -0x7FFFFFFF, few = 0x7FFFFFFF;
#pragma unroll
        for (int n = 0; n < QB; ++n) {
            at[n] = query_of(a, b, unit, tile_q * TILE + (wave * QB + n) * 16 + col);
            bias[n] = a.bias + ((long)table * a.heads + at[n].h) * a.codes;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                qf[n][s] = (V8<T>)((T)0.0f);
                if (at[n].there) qf[n][s] = eight(q + at[n].h * a.p_q.head + at[n].i * a.p_q.row, s * 32 + g * 8, a.width);
            }
            if (at[n].there && a.groups) {
                lowest = at[n].group < lowest ? at[n].group : lowest;
                highest = at[n].group > highest ? at[n].group : highest;
            }
        }
        int low = 0, high = 0;
        if (a.groups) {
            int l2, h2;
            range_of(lowest, true, room, low, h2);
            __syncthreads();
            range_of(highest, true, room, l2, high);
        }
        // keys that any row of this workgroup may see by order, and up to which all of them may
        const int end_row = (tile_q + 1) * TILE < rows ? (tile_q + 1) * TILE : rows, last_i = (end_row - 1) / a.pack, first_i = tile_q * TILE / a.pack;
        int visible = a.causal ? last_i + a.keys - a.queries + 1 : a.keys;
        visible = visible < 0 ? 0 : (visible > a.keys ? a.keys : visible);
        few = a.causal ? first_i + a.keys - a.queries + 1 : a.keys;
        if (few > a.keys) few = a.keys;
        const int all_tiles = (visible + KT - 1) / KT, share = (all_tiles + a.splits - 1) / a.splits;
        const int end_tile = (split + 1) * share < all_tiles ? (split + 1) * share : all_tiles;

        // the next tile that holds a key of a group of these rows
        auto wanted = [&](int tile) {
            if (a.groups)
                for (; tile < end_tile; ++tile) {
                    const int j = tile * KT + lane;
                    const int group = lane < KT && j < a.keys ? kg[j] : -1;
                    if (__ballot(group >= 0 && group >= low && group <= high)) break;
                }
            return tile;
        };
        Fetch<T, DP, KT, THREADS> next_k, next_v;
        int next_code = 0, next_group = 0;
        auto ask = [&](int tile) {
            if (tile >= end_tile) return;
            auto there = [&](int j) { return j < a.keys && (!kg || kg[j] >= 0); };
            next_k.ask(k, a.p_k.row, tile * KT, a.width, there);
            next_v.ask(v, a.p_v.row, tile * KT, a.width, there);
            const int j = tile * KT + (int)threadIdx.x;
            if ((int)threadIdx.x < KT) {
                next_code = a.tables && j < a.keys ? a.key_code[j] : 0;
                next_group = a.groups ? (j < a.keys ? kg[j] : -1) : 0;
            }
        };

        Block16<T> o[DB][QB];
        float m[QB], l[QB];
#pragma unroll
        for (int n = 0; n < QB; ++n) {
            m[n] = kNone;
            l[n] = 0.0f;
        }
        int tile = wanted(split * share);
        ask(tile);
        while (tile < end_tile) {
            __syncthreads();
            next_k.put(k_tile);
            next_v.put(v_tile);
            if ((int)threadIdx.x < KT) {
                codes[threadIdx.x] = next_code;
                groups[threadIdx.x] = next_group;
            }
            __syncthreads();
            const int k0 = tile * KT;
            tile = wanted(tile + 1);
            ask(tile);

            Block16<T> acc[KB][QB];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const V8<T> f = R::along(k_tile, kb * 16, s, lane);
#pragma unroll
                    for (int n = 0; n < QB; ++n) acc[kb][n].mac(f, qf[n][s]);
                }
            const Settled settled;
            float z[KB][QB][4], top[QB];
#pragma unroll
            for (int n = 0; n < QB; ++n) top[n] = kNone;
            const bool edge = k0 + KT > few;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const i4 kc = *reinterpret_cast<const i4 *>(codes + kb * 16 + g * 4);
                const i4 kgr = *reinterpret_cast<const i4 *>(groups + kb * 16 + g * 4);
#pragma unroll
                for (int n = 0; n < QB; ++n) {
                    const f4 s = acc[kb][n].read(settled);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float add = 0.0f;
                        if (a.tables) {
                            const unsigned at_code = (unsigned)(at[n].code - kc[i]), last = (unsigned)a.codes - 1u;
                            add = bias[n][at_code < last ? at_code : last];
                        }
                        float x = __builtin_fmaf(s[i], a.scale, add);
                        if (edge && k0 + kb * 16 + g * 4 + i > at[n].last) x = kNone;
                        if (a.groups && kgr[i] != at[n].group) x = kNone;
                        z[kb][n][i] = x;
                        top[n] = __builtin_fmaxf(top[n], x);
                    }
                }
            }
            float base[QB];
#pragma unroll
            for (int n = 0; n < QB; ++n) {
                top[n] = __builtin_fmaxf(top[n], __shfl_xor(top[n], 16));
                top[n] = __builtin_fmaxf(top[n], __shfl_xor(top[n], 32));
                const float now = __builtin_fmaxf(m[n], top[n]);
                base[n] = now == kNone ? 0.0f : now;
                if (__ballot(now > m[n])) {
                    const float by = two_to(m[n] - base[n]);
                    l[n] *= by;
#pragma unroll
                    for (int d = 0; d < DB; ++d) o[d][n].scale(settled, by);
                }
                m[n] = now;
            }
#pragma unroll
            for (int c = 0; c < KT / 32; ++c) {
                Pieces<T> p[QB];
#pragma unroll
                for (int n = 0; n < QB; ++n)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float e = two_to(z[2 * c + (i >> 2)][n][i & 3] - base[n] + kShift<T>);
                        l[n] += e;
                        p[n].set(i, e);
                    }
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const V8<T> f = R::across(v_tile, c * 32, d * 16, lane);
#pragma unroll
                    for (int n = 0; n < QB; ++n) p[n].mac(o[d][n], f);
                }
            }
        }
        const Settled settled;
#pragma unroll
        for (int n = 0; n < QB; ++n) {
            l[n] += __shfl_xor(l[n], 16);
            l[n] += __shfl_xor(l[n], 32);
            const int row = tile_q * TILE + (wave * QB + n) * 16 + col;
            if (row >= rows) continue;
            // (a row that sees nothing, or is of no group: zeros)
            const int i = row / a.pack, h = unit * a.pack + (row - i * a.pack);
            const long whole = ((long)b * a.heads + h) * a.queries + i;
            if (a.splits > 1) {
                float *const part = a.part_o + ((long)split * a.all_rows + whole) * a.width;
#pragma unroll
                for (int d = 0; d < DB; ++d) four(part, d * 16 + g * 4, a.width, o[d][n].read(settled));
                if (g == 0) {
                    a.part_ml[2 * ((long)split * a.all_rows + whole)] = m[n];
                    a.part_ml[2 * ((long)split * a.all_rows + whole) + 1] = l[n];
                }
                continue;
            }
            const float by = l[n] == 0.0f ? 0.0f : 1.0f / l[n];
            T *const to = static_cast<T *>(a.o) + b * a.p_o.batch + h * a.p_o.head + i * a.p_o.row;
            T *const rest = a.rest ? static_cast<T *>(a.rest) + b * a.p_o.batch + h * a.p_o.head + i * a.p_o.row : nullptr;
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                f4 x = o[d][n].read(settled);
                f4 left;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[j] = l[n] == 0.0f ? 0.0f : x[j] * by;
                    left[j] = x[j] - (float)(T)x[j];
                }
                four(to, d * 16 + g * 4, a.width, x);
                if (rest) four(rest, d * 16 + g * 4, a.width, left);
            }
            if (g == 0 && a.stats) {
                a.stats[2 * whole] = l[n] == 0.0f ? 0.0f : m[n];
                a.stats[2 * whole + 1] = l[n] == 0.0f ? __builtin_inff() : __builtin_log2f(l[n]) - kShift<T>;
            }
        }
        __syncthreads();
    }
}

// The splits' results joined: sixteen lanes to a row
template <class T>
__global__ void __launch_bounds__(256)
hot_attention_join_kernel(AttentionArgs a)
{
    const int t = (int)threadIdx.x & 15;
    for (long row = (long)blockIdx.x * 16 + ((int)threadIdx.x >> 4); row < a.all_rows; row += (long)gridDim.x * 16) {
        const int i = (int)(row % a.queries), h = (int)(row / a.queries % a.heads), b = (int)(row / a.queries / a.heads);
        float m = kNone;
        for (int s = 0; s < a.splits; ++s) m = __builtin_fmaxf(m, a.part_ml[2 * ((long)s * a.all_rows + row)]);
        const float base = m == kNone ? 0.0f : m;
        float l = 0.0f, o[8] = {};
        for (int s = 0; s < a.splits; ++s) {
            const long at = (long)s * a.all_rows + row;
            const float by = two_to(a.part_ml[2 * at] - base);
            l = __builtin_fmaf(a.part_ml[2 * at + 1], by, l);
            const V8<float> v = eight(a.part_o + at * a.width, t * 8, a.width);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = __builtin_fmaf(v[j], by, o[j]);
        }
        const float by = l == 0.0f ? 0.0f : 1.0f / l;
        T *const to = static_cast<T *>(a.o) + b * a.p_o.batch + h * a.p_o.head + i * a.p_o.row;
        T *const rest = a.rest ? static_cast<T *>(a.rest) + b * a.p_o.batch + h * a.p_o.head + i * a.p_o.row : nullptr;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            f4 x, left;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = l == 0.0f ? 0.0f : o[4 * c + j] * by;
                left[j] = x[j] - (float)(T)x[j];
            }
            four(to, t * 8 + c * 4, a.width, x);
            if (rest) four(rest, t * 8 + c * 4, a.width, left);
        }
        if (t == 0 && a.stats) {
            a.stats[2 * row] = l == 0.0f ? 0.0f : m;
            a.stats[2 * row + 1] = l == 0.0f ? __builtin_inff() : __builtin_log2f(l) - kShift<T>;
        }
    }
}

// ---------------------------------------------------------------------------------
// D of every query, sixteen lanes to a row; for fp16 also the largest |do_i|^2 of every head and the largest |v_j|^2 of every key head
template <class T>
__global__ void __launch_bounds__(256)
hot_attention_prepare_kernel(AttentionArgs a)
{
    const int t = (int)threadIdx.x & 15;
    const long keys = __is_same(T, _Float16) ? (long)a.batch * a.kv_heads * a.keys : 0, all = a.all_rows + keys;
    for (long row = (long)blockIdx.x * 16 + ((int)threadIdx.x >> 4); row < all; row += (long)gridDim.x * 16) {
        float sum = 0.0f, square = 0.0f;
        unsigned *bound;
        if (row < a.all_rows) {
            const int i = (int)(row % a.queries), h = (int)(row / a.queries % a.heads), b = (int)(row / a.queries / a.heads);
            const bool there = !a.groups || a.query_groups[(long)(b % a.groups) * a.queries + i] >= 0;
            bound = a.bounds + (long)b * a.heads + h;
            if (there) {
                const long o_at = b * a.p_o.batch + h * a.p_o.head + i * a.p_o.row;
                const V8<T> up = eight(static_cast<const T *>(a.grad_o) + b * a.p_go.batch + h * a.p_go.head + i * a.p_go.row, t * 8, a.width);
                const V8<T> o = eight(static_cast<const T *>(a.o) + o_at, t * 8, a.width);
                V8<T> rest = (V8<T>)((T)0.0f);
                if (a.rest) rest = eight(static_cast<const T *>(a.rest) + o_at, t * 8, a.width);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sum = __builtin_fmaf((float)up[j], (float)o[j] + (float)rest[j], sum);
                    square = __builtin_fmaf((float)up[j], (float)up[j], square);
                }
            }
        } else {
            const long at = row - a.all_rows;
            const int j0 = (int)(at % a.keys), h = (int)(at / a.keys % a.kv_heads), b = (int)(at / a.keys / a.kv_heads);
            bound = a.bounds + (long)a.batch * a.heads + (long)b * a.kv_heads + h;
            if (!a.groups || a.key_groups[(long)(b % a.groups) * a.keys + j0] >= 0) {
                const V8<T> v = eight(static_cast<const T *>(a.v) + b * a.p_v.batch + h * a.p_v.head + j0 * a.p_v.row, t * 8, a.width);
#pragma unroll
                for (int j = 0; j < 8; ++j) square = __builtin_fmaf((float)v[j], (float)v[j], square);
            }
        }
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) {
            sum += __shfl_xor(sum, off);
            square += __shfl_xor(square, off);
        }
        if (t) continue;
        if (row < a.all_rows) a.d[row] = sum;
        // (positive floats are ordered as their bits are, and the largest does not depend on the order; nan and infinity are left out)
        if constexpr (__is_same(T, _Float16))
            if (square < 3.0e38f) atomicMax(bound, __builtin_bit_cast(unsigned, square));
    }
}

// The power of two that dz of `count` heads of one key head is multiplied by before it is cut: a bound on it becomes 2^13 to 2^14
template <class T>
__device__ __forceinline__ float unit_of(const AttentionArgs &a, int b, int h, int count)
{
    if constexpr (!__is_same(T, _Float16)) return 1.0f;
    unsigned most = 0;
    for (int i = 0; i < count; ++i) {
        const unsigned bits = a.bounds[(long)b * a.heads + h + i];
        most = bits > most ? bits : most;
    }
    const float up = __builtin_bit_cast(float, most);
    const float v = __builtin_bit_cast(float, a.bounds[(long)a.batch * a.heads + (long)b * a.kv_heads + h / a.per]);
    const float bound = 2.0f * __builtin_sqrtf(up) * __builtin_sqrtf(v);
    if (!(bound > 0.0f) || !(bound < 3.0e38f)) return 1.0f;
    int e = (int)(__builtin_bit_cast(unsigned, bound) >> 23) - 126;             // bound < 2^e
    e = e < -100 ? -100 : (e > 100 ? 100 : e);
    return __builtin_bit_cast(float, (unsigned)(127 + 14 - e) << 23);
}

// ---------------------------------------------------------------------------------
// dk and dv: a wave holds KB blocks of sixteen keys, and their k and v as operands; the queries of every head that reads them go by in LDS.
template <class T, int DP, int KB, int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
hot_attention_keys_kernel(AttentionArgs a)
{
    constexpr int THREADS = 64 * WAVES, KS = DP / 32, DB = DP / 16, TILE = WAVES * KB * 16, QT = 64;
    typedef Rows<T, DP> R;
    __shared__ __attribute__((aligned(16))) char q_tile[QT * R::kPitch];
    __shared__ __attribute__((aligned(16))) char up_tile[QT * R::kPitch];
    __shared__ __attribute__((aligned(16))) float ms[QT], ls[QT], ds[QT];
    __shared__ __attribute__((aligned(16))) int codes[QT], groups[QT];
    __shared__ int room[2];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
    const int tiles_q = (a.queries + QT - 1) / QT;

    for (long id = blockIdx.x; id < ((a.items + 7) & ~7L); id += gridDim.x) {
        long item = item_of(id, a.items);
        if (item < 0) continue;
        const int tile_k = (int)(item % a.tiles_k);
        item /= a.tiles_k;
        const int kvh = (int)(item % a.kv_heads), b = (int)(item / a.kv_heads), table = a.tables ? b / a.entries : 0;
        const T *const k = static_cast<const T *>(a.k) + b * a.p_k.batch + kvh * a.p_k.head;
        const T *const v = static_cast<const T *>(a.v) + b * a.p_v.batch + kvh * a.p_v.head;
        const int *const kg = a.groups ? a.key_groups + (long)(b % a.groups) * a.keys : nullptr;
        const int *const qg = a.groups ? a.query_groups + (long)(b % a.groups) * a.queries : nullptr;
        const int past = a.keys - a.queries;

        int key[KB], code[KB], group[KB];
        V8<T> kf[KB][KS], vf[KB][KS];
        int lowest = 0x7FFFFFFF, highest = -0x7FFFFFFF;
#pragma unroll
        for (int n = 0; n < KB; ++n) {
            key[n] = tile_k * TILE + (wave * KB + n) * 16 + col;
            const bool in = key[n] < a.keys;
            code[n] = a.tables && in ? a.key_code[key[n]] : 0;
            group[n] = in ? (kg ? kg[key[n]] : 0) : -1;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                kf[n][s] = vf[n][s] = (V8<T>)((T)0.0f);
                if (group[n] >= 0) {
                    kf[n][s] = eight(k + key[n] * a.p_k.row, s * 32 + g * 8, a.width);
                    vf[n][s] = eight(v + key[n] * a.p_v.row, s * 32 + g * 8, a.width);
                }
            }
            if (group[n] >= 0) {
                lowest = group[n] < lowest ? group[n] : lowest;
                highest = group[n] > highest ? group[n] : highest;
            }
        }
        int low = 0, high = 0;
        if (a.groups) {
            int l2, h2;
            range_of(lowest, true, room, low, h2);
            __syncthreads();
            range_of(highest, true, room, l2, high);
        }
        Block16<T> dk[DB][KB], dv[DB][KB];
        const float unit = unit_of<T>(a, b, kvh * a.per, a.per);
        // the first query that sees a key of this tile
        int first = a.causal ? tile_k * TILE - past : 0;
        first = first < 0 ? 0 : first;
        const int first_tile = first / QT;

        for (int h = kvh * a.per; h < (kvh + 1) * a.per; ++h) {
            const T *const q = static_cast<const T *>(a.q) + b * a.p_q.batch + h * a.p_q.head;
            const T *const up = static_cast<const T *>(a.grad_o) + b * a.p_go.batch + h * a.p_go.head;
            const float *const bias = a.bias + ((long)table * a.heads + h) * a.codes;
            const long stat0 = ((long)b * a.heads + h) * a.queries;
            auto wanted = [&](int tile) {
                if (a.groups)
                    for (; tile < tiles_q; ++tile) {
                        const int i = tile * QT + lane;
                        const int x = i < a.queries ? qg[i] : -1;
                        if (__ballot(x >= 0 && x >= low && x <= high)) break;
                    }
                return tile;
            };
            Fetch<T, DP, QT, THREADS> next_q, next_up;
            float next_m = 0.0f, next_l = 0.0f, next_d = 0.0f;
            int next_code = 0, next_group = 0;
            auto ask = [&](int tile) {
                if (tile >= tiles_q) return;
                auto there = [&](int i) { return i < a.queries && (!qg || qg[i] >= 0); };
                next_q.ask(q, a.p_q.row, tile * QT, a.width, there);
                next_up.ask(up, a.p_go.row, tile * QT, a.width, there);
                const int i = tile * QT + (int)threadIdx.x;
                if ((int)threadIdx.x < QT) {
                    const bool in = i < a.queries;
                    next_m = in ? a.stats[2 * (stat0 + i)] : 0.0f;
                    next_l = in ? a.stats[2 * (stat0 + i) + 1] : __builtin_inff();
                    next_d = in ? a.d[stat0 + i] : 0.0f;
                    next_code = a.tables && in ? a.query_code[i] : 0;
                    next_group = in ? (qg ? qg[i] : 0) : -2;
                }
            };
            int tile = wanted(first_tile);
            ask(tile);
            while (tile < tiles_q) {
                __syncthreads();
                next_q.put(q_tile);
                next_up.put(up_tile);
                if ((int)threadIdx.x < QT) {
                    ms[threadIdx.x] = next_m;
                    ls[threadIdx.x] = next_l;
                    ds[threadIdx.x] = next_d;
                    codes[threadIdx.x] = next_code;
                    groups[threadIdx.x] = next_group;
                }
                __syncthreads();
                const int i0 = tile * QT;
                tile = wanted(tile + 1);
                ask(tile);
                // whether some pair is not to be seen by order, or by the ends
                const bool edge = a.causal && i0 + past < tile_k * TILE + TILE - 1;
#pragma unroll
                for (int c = 0; c < QT / 32; ++c) {
                    Block16<T> s[2][KB], dp[2][KB];
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int x = 0; x < KS; ++x) {
                            const V8<T> fq = R::along(q_tile, c * 32 + u * 16, x, lane), fu = R::along(up_tile, c * 32 + u * 16, x, lane);
#pragma unroll
                            for (int n = 0; n < KB; ++n) {
                                s[u][n].mac(fq, kf[n][x]);
                                dp[u][n].mac(fu, vf[n][x]);
                            }
                        }
                    const Settled settled;
                    Pieces<T> p[KB], dz[KB];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int row0 = c * 32 + u * 16 + g * 4;
                        const f4 m = *reinterpret_cast<const f4 *>(ms + row0), l = *reinterpret_cast<const f4 *>(ls + row0), d = *reinterpret_cast<const f4 *>(ds + row0);
                        const i4 qc = *reinterpret_cast<const i4 *>(codes + row0), qgr = *reinterpret_cast<const i4 *>(groups + row0);
#pragma unroll
                        for (int n = 0; n < KB; ++n) {
                            const f4 zs = s[u][n].read(settled), dps = dp[u][n].read(settled);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float add = 0.0f;
                                if (a.tables) {
                                    const unsigned at_code = (unsigned)(qc[i] - code[n]), last = (unsigned)a.codes - 1u;
                                    add = bias[at_code < last ? at_code : last];
                                }
                                float e = two_to(__builtin_fmaf(zs[i], a.scale, add) - m[i] - l[i] + kShift<T>);
                                if (group[n] != qgr[i] || (edge && key[n] > i0 + row0 + i + past)) e = 0.0f;
                                p[n].set(u * 4 + i, e);
                                dz[n].set(u * 4 + i, e * ((dps[i] - d[i]) * (unit * (__is_same(T, _Float16) ? 0x1p-14f : 1.0f))));
                            }
                        }
                    }
#pragma unroll
                    for (int x = 0; x < DB; ++x) {
                        const V8<T> fu = R::across(up_tile, c * 32, x * 16, lane), fq = R::across(q_tile, c * 32, x * 16, lane);
#pragma unroll
                        for (int n = 0; n < KB; ++n) {
                            p[n].mac(dv[x][n], fu);
                            dz[n].mac(dk[x][n], fq);
                        }
                    }
                }
            }
        }
        const Settled settled;
#pragma unroll
        for (int n = 0; n < KB; ++n) {
            if (key[n] >= a.keys) continue;
            T *const to_k = a.grad_k ? static_cast<T *>(a.grad_k) + b * a.p_gk.batch + kvh * a.p_gk.head + key[n] * a.p_gk.row : nullptr;
            T *const to_v = a.grad_v ? static_cast<T *>(a.grad_v) + b * a.p_gv.batch + kvh * a.p_gv.head + key[n] * a.p_gv.row : nullptr;
#pragma unroll
            for (int x = 0; x < DB; ++x) {
                if (to_k) four(to_k, x * 16 + g * 4, a.width, dk[x][n].read(settled) * (a.plain_scale / unit));
                if (to_v) four(to_v, x * 16 + g * 4, a.width, dv[x][n].read(settled) * (__is_same(T, _Float16) ? 0x1p-14f : 1.0f));
            }
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------
// dq, and what the table's gradient is made of.  A workgroup holds the queries of one tile and head, of several entries of the batch one after the other; every
// pair's dz is added to its difference of codes in bins of the wave's own (LDS works a wave's additions one after the other), the waves' bins are
// added up in their order and go to the table's buckets, which one wave alone adds to.
template <class T, int DP, int QB, int WAVES, bool TABLE>
__global__ void __launch_bounds__(64 * WAVES)
hot_attention_queries_kernel(AttentionArgs a)
{
    constexpr int THREADS = 64 * WAVES, KS = DP / 32, DB = DP / 16, KT = 64, TILE = WAVES * QB * 16;
    typedef Rows<T, DP> R;
    __shared__ __attribute__((aligned(16))) char k_tile[KT * R::kPitch];
    __shared__ __attribute__((aligned(16))) char v_tile[KT * R::kPitch];
    __shared__ __attribute__((aligned(16))) int codes[KT], groups[KT];
    __shared__ int room[2];
    __shared__ float bins[TABLE ? WAVES : 1][TABLE ? kBins : 1];
    extern __shared__ float buckets[];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, g = lane >> 4, col = lane & 15;

    for (long id = blockIdx.x; id < ((a.items + 7) & ~7L); id += gridDim.x) {
        long item = item_of(id, a.items);
        if (item < 0) continue;
        const long unit_item = item;
        const int tile_q = a.tiles_q - 1 - (int)(item % a.tiles_q);
        item /= a.tiles_q;
        const int h = (int)(item % a.heads), chunk = (int)(item / a.heads), kvh = h / a.per;
        const int per_table = (a.entries + a.chunk - 1) / a.chunk, table = chunk / per_table;
        const int first_b = table * a.entries + chunk % per_table * a.chunk;
        const int end_b = first_b + a.chunk < (table + 1) * a.entries ? first_b + a.chunk : (table + 1) * a.entries;
        const float *const bias = a.bias + ((long)table * a.heads + h) * a.codes;
        if constexpr (TABLE) {
            for (int i = (int)threadIdx.x; i < a.buckets; i += THREADS) buckets[i] = 0.0f;
            for (int i = lane; i < kBins; i += 64) bins[wave][i] = 0.0f;
        }
        for (int b = first_b; b < end_b; ++b) {
            const T *const q = static_cast<const T *>(a.q) + b * a.p_q.batch + h * a.p_q.head;
            const T *const up = static_cast<const T *>(a.grad_o) + b * a.p_go.batch + h * a.p_go.head;
            const T *const k = static_cast<const T *>(a.k) + b * a.p_k.batch + kvh * a.p_k.head;
            const T *const v = static_cast<const T *>(a.v) + b * a.p_v.batch + kvh * a.p_v.head;
            const int *const kg = a.groups ? a.key_groups + (long)(b % a.groups) * a.keys : nullptr;
            const float unit = unit_of<T>(a, b, h, 1);
            Query at[QB];
            V8<T> qf[QB][KS], uf[QB][KS];
            float m[QB], l[QB], dd[QB];
            int lowest = 0x7FFFFFFF, highest = -0x7FFFFFFF, code_low = 0x7FFFFFFF, code_high = -0x7FFFFFFF;
#pragma unroll
            for (int n = 0; n < QB; ++n) {
                at[n] = query_of(a, b, h, tile_q * TILE + (wave * QB + n) * 16 + col);
                m[n] = dd[n] = 0.0f;
                l[n] = __builtin_inff();
                if (at[n].there) {
                    const long row = ((long)b * a.heads + h) * a.queries + at[n].i;
                    m[n] = a.stats[2 * row];
                    l[n] = a.stats[2 * row + 1];
                    dd[n] = a.d[row];
                    lowest = at[n].group < lowest ? at[n].group : lowest;
                    highest = at[n].group > highest ? at[n].group : highest;
                    code_low = at[n].code < code_low ? at[n].code : code_low;
                    code_high = at[n].code > code_high ? at[n].code : code_high;
                }
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    qf[n][s] = uf[n][s] = (V8<T>)((T)0.0f);
                    if (at[n].there) {
                        qf[n][s] = eight(q + at[n].i * a.p_q.row, s * 32 + g * 8, a.width);
                        uf[n][s] = eight(up + at[n].i * a.p_go.row, s * 32 + g * 8, a.width);
                    }
                }
            }
            int low = 0, high = 0, qc_low = 0, qc_high = 0, unused;
            if (a.groups) {
                range_of(lowest, true, room, low, unused);
                __syncthreads();
                range_of(highest, true, room, unused, high);
                __syncthreads();
            }
            if constexpr (TABLE) {
                range_of(code_low, true, room, qc_low, unused);
                __syncthreads();
                range_of(code_high, true, room, unused, qc_high);
                __syncthreads();
            }
            const int end_row = (tile_q + 1) * TILE < a.queries ? (tile_q + 1) * TILE : a.queries;
            int visible = a.causal ? end_row - 1 + a.keys - a.queries + 1 : a.keys;
            visible = visible < 0 ? 0 : (visible > a.keys ? a.keys : visible);
            int few = a.causal ? tile_q * TILE + a.keys - a.queries + 1 : a.keys;
            if (few > a.keys) few = a.keys;
            const int end_tile = (visible + KT - 1) / KT;
            auto wanted = [&](int tile) {
                if (a.groups)
                    for (; tile < end_tile; ++tile) {
                        const int j = tile * KT + lane;
                        const int x = j < a.keys ? kg[j] : -1;
                        if (__ballot(x >= 0 && x >= low && x <= high)) break;
                    }
                return tile;
            };
            Fetch<T, DP, KT, THREADS> next_k, next_v;
            int next_code = 0, next_group = 0;
            auto ask = [&](int tile) {
                if (tile >= end_tile) return;
                auto there = [&](int j) { return j < a.keys && (!kg || kg[j] >= 0); };
                next_k.ask(k, a.p_k.row, tile * KT, a.width, there);
                next_v.ask(v, a.p_v.row, tile * KT, a.width, there);
                const int j = tile * KT + (int)threadIdx.x;
                if ((int)threadIdx.x < KT) {
                    next_code = a.tables && j < a.keys ? a.key_code[j] : 0;
                    next_group = a.groups ? (j < a.keys ? kg[j] : -1) : 0;
                }
            };
            Block16<T> dq[DB][QB];
            int tile = wanted(0);
            ask(tile);
            while (tile < end_tile) {
                __syncthreads();
                next_k.put(k_tile);
                next_v.put(v_tile);
                if ((int)threadIdx.x < KT) {
                    codes[threadIdx.x] = next_code;
                    groups[threadIdx.x] = next_group;
                }
                __syncthreads();
                const int k0 = tile * KT, here = tile;
                tile = wanted(tile + 1);
                ask(tile);
                const bool edge = k0 + KT > few;
                int bin_low = 0, bins_all = 0;
                if constexpr (TABLE) {
                    bin_low = qc_low - a.key_range[2 * here + 1];
                    bins_all = qc_high - a.key_range[2 * here] - bin_low + 1;
                }
                float grad[TABLE ? KT / 16 : 1][QB][4];
#pragma unroll
                for (int c = 0; c < KT / 32; ++c) {
                    Block16<T> s[2][QB], dp[2][QB];
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int x = 0; x < KS; ++x) {
                            const V8<T> fk = R::along(k_tile, c * 32 + u * 16, x, lane), fv = R::along(v_tile, c * 32 + u * 16, x, lane);
#pragma unroll
                            for (int n = 0; n < QB; ++n) {
                                s[u][n].mac(fk, qf[n][x]);
                                dp[u][n].mac(fv, uf[n][x]);
                            }
                        }
                    const Settled settled;
                    Pieces<T> dz[QB];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int row0 = c * 32 + u * 16 + g * 4;
                        const i4 kc = *reinterpret_cast<const i4 *>(codes + row0), kgr = *reinterpret_cast<const i4 *>(groups + row0);
#pragma unroll
                        for (int n = 0; n < QB; ++n) {
                            const f4 zs = s[u][n].read(settled), dps = dp[u][n].read(settled);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float add = 0.0f;
                                if (a.tables) {
                                    const unsigned at_code = (unsigned)(at[n].code - kc[i]), last = (unsigned)a.codes - 1u;
                                    add = bias[at_code < last ? at_code : last];
                                }
                                float e = two_to(__builtin_fmaf(zs[i], a.scale, add) - m[n] - l[n]);
                                if (edge && k0 + row0 + i > at[n].last) e = 0.0f;
                                if (a.groups && kgr[i] != at[n].group) e = 0.0f;
                                const float w = e * (dps[i] - dd[n]);
                                if constexpr (TABLE) grad[2 * c + u][n][i] = w;
                                dz[n].set(u * 4 + i, w * unit);
                            }
                        }
                    }
#pragma unroll
                    for (int x = 0; x < DB; ++x) {
                        const V8<T> f = R::across(k_tile, c * 32, x * 16, lane);
#pragma unroll
                        for (int n = 0; n < QB; ++n) dz[n].mac(dq[x][n], f);
                    }
                }
                if constexpr (TABLE) {
                    // (as many bins at a time as there are; differences beyond them wait for their turn)
                    for (int done = 0; done < bins_all; done += kBins) {
                        const int now = bins_all - done < kBins ? bins_all - done : kBins;
#pragma unroll
                        for (int x = 0; x < KT / 16; ++x) {
                            const i4 kc = *reinterpret_cast<const i4 *>(codes + x * 16 + g * 4);
#pragma unroll
                            for (int n = 0; n < QB; ++n)
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const int bin = at[n].code - kc[i] - bin_low - done;
                                    if (at[n].there && (unsigned)bin < (unsigned)now) __hip_atomic_fetch_add(&bins[wave][bin], grad[x][n][i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                                }
                        }
                        __syncthreads();
                        if (wave == 0)
                            for (int i = lane; i < now; i += 64) {
                                float sum = 0.0f;
#pragma unroll
                                for (int w = 0; w < WAVES; ++w) {
                                    sum += bins[w][i];
                                    bins[w][i] = 0.0f;
                                }
                                const unsigned code = (unsigned)(bin_low + done + i), last = (unsigned)a.codes - 1u;
                                const unsigned bucket = (unsigned)a.bucket[code < last ? code : last], most = (unsigned)a.buckets - 1u;
                                __hip_atomic_fetch_add(&buckets[bucket < most ? bucket : most], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                            }
                        __syncthreads();
                    }
                }
            }
            const Settled settled;
            if (a.grad_q)
#pragma unroll
                for (int n = 0; n < QB; ++n) {
                    const int row = tile_q * TILE + (wave * QB + n) * 16 + col;
                    if (row >= a.queries) continue;
                    T *const to = static_cast<T *>(a.grad_q) + b * a.p_gq.batch + h * a.p_gq.head + row * a.p_gq.row;
#pragma unroll
                    for (int x = 0; x < DB; ++x) four(to, x * 16 + g * 4, a.width, dq[x][n].read(settled) * (a.plain_scale / unit));
                }
            __syncthreads();
        }
        if constexpr (TABLE) {
            float *const to = a.parts + unit_item * a.buckets;
            for (int i = (int)threadIdx.x; i < a.buckets; i += THREADS) to[i] = buckets[i];
            __syncthreads();
        }
    }
}

// The table's gradient: the workgroups' sums, 64 buckets and 16 runs of workgroups at a time
__global__ void __launch_bounds__(1024)
hot_attention_table_kernel(AttentionArgs a)
{
    __shared__ float runs[16][64];
    const int lane = (int)threadIdx.x & 63, run = (int)threadIdx.x >> 6, h = (int)blockIdx.y, table = (int)blockIdx.z;
    const int col = (int)blockIdx.x * 64 + lane, per_table = (a.entries + a.chunk - 1) / a.chunk;
    float sum = 0.0f;
    if (col < a.buckets)
        for (long u = run; u < (long)per_table * a.tiles_q; u += 16) {
            const long chunk = (long)table * per_table + u / a.tiles_q, unit = (chunk * a.heads + h) * a.tiles_q + u % a.tiles_q;
            sum += a.parts[unit * a.buckets + col];
        }
    runs[run][lane] = sum;
    __syncthreads();
    if (run || col >= a.buckets) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += runs[i][lane];
    store_as(a.grad_table, a.table_type, ((long)table * a.buckets + col) * a.heads + h, sum);
}

// ---------------------------------------------------------------------------------
// Host side: what is launched for one type

inline unsigned blocks_for(long items)
{
    const long most = 1L << 20, up = (items + 7) & ~7L;
    return (unsigned)(up < most ? up : most);
}

template <class T, int DP>
void forward_go(const AttentionArgs &a, hipStream_t s)
{
    if (a.shape == 0) hot_attention_forward_kernel<T, DP, 1, 1, 32><<<blocks_for(a.items), 64, 0, s>>>(a);
    else if (a.shape == 1) hot_attention_forward_kernel<T, DP, 1, 4, 64><<<blocks_for(a.items), 256, 0, s>>>(a);
    else hot_attention_forward_kernel<T, DP, 2, 4, 64><<<blocks_for(a.items), 256, 0, s>>>(a);
}

template <class T, int DP>
void queries_go(const AttentionArgs &a, hipStream_t s)
{
    const unsigned blocks = blocks_for(a.items);
    if (a.grad_table) {
        if (a.shape == 1) hot_attention_queries_kernel<T, DP, 1, 4, true><<<blocks, 256, a.buckets * 4, s>>>(a);
        else hot_attention_queries_kernel<T, DP, 2, 4, true><<<blocks, 256, a.buckets * 4, s>>>(a);
    } else if (a.shape == 1) hot_attention_queries_kernel<T, DP, 1, 4, false><<<blocks, 256, 0, s>>>(a);
    else hot_attention_queries_kernel<T, DP, 2, 4, false><<<blocks, 256, 0, s>>>(a);
}

template <class T, int DP>
void keys_go(const AttentionArgs &a, hipStream_t s)
{
    hot_attention_keys_kernel<T, DP, 1, 4><<<blocks_for(a.items), 256, 0, s>>>(a);
}

#define HOT_BY_WIDTH(GO)                    \
    if (a.width <= 32) GO<T, 32>(a, s);     \
    else if (a.width <= 64) GO<T, 64>(a, s); \
    else if (a.width <= 96) GO<T, 96>(a, s); \
    else GO<T, 128>(a, s)

}  // namespace

namespace hot_detail {

template <class T>
void attention_begin(const AttentionArgs &a, hipStream_t s)
{
    const long n = (long)a.tables * a.heads * a.codes, all = n > a.bounds_count ? n : a.bounds_count;
    if (!all) return;
    const long blocks = (all + 255) / 256;
    hot_attention_begin_kernel<<<(unsigned)(blocks < 2048 ? blocks : 2048), 256, 0, s>>>(a);
}

template <class T>
void attention_forward(const AttentionArgs &a, hipStream_t s)
{
    HOT_BY_WIDTH(forward_go);
    if (a.splits > 1) {
        const long blocks = (a.all_rows + 15) / 16;
        hot_attention_join_kernel<T><<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, s>>>(a);
    }
}

template <class T>
void attention_prepare(const AttentionArgs &a, hipStream_t s)
{
    const long blocks = (a.all_rows + (__is_same(T, _Float16) ? (long)a.batch * a.kv_heads * a.keys : 0) + 15) / 16;
    hot_attention_prepare_kernel<T><<<(unsigned)(blocks < 8192 ? blocks : 8192), 256, 0, s>>>(a);
}

template <class T>
void attention_keys(const AttentionArgs &a, hipStream_t s)
{
    HOT_BY_WIDTH(keys_go);
}

template <class T>
void attention_queries(const AttentionArgs &a, hipStream_t s)
{
    if (a.items) {
        HOT_BY_WIDTH(queries_go);
    }
    if (a.grad_table) hot_attention_table_kernel<<<dim3((unsigned)((a.buckets + 63) / 64), (unsigned)a.heads, (unsigned)a.tables), 1024, 0, s>>>(a);
}

}  // namespace hot_detail

#define HOT_ATTENTION_OF(T)                                                       \
    template void hot_detail::attention_begin<T>(const AttentionArgs &, hipStream_t);   \
    template void hot_detail::attention_forward<T>(const AttentionArgs &, hipStream_t); \
    template void hot_detail::attention_prepare<T>(const AttentionArgs &, hipStream_t); \
    template void hot_detail::attention_keys<T>(const AttentionArgs &, hipStream_t);    \
    template void hot_detail::attention_queries<T>(const AttentionArgs &, hipStream_t)

#endif  // HOT_ATTENTION_H
