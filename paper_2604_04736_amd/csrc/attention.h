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
// The backward kernels round as the forward one did: z first, then z - m, then - log2 l.  (m + log2 l as one number is shorter by one addition, but where |m| is large, by a bias or a product that a row's keys
// share, log2 l is lost in it, and z keeps what the forward pass rounded off: p then added up to anything but one.)
// fp16's pieces end at 2^-24: p is held times 2^14, dz in units of a bound on it, 2 max |do_i| max |v_j| of the head.
#ifndef HOT_ATTENTION_H
#define HOT_ATTENTION_H

#include <hip/hip_runtime.h>

#include "attention_args.h"
#include "element.h"
#include "fragment.h"

namespace {

using hot_detail::AttentionArgs;

constexpr int kMostCode = 1 << 28;               // beyond every code, and far enough from the ends of int to be added to
constexpr float kNone = -__builtin_inff();
template <class T>
constexpr float kShift = __is_same(T, _Float16) ? 14.0f : 0.0f;
// what o's rounding leaves over is held in units of 1 / kFiner: of fp16 it is at most 16, and at 2^-24 its steps would end where o is some 2^-13
template <class T>
constexpr float kFiner = __is_same(T, _Float16) ? 2048.0f : 1.0f;

__device__ __forceinline__ float two_to(float x) { return __builtin_amdgcn_exp2f(x); }

// ... times 2^kShift (for the other types no addition of zero, which the compiler would keep)
template <class T>
__device__ __forceinline__ float shifted(float x)
{
    if constexpr (__is_same(T, _Float16)) x += kShift<T>;
    return two_to(x);
}

// Which item a workgroup takes.  Splits of one tile lie side by side, then the heads (of all entries), then the tiles, those with the most work first where causal order
// makes them unequal: the last ones to finish are short, and since workgroups go to the eight dies in turn, a head's tiles stay on one die where heads are a multiple of eight.
__device__ __forceinline__ long item_of(long items)
{
    const long id = (long)blockIdx.y * gridDim.x + blockIdx.x;
    return id < items ? id : -1;
}

// The same number, of which the compiler does not know it: what is made of it is made where it stands.  (Moved out of loops, places in LDS took a hundred registers, for
// which others were spilled.)
__device__ __forceinline__ int fresh_lane(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// Whether 32 keys' part of o, and 32 queries' part of dk and dv, is added up by itself before it goes to the sum.  float32's instruction takes four of them, so that o was one chain of 1024 additions over 4096
// keys, dk and dv one of all queries of the heads that share a key.  What o's leave off is in D, alike for all keys of a row, and the sums of the table's gradient do not average it out (16 heads x 4096 tokens
// whose values have a common part: 3 times as far from 64 bits).  Now 128 additions of sums of eight: 16 heads x 4096 x 128 in causal order 0.95 -> 1.00 ms forward, 3.42 -> 3.48 a pass for dk and dv.
// The instruction of 16-bit types takes 32 keys anyway.
template <class T>
constexpr bool kFresh = sizeof(T) == 4;

// Tiles in LDS: two of 16-bit elements, one on its way while the other is worked on; one of float32, whose products take longer than its way
template <class T>
constexpr int kStages = sizeof(T) == 2 ? 2 : 1;

// Two tiles of ROWS rows straight from memory to LDS, one behind the other, 1024 bytes of LDS to an instruction of a wave, sixteen of them a lane.  What is no element, rows behind the
// last and rows of negative groups are zeros: the hardware's answer to an offset outside its window.  A lane's places do not change from tile to tile.
// What of a row is no whole piece goes through registers (tail).
constexpr unsigned kBeyond = 0x80000000u;
typedef __amdgpu_buffer_rsrc_t Window;

template <class T, int DP, int ROWS, int WAVES>
struct Bring {
    typedef Rows<T, DP, ROWS> R;
    static constexpr int N = 16 / (int)sizeof(T), kLoads = R::kBytes / 1024, kEach = (kLoads + WAVES - 1) / WAVES;
    static_assert(64 * WAVES >= 2 * ROWS, "a thread to a row's tail");
    int row[kEach];
    unsigned off[2][kEach];
    T ends[N - 1];

    __device__ __forceinline__ void begin(long pitch0, long pitch1, int width)
    {
        const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            int at;
            const bool is = R::at_byte((wave + i * WAVES) * 1024 + lane * 16, row[i], at);
            off[0][i] = (unsigned)(row[i] * (int)pitch0 + at) * (unsigned)sizeof(T);
            off[1][i] = (unsigned)(row[i] * (int)pitch1 + at) * (unsigned)sizeof(T);
            if (!is || at + N > width) row[i] = 0x7FFFFFFF;
        }
    }
    // base0, base1: the tiles' first rows; last: their last row that is there; groups: those of the rows, or null
    __device__ __forceinline__ void ask(const T *base0, long pitch0, const T *base1, long pitch1, int width, int last, const int *groups, lds_char *to)
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        if (width % N) {
            const int r = (int)threadIdx.x % ROWS, from = r < last ? r : last;
            const T *const end = ((int)threadIdx.x < ROWS ? base0 + from * pitch0 : base1 + from * pitch1) + width / N * N;
#pragma unroll
            for (int j = 0; j < N - 1; ++j) ends[j] = end[j < width % N ? j : 0];
            const bool there = (int)threadIdx.x < 2 * ROWS && r <= last && (!groups || groups[from] >= 0);
#pragma unroll
            for (int j = 0; j < N - 1; ++j) ends[j] = there ? ends[j] : (T)0.0f;
        }
        int g[kEach];
        if (groups)
#pragma unroll
            for (int i = 0; i < kEach; ++i) g[i] = groups[row[i] <= last ? row[i] : 0];
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const Window window = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(which ? base1 : base0), 0, (int)kBeyond, 0x00020000);
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                if (kLoads % WAVES && wave + i * WAVES >= kLoads) break;
                bool there = row[i] <= last;
                if (groups) there = there & (g[i] >= 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(window, (__attribute__((address_space(3))) void *)(to + which * R::kBytes + (wave + i * WAVES) * 1024), 16,
                                                         there ? (int)off[which][i] : (int)kBeyond, 0, 0, 0);
            }
        }
    }
    // the rows' tails, once the tiles have arrived (a barrier behind them)
    __device__ __forceinline__ void tail(lds_char *tile, int width) const
    {
        if (width % N == 0) return;
        const int r = (int)threadIdx.x % ROWS, which = (int)threadIdx.x / ROWS;
        if (which < 2)
#pragma unroll
            for (int j = 0; j < N - 1; ++j)
                if (j < width % N) *(__attribute__((address_space(3))) T *)(tile + which * R::kBytes + R::place(r, width / N * N + j)) = ends[j];
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
};

// Everything that was sent for has come, to all waves.  (The builtin, not an instruction of our own: the compiler has to know that nothing is on its way any more, or it waits
// in the loops behind for what came before them.)
__device__ __forceinline__ void arrive()
{
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0)
    __syncthreads();
}

// What all lanes read alike, and nobody writes meanwhile, through the scalar cache: vector loads come back in order, and one that is waited for would wait for the tile on its way
typedef int i2 __attribute__((ext_vector_type(2)));
template <class X>
__device__ __forceinline__ X alike_as(const void *p)
{
    return *(const __attribute__((address_space(4))) X *)(uintptr_t)p;
}
__device__ __forceinline__ float alike(const float *p) { return alike_as<float>(p); }
__device__ __forceinline__ int2 alike(const int2 *p)
{
    const i2 v = alike_as<i2>(p);
    return int2{v[0], v[1]};
}
__device__ __forceinline__ int4 alike(const int4 *p)
{
    const i4 v = alike_as<i4>(p);
    return int4{v[0], v[1], v[2], v[3]};
}

// ... of codes, whose entries also say whether codes go up by one from token to token (z)
__device__ __forceinline__ int2 codes_over(const int4 *ranges, int first, int last, bool &line)
{
    int4 s = alike(ranges + (first >> 6));
    for (int t = (first >> 6) + 1; t <= last >> 6; ++t) {
        const int4 u = alike(ranges + t);
        s.x = u.x < s.x ? u.x : s.x;
        s.y = u.y > s.y ? u.y : s.y;
        s.z &= u.z;
    }
    line = s.z != 0;
    return int2{s.x, s.y};
}

// Smallest and largest group of 64 rows each, and whether some are of a negative one (z), from the 64 of row `first` to those of row `last`
__device__ __forceinline__ int4 span_over(const int4 *spans, int first, int last)
{
    int4 s = alike(spans + (first >> 6));
    for (int t = (first >> 6) + 1; t <= last >> 6; ++t) {
        const int4 u = alike(spans + t);
        s.x = u.x < s.x ? u.x : s.x;
        s.y = u.y > s.y ? u.y : s.y;
        s.z |= u.z;
    }
    return s;
}

// Whether all rows of both spans are of one group: every pair may see each other, by groups
__device__ __forceinline__ bool together(int4 a, int4 b) { return (a.z | b.z) == 0 && a.x == a.y && b.x == b.y && a.x == b.x; }

// The tiles first .. end - 1 of T rows whose groups can meet those of `mine`, one after the other: sixty-four are looked at at once
template <int T>
struct Walk {
    const int4 *spans;           // of 64 rows each; null: all tiles
    int4 mine;
    int base, end;
    unsigned long mask;

    __device__ __forceinline__ void look(int from)
    {
        base = from;
        const int t = from + ((int)threadIdx.x & 63);
        bool meets = t < end;
        if (meets && spans) {
            const int4 s = spans[t * T >> 6];
            meets = s.x <= s.y && s.x <= mine.y && s.y >= mine.x;
        }
        mask = __ballot(meets);
    }
    __device__ __forceinline__ int begin(const int4 *spans_, int4 mine_, int first, int end_)
    {
        spans = spans_;
        mine = mine_;
        end = end_;
        if (!spans) return first;
        look(first);
        return next(0);
    }
    __device__ __forceinline__ int next(int now)
    {
        if (!spans) return now + 1;
        while (!mask) {
            if (base + 64 >= end) return end;
            look(base + 64);
        }
        const int t = base + __builtin_ctzl(mask);
        mask &= mask - 1;
        return t;
    }
};

// How the bias of a tile of pairs is had.  The differences of codes between the two sides' ranges lie in low .. high: if they are of one bucket it is one number; if they are
// few they are staged in LDS; else each pair goes to memory.
constexpr int kOne = 0, kStaged = 1, kFar = 2;

// ROOM: how many are staged at most.  640 hold a window of 12 x 12 tokens; beside tiles of 128 16-bit elements 384, so that two workgroups' share a compute unit's LDS.
template <int THREADS, int ROOM>
struct Bias {
    static constexpr int kRoom = ROOM;
    float v, one;
    int bucket, low, count, form, all;

    // (the first THREADS of what is staged come with the tile's rows; more there are only in wide windows)
    template <bool BUCKETS>
    __device__ __forceinline__ void ask(const AttentionArgs &a, const float *bias, int2 queries, int2 keys, int heads)
    {
        form = kOne;
        one = 0.0f;
        if (!a.tables) return;
        low = queries.x - keys.y;
        int high = queries.y - keys.x;
        low = low < 0 ? 0 : (low < a.codes ? low : a.codes - 1);
        high = high < low ? low : (high < a.codes ? high : a.codes - 1);
        count = high - low + 1;
        const int2 run = alike(a.bucket + low);
        all = run.x;
        one = alike(bias + low);
        form = run.y >= high ? kOne : (heads == 1 ? (count <= kRoom ? kStaged : kFar) : (count * heads <= kRoom ? kStaged : kFar));
        const int at = low + ((int)threadIdx.x < count ? (int)threadIdx.x : 0);
        v = bias[at];
        if constexpr (BUCKETS) bucket = a.bucket[at].x;
    }
    template <bool BUCKETS>
    __device__ __forceinline__ void put(const AttentionArgs &a, const float *bias, float *room, unsigned short *buckets, int heads) const
    {
        if (form != kStaged) return;
        const auto within = [&](int b) { return (unsigned short)((unsigned)b < (unsigned)a.buckets ? b : a.buckets - 1); };
        if ((int)threadIdx.x < count) {
            room[threadIdx.x] = v;
            if constexpr (BUCKETS) buckets[threadIdx.x] = within(bucket);
        }
#pragma unroll 1
        for (int at = (int)threadIdx.x + THREADS; at < count; at += THREADS) {
            room[at] = bias[low + at];
            if constexpr (BUCKETS) buckets[at] = within(a.bucket[low + at].x);
        }
        // (the biases of further heads behind those of the first)
#pragma unroll 1
        for (int h = 1; h < heads; ++h)
#pragma unroll 1
            for (int at = (int)threadIdx.x; at < count; at += THREADS) room[h * count + at] = bias[(long)h * a.codes + low + at];
    }
};

template <int FORM, bool MASKED>
struct Form {
    static constexpr int kForm = FORM;
    static constexpr bool kMasked = MASKED;
};

// go(Form<...>) for what a tile asks for
template <class Go>
__device__ __forceinline__ void by_form(int form, bool masked, Go go)
{
    if (form == kOne) {
        if (masked) go(Form<kOne, true>{});
        else go(Form<kOne, false>{});
    } else if (form == kStaged) {
        if (masked) go(Form<kStaged, true>{});
        else go(Form<kStaged, false>{});
    } else go(Form<kFar, true>{});
}

// ---------------------------------------------------------------------------------
// The table as a vector over differences of codes, in units of log 2; what a type's lowest value would overflow to stays finite, so that it is no mask.
// Smallest and largest group of 64 queries and of 64 keys each (those that are not negative).  And zeros for the bounds of fp16 (see above).
__global__ void __launch_bounds__(256)
hot_attention_begin_kernel(AttentionArgs a)
{
    const long n = (long)a.tables * a.heads * a.codes;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) {
        const int code = (int)(i % a.codes), h = (int)(i / a.codes % a.heads), t = (int)(i / a.codes / a.heads);
        const unsigned b = (unsigned)a.bucket[code].x, last = (unsigned)a.buckets - 1u;
        const long at = ((long)t * a.buckets + (b < last ? b : last)) * a.heads + h;
        const float v = a.table_type == HOT_F32 ? static_cast<const float *>(a.table)[at]
                                                : (a.table_type == HOT_BF16 ? (float)static_cast<const __bf16 *>(a.table)[at] : (float)static_cast<const _Float16 *>(a.table)[at]);
        float u = v * 1.4426950408889634f;
        if (__builtin_isfinite(v)) u = u > 3.4028234e38f ? 3.4028234e38f : (u < -3.4028234e38f ? -3.4028234e38f : u);
        a.bias[i] = u;
    }
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < a.bounds_count; i += (long)gridDim.x * 256) a.bounds[i] = 0u;
    if (!a.groups) return;
    const int tiles_q = (a.queries + 63) >> 6, tiles_k = (a.keys + 63) >> 6, lane = (int)threadIdx.x & 63;
    const long all = (long)a.groups * (tiles_q + tiles_k);
    for (long i = (long)blockIdx.x * 4 + (threadIdx.x >> 6); i < all; i += (long)gridDim.x * 4) {
        const bool of_keys = i >= (long)a.groups * tiles_q;
        const long at = of_keys ? i - (long)a.groups * tiles_q : i;
        const int tiles = of_keys ? tiles_k : tiles_q, count = of_keys ? a.keys : a.queries, row = (int)(at / tiles), r = (int)(at % tiles) * 64 + lane;
        const int g = r < count ? (of_keys ? a.key_groups : a.query_groups)[(long)row * count + r] : -1;
        int low = g < 0 ? 0x7FFFFFFF : g, high = g;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            const int l = __shfl_xor(low, off), h = __shfl_xor(high, off);
            low = l < low ? l : low;
            high = h > high ? h : high;
        }
        const int none = __ballot(r < count && g < 0) != 0;
        if (lane == 0) (of_keys ? a.key_spans : a.query_spans)[at] = int4{low, high, none, 0};
    }
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
    row = q.there ? row : 0;
    q.i = row / a.pack;
    q.h = unit * a.pack + (row - q.i * a.pack);
    q.code = a.tables ? a.query_code[q.i] : 0;
    q.group = a.groups ? a.query_groups[(long)(b % a.groups) * a.queries + q.i] : 0;
    if (q.group < 0) q.there = false;
    if (!q.there) q.group = -3;            // (that of no key)
    q.last = !q.there ? -1 : (a.causal ? q.i + (a.keys - a.queries) : a.keys - 1);
    return q;
}

// The range of codes of queries first .. last of an entry: that of the 64s of the whole line which they lie in
__device__ __forceinline__ int2 query_codes(const AttentionArgs &a, int first, int last, bool &line)
{
    return a.tables ? codes_over(a.query_range, a.first_query + first, a.first_query + last, line) : int2{0, 0};
}

// ---------------------------------------------------------------------------------
// o, and the rows' statistics.  A wave holds QB blocks of sixteen queries as operands and their o in registers; KT keys and values at a time go by in LDS, the next tile of 16-bit
// types on its way meanwhile.  Two products of 16 x 16 x DP for a block of sixteen keys, and a third one for p's second piece: with 16 heads x 8192 tokens x 128 bf16 in causal
// order 0.63 ms, half of the matrix rate that a large product reaches for these three, the rest being what softmax issues beside them (0.70 with every p converted by itself, and once
// more for its second piece).
// Two blocks of queries to a wave halve LDS's reading at width 128 (one block and eight waves: 0.75 ms where this was 0.70); up to 96 elements eight waves of one block have the registers to be four to a
// unit's quarter (two texts' rows of 3001 x 8 heads x 80 fp16, packed, 93 -> 78 us; such few tiles are 64 rows now).
// One wave and 32 keys where a tile has up to sixteen rows: bound by memory, 335 MB of eight caches of up to 16384 x 8 heads x 128 bf16 in 80 to 83 us, 4.1 TB/s (four waves with 64 keys, three of them without
// rows: 124 us).
template <class T, int DP, int QB, int WAVES, int KT>
__global__ void __launch_bounds__(64 * WAVES, WAVES == 8 ? 4 : 2)
hot_attention_forward_kernel(AttentionArgs a)
{
    constexpr int THREADS = 64 * WAVES, KS = DP / 32, DB = DP / 16, TILE = WAVES * QB * 16;
    typedef Rows<T, DP, KT> R;
    typedef Bring<T, DP, KT, WAVES> B;
    // (one wave with few rows: twice as many of them to a compute unit bring more than a second tile of each)
    constexpr int STAGES = WAVES == 1 ? 1 : kStages<T>;
    typedef Bias<THREADS, THREADS < 256 ? 256 : (sizeof(T) == 2 && DP > 64 ? 384 : 640)> Staging;
    __shared__ __attribute__((aligned(1024))) char tiles[STAGES * 2 * R::kBytes];
    __shared__ __attribute__((aligned(16))) int all_codes[STAGES * KT], all_groups[STAGES * KT];
    __shared__ float all_staged[STAGES * Staging::kRoom];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
    const int rows = a.queries * a.pack;

    long item = item_of(a.items);
    if (item < 0) return;
    const int split = (int)(item % a.splits);
    item /= a.splits;
    const int units = a.heads / a.pack, unit = (int)(item % units);
    item /= units;
    const int b = (int)(item % a.batch), tile_q = a.tiles_q - 1 - (int)(item / a.batch), kvh = unit * a.pack / a.per, table = a.tables ? b / a.entries : 0;
    const T *const q = static_cast<const T *>(a.q) + b * a.p_q.batch;
    const T *const k = static_cast<const T *>(a.k) + b * a.p_k.batch + kvh * a.p_k.head;
    const T *const v = static_cast<const T *>(a.v) + b * a.p_v.batch + kvh * a.p_v.head;
    const int *const kg = a.groups ? a.key_groups + (long)(b % a.groups) * a.keys : nullptr;
    const int end_row = (tile_q + 1) * TILE < rows ? (tile_q + 1) * TILE : rows, last_i = (end_row - 1) / a.pack, first_i = tile_q * TILE / a.pack;

    Query at[QB];
    V8<T> qf[QB][KS];
#pragma unroll
    for (int n = 0; n < QB; ++n) {
        at[n] = query_of(a, b, unit, tile_q * TILE + (wave * QB + n) * 16 + col);
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[n][s] = eight(q + at[n].h * a.p_q.head + at[n].i * a.p_q.row, s * 32 + g * 8, a.width, at[n].there);
    }
    // (of the first of heads side by side)
    const float *const bias = a.bias + ((long)table * a.heads + unit * a.pack) * a.codes;
    bool line = false;
    const int2 mine = query_codes(a, first_i, last_i, line);
    // keys that any row of this workgroup may see by order, and up to which all of them may
    int visible = a.causal ? last_i + (a.keys - a.queries) + 1 : a.keys, few = a.causal ? first_i + (a.keys - a.queries) + 1 : a.keys;
    visible = visible < 0 ? 0 : (visible > a.keys ? a.keys : visible);
    if (few > a.keys) few = a.keys;
    const int all_tiles = (visible + KT - 1) / KT, share = (all_tiles + a.splits - 1) / a.splits;
    const int end_tile = (split + 1) * share < all_tiles ? (split + 1) * share : all_tiles;

    const int4 *const spans = a.groups ? a.key_spans + (long)(b % a.groups) * ((a.keys + 63) >> 6) : nullptr;
    const int4 my_groups = a.groups ? span_over(a.query_spans + (long)(b % a.groups) * ((a.queries + 63) >> 6), first_i, last_i) : int4{0, 0, 0, 0};
    bool next_apart = false;             // whether groups keep some pairs of the next tile apart
    Walk<KT> walk;
    B bring;
    bring.begin(a.p_k.row, a.p_v.row, a.width);
    Staging next_bias;
    float next_one[QB] = {};
    int next_code = 0, next_group = 0;
    auto ask = [&](int tile, lds_char *to) {
        if (tile >= end_tile) return;
        const int last = a.keys - 1 - tile * KT;
        const int4 span = a.groups ? alike(spans + (tile * KT >> 6)) : int4{0, 0, 0, 0};
        next_apart = a.groups && !together(span, my_groups);
        bring.ask(k + (long)tile * KT * a.p_k.row, a.p_k.row, v + (long)tile * KT * a.p_v.row, a.p_v.row, a.width, last, span.z ? kg + tile * KT : nullptr, to);
        if ((int)threadIdx.x < KT) {
            const int j = tile * KT + ((int)threadIdx.x < last ? (int)threadIdx.x : last);
            next_code = a.tables ? a.key_code[j] : 0;
            next_group = kg ? kg[j] : 0;
            if ((int)threadIdx.x > last) next_group = -1;
        }
        next_bias.template ask<false>(a, bias, mine, a.tables ? codes_over(a.key_range, tile * KT, tile * KT, line) : int2{0, 0}, a.pack);
        if (a.tables)
#pragma unroll
            for (int n = 0; n < QB; ++n) next_one[n] = bias[(long)(at[n].h - unit * a.pack) * a.codes + next_bias.low];
    };

    Block16<T> o[DB][QB];
    float m[QB], l[QB];
#pragma unroll
    for (int n = 0; n < QB; ++n) {
        m[n] = kNone;
        l[n] = 0.0f;
    }
    bool any = false;
#pragma unroll
    for (int n = 0; n < QB; ++n) any = any || at[n].there;
    const bool busy = __ballot(any) != 0;            // (waves without queries only bring tiles)
    int tile = walk.begin(spans, my_groups, split * share, end_tile);
    // One tile: the products of what is `here`, while the next one comes to `there`
    auto step = [&](lds_char *__restrict here_tile, lds_char *__restrict there_tile, int buffer) {
        int *const codes = all_codes + buffer * KT, *const groups = all_groups + buffer * KT;
        float *const staged = all_staged + buffer * Staging::kRoom;
        if ((int)threadIdx.x < KT) {
            codes[threadIdx.x] = next_code;
            groups[threadIdx.x] = next_group;
        }
        next_bias.template put<false>(a, bias, staged, nullptr, a.pack);
        const int form = __builtin_amdgcn_readfirstlane(next_bias.form), low = __builtin_amdgcn_readfirstlane(next_bias.low);
        float one[QB];
        int own[QB];                     // where the biases of the row's head are staged, from its code on
#pragma unroll
        for (int n = 0; n < QB; ++n) {
            one[n] = next_one[n];
            own[n] = (at[n].h - unit * a.pack) * next_bias.count + at[n].code - low;
        }
        const bool apart = next_apart;
        arrive();
        bring.tail(here_tile, a.width);
        const int k0 = tile * KT;
        tile = walk.next(tile);
        if constexpr (STAGES == 2) ask(tile, there_tile);
        if (!busy) return;
        // 32 keys at a time: their scores and pieces are as many registers as there is room for beside the sums
        const int here = fresh_lane(lane);
#pragma unroll 1
        for (int c = 0; c < KT / 32; ++c) {
            Block16<T> acc[2][QB];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const V8<T> f = R::along(here_tile, c, u, s, here);
#pragma unroll
                    for (int n = 0; n < QB; ++n) acc[u][n].mac(f, qf[n][s]);
                }
            const Settled settled;
            float z[QB][8], top[QB];
#pragma unroll
            for (int n = 0; n < QB; ++n) top[n] = kNone;
            by_form(form, k0 + KT > few || apart, [&](auto how) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int row0 = R::row_of(c, u, g);
                    i4 kc = i4(0), kgr = i4(0);
                    if constexpr (how.kForm != kOne) kc = *reinterpret_cast<const i4 *>(codes + row0);
                    if constexpr (how.kMasked) kgr = *reinterpret_cast<const i4 *>(groups + row0);
#pragma unroll
                    for (int n = 0; n < QB; ++n) {
                        const f4 s = acc[u][n].read(settled);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float add = one[n];
                            if constexpr (how.kForm == kStaged) {
                                const unsigned at_code = (unsigned)(own[n] - kc[i]), last = Staging::kRoom - 1;
                                add = staged[at_code < last ? at_code : last];
                            } else if constexpr (how.kForm == kFar) {
                                const unsigned at_code = (unsigned)(at[n].code - kc[i]), last = (unsigned)a.codes - 1u;
                                add = a.tables ? bias[(long)(at[n].h - unit * a.pack) * a.codes + (at_code < last ? at_code : last)] : 0.0f;
                            }
                            float x = __builtin_fmaf(s[i], a.scale, add);
                            if constexpr (how.kMasked) x = (k0 + row0 + i > at[n].last) | (kgr[i] != at[n].group) ? kNone : x;
                            z[n][u * 4 + i] = x;
                            top[n] = __builtin_fmaxf(top[n], x);
                        }
                    }
                }
            });
            Pieces<T> p[QB];
#pragma unroll
            for (int n = 0; n < QB; ++n) {
                top[n] = __builtin_fmaxf(top[n], __shfl_xor(top[n], 16));
                top[n] = __builtin_fmaxf(top[n], __shfl_xor(top[n], 32));
                const float now = __builtin_fmaxf(m[n], top[n]), base = now == kNone ? 0.0f : now;
                if (__ballot(now > m[n])) {
                    const float by = two_to(m[n] - base);
                    l[n] *= by;
#pragma unroll
                    for (int d = 0; d < DB; ++d) o[d][n].scale(settled, by);
                }
                m[n] = now;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const float e = shifted<T>(z[n][i] - base), f = shifted<T>(z[n][i + 1] - base);
                    sum += e;
                    sum += f;
                    p[n].set(i, e, f);
                }
                l[n] += sum;
            }
            if constexpr (kFresh<T>) {
#pragma unroll
                for (int d = 0; d < DB; d += 2) {
                    Block16<T> part[2][QB];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const V8<T> f = R::across(here_tile + R::kBytes, c, (d + x) * 16, here);
#pragma unroll
                        for (int n = 0; n < QB; ++n) p[n].mac(part[x][n], f);
                    }
                    const Settled summed;
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int n = 0; n < QB; ++n) o[d + x][n].add(summed, part[x][n]);
                }
            } else {
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const V8<T> f = R::across(here_tile + R::kBytes, c, d * 16, here);
#pragma unroll
                    for (int n = 0; n < QB; ++n) p[n].mac(o[d][n], f);
                }
            }
        }
    };
    lds_char *const lds = (lds_char *)tiles;
    if constexpr (STAGES == 2) ask(tile, lds);
    int buffer = 0;
    while (tile < end_tile) {
        if constexpr (STAGES == 2) {
            step(lds + buffer * 2 * R::kBytes, lds + (1 - buffer) * 2 * R::kBytes, buffer);
            buffer = 1 - buffer;
        } else {
            __syncthreads();
            ask(tile, lds);
            step(lds, lds, 0);
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
        const long place = ((long)b * a.heads + h) * a.queries + i;
        if (a.splits > 1) {
            float *const part = a.part_o + ((long)split * a.all_rows + place) * a.width;
#pragma unroll
            for (int d = 0; d < DB; ++d) four(part, d * 16 + g * 4, a.width, o[d][n].read(settled));
            if (g == 0) {
                a.part_ml[2 * ((long)split * a.all_rows + place)] = m[n];
                a.part_ml[2 * ((long)split * a.all_rows + place) + 1] = l[n];
            }
            continue;
        }
        const float by = 1.0f / l[n];
        T *const to = static_cast<T *>(a.o) + b * a.p_o.batch + h * a.p_o.head + i * a.p_o.row;
        T *const rest = a.rest ? static_cast<T *>(a.rest) + b * a.p_o.batch + h * a.p_o.head + i * a.p_o.row : nullptr;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            f4 x = o[d][n].read(settled);
            f4 left;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = as_it_is<T>(l[n] == 0.0f ? 0.0f : x[j] * by);
                left[j] = (x[j] - (float)(T)x[j]) * kFiner<T>;
            }
            four(to, d * 16 + g * 4, a.width, x);
            if (rest) four(rest, d * 16 + g * 4, a.width, left);
        }
        if (g == 0 && a.stats) {
            a.stats[2 * place] = l[n] == 0.0f ? 0.0f : m[n];
            a.stats[2 * place + 1] = l[n] == 0.0f ? __builtin_inff() : __builtin_log2f(l[n]) - kShift<T>;
        }
    }
}

// The splits' results joined: a workgroup to a row, sixteen lanes to its elements and sixteen runs of splits, whose sums are added in their order.  Few rows and up to 128 splits, so what
// counts is how many loads are on their way (256 rows x 32 splits 5 us; sixteen lanes to a row 11).
template <class T>
__global__ void __launch_bounds__(256)
hot_attention_join_kernel(AttentionArgs a)
{
    __shared__ float sums[16][16 * 8 + 1], totals[16], tops[16];
    const int t = (int)threadIdx.x & 15, run = (int)threadIdx.x >> 4;
    for (long row = blockIdx.x; row < a.all_rows; row += gridDim.x) {
        const int i = (int)(row % a.queries), h = (int)(row / a.queries % a.heads), b = (int)(row / a.queries / a.heads);
        float m = kNone;
        for (int s = run; s < a.splits; s += 16) m = __builtin_fmaxf(m, a.part_ml[2 * ((long)s * a.all_rows + row)]);
        if (t == 0) tops[run] = m;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k) m = __builtin_fmaxf(m, tops[k]);
        const float base = m == kNone ? 0.0f : m;
        float l = 0.0f, o[8] = {};
#pragma unroll 4
        for (int s = run; s < a.splits; s += 16) {
            const long at = (long)s * a.all_rows + row;
            const float by = two_to(a.part_ml[2 * at] - base);
            l = __builtin_fmaf(a.part_ml[2 * at + 1], by, l);
            const V8<float> v = eight(a.part_o + at * a.width, t * 8, a.width, true);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = __builtin_fmaf(v[j], by, o[j]);
        }
        if (t == 0) totals[run] = l;
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[run][t * 8 + j] = o[j];
        __syncthreads();
        if ((int)threadIdx.x < a.width) {
            l = 0.0f;
            float x = 0.0f;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                l += totals[k];
                x += sums[k][threadIdx.x];
            }
            x = as_it_is<T>(l == 0.0f ? 0.0f : x / l);
            const long to = b * a.p_o.batch + h * a.p_o.head + i * a.p_o.row + (long)threadIdx.x;
            static_cast<T *>(a.o)[to] = (T)x;
            if (a.rest) static_cast<T *>(a.rest)[to] = (T)((x - (float)(T)x) * kFiner<T>);
            if (threadIdx.x == 0 && a.stats) {
                a.stats[2 * row] = l == 0.0f ? 0.0f : m;
                a.stats[2 * row + 1] = l == 0.0f ? __builtin_inff() : __builtin_log2f(l) - kShift<T>;
            }
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------
// D of every query, sixteen lanes to a row; for fp16 also the largest |do_i|^2 of every head and the largest |v_j|^2 of every key head (kPrepareRows rows to a workgroup, so
// that few of them meet at one address).  Bound by memory and its latency: 16 x 8192 rows of 128 bf16 18 us, 5.6 TB/s with what the caches still hold; four rows to a quarter of a wave,
// two of them on their way (eight rows one after the other, places by divisions of 64 bits: 18 us, and where there are few rows 22 instead of 16).
constexpr int kPrepareRows = 64;

template <class T>
__global__ void __launch_bounds__(256)
hot_attention_prepare_kernel(AttentionArgs a)
{
    constexpr bool BOUNDS = __is_same(T, _Float16);
    __shared__ float most[16];
    const int t = (int)threadIdx.x & 15, lane_row = (int)threadIdx.x >> 4;
    const unsigned rows = (unsigned)a.all_rows, all = rows + (BOUNDS ? (unsigned)((long)a.batch * a.kv_heads * a.keys) : 0u);      // (each less than 2^31)
    const unsigned step = gridDim.x * kPrepareRows;
    for (unsigned first = blockIdx.x * kPrepareRows; first < all; first = all - first > step ? first + step : all) {
        // whose maximum row `r` goes to
        auto owner = [&](unsigned r) { return r < rows ? (long)(r / (unsigned)a.queries) : (long)a.batch * a.heads + (r - rows) / (unsigned)a.keys; };
        const unsigned end = all - first > kPrepareRows ? first + kPrepareRows : all;
        const bool alone = BOUNDS && owner(first) == owner(end - 1);
        float largest = 0.0f;
#pragma unroll 2
        for (unsigned row = first + lane_row; row < end; row += 16) {
            float sum = 0.0f, square = 0.0f;
            if (row < rows) {
                const unsigned of = row / (unsigned)a.queries;
                const int i = (int)(row - of * (unsigned)a.queries), h = (int)(of % (unsigned)a.heads), b = (int)(of / (unsigned)a.heads);
                const bool there = !a.groups || a.query_groups[(long)(b % a.groups) * a.queries + i] >= 0;
                const long o_at = b * a.p_o.batch + h * a.p_o.head + i * a.p_o.row;
                const V8<T> up = eight(static_cast<const T *>(a.grad_o) + b * a.p_go.batch + h * a.p_go.head + i * a.p_go.row, t * 8, a.width, there);
                const V8<T> o = eight(static_cast<const T *>(a.o) + o_at, t * 8, a.width, there);
                V8<T> rest = (V8<T>)((T)0.0f);
                if (a.rest) rest = eight(static_cast<const T *>(a.rest) + o_at, t * 8, a.width, there);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sum = __builtin_fmaf((float)up[j], __builtin_fmaf((float)rest[j], 1.0f / kFiner<T>, (float)o[j]), sum);
                    square = __builtin_fmaf((float)up[j], (float)up[j], square);
                }
            } else if constexpr (BOUNDS) {
                const unsigned at = row - rows, of = at / (unsigned)a.keys;
                const int j0 = (int)(at - of * (unsigned)a.keys), h = (int)(of % (unsigned)a.kv_heads), b = (int)(of / (unsigned)a.kv_heads);
                const bool there = !a.groups || a.key_groups[(long)(b % a.groups) * a.keys + j0] >= 0;
                const V8<T> v = eight(static_cast<const T *>(a.v) + b * a.p_v.batch + h * a.p_v.head + j0 * a.p_v.row, t * 8, a.width, there);
#pragma unroll
                for (int j = 0; j < 8; ++j) square = __builtin_fmaf((float)v[j], (float)v[j], square);
            }
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) {
                sum += __shfl_xor(sum, off);
                if constexpr (BOUNDS) square += __shfl_xor(square, off);
            }
            if (t == 0 && row < rows) a.d[row] = sum;
            // (positive floats are ordered as their bits are, and the largest does not depend on the order; nan and infinity are left out)
            if constexpr (BOUNDS) {
                if (!(square < 3.0e38f)) square = 0.0f;
                if (alone) largest = __builtin_fmaxf(largest, square);
                else if (t == 0) atomicMax(a.bounds + owner(row), __builtin_bit_cast(unsigned, square));
            }
        }
        if constexpr (BOUNDS) {
            if (t == 0) most[lane_row] = largest;
            __syncthreads();
            if (threadIdx.x == 0 && alone) {
                for (int i = 1; i < 16; ++i) largest = __builtin_fmaxf(largest, most[i]);
                atomicMax(a.bounds + owner(first), __builtin_bit_cast(unsigned, largest));
            }
            __syncthreads();
        }
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
// dk and dv: a wave holds KB blocks of sixteen keys, and their k and v as operands; the queries of the heads that read them go by in LDS.  Where that gives too few
// workgroups, the heads and runs of queries are split and the parts are added in their order (hot_attention_sum_kernel).
// z and dp, then dv and dk with two pieces of p and dz: six products, of which 16 heads x 8192 tokens x 128 bf16 in causal order do 0.83 TFLOP in 1.17 ms, 58 % of what a large product
// reaches (pieces one at a time: 1.25).  Two waves to a unit's quarter and 32 queries in registers at a time; with KB = 2 (half of the reading of LDS) registers are spilled or one wave is left: 2.1 ms where this was 1.25;
// eight waves to a tile 1.31, six and a third wave to a quarter 2.3.
template <class T, int DP, int KB, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 2)
hot_attention_keys_kernel(AttentionArgs a)
{
    constexpr int THREADS = 64 * WAVES, KS = DP / 32, DB = DP / 16, TILE = WAVES * KB * 16, QT = 64;
    typedef Rows<T, DP, QT> R;
    typedef Bring<T, DP, QT, WAVES> B;
    constexpr int STAGES = kStages<T>;
    typedef Bias<THREADS, THREADS < 256 ? 256 : (sizeof(T) == 2 && DP > 64 ? 384 : 640)> Staging;
    __shared__ __attribute__((aligned(1024))) char tiles[STAGES * 2 * R::kBytes];
    __shared__ __attribute__((aligned(16))) float all_ms[STAGES * QT], all_ls[STAGES * QT], all_ds[STAGES * QT];
    __shared__ __attribute__((aligned(16))) int all_codes[STAGES * QT], all_groups[STAGES * QT];
    __shared__ float all_staged[STAGES * Staging::kRoom];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
    const int tiles_q = (a.queries + QT - 1) / QT, past = a.keys - a.queries, reach = a.causal ? past : 0x7FFFFF00;        // (added to less than 256)

    long item = item_of(a.items);
    if (item < 0) return;
    const int split = (int)(item % a.splits);
    item /= a.splits;
    const int kvh = (int)(item % a.kv_heads);
    item /= a.kv_heads;
    const int b = (int)(item % a.batch), tile_k = (int)(item / a.batch), table = a.tables ? b / a.entries : 0;
    // one head of the key head's, or all; a run of its queries
    const int runs = a.by_head ? a.splits / a.per : a.splits, run = a.by_head ? split / a.per : split;
    const int first_h = kvh * a.per + (a.by_head ? split % a.per : 0), end_h = a.by_head ? first_h + 1 : first_h + a.per;
    const T *const k = static_cast<const T *>(a.k) + b * a.p_k.batch + kvh * a.p_k.head;
    const T *const v = static_cast<const T *>(a.v) + b * a.p_v.batch + kvh * a.p_v.head;
    const int *const kg = a.groups ? a.key_groups + (long)(b % a.groups) * a.keys : nullptr;
    const int *const qg = a.groups ? a.query_groups + (long)(b % a.groups) * a.queries : nullptr;

    int key[KB], code[KB], group[KB];
    V8<T> kf[KB][KS], vf[KB][KS];
#pragma unroll
    for (int n = 0; n < KB; ++n) {
        key[n] = tile_k * TILE + (wave * KB + n) * 16 + col;
        const bool in = key[n] < a.keys;
        const int j = in ? key[n] : a.keys - 1;
        code[n] = a.tables ? a.key_code[j] : 0;
        group[n] = kg ? kg[j] : 0;
        if (!in) group[n] = -1;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            kf[n][s] = eight(k + j * a.p_k.row, s * 32 + g * 8, a.width, group[n] >= 0);
            vf[n][s] = eight(v + j * a.p_v.row, s * 32 + g * 8, a.width, group[n] >= 0);
        }
    }
    const int last_key = (tile_k + 1) * TILE < a.keys ? (tile_k + 1) * TILE - 1 : a.keys - 1;
    bool line = false;
    const int2 key_codes = a.tables ? codes_over(a.key_range, tile_k * TILE, last_key, line) : int2{0, 0};
    const int4 *const spans = a.groups ? a.query_spans + (long)(b % a.groups) * tiles_q : nullptr;
    const int4 my_groups = a.groups ? span_over(a.key_spans + (long)(b % a.groups) * ((a.keys + 63) >> 6), tile_k * TILE, last_key) : int4{0, 0, 0, 0};
    bool next_apart = false;             // whether groups keep some pairs of the next tile apart
    bool any = false;
#pragma unroll
    for (int n = 0; n < KB; ++n) any = any || group[n] >= 0;
    const bool busy = __ballot(any) != 0;                // (waves without keys only bring tiles)
    Block16<T> dk[DB][KB], dv[DB][KB];
    const float unit = unit_of<T>(a, b, kvh * a.per, a.per);
    // from the first query that sees a key of this tile on
    const int first = a.causal && tile_k * TILE > past ? (tile_k * TILE - past) / QT : 0, left = tiles_q > first ? tiles_q - first : 0, share = (left + runs - 1) / runs;
    const int first_tile = first + run * share, end_tile = first_tile + share < tiles_q ? first_tile + share : tiles_q;

    B bring;
    bring.begin(a.p_q.row, a.p_go.row, a.width);
    lds_char *const lds = (lds_char *)tiles;
    for (int h = first_h; h < end_h; ++h) {
        const T *const q = static_cast<const T *>(a.q) + b * a.p_q.batch + h * a.p_q.head;
        const T *const up = static_cast<const T *>(a.grad_o) + b * a.p_go.batch + h * a.p_go.head;
        const float *const bias = a.bias + ((long)table * a.heads + h) * a.codes;
        const long stat0 = ((long)b * a.heads + h) * a.queries;
        Walk<QT> walk;
        Staging next_bias;
        float next_m = 0.0f, next_l = 0.0f, next_d = 0.0f;
        int next_code = 0, next_group = 0;
        auto ask = [&](int tile, lds_char *to) {
            if (tile >= end_tile) return;
            const int last = a.queries - 1 - tile * QT;
            const int4 span = a.groups ? alike(spans + tile) : int4{0, 0, 0, 0};
            next_apart = a.groups && !together(span, my_groups);
            bring.ask(q + (long)tile * QT * a.p_q.row, a.p_q.row, up + (long)tile * QT * a.p_go.row, a.p_go.row, a.width, last, span.z ? qg + tile * QT : nullptr, to);
            if ((int)threadIdx.x < QT) {
                const int i = tile * QT + ((int)threadIdx.x < last ? (int)threadIdx.x : last);
                next_m = a.stats[2 * (stat0 + i)];
                next_l = a.stats[2 * (stat0 + i) + 1];
                next_d = a.d[stat0 + i];
                next_code = a.tables ? a.query_code[i] : 0;
                next_group = qg ? qg[i] : 0;
                if ((int)threadIdx.x > last) {
                    next_l = __builtin_inff();
                    next_group = -2;
                }
            }
            next_bias.template ask<false>(a, bias, query_codes(a, tile * QT, tile * QT + (last < QT - 1 ? last : QT - 1), line), key_codes, 1);
        };
        int tile = walk.begin(spans, my_groups, first_tile, end_tile);
        // One tile: the products of what is `here`, while the next one comes to `there`
        auto step = [&](lds_char *__restrict here, lds_char *__restrict there, int buffer) {
            int *const codes = all_codes + buffer * QT, *const groups = all_groups + buffer * QT;
            float *const ms = all_ms + buffer * QT, *const ls = all_ls + buffer * QT, *const ds = all_ds + buffer * QT, *const staged = all_staged + buffer * Staging::kRoom;
            if ((int)threadIdx.x < QT) {
                ms[threadIdx.x] = next_m;
                ls[threadIdx.x] = next_l - kShift<T>;
                ds[threadIdx.x] = next_d;
                codes[threadIdx.x] = next_code;
                groups[threadIdx.x] = next_group;
            }
            next_bias.template put<false>(a, bias, staged, nullptr, 1);
            const int form = __builtin_amdgcn_readfirstlane(next_bias.form), low = __builtin_amdgcn_readfirstlane(next_bias.low);
            const float one = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, next_bias.one)));
            const bool apart = next_apart;
            arrive();
            bring.tail(here, a.width);
            const int i0 = tile * QT;
            tile = walk.next(tile);
            if constexpr (STAGES == 2) ask(tile, there);
            if (!busy) return;
            // (queries behind the last have l = infinity, keys behind the last are zeros and are not stored)
            const bool masked = apart || (a.causal && i0 + past < last_key);
            const int at = fresh_lane(lane);
#pragma unroll 1
            for (int c = 0; c < QT / 32; ++c) {
                Block16<T> s[2][KB], dp[2][KB];
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int x = 0; x < KS; ++x) {
                        const V8<T> fq = R::along(here, c, u, x, at), fu = R::along(here + R::kBytes, c, u, x, at);
#pragma unroll
                        for (int n = 0; n < KB; ++n) {
                            s[u][n].mac(fq, kf[n][x]);
                            dp[u][n].mac(fu, vf[n][x]);
                        }
                    }
                const Settled settled;
                Pieces<T> p[KB], dz[KB];
                by_form(form, masked, [&](auto how) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int row0 = R::row_of(c, u, g);
                        const f4 m = *reinterpret_cast<const f4 *>(ms + row0), l = *reinterpret_cast<const f4 *>(ls + row0), d = *reinterpret_cast<const f4 *>(ds + row0);
                        i4 qc = i4(0), qgr = i4(0);
                        if constexpr (how.kForm != kOne) qc = *reinterpret_cast<const i4 *>(codes + row0);
                        if constexpr (how.kMasked) qgr = *reinterpret_cast<const i4 *>(groups + row0);
#pragma unroll
                        for (int n = 0; n < KB; ++n) {
                            const f4 zs = s[u][n].read(settled), dps = dp[u][n].read(settled);
                            float es[4], ws[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float add = one;
                                if constexpr (how.kForm == kStaged) {
                                    const unsigned at_code = (unsigned)(qc[i] - (code[n] + low)), last = Staging::kRoom - 1;
                                    add = staged[at_code < last ? at_code : last];
                                } else if constexpr (how.kForm == kFar) {
                                    const unsigned at_code = (unsigned)(qc[i] - code[n]), last = (unsigned)a.codes - 1u;
                                    add = bias[at_code < last ? at_code : last];
                                }
                                float e = two_to(__builtin_fmaf(zs[i], a.scale, add) - m[i] - l[i]);
                                float w = e * ((dps[i] - d[i]) * (unit * (__is_same(T, _Float16) ? 0x1p-14f : 1.0f)));
                                if constexpr (how.kMasked)
                                    if ((group[n] != qgr[i]) | (key[n] - i0 > row0 + i + reach)) e = w = 0.0f;
                                es[i] = e;
                                ws[i] = w;
                            }
#pragma unroll
                            for (int i = 0; i < 4; i += 2) {
                                p[n].set(u * 4 + i, es[i], es[i + 1]);
                                dz[n].set(u * 4 + i, ws[i], ws[i + 1]);
                            }
                        }
                    }
                });
#pragma unroll
                for (int x = 0; x < DB; ++x) {
                    const V8<T> fu = R::across(here + R::kBytes, c, x * 16, at), fq = R::across(here, c, x * 16, at);
                    if constexpr (kFresh<T>) {
                        Block16<T> part_v[KB], part_k[KB];
#pragma unroll
                        for (int n = 0; n < KB; ++n) {
                            p[n].mac(part_v[n], fu);
                            dz[n].mac(part_k[n], fq);
                        }
                        const Settled summed;
#pragma unroll
                        for (int n = 0; n < KB; ++n) {
                            dv[x][n].add(summed, part_v[n]);
                            dk[x][n].add(summed, part_k[n]);
                        }
                    } else {
#pragma unroll
                        for (int n = 0; n < KB; ++n) {
                            p[n].mac(dv[x][n], fu);
                            dz[n].mac(dk[x][n], fq);
                        }
                    }
                }
            }
        };
        // (the waves have done with the last head's tiles)
        __syncthreads();
        if constexpr (STAGES == 2) ask(tile, lds);
        int buffer = 0;
        while (tile < end_tile) {
            if constexpr (STAGES == 2) {
                step(lds + buffer * 2 * R::kBytes, lds + (1 - buffer) * 2 * R::kBytes, buffer);
                buffer = 1 - buffer;
            } else {
                __syncthreads();
                ask(tile, lds);
                step(lds, lds, 0);
            }
        }
    }
    const Settled settled;
    const float by_k = a.plain_scale / unit, by_v = __is_same(T, _Float16) ? 0x1p-14f : 1.0f;
#pragma unroll
    for (int n = 0; n < KB; ++n) {
        if (key[n] >= a.keys) continue;
        if (a.splits > 1) {
            const long at = ((((long)split * a.batch + b) * a.kv_heads + kvh) * a.keys + key[n]) * a.width;
#pragma unroll
            for (int x = 0; x < DB; ++x) {
                if (a.grad_k) four(a.part_k + at, x * 16 + g * 4, a.width, dk[x][n].read(settled) * by_k);
                if (a.grad_v) four(a.part_v + at, x * 16 + g * 4, a.width, dv[x][n].read(settled) * by_v);
            }
            continue;
        }
        T *const to_k = a.grad_k ? static_cast<T *>(a.grad_k) + b * a.p_gk.batch + kvh * a.p_gk.head + key[n] * a.p_gk.row : nullptr;
        T *const to_v = a.grad_v ? static_cast<T *>(a.grad_v) + b * a.p_gv.batch + kvh * a.p_gv.head + key[n] * a.p_gv.row : nullptr;
#pragma unroll
        for (int x = 0; x < DB; ++x) {
            if (to_k) four(to_k, x * 16 + g * 4, a.width, dk[x][n].read(settled) * by_k);
            if (to_v) four(to_v, x * 16 + g * 4, a.width, dv[x][n].read(settled) * by_v);
        }
    }
}

// Parts of gradients of rows of `count` tokens and `heads` heads an entry added up in their order, sixteen lanes to a row (dk and dv of 8192 x 4 rows x 128 in four parts: 151 MB in 23 us)
struct SumArgs {
    const float *parts;
    void *to;
    hot_pitch pitch;
    int splits, count, heads, width;
    long rows;
};

template <class T>
__global__ void __launch_bounds__(256)
hot_attention_sum_kernel(SumArgs first, SumArgs second)
{
    const SumArgs a = blockIdx.y ? second : first;
    if (!a.to) return;
    const int t = (int)threadIdx.x & 15;
    for (long row = (long)blockIdx.x * 16 + ((int)threadIdx.x >> 4); row < a.rows; row += (long)gridDim.x * 16) {
        const int i = (int)(row % a.count), h = (int)(row / a.count % a.heads), b = (int)(row / a.count / a.heads);
        float o[8] = {};
#pragma unroll 4
        for (int s = 0; s < a.splits; ++s) {
            const V8<float> v = eight(a.parts + ((long)s * a.rows + row) * a.width, t * 8, a.width, true);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] += v[j];
        }
        T *const to = static_cast<T *>(a.to) + b * a.pitch.batch + h * a.pitch.head + i * a.pitch.row;
#pragma unroll
        for (int c = 0; c < 2; ++c) four(to, t * 8 + c * 4, a.width, f4{o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]});
    }
}

// same_row += sum over e >= E of v[e] of lane L + e of this lane's sixteen, next_row += that of lane L + e - 16
template <int E>
__device__ __forceinline__ void sum_along(const float (&v)[8], float &same_row, float &next_row)
{
    const int bits = __builtin_bit_cast(int, v[E]);
    same_row += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, bits, 0x100 | E, 0xF, 0xF, true));
    next_row += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, bits, 0x110 | (16 - E), 0xF, 0xF, true));
    if constexpr (E < 7) sum_along<E + 1>(v, same_row, next_row);
}

// ---------------------------------------------------------------------------------
// dq, and what the table's gradient is made of.  A workgroup holds the queries of one tile and head, of several entries of the batch one after the other.  Where a tile of
// pairs is of one bucket its dz are added up in registers (in 64 bits from tile to tile); else each goes to its difference of codes in bins of the wave's own, and from
// there to the wave's sums of the buckets.  No two waves add to one place, and LDS works a wave's additions in the order that they are issued in.
// Four products (z, dp, dz's two pieces times k): 16 heads x 8192 tokens x 128 bf16 in causal order 0.76 ms, 59 % of the rate of a large product; a block of sixteen queries to a wave
// where there are no more than 64 of them, else two (one at 8192 tokens: 1.10 ms where this was 0.80).  Of the sums over one distance each, lines of a tile are summed along lanes first: LDS's own
// additions of floats take some 270 cycles an instruction.
template <class T, int DP, int QB, int WAVES, bool TABLE>
__global__ void __launch_bounds__(64 * WAVES, 2)
hot_attention_queries_kernel(AttentionArgs a)
{
    constexpr int THREADS = 64 * WAVES, KS = DP / 32, DB = DP / 16, KT = 64, TILE = WAVES * QB * 16;
    typedef Rows<T, DP, KT> R;
    typedef Bring<T, DP, KT, WAVES> B;
    constexpr int STAGES = kStages<T>;
    typedef Bias<THREADS, THREADS < 256 ? 256 : (sizeof(T) == 2 && DP > 64 ? 384 : 640)> Staging;
    constexpr int BINS = TABLE ? Staging::kRoom : 1;
    __shared__ __attribute__((aligned(1024))) char tiles[STAGES * 2 * R::kBytes];
    __shared__ __attribute__((aligned(16))) int all_codes[STAGES * KT], all_groups[STAGES * KT];
    __shared__ float all_staged[STAGES * (Staging::kRoom + 64)];          // (the last 64, and those of the bins, are for pairs that do not count: a place for each lane)
    __shared__ unsigned short all_staged_bucket[STAGES * BINS];
    __shared__ float all_bins[WAVES * (BINS + 64)];
    extern __shared__ float all_sums[];          // [waves, buckets]
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
    float *const bins = all_bins + wave * (BINS + 64), *const sums = all_sums + wave * a.buckets;
    if constexpr (TABLE)
        for (int i = lane; i < BINS + 64; i += 64) bins[i] = 0.0f;
    for (int i = 0; i < STAGES; ++i) all_staged[i * (Staging::kRoom + 64) + Staging::kRoom + lane] = 0.0f;
    auto add = [](float *to, float x) { __hip_atomic_fetch_add(to, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT); };

    long item = item_of(a.items);
    if (item < 0) return;
    const int chunks = (int)(a.items / ((long)a.splits * a.tiles_q * a.heads)), split = (int)(item % a.splits);
    item /= a.splits;
    const int h = (int)(item % a.heads), kvh = h / a.per;
    item /= a.heads;
    const int chunk = (int)(item % chunks), tile_q = a.tiles_q - 1 - (int)(item / chunks);
    const int per_table = (a.entries + a.chunk - 1) / a.chunk, table = chunk / per_table;
    const int first_b = table * a.entries + chunk % per_table * a.chunk;
    const int end_b = first_b + a.chunk < (table + 1) * a.entries ? first_b + a.chunk : (table + 1) * a.entries;
    const float *const bias = a.bias + ((long)table * a.heads + h) * a.codes;
    const int end_row = (tile_q + 1) * TILE < a.queries ? (tile_q + 1) * TILE : a.queries, first_i = tile_q * TILE, last_i = end_row - 1;
    int visible = a.causal ? last_i + (a.keys - a.queries) + 1 : a.keys, few = a.causal ? first_i + (a.keys - a.queries) + 1 : a.keys;
    visible = visible < 0 ? 0 : (visible > a.keys ? a.keys : visible);
    if (few > a.keys) few = a.keys;
    const int all_tiles = (visible + KT - 1) / KT, share = (all_tiles + a.splits - 1) / a.splits;
    const int end_tile = (split + 1) * share < all_tiles ? (split + 1) * share : all_tiles;
    bool line = false;               // whether the queries' codes go up by one
    const int2 mine_codes = query_codes(a, first_i, last_i, line);
    const int line_code = TABLE ? a.query_code[first_i] : 0;
    double same = 0.0;               // this lane's part of the sum of bucket `same_bucket`
    int same_bucket = -1;
    auto flush = [&]() {
        if (same_bucket < 0) return;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) same += __shfl_xor(same, off);
        if (lane == 0) add(sums + same_bucket, (float)same);
        same = 0.0;
    };
    if constexpr (TABLE)
        for (int i = lane; i < a.buckets; i += 64) sums[i] = 0.0f;
    B bring;
    bring.begin(a.p_k.row, a.p_v.row, a.width);
    lds_char *const lds = (lds_char *)tiles;
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
        int code_low = kMostCode, code_high = -1;             // of this wave's queries
#pragma unroll
        for (int n = 0; n < QB; ++n) {
            at[n] = query_of(a, b, h, tile_q * TILE + (wave * QB + n) * 16 + col);
            const long row = ((long)b * a.heads + h) * a.queries + at[n].i;
            m[n] = a.stats[2 * row];
            l[n] = a.stats[2 * row + 1];
            dd[n] = a.d[row];
            if (!at[n].there) {
                m[n] = dd[n] = 0.0f;
                l[n] = __builtin_inff();
                at[n].code = kMostCode;          // (beyond what is staged)
            } else {
                code_low = at[n].code < code_low ? at[n].code : code_low;
                code_high = at[n].code > code_high ? at[n].code : code_high;
            }
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                qf[n][s] = eight(q + at[n].i * a.p_q.row, s * 32 + g * 8, a.width, at[n].there);
                uf[n][s] = eight(up + at[n].i * a.p_go.row, s * 32 + g * 8, a.width, at[n].there);
            }
        }
        if constexpr (TABLE) {
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) {
                const int x = __shfl_xor(code_low, off), y = __shfl_xor(code_high, off);
                code_low = x < code_low ? x : code_low;
                code_high = y > code_high ? y : code_high;
            }
        }
        const int4 *const spans = a.groups ? a.key_spans + (long)(b % a.groups) * ((a.keys + 63) >> 6) : nullptr;
        const int4 my_groups = a.groups ? span_over(a.query_spans + (long)(b % a.groups) * ((a.queries + 63) >> 6), first_i, last_i) : int4{0, 0, 0, 0};
        bool next_apart = false;             // whether groups keep some pairs of the next tile apart
        Walk<KT> walk;
        Staging next_bias;
        int next_code = 0, next_group = 0;
        int2 next_range = int2{0, 0};
        bool next_line = false;
        auto ask = [&](int tile, lds_char *to) {
            if (tile >= end_tile) return;
            const int last = a.keys - 1 - tile * KT;
            const int4 span = a.groups ? alike(spans + (tile * KT >> 6)) : int4{0, 0, 0, 0};
            next_apart = a.groups && !together(span, my_groups);
            bring.ask(k + (long)tile * KT * a.p_k.row, a.p_k.row, v + (long)tile * KT * a.p_v.row, a.p_v.row, a.width, last, span.z ? kg + tile * KT : nullptr, to);
            if ((int)threadIdx.x < KT) {
                const int j = tile * KT + ((int)threadIdx.x < last ? (int)threadIdx.x : last);
                next_code = a.tables ? a.key_code[j] : 0;
                next_group = kg ? kg[j] : 0;
                if ((int)threadIdx.x > last) next_group = -1;
            }
            next_range = a.tables ? codes_over(a.key_range, tile * KT, tile * KT, next_line) : int2{0, 0};
            next_bias.template ask<TABLE>(a, bias, mine_codes, next_range, 1);
        };
        bool any = false;
#pragma unroll
        for (int n = 0; n < QB; ++n) any = any || at[n].there;
        const bool busy = __ballot(any) != 0;            // (waves without queries only bring tiles)
        Block16<T> dq[DB][QB];
        int tile = walk.begin(spans, my_groups, split * share, end_tile);
        // One tile: the products of what is `here`, while the next one comes to `there`
        auto step = [&](lds_char *__restrict here_tile, lds_char *__restrict there_tile, int buffer) {
            int *const codes = all_codes + buffer * KT, *const groups = all_groups + buffer * KT;
            float *const staged = all_staged + buffer * (Staging::kRoom + 64);
            unsigned short *const staged_bucket = all_staged_bucket + buffer * BINS;
            if ((int)threadIdx.x < KT) {
                codes[threadIdx.x] = next_code;
                groups[threadIdx.x] = next_group;
            }
            next_bias.template put<TABLE>(a, bias, staged, staged_bucket, 1);
            const int form = __builtin_amdgcn_readfirstlane(next_bias.form), low = __builtin_amdgcn_readfirstlane(next_bias.low), bucket = __builtin_amdgcn_readfirstlane(next_bias.all);
            const int2 range = next_range;
            const bool lined = TABLE && line && next_line;
            const float one = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, next_bias.one)));
            const bool apart = next_apart;
            arrive();
            bring.tail(here_tile, a.width);
            const int k0 = tile * KT;
            tile = walk.next(tile);
            if constexpr (STAGES == 2) ask(tile, there_tile);
            if (!busy) return;
            const bool masked = k0 + KT > few || apart;
            float here = 0.0f;
#pragma unroll 1
            for (int c = 0; c < KT / 32; ++c) {
                const int own = fresh_lane(lane);
                Block16<T> s[2][QB], dp[2][QB];
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int x = 0; x < KS; ++x) {
                        const V8<T> fk = R::along(here_tile, c, u, x, own), fv = R::along(here_tile + R::kBytes, c, u, x, own);
#pragma unroll
                        for (int n = 0; n < QB; ++n) {
                            s[u][n].mac(fk, qf[n][x]);
                            dp[u][n].mac(fv, uf[n][x]);
                        }
                    }
                const Settled settled;
                Pieces<T> dz[QB];
                const unsigned none = (unsigned)(Staging::kRoom + lane);           // where what is beyond the bins goes
                float counts[TABLE ? QB : 1][8];
                by_form(form, masked, [&](auto how) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int row0 = R::row_of(c, u, g);
                        i4 kc = i4(0), kgr = i4(0);
                        if constexpr (how.kForm != kOne) kc = *reinterpret_cast<const i4 *>(codes + row0);
                        if constexpr (how.kMasked) kgr = *reinterpret_cast<const i4 *>(groups + row0);
#pragma unroll
                        for (int n = 0; n < QB; ++n) {
                            const f4 zs = s[u][n].read(settled), dps = dp[u][n].read(settled);
                            float before = 0.0f;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float bias_here = one;
                                unsigned at_code = 0;
                                const bool sees = !how.kMasked || !((k0 + row0 + i > at[n].last) | (kgr[i] != at[n].group));
                                if constexpr (how.kForm == kStaged) {
                                    at_code = (unsigned)(at[n].code - low - kc[i]);
                                    at_code = at_code < none ? at_code : none;
                                    bias_here = staged[at_code];
                                } else if constexpr (how.kForm == kFar) {
                                    const unsigned last = (unsigned)a.codes - 1u;
                                    at_code = (unsigned)(at[n].code - kc[i]);
                                    at_code = at_code < last ? at_code : last;
                                    bias_here = bias[at_code];
                                }
                                const float e = two_to(__builtin_fmaf(zs[i], a.scale, bias_here) - m[n] - l[n]);
                                float w = e * (dps[i] - dd[n]);
                                if constexpr (how.kMasked) w = sees ? w : 0.0f;
                                if (i & 1) dz[n].set(u * 4 + i - 1, before, w * unit);
                                before = w * unit;
                                if constexpr (TABLE) {
                                    if constexpr (how.kForm == kOne) here += w;
                                    else if constexpr (how.kForm == kStaged) {
                                        counts[n][u * 4 + i] = w;
                                    } else {
                                        const unsigned to = (unsigned)a.bucket[at_code].x, most = (unsigned)a.buckets - 1u;
                                        add(sums + (to < most ? to : most), w);
                                    }
                                }
                            }
                        }
                    }
                    if constexpr (TABLE && how.kForm == kStaged) {
                        const int row0 = R::row_of(c, 0, g);
                        if (lined) {
                            // Queries L of a block and eight neighbouring keys: distance D + L of the first key is that of key e and query L + e, which is a lane of this
                            // block's row or, sixteen distances on, one of the next: two sums over eight lanes each, and the blocks' overlap added up.  Three
                            // additions to LDS where single pairs took sixteen (some 270 cycles each: LDS adds floats one lane after the other).
                            const int from = line_code + wave * QB * 16 + col - low - codes[row0];
                            float carry = 0.0f;
#pragma unroll
                            for (int n = QB - 1; n >= 0; --n) {
                                float same_row = counts[n][0], next_row = 0.0f;
                                sum_along<1>(counts[n], same_row, next_row);
                                const unsigned bin = (unsigned)(from + n * 16);
                                add(bins + (bin < none ? bin : none), same_row + carry);
                                carry = next_row;
                            }
                            const unsigned bin = (unsigned)(from - 16);
                            add(bins + (bin < none ? bin : none), carry);
                        } else {
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                const i4 kc = *reinterpret_cast<const i4 *>(codes + row0 + 4 * u);
#pragma unroll
                                for (int n = 0; n < QB; ++n)
#pragma unroll
                                    for (int i = 0; i < 4; ++i) {
                                        const float w = counts[n][u * 4 + i];
                                        unsigned bin = (unsigned)(at[n].code - low - kc[i]);
                                        bin = w != 0.0f && bin < none ? bin : none;
                                        add(bins + bin, w);
                                    }
                            }
                        }
                    }
                });
#pragma unroll
                for (int x = 0; x < DB; ++x) {
                    const V8<T> f = R::across(here_tile, c, x * 16, own);
#pragma unroll
                    for (int n = 0; n < QB; ++n) dz[n].mac(dq[x][n], f);
                }
            }
            if constexpr (TABLE) {
                if (form == kOne) {
                    if (bucket != same_bucket) {
                        flush();
                        same_bucket = bucket < 0 ? 0 : (bucket < a.buckets ? bucket : a.buckets - 1);
                    }
                    same += (double)here;
                } else if (form == kStaged) {
                    // the bins that this wave's queries reach
                    // (none where the wave has no queries: code_high is -1)
                    int first = code_low - range.y - low, end = code_high - range.x - low + 1;
                    first = first < 0 ? 0 : first;
                    end = code_high < 0 ? 0 : (end < BINS ? end : BINS);
                    for (int i = first + lane; i < end; i += 64) {
                        const float x = bins[i];
                        bins[i] = 0.0f;
                        add(sums + staged_bucket[i], x);
                    }
                }
            }
        };
        if constexpr (STAGES == 2) ask(tile, lds);
        int buffer = 0;
        while (tile < end_tile) {
            if constexpr (STAGES == 2) {
                step(lds + buffer * 2 * R::kBytes, lds + (1 - buffer) * 2 * R::kBytes, buffer);
                buffer = 1 - buffer;
            } else {
                __syncthreads();
                ask(tile, lds);
                step(lds, lds, 0);
            }
        }
        const Settled settled;
        if (a.grad_q)
#pragma unroll
            for (int n = 0; n < QB; ++n) {
                const int row = tile_q * TILE + (wave * QB + n) * 16 + col;
                if (row >= a.queries) continue;
                if (a.splits > 1) {
                    float *const part = a.part_o + ((long)split * a.all_rows + ((long)b * a.heads + h) * a.queries + row) * a.width;
#pragma unroll
                    for (int x = 0; x < DB; ++x) four(part, x * 16 + g * 4, a.width, dq[x][n].read(settled) * (a.plain_scale / unit));
                    continue;
                }
                T *const to = static_cast<T *>(a.grad_q) + b * a.p_gq.batch + h * a.p_gq.head + row * a.p_gq.row;
#pragma unroll
                for (int x = 0; x < DB; ++x) four(to, x * 16 + g * 4, a.width, dq[x][n].read(settled) * (a.plain_scale / unit));
            }
        __syncthreads();
    }
    if constexpr (TABLE) {
        flush();
        __syncthreads();
        float *const to = a.parts + ((((long)chunk * a.heads + h) * a.tiles_q + tile_q) * a.splits + split) * a.buckets;
        for (int i = (int)threadIdx.x; i < a.buckets; i += THREADS) {
            float sum = all_sums[i];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) sum += all_sums[w * a.buckets + i];
            to[i] = sum;
        }
        __syncthreads();
    }
}

// The table's gradient: the workgroups' sums, 64 buckets and 16 runs of workgroups at a time
__global__ void __launch_bounds__(1024)
hot_attention_table_kernel(AttentionArgs a)
{
    __shared__ double runs[16][64];
    const int lane = (int)threadIdx.x & 63, run = (int)threadIdx.x >> 6, h = (int)blockIdx.y, table = (int)blockIdx.z;
    const int col = (int)blockIdx.x * 64 + lane, per_table = (a.entries + a.chunk - 1) / a.chunk, each = a.tiles_q * a.splits;
    double sum = 0.0;
    if (col < a.buckets) {
        const long all = (long)per_table * each;
        for (long u = run; u < all; u += 64) {
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const long w = u + 16 * j < all ? u + 16 * j : u, chunk = (long)table * per_table + w / each;
                v[j] = a.parts[((chunk * a.heads + h) * each + w % each) * a.buckets + col];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) sum += u + 16 * j < all ? (double)v[j] : 0.0;
        }
    }
    runs[run][lane] = sum;
    __syncthreads();
    if (run || col >= a.buckets) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += runs[i][lane];
    store_as(a.grad_table, a.table_type, ((long)table * a.buckets + col) * a.heads + h, (float)sum);
}

// ---------------------------------------------------------------------------------
// Host side: what is launched for one type

inline dim3 blocks_for(long items)
{
    const long most = 1L << 20, up = items;
    return up <= most ? dim3((unsigned)up) : dim3((unsigned)most, (unsigned)((up + most - 1) / most));
}

template <class T, int DP>
void forward_go(const AttentionArgs &a, hipStream_t s)
{
    if (a.shape == 0) hot_attention_forward_kernel<T, DP, 1, 1, 32><<<blocks_for(a.items), 64, 0, s>>>(a);
    else if (a.shape == 1) hot_attention_forward_kernel<T, DP, 1, 4, 64><<<blocks_for(a.items), 256, 0, s>>>(a);
    else if constexpr (DP <= 96 && sizeof(T) == 2) hot_attention_forward_kernel<T, DP, 1, 8, 64><<<blocks_for(a.items), 512, 0, s>>>(a);
    else hot_attention_forward_kernel<T, DP, 2, 4, 64><<<blocks_for(a.items), 256, 0, s>>>(a);
}

template <class T, int DP>
void queries_go(const AttentionArgs &a, hipStream_t s)
{
    const dim3 blocks = blocks_for(a.items);
    if (a.grad_table) {
        if (a.shape == 1) hot_attention_queries_kernel<T, DP, 1, 4, true><<<blocks, 256, 4 * a.buckets * 4, s>>>(a);
        else hot_attention_queries_kernel<T, DP, 2, 4, true><<<blocks, 256, 4 * a.buckets * 4, s>>>(a);
    } else if (a.shape == 1) hot_attention_queries_kernel<T, DP, 1, 4, false><<<blocks, 256, 0, s>>>(a);
    else hot_attention_queries_kernel<T, DP, 2, 4, false><<<blocks, 256, 0, s>>>(a);
}

template <class T, int DP>
void keys_go(const AttentionArgs &a, hipStream_t s)
{
    hot_attention_keys_kernel<T, DP, 1, 4><<<blocks_for(a.items), 256, 0, s>>>(a);
}

template <class T>
void sum_go(const SumArgs &x, const SumArgs &y, hipStream_t s)
{
    const long blocks = (x.rows + 15) / 16;
    hot_attention_sum_kernel<T><<<dim3((unsigned)(blocks < 8192 ? blocks : 8192), y.to ? 2 : 1), 256, 0, s>>>(x, y);
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
    const long n = (long)a.tables * a.heads * a.codes, spans = 64L * a.groups * (((a.queries + 63) >> 6) + ((a.keys + 63) >> 6));
    long all = n > a.bounds_count ? n : a.bounds_count;
    all = all > spans ? all : spans;
    if (!all) return;
    const long blocks = (all + 255) / 256;
    hot_attention_begin_kernel<<<(unsigned)(blocks < 2048 ? blocks : 2048), 256, 0, s>>>(a);
}

template <class T>
void attention_forward(const AttentionArgs &a, hipStream_t s)
{
    HOT_BY_WIDTH(forward_go);
    if (a.splits > 1) {
        hot_attention_join_kernel<T><<<(unsigned)(a.all_rows < 8192 ? a.all_rows : 8192), 256, 0, s>>>(a);
    }
}

template <class T>
void attention_prepare(const AttentionArgs &a, hipStream_t s)
{
    const long blocks = (a.all_rows + (__is_same(T, _Float16) ? (long)a.batch * a.kv_heads * a.keys : 0) + kPrepareRows - 1) / kPrepareRows;
    hot_attention_prepare_kernel<T><<<(unsigned)(blocks < 8192 ? blocks : 8192), 256, 0, s>>>(a);
}

template <class T>
void attention_keys(const AttentionArgs &a, hipStream_t s)
{
    HOT_BY_WIDTH(keys_go);
    if (a.splits > 1) {
        const long rows = (long)a.batch * a.kv_heads * a.keys;
        const SumArgs k = {a.part_k, a.grad_k, a.p_gk, a.splits, a.keys, a.kv_heads, a.width, rows}, v = {a.part_v, a.grad_v, a.p_gv, a.splits, a.keys, a.kv_heads, a.width, rows};
        sum_go<T>(k, v, s);
    }
}

template <class T>
void attention_queries(const AttentionArgs &a, hipStream_t s)
{
    if (a.items) {
        HOT_BY_WIDTH(queries_go);
    }
    if (a.items && a.grad_q && a.splits > 1) {
        const SumArgs q = {a.part_o, a.grad_q, a.p_gq, a.splits, a.queries, a.heads, a.width, a.all_rows};
        sum_go<T>(q, SumArgs{}, s);
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
