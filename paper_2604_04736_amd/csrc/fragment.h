// Blocks of 16 x 16 results of the matrix instruction, for the kernels of attention.h, and their operands out of LDS.
//
// An instruction contracts 32 indices: lane l brings line l % 16 of its operand at indices 8 (l / 16) .. + 7, and receives results (4 (l / 16) + i, l % 16),
// i = 0 .. 3, the second index being B's line.  Two blocks of results thus leave eight rows of one column in a lane, which is the
// form of an operand that contracts those 32 rows, if the other operand takes them in the same order (Rows).  So the softmax's results go from one product into the next without leaving their lanes.
// float32 is multiplied by the instruction of its own, four indices at a time, on the same operands.
#ifndef HOT_FRAGMENT_H
#define HOT_FRAGMENT_H

#include <hip/hip_runtime.h>

#include "vec.h"

namespace {

template <class T>
struct Eight {
    typedef T V __attribute__((ext_vector_type(8)));
};
template <class T>
using V8 = typename Eight<T>::V;

typedef short s4v __attribute__((ext_vector_type(4)));
typedef short s8v __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) s4v lds_s4v;
typedef __attribute__((address_space(3))) f4 lds_f4;

// The wait states between a run of matrix instructions and the first read of their results: 32, which the scheduler may not move
// (the compiler's own can be missing where a branch lies between).  Blocks hand their registers out only against one of these.
struct Settled {
    __device__ __forceinline__ Settled()
    {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    }
    Settled(const Settled &) = delete;
    Settled &operator=(const Settled &) = delete;
};

template <class T>
class Block16 {
    f4 v_;

public:
    __device__ __forceinline__ Block16() : v_(0.0f) {}
    __device__ __forceinline__ void mac(V8<T> a, V8<T> b)
    {
        if constexpr (__is_same(T, float)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v_ = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], v_, 0, 0, 0);
        } else if constexpr (__is_same(T, _Float16)) v_ = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, v_, 0, 0, 0);
        else v_ = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, v_, 0, 0, 0);
    }
    __device__ __forceinline__ f4 read(const Settled &) const { return v_; }
    __device__ __forceinline__ void add(const Settled &, const Block16 &b)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v_[i] += b.v_[i];
    }
    __device__ __forceinline__ void scale(const Settled &, float by)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v_[i] *= by;
    }
};

// x, once.  The compiler joins a product with its rounding to fp16 (one rounding for two), at some of the product's uses and not at others: two pieces of a number
// would then be of different numbers, a step of the first piece apart where that is nearly a tie.
template <class T>
__device__ __forceinline__ float as_it_is(float x)
{
    if constexpr (__is_same(T, _Float16)) asm("" : "+v"(x));
    return x;
}

// Eight results as an operand: as they are for float32, in two pieces for 16-bit types (bf16: 2^-17 of each is left over; fp16: 2^-23, or half a step of 2^-24)
template <class T>
struct Pieces {
    static constexpr int N = __is_same(T, float) ? 1 : 2;
    V8<T> p[N];

    // results i and i + 1, i even: one conversion for both (one at a time, each was converted once more for its second piece)
    __device__ __forceinline__ void set(int i, float x, float y)
    {
        if constexpr (N == 1) {
            p[0][i] = x;
            p[0][i + 1] = y;
        } else {
#pragma clang fp contract(off)     // (of the product's rounding in every form of a kernel, or the forms' results differ in the last place)
            typedef T T2 __attribute__((ext_vector_type(2)));
            typedef float F2 __attribute__((ext_vector_type(2)));
            typedef unsigned U4 __attribute__((ext_vector_type(4)));
            const F2 v = {as_it_is<T>(x), as_it_is<T>(y)};
            const unsigned high = __builtin_bit_cast(unsigned, __builtin_convertvector(v, T2));
            F2 back;
            if constexpr (__is_same(T, _Float16)) back = __builtin_convertvector(__builtin_bit_cast(T2, high), F2);
            else back = F2{__builtin_bit_cast(float, high << 16), __builtin_bit_cast(float, high & 0xffff0000u)};
            const unsigned low = __builtin_bit_cast(unsigned, __builtin_convertvector((F2){v.x - back.x, v.y - back.y}, T2));
            U4 first = __builtin_bit_cast(U4, p[0]), second = __builtin_bit_cast(U4, p[1]);
            first[i / 2] = high;
            second[i / 2] = low;
            p[0] = __builtin_bit_cast(V8<T>, first);
            p[1] = __builtin_bit_cast(V8<T>, second);
        }
    }
    // c += a (the pieces)
    __device__ __forceinline__ void mac(Block16<T> &c, V8<T> a) const
    {
#pragma unroll
        for (int k = N - 1; k >= 0; --k) c.mac(a, p[k]);
    }
};

// A tile of ROWS rows of DP elements in LDS, and the order in which products take its rows: line 4 a + b of block u of sixteen lines (two blocks to 32 rows c) is row
// kSpread a + 8 c + 4 u + b.  A lane thus holds the results of eight neighbouring rows, and the four lanes of one column those of rows kSpread apart, so that
// where rows and columns are tokens of a line, sixty-four lanes have sixty-four different distances.
// LDS serves 256 bytes at once if they are in different banks: sixteen bytes each of the sixteen rows of a block (along), or 32 bytes each of eight rows
// (the transposing read across; float32: 64 bytes of four).  Pieces of sixteen bytes are permuted by the row so that both are.
template <class T, int DP, int ROWS>
struct Rows {
    static constexpr bool kSmall = sizeof(T) == 2;
    static constexpr int kSpread = ROWS / 4;
    static constexpr int kPitch = kSmall ? (DP <= 32 ? 64 : (DP <= 64 ? 128 : 256)) : DP * 4 + 64;
    static constexpr int kBytes = (ROWS * kPitch + (kSmall ? 0 : 4 * 64) + 1023) / 1024 * 1024;         // (whole loads of a wave)

    static __device__ __forceinline__ int row_of(int c, int u, int a) { return kSpread * a + 8 * c + 4 * u; }

    // the byte of element `at` of a row
    static __device__ __forceinline__ int place(int row, int at)
    {
        const int byte = at * (int)sizeof(T), a = row / kSpread & 3;
        if constexpr (!kSmall) return row * kPitch + a * 64 + (byte ^ a << 4);
        else {
            const int high = a >> 1, low = a & 1;
            int turn;
            if constexpr (kPitch == 256) turn = (row & 3) << 1 | low << 3 | high;
            else if constexpr (kPitch == 128) turn = (row & 2) | low << 2 | high;
            else turn = low << 1 | high;
            return row * kPitch + (byte ^ turn << 4);
        }
    }
    // ... and back: which row and element lie at a byte; false for what belongs to none
    static __device__ __forceinline__ bool at_byte(int byte, int &row, int &at)
    {
        if constexpr (kSmall) {
            row = byte / kPitch;
            at = (place(row, 0) - row * kPitch ^ byte % kPitch) / 2;
            return row < ROWS && at < DP;
        } else {
            constexpr int SEGMENT = kSpread * kPitch + 64;
            const int a = byte / SEGMENT, in = byte % SEGMENT, of_row = in % kPitch;
            row = a * kSpread + in / kPitch;
            at = (of_row ^ a << 4) / 4;
            return a < 4 && in < kSpread * kPitch && of_row < DP * 4;
        }
    }
    // operand of the sixteen lines of block u of rows c at elements 32 ks ..
    static __device__ __forceinline__ V8<T> along(const lds_char *tile, int c, int u, int ks, int lane)
    {
        const int row = row_of(c, u, lane >> 2 & 3) + (lane & 3), at = ks * 32 + (lane >> 4) * 8;
        if constexpr (kSmall) return *(const __attribute__((address_space(3))) V8<T> *)(tile + place(row, at));
        else {
            const f4 low = *(const lds_f4 *)(tile + place(row, at)), high = *(const lds_f4 *)(tile + place(row, at + 4));
            return __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    // operand whose lines are elements e0 .. + 15 and whose 32 indices are rows c, in the order of a lane's results of both blocks
    static __device__ __forceinline__ V8<T> across(const lds_char *tile, int c, int e0, int lane)
    {
        const int row = row_of(c, 0, lane >> 4), i = lane & 15;
        if constexpr (kSmall) {
            // (a transposing read: of four rows of sixteen elements that sixteen lanes name, lane i receives element i of each)
            const lds_char *const at = tile + place(row + (i >> 2), e0 + (i & 3) * 4);
            const s4v up = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v *)at);
            const s4v low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v *)(at + 4 * kPitch));
            return __builtin_bit_cast(V8<T>, __builtin_shufflevector(up, low, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            V8<T> v;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = *(const __attribute__((address_space(3))) T *)(tile + place(row, e0 + i) + j * kPitch);
            return v;
        }
    }
};

// The N elements of a vector moved down by `by` (the same for all lanes), zeros behind them
template <int N, class V>
__device__ __forceinline__ V moved_down(V v, int by)
{
#pragma unroll 1
    for (; by > 0; --by) {
#pragma unroll
        for (int j = 0; j + 1 < N; ++j) v[j] = v[j + 1];
        v[N - 1] = 0;
    }
    return v;
}

// Eight neighbouring elements of a row of n >= 8 in memory, zeros behind its end and where `there` is false, on any element's address.  Nothing branches around a
// load: the compiler would wait for each before the next (a row of the tensor is there to be read in any case, what was read is dropped).  Pieces behind
// the row's end are read from where it ends.
template <class T>
__device__ __forceinline__ V8<T> eight(const T *row, int at, int n, bool there)
{
    typedef V8<T> Loose __attribute__((aligned(sizeof(T))));
    V8<T> v;
    v = *reinterpret_cast<const Loose *>(row + (at + 8 <= n ? at : n - 8));
    if (n & 7) {
        const V8<T> low = moved_down<8>(v, 8 - (n & 7));
        if (at + 8 > n) v = low;
    }
    if (!there || at >= n) v = (V8<T>)((T)0.0f);
    return v;
}

// Four results to a row of n elements
template <class T>
__device__ __forceinline__ void four(T *row, int at, int n, f4 v)
{
    typedef T F __attribute__((ext_vector_type(4)));
    typedef F Loose __attribute__((aligned(sizeof(T))));
    if (at + 4 <= n) {
        *reinterpret_cast<Loose *>(row + at) = __builtin_convertvector(v, F);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (at + j < n) row[at + j] = (T)v[j];
}

}  // namespace

#endif  // HOT_FRAGMENT_H
