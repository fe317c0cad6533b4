// libhot: dropout of activations by a counter, and the end of a transformer block fused with the norm that begins the next one:
//
//   t = norm'(branch),  d = dropout(t),  h = x + scale gate d,  y = norm(h)
//
// norm and norm' are layer norms, root-mean-square norms or nothing; gate and the norms' weights and biases are shared by all rows or one set per
// sample.  With n, n' the normalised rows and r, r' what they were multiplied by:
//   du = dh + r (u - n mean(u n) - mean u),  u = dy weight     (mean u: layer norm only)
//   dx = du,  dgate = scale sum du d,  dt = dropout(scale gate du),  dbranch = dt, or the same form of v = dt branch_weight with n' and r'
//   dweight = sum dy n,  dbias = sum dy,  dbranch_weight = sum dt n',  dbranch_bias = sum dt
//
// A mask is never stored: element c of row r of a sample is kept where sixteen bits of the generator (draw.h) at a counter made from (r, c div 8) lie
// below round(65536 keep), so eight elements share one call of it, forward and backward alike.  Sixteen bits, since with a word for each element the
// generator's multiplications, not memory, bound 16-bit types; kept elements are multiplied by 65536 / round(65536 keep), so the mean is right for the
// probability that is used.  The counters' top bit is set, which the draw of weights never does: one seed serves both.
//
// What bounds the kernels is memory.  A row lies in registers between its loads and its stores: eight elements a thread (sixteen beyond 8192), so that
// one call of the generator serves a thread's elements; the next row is on its way meanwhile.  The backward pass forms h again from x and branch
// instead of reading h, which is rounded: the same bytes, and n as exact as the forward pass had it.  The vectors' sums stay in the registers of the
// threads that own the columns; every workgroup leaves one row of them in scratch memory and a second kernel adds these in a fixed order.
#include <hip/hip_runtime.h>

#include "hot.h"
#include "vec.h"
#include "draw.h"
#include "element.h"

// (a product that is rounded here and contracted there would leave u - mean u other than zero where all u are the same)
#pragma clang fp contract(off)

namespace {

constexpr int kBlockThreads = 256;
constexpr int kUnits = 256;                  // compute units
typedef float f8 __attribute__((ext_vector_type(8)));

// Eight neighbouring elements, on any element's address
template <class T>
struct Octet {
    typedef T V __attribute__((ext_vector_type(8)));
    typedef V Loose __attribute__((aligned(sizeof(T))));
    V v;

    __device__ __forceinline__ void take(const T *row, long at, long n)
    {
        if (at + 8 <= n) {
            v = *reinterpret_cast<const Loose *>(row + at);
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = at + j < n ? row[at + j] : (T)0.0f;
    }
    __device__ __forceinline__ f8 floats() const { return __builtin_convertvector(v, f8); }
    static __device__ __forceinline__ void store(T *row, long at, long n, f8 f)
    {
        const V o = __builtin_convertvector(f, V);
        if (at + 8 <= n) {
            *reinterpret_cast<Loose *>(row + at) = o;
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (at + j < n) row[at + j] = o[j];
    }
};

struct Drop {
    Rng rng;
    unsigned long long offset;
    unsigned threshold;          // 65536: everything is kept
    float up;
};

// ... which of the eight elements of octet `at` of sample s stay
__device__ __forceinline__ void kept_of(const Drop &d, unsigned long long at, int s, bool (&kept)[8])
{
    const unsigned long long i = d.offset + at;
    const u4 x = philox4x32_10((unsigned)i, (unsigned)(i >> 32) | 0x80000000u, d.rng.first_sample + (unsigned)s, d.rng.step, d.rng.k0, d.rng.k1);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        kept[2 * j] = (x[j] & 0xFFFFu) < d.threshold;
        kept[2 * j + 1] = (x[j] >> 16) < d.threshold;
    }
}

__device__ __forceinline__ void drop(f8 &v, const bool (&kept)[8], float up)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = kept[j] ? v[j] * up : 0.0f;
}

// ---------------------------------------------------------------------------------
// Dropout alone.  `tpr` threads to a row (of one sample, blockIdx.y), each with an octet of every `tpr`; workgroups along z share long rows.
// Rows of whole octets are one long row.  Bound by memory: 32768 x 4096 bf16 in 98 us, 5.5 TB/s, as fast as they are copied.  (10007 x 1531 fp16, whose rows begin on any element: 15 us.)
// (x and y may be one array: every thread reads its octet before it writes it, and no other thread's.)
template <class T>
__global__ void __launch_bounds__(kBlockThreads)
hot_dropout_kernel(const T *x, T *y, long rows, long width, long octets, int tpr, Drop d)
{
    const int s = (int)blockIdx.y;
    x += (size_t)s * (size_t)rows * (size_t)width;
    y += (size_t)s * (size_t)rows * (size_t)width;
    const int groups = kBlockThreads / tpr, t = (int)threadIdx.x % tpr;
    const long along = (octets + tpr - 1) / tpr;
    for (long row = (long)blockIdx.x * groups + (int)threadIdx.x / tpr; row < rows; row += (long)gridDim.x * groups) {
        const T *const from = x + (size_t)row * (size_t)width;
        T *const to = y + (size_t)row * (size_t)width;
        for (long c = blockIdx.z; c < along; c += gridDim.z) {
            const long o = c * tpr + t;
            if (o >= octets) break;
            Octet<T> v;
            v.take(from, o * 8, width);
            bool kept[8];
            kept_of(d, (unsigned long long)row * (unsigned long long)octets + (unsigned long long)o, s, kept);
            f8 f = v.floats();
            drop(f, kept, d.up);
            Octet<T>::store(to, o * 8, width, f);
        }
    }
}

// ---------------------------------------------------------------------------------
struct BlockArgs {
    long rows, width;
    long weight_sample, bias_sample, gate_sample, branch_weight_sample, branch_bias_sample;
    float inv_width, eps, scale;
    int vector_type;
    bool layer, branch_layer, norm;      // whether the norms take the mean off; whether there is one behind the sum
    Drop d;
    const void *x, *branch, *weight, *bias, *gate, *branch_weight, *branch_bias, *dh, *dy;
    void *h, *y;                         // or dx, dbranch
    float *stats;                        // [samples, rows, 4]: mean and r of h, mean and r of the branch
    float *parts;                        // [samples, gridDim.x, kSums, width]
};

constexpr int kSums = 5;                 // gradients of weight, bias, gate, branch_weight, branch_bias
enum { kWeight, kBias, kGate, kBranchWeight, kBranchBias };

// Sums of N values over the TPR threads of a row.  `turn` alternates between two sets of slots, so that one barrier per sum is enough.
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float (*slots)[2], int &turn)
{
    constexpr int W = TPR < 64 ? TPR : 64;
#pragma unroll
    for (int off = W / 2; off > 0; off >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], off);
    if constexpr (TPR > 64) {
        constexpr int WAVES = TPR / 64;
        const int base = (int)(threadIdx.x / TPR) * 2 * WAVES + turn * WAVES;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) slots[base + (threadIdx.x % TPR >> 6)][k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) v[k] += slots[base + i][k];
        }
    }
}

// Eight elements of a vector: of the rows' type or float32
template <class T>
__device__ __forceinline__ f8 vector_of(const void *p, int type, long sample, long at, long n, float without)
{
    if (!p) return f8(without);
    if (type == HOT_F32) {
        Octet<float> v;
        v.take(static_cast<const float *>(p) + sample, at, n);
        return v.floats();
    }
    Octet<T> v;
    v.take(static_cast<const T *>(p) + sample, at, n);
    return v.floats();
}

__device__ __forceinline__ void clip(f8 &v, long valid)
{
    if (valid >= 8) return;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j >= valid) v[j] = 0.0f;
}

// Normalises a row's VPT octets a thread in place and says by which mean and factor
template <int TPR, int VPT>
__device__ __forceinline__ void normalise(f8 (&v)[VPT], bool layer, const BlockArgs &a, long at, float (*slots)[2], int &turn, float &mean, float &r)
{
    mean = 0.0f;
    if (layer) {
        float sum[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[0] += v[i][j];
        row_sum<TPR, 1>(sum, slots, turn);
        mean = sum[0] * a.inv_width;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            v[i] -= mean;
            clip(v[i], a.width - (at + (long)i * TPR * 8));
        }
    }
    float sq[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sq[0] = __builtin_fmaf(v[i][j], v[i][j], sq[0]);
    row_sum<TPR, 1>(sq, slots, turn);
    r = 1.0f / __builtin_sqrtf(__builtin_fmaf(sq[0], a.inv_width, a.eps));
#pragma unroll
    for (int i = 0; i < VPT; ++i) v[i] *= r;
}

template <int TPR>
constexpr int threads_of() { return TPR > kBlockThreads ? TPR : kBlockThreads; }

// waves of a workgroup's rows times two turns
template <int TPR>
constexpr int slots_of() { return TPR > 64 ? 2 * threads_of<TPR>() / 64 : 1; }

template <class T, int TPR, int VPT, bool BRANCH>
__global__ void __launch_bounds__(threads_of<TPR>())
hot_block_forward_kernel(BlockArgs a)
{
    constexpr int GROUPS = threads_of<TPR>() / TPR;
    __shared__ float slots[slots_of<TPR>()][2];
    int turn = 0;
    const int s = (int)blockIdx.y, t = (int)threadIdx.x % TPR;
    const long n = a.width, at = (long)t * 8, octets = (n + 7) / 8;
    const size_t base = (size_t)s * (size_t)a.rows * (size_t)n;
    const T *const xs = static_cast<const T *>(a.x) + base, *const bs = static_cast<const T *>(a.branch) + base;
    T *const hs = static_cast<T *>(a.h) + base, *const ys = a.y ? static_cast<T *>(a.y) + base : nullptr;
    const bool drops = a.d.threshold < 65536u;
    // (all groups of a workgroup walk equally far: rows are shared by its barriers)
    const long stride = (long)gridDim.x * GROUPS, first = (long)blockIdx.x * GROUPS;
    const long mine = first + (int)threadIdx.x / TPR;
    Octet<T> next_x[VPT], next_b[VPT];
    auto ask = [&](long row) {
        if (row >= a.rows) return;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            next_x[i].take(xs + (size_t)row * (size_t)n, at + (long)i * TPR * 8, n);
            next_b[i].take(bs + (size_t)row * (size_t)n, at + (long)i * TPR * 8, n);
        }
    };
    ask(mine);
    f8 gate[VPT], w[VPT], b[VPT], bw[VPT], bb[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const long c = at + (long)i * TPR * 8;
        gate[i] = vector_of<T>(a.gate, a.vector_type, s * a.gate_sample, c, n, 1.0f) * a.scale;
        if (ys) {
            w[i] = vector_of<T>(a.weight, a.vector_type, s * a.weight_sample, c, n, 1.0f);
            b[i] = vector_of<T>(a.bias, a.vector_type, s * a.bias_sample, c, n, 0.0f);
        }
        if constexpr (BRANCH) {
            bw[i] = vector_of<T>(a.branch_weight, a.vector_type, s * a.branch_weight_sample, c, n, 1.0f);
            bb[i] = vector_of<T>(a.branch_bias, a.vector_type, s * a.branch_bias_sample, c, n, 0.0f);
        }
    }
    for (long top = first; top < a.rows; top += stride) {
        const long row = top + (int)threadIdx.x / TPR;
        const bool there = row < a.rows;
        f8 h[VPT], d[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            h[i] = next_x[i].floats();
            d[i] = next_b[i].floats();
        }
        ask(row + stride);
        float mean = 0.0f, r = 0.0f, branch_mean = 0.0f, branch_r = 0.0f;
        if constexpr (BRANCH) {
            normalise<TPR, VPT>(d, a.branch_layer, a, at, slots, turn, branch_mean, branch_r);
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) d[i][j] = __builtin_fmaf(d[i][j], bw[i][j], bb[i][j]);
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const long c = at + (long)i * TPR * 8;
            if (drops) {
                bool kept[8];
                kept_of(a.d, (unsigned long long)row * (unsigned long long)octets + (unsigned long long)(c / 8), s, kept);
                drop(d[i], kept, a.d.up);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) h[i][j] = __builtin_fmaf(gate[i][j], d[i][j], h[i][j]);
            clip(h[i], n - c);
            if (there) Octet<T>::store(hs + (size_t)row * (size_t)n, c, n, h[i]);
        }
        if (ys) {
            normalise<TPR, VPT>(h, a.layer, a, at, slots, turn, mean, r);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                f8 y;
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = __builtin_fmaf(h[i][j], w[i][j], b[i][j]);
                if (there) Octet<T>::store(ys + (size_t)row * (size_t)n, at + (long)i * TPR * 8, n, y);
            }
        }
        if (t == 0 && there && a.stats) {
            f4 *const to = reinterpret_cast<f4 *>(a.stats) + (size_t)s * (size_t)a.rows + (size_t)row;
            *to = f4{mean, r, branch_mean, branch_r};
        }
    }
}

// The sums that a call asks for are known by the parts' pointers alone; those that cannot be (no branch norm) are left out of the code.
// 32768 x 8192 bf16, four arrays read and two written: 0.62 ms, 5.2 TB/s (the forward kernel's four arrays 0.42 ms, as much): a copy's rate.
template <class T, int TPR, int VPT, bool BRANCH>
__global__ void __launch_bounds__(threads_of<TPR>())
hot_block_backward_kernel(BlockArgs a)
{
    constexpr int THREADS = threads_of<TPR>(), GROUPS = THREADS / TPR, COLS = TPR * VPT * 8, SUMS = BRANCH ? 5 : 3;
    __shared__ float slots[slots_of<TPR>()][2];
    __shared__ float joined[TPR < THREADS ? THREADS / 64 * (TPR <= 64 ? COLS : COLS * 64 / TPR) : 1];
    int turn = 0;
    const int s = (int)blockIdx.y, t = (int)threadIdx.x % TPR;
    const long n = a.width, at = (long)t * 8, octets = (n + 7) / 8;
    const size_t base = (size_t)s * (size_t)a.rows * (size_t)n;
    const T *const xs = static_cast<const T *>(a.x) + base, *const bs = static_cast<const T *>(a.branch) + base;
    const T *const dhs = a.dh ? static_cast<const T *>(a.dh) + base : nullptr, *const dys = a.dy ? static_cast<const T *>(a.dy) + base : nullptr;
    T *const dxs = a.h ? static_cast<T *>(a.h) + base : nullptr, *const dbs = a.y ? static_cast<T *>(a.y) + base : nullptr;
    const bool drops = a.d.threshold < 65536u;
    const long stride = (long)gridDim.x * GROUPS, first = (long)blockIdx.x * GROUPS;
    Octet<T> next_x[VPT], next_b[VPT], next_dh[VPT], next_dy[VPT];
    f4 next_stats = f4(0.0f);
#pragma unroll
    for (int i = 0; i < VPT; ++i) next_x[i].v = next_b[i].v = next_dh[i].v = next_dy[i].v = (typename Octet<T>::V)((T)0.0f);
    auto ask = [&](long row) {
        if (row >= a.rows) return;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const long c = at + (long)i * TPR * 8;
            next_b[i].take(bs + (size_t)row * (size_t)n, c, n);
            if (dhs) next_dh[i].take(dhs + (size_t)row * (size_t)n, c, n);
            if (dys) {
                next_dy[i].take(dys + (size_t)row * (size_t)n, c, n);
                next_x[i].take(xs + (size_t)row * (size_t)n, c, n);
            }
        }
        next_stats = *(reinterpret_cast<const f4 *>(a.stats) + (size_t)s * (size_t)a.rows + (size_t)row);
    };
    ask(first + (int)threadIdx.x / TPR);
    f8 gate[VPT], w[VPT], bw[VPT], bb[VPT], sums[SUMS][VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const long c = at + (long)i * TPR * 8;
        gate[i] = vector_of<T>(a.gate, a.vector_type, s * a.gate_sample, c, n, 1.0f) * a.scale;
        w[i] = vector_of<T>(a.weight, a.vector_type, s * a.weight_sample, c, n, 1.0f);
        if constexpr (BRANCH) {
            bw[i] = vector_of<T>(a.branch_weight, a.vector_type, s * a.branch_weight_sample, c, n, 1.0f);
            bb[i] = vector_of<T>(a.branch_bias, a.vector_type, s * a.branch_bias_sample, c, n, 0.0f);
        }
#pragma unroll
        for (int k = 0; k < SUMS; ++k) sums[k][i] = f8(0.0f);
    }
    for (long top = first; top < a.rows; top += stride) {
        const long row = top + (int)threadIdx.x / TPR;
        const bool there = row < a.rows;
        // (a row that is not there: its loads were not made, the row before is still in the registers)
        f8 h[VPT], d[VPT], du[VPT], u[VPT], tn[VPT];
        const f4 st = next_stats;
        const float mean = st[0], r = st[1], branch_mean = st[2], branch_r = st[3];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            h[i] = next_x[i].floats();
            d[i] = next_b[i].floats();
            du[i] = next_dh[i].floats();
            u[i] = next_dy[i].floats();
            if (!there) du[i] = u[i] = f8(0.0f);
        }
        ask(row + stride);
        unsigned mask[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const long c = at + (long)i * TPR * 8;
            mask[i] = 0xFFu;
            if constexpr (BRANCH) {
                tn[i] = (d[i] - branch_mean) * branch_r;
                clip(tn[i], n - c);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[i][j] = __builtin_fmaf(tn[i][j], bw[i][j], bb[i][j]);
            }
            if (drops) {
                bool kept[8];
                kept_of(a.d, (unsigned long long)row * (unsigned long long)octets + (unsigned long long)(c / 8), s, kept);
                drop(d[i], kept, a.d.up);
                mask[i] = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) mask[i] |= (unsigned)kept[j] << j;
            }
        }
        if (dys) {
            float sum[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = (__builtin_fmaf(gate[i][j], d[i][j], h[i][j]) - mean) * r;
                clip(h[i], n - (at + (long)i * TPR * 8));
                if (!there) h[i] = f8(0.0f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sums[kBias][i][j] += u[i][j];
                    sums[kWeight][i][j] = __builtin_fmaf(u[i][j], h[i][j], sums[kWeight][i][j]);
                    u[i][j] *= w[i][j];
                    sum[0] += u[i][j];
                    sum[1] = __builtin_fmaf(u[i][j], h[i][j], sum[1]);
                }
            }
            row_sum<TPR, 2>(sum, slots, turn);
            const float c1 = a.layer ? sum[0] * a.inv_width : 0.0f, c2 = sum[1] * a.inv_width;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) du[i][j] = __builtin_fmaf(r, u[i][j] - __builtin_fmaf(h[i][j], c2, c1), du[i][j]);
        }
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const long c = at + (long)i * TPR * 8;
            if (!there) du[i] = d[i] = f8(0.0f);
            clip(du[i], n - c);
            if (dxs && there) Octet<T>::store(dxs + (size_t)row * (size_t)n, c, n, du[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sums[kGate][i][j] = __builtin_fmaf(du[i][j], d[i][j], sums[kGate][i][j]);
                du[i][j] = mask[i] >> j & 1u ? du[i][j] * gate[i][j] * a.d.up : 0.0f;
            }
            if constexpr (BRANCH) {
                if (!there) tn[i] = f8(0.0f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sums[kBranchBias][i][j] += du[i][j];
                    sums[kBranchWeight][i][j] = __builtin_fmaf(du[i][j], tn[i][j], sums[kBranchWeight][i][j]);
                    du[i][j] *= bw[i][j];
                    sum[0] += du[i][j];
                    sum[1] = __builtin_fmaf(du[i][j], tn[i][j], sum[1]);
                }
            }
        }
        if constexpr (BRANCH) {
            row_sum<TPR, 2>(sum, slots, turn);
            const float c1 = a.branch_layer ? sum[0] * a.inv_width : 0.0f, c2 = sum[1] * a.inv_width;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) du[i][j] = branch_r * (du[i][j] - __builtin_fmaf(tn[i][j], c2, c1));
        }
        if (dbs && there)
#pragma unroll
            for (int i = 0; i < VPT; ++i) Octet<T>::store(dbs + (size_t)row * (size_t)n, at + (long)i * TPR * 8, n, du[i]);
    }
    if (!a.parts) return;
    float *const part = a.parts + ((size_t)s * gridDim.x + blockIdx.x) * kSums * (size_t)n;
#pragma unroll
    for (int k = 0; k < SUMS; ++k) {
        if (k == kGate)
#pragma unroll
            for (int i = 0; i < VPT; ++i) sums[k][i] *= a.scale;
        if constexpr (TPR >= THREADS) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const long c = at + (long)i * TPR * 8 + j;
                    if (c < n) part[(size_t)k * (size_t)n + (size_t)c] = sums[k][i][j];
                }
        } else {
            // the rows that lanes and waves of the workgroup held side by side
            constexpr int W = TPR < 64 ? TPR : 64, WIDE = W * VPT * 8;           // columns of a wave
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
#pragma unroll
                    for (int off = W; off < 64; off <<= 1) sums[k][i][j] += __shfl_xor(sums[k][i][j], off);
                    if ((threadIdx.x & 63) < W) joined[(threadIdx.x >> 6) * WIDE + (i * W + (threadIdx.x & 63)) * 8 + j] = sums[k][i][j];
                }
            __syncthreads();
            constexpr int PER = TPR > 64 ? TPR / 64 : 1, ROWS = THREADS / 64 / PER;      // waves to a row, rows side by side
            for (int c = (int)threadIdx.x; c < COLS; c += THREADS) {
                // column c of a row lies with thread c / 8 % TPR, its octet c / 8 / TPR
                const int octet = c / 8 % TPR, i = c / 8 / TPR, wave = octet / 64, lane = octet % 64;
                float sum = 0.0f;
#pragma unroll
                for (int g = 0; g < ROWS; ++g) sum += joined[(g * PER + wave) * WIDE + (i * W + lane) * 8 + c % 8];
                if (c < n) part[(size_t)k * (size_t)n + (size_t)c] = sum;
            }
            __syncthreads();
        }
    }
}

// The vectors' gradients: sums of the workgroups' rows of partial sums, 64 columns and 16 runs of rows to a workgroup.
constexpr int kRuns = 16;

struct JoinArgs {
    const float *parts;
    long blocks, width;
    int samples, type;
    void *to[kSums];
    long sample[kSums];          // 0: one vector for all samples
};

__global__ void __launch_bounds__(64 * kRuns)
hot_block_join_kernel(JoinArgs a)
{
    __shared__ float runs[kRuns][64];
    const int lane = (int)threadIdx.x & 63, run = (int)threadIdx.x >> 6, k = (int)blockIdx.y, s = (int)blockIdx.z;
    void *const out = a.to[k];
    const bool own = a.sample[k] > 0;
    if (!out || (!own && s > 0)) return;                    // (the whole workgroup)
    const long col = (long)blockIdx.x * 64 + lane, count = own ? a.blocks : a.blocks * a.samples;
    float sum = 0.0f;
    if (col < a.width) {
        const float *p = a.parts + (((size_t)s * (size_t)a.blocks) * kSums + (size_t)k) * (size_t)a.width + (size_t)col;
        for (long i = run; i < count; i += 4 * kRuns) {
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = i + j * kRuns < count ? p[(size_t)(i + j * kRuns) * kSums * (size_t)a.width] : 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) sum += v[j];
        }
    }
    runs[run][lane] = sum;
    __syncthreads();
    if (run || col >= a.width) return;
#pragma unroll
    for (int i = 1; i < kRuns; ++i) sum += runs[i][lane];
    store_as(out, a.type, s * a.sample[k] + col, sum);
}

// ---------------------------------------------------------------------------------
// Host side

bool make_drop(const hot_rng *rng, int samples, double keep, int64_t offset, double calls, Drop &d)
{
    if (!(keep > 0.0 && keep <= 1.0) || offset < 0 || (double)offset + calls > 9.2e18) return false;
    d = {};
    const double most = keep * 65536.0 + 0.5;
    d.threshold = most < 1.0 ? 1u : (unsigned)most;
    // (the nearest whole number; a tie goes to the even one)
    if ((double)d.threshold == most && (d.threshold & 1u)) --d.threshold;
    if (d.threshold < 1u) d.threshold = 1u;
    d.up = (float)(65536.0 / d.threshold);
    d.offset = (unsigned long long)offset;
    return d.threshold >= 65536u || make_rng(rng, samples, d.rng);
}

template <class T>
void dropout_run(const hot_dropout_desc &d, const Drop &drops, const void *x, void *y, hipStream_t s)
{
    long rows = d.rows, width = d.width;
    if (width % 8 == 0) {
        width *= rows;
        rows = 1;
    }
    const long octets = (width + 7) / 8;
    int tpr = kBlockThreads;
    if (rows > 1)
        while (tpr > 1 && tpr / 2 >= octets) tpr /= 2;
    // as many workgroups as are resident twice over: along the rows' number, and along the rows where there are few
    const long most = 16L * kUnits, groups = kBlockThreads / tpr, down = (rows + groups - 1) / groups, along = (octets + tpr - 1) / tpr;
    const long x_blocks = down < most ? down : most, room = most / x_blocks, z_blocks = along < room ? along : room;
    hot_dropout_kernel<T><<<dim3((unsigned)x_blocks, (unsigned)d.samples, (unsigned)z_blocks), kBlockThreads, 0, s>>>(
        static_cast<const T *>(x), static_cast<T *>(y), rows, width, octets, tpr, drops);
}

// Threads to a row and octets to a thread
struct BlockShape {
    int tpr, vpt;
};

BlockShape block_shape(long width)
{
    const long octets = (width + 7) / 8;
    for (int tpr : {8, 16, 32, 64, 128, 256, 512, 1024})
        if (octets <= tpr) return {tpr, 1};
    return {1024, 2};
}

long block_backward_blocks(const hot_block_desc &d)
{
    const BlockShape h = block_shape(d.width);
    const long groups = h.tpr < kBlockThreads ? kBlockThreads / h.tpr : 1, want = (d.rows + groups - 1) / groups;
    const long resident = (h.tpr > 512 ? 1 : (h.tpr > kBlockThreads ? 2 : 4)) * (long)kUnits;
    const long most = (resident + d.samples - 1) / d.samples;
    return want < 1 ? 1 : (want < most ? want : most);
}

bool one_or_own(int64_t pitch, int64_t width) { return pitch == 0 || pitch >= width; }

bool block_ok(const hot_block_desc *d)
{
    return d && d->rows >= 0 && d->rows <= (1L << 40) && d->width >= 1 && d->width <= HOT_BLOCK_MOST_WIDTH && d->samples >= 1 && d->samples <= 65535 && known_type(d->dtype) &&
           (d->vector_dtype == d->dtype || d->vector_dtype == HOT_F32) && one_or_own(d->weight_sample, d->width) && one_or_own(d->bias_sample, d->width) &&
           one_or_own(d->gate_sample, d->width) && one_or_own(d->branch_weight_sample, d->width) && one_or_own(d->branch_bias_sample, d->width) && d->eps >= 0.0 &&
           d->eps <= 3.0e38 && d->scale >= -3.0e38 && d->scale <= 3.0e38 && d->norm >= HOT_NORM_NONE && d->norm <= HOT_NORM_RMS && d->branch_norm >= HOT_NORM_NONE &&
           d->branch_norm <= HOT_NORM_RMS;
}

bool block_args(const hot_block_desc &d, const hot_rng *rng, BlockArgs &a)
{
    a = {};
    if (!make_drop(rng, d.samples, d.keep, d.offset, (double)d.rows * (double)((d.width + 7) / 8), a.d)) return false;
    a.rows = d.rows;
    a.width = d.width;
    a.weight_sample = d.weight_sample;
    a.bias_sample = d.bias_sample;
    a.gate_sample = d.gate_sample;
    a.branch_weight_sample = d.branch_weight_sample;
    a.branch_bias_sample = d.branch_bias_sample;
    a.inv_width = (float)(1.0 / (double)d.width);
    a.eps = (float)d.eps;
    a.scale = (float)d.scale;
    a.vector_type = d.vector_dtype;
    a.layer = d.norm == HOT_NORM_LAYER;
    a.norm = d.norm != HOT_NORM_NONE;
    a.branch_layer = d.branch_norm == HOT_NORM_LAYER;
    return true;
}

template <class T, int TPR, int VPT>
void block_go(const hot_block_desc &d, bool backward, const BlockArgs &a, hipStream_t s)
{
    constexpr int THREADS = threads_of<TPR>();
    const long groups = THREADS / TPR, want = (d.rows + groups - 1) / groups, most = 16L * kUnits;
    const dim3 grid((unsigned)(backward ? block_backward_blocks(d) : (want < most ? want : most)), (unsigned)d.samples);
    if (backward) {
        if (d.branch_norm != HOT_NORM_NONE) hot_block_backward_kernel<T, TPR, VPT, true><<<grid, THREADS, 0, s>>>(a);
        else hot_block_backward_kernel<T, TPR, VPT, false><<<grid, THREADS, 0, s>>>(a);
    } else if (d.branch_norm != HOT_NORM_NONE) hot_block_forward_kernel<T, TPR, VPT, true><<<grid, THREADS, 0, s>>>(a);
    else hot_block_forward_kernel<T, TPR, VPT, false><<<grid, THREADS, 0, s>>>(a);
}

template <class T>
void block_run(const hot_block_desc &d, bool backward, const BlockArgs &a, hipStream_t s)
{
    const BlockShape h = block_shape(d.width);
    if (h.vpt == 2) block_go<T, 1024, 2>(d, backward, a, s);
    else if (h.tpr == 8) block_go<T, 8, 1>(d, backward, a, s);
    else if (h.tpr == 16) block_go<T, 16, 1>(d, backward, a, s);
    else if (h.tpr == 32) block_go<T, 32, 1>(d, backward, a, s);
    else if (h.tpr == 64) block_go<T, 64, 1>(d, backward, a, s);
    else if (h.tpr == 128) block_go<T, 128, 1>(d, backward, a, s);
    else if (h.tpr == 256) block_go<T, 256, 1>(d, backward, a, s);
    else if (h.tpr == 512) block_go<T, 512, 1>(d, backward, a, s);
    else block_go<T, 1024, 1>(d, backward, a, s);
}

void block_run(const hot_block_desc &d, bool backward, const BlockArgs &a, hipStream_t s)
{
    if (d.dtype == HOT_F32) block_run<float>(d, backward, a, s);
    else if (d.dtype == HOT_BF16) block_run<__bf16>(d, backward, a, s);
    else block_run<_Float16>(d, backward, a, s);
}

}  // namespace

extern "C" {

int hot_dropout(const hot_dropout_desc *desc, const hot_rng *rng, const void *x, void *y, void *stream)
{
    if (!desc || desc->rows < 0 || desc->rows > (1L << 40) || desc->width < 1 || desc->width > (1L << 40) || desc->samples < 1 || desc->samples > 65535 ||
        !known_type(desc->dtype))
        return HOT_EINVAL;
    const double octets = (double)desc->rows * (double)((desc->width + 7) / 8);
    Drop d;
    if (octets * 8 * desc->samples > 1.0e18 || !make_drop(rng, desc->samples, desc->keep, desc->offset, octets, d)) return HOT_EINVAL;
    if (desc->rows == 0) return HOT_OK;
    if (!x || !y || !on_element(x, desc->dtype) || !on_element(y, desc->dtype)) return HOT_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (desc->dtype == HOT_F32) dropout_run<float>(*desc, d, x, y, s);
    else if (desc->dtype == HOT_BF16) dropout_run<__bf16>(*desc, d, x, y, s);
    else dropout_run<_Float16>(*desc, d, x, y, s);
    return hot_detail::note_hip(hipGetLastError());
}

int hot_block_forward(const hot_block_desc *desc, const hot_rng *rng, const void *x, const void *branch, const void *weight, const void *bias, const void *gate,
                      const void *branch_weight, const void *branch_bias, void *h, void *y, float *stats, void *stream)
{
    BlockArgs a;
    if (!block_ok(desc) || !block_args(*desc, rng, a)) return HOT_EINVAL;
    if (desc->rows == 0) return HOT_OK;
    const int t = desc->dtype, v = desc->vector_dtype;
    if (!x || !branch || !h || (y != nullptr) != a.norm || !on_element(x, t) || !on_element(branch, t) || !on_element(h, t) || !on_element(y, t) || !on_element(weight, v) ||
        !on_element(bias, v) || !on_element(gate, v) || !on_element(branch_weight, v) || !on_element(branch_bias, v) || !aligned16(stats))
        return HOT_EINVAL;
    a.x = x;
    a.branch = branch;
    a.weight = weight;
    a.bias = bias;
    a.gate = gate;
    a.branch_weight = branch_weight;
    a.branch_bias = branch_bias;
    a.h = h;
    a.y = y;
    a.stats = stats;
    block_run(*desc, false, a, static_cast<hipStream_t>(stream));
    return hot_detail::note_hip(hipGetLastError());
}

int64_t hot_block_backward_workspace_bytes(const hot_block_desc *desc)
{
    if (!block_ok(desc)) return HOT_EINVAL;
    return block_backward_blocks(*desc) * desc->samples * kSums * desc->width * 4;
}

int hot_block_backward(const hot_block_desc *desc, const hot_rng *rng, const void *x, const void *branch, const void *weight, const void *gate,
                       const void *branch_weight, const void *branch_bias, const float *stats, const void *dh, const void *dy, void *dx, void *dbranch,
                       void *grad_weight, void *grad_bias, void *grad_gate, void *grad_branch_weight, void *grad_branch_bias, void *workspace,
                       int64_t workspace_bytes, void *stream)
{
    BlockArgs a;
    if (!block_ok(desc) || !block_args(*desc, rng, a)) return HOT_EINVAL;
    const int t = desc->dtype, v = desc->vector_dtype;
    void *const grads[kSums] = {grad_weight, grad_bias, grad_gate, grad_branch_weight, grad_branch_bias};
    bool sums = false;
    for (void *g : grads) {
        if (!on_element(g, v)) return HOT_EINVAL;
        sums = sums || g;
    }
    if ((grad_weight || grad_bias) && !a.norm) return HOT_EINVAL;
    if ((grad_branch_weight || grad_branch_bias) && desc->branch_norm == HOT_NORM_NONE) return HOT_EINVAL;
    if (sums && (!workspace || !aligned4(workspace) || workspace_bytes < hot_block_backward_workspace_bytes(desc))) return HOT_EINVAL;
    if (desc->rows > 0 && (!x || !branch || !stats || (dy && !a.norm) || !on_element(x, t) || !on_element(branch, t) || !on_element(dh, t) || !on_element(dy, t) ||
                           !on_element(dx, t) || !on_element(dbranch, t) || !on_element(weight, v) || !on_element(gate, v) || !on_element(branch_weight, v) ||
                           !on_element(branch_bias, v) || !aligned16(stats)))
        return HOT_EINVAL;
    a.x = x;
    a.branch = branch;
    a.weight = weight;
    a.gate = gate;
    a.branch_weight = branch_weight;
    a.branch_bias = branch_bias;
    a.dh = dh;
    a.dy = dy;
    a.h = dx;
    a.y = dbranch;
    a.stats = const_cast<float *>(stats);
    a.parts = sums ? static_cast<float *>(workspace) : nullptr;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (desc->rows > 0 && (dx || dbranch || sums)) block_run(*desc, true, a, s);
    if (sums) {
        JoinArgs j = {};
        j.parts = a.parts;
        j.blocks = desc->rows > 0 ? block_backward_blocks(*desc) : 0;        // (no rows: no partial sums to add, which gives zeros)
        j.width = desc->width;
        j.samples = desc->samples;
        j.type = v;
        const int64_t own[kSums] = {desc->weight_sample, desc->bias_sample, desc->gate_sample, desc->branch_weight_sample, desc->branch_bias_sample};
        bool any = false;
        for (int k = 0; k < kSums; ++k) {
            j.to[k] = grads[k];
            j.sample[k] = own[k];
            any = any || (grads[k] && own[k] > 0);
        }
        hot_block_join_kernel<<<dim3((unsigned)((desc->width + 63) / 64), kSums, any ? (unsigned)desc->samples : 1u), 64 * kRuns, 0, s>>>(j);
    }
    return hot_detail::note_hip(hipGetLastError());
}

}  // extern "C"
