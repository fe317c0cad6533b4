// libhot: layer norm over the last axis, forward and backward, with weights shared by all rows or one set per weight sample.
//
//   forward   m = mean x,  r = 1/sqrt(mean (x - m)^2 + eps),  h = (x - m) r,  y = h w + b
//   backward  u = dy w,  dx = r (u - mean u - h mean(u h)),  dw = sum over rows dy h,  db = sum over rows dy
//
// What bounds both is memory: a row is read once, kept in registers through mean, variance and result, and written once, while the next
// row of the same threads is on its way.  32768 x 8192 in bf16: forward 244 us (4.4 TB/s), backward 314 (5.1); a copy of that size runs at
// 4.8 to 5.2.  TPR threads share a row, each with VPT pieces of sixteen bytes; rows shorter than a wavefront's reach share one
// (TPR = 16), longer ones take a workgroup.  Mean, then variance of what was read (two passes over registers, no cancellation), in fp32.
// The sums for dw and db stay in registers of the threads that own the columns while a workgroup walks its rows; every workgroup
// leaves one row of partial sums in scratch memory and a second kernel adds them in a fixed order.
#include <hip/hip_runtime.h>

#include "hot.h"
#include "vec.h"
#include "element.h"

// (a product that is rounded here and contracted there would leave u - mean u other than zero where all u are the same)
#pragma clang fp contract(off)

namespace {

constexpr int kNormBlock = 256;
constexpr int kComputeUnits = 256;

struct NormArgs {
    long rows;                   // of one sample
    long width;
    long ldx, x_sample, w_sample, ldy, y_sample;      // elements; ldy / y_sample: dy of the backward pass (y and dx are dense)
    float inv_width, eps;
    int w_type;
    const void *x, *w, *b, *dy;
    void *out;                   // y or dx, [samples, rows, width]
    float *mean, *rstd;          // [samples, rows]
    float *parts;                // [samples, gridDim.x, 2, width]
};

// Sums of N values over the TPR threads of a row.  `turn` alternates between two sets of slots, so that one barrier per sum is enough.
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float (*slots)[N], int &turn)
{
    constexpr int W = TPR < 64 ? TPR : 64;
#pragma unroll
    for (int off = W / 2; off > 0; off >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], off);
    if constexpr (TPR > 64) {
        constexpr int WAVES = TPR / 64;
        float (*const s)[N] = slots + turn * WAVES;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) s[threadIdx.x >> 6][k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) v[k] += s[i][k];
        }
    }
}

// zeros behind the row's end, where a piece reaches there
template <int N, class F>
__device__ __forceinline__ void clip(F &v, int valid)
{
    if (valid >= N) return;
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j >= valid) v[j] = 0.0f;
}

template <class T, int TPR, int VPT>
__global__ void __launch_bounds__(TPR > kNormBlock ? TPR : kNormBlock)
hot_norm_forward_kernel(NormArgs a)
{
    typedef Piece<T> P;
    typedef typename P::F F;
    constexpr int N = P::N, BLOCK = TPR > kNormBlock ? TPR : kNormBlock, GROUPS = BLOCK / TPR;
    __shared__ float slots[2 * (TPR > 64 ? TPR / 64 : 1)][1];
    int turn = 0;
    const int t = (int)threadIdx.x % TPR, s = (int)blockIdx.y, n = (int)a.width;
    const T *const xs = static_cast<const T *>(a.x) + (size_t)s * (size_t)a.x_sample;
    T *const ys = static_cast<T *>(a.out) + (size_t)s * (size_t)a.rows * (size_t)n;
    const long stride = (long)gridDim.x * GROUPS;
    long row = (long)blockIdx.x * GROUPS + threadIdx.x / TPR;
    typename P::V next[VPT];
    auto ask = [&](long r) {
        if (r >= a.rows) return;
#pragma unroll
        for (int i = 0; i < VPT; ++i) next[i] = P::take(xs + (size_t)r * (size_t)a.ldx, (i * TPR + t) * N, n);
    };
    ask(row);
    F w[VPT], b[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const long at = s * a.w_sample + (i * TPR + t) * N, end = s * a.w_sample + n;
        w[i] = a.w ? load_as<N, F>(a.w, a.w_type, at, end) : F(1.0f);
        b[i] = a.b ? load_as<N, F>(a.b, a.w_type, at, end) : F(0.0f);
    }
    for (; row < a.rows; row += stride) {
        F v[VPT];
        float sum[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            v[i] = __builtin_convertvector(next[i], F);
#pragma unroll
            for (int j = 0; j < N; ++j) sum[0] += v[i][j];
        }
        ask(row + stride);
        row_sum<TPR, 1>(sum, slots, turn);
        const float mean = sum[0] * a.inv_width;
        float sq[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            v[i] -= mean;
            clip<N>(v[i], n - (i * TPR + t) * N);
#pragma unroll
            for (int j = 0; j < N; ++j) sq[0] = __builtin_fmaf(v[i][j], v[i][j], sq[0]);
        }
        row_sum<TPR, 1>(sq, slots, turn);
        const float rstd = 1.0f / __builtin_sqrtf(__builtin_fmaf(sq[0], a.inv_width, a.eps));
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            F o;
#pragma unroll
            for (int j = 0; j < N; ++j) o[j] = __builtin_fmaf(v[i][j] * rstd, w[i][j], b[i][j]);
            P::store(ys + (size_t)row * (size_t)n, (i * TPR + t) * N, n, o);
        }
        if (t == 0 && a.mean) {
            a.mean[s * a.rows + row] = mean;
            a.rstd[s * a.rows + row] = rstd;
        }
    }
}

template <class T, int TPR, int VPT>
__global__ void __launch_bounds__(TPR > kNormBlock ? TPR : kNormBlock)
hot_norm_backward_kernel(NormArgs a)
{
    typedef Piece<T> P;
    typedef typename P::F F;
    constexpr int N = P::N, BLOCK = TPR > kNormBlock ? TPR : kNormBlock, GROUPS = BLOCK / TPR, COLS = TPR * VPT * N;
    __shared__ float slots[2 * (TPR > 64 ? TPR / 64 : 1)][2];
    __shared__ float joined[TPR <= 64 ? BLOCK / 64 * COLS : 1];
    int turn = 0;
    const int t = (int)threadIdx.x % TPR, s = (int)blockIdx.y, n = (int)a.width;
    const T *const xs = static_cast<const T *>(a.x) + (size_t)s * (size_t)a.x_sample;
    const T *const dys = static_cast<const T *>(a.dy) + (size_t)s * (size_t)a.y_sample;
    T *const dxs = static_cast<T *>(a.out) + (size_t)s * (size_t)a.rows * (size_t)n;
    const long stride = (long)gridDim.x * GROUPS;
    long row = (long)blockIdx.x * GROUPS + threadIdx.x / TPR;
    typename P::V next_x[VPT], next_dy[VPT];
    float next_mean = 0.0f, next_rstd = 0.0f;
    auto ask = [&](long r) {
        if (r >= a.rows) return;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            next_x[i] = P::take(xs + (size_t)r * (size_t)a.ldx, (i * TPR + t) * N, n);
            next_dy[i] = P::take(dys + (size_t)r * (size_t)a.ldy, (i * TPR + t) * N, n);
        }
        next_mean = a.mean[s * a.rows + r];
        next_rstd = a.rstd[s * a.rows + r];
    };
    ask(row);
    F w[VPT], dw[VPT], db[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        dw[i] = db[i] = F(0.0f);
        w[i] = a.w ? load_as<N, F>(a.w, a.w_type, s * a.w_sample + (i * TPR + t) * N, s * a.w_sample + n) : F(1.0f);
    }
    for (; row < a.rows; row += stride) {
        F h[VPT], u[VPT];
        const float mean = next_mean, rstd = next_rstd;
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            u[i] = __builtin_convertvector(next_dy[i], F);
            h[i] = (__builtin_convertvector(next_x[i], F) - mean) * rstd;
            // (behind the row's end dy is zero, and h is made so: the row's own statistics need not be finite)
            clip<N>(h[i], n - (i * TPR + t) * N);
        }
        ask(row + stride);
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                db[i][j] += u[i][j];
                dw[i][j] = __builtin_fmaf(u[i][j], h[i][j], dw[i][j]);
                u[i][j] *= w[i][j];
                sum[0] += u[i][j];
                sum[1] = __builtin_fmaf(u[i][j], h[i][j], sum[1]);
            }
        if (!a.out) continue;
        row_sum<TPR, 2>(sum, slots, turn);
        const float c1 = sum[0] * a.inv_width, c2 = sum[1] * a.inv_width;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            F o;
#pragma unroll
            for (int j = 0; j < N; ++j) o[j] = rstd * (u[i][j] - __builtin_fmaf(h[i][j], c2, c1));
            P::store(dxs + (size_t)row * (size_t)n, (i * TPR + t) * N, n, o);
        }
    }
    if (!a.parts) return;
    float *const part = a.parts + ((size_t)s * gridDim.x + blockIdx.x) * 2 * (size_t)n;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        F (&v)[VPT] = which ? db : dw;
        if constexpr (TPR > 64) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const long at = (long)(i * TPR + t) * N + j;
                    if (at < n) part[which * n + at] = v[i][j];
                }
        } else {
            // the rows that lanes and waves of the workgroup held side by side
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
#pragma unroll
                    for (int off = TPR; off < 64; off <<= 1) v[i][j] += __shfl_xor(v[i][j], off);
                    if ((threadIdx.x & 63) < TPR) joined[(threadIdx.x >> 6) * COLS + (i * TPR + t) * N + j] = v[i][j];
                }
            __syncthreads();
            for (int at = (int)threadIdx.x; at < COLS && at < n; at += BLOCK) {
                float sum = 0.0f;
#pragma unroll
                for (int k = 0; k < BLOCK / 64; ++k) sum += joined[k * COLS + at];
                part[which * n + at] = sum;
            }
            __syncthreads();
        }
    }
}

// Rows too long for a workgroup's registers: three passes over the row, the second and third of which find it in the caches.
constexpr int kWideBlock = 1024;

template <class T, bool BACKWARD>
__global__ void __launch_bounds__(kWideBlock)
hot_norm_wide_kernel(NormArgs a)
{
    typedef Piece<T> P;
    constexpr int N = P::N;
    __shared__ float slots[2 * kWideBlock / 64][2];
    int turn = 0;
    const int s = (int)blockIdx.y;
    const long n = a.width, step = (long)kWideBlock * N, first = (long)threadIdx.x * N;
    for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *const x = static_cast<const T *>(a.x) + (size_t)s * (size_t)a.x_sample + (size_t)row * (size_t)a.ldx;
        const T *const dy = BACKWARD ? static_cast<const T *>(a.dy) + (size_t)s * (size_t)a.y_sample + (size_t)row * (size_t)a.ldy : nullptr;
        T *const out = static_cast<T *>(a.out) + ((size_t)s * (size_t)a.rows + (size_t)row) * (size_t)n;
        float mean, rstd, sum[2] = {0.0f, 0.0f};
        auto weights = [&](const void *w, long at) { return load_as<N, typename P::F>(w, a.w_type, s * a.w_sample + at, s * a.w_sample + n); };
        if constexpr (!BACKWARD) {
            for (long at = first; at < n; at += step) {
                const typename P::F v = P::load(x, at, n);
#pragma unroll
                for (int j = 0; j < N; ++j) sum[0] += v[j];
            }
            row_sum<kWideBlock, 2>(sum, slots, turn);
            mean = sum[0] * a.inv_width;
            float sq[2] = {0.0f, 0.0f};
            for (long at = first; at < n; at += step) {
                const typename P::F v = P::load(x, at, n);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float c = at + j < n ? v[j] - mean : 0.0f;
                    sq[0] = __builtin_fmaf(c, c, sq[0]);
                }
            }
            row_sum<kWideBlock, 2>(sq, slots, turn);
            rstd = 1.0f / __builtin_sqrtf(__builtin_fmaf(sq[0], a.inv_width, a.eps));
            for (long at = first; at < n; at += step) {
                const typename P::F v = P::load(x, at, n), w = a.w ? weights(a.w, at) : typename P::F(1.0f), b = a.b ? weights(a.b, at) : typename P::F(0.0f);
                typename P::F o;
#pragma unroll
                for (int j = 0; j < N; ++j) o[j] = __builtin_fmaf((v[j] - mean) * rstd, w[j], b[j]);
                P::store(out, at, n, o);
            }
            if (threadIdx.x == 0 && a.mean) {
                a.mean[s * a.rows + row] = mean;
                a.rstd[s * a.rows + row] = rstd;
            }
        } else {
            mean = a.mean[s * a.rows + row];
            rstd = a.rstd[s * a.rows + row];
            for (long at = first; at < n; at += step) {
                const typename P::F v = P::load(x, at, n), d = P::load(dy, at, n), w = a.w ? weights(a.w, at) : typename P::F(1.0f);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float u = d[j] * w[j], h = at + j < n ? (v[j] - mean) * rstd : 0.0f;
                    sum[0] += u;
                    sum[1] = __builtin_fmaf(u, h, sum[1]);
                }
            }
            row_sum<kWideBlock, 2>(sum, slots, turn);
            const float c1 = sum[0] * a.inv_width, c2 = sum[1] * a.inv_width;
            for (long at = first; at < n; at += step) {
                const typename P::F v = P::load(x, at, n), d = P::load(dy, at, n), w = a.w ? weights(a.w, at) : typename P::F(1.0f);
                typename P::F o;
#pragma unroll
                for (int j = 0; j < N; ++j) o[j] = rstd * (d[j] * w[j] - __builtin_fmaf((v[j] - mean) * rstd, c2, c1));
                P::store(out, at, n, o);
            }
        }
    }
}

// ... and their weights' sums: threads own columns, workgroups along y the rows y, y + gridDim.y, ...
template <class T>
__global__ void __launch_bounds__(kNormBlock)
hot_norm_wide_weights_kernel(NormArgs a)
{
    typedef Piece<T> P;
    constexpr int N = P::N;
    const int s = (int)blockIdx.z;
    const long n = a.width, at = ((long)blockIdx.x * kNormBlock + threadIdx.x) * N;
    if (at >= n) return;
    typename P::F dw = typename P::F(0.0f), db = dw;
    for (long row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const typename P::F v = P::load(static_cast<const T *>(a.x) + (size_t)s * (size_t)a.x_sample + (size_t)row * (size_t)a.ldx, at, n);
        const typename P::F d = P::load(static_cast<const T *>(a.dy) + (size_t)s * (size_t)a.y_sample + (size_t)row * (size_t)a.ldy, at, n);
        const float mean = a.mean[s * a.rows + row], rstd = a.rstd[s * a.rows + row];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            db[j] += d[j];
            dw[j] = __builtin_fmaf(d[j], (v[j] - mean) * rstd, dw[j]);
        }
    }
    float *const part = a.parts + ((size_t)s * gridDim.y + blockIdx.y) * 2 * (size_t)n;
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (at + j < n) {
            part[at + j] = dw[j];
            part[n + at + j] = db[j];
        }
}

// dw and db: the sums of `parts` rows of partial sums, 64 columns and 16 runs of rows to a workgroup (that takes several blocks of columns beyond kMostJoinBlocks:
// a grid's dimension holds fewer than 2^32 threads).
constexpr int kJoinRuns = 16;
constexpr long kMostJoinBlocks = 1L << 20;

__global__ void __launch_bounds__(64 * kJoinRuns)
hot_norm_join_kernel(const float *__restrict__ parts, long count, long width, long out_sample, int type, void *dw, void *db)
{
    __shared__ float runs[kJoinRuns][64];
    const int lane = (int)threadIdx.x & 63, run = (int)threadIdx.x >> 6, which = (int)blockIdx.y, s = (int)blockIdx.z;
    void *const out = which ? db : dw;
    if (!out) return;                    // (the whole workgroup)
    for (long first = (long)blockIdx.x * 64; first < width; first += (long)gridDim.x * 64) {
        const long col = first + lane;
        float sum = 0.0f;
        if (col < width) {
            const float *p = parts + ((size_t)s * (size_t)count * 2 + (size_t)which) * (size_t)width + (size_t)col;
            for (long k = run; k < count; k += 4 * kJoinRuns) {
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = k + i * kJoinRuns < count ? p[(size_t)(k + i * kJoinRuns) * 2 * (size_t)width] : 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += v[i];
            }
        }
        if (first != (long)blockIdx.x * 64) __syncthreads();
        runs[run][lane] = sum;
        __syncthreads();
        if (run || col >= width) continue;
#pragma unroll
        for (int i = 1; i < kJoinRuns; ++i) sum += runs[i][lane];
        store_as(out, type, s * out_sample + col, sum);
    }
}

// ---------------------------------------------------------------------------------
// Host side.  Threads to a row and pieces to a thread: the fewest threads, since a thread's own additions are cheaper than those across
// threads, as long as its elements fit its registers (65536 x 1024 bf16 backward: 64 threads 87 us, 256 threads 106).

struct NormShape {
    int tpr, vpt;        // 0: the wide kernels
    long groups;         // rows that a workgroup holds at once
};

// Elements of a thread that fit: the backward pass holds seven numbers for each, the forward pass four.  In workgroups of 256 threads on
// the backward pass takes eight (65536 x 4096 bf16 on 512 x 8: 310 us; sixteen on 256 threads spill where four waves share a
// SIMD, 529 us, and leave two waves otherwise; 32768 x 8192 on 256 x 32 499 us, on 1024 x 8 314), the forward pass sixteen (eight: 262 us for 244).
constexpr bool norm_fits(bool backward, int tpr, int vpt, int per) { return vpt * per <= (tpr < 256 ? 16 : (backward ? 8 : 16)); }

NormShape norm_shape(bool backward, int type, long width)
{
    const int per = 16 / type_bytes(type);
    const long pieces = (width + per - 1) / per;
    for (int tpr : {16, 64, 256, 512, 1024})
        for (int vpt : {1, 2, 4})
            if (pieces <= (long)tpr * vpt && norm_fits(backward, tpr, vpt, per)) return {tpr, vpt, tpr < kNormBlock ? kNormBlock / tpr : 1};
    return {0, 0, 1};
}

constexpr long kWideRowRuns = 64;

// Workgroups along the rows of a sample: of the backward pass, whose partial sums want few of them.
long norm_backward_blocks(const hot_norm_desc &d)
{
    const NormShape h = norm_shape(true, d.dtype, d.width);
    if (!h.tpr) return d.rows < kWideRowRuns ? (d.rows > 0 ? d.rows : 1) : kWideRowRuns;
    const long want = (d.rows + h.groups - 1) / h.groups;
    const long resident = (h.tpr > 512 ? 1 : (h.tpr > kNormBlock ? 2 : 4)) * (long)kComputeUnits;
    const long most = (resident + d.samples - 1) / d.samples;
    return want < 1 ? 1 : (want < most ? want : most);
}

bool norm_ok(const hot_norm_desc *d)
{
    return d && d->rows >= 0 && d->rows <= (1L << 40) && d->width >= 1 && d->width <= (1L << 31) && d->samples >= 1 && d->samples <= 65535 && known_type(d->dtype) &&
           known_type(d->weight_dtype) && d->ldx >= 0 && d->x_sample >= 0 && d->ldy >= 0 && d->y_sample >= 0 && d->w_sample >= 0 &&
           (d->w_sample == 0 || d->w_sample >= d->width) && d->eps >= 0.0;
}

NormArgs norm_args(const hot_norm_desc &d)
{
    NormArgs a = {};
    a.rows = d.rows;
    a.width = d.width;
    a.ldx = d.ldx;
    a.x_sample = d.x_sample;
    a.w_sample = d.w_sample;
    a.ldy = d.ldy;
    a.y_sample = d.y_sample;
    a.inv_width = (float)(1.0 / (double)d.width);
    a.eps = (float)d.eps;
    a.w_type = d.weight_dtype;
    return a;
}

template <class T, int TPR, int VPT>
void norm_go(bool backward, const NormArgs &a, long blocks, int samples, hipStream_t s)
{
    const dim3 grid((unsigned)blocks, (unsigned)samples), block(TPR > kNormBlock ? TPR : kNormBlock);
    if (backward) {
        if constexpr (norm_fits(true, TPR, VPT, Piece<T>::N)) hot_norm_backward_kernel<T, TPR, VPT><<<grid, block, 0, s>>>(a);
    } else if constexpr (norm_fits(false, TPR, VPT, Piece<T>::N)) hot_norm_forward_kernel<T, TPR, VPT><<<grid, block, 0, s>>>(a);
}

template <class T, int TPR>
void norm_go(int vpt, bool backward, const NormArgs &a, long blocks, int samples, hipStream_t s)
{
    if (vpt == 1) norm_go<T, TPR, 1>(backward, a, blocks, samples, s);
    else if (vpt == 2) norm_go<T, TPR, 2>(backward, a, blocks, samples, s);
    else norm_go<T, TPR, 4>(backward, a, blocks, samples, s);
}

template <class T>
void norm_run(const hot_norm_desc &d, bool backward, const NormArgs &a, hipStream_t s)
{
    const NormShape h = norm_shape(backward, d.dtype, d.width);
    if (!h.tpr) {
        const long most = 4 * (long)kComputeUnits, blocks = d.rows < most ? d.rows : most;
        const dim3 grid((unsigned)blocks, (unsigned)d.samples);
        if (!backward) hot_norm_wide_kernel<T, false><<<grid, kWideBlock, 0, s>>>(a);
        else {
            if (a.out) hot_norm_wide_kernel<T, true><<<grid, kWideBlock, 0, s>>>(a);
            if (a.parts) {
                const long per = (long)kNormBlock * Piece<T>::N;
                hot_norm_wide_weights_kernel<T><<<dim3((unsigned)((d.width + per - 1) / per), (unsigned)norm_backward_blocks(d), (unsigned)d.samples), kNormBlock, 0, s>>>(a);
            }
        }
        return;
    }
    long blocks;
    if (backward) blocks = norm_backward_blocks(d);
    else {
        const long want = (d.rows + h.groups - 1) / h.groups, most = 16 * (long)kComputeUnits;
        blocks = want < most ? want : most;
    }
    if (h.tpr == 16) norm_go<T, 16>(h.vpt, backward, a, blocks, d.samples, s);
    else if (h.tpr == 64) norm_go<T, 64>(h.vpt, backward, a, blocks, d.samples, s);
    else if (h.tpr == 256) norm_go<T, 256>(h.vpt, backward, a, blocks, d.samples, s);
    else if (h.tpr == 512) norm_go<T, 512>(h.vpt, backward, a, blocks, d.samples, s);
    else norm_go<T, 1024>(h.vpt, backward, a, blocks, d.samples, s);
}

void norm_run(const hot_norm_desc &d, bool backward, const NormArgs &a, hipStream_t s)
{
    if (d.dtype == HOT_F32) norm_run<float>(d, backward, a, s);
    else if (d.dtype == HOT_BF16) norm_run<__bf16>(d, backward, a, s);
    else norm_run<_Float16>(d, backward, a, s);
}

}  // namespace

extern "C" {

int hot_norm_forward(const hot_norm_desc *desc, const void *x, const void *weight, const void *bias, void *y, float *mean, float *rstd, void *stream)
{
    if (!norm_ok(desc) || (mean == nullptr) != (rstd == nullptr)) return HOT_EINVAL;
    if (desc->rows == 0) return HOT_OK;
    if (!x || !y || !on_element(x, desc->dtype) || !on_element(y, desc->dtype) || !on_element(weight, desc->weight_dtype) || !on_element(bias, desc->weight_dtype) ||
        !aligned4(mean) || !aligned4(rstd))
        return HOT_EINVAL;
    NormArgs a = norm_args(*desc);
    a.x = x;
    a.w = weight;
    a.b = bias;
    a.out = y;
    a.mean = mean;
    a.rstd = rstd;
    norm_run(*desc, false, a, static_cast<hipStream_t>(stream));
    return hot_detail::note_hip(hipGetLastError());
}

int64_t hot_norm_backward_workspace_bytes(const hot_norm_desc *desc)
{
    if (!norm_ok(desc)) return HOT_EINVAL;
    return norm_backward_blocks(*desc) * desc->samples * 2 * desc->width * 4;
}

int hot_norm_backward(const hot_norm_desc *desc, const void *x, const void *weight, const float *mean, const float *rstd, const void *dy, void *dx,
                      void *grad_weight, void *grad_bias, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (!norm_ok(desc)) return HOT_EINVAL;
    const bool sums = grad_weight || grad_bias;
    if (!on_element(dx, desc->dtype) || !on_element(weight, desc->weight_dtype) || !on_element(grad_weight, desc->weight_dtype) ||
        !on_element(grad_bias, desc->weight_dtype))
        return HOT_EINVAL;
    if (sums && (!workspace || !aligned4(workspace) || workspace_bytes < hot_norm_backward_workspace_bytes(desc))) return HOT_EINVAL;
    if (desc->rows > 0 && (!x || !mean || !rstd || !dy || !on_element(x, desc->dtype) || !on_element(dy, desc->dtype) || !aligned4(mean) || !aligned4(rstd)))
        return HOT_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    NormArgs a = norm_args(*desc);
    a.x = x;
    a.w = weight;
    a.dy = dy;
    a.out = dx;
    a.mean = const_cast<float *>(mean);
    a.rstd = const_cast<float *>(rstd);
    a.parts = sums ? static_cast<float *>(workspace) : nullptr;
    if (desc->rows > 0 && (dx || sums)) norm_run(*desc, true, a, s);
    if (sums) {
        // (no rows: no partial sums to add, which gives zeros)
        const long blocks = desc->rows > 0 ? norm_backward_blocks(*desc) : 0;
        const bool own = desc->w_sample > 0;
        const long columns = (desc->width + 63) / 64;
        hot_norm_join_kernel<<<dim3((unsigned)(columns < kMostJoinBlocks ? columns : kMostJoinBlocks), 2, own ? (unsigned)desc->samples : 1u), 64 * kJoinRuns, 0, s>>>(
            a.parts, own ? blocks : blocks * desc->samples, desc->width, desc->w_sample, desc->weight_dtype, grad_weight, grad_bias);
    }
    return hot_detail::note_hip(hipGetLastError());
}

}  // extern "C"
