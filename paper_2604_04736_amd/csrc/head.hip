// libhot: a linear head's loss over a vocabulary and its gradients, from the features in front of the head, without logits in memory.
//
//   z[r, v] = x[r] . W[v] + b[v],  q = softmax(z / T),  a row's targets are entries (i_j, p_j) with sum p_j = 1:
//   loss[r] = T^2 sum_j p_j (ln p_j - ln q[i_j]) = T^2 (sum_j p_j ln p_j + lse(z / T) - sum_j p_j z[i_j] / T)
//   dz = g T (q - sum_j p_j delta_(i_j)),  dx = dz W,  dW = dz^T x,  db = sum_r dz
// A label is one entry of weight one at T = 1 (the cross entropy); a teacher's top logits t give p = softmax(t / T) over the words listed.
//
// The forward pass multiplies tiles of vocabulary by tiles of rows; a tile leaves per row its largest logit m, its sum of exponentials of (z - m) / T, its
// share of sum_j p_j (z - m) and of sum_j p_j, which a second kernel joins.  Logits are subtracted before anything multiplies them, so that words masked with the
// type's lowest value, or all logits together, may lie anywhere.  The backward pass walks the vocabulary in pieces: it forms a piece's logits again,
// leaves dz of that piece in scratch memory (two 16-bit pieces, or three bf16 pieces of float32) and multiplies it with W and with x.  Its
// products are 2 R V K operations each, one forward and five backward (the two with dz twice over); what bounds them is the matrix pipes from
// some hundred rows on, below that reading W.
// Rows without entries are left out before anything is multiplied, so what they hold (NaN too) reaches no result and costs nothing.
#include <hip/hip_runtime.h>

#include <climits>

#include "hot.h"
#include "vec.h"
#include "element.h"
#include "tile.h"

namespace {

constexpr int kComputeUnits = 256;
constexpr int kMostTop = 1024;           // entries of a row (they are sorted in LDS)
constexpr int kStartStep = 128;          // words between the marks into a row's sorted entries
// fp16: dz is held in units of 2^-15 of a sample's largest gradient (|q - p| <= 1: no overflow), its two pieces in steps of 2^-39 of it
constexpr float kHalfScale = 32768.0f;

inline __host__ __device__ long up(long n, long to) { return (n + to - 1) / to * to; }

// --------------------------------------------------------------------------- a teacher's entries

struct ListArgs {
    long rows;                         // lists = rows x (samples or one)
    long idx_sample, idx_row, logit_sample, logit_row;
    int top, logit_type, marks;        // marks = vocabulary / kStartStep, rounded up
    long vocab;
    float inv_temperature;
    const int64_t *index;
    const void *logit;
    int *word;                         // [lists, top] ascending
    float *weight;                     // [lists, top]
    int *count;                        // [lists]
    double *sums;                      // [lists, 2]: sum p ln p, sum p
    unsigned short *start;             // [lists, marks + 1]: entries below word kStartStep * k
};

constexpr int kListWaves = 4;

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}

__device__ __forceinline__ double wave_total(double v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// One wave to a row: softmax of what is listed, entries of weight zero dropped, the others sorted by word (rank by comparison with all).
// MOST: the longest list that fits (12 bytes of LDS an entry decide how many rows a compute unit has under way).
template <int MOST>
__global__ void __launch_bounds__(64 * kListWaves)
hot_head_lists_kernel(ListArgs a)
{
    __shared__ __attribute__((aligned(16))) int words[kListWaves][MOST], sorted[kListWaves][MOST];
    __shared__ float scaled[kListWaves][MOST];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const long s = blockIdx.y, row = (long)blockIdx.x * kListWaves + wave, list = s * a.rows + row;
    int *const w = words[wave], *const in_order = sorted[wave];
    float *const t = scaled[wave];
    if (row < a.rows) {
        const int64_t *const index = a.index + s * a.idx_sample + row * a.idx_row;
        const long logit0 = s * a.logit_sample + row * a.logit_row;
        float most = -__builtin_inff();
        bool outside = false, nan = false;
        for (int j = lane; j < (a.top + 3 & ~3); j += 64) {
            typedef float F1 __attribute__((ext_vector_type(1)));
            const int64_t i = j < a.top ? index[j] : -1;
            const float v = i < 0 ? -__builtin_inff() : load_as<1, F1>(a.logit, a.logit_type, logit0 + j, logit0 + a.top)[0];
            outside |= i >= a.vocab;
            nan |= v != v;
            most = fmaxf(most, v);
            w[j] = i < 0 || i >= a.vocab ? -1 : (int)i;
            t[j] = v;
        }
        most = wave_max(most);
        // a word outside the vocabulary or a logit that is no number leaves a row that is none; nothing listed, or nothing but -inf, no entries
        const bool broken = __builtin_amdgcn_ballot_w64(outside || nan) != 0 || most == __builtin_inff();
        const bool empty = !broken && most == -__builtin_inff();
        double total = 0.0, entropy = 0.0, sum = 0.0;
        for (int j = lane; j < a.top; j += 64) {
            t[j] = expf((t[j] - most) * a.inv_temperature);         // (in this order: the lowest value of a type, over a small T, is no infinity)
            total += (double)t[j];
        }
        total = wave_total(total);
        for (int j = lane; j < a.top; j += 64) {
            const float p = broken || empty ? 0.0f : (float)((double)t[j] / total);
            if (p > 0.0f) {
                entropy += (double)p * log((double)t[j] / total);
                sum += (double)p;
            } else w[j] = -1;
            t[j] = p;
        }
        entropy = wave_total(entropy);
        sum = wave_total(sum);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        int kept = 0;
        for (int j0 = 0; j0 < a.top; j0 += 64) {
            const int j = j0 + lane, mine = j < a.top ? w[j] : -1;
            kept += __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine >= 0));
            if (mine < 0) continue;
            int rank = 0;
#pragma unroll 4
            for (int k = 0; k < a.top; k += 4) {        // (entries that are not there are -1, as unsigned numbers above all words)
                const i4 q = *reinterpret_cast<const i4 *>(w + k);
#pragma unroll
                for (int i = 0; i < 4; ++i) rank += (unsigned)q[i] < (unsigned)mine || (q[i] == mine && k + i < j);
            }
            in_order[rank] = mine;
            a.word[list * a.top + rank] = mine;
            a.weight[list * a.top + rank] = t[j];
        }
        if (broken) {
            if (lane == 0) {
                in_order[0] = 0;
                a.word[list * a.top] = 0;
                a.weight[list * a.top] = __builtin_nanf("");
            }
            kept = 1;
            entropy = sum = (double)__builtin_nanf("");
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (lane == 0) {
            a.count[list] = kept;
            a.sums[2 * list] = entropy;
            a.sums[2 * list + 1] = sum;
        }
        for (int m = lane; m <= a.marks; m += 64) {
            const int word = m * kStartStep;
            int at = 0, hi = kept;
            while (at < hi) {
                const int mid = (at + hi) >> 1;
                if (in_order[mid] < word) at = mid + 1;
                else hi = mid;
            }
            a.start[list * (a.marks + 1) + m] = (unsigned short)at;
        }
    }
}

// --------------------------------------------------------------------------- the rows that count

// The features' gradients: a run of a piece's words to a workgroup.  A round of workgroups takes its steps of 64 words, and as long as some twenty
// of them for its start and for adding to the sums in memory; of the numbers of runs up to 64 the one with the fewest such steps is taken, by the host for all
// rows (workgroups and sums of that many), and by the device for the rows that count within what the host gave (all passes of
// 900 x 768 x 20000 float32 of which 65 % are left out: 383 -> 357 us, 2048 x 1024 x 30000 bf16, 70 %: 388 -> 337).
struct WordRuns {
    int rows_log, at_once_log;     // rows of a tile and workgroups that run at once, powers of two
    int width_tiles, samples, piece;
    long workgroups, sums;         // of one sample: workgroups, rows of sums
    int *depth;                    // [samples]: words of a run; null in the forward pass
};

__host__ __device__ inline long up_shift(long n, int log) { return (n + (1L << log) - 1) >> log; }

__host__ __device__ inline int run_depth(int piece, int runs) { return (int)(((unsigned)(piece + runs - 1) / (unsigned)runs + 63) & ~63u); }

__host__ __device__ inline bool run_possible(const WordRuns &a, long rows, int runs)
{
    return runs == 1 || (runs * 256 <= a.piece && runs * place_blocks(a.width_tiles, up_shift(rows, a.rows_log)) <= a.workgroups && runs * rows <= a.sums);
}

__host__ __device__ inline long run_steps(const WordRuns &a, long rows, int runs)
{
    return up_shift(up_shift(rows, a.rows_log) * a.width_tiles * a.samples * runs, a.at_once_log) * (run_depth(a.piece, runs) / 64 + 20);
}

// by one wave, a number of runs to a lane
__device__ __forceinline__ void choose_runs(const WordRuns &a, long s, int rows)
{
    const int runs = ((int)threadIdx.x & 63) + 1;
    unsigned long long best = run_possible(a, rows, runs) ? (unsigned long long)run_steps(a, rows, runs) << 6 | (unsigned)(runs - 1) : ~0ull;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const unsigned long long other = __shfl_xor(best, d);
        best = other < best ? other : best;
    }
    if (runs == 1) a.depth[s] = run_depth(a.piece, (int)(best & 63) + 1);
}

// A row's largest logit, as what others are taken from: zero where nothing but -inf is there
__device__ __forceinline__ float level(float most) { return most == -__builtin_inff() ? 0.0f : most; }

// lse = largest / T + ln_sum in 64 bits holds ln_sum to 2^-26 as long as largest / T is below 2^27.  Beyond (every word masked with the lowest value, say) the two
// lie side by side: the float's value times 2^200, and in the 29 bits that a float leaves free in a double 2^24 ln_sum (at most ln 2^24).
constexpr unsigned long long kFreeBits = (1ull << 29) - 1;

__device__ __forceinline__ double put_lse(float largest, double ln_sum, double temperature)
{
    const double at = (double)largest / temperature;
    if (!(__builtin_fabs(at) >= 0x1p27) || __builtin_isinf(largest) || !(ln_sum >= 0.0)) return at + ln_sum;
    return __builtin_bit_cast(double, __builtin_bit_cast(unsigned long long, (double)largest * 0x1p200) | (unsigned long long)(ln_sum * 0x1p24 + 0.5));
}

// (z - base) log2(e) / T - rest is the logarithm to base 2 of a word's probability
__device__ __forceinline__ void get_lse(double lse, double temperature, float &base, float &rest)
{
    constexpr double LOG2E = 1.44269504088896340736;
    if (__builtin_fabs(lse) >= 0x1p160 && __builtin_isfinite(lse)) {
        const unsigned long long bits = __builtin_bit_cast(unsigned long long, lse);
        base = (float)(__builtin_bit_cast(double, bits & ~kFreeBits) * 0x1p-200);
        rest = (float)((double)(bits & kFreeBits) * 0x1p-24 * LOG2E);
        return;
    }
    const double at = lse * temperature;
    base = (float)at;
    rest = __builtin_isfinite(base) ? (float)((at - (double)base) * LOG2E / temperature) : 0.0f;
}

struct RowArgs {
    long rows, vocab;
    double temperature;
    long idx_sample, idx_row;
    int64_t ignore;
    const int64_t *index;          // labels, or
    const int *list_count;         // entries of every list
    long list_sample;              // lists between samples
    const double *lse;             // backward: [samples, rows] and the gradients of the losses
    const float *g;
    long g_sample, g_row;
    float scale_to;                // what the largest gradient is held as
    int *count;                    // [samples]
    int *row_of, *place_of;        // [samples, rows]: the row at a place, the place of a row (-1: left out)
    int *label;                    // [samples, rows] by place (-1: no word)
    float *base, *rest, *grad;     // by place: lse as get_lse gives it, the row's gradient
    float *scale;                  // [samples, 2]: what gradients are multiplied with, and what results are multiplied with in turn
    WordRuns runs;
};

// The rows of sample s that count, in order: how many, and (WRITE) the arrays by place.  `map` (LDS, rows of them, or null): the row at a place.
template <int BLOCK, bool WRITE>
__device__ __forceinline__ int find_rows(const RowArgs &a, long s, unsigned short *map)
{
    __shared__ int totals[2][BLOCK / 64];
    __shared__ float most[BLOCK / 64];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const long base = s * a.rows;
    int before = 0, turn = 0;
    float largest = 0.0f;
    for (long r0 = 0; r0 < a.rows; r0 += BLOCK) {
        const long row = r0 + threadIdx.x;
        bool counts = false;
        int label = -1;
        if (row < a.rows) {
            if (a.list_count) counts = a.list_count[s * a.list_sample + row] > 0;
            else {
                const int64_t t = a.index[s * a.idx_sample + row * a.idx_row];
                counts = t != a.ignore;
                label = t >= 0 && t < a.vocab ? (int)t : -1;
            }
        }
        const unsigned long long mask = __builtin_amdgcn_ballot_w64(counts);
        if (lane == 0) totals[turn][wave] = __builtin_popcountll(mask);
        __syncthreads();
        int at = before + __builtin_popcountll(mask & ((1ull << lane) - 1));
#pragma unroll
        for (int i = 0; i < BLOCK / 64; ++i) {
            if (i < wave) at += totals[turn][i];
            before += totals[turn][i];
        }
        turn ^= 1;
        if (row < a.rows && counts && map) map[at] = (unsigned short)row;
        if constexpr (WRITE)
            if (row < a.rows) {
                a.place_of[base + row] = counts ? at : -1;
                if (counts) {
                    a.row_of[base + at] = (int)row;
                    if (a.label) a.label[base + at] = label;
                    if (a.lse) {
                        get_lse(a.lse[base + row], a.temperature, a.base[base + at], a.rest[base + at]);
                        float g = a.g[s * a.g_sample + row * a.g_row];
                        if (!a.list_count && label < 0) g = __builtin_nanf("");
                        a.grad[base + at] = g;
                        largest = fmaxf(largest, __builtin_fabsf(g));
                    }
                }
            }
    }
    if constexpr (WRITE) {
        if (threadIdx.x == 0) a.count[s] = before;
        if (wave == 0 && a.runs.depth) choose_runs(a.runs, s, before);
        if (a.lse) {
            largest = wave_max(largest);
            if (lane == 0) most[wave] = largest;
            __syncthreads();
            if (threadIdx.x == 0) {
#pragma unroll
                for (int i = 0; i < BLOCK / 64; ++i) largest = fmaxf(largest, most[i]);
                // (where that factor would leave the normal numbers, and where nothing but zeros or infinities come in, it is scale_to)
                const float by = a.scale_to / largest;
                const bool usable = by >= 0x1p-126f && by <= 0x1p127f;
                a.scale[2 * s] = usable ? by : a.scale_to;
                a.scale[2 * s + 1] = usable ? largest / a.scale_to : 1.0f / a.scale_to;
            }
        }
    }
    return before;
}

constexpr int kRowBlock = 1024;

__global__ void __launch_bounds__(kRowBlock) hot_head_rows_kernel(RowArgs a) { find_rows<kRowBlock, true>(a, blockIdx.x, nullptr); }

// --------------------------------------------------------------------------- operands as the tiles read them

struct PackArgs {
    const void *from;
    long from_row, from_sample;    // elements
    const int *row_of;             // [samples, rows] or null: rows as they are
    const int *count;              // with row_of: how many of them
    long rows;
    int width;
    char *to;                      // [samples], pieces `plane` apart: blocks of `columns` columns, each all rows
    long to_sample, plane, block;
    int columns;
};

// Workgroup `first` of `blocks`.  A wave packs a run of rows of one block of columns: what it writes is one run of memory.
template <class T>
__device__ __forceinline__ void pack(const PackArgs &a, long s, long n, const unsigned short *map, long first, long blocks)
{
    const int per_row = a.columns / 8, in_block = (int)threadIdx.x % per_row;
    const int column_blocks = (a.width + a.columns - 1) / a.columns;
    const long rows_at_once = 256 / per_row, row_groups = (n + rows_at_once - 1) / rows_at_once, items = row_groups * column_blocks;
    for (long item = first; item < items; item += blocks) {
        const long place = item / column_blocks * rows_at_once + threadIdx.x / per_row, block = item % column_blocks;
        const int col = (int)block * a.columns + in_block * 8;
        if (place >= n || col >= a.width) continue;
        const long row = map ? map[place] : (a.row_of ? a.row_of[s * a.rows + place] : place);
        const T *const from = static_cast<const T *>(a.from) + (size_t)s * (size_t)a.from_sample + (size_t)row * (size_t)a.from_row;
        char *const to = a.to + (size_t)s * (size_t)a.to_sample + (size_t)block * (size_t)a.block + ((size_t)place * (size_t)per_row + (size_t)in_block) * 16;
        if constexpr (sizeof(T) == 2) {
            typedef T V __attribute__((ext_vector_type(8)));
            *reinterpret_cast<V *>(to) = Piece<T>::take(from, col, a.width);
        } else {
            typedef __bf16 V __attribute__((ext_vector_type(8)));
            V p[3];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const typename Piece<T>::F v = Piece<T>::load(from, col + 4 * h, a.width);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    __bf16 q[3];
                    split_bf16(v[j], q);
#pragma unroll
                    for (int i = 0; i < 3; ++i) p[i][4 * h + j] = q[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 3; ++i) *reinterpret_cast<V *>(to + (size_t)i * (size_t)a.plane) = p[i];
        }
    }
}

template <class T>
__global__ void __launch_bounds__(256) hot_head_pack_kernel(PackArgs a)
{
    const long s = blockIdx.y;
    pack<T>(a, s, a.row_of ? a.count[s] : a.rows, nullptr, blockIdx.x, gridDim.x);
}

// Up to kFewRows rows: rows found, features packed and (the first piece's) weights packed in one launch.  Every workgroup that packs
// features finds the rows by itself; the first one writes them down.
constexpr int kFewRows = 1024;

template <class T>
__global__ void __launch_bounds__(256) hot_head_prepare_kernel(RowArgs rows, PackArgs x, PackArgs w, int x_blocks)
{
    __shared__ unsigned short map[kFewRows];
    const long s = blockIdx.y;
    if ((int)blockIdx.x >= x_blocks) return pack<T>(w, s, w.rows, nullptr, (int)blockIdx.x - x_blocks, (int)gridDim.x - x_blocks);
    const int count = blockIdx.x == 0 ? find_rows<256, true>(rows, s, map) : find_rows<256, false>(rows, s, map);
    __syncthreads();
    pack<T>(x, s, count, map, blockIdx.x, x_blocks);
}

// --------------------------------------------------------------------------- logits: statistics, or their gradients

struct HeadArgs {
    Matrix w, x;                   // 16-bit elements; w begins at word v_begin
    long w_sample, x_sample;       // bytes
    int width;
    int vocab, v_begin, v_count;   // the piece of the vocabulary
    long rows, places;             // rows a sample, and that rounded up to 256
    const int *count, *row_of, *label;
    const void *bias;
    long bias_sample;
    int bias_type;
    float scale;                   // log2(e) / temperature
    // a teacher's entries
    const int *word;
    const float *weight;
    const unsigned short *start;
    int top, marks;
    long list_sample;
    // forward: partials[sample][tile][4][place]
    float *partials;
    int v_tiles;
    // backward
    const float *base, *rest, *grad, *to_scale;
    char *dz;                      // [sample] blocks of BK words, each all places
    long dz_block, dz_plane, dz_sample;
    float *sums;                   // for db, or null: dz summed over a tile's rows, [sample][tile of rows][word of the piece]
    int row_tiles, v_piece;
};

// This lane's rows (one in each block of 32) and where their targets are, read before the product so that nothing waits for them behind it.
template <class TILE, bool LISTS>
struct Rows {
    bool live[TILE::NB];
    int place[TILE::NB];
    int word[TILE::NB];            // the label, or the first entry in the tile
    float weight[TILE::NB];
    long entry[TILE::NB];          // of the list
    int left[TILE::NB];
    float covered[TILE::NB];       // weight of the targets that targets() met in this wave's words

    __device__ __forceinline__ Rows(const HeadArgs &a, long s, int count, int v0, int r0)
    {
#pragma unroll
        for (int n = 0; n < TILE::NB; ++n) {
            place[n] = r0 + TILE::n0() + 32 * n + (TILE::lane() & 31);
            live[n] = place[n] < count;
            word[n] = -1;
            weight[n] = 0.0f;
            entry[n] = 0;
            left[n] = 0;
            covered[n] = 0.0f;
            if (!live[n]) continue;
            if constexpr (!LISTS) word[n] = a.label[s * a.rows + place[n]];
            else {
                const long list = s * a.list_sample + a.row_of[s * a.rows + place[n]];
                const unsigned short *const start = a.start + list * (a.marks + 1);
                // (a tile of 64 words walks the entries of its neighbour too, which match none of its results)
                const int mark = v0 / kStartStep, last = (v0 + TILE::BM + kStartStep - 1) / kStartStep, first = start[mark];
                entry[n] = list * a.top + first;
                left[n] = start[last < a.marks ? last : a.marks] - first;
                if (left[n] > 0) {
                    word[n] = a.word[entry[n]];
                    weight[n] = a.weight[entry[n]];
                }
            }
        }
    }

    // f(n, m, i, mine, weight) for every result (m, n, i) of the wave that some lane's target may be; `mine` where it is this lane's
    template <class F>
    __device__ __forceinline__ void targets(const HeadArgs &a, int v0, const F &f)
    {
        const int first = v0 + TILE::m0(), low = 4 * (TILE::lane() >> 5);
#pragma unroll
        for (int n = 0; n < TILE::NB; ++n) {
            auto meet = [&](int in, float w) {
                covered[n] += in >= 0 && in < TILE::WM ? w : 0.0f;
#pragma unroll
                for (int m = 0; m < TILE::MB; ++m) {
                    if (__builtin_amdgcn_ballot_w64(in >= 32 * m && in < 32 * m + 32) == 0) continue;
#pragma unroll
                    for (int i = 0; i < 16; ++i) f(n, m, i, in - low == 32 * m + 8 * (i >> 2) + (i & 3), w);
                }
            };
            if constexpr (!LISTS) meet(word[n] - first, 1.0f);
            else
                while (__builtin_amdgcn_ballot_w64(left[n] > 0) != 0) {
                    const int in = left[n] > 0 ? word[n] - first : -1;
                    const float w = weight[n];
                    ++entry[n];
                    if (--left[n] > 0) {
                        word[n] = a.word[entry[n]];
                        weight[n] = a.weight[entry[n]];
                    }
                    meet(in, w);
                }
        }
    }
};

// The bias of a tile's words, -inf for words beyond the vocabulary: loaded before the product, added behind it; most tiles have neither
template <class TILE>
__device__ __forceinline__ bool ask_bias(const HeadArgs &a, long s, int v0, float *bias)
{
    if (!a.bias && v0 + TILE::BM <= a.vocab) return false;
    for (int i = (int)threadIdx.x; i < TILE::BM; i += TILE::THREADS) {
        typedef float F1 __attribute__((ext_vector_type(1)));
        const int v = v0 + i;
        float b = v < a.vocab ? 0.0f : -__builtin_inff();
        if (a.bias && v < a.vocab) b = load_as<1, F1>(a.bias, a.bias_type, s * a.bias_sample + v, s * a.bias_sample + a.vocab)[0];
        bias[i] = b;
    }
    return true;
}

template <class TILE>
__device__ __forceinline__ void add_bias(const float *bias, f16v (&acc)[TILE::MB][TILE::NB])
{
#pragma unroll
    for (int m = 0; m < TILE::MB; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float b = bias[TILE::m0() + 32 * m + TILE::row(i)];
#pragma unroll
            for (int n = 0; n < TILE::NB; ++n) acc[m][n][i] += b;
        }
}

__device__ __forceinline__ Matrix part(const Matrix &m, long bytes) { return {m.at + bytes, m.pitch, m.block, m.plane}; }

// where a workgroup's tile of logits begins
struct TileOf {
    bool any;
    int v0, r0;
};

template <class TILE>
__device__ __forceinline__ TileOf tile_of(const HeadArgs &a, int count)
{
    const Place at = place((a.v_count + TILE::BM - 1) / TILE::BM, (count + TILE::BN - 1) / TILE::BN);
    return {at.any, a.v_begin + at.m * TILE::BM, at.n * TILE::BN};
}

template <class TILE>
__device__ __forceinline__ void logits(const HeadArgs &a, char *lds, float *bias, long s, int count, const TileOf &t, f16v (&acc)[TILE::MB][TILE::NB])
{
    const bool biased = ask_bias<TILE>(a, s, t.v0, bias);
    const Operand w = {part(a.w, s * a.w_sample + (t.v0 - a.v_begin) * a.w.pitch), a.v_begin + a.v_count - t.v0, a.width};
    const Operand x = {part(a.x, s * a.x_sample + t.r0 * a.x.pitch), count - t.r0, a.width};
    TILE::product((lds_char *)lds, w, x, a.width, acc);        // (with barriers between the writing of the bias and this)
    if (biased) add_bias<TILE>(bias, acc);
}

template <class TILE, bool LISTS>
__global__ void __launch_bounds__(TILE::THREADS)
hot_head_forward_kernel(HeadArgs a)
{
    constexpr int NEED = 4 * TILE::WAVES_M * TILE::BN * 4;
    // (one array: beside a second one the compiler would wait for every load in flight before it reads either)
    constexpr int ROOM = TILE::kLds > NEED ? TILE::kLds : NEED;
    __shared__ __attribute__((aligned(1024))) char memory[ROOM + TILE::BM * 4];
    const long s = blockIdx.y;
    const int count = a.count[s];
    const TileOf tile = tile_of<TILE>(a, count);
    if (!tile.any) return;
    Rows<TILE, LISTS> rows(a, s, count, tile.v0, tile.r0);
    f16v acc[TILE::MB][TILE::NB];
    logits<TILE>(a, memory, reinterpret_cast<float *>(memory + ROOM), s, count, tile, acc);
    const int r0 = tile.r0, v0 = tile.v0;
    float most[TILE::NB], dot[TILE::NB] = {};
#pragma unroll
    for (int n = 0; n < TILE::NB; ++n) {
        most[n] = acc[0][n][0];
#pragma unroll
        for (int m = 0; m < TILE::MB; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) most[n] = fmaxf(most[n], acc[m][n][i]);
        most[n] = fmaxf(most[n], __shfl_xor(most[n], 32));
        const float from = level(most[n]);        // (nothing but -inf: a sum of zero)
#pragma unroll
        for (int m = 0; m < TILE::MB; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][n][i] -= from;
    }
    rows.targets(a, v0, [&](int n, int m, int i, bool mine, float weight) { dot[n] += mine ? weight * acc[m][n][i] : 0.0f; });
    float (*const part)[TILE::WAVES_M][TILE::BN] = reinterpret_cast<float (*)[TILE::WAVES_M][TILE::BN]>(memory);
#pragma unroll
    for (int n = 0; n < TILE::NB; ++n) {
        float sum = 0.0f;
#pragma unroll
        for (int m = 0; m < TILE::MB; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f(acc[m][n][i] * a.scale);
        sum += __shfl_xor(sum, 32);
        dot[n] += __shfl_xor(dot[n], 32);
        if (TILE::lane() < 32) {
            const int wm = TILE::wave() / TILE::WAVES_N, col = TILE::n0() + 32 * n + TILE::lane();
            part[0][wm][col] = most[n];
            part[1][wm][col] = sum;
            part[2][wm][col] = dot[n];
            part[3][wm][col] = rows.covered[n];
        }
    }
    __syncthreads();
    for (int col = (int)threadIdx.x; col < TILE::BN; col += TILE::THREADS) {
        if (r0 + col >= count) break;
        float top = part[0][0][col];
#pragma unroll
        for (int k = 1; k < TILE::WAVES_M; ++k) top = fmaxf(top, part[0][k][col]);
        float sum = 0.0f, d = 0.0f, covered = 0.0f;
#pragma unroll
        for (int k = 0; k < TILE::WAVES_M; ++k) {
            const float m = part[0][k][col], w = part[3][k][col];
            // (a largest logit of -inf: a sum of zero, or none where a logit is no number)
            sum += m == -__builtin_inff() ? part[1][k][col] : part[1][k][col] * __builtin_amdgcn_exp2f((m - top) * a.scale);
            d += part[2][k][col] + (w > 0.0f ? w * (level(m) - level(top)) : 0.0f);
            covered += w;
        }
        float *const out = a.partials + (((size_t)s * (size_t)a.v_tiles + (size_t)(v0 / TILE::BM)) * 4) * (size_t)a.places + (size_t)(r0 + col);
        out[0] = top;
        out[a.places] = sum;
        out[2 * a.places] = d;
        out[3 * a.places] = covered;
    }
}

// A product that is rounded to float32 wherever it is used.  (The compiler fuses a product with the conversion of the result to fp16, in one of its uses:
// the first piece was then rounded once, and the second formed from what a piece rounded twice left, near the middle of two numbers another one.)
__device__ __forceinline__ float rounded_product(float a, float b)
{
    float v = a * b;
    asm volatile("" : "+v"(v));
    return v;
}

template <class TILE, bool LISTS, int PIECES>
__global__ void __launch_bounds__(TILE::THREADS)
hot_head_dz_kernel(HeadArgs a)
{
    constexpr int PITCH = TILE::BM * 2 + 16;       // (16 bytes on: rows of a column of lanes lie in different banks)
    constexpr int ROWS = TILE::WAVES_N * 32, NEED = PIECES * ROWS * PITCH;
    // (one array: beside a second one the compiler would wait for every load in flight before it reads either)
    constexpr int ROOM = TILE::kLds > NEED ? TILE::kLds : NEED;
    __shared__ __attribute__((aligned(1024))) char memory[ROOM + TILE::BM * 4];
    const long s = blockIdx.y;
    const int count = a.count[s];
    const TileOf tile = tile_of<TILE>(a, count);
    if (!tile.any) return;
    Rows<TILE, LISTS> rows(a, s, count, tile.v0, tile.r0);
    float base[TILE::NB], rest[TILE::NB], g[TILE::NB];
    const float to_scale = a.to_scale[2 * s];
#pragma unroll
    for (int n = 0; n < TILE::NB; ++n) {
        const long at = s * a.rows + rows.place[n];
        base[n] = rows.live[n] ? a.base[at] : __builtin_inff();
        rest[n] = rows.live[n] ? a.rest[at] : 0.0f;
        g[n] = rows.live[n] ? a.grad[at] * to_scale : 0.0f;
    }
    f16v acc[TILE::MB][TILE::NB];
    logits<TILE>(a, memory, reinterpret_cast<float *>(memory + ROOM), s, count, tile, acc);
    const int v0 = tile.v0, r0 = tile.r0;
#pragma unroll
    for (int m = 0; m < TILE::MB; ++m)
#pragma unroll
        for (int n = 0; n < TILE::NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[m][n][i] - base[n], a.scale, -rest[n]));
    rows.targets(a, v0, [&](int n, int m, int i, bool mine, float weight) { acc[m][n][i] -= mine ? weight : 0.0f; });
    // to rows of words through LDS, all pieces of a block of rows of every wave at once
    typedef typename TILE::T T;
    typedef T V4 __attribute__((ext_vector_type(4)));
    typedef T V8 __attribute__((ext_vector_type(8)));
    constexpr int BK = TILE::BK, PAIRS = TILE::BM / 2, RUNS = TILE::THREADS / PAIRS, CHUNKS = TILE::BM / 8;
    float sum[2] = {0.0f, 0.0f};
    char *const out = a.dz + (size_t)s * (size_t)a.dz_sample + (size_t)((v0 - a.v_begin) / BK) * (size_t)a.dz_block + (size_t)r0 * (BK * 2);
    const int mine = TILE::n0() / TILE::WN * 32 + (TILE::lane() & 31);
#pragma unroll
    for (int n = 0; n < TILE::NB; ++n) {
        if (n) __syncthreads();
#pragma unroll
        for (int m = 0; m < TILE::MB; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                V4 o[PIECES];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = rounded_product(acc[m][n][4 * q + i], g[n]);
#pragma unroll
                    for (int p = 0; p < PIECES; ++p) {
                        o[p][i] = (T)v;
                        v = __builtin_isfinite((float)o[p][i]) ? v - (float)o[p][i] : 0.0f;
                    }
                }
#pragma unroll
                for (int p = 0; p < PIECES; ++p) *reinterpret_cast<V4 *>(memory + (p * ROWS + mine) * PITCH + (TILE::m0() + 32 * m + TILE::row(4 * q)) * 2) = o[p];
            }
        __syncthreads();
#pragma unroll 4
        for (int k = (int)threadIdx.x; k < PIECES * ROWS * CHUNKS; k += TILE::THREADS) {
            const int p = k / (ROWS * CHUNKS), block = k / (ROWS * BK / 8) % (TILE::BM / BK), in = k % (ROWS * BK / 8), row = in / (BK / 8), chunk = in % (BK / 8);
            *reinterpret_cast<V8 *>(out + (size_t)p * (size_t)a.dz_plane + (size_t)block * (size_t)a.dz_block + (row / 32 * TILE::WN + 32 * n + row % 32) * (BK * 2) + chunk * 16) =
                *reinterpret_cast<const V8 *>(memory + (p * ROWS + row) * PITCH + block * (BK * 2) + chunk * 16);
        }
        if (a.sums) {       // two words to a thread, a run of rows each
            typedef T V2 __attribute__((ext_vector_type(2)));
            const int pair = (int)threadIdx.x % PAIRS, run = (int)threadIdx.x / PAIRS;
#pragma unroll 8
            for (int r = run; r < PIECES * ROWS; r += RUNS) {
                const V2 v = *reinterpret_cast<const V2 *>(memory + r * PITCH + pair * 4);
                sum[0] += (float)v[0];
                sum[1] += (float)v[1];
            }
        }
    }
    if (!a.sums) return;
    __syncthreads();
    float (*const runs)[TILE::BM] = reinterpret_cast<float (*)[TILE::BM]>(memory);
    const int pair = (int)threadIdx.x % PAIRS;
    runs[threadIdx.x / PAIRS][2 * pair] = sum[0];
    runs[threadIdx.x / PAIRS][2 * pair + 1] = sum[1];
    __syncthreads();
    for (int i = (int)threadIdx.x; i < TILE::BM; i += TILE::THREADS) {
        float total = 0.0f;
#pragma unroll
        for (int k = 0; k < RUNS; ++k) total += runs[k][i];
        a.sums[((size_t)s * (size_t)a.row_tiles + (size_t)(r0 / TILE::BN)) * (size_t)a.v_piece + (size_t)(v0 - a.v_begin + i)] = total;
    }
}

// --------------------------------------------------------------------------- joining a row's partial statistics

struct JoinArgs {
    long rows, places;
    int tiles, lanes;              // lanes: threads to a row
    float scale;                   // log2(e) / temperature
    const float *partials;
    const int *place_of, *label;
    const double *sums;            // of the lists, or null
    long list_sample;
    double temperature;
    float *loss;
    double *lse;
};

// What some of a row's words leave: largest logit, sum of exp2((z - most) scale), sum of p (z - most), sum of p
template <class SUM>
struct Share {
    float most;
    SUM sum;
    double dot, covered;

    template <class OTHER>
    __device__ __forceinline__ void join(const Share<OTHER> &o, float scale)
    {
        const float top = o.most > most || o.most != o.most ? o.most : most;
        const SUM there = (SUM)o.sum;
        sum = top == -__builtin_inff() ? sum + there : sum * (SUM)__builtin_amdgcn_exp2f((most - top) * scale) + there * (SUM)__builtin_amdgcn_exp2f((o.most - top) * scale);
        dot = moved(dot, covered, most, top) + moved(o.dot, o.covered, o.most, top);
        covered += o.covered;
        most = top;
    }
    static __device__ __forceinline__ double moved(double dot, double covered, float from, float to)
    {
        return covered > 0.0 ? dot + covered * ((double)level(from) - (double)level(to)) : dot;
    }
};

__global__ void __launch_bounds__(256)
hot_head_join_kernel(JoinArgs a)
{
    __shared__ Share<double> shares[256];
    const int per = 256 / a.lanes, r = (int)threadIdx.x % per, lane = (int)threadIdx.x / per;
    const long s = blockIdx.y, row = (long)blockIdx.x * per + r;
    const int at = row < a.rows ? a.place_of[s * a.rows + row] : -1;
    Share<float> mine = {-__builtin_inff(), 0.0f, 0.0, 0.0};
    if (at >= 0)
#pragma unroll 4
        for (int k = lane; k < a.tiles; k += a.lanes) {
            const float *const p = a.partials + ((size_t)s * (size_t)a.tiles + (size_t)k) * 4 * (size_t)a.places + (size_t)at;
            mine.join(Share<float>{p[0], p[a.places], (double)p[2 * a.places], (double)p[3 * a.places]}, a.scale);
        }
    Share<double> all = {mine.most, (double)mine.sum, mine.dot, mine.covered};
    // the row's threads, in halves
    for (int half = a.lanes / 2; half > 0; half /= 2) {
        if (lane >= half && lane < 2 * half) shares[threadIdx.x] = all;
        __syncthreads();
        if (lane < half) all.join(shares[(int)threadIdx.x + half * per], a.scale);
        __syncthreads();
    }
    if (lane || row >= a.rows) return;
    float loss = 0.0f;
    double lse = 0.0;
    if (at >= 0) {
        const double ln_sum = log2(all.sum) * 0.69314718055994530942;
        lse = put_lse(all.most, ln_sum, a.temperature);
        double entropy = 0.0, weight = 1.0;
        if (a.sums) {
            const long list = s * a.list_sample + row;
            entropy = a.sums[2 * list];
            weight = a.sums[2 * list + 1];
        } else if (a.label[s * a.rows + at] < 0) entropy = (double)__builtin_nanf("");
        loss = (float)(a.temperature * a.temperature * (entropy + weight * ln_sum - all.dot / a.temperature));
    }
    a.loss[s * a.rows + row] = loss;
    if (a.lse) a.lse[s * a.rows + row] = lse;
}

// --------------------------------------------------------------------------- gradients of features, weights and bias

struct GradArgs {
    Matrix dz, other;              // other: W (from word v_begin) or the packed features
    long dz_sample, sample;
    int width, v_begin, v_count;
    const int *count;
    WordRuns runs;                 // of words
    bool first;                    // of the pieces: sums begin with it
    float *sums;                   // dx: [sample], its runs.sums rows: [run][place][width]
    void *out;                     // dW, or its partial sums: [run of rows] out_split apart, [sample], words from out_first on
    long out_sample, out_split;
    int out_first, row_depth;      // rows of a run
    const float *scale;            // [samples, 2]
    float temperature;
};

// dx's share of one piece of the vocabulary (and of one run of it): rows x width, contracted over words
template <class TILE>
__global__ void __launch_bounds__(TILE::THREADS)
hot_head_dx_kernel(GradArgs a)
{
    __shared__ __attribute__((aligned(1024))) char memory[TILE::kLds];
    const long s = blockIdx.y;
    const int count = a.count[s], each = a.runs.depth[s], k_tiles = (a.width + TILE::BN - 1) / TILE::BN, r_tiles = (count + TILE::BM - 1) / TILE::BM;
    if (count == 0) return;
    const int id = (int)(blockIdx.x + gridDim.x * blockIdx.z), tiles = (int)place_blocks(k_tiles, r_tiles), run = id / tiles;
    const Place at = place(k_tiles, r_tiles, id - run * tiles, (int)blockIdx.y + run * (int)gridDim.y);
    if (run >= (a.runs.piece + each - 1) / each || !at.any) return;
    const int r0 = at.n * TILE::BM, k0 = at.m * TILE::BN, v = run * each, depth = a.v_count - v < each ? a.v_count - v : each;
    f16v acc[TILE::MB][TILE::NB];
    const Operand dz = {part(a.dz, s * a.dz_sample + v / TILE::BK * a.dz.block + r0 * a.dz.pitch), count - r0, depth};
    const Operand w = {part(a.other, s * a.sample + v * a.other.pitch + k0 / TILE::BK * a.other.block), a.width - k0, depth};
    TILE::product((lds_char *)memory, dz, w, depth, acc);
    float *const sums = a.sums + ((size_t)s * (size_t)a.runs.sums + (size_t)run * (size_t)count) * (size_t)a.width;
#pragma unroll
    for (int m = 0; m < TILE::MB; ++m)
#pragma unroll
        for (int n = 0; n < TILE::NB; ++n) {
            const int k = k0 + TILE::n0() + 32 * n + (TILE::lane() & 31);
            if (k >= a.width) continue;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = r0 + TILE::m0() + 32 * m + TILE::row(i);
                if (r >= count) continue;
                float *const p = sums + (size_t)r * (size_t)a.width + (size_t)k;
                *p = a.first ? acc[m][n][i] : *p + acc[m][n][i];
            }
        }
}

// dW of one piece of the vocabulary: words x width, contracted over rows.  M = width, so that a lane's neighbouring results are
// neighbours in memory; OUT: the type of W.
template <class TILE, class OUT>
__global__ void __launch_bounds__(TILE::THREADS)
hot_head_dw_kernel(GradArgs a)
{
    constexpr int PITCH = TILE::BM * (int)sizeof(OUT) + 16, NEED = TILE::BN * PITCH;
    __shared__ __attribute__((aligned(1024))) char memory[TILE::kLds > NEED ? TILE::kLds : NEED];
    const long s = blockIdx.y;
    const int count = a.count[s];
    const Place at = place((a.v_count + TILE::BN - 1) / TILE::BN, (a.width + TILE::BM - 1) / TILE::BM);
    if (!at.any) return;
    const int in = at.m * TILE::BN, k0 = at.n * TILE::BM;
    f16v acc[TILE::MB][TILE::NB];
    const int r0 = (int)blockIdx.z * a.row_depth, left = count - r0, depth = left < 0 ? 0 : (left < a.row_depth ? left : a.row_depth);
    const Operand x = {part(a.other, s * a.sample + k0 / TILE::BK * a.other.block + r0 * a.other.pitch), a.width - k0, depth};
    const Operand dz = {part(a.dz, s * a.dz_sample + in / TILE::BK * a.dz.block + r0 * a.dz.pitch), a.v_count - in, depth};
    TILE::product((lds_char *)memory, x, dz, depth, acc);
    const float scale = a.scale[2 * s + 1] * a.temperature;
    typedef OUT V4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int n = 0; n < TILE::NB; ++n)
#pragma unroll
        for (int m = 0; m < TILE::MB; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                V4 o;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = (OUT)(acc[m][n][4 * q + i] * scale);
                *reinterpret_cast<V4 *>(memory + (TILE::n0() + 32 * n + (TILE::lane() & 31)) * PITCH + (TILE::m0() + 32 * m + TILE::row(4 * q)) * (int)sizeof(OUT)) = o;
            }
    __syncthreads();
    constexpr int N = Piece<OUT>::N, CHUNKS = TILE::BM / N;
    OUT *const out = static_cast<OUT *>(a.out) + (size_t)blockIdx.z * (size_t)a.out_split + (size_t)s * (size_t)a.out_sample + (size_t)(a.out_first + in) * (size_t)a.width;
    for (int k = (int)threadIdx.x; k < TILE::BN * CHUNKS; k += TILE::THREADS) {
        const int row = k / CHUNKS, col = k0 + k % CHUNKS * N;
        if (in + row >= a.v_count || col >= a.width) continue;
        OUT *const to = out + (size_t)row * (size_t)a.width;
        const typename Piece<OUT>::V v = *reinterpret_cast<const typename Piece<OUT>::V *>(memory + row * PITCH + k % CHUNKS * 16);
        if (col + N <= a.width) *reinterpret_cast<typename Piece<OUT>::Loose *>(to + col) = v;
        else
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (col + j < a.width) to[col + j] = v[j];
    }
}

// dW of one piece from the partial sums of its runs of rows
struct RunArgs {
    const float *parts;            // [run][sample][words of the piece][width]
    long words_width, part_sample, part_run, out_sample;
    int runs;
    void *out;                     // from the piece's first word on
};

template <class T>
__global__ void __launch_bounds__(256) hot_head_runs_kernel(RunArgs a)
{
    constexpr int N = Piece<T>::N;
    const long s = blockIdx.y, items = (a.words_width + N - 1) / N;
    for (long item = (long)blockIdx.x * 256 + threadIdx.x; item < items; item += (long)gridDim.x * 256) {
        typename Piece<T>::F sum = typename Piece<T>::F(0.0f);
        for (int k = 0; k < a.runs; ++k) {
            const float *const p = a.parts + (size_t)k * (size_t)a.part_run + (size_t)s * (size_t)a.part_sample;
#pragma unroll
            for (int h = 0; h < N; h += 4) {
                const Piece<float>::F v = Piece<float>::load(p, item * N + h, a.words_width);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[h + j] += v[j];
            }
        }
        Piece<T>::store(static_cast<T *>(a.out) + (size_t)s * (size_t)a.out_sample, item * N, a.words_width, sum);
    }
}

// db of one piece: the sums of its tiles of rows added up
struct BiasArgs {
    const float *sums;
    int row_tiles, tile_rows, v_piece, v_begin, v_count;
    const int *count;
    const float *scale;
    float temperature;
    void *out;
    long out_sample;
    int type;
};

__device__ __forceinline__ void bias_gradient(const BiasArgs &a, long s, int first)
{
    const int word = first * 256 + (int)threadIdx.x, tiles = (a.count[s] + a.tile_rows - 1) / a.tile_rows;
    if (word >= a.v_count) return;
    float total = 0.0f;
#pragma unroll 8
    for (int k = 0; k < tiles; ++k) total += a.sums[((size_t)s * (size_t)a.row_tiles + (size_t)k) * (size_t)a.v_piece + (size_t)word];
    store_as(a.out, a.type, s * a.out_sample + a.v_begin + word, total * (a.scale[2 * s + 1] * a.temperature));
}

struct FeatureArgs {
    const float *sums;             // as above
    const int *place_of, *count;
    WordRuns runs;
    const float *scale;
    float temperature;
    long rows, width;
    int samples;
    bool shared;                   // all samples have the same features: their gradients are added
    void *out;
};

// dx: the sums of its runs of words, at the rows' own places, and zeros for the rows that were left out
template <class T>
__device__ __forceinline__ void feature_gradient(const FeatureArgs &a, long sample, long first, long blocks)
{
    constexpr int N = Piece<T>::N;
    if (a.shared && sample > 0) return;
    const long chunks = (a.width + N - 1) / N, items = a.rows * chunks;
    for (long item = first * 256 + threadIdx.x; item < items; item += blocks * 256) {
        const long row = item / chunks, col = (item - row * chunks) * N;
        const long s0 = a.shared ? 0 : sample, s1 = a.shared ? a.samples : s0 + 1;
        typename Piece<T>::F total = typename Piece<T>::F(0.0f);
        for (long s = s0; s < s1; ++s) {
            const int at = a.place_of[s * a.rows + row];
            if (at < 0) continue;
            typename Piece<T>::F sum = typename Piece<T>::F(0.0f);
            const int runs = (a.runs.piece + a.runs.depth[s] - 1) / a.runs.depth[s], count = a.count[s];
            for (int k = 0; k < runs; ++k) {
                const float *const p = a.sums + ((size_t)s * (size_t)a.runs.sums + (size_t)k * (size_t)count + (size_t)at) * (size_t)a.width;
#pragma unroll
                for (int h = 0; h < N; h += 4) {
                    const Piece<float>::F v = Piece<float>::load(p, col + h, a.width);
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[h + j] += v[j];
                }
            }
            total += sum * (a.scale[2 * s + 1] * a.temperature);
        }
        Piece<T>::store(static_cast<T *>(a.out) + ((size_t)s0 * (size_t)a.rows + (size_t)row) * (size_t)a.width, col, a.width, total);
    }
}

// both, behind a piece's products: the first x_blocks workgroups have dx (behind the last piece)
template <class T>
__global__ void __launch_bounds__(256) hot_head_finish_kernel(FeatureArgs x, BiasArgs b, int x_blocks)
{
    const long s = blockIdx.y;
    if ((int)blockIdx.x < x_blocks) feature_gradient<T>(x, s, blockIdx.x, x_blocks);
    else bias_gradient(b, s, (int)blockIdx.x - x_blocks);
}

__global__ void __launch_bounds__(256) hot_head_zero_kernel(char *p, long bytes)
{
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < bytes; i += (long)gridDim.x * 256) p[i] = 0;
}

// ---------------------------------------------------------------------------------
// Host side.

constexpr long kMostTiles = 1L << 22;                    // of up to 512 threads in a launch (one grid dimension holds fewer than 2^32), and of 256 x 256 logits in a call
// Of dz and packed weights: twice what the memory-side cache holds.  Half of it adds the features' gradients up in twice as many passes over their sums
// (8192 x 4096 x 131072 bf16 forward and backward 41.8 ms, 41.0 so; 1000 x 768 x 32768 float32 1138 us, 1067 so).
constexpr int64_t kPieceBytes = (int64_t)512 << 20;

// Sizes of tiles (of logits: words x rows): 256 x 32 for up to 32 rows, 64 x 64 and 128 x 128 where larger ones leave the chip empty, 256 x 256
// (256 x 128 in three pieces).
// Float32 heads of up to 128 rows with 256 tiles of words have 256 x 128 with the weights read as they lie (128 x 1024 x 65536 forward and backward: 842 us packed, 585 so; with half as
// many tiles, 64 x 768 x 32768, whose packed weights stay in the memory-side cache, 281 packed, 278 so).
// Tiles of the gradients are the same, but with half as many words (weights') or rows (features') where two pieces of dz would take twice the room: 256 x 128, and 128 x 64
// for 128 x 128 (512 x 1024 x 11000 bf16 forward and backward 140 us; with all 128, one workgroup to a compute unit, 153, with 64 x 64 150).
enum { kFew, kSmall, kMiddle, kLarge, kTall };

struct HeadPlan {
    int pieces, dz_pieces;   // of an element, and of dz
    bool pack_w, raw_w;      // weights packed; float32 weights of few rows, read as they lie
    int columns;             // of a block of what is packed
    long row_bytes;          // of a packed row: whole blocks
    long places;
    int v_piece;             // words of a piece
    int size;                // kFew ... kTall
    int v_tile, r_tile;      // words and rows of a tile of logits
    int x_tile;              // rows of a tile of the features' gradients
    int row_tiles;
    WordRuns word_runs;       // runs of words of the features' gradients
    int most_word_runs;
    int runs, run_depth;     // runs of rows of the weights' gradients, and their length
    // where things lie in the workspace
    int64_t word, weight, list_count, sums, start, count, word_run, row_of, place_of, label, base, rest, grad, scale, x, w, dz, partials, dx, db, dw, bytes;
};

struct Layout {
    int64_t at = 0;
    int64_t take(int64_t bytes)
    {
        const int64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    }
};

bool head_ok(const hot_head_desc *d)
{
    if (!d || d->rows < 0 || d->rows > (1L << 20) || d->width < 1 || d->width > (1L << 19) || d->vocab < 1 || d->vocab > (1L << 24) || d->samples < 1 || d->samples > 4096 ||
        !known_type(d->dtype) || d->ldx < 0 || d->x_sample < 0 || d->ldw < d->width || d->w_sample < 0 || d->bias_sample < 0 || d->index_row < 0 || d->index_sample < 0)
        return false;
    if (d->samples > 1 && (d->w_sample < (d->vocab - 1) * d->ldw + d->width || (d->bias_sample != 0 && d->bias_sample < d->vocab))) return false;
    if (d->top < 0 || d->top > kMostTop || d->samples * d->rows > (1L << 30)) return false;
    if (d->top > 0 && (!known_type(d->logit_dtype) || d->logit_row < 0 || d->logit_sample < 0)) return false;
    if (up(d->rows, 256) / 256 * (up(d->vocab, 256) / 256) > kMostTiles) return false;
    if (!(d->temperature > 0.0) || !(d->temperature <= 1e4) || !(d->temperature >= 1e-4) || (d->top == 0 && d->temperature != 1.0)) return false;
    return true;
}

HeadPlan head_plan(const hot_head_desc &d, bool backward, bool with_dx)
{
    HeadPlan p = {};
    const long S = d.samples, R = d.rows, V = d.vocab, K = d.width;
    p.pieces = d.dtype == HOT_F32 ? 3 : 1;
    const bool whole = d.w_aligned && K % 4 == 0 && d.ldw % 4 == 0 && (S == 1 || d.w_sample % 4 == 0) && d.ldw <= (1L << 20);
    p.raw_w = p.pieces == 3 && whole && (R <= 32 || (R <= 128 && up(V, 256) / 256 * S >= kComputeUnits));
    p.pack_w = (p.pieces == 3 && !p.raw_w) || (p.pieces == 1 && (!d.w_aligned || K % 8 || d.ldw % 8 || (S > 1 && d.w_sample % 8) || d.ldw > (1L << 21)));
    p.columns = p.pieces == 3 ? 32 : 64;
    p.row_bytes = up(K, p.columns) * 2;
    p.places = up(R, 256);
    // The time of a size: rounds of workgroups times what a round takes (a round of large tiles is one; smaller tiles run at lower rates, two of them
    // to a compute unit but for three pieces of 128 x 128).
    auto rounds = [&](long v, long r, long to_a_unit) { return (double)((((V + v - 1) / v) * ((R + r - 1) / r) * S + to_a_unit * kComputeUnits - 1) / (to_a_unit * kComputeUnits)); };
    const bool three = p.pieces == 3;
    const double large = rounds(256, three ? 128 : 256, 1), middle = rounds(128, 128, three ? 1 : 2) * (three ? 0.62 : 0.67), small = rounds(64, 64, 2) * (three ? 0.42 : 0.25);
    p.size = R <= 32 ? kFew : p.raw_w ? kTall : (large <= middle && large <= small ? kLarge : (middle <= small ? kMiddle : kSmall));
    p.dz_pieces = three ? 3 : 2;
    constexpr int V_TILE[] = {256, 64, 128, 256, 256}, R_TILE[] = {32, 64, 128, 256, 128};
    p.v_tile = V_TILE[p.size];
    p.r_tile = p.size == kLarge && three ? 128 : R_TILE[p.size];
    p.x_tile = p.size == kLarge ? 128 : (p.size == kMiddle && !three ? 64 : p.r_tile);
    p.row_tiles = (int)((R + p.r_tile - 1) / p.r_tile);
    long piece = up(V, 256);
    if (backward || p.pack_w) {
        const int64_t per_word = S * ((backward ? p.places * 2 * p.dz_pieces : 0) + (p.pack_w ? p.row_bytes * p.pieces : 0));
        const long most = kPieceBytes / per_word / 256 * 256;
        const long least = 1024;
        const long n = (piece + (most > least ? most : least) - 1) / (most > least ? most : least);
        piece = up((V + n - 1) / n, 256);
    }
    // tiles of the weights' gradients: width and words
    const int wt = p.size >= kLarge ? 256 : (p.size == kMiddle ? 128 : 64), wv = p.size >= kLarge ? 128 : (three ? wt : 64);
    // (float32, 2^20 rows and 2^18 words: 2^23 tiles of logits)
    const long logits = kMostTiles / p.row_tiles * p.v_tile, weights = kMostTiles / ((K + wt - 1) / wt) * wv, most = (logits < weights || !backward ? logits : weights) / 256 * 256;
    piece = piece < most ? piece : most;
    p.v_piece = (int)piece;
    // as many workgroups and sums as the best number of runs needs for all rows
    WordRuns &w = p.word_runs;
    static_assert(kComputeUnits == 256, "");
    w = {__builtin_ctz((unsigned)p.x_tile), p.size == kLarge || p.pieces == 3 ? 8 : 9, (int)((K + V_TILE[p.size] - 1) / V_TILE[p.size]), (int)S, (int)piece, LONG_MAX, LONG_MAX, nullptr};
    int best_runs = 1;
    for (int runs = 2; runs <= 64 && run_possible(w, R, runs); ++runs)
        if (run_steps(w, R, runs) < run_steps(w, R, best_runs)) best_runs = runs;
    best_runs = (int)((piece + run_depth((int)piece, best_runs) - 1) / run_depth((int)piece, best_runs));
    p.most_word_runs = best_runs;
    w.workgroups = best_runs * place_blocks(w.width_tiles, (R + p.x_tile - 1) / p.x_tile);
    w.sums = best_runs * R;
    long best = 0;

    // The weights' gradients: as many runs of rows as leave the fewest steps of BK rows in all rounds, twenty more to each run, and as long as their
    // partial sums are no more than two rounds of tiles (5569 x 42 x 1227 float32, forward and backward: 403 us on ten workgroups, 153 so)
    const long w_tiles = ((piece + wv - 1) / wv < (V + wv - 1) / wv ? (piece + wv - 1) / wv : (V + wv - 1) / wv) * ((K + wt - 1) / wt) * S;
    for (long runs = 1; runs <= 256 && (runs == 1 || (runs * 4 * p.columns <= R && runs * w_tiles <= 2 * kComputeUnits)); ++runs) {
        const long depth = up((R + runs - 1) / runs, p.columns), cost = (w_tiles * runs + kComputeUnits - 1) / kComputeUnits * (depth / p.columns + 20);
        if (runs == 1 || cost < best) {
            best = cost;
            p.run_depth = (int)depth;
        }
    }
    p.runs = (int)((R + p.run_depth - 1) / p.run_depth);

    Layout l;
    const long lists = d.top > 0 ? (d.index_sample > 0 || d.logit_sample > 0 ? S : 1) * R : 0, marks = (V + kStartStep - 1) / kStartStep;
    p.word = l.take(lists * d.top * 4);
    p.weight = l.take(lists * d.top * 4);
    p.list_count = l.take(lists * 4);
    p.sums = l.take(lists * 16);
    p.start = l.take(lists * (marks + 1) * 2);
    p.count = l.take(S * 4);
    p.word_run = l.take(S * 4);
    p.row_of = l.take(S * R * 4);
    p.place_of = l.take(S * R * 4);
    p.label = l.take(d.top > 0 ? 0 : S * R * 4);
    if (backward) {
        p.base = l.take(S * R * 4);
        p.rest = l.take(S * R * 4);
        p.grad = l.take(S * R * 4);
        p.scale = l.take(S * 8);
    }
    p.x = l.take(S * p.places * p.row_bytes * p.pieces);
    p.w = l.take(p.pack_w ? S * piece * p.row_bytes * p.pieces : 0);
    if (backward) {
        p.dz = l.take(S * p.places * piece * 2 * p.dz_pieces);
        p.db = l.take(S * p.row_tiles * piece * 4);
        p.dw = l.take(p.runs > 1 ? (int64_t)p.runs * S * (piece < V ? piece : V) * K * 4 : 0);
        if (with_dx) p.dx = l.take(p.word_runs.sums * S * K * 4);
    } else {
        p.partials = l.take(S * ((V + p.v_tile - 1) / p.v_tile) * 4 * p.places * 4);
    }
    p.bytes = l.at;
    return p;
}

struct HeadCall {
    const hot_head_desc &d;
    const HeadPlan &p;
    char *ws;
    hipStream_t stream;
    const void *x, *w, *bias;
    const int64_t *index;
    const void *logit;
    long list_sample;

    template <class V>
    V *in(int64_t at) const { return reinterpret_cast<V *>(ws + at); }
};

unsigned grid_for(long items, long most = 8192)
{
    const long n = (items + 255) / 256;
    return (unsigned)(n < 1 ? 1 : (n < most ? n : most));
}

void head_lists(const HeadCall &c)
{
    const hot_head_desc &d = c.d;
    const HeadPlan &p = c.p;
    if (d.top == 0) return;
    ListArgs a;
    a.rows = d.rows;
    a.idx_sample = d.index_sample;
    a.idx_row = d.index_row;
    a.logit_sample = d.logit_sample;
    a.logit_row = d.logit_row;
    a.top = (int)d.top;
    a.logit_type = d.logit_dtype;
    a.marks = (int)((d.vocab + kStartStep - 1) / kStartStep);
    a.vocab = d.vocab;
    a.inv_temperature = (float)(1.0 / d.temperature);
    a.index = c.index;
    a.logit = c.logit;
    a.word = c.in<int>(p.word);
    a.weight = c.in<float>(p.weight);
    a.count = c.in<int>(p.list_count);
    a.sums = c.in<double>(p.sums);
    a.start = c.in<unsigned short>(p.start);
    // (samples along y: a grid's dimension holds fewer than 2^32 threads)
    const dim3 grid((unsigned)((a.rows + kListWaves - 1) / kListWaves), c.list_sample > 0 ? (unsigned)d.samples : 1u), block(64 * kListWaves);
    if (a.top <= 64) hot_head_lists_kernel<64><<<grid, block, 0, c.stream>>>(a);
    else if (a.top <= 256) hot_head_lists_kernel<256><<<grid, block, 0, c.stream>>>(a);
    else hot_head_lists_kernel<kMostTop><<<grid, block, 0, c.stream>>>(a);
}

WordRuns head_runs(const HeadCall &c)
{
    WordRuns a = c.p.word_runs;
    a.depth = c.in<int>(c.p.word_run);
    return a;
}

RowArgs head_rows(const HeadCall &c, const double *lse, const float *g, long g_sample, long g_row)
{
    const hot_head_desc &d = c.d;
    const HeadPlan &p = c.p;
    RowArgs a = {};
    a.rows = d.rows;
    a.vocab = d.vocab;
    a.temperature = d.temperature;
    a.idx_sample = d.index_sample;
    a.idx_row = d.index_row;
    a.ignore = d.ignore_index;
    a.index = c.index;
    a.list_count = d.top > 0 ? c.in<int>(p.list_count) : nullptr;
    a.list_sample = c.list_sample;
    a.lse = lse;
    a.g = g;
    a.g_sample = g_sample;
    a.g_row = g_row;
    a.scale_to = d.dtype == HOT_F16 ? kHalfScale : 1.0f;
    a.count = c.in<int>(p.count);
    a.row_of = c.in<int>(p.row_of);
    a.place_of = c.in<int>(p.place_of);
    a.label = d.top > 0 ? nullptr : c.in<int>(p.label);
    a.base = c.in<float>(p.base);
    a.rest = c.in<float>(p.rest);
    a.grad = c.in<float>(p.grad);
    a.scale = c.in<float>(p.scale);
    if (lse) a.runs = head_runs(c);
    return a;
}

PackArgs head_pack_x(const HeadCall &c)
{
    PackArgs a;
    a.from = c.x;
    a.from_row = c.d.ldx;
    a.from_sample = c.d.x_sample;
    a.row_of = c.in<int>(c.p.row_of);
    a.count = c.in<int>(c.p.count);
    a.rows = c.d.rows;
    a.width = (int)c.d.width;
    a.to = c.in<char>(c.p.x);
    a.columns = c.p.columns;
    a.block = c.p.places * c.p.columns * 2L;
    a.to_sample = c.p.places * c.p.row_bytes;
    a.plane = c.d.samples * a.to_sample;
    return a;
}

PackArgs head_pack_w(const HeadCall &c, long v_begin, long v_count)
{
    PackArgs a = {};
    a.from = static_cast<const char *>(c.w) + (size_t)v_begin * (size_t)c.d.ldw * (size_t)type_bytes(c.d.dtype);
    a.from_row = c.d.ldw;
    a.from_sample = c.d.w_sample;
    a.rows = v_count;
    a.width = (int)c.d.width;
    a.to = c.in<char>(c.p.w);
    a.columns = c.p.columns;
    a.block = c.p.v_piece * c.p.columns * 2L;
    a.to_sample = c.p.v_piece * c.p.row_bytes;
    a.plane = c.d.samples * a.to_sample;
    return a;
}

// workgroups that pack an array: a run of rows of a block of columns to each, as long as that leaves enough of them
long pack_blocks(const PackArgs &a)
{
    const long at_once = 256 / (a.columns / 8), items = (a.rows + at_once - 1) / at_once * ((a.width + a.columns - 1) / a.columns);
    return items < 8192 ? items : 8192;
}

template <class T>
void head_pack(const HeadCall &c, const PackArgs &a)
{
    hot_head_pack_kernel<T><<<dim3((unsigned)pack_blocks(a), (unsigned)c.d.samples), 256, 0, c.stream>>>(a);
}

// Everything in front of the products: entries, rows, the packed features and the first piece's packed weights
template <class T>
void head_prepare(const HeadCall &c, const RowArgs &rows, long first_words)
{
    head_lists(c);
    const PackArgs x = head_pack_x(c), w = head_pack_w(c, 0, first_words);
    const long xb = pack_blocks(x), wb = c.p.pack_w ? pack_blocks(w) : 0;
    if (c.d.rows <= kFewRows) {
        hot_head_prepare_kernel<T><<<dim3((unsigned)(xb + wb), (unsigned)c.d.samples), 256, 0, c.stream>>>(rows, x, w, (int)xb);
        return;
    }
    hot_head_rows_kernel<<<dim3((unsigned)c.d.samples), kRowBlock, 0, c.stream>>>(rows);
    head_pack<T>(c, x);
    if (c.p.pack_w) head_pack<T>(c, w);
}

// the weights from word v_begin on as the kernels read them: as they lie, or packed
Matrix head_weights(const HeadCall &c, long v_begin, long &sample)
{
    const long columns = c.p.columns;
    const long size = type_bytes(c.d.dtype);
    sample = c.p.pack_w ? c.p.v_piece * c.p.row_bytes : c.d.w_sample * size;
    if (!c.p.pack_w) return {static_cast<const char *>(c.w) + (size_t)v_begin * (size_t)c.d.ldw * (size_t)size, c.d.ldw * size, columns * size, 0};
    return {c.in<char>(c.p.w), columns * 2, c.p.v_piece * columns * 2, c.d.samples * sample};
}

HeadArgs head_args(const HeadCall &c, long v_begin, long v_count)
{
    const hot_head_desc &d = c.d;
    const HeadPlan &p = c.p;
    HeadArgs a = {};
    a.w = head_weights(c, v_begin, a.w_sample);
    a.x_sample = p.places * p.row_bytes;
    a.x = {c.in<char>(p.x), p.columns * 2L, p.places * p.columns * 2L, d.samples * a.x_sample};
    a.width = (int)d.width;
    a.vocab = (int)d.vocab;
    a.v_begin = (int)v_begin;
    a.v_count = (int)v_count;
    a.rows = d.rows;
    a.places = p.places;
    a.count = c.in<int>(p.count);
    a.row_of = c.in<int>(p.row_of);
    a.label = c.in<int>(p.label);
    a.bias = c.bias;
    a.bias_sample = d.bias_sample;
    a.bias_type = d.dtype;
    a.scale = (float)(1.44269504088896340736 / d.temperature);
    a.word = c.in<int>(p.word);
    a.weight = c.in<float>(p.weight);
    a.start = c.in<unsigned short>(p.start);
    a.top = (int)d.top;
    a.marks = (int)((d.vocab + kStartStep - 1) / kStartStep);
    a.list_sample = c.list_sample;
    a.partials = c.in<float>(p.partials);
    a.v_tiles = (int)((d.vocab + p.v_tile - 1) / p.v_tile);
    a.base = c.in<float>(p.base);
    a.rest = c.in<float>(p.rest);
    a.grad = c.in<float>(p.grad);
    a.to_scale = c.in<float>(p.scale);
    a.row_tiles = p.row_tiles;
    a.v_piece = p.v_piece;
    a.dz = c.in<char>(p.dz);
    a.dz_block = p.places * p.columns * 2L;
    a.dz_sample = p.places * p.v_piece * 2L;
    a.dz_plane = d.samples * a.dz_sample;
    return a;
}

template <int PIECES>
constexpr int kSmallStages = PIECES == 1 ? 4 : 3;

// Pieces in which dz is held.  One rounding of dz to 16 bits would show in gradients of 16 bits beside their own: a word's is made by the few rows that
// carry or list it, a row's by its few likely words, and there is nothing that averages out (1.4 times the error of a float32 dz
// over 4096 rows, up to three times it over a handful).
template <int PIECES>
constexpr int kDz = PIECES == 1 ? 2 : PIECES;

template <class TILE>
void logits_go(const HeadCall &c, const HeadArgs &a, bool backward)
{
    const dim3 grid((unsigned)place_blocks((a.v_count + TILE::BM - 1) / TILE::BM, (c.d.rows + TILE::BN - 1) / TILE::BN), (unsigned)c.d.samples), block(TILE::THREADS);
    if (c.d.top > 0) {
        if (backward) hot_head_dz_kernel<TILE, true, kDz<TILE::PIECES_A>><<<grid, block, 0, c.stream>>>(a);
        else hot_head_forward_kernel<TILE, true><<<grid, block, 0, c.stream>>>(a);
    } else {
        if (backward) hot_head_dz_kernel<TILE, false, kDz<TILE::PIECES_A>><<<grid, block, 0, c.stream>>>(a);
        else hot_head_forward_kernel<TILE, false><<<grid, block, 0, c.stream>>>(a);
    }
}

template <class T, int PIECES>
void head_logits(const HeadCall &c, const HeadArgs &a, bool backward)
{
    if constexpr (PIECES == 3) {
        if (c.p.size == kTall) return logits_go<Tile<T, PIECES, PIECES, true, true, 256, 128, 8, 1, 2, true, false>>(c, a, backward);
        if (c.p.raw_w) return logits_go<Tile<T, PIECES, PIECES, true, true, 256, 32, 8, 1, 4, true, false>>(c, a, backward);
        if (c.p.size == kFew) return logits_go<Tile<T, PIECES, PIECES, true, true, 256, 32, 8, 1>>(c, a, backward);
    } else if (c.p.size == kFew) return logits_go<Tile<T, PIECES, PIECES, true, true, 256, 32, 8, 1, 4>>(c, a, backward);
    if (c.p.size == kSmall) logits_go<Tile<T, PIECES, PIECES, true, true, 64, 64, 2, 2, kSmallStages<PIECES>>>(c, a, backward);
    else if (c.p.size == kMiddle) logits_go<Tile<T, PIECES, PIECES, true, true, 128, 128, 2, 2>>(c, a, backward);
    else if constexpr (PIECES == 1) logits_go<Tile<T, PIECES, PIECES, true, true, 256, 256, 2, 4>>(c, a, backward);
    else logits_go<Tile<T, PIECES, PIECES, true, true, 256, 128, 4, 2>>(c, a, backward);
}

template <class TILE>
void head_dx(const HeadCall &c, const GradArgs &a)
{
    hot_head_dx_kernel<TILE><<<dim3((unsigned)place_blocks((c.d.width + TILE::BN - 1) / TILE::BN, (c.d.rows + TILE::BM - 1) / TILE::BM), (unsigned)c.d.samples, (unsigned)c.p.most_word_runs),
                               TILE::THREADS, 0, c.stream>>>(a);
}

template <class TILE, class OUT>
void dw_go(const HeadCall &c, const GradArgs &a)
{
    hot_head_dw_kernel<TILE, OUT><<<dim3((unsigned)place_blocks((a.v_count + TILE::BN - 1) / TILE::BN, (c.d.width + TILE::BM - 1) / TILE::BM), (unsigned)c.d.samples, (unsigned)c.p.runs),
                                    TILE::THREADS, 0, c.stream>>>(a);
}

// dW on tiles of TILE, or (RUNS) as partial sums in float32 that are then added up
template <class TILE, class T, bool RUNS = true>
void head_dw(const HeadCall &c, GradArgs a, void *dw)
{
    const long part = (long)a.v_count * c.d.width;
    a.row_depth = c.p.run_depth;
    if (!RUNS || c.p.runs == 1) {
        a.out = dw;
        a.out_sample = c.d.vocab * c.d.width;
        a.out_first = a.v_begin;
        return dw_go<TILE, T>(c, a);
    }
    if constexpr (RUNS) {
        float *const parts = c.in<float>(c.p.dw);
        a.out = parts;
        a.out_sample = part;
        a.out_split = c.d.samples * part;
        a.out_first = 0;
        dw_go<TILE, float>(c, a);
        const RunArgs r = {parts, part, part, a.out_split, c.d.vocab * c.d.width, c.p.runs, static_cast<T *>(dw) + (size_t)a.v_begin * (size_t)c.d.width};
        hot_head_runs_kernel<T><<<dim3(grid_for((part + Piece<T>::N - 1) / Piece<T>::N), (unsigned)c.d.samples), 256, 0, c.stream>>>(r);
    }
}

// T: the type of the tensors; E: of the tiles' elements
template <class T, class E, int PIECES>
void head_forward(const HeadCall &c, float *loss, double *lse)
{
    head_prepare<T>(c, head_rows(c, nullptr, nullptr, 0, 0), c.d.vocab < c.p.v_piece ? c.d.vocab : c.p.v_piece);
    for (long v = 0; v < c.d.vocab; v += c.p.v_piece) {
        const long n = c.d.vocab - v < c.p.v_piece ? c.d.vocab - v : c.p.v_piece;
        if (c.p.pack_w && v > 0) head_pack<T>(c, head_pack_w(c, v, n));
        head_logits<E, PIECES>(c, head_args(c, v, n), false);
    }
    JoinArgs a;
    a.rows = c.d.rows;
    a.places = c.p.places;
    a.tiles = (int)((c.d.vocab + c.p.v_tile - 1) / c.p.v_tile);
    a.lanes = 4;
    while (a.lanes < 256 && (c.d.rows + 256 / a.lanes - 1) / (256 / a.lanes) * c.d.samples < kComputeUnits && a.lanes * 2 <= a.tiles) a.lanes *= 2;
    a.scale = (float)(1.44269504088896340736 / c.d.temperature);
    a.partials = c.in<float>(c.p.partials);
    a.place_of = c.in<int>(c.p.place_of);
    a.label = c.in<int>(c.p.label);
    a.sums = c.d.top > 0 ? c.in<double>(c.p.sums) : nullptr;
    a.list_sample = c.list_sample;
    a.temperature = c.d.temperature;
    a.loss = loss;
    a.lse = lse;
    hot_head_join_kernel<<<dim3((unsigned)((c.d.rows + 256 / a.lanes - 1) / (256 / a.lanes)), (unsigned)c.d.samples), 256, 0, c.stream>>>(a);
}

template <class T, class E, int PIECES>
void head_backward(const HeadCall &c, const double *lse, const float *g, long g_sample, long g_row, void *dx, void *dw, void *db)
{
    head_prepare<T>(c, head_rows(c, lse, g, g_sample, g_row), c.d.vocab < c.p.v_piece ? c.d.vocab : c.p.v_piece);
    const float *const scale = c.in<float>(c.p.scale);
    for (long v = 0; v < c.d.vocab; v += c.p.v_piece) {
        const long n = c.d.vocab - v < c.p.v_piece ? c.d.vocab - v : c.p.v_piece;
        if (c.p.pack_w && v > 0) head_pack<T>(c, head_pack_w(c, v, n));
        HeadArgs h = head_args(c, v, n);
        if (db) h.sums = c.in<float>(c.p.db);
        head_logits<E, PIECES>(c, h, true);
        GradArgs a = {};
        a.dz = {h.dz, c.p.columns * 2L, h.dz_block, h.dz_plane};
        a.dz_sample = h.dz_sample;
        a.width = h.width;
        a.v_begin = h.v_begin;
        a.v_count = h.v_count;
        a.count = h.count;
        a.runs = head_runs(c);
        a.first = v == 0;
        a.sums = c.in<float>(c.p.dx);
        a.scale = scale;
        a.temperature = (float)c.d.temperature;
        if (dx) {
            a.other = h.w;
            a.sample = h.w_sample;
            if (c.p.size == kTall) {
                if constexpr (PIECES == 3) head_dx<Tile<E, PIECES, PIECES, true, false, 128, 256, 1, 8, 2, false, true>>(c, a);
            } else if (c.p.raw_w) {
                if constexpr (PIECES == 3) head_dx<Tile<E, PIECES, PIECES, true, false, 32, 256, 1, 8, 4, false, true>>(c, a);
            } else if (c.p.size == kFew) head_dx<Tile<E, kDz<PIECES>, PIECES, true, false, 32, 256, 1, 8, PIECES == 1 ? 3 : 2>>(c, a);
            else if (c.p.size == kSmall) head_dx<Tile<E, kDz<PIECES>, PIECES, true, false, 64, 64, 2, 2, 3>>(c, a);
            else if (c.p.size == kMiddle) head_dx<Tile<E, kDz<PIECES>, PIECES, true, false, PIECES == 1 ? 64 : 128, 128, 2, 2>>(c, a);
            else head_dx<Tile<E, kDz<PIECES>, PIECES, true, false, 128, 256, 2, 4>>(c, a);
        }
        if (dw) {
            a.other = h.x;
            a.sample = h.x_sample;
            if (c.p.size == kFew) head_dw<Tile<E, PIECES, kDz<PIECES>, false, false, 256, 64, 4, 1, 1>, T, false>(c, a, dw);
            else if (c.p.size == kSmall) head_dw<Tile<E, PIECES, kDz<PIECES>, false, false, 64, 64, 2, 2, 3>, T>(c, a, dw);
            else if (c.p.size == kMiddle) head_dw<Tile<E, PIECES, kDz<PIECES>, false, false, 128, PIECES == 1 ? 64 : 128, 2, 2>, T>(c, a, dw);
            else head_dw<Tile<E, PIECES, kDz<PIECES>, false, false, 256, 128, 4, 2>, T>(c, a, dw);
        }
        const bool finish_x = dx && v + n >= c.d.vocab;
        if (!db && !finish_x) continue;
        const BiasArgs b = {h.sums, c.p.row_tiles, c.p.r_tile, c.p.v_piece, h.v_begin, h.v_count, h.count, scale, a.temperature, db, c.d.vocab, c.d.dtype};
        const FeatureArgs f = {c.in<float>(c.p.dx), c.in<int>(c.p.place_of), h.count, a.runs, scale, a.temperature, c.d.rows, c.d.width, (int)c.d.samples,
                               c.d.samples > 1 && c.d.x_sample == 0, dx};
        const unsigned xb = finish_x ? grid_for(c.d.rows * ((c.d.width + Piece<T>::N - 1) / Piece<T>::N)) : 0, bb = db ? (unsigned)((n + 255) / 256) : 0;
        hot_head_finish_kernel<T><<<dim3(xb + bb, (unsigned)c.d.samples), 256, 0, c.stream>>>(f, b, (int)xb);
    }
}

bool head_inputs_ok(const hot_head_desc &d, const void *x, const void *w, const void *bias, const int64_t *index, const void *logit)
{
    if (!w || !on_element(w, d.dtype) || !on_element(bias, d.dtype)) return false;
    if (bias && d.samples > 1 && d.bias_sample == 0) return false;
    if (d.w_aligned && !aligned16(w)) return false;
    if (d.rows == 0) return true;
    if (!x || !on_element(x, d.dtype) || !index || (reinterpret_cast<uintptr_t>(index) & 7u)) return false;
    if (d.top > 0 && (!logit || !on_element(logit, d.logit_dtype))) return false;
    return true;
}

HeadCall head_call(const hot_head_desc &d, const HeadPlan &p, const void *x, const void *w, const void *bias, const int64_t *index, const void *logit, void *workspace,
                   void *stream)
{
    return {d, p, static_cast<char *>(workspace), static_cast<hipStream_t>(stream), x, w, bias, index, logit, d.index_sample > 0 || d.logit_sample > 0 ? d.rows : 0};
}

bool workspace_ok(const HeadPlan &p, const void *workspace, int64_t bytes) { return workspace && aligned16(workspace) && bytes >= p.bytes; }

}  // namespace

extern "C" {

int64_t hot_head_workspace_bytes(const hot_head_desc *desc, int which)
{
    if (!head_ok(desc) || which < 0 || which > 2) return HOT_EINVAL;
    if (desc->rows == 0) return 0;
    return head_plan(*desc, which > 0, which == 1).bytes;
}

int hot_head_forward(const hot_head_desc *desc, const void *x, const void *weight, const void *bias, const int64_t *index, const void *logit, float *loss,
                     double *lse, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (!head_ok(desc) || !head_inputs_ok(*desc, x, weight, bias, index, logit)) return HOT_EINVAL;
    if (desc->rows == 0) return HOT_OK;
    const HeadPlan p = head_plan(*desc, false, false);
    if (!loss || !aligned4(loss) || (reinterpret_cast<uintptr_t>(lse) & 7u) || !workspace_ok(p, workspace, workspace_bytes)) return HOT_EINVAL;
    const HeadCall c = head_call(*desc, p, x, weight, bias, index, logit, workspace, stream);
    if (desc->dtype == HOT_F32) head_forward<float, __bf16, 3>(c, loss, lse);
    else if (desc->dtype == HOT_BF16) head_forward<__bf16, __bf16, 1>(c, loss, lse);
    else head_forward<_Float16, _Float16, 1>(c, loss, lse);
    return hot_detail::note_hip(hipGetLastError());
}

int hot_head_backward(const hot_head_desc *desc, const void *x, const void *weight, const void *bias, const int64_t *index, const void *logit,
                      const double *lse, const float *grad_loss, int64_t grad_sample, int64_t grad_row, void *dx, void *grad_weight, void *grad_bias,
                      void *workspace, int64_t workspace_bytes, void *stream)
{
    if (!head_ok(desc) || !head_inputs_ok(*desc, x, weight, bias, index, logit) || grad_sample < 0 || grad_row < 0) return HOT_EINVAL;
    if (!on_element(dx, desc->dtype) || !on_element(grad_weight, desc->dtype) || !on_element(grad_bias, desc->dtype)) return HOT_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (desc->rows == 0) {        // sums over no rows
        const int64_t words = desc->samples * desc->vocab, size = type_bytes(desc->dtype);
        if (grad_weight) hot_head_zero_kernel<<<grid_for(words * desc->width * size), 256, 0, s>>>(static_cast<char *>(grad_weight), words * desc->width * size);
        if (grad_bias) hot_head_zero_kernel<<<grid_for(words * size), 256, 0, s>>>(static_cast<char *>(grad_bias), words * size);
        return hot_detail::note_hip(hipGetLastError());
    }
    if (!dx && !grad_weight && !grad_bias) return HOT_OK;
    const HeadPlan p = head_plan(*desc, true, dx != nullptr);
    if (!lse || (reinterpret_cast<uintptr_t>(lse) & 7u) || !grad_loss || !aligned4(grad_loss) || !workspace_ok(p, workspace, workspace_bytes)) return HOT_EINVAL;
    const HeadCall c = head_call(*desc, p, x, weight, bias, index, logit, workspace, stream);
    if (desc->dtype == HOT_F32) head_backward<float, __bf16, 3>(c, lse, grad_loss, grad_sample, grad_row, dx, grad_weight, grad_bias);
    else if (desc->dtype == HOT_BF16) head_backward<__bf16, __bf16, 1>(c, lse, grad_loss, grad_sample, grad_row, dx, grad_weight, grad_bias);
    else head_backward<_Float16, _Float16, 1>(c, lse, grad_loss, grad_sample, grad_row, dx, grad_weight, grad_bias);
    return hot_detail::note_hip(hipGetLastError());
}

}  // extern "C"
