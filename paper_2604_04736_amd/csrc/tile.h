// Tiles of a matrix product on the 16-bit matrix instruction, for the kernels of head.hip: BM x BN results of a workgroup, both
// operands staged through LDS straight from memory, sixteen bytes a lane, while the tile before is multiplied.
//
// An operand lies in memory with its contraction index running along its rows (ALONG: weights and features for the logits, their gradients
// for the features' gradients) or across them (weights for the features' gradients, features and the logits' gradients for the weights').
// Along, a lane's eight contraction indices are one 16-byte read of LDS; across, two transposing reads, so no operand is ever
// transposed in memory.  Sixteen-byte pieces of LDS are permuted so that neither form of reading meets its own banks.
// Pieces of an operand (planes of equal layout): three bf16 pieces of float32 in both, multiplied as the six products that carry 24 bits, from
// the smallest on; one of bf16 and fp16 operands as they are; two where an operand is a result that is held in twice its type's bits.
#ifndef HOT_TILE_H
#define HOT_TILE_H

#include <hip/hip_runtime.h>

namespace {

typedef short s4v __attribute__((ext_vector_type(4)));
typedef short s8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) s4v lds_s4v;
typedef __attribute__((address_space(3))) s8v lds_s8v;

constexpr unsigned kBeyond = 0x80000000u;        // an offset outside every window: such lanes receive zeros

// The wait states between a run of matrix instructions and the first read of their results: 32, which the scheduler may not move
// (the compiler's own can be missing where a branch lies between).  Accumulators hand their registers out only against one of these.
struct TileSettled {
    __device__ __forceinline__ TileSettled()
    {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    }
    TileSettled(const TileSettled &) = delete;
    TileSettled &operator=(const TileSettled &) = delete;
};

// 32 x 32 results, sixteen to a lane, over sixteen contraction indices an instruction
template <class T>
class TileAcc {
    f16v v_;

public:
    __device__ __forceinline__ TileAcc() : v_(0.0f) {}
    __device__ __forceinline__ void mac(s8v a, s8v b)
    {
        if constexpr (__is_same(T, _Float16)) v_ = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), v_, 0, 0, 0);
        else v_ = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), v_, 0, 0, 0);
    }
    __device__ __forceinline__ f16v read(const TileSettled &) const { return v_; }
};

// A matrix in memory: element (row, col) at col / BK * block + row * pitch + col % BK * size, `plane` bytes between pieces.  Rows as they usually
// lie have a block of BK elements; what is written here for the tiles to read has rows of BK elements, one block of columns after another,
// so that a tile's loads are one run of memory (or four).
struct Matrix {
    const char *at;
    long pitch, block, plane;
};

// One operand's part of a tile: T of its rows or columns ("lines": what is not contracted) from `at` on.
struct Operand {
    Matrix m;            // from the first line and the first contraction index on (a multiple of BK if it is a column)
    int lines;           // how many lines there are; the tile's others are zeros
    int depth;           // how many contraction indices there are; the others are zeros
};

// Which of a row's chunks lies where (exclusive or), so that the lanes that LDS serves at once, 256 bytes, are in different banks: sixteen rows read sixteen bytes
// each along; across, four rows 64 bytes each, or, of float32, two rows eight apart.  (With only eight rows and 128 bytes told apart, half of the cycles that
// LDS worked were conflicts.)
template <int PER_ROW>
__device__ __forceinline__ int chunk_along(int row)
{
    return PER_ROW == 8 ? row >> 1 & 7 : row >> 2 & 3;
}

template <int T, bool RAW>
__device__ __forceinline__ int chunk_across(int row)
{
    static_assert(T >= 64, "a row holds the chunks told apart");
    return RAW ? (row >> 3 & 1) << 3 : (T >= 128 ? (row & 3) << 2 : (row >> 1 & 1) << 2);
}

// Lines and indices are taken sixteen bytes at a time along memory: a row may be read up to the next multiple of that, and must be finite there or
// meet zeros of the other operand.  RAW: float32 as it lies, cut into pieces only where a wave reads its operands from LDS.
template <int T, int BK, bool ALONG, int PIECES, int WAVES, bool RAW>
struct Stage {
    static constexpr int kSize = RAW ? 4 : 2, kChunk = 16 / kSize, kPlanes = RAW ? 1 : PIECES;
    static constexpr int kBytes = T * BK * kSize;                          // of one plane
    static constexpr int kPerRow = (ALONG ? BK : T) * kSize / 16;          // 16-byte chunks in a row of LDS
    static constexpr int kRows = 64 / kPerRow;                             // rows that one instruction of a wave fills
    // loads of a plane, and how many each wave issues (a plane of fewer loads than waves is loaded by several, to the same place)
    static constexpr int kLoads = kBytes / 1024, kEach = kLoads >= WAVES ? kLoads / WAVES : 1;
    static_assert(kPerRow <= 64 && kBytes % 1024 == 0 && (ALONG || T >= 64) && (kLoads % WAVES == 0 || WAVES % kLoads == 0), "");

    unsigned off[kEach];
    int index[ALONG ? 1 : kEach];          // the contraction index of this lane's loads in a tile
    int wave;

    // the order of a row's chunks
    static __device__ __forceinline__ int permuted(int row)
    {
        if constexpr (ALONG) return chunk_along<kPerRow>(row);
        else return chunk_across<T, RAW>(row);
    }

    __device__ __forceinline__ int load(int i) const { return (wave + i * WAVES) % kLoads; }

    __device__ __forceinline__ Stage(const Operand &o, int wave_, int lane) : wave(wave_)
    {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int row = load(j) * kRows + lane / kPerRow, col = (lane % kPerRow ^ permuted(row)) * kChunk;
            const int line = ALONG ? row : col;
            off[j] = line < o.lines ? (unsigned)(col / BK * o.m.block + row * o.m.pitch + col % BK * kSize) : kBeyond;
            if constexpr (ALONG) index[0] = col;
            else index[j] = row;
        }
    }

    // Sends for load `j` of kAll of the tile that begins at contraction index k0 (beyond the last index: for zeros).
    static constexpr int kAll = kEach * kPlanes;
    __device__ __forceinline__ void ask(const Operand &o, int k0, lds_char *to, int j) const
    {
        const int p = j / kEach, i = j % kEach;
        const char *const from = o.m.at + p * o.m.plane + (ALONG ? k0 / BK * o.m.block : k0 * o.m.pitch);
        const __amdgpu_buffer_rsrc_t win = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(from), 0, (int)kBeyond, 0x00020000);
        const unsigned at = index[ALONG ? 0 : i] < o.depth - k0 ? off[i] : kBeyond;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(win, (__attribute__((address_space(3))) void *)(to + p * kBytes + load(i) * 1024), 16, (int)at, 0, 0, 0);
    }
};

// the three bf16 pieces of a float, whose sum it is up to 2^-25 of it; what is not finite stays in the first
__device__ __forceinline__ void split_bf16(float x, __bf16 (&p)[3])
{
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        p[i] = (__bf16)x;
        const float back = (float)p[i];
        x = __builtin_isfinite(back) ? x - back : 0.0f;
    }
}

// Lane l's operand of the matrix instruction: line l % 32 of a block of 32, contraction indices 8 (l / 32) .. + 7 of sixteen.
template <int T, int BK, bool ALONG>
__device__ __forceinline__ s8v fragment(const lds_char *tile, int line0, int ks, int lane)
{
    const int half = lane >> 5;
    if constexpr (ALONG) {
        const int row = line0 + (lane & 31), chunk = ks * 2 + half;
        return *(const lds_s8v *)(tile + row * (BK * 2) + ((chunk ^ chunk_along<BK / 8>(row)) << 4));
    } else {
        const int i = lane & 15, row = ks * 16 + half * 8 + (i >> 2);
        const int byte = (line0 + (lane & 16) + (i & 3) * 4) * 2 ^ chunk_across<T, false>(i >> 2) << 4;        // (the same for row + 4)
        const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v *)(tile + row * (T * 2) + byte));
        const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v *)(tile + (row + 4) * (T * 2) + byte));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
}

// The same of float32: eight of its elements, cut into three pieces
template <int T, int BK, bool ALONG>
__device__ __forceinline__ void raw_fragment(const lds_char *tile, int line0, int ks, int lane, s8v &p0, s8v &p1, s8v &p2)
{
    typedef float f4v __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) f4v lds_f4v;
    typedef __attribute__((address_space(3))) float lds_float;
    const int half = lane >> 5, line = line0 + (lane & 31);
    float v[8];
    if constexpr (ALONG) {
        static_assert(BK == 32, "");
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f4v q = *(const lds_f4v *)(tile + line * (BK * 4) + (((ks * 2 + half) * 2 + h) ^ chunk_along<8>(line)) * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * h + j] = q[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = *(const lds_float *)(tile + (ks * 16 + half * 8 + j) * (T * 4) + (line * 4 ^ chunk_across<T, true>(half * 8) << 4));
    }
    bf16x8 p[3];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        __bf16 q[3];
        split_bf16(v[j], q);
#pragma unroll
        for (int i = 0; i < 3; ++i) p[i][j] = q[i];
    }
    p0 = __builtin_bit_cast(s8v, p[0]);
    p1 = __builtin_bit_cast(s8v, p[1]);
    p2 = __builtin_bit_cast(s8v, p[2]);
}

// STAGES tiles lie in LDS: two, or more where a tile is short work and latency counts; the loads of STAGES - 1 of them are under way.  One: the
// contraction has no more than BK indices.
template <class T_, int PIECES_A_, int PIECES_B_, bool A_ALONG_, bool B_ALONG_, int BM_, int BN_, int WAVES_M_, int WAVES_N_, int STAGES_ = 2, bool RAW_A_ = false, bool RAW_B_ = false>
struct Tile {
    typedef T_ T;
    static constexpr int PIECES_A = PIECES_A_, PIECES_B = PIECES_B_, BM = BM_, BN = BN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_;
    static constexpr int STAGES = STAGES_;
    static constexpr bool A_ALONG = A_ALONG_, B_ALONG = B_ALONG_, RAW_A = RAW_A_, RAW_B = RAW_B_;
    static_assert(STAGES >= 1 && (!RAW_A || PIECES_A == 3) && (!RAW_B || PIECES_B == 3), "");
    static constexpr int BK = PIECES_A == 3 ? 32 : 64;
    static constexpr int WAVES = WAVES_M * WAVES_N, THREADS = 64 * WAVES, WM = BM / WAVES_M, WN = BN / WAVES_N, MB = WM / 32, NB = WN / 32;
    typedef Stage<BM, BK, A_ALONG, PIECES_A, WAVES, RAW_A> StageA;
    typedef Stage<BN, BK, B_ALONG, PIECES_B, WAVES, RAW_B> StageB;
    static constexpr int kA = StageA::kPlanes * StageA::kBytes, kStage = kA + StageB::kPlanes * StageB::kBytes, kLds = STAGES * kStage;

    static __device__ __forceinline__ int lane() { return (int)threadIdx.x & 63; }
    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }
    // where this wave's results begin, and the row within a block of 32 x 32 of result i of a lane (its column is lane % 32)
    static __device__ __forceinline__ int m0() { return wave() / WAVES_N * WM; }
    static __device__ __forceinline__ int n0() { return wave() % WAVES_N * WN; }
    static __device__ __forceinline__ int row(int i) { return 8 * (i >> 2) + 4 * (lane() >> 5) + (i & 3); }

    // everything sent for has come, to all waves, but for the last PENDING loads of each
    template <int PENDING = 0>
    static __device__ __forceinline__ void arrive()
    {
        static_assert(PENDING < 64, "");
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(PENDING) : "memory");
    }

    static constexpr int kReadsB = StageB::kPlanes * NB;

    // The operands of one matrix step of sixteen contraction indices: those of B, then those of A
    struct Operands {
        s8v a[PIECES_A][MB], b[PIECES_B][NB];
        __device__ __forceinline__ void read(const lds_char *tile, int ks, int i)
        {
            const int l = lane();
            if (i < kReadsB) {
                if constexpr (RAW_B) raw_fragment<BN, BK, B_ALONG>(tile + kA, n0() + 32 * i, ks, l, b[0][i], b[1][i], b[2][i]);
                else b[i / NB][i % NB] = fragment<BN, BK, B_ALONG>(tile + kA + i / NB * StageB::kBytes, n0() + 32 * (i % NB), ks, l);
            } else {
                i -= kReadsB;
                if constexpr (RAW_A) raw_fragment<BM, BK, A_ALONG>(tile, m0() + 32 * i, ks, l, a[0][i], a[1][i], a[2][i]);
                else a[i / MB][i % MB] = fragment<BM, BK, A_ALONG>(tile + i / MB * StageA::kBytes, m0() + 32 * (i % MB), ks, l);
            }
        }
    };
    static constexpr int kReads = kReadsB + StageA::kPlanes * MB, kLoads = StageA::kAll + StageB::kAll;
    // a step's products in parts, between which reads and loads are issued: rows of blocks (of the smaller piece before those of the larger), or the products of
    // three pieces
    static constexpr int kParts = PIECES_A == 3 ? 6 : MB * PIECES_A * PIECES_B;
    static_assert(PIECES_A * PIECES_B <= 2 || (PIECES_A == 3 && PIECES_B == 3), "");

    static __device__ __forceinline__ void multiply(const Operands &o, TileAcc<T> (&acc)[MB][NB], int part)
    {
        if constexpr (PIECES_A == 3) {
            constexpr int PA[6] = {2, 1, 0, 1, 0, 0}, PB[6] = {0, 1, 2, 0, 1, 0};
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int n = 0; n < NB; ++n) acc[m][n].mac(o.a[PA[part]][m], o.b[PB[part]][n]);
        } else {
            const int piece = part / MB, m = part % MB, pa = PIECES_A == 2 ? 1 - piece : 0, pb = PIECES_B == 2 ? 1 - piece : 0;
#pragma unroll
            for (int n = 0; n < NB; ++n) acc[m][n].mac(o.a[pa][m], o.b[pb][n]);
        }
    }

    // One tile of contraction indices: the tile `here`, while the ones behind it are on their way.  `before`: the room of the tile before, which the
    // rest of tile STAGES - 1 from here goes to (with two stages that is `next`).
    static constexpr int kSteps = BK / 16, kEarly = (kLoads + 1) / 2, kAhead = STAGES > 2 ? (STAGES - 2) * kLoads : 0;
    static __device__ __forceinline__ void ask(const Operand &a, const Operand &b, const StageA &sa, const StageB &sb, int k0, lds_char *to, int j)
    {
        if (j < StageA::kAll) sa.ask(a, k0, to, j);
        else sb.ask(b, k0, to + kA, j - StageA::kAll);
    }
    static __device__ __forceinline__ void step(lds_char *__restrict here, lds_char *__restrict next, lds_char *before, const Operand &a, const Operand &b, const StageA &sa,
                                                const StageB &sb, int k0, Operands (&now)[2], TileAcc<T> (&acc)[MB][NB])
    {
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
            const bool last = ks + 1 == kSteps;
            __builtin_amdgcn_sched_barrier(0);
            if (last) arrive<kAhead>();
#pragma unroll
            for (int part = 0; part < kParts; ++part) {
                // reads in the first half of the parts, loads in all of them
                constexpr int HALF = (kParts + 1) / 2;
#pragma unroll
                for (int i = 0; i < kReads; ++i)
                    if (i * HALF / kReads == part) {
                        if (last) now[(ks + 1) & 1].read(next, 0, i);
                        else now[(ks + 1) & 1].read(here, ks + 1, i);
                    }
                if (last)
#pragma unroll
                    for (int j = 0; j < kEarly; ++j)
                        if (j * kParts / kEarly == part) ask(a, b, sa, sb, k0 + STAGES * BK, here, j);
                if (ks == 0)
#pragma unroll
                    for (int j = kEarly; j < kLoads; ++j)
                        if ((j - kEarly) * kParts / (kLoads - kEarly) == part) ask(a, b, sa, sb, k0 + (STAGES - 1) * BK, STAGES == 2 ? next : before, j);
                multiply(now[ks & 1], acc, part);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }

    // results = A B over `depth` contraction indices; LDS is free when it returns.  Two sets of operands in registers.  Between the parts of
    // a step's products the next step's operands are read; the last step of a tile begins with the barrier behind which the tile's room
    // is free: the loads that go there are issued in that step and the one behind it.  Tiles of 8192 x 4096 x 131072 in bf16 run at 1.33 to
    // 1.37 PFLOP/s along (256 x 256), 1.23 and 1.26 across (256 x 128, two pieces; a library's product 1.48).  For one piece four waves with 128 x 128 results each
    // were slower (1.06 to 1.3), so were tiles of 256 x 128 with two workgroups to a compute unit (1.06).
    static __device__ __forceinline__ void product(lds_char *lds, const Operand &a, const Operand &b, int depth, f16v (&results)[MB][NB])
    {
        const int l = lane(), w = wave();
        const StageA sa(a, w, l);
        const StageB sb(b, w, l);
        TileAcc<T> acc[MB][NB];
        Operands now[2];
        if constexpr (STAGES == 1) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) ask(a, b, sa, sb, 0, lds, j);
            arrive();
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) {
#pragma unroll
                for (int i = 0; i < kReads; ++i) now[ks & 1].read(lds, ks, i);
#pragma unroll
                for (int part = 0; part < kParts; ++part) multiply(now[ks & 1], acc, part);
            }
        } else {
#pragma unroll
            for (int t = 0; t < STAGES - 1; ++t)
#pragma unroll
                for (int j = 0; j < kLoads; ++j) ask(a, b, sa, sb, t * BK, lds + t * kStage, j);
            arrive<kAhead>();
#pragma unroll
            for (int j = 0; j < kEarly; ++j) ask(a, b, sa, sb, (STAGES - 1) * BK, lds + (STAGES - 1) * kStage, j);
#pragma unroll
            for (int i = 0; i < kReads; ++i) now[0].read(lds, 0, i);         // (of zeros where depth is 0)
            int at = 0;
            for (int k0 = 0; k0 < depth; k0 += BK) {
                const int behind = at + kStage < kLds ? at + kStage : 0, before = at > 0 ? at - kStage : kLds - kStage;
                step(lds + at, lds + behind, lds + before, a, b, sa, sb, k0, now, acc);
                at = behind;
            }
        }
        arrive();
        const TileSettled settled;
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int n = 0; n < NB; ++n) results[m][n] = acc[m][n].read(settled);
    }
};

// Which tile a workgroup takes.  Workgroups go to the eight dies in turn; each die gets a run of tiles and walks it with up to eight
// tiles of the second dimension side by side, so that tiles that run together share their operands in the die's L2.  Where the grid's other
// dimensions (whose steps are multiples of eight workgroups) have few tiles each, the die that begins turns with them.
struct Place {
    int m, n;
    bool any;
};

__device__ __forceinline__ Place place(int m_tiles, int n_tiles, int id, int turn)
{
    const int die = (id + turn) % 8;
    const int items = m_tiles * n_tiles, per_die = (items + 7) / 8, item = die * per_die + id / 8;
    if (id / 8 >= per_die || item >= items) return {0, 0, false};
    const int group = item / (8 * m_tiles), first = group * 8, wide = n_tiles - first < 8 ? n_tiles - first : 8, in = item - group * 8 * m_tiles;
    return {in / wide, first + in % wide, true};
}

__device__ __forceinline__ Place place(int m_tiles, int n_tiles) { return place(m_tiles, n_tiles, (int)blockIdx.x, (int)(blockIdx.y + blockIdx.z * gridDim.y)); }

__host__ __device__ inline long place_blocks(long m_tiles, long n_tiles) { return (m_tiles * n_tiles + 7) & ~7L; }

}  // namespace

#endif  // HOT_TILE_H
