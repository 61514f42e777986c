// A block's tile of a product C [m x n] = A B on the matrix cores, for operands in bfloat16 or float whose rows start on any element.
//
// An operand is seen as outer index times reduction index k.  It lies in memory either with k side by side (ACROSS = false) or with the outer
// index side by side (ACROSS = true); a tile is copied to LDS as it lies, in pieces of 16 bytes:
//   k side by side      [outer][128 or 64 bytes of k]: a lane's part of a row is one 16-byte read.  Rows that are read together would meet in
//                       the same banks: the pieces of a row are kept in an order that its number turns.
//   outer side by side  [k][outer]: bfloat16 is turned by the LDS's transposing read (ds_read_b64_tr_b16: 16 lanes read 4 rows of k by 16
//                       columns, each gets its column's 4 values); floats are read one by one.  32-byte segment s of row k at s ^ f(k), so that the four
//                       rows of a read and those of its neighbours lie in different banks.
// Products: v_mfma_f32_32x32x16_bf16 and v_mfma_f32_32x32x2_f32, sums in float.  The B operand is given to the instruction as its rows, so that a
// lane ends up with four neighbouring columns of a row of C.
#pragma once
#include "common.hpp"
#include "row_pieces.hpp"

namespace csgs {

#define CSGS_LDS __attribute__((address_space(3)))
#define CSGS_INLINE __attribute__((always_inline))     // (of a lambda: what it captures stays in registers)
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// f(0), f(1) .. f(N - 1) with the numbers as constants: an array that is indexed so is registers from the first pass of the compiler on, however large what surrounds it.
template <int N, typename F>
__device__ CSGS_INLINE inline void each_of(F f)
{
    if constexpr (N > 0) {
        each_of<N - 1>(f);
        f(std::integral_constant<int, N - 1>());
    }
}

// An operand: element (o, k) at p[o * ld + k], or p[k * ld + o] where the outer index lies side by side.
struct Operand {
    const void *p;
    int64_t ld;
};


// Which 32-byte segment of a row of k holds segment s (R outer entries of bfloat16 a row).
template <int R>
__device__ inline int across_turn(int k)
{
    if constexpr (R * 2 >= 256) return 2 * (k & 3) | ((k >> 3) & 1);
    return 2 * ((k >> 1) & 1) | ((k >> 3) & 1);
}

// Where piece 0 of row r is kept among the pieces of its row (rows of ROWB bytes): rows that share banks differ.
template <int ROWB>
__device__ inline int along_turn(int row)
{
    static_assert(ROWB == 128 || ROWB == 64, "rows of 128 or 64 bytes");
    return ROWB == 128 ? (row >> 1) & 7 : (row >> 2) & 3;
}

// R outer entries by BK of an operand, ROWB bytes of k: copied to LDS by NT threads, read from there by wavefronts.
template <typename T, int R, bool ACROSS, int NT, int ROWB>
struct TileSide {
    static constexpr int BK = ROWB / (int)sizeof(T), PIECE = 16 / (int)sizeof(T);
    static constexpr int BYTES = R * ROWB;
    static constexpr int PIECES = R * (ROWB / 16) / NT;     // a thread's
    static_assert(R * (ROWB / 16) % NT == 0 && PIECES >= 1, "whole pieces for every thread");
    static constexpr int ROW_PIECES = ACROSS ? R / PIECE : ROWB / 16;

    // The first element of the piece that belongs to place `id` of the tile.
    static __device__ inline void piece(int id, int *o, int *k)
    {
        const int row = id / ROW_PIECES, place = id % ROW_PIECES;
        if constexpr (!ACROSS) {
            *o = row;
            *k = (place ^ along_turn<ROWB>(row)) * PIECE;
        } else {
            *k = row;
            if constexpr (sizeof(T) == 2) *o = (((((place >> 1) ^ across_turn<R>(row)) << 1) | (place & 1))) * PIECE;
            else *o = place * PIECE;
        }
    }

    // Pieces by way of registers: anything outside the operand is zero.
    u32x4 held[PIECES];
    __device__ CSGS_INLINE void ask(int tid, const Operand &op, int64_t o0, int64_t outer, int64_t k0, int64_t red)
    {
        const T *base = (const T *)op.p;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            int po, pk;
            piece(tid + i * NT, &po, &pk);
            const int64_t o = o0 + po, k = k0 + pk;
            const int64_t at = ACROSS ? k * op.ld + o : o * op.ld + k;
            const int64_t rest = ACROSS ? (k < red ? outer - o : 0) : (o < outer ? red - k : 0);
            if (rest >= PIECE) {
                held[i] = load_global<u32x4, (int)sizeof(T)>(base + at);
            } else {
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < PIECE; ++e)
                    if (e < rest) {
                        if constexpr (sizeof(T) == 4) w[e] = load_global<uint32_t>(base + at + e);
                        else w[e / 2] |= (uint32_t)load_global<uint16_t>(base + at + e) << (16 * (e & 1));
                    }
                held[i] = u32x4{w[0], w[1], w[2], w[3]};
            }
        }
    }
    __device__ CSGS_INLINE void put(int tid, char *lds) const
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) *(u32x4 *)(lds + (tid + i * NT) * 16) = held[i];
    }

    // What a lane gives the matrix cores for the 32 outer entries from `first` on, of k from 16 * step (bfloat16) or 8 * step (floats) on.
    static __device__ CSGS_INLINE inline bf16x8 fragment(const char *lds, int first, int step, int lane)
    {
        static_assert(sizeof(T) == 2, "bfloat16");
        if constexpr (!ACROSS) {
            const int row = first + (lane & 31), g = 2 * step + (lane >> 5);
            return *(const bf16x8 *)(lds + row * ROWB + ((g ^ along_turn<ROWB>(row)) << 4));
        } else {
            const int i = lane & 15, k = step * 16 + 8 * (lane >> 5) + (i >> 2);
            const int segment = first / 16 + ((lane >> 4) & 1);
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            s16x4 part[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int kk = k + 4 * h;
                const char *at = lds + kk * (R * 2) + ((segment ^ across_turn<R>(kk)) << 5) + (i & 3) * 8;
                part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((CSGS_LDS s16x4 *)(CSGS_LDS void *)at);
            }
            const s16x8 both = {part[0].x, part[0].y, part[0].z, part[0].w, part[1].x, part[1].y, part[1].z, part[1].w};
            return __builtin_bit_cast(bf16x8, both);
        }
    }
    static __device__ CSGS_INLINE inline f32x4 fragment_f32(const char *lds, int first, int step, int lane)
    {
        static_assert(sizeof(T) == 4, "floats");
        if constexpr (!ACROSS) {
            const int row = first + (lane & 31), g = 2 * step + (lane >> 5);
            return *(const f32x4 *)(lds + row * ROWB + ((g ^ along_turn<ROWB>(row)) << 4));
        } else {
            const float *at = (const float *)lds + (step * 8 + 4 * (lane >> 5)) * R + first + (lane & 31);
            return f32x4{at[0], at[R], at[2 * R], at[3 * R]};
        }
    }
};

// The tile: BM rows and, of each of NB matrices B, BN columns; WM x WN wavefronts, KG times: where there are few tiles of long sums, KG groups of wavefronts take
// the chunks of k in turn, and the first one adds up what they have, in their order, and gives it out.
template <typename T, int BM, int BN, int WM, int WN, bool A_ACROSS, bool B_ACROSS, int NB, int ROWB = 128, int KG = 1>
struct MatrixTile {
    static constexpr int ROWS = BM, COLS = BN, WAVES_M = WM, WAVES_N = WN, NT = WM * WN * WAVE, THREADS = NT * KG, BK = ROWB / (int)sizeof(T), STEPS = ROWB / 32;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;     // 32 x 32 tiles of a wavefront
    static_assert(TM >= 1 && TN >= 1 && TM * 32 * WM == BM && TN * 32 * WN == BN, "whole tiles");
    using SideA = TileSide<T, BM, A_ACROSS, NT, ROWB>;
    using SideB = TileSide<T, BN, B_ACROSS, NT, ROWB>;
    // sums on their way out: 32 rows of a wavefront, rows 16 bytes further apart than they are long (lanes that write one below the other would meet in a bank)
    static constexpr int ROW_LANES = TN * 8, PITCH = TN * 32 + 4, STRIP = NB * 32 * PITCH * 4;
    static constexpr int TILE_BYTES = SideA::BYTES + NB * SideB::BYTES, OUT_BYTES = WM * WN * STRIP;
    static constexpr int SUMS = NB * TN * TM * 16, JOIN_BYTES = (KG - 1) * SUMS * NT * 4;
    static constexpr int larger(int a, int b) { return a > b ? a : b; }
    static constexpr int LDS_BYTES = larger(KG * TILE_BYTES, larger(OUT_BYTES, JOIN_BYTES));

    // This thread in its group, and the group.
    static __device__ inline int my_id() { return KG == 1 ? (int)threadIdx.x : (int)threadIdx.x % NT; }
    static __device__ inline int my_group() { return KG == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / NT); }
    static __device__ inline int my_wave() { return my_id() / WAVE; }

    static constexpr int WAVES = THREADS > 512 ? THREADS / 256 : 2;       // wavefronts that a SIMD is to hold

    f32x16 acc[NB][TN][TM];

    __device__ CSGS_INLINE void clear()
    {
        each_of<NB * TN * TM>([&](auto i) CSGS_INLINE { acc[i / (TN * TM)][i / TM % TN][i % TM] = f32x16{}; });
    }

    __device__ CSGS_INLINE void multiply(const char *lds)
    {
        const int lane = (int)threadIdx.x & (WAVE - 1), wave = my_wave();
        const int m0 = wave / WN * (TM * 32), n0 = wave % WN * (TN * 32);
        each_of<STEPS>([&](auto step) CSGS_INLINE {
            if constexpr (sizeof(T) == 2) {
                bf16x8 a[TM];
                each_of<TM>([&](auto m) CSGS_INLINE { a[m] = SideA::fragment(lds, m0 + 32 * m, step, lane); });
                each_of<NB * TN>([&](auto i) CSGS_INLINE {
                    constexpr int b = i / TN, n = i % TN;
                    const bf16x8 f = SideB::fragment(lds + SideA::BYTES + b * SideB::BYTES, n0 + 32 * n, step, lane);
                    each_of<TM>([&](auto m) CSGS_INLINE { acc[b][n][m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, a[m], acc[b][n][m], 0, 0, 0); });
                });
            } else {
                f32x4 a[TM];
                each_of<TM>([&](auto m) CSGS_INLINE { a[m] = SideA::fragment_f32(lds, m0 + 32 * m, step, lane); });
                each_of<NB * TN>([&](auto i) CSGS_INLINE {
                    constexpr int b = i / TN, n = i % TN;
                    const f32x4 f = SideB::fragment_f32(lds + SideA::BYTES + b * SideB::BYTES, n0 + 32 * n, step, lane);
                    each_of<4 * TM>([&](auto j) CSGS_INLINE {
                        constexpr int k = j / TM, m = j % TM;
                        acc[b][n][m] = __builtin_amdgcn_mfma_f32_32x32x2f32(f[k], a[m][k], acc[b][n][m], 0, 0, 0);
                    });
                });
            }
        });
    }

    // Adds the products over k in [k0, k1): rows from m0 on of `rows`, columns from n0 on of `cols`.  One buffer in LDS: the next pieces are on their way
    // while this one's products are formed.
    __device__ CSGS_INLINE void accumulate(char *lds, const Operand &a, const Operand *b, int64_t m0, int64_t rows, int64_t n0, int64_t cols, int64_t k0, int64_t k1)
    {
        SideA sa;
        SideB sb[NB];
        const int tid = my_id(), group = my_group();
        const auto ask = [&](int64_t k) CSGS_INLINE {
            sa.ask(tid, a, m0, rows, k, k1);
            each_of<NB>([&](auto i) CSGS_INLINE { sb[i].ask(tid, b[i], n0, cols, k, k1); });
        };
        if (k0 >= k1) return;
        char *mine = lds + group * TILE_BYTES;
        const int64_t first = k0 + group * BK;
        ask(first);
        // (all groups go round equally often: k past the end is zeros)
        for (int64_t k = k0; k < k1; k += KG * BK) {
            __syncthreads();       // (the buffer's last readers are done)
            sa.put(tid, mine);
            each_of<NB>([&](auto i) CSGS_INLINE { sb[i].put(tid, mine + SideA::BYTES + i * SideB::BYTES); });
            __syncthreads();
            if (k + KG * BK < k1) ask(k + (KG + group) * BK);
            multiply(mine);
        }
    }
    // The groups' sums, in the first one.
    __device__ CSGS_INLINE void join(char *lds)
    {
        if constexpr (KG > 1) {
            float *at = (float *)lds + my_id();
            const int group = my_group();
            __syncthreads();
            if (group > 0)
                each_of<SUMS>([&](auto i) CSGS_INLINE { at[((group - 1) * SUMS + i) * NT] = acc[i / 16 / (TN * TM)][i / 16 / TM % TN][i / 16 % TM][i % 16]; });
            __syncthreads();
            if (group == 0)
                each_of<SUMS>([&](auto i) CSGS_INLINE {
                    float x = acc[i / 16 / (TN * TM)][i / 16 / TM % TN][i / 16 % TM][i % 16];
#pragma unroll
                    for (int g = 0; g < KG - 1; ++g) x += at[(g * SUMS + i) * NT];
                    acc[i / 16 / (TN * TM)][i / 16 / TM % TN][i / 16 % TM][i % 16] = x;
                });
        }
    }

    // Whether sums have to be formed again: never here.
    __device__ CSGS_INLINE bool settle(char *lds)
    {
        join(lds);
        return false;
    }
    template <typename F>
    __device__ CSGS_INLINE void again(char *, F) {}

    // give(row in the tile, first of four columns in it, the values of the NB matrices, what ask(row, column) has answered) for all of the tile.  A wavefront's sums go through
    // LDS, 32 rows at a time, so that its lanes take whole rows of what is read and written beside them; a lane's columns are the same in every call.  What is asked for
    // is asked for together, a group of rows ahead of where it is needed: few wavefronts are here to wait for it.
    template <typename Ask, typename Give>
    __device__ CSGS_INLINE void each(char *lds, Ask ask, Give give) const
    {
        const int lane = (int)threadIdx.x & (WAVE - 1), wave = my_wave();
        const int m0 = wave / WN * (TM * 32) + lane / ROW_LANES, n0 = my_column();
        float *strip = (float *)lds + wave * (STRIP / 4);
        const float *mine = strip + lane / ROW_LANES * PITCH + lane % ROW_LANES * 4;
        constexpr int STEP = WAVE / ROW_LANES, GROUP = 16 / STEP;      // two groups of rows of a strip
        using Held = decltype(ask(0, 0));
        Held held[2][GROUP];
        __syncthreads();           // (the tiles' readers are done)
        if (my_group() > 0) return;
        each_of<GROUP>([&](auto i) CSGS_INLINE { held[0][i] = ask(m0 + i * STEP, n0); });
#pragma unroll 1
        for (int m = 0; m < TM; ++m) {
            // (a branch for each of them: registers have no index.  The empty statement differs from branch to branch, so that they are not made one, of an index, again)
            each_of<TM>([&](auto k) CSGS_INLINE {
                if (k == m) {
                    each_of<NB * TN * 4>([&](auto i) CSGS_INLINE {
                        constexpr int b = i / (TN * 4), n = i / 4 % TN, q = i % 4;
                        const f32x16 x = acc[b][n][k];
                        *(f32x4 *)(strip + (b * 32 + (lane & 31)) * PITCH + 32 * n + 8 * q + 4 * (lane >> 5)) = f32x4{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
                    });
                    asm volatile("; rows %0" ::"n"(32 * decltype(k)::value));
                }
            });
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            each_of<2>([&](auto g) CSGS_INLINE {
                const int next = 32 * m + 16 * (g + 1);
                if (next < 32 * TM) each_of<GROUP>([&](auto i) CSGS_INLINE { held[g ^ 1][i] = ask(m0 + next + i * STEP, n0); });
                each_of<GROUP>([&](auto i) CSGS_INLINE {
                    float v[NB][4];
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        const f32x4 x = *(const f32x4 *)(mine + (b * 32 + 16 * g + i * STEP) * PITCH);
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[b][e] = x[e];
                    }
                    give(m0 + 32 * m + 16 * g + i * STEP, n0, v, held[g][i]);
                });
            });
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    // The first of the four columns of the tile that this lane is given.
    static __device__ inline int my_column()
    {
        const int lane = (int)threadIdx.x & (WAVE - 1), wave = my_wave();
        return wave % WN * (TN * 32) + lane % ROW_LANES * 4;
    }
    // What the lanes of a wavefront hold for their columns, added up in a fixed order; f(first of four columns, sums) in one lane of each.
    template <typename F>
    static __device__ CSGS_INLINE void columns(float (&s)[4], F f)
    {
        const int lane = (int)threadIdx.x & (WAVE - 1);
        if (my_group() > 0) return;
#pragma unroll
        for (int d = ROW_LANES; d < WAVE; d <<= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += __shfl_xor(s[i], d);
        if (lane < ROW_LANES) f(my_column(), s);
    }
};

}  // namespace csgs
