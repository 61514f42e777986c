// A block's tile of a product of bfloat16 operands whose pieces of 16 bytes start on multiples of 4 bytes: copied from memory to LDS without passing through
// registers (buffer_load ... lds), into two or three buffers in turn.
//
// The tile's layout in LDS is that of matrix_tile.hpp.  The copy writes a wavefront's 64 pieces side by side, so a lane asks for the piece that belongs to
// its place.  What lies outside of an operand is asked for outside of the buffer's bounds and arrives as zero: rows past the end by the bounds themselves, k past the
// end of a row by an offset that is never inside.
//
// Bound by the matrix cores' rate at the clock that they leave (1.6 - 1.9 GHz) and by what of the copies is not hidden.  Measured on 65536 rows of 4096 by 1024: tiles of 128 by 128 by way of
// registers 835 us; 256 by 256 copied straight, four wavefronts, 614; eight wavefronts, two on each of the unit's four cores, 521 (1056 TFLOP/s; a large library product of
// these sizes reaches 1254).  Chunks of 32 k in three or four buffers, and two blocks of 128 rows a compute unit, were no faster.
//
// A chunk of 64 k is four steps.  A step's fragments are read from LDS while the products of the step before are formed; one wait and one barrier a chunk, in front of
// its last step, where all fragments of the chunk are in registers and the next chunk has arrived: behind it the copy of the chunk after that may go into the buffer
// that has just been read.
#pragma once
#include "matrix_tile.hpp"

namespace csgs {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// A wavefront's 64 pieces of 16 bytes to LDS, side by side from `lds` on (a byte offset, the same in all lanes).  Arrives unseen by the compiler: waited for by
// wait_and_meet.  (Between a write of m0 and its use one wait state.)
__device__ inline void copy_to_lds(i32x4 buffer, uint32_t offset, uint32_t base, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(buffer), "s"(base) : "memory");
}
// All but the last `LEFT` copies of this wavefront have arrived (they arrive in order) and every fragment is in registers; then the same of the block.
template <int LEFT>
__device__ inline void wait_and_meet()
{
    static_assert(LEFT < 64, "the counter's range");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}
__device__ inline uint32_t lds_offset(const void *p) { return (uint32_t)(uintptr_t)(CSGS_LDS const void *)p; }
__device__ inline int32_t one_for_all(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

constexpr uint32_t NOWHERE = 0x7FFFFFF0u;     // an offset outside of every buffer

template <int R, bool ACROSS, int NT, int ROWB>
struct DirectSide {
    using Layout = TileSide<uint16_t, R, ACROSS, NT, ROWB>;
    static constexpr int PIECES = Layout::PIECES, BK = Layout::BK;
    // pieces of a thread lie NT places apart: this many rows of the tile.  Rows 16 apart are turned alike
    static constexpr int ROWS = NT / Layout::ROW_PIECES, TURNS = ROWS % 16 == 0 ? 1 : 2;
    static_assert(ACROSS || TURNS == 1, "one k for all pieces of a lane");
    static_assert(NT % Layout::ROW_PIECES == 0 && ROWS % 8 == 0, "rows that are turned alike, or every second one");

    const char *base;      // of the tile's first row and k = 0
    int64_t bytes;         // from there to the end of the operand's last entry
    uint32_t offset[TURNS], row_bytes;
    int32_t my_k;          // of this lane's pieces (k side by side)

    // Entries o0 .. of `outer`, k from 0 to red.
    __device__ CSGS_INLINE void start(const Operand &op, int64_t o0, int64_t outer, int64_t red)
    {
        row_bytes = (uint32_t)(op.ld * 2);
        base = (const char *)op.p + (ACROSS ? o0 : o0 * op.ld) * 2;
        bytes = (ACROSS ? (red - 1) * op.ld + outer - o0 : (outer - 1 - o0) * op.ld + red) * 2;
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            int o, k;
            Layout::piece((int)threadIdx.x + i * NT, &o, &k);
            // (relative to row i * ROWS of the tile, which `base` of copy_to_lds adds)
            if constexpr (!ACROSS) {
                my_k = k;
                offset[i] = (uint32_t)(o - i * ROWS) * row_bytes + (uint32_t)k * 2;
            } else {
                offset[i] = o0 + o < outer ? (uint32_t)(k - i * ROWS) * row_bytes + (uint32_t)o * 2 : NOWHERE;
            }
        }
    }
    // Piece i of this thread of the k from `k` on, below red, to a buffer.
    __device__ CSGS_INLINE void copy(int i, int64_t k, int64_t red, uint32_t lds) const
    {
        const int64_t skip = ACROSS ? k * (int64_t)row_bytes : k * 2, left = bytes - skip;
        const char *from = base + skip;
        const i32x4 buffer = {one_for_all((int32_t)(uintptr_t)from), one_for_all((int32_t)((uintptr_t)from >> 32)),
                              one_for_all(left < 0 ? 0 : left < NOWHERE ? (int32_t)left : (int32_t)NOWHERE), 0x00020000};
        const bool inside = ACROSS || k + my_k < red;
        const uint32_t to = (uint32_t)one_for_all((int32_t)(lds + (threadIdx.x / WAVE) * (WAVE * 16)));
        copy_to_lds(buffer, inside ? offset[i % TURNS] : NOWHERE, (uint32_t)one_for_all((int32_t)(i * ROWS * row_bytes)), to + i * NT * 16);
    }
};

template <int BM, int BN, int WM, int WN, bool A_ACROSS, bool B_ACROSS, int NB, int ROWB, int BUFFERS>
struct DirectTile : MatrixTile<uint16_t, BM, BN, WM, WN, A_ACROSS, B_ACROSS, NB, ROWB> {
    using Base = MatrixTile<uint16_t, BM, BN, WM, WN, A_ACROSS, B_ACROSS, NB, ROWB>;
    using Base::acc;
    using Base::NT;
    using Base::TM;
    using Base::TN;
    using LayoutA = typename Base::SideA;
    using LayoutB = typename Base::SideB;
    static constexpr int BUFFER = Base::TILE_BYTES, LDS_BYTES = BUFFERS * BUFFER > Base::OUT_BYTES ? BUFFERS * BUFFER : Base::OUT_BYTES, BK = Base::BK;
    static constexpr int STEPS = Base::STEPS, WAVES = LDS_BYTES > 80 * 1024 ? NT / 256 : 2;     // (one block a compute unit, or two)
    using SideA = DirectSide<BM, A_ACROSS, NT, ROWB>;
    using SideB = DirectSide<BN, B_ACROSS, NT, ROWB>;

    static constexpr int PRODUCTS = NB * TN * TM, READS = NB * TN + TM;
    struct Fragments {
        bf16x8 a[TM], b[NB * TN];
    };
    // Fragment i of a step, in the order in which the products below ask for them.
    static __device__ CSGS_INLINE inline void read(Fragments &f, int i, const char *lds, int step, int m0, int n0, int lane)
    {
        if (i == 0 || i > TM) {
            const int n = i == 0 ? 0 : i - TM;
            f.b[n] = LayoutB::fragment(lds + LayoutA::BYTES + n / TN * LayoutB::BYTES, n0 + 32 * (n % TN), step, lane);
        } else {
            f.a[i - 1] = LayoutA::fragment(lds, m0 + 32 * (i - 1), step, lane);
        }
    }
    // A step's products, `beside(i)` behind the i-th of them: what is asked for there is on its way while the next ones are formed.  (The order is kept: left to itself
    // the compiler puts a step's reads behind its products and waits for them.)
    template <typename F>
    __device__ CSGS_INLINE inline void products(const Fragments &f, F beside)
    {
        each_of<PRODUCTS>([&](auto i) CSGS_INLINE {
            constexpr int n = i / TM, m = i % TM;
            acc[n / TN][n % TN][m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.b[n], f.a[m], acc[n / TN][n % TN][m], 0, 0, 0);
            beside(i);
            __builtin_amdgcn_sched_barrier(0);
        });
    }

    __device__ CSGS_INLINE void accumulate(char *lds, const Operand &a, const Operand *b, int64_t m0, int64_t rows, int64_t n0, int64_t cols, int64_t k0, int64_t k1)
    {
        if (k0 >= k1) return;
        const int lane = (int)threadIdx.x & (WAVE - 1), wave = (int)threadIdx.x / WAVE;
        const int wm = wave / WN * (TM * 32), wn = wave % WN * (TN * 32);
        SideA sa;
        SideB sb[NB];
        sa.start(a, m0, rows, k1);
#pragma unroll
        for (int i = 0; i < NB; ++i) sb[i].start(b[i], n0, cols, k1);
        const uint32_t first = lds_offset(lds);
        // one of the pieces that a thread copies of a chunk
        constexpr int COPIES = SideA::PIECES + NB * SideB::PIECES;
        auto copy = [&](int i, int64_t k, uint32_t to) CSGS_INLINE {
            if (i < SideA::PIECES) sa.copy(i, k, k1, to);
            else sb[(i - SideA::PIECES) / SideB::PIECES].copy((i - SideA::PIECES) % SideB::PIECES, k, k1, to + LayoutA::BYTES + (i - SideA::PIECES) / SideB::PIECES * LayoutB::BYTES);
        };
        const int32_t chunks = (int32_t)((k1 - k0 + BK - 1) / BK);
        int64_t k = k0;                 // of the next chunk to be copied; past the last one: zeros
        wait_and_meet<0>();             // (the buffers' readers of an earlier call are done)
        each_of<BUFFERS>([&](auto n) CSGS_INLINE {
            each_of<COPIES>([&](auto i) CSGS_INLINE { copy(i, k, first + n * BUFFER); });
            k += BK;
        });
        wait_and_meet<(BUFFERS - 1) * COPIES>();
        Fragments f[2];
        each_of<READS>([&](auto i) CSGS_INLINE { read(f[0], i, lds, 0, wm, wn, lane); });
        int32_t here = 0;               // the buffer's place in LDS
        for (int32_t c = 0; c < chunks; ++c) {
            each_of<STEPS - 1>([&](auto step) CSGS_INLINE {
                products(f[step & 1], [&](int i) CSGS_INLINE {
                    if (i < READS) read(f[(step & 1) ^ 1], i, lds + here, step + 1, wm, wn, lane);
                });
            });
            wait_and_meet<(BUFFERS - 2) * COPIES>();
            // (behind the last chunks: zeros, and fragments that no product takes)
            const int32_t next = here + BUFFER < BUFFERS * BUFFER ? here + BUFFER : 0;
            products(f[(STEPS - 1) & 1], [&](int i) CSGS_INLINE {
                if (i < READS) read(f[STEPS & 1], i, lds + next, 0, wm, wn, lane);
#pragma unroll
                for (int j = i * COPIES / PRODUCTS; j < (i + 1) * COPIES / PRODUCTS; ++j) copy(j, k, first + here);
            });
            k += BK;
            here = next;
        }
        wait_and_meet<0>();
    }
    static_assert(STEPS % 2 == 0 && READS <= PRODUCTS, "fragments in turn, all asked for beside a step's products");
};

// Whether an operand's tiles can be copied so: outer by red entries, at most `tile` of the former in one tile.
inline bool direct_operand(const Operand &op, bool across, int64_t outer, int64_t red, int64_t tile)
{
    if (((uintptr_t)op.p & 3) || op.ld % 2 || op.ld > (int64_t)1 << 30) return false;
    if (across) return outer % 2 == 0 && (64 * op.ld + tile) * 2 < (int64_t)NOWHERE;
    return red % 8 == 0 && (tile * op.ld + red) * 2 < (int64_t)NOWHERE;
}

}  // namespace csgs
