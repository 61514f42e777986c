// A block's tile of a product of floats, on the bfloat16 matrix cores.
//
// A float is the sum of three bfloat16 numbers, exactly: itself rounded, h; what that leaves rounded, m; and l = x - h - m, of which 7 bits are left.  Rounded to nearest, for x in [1, 2)
// |m| <= 2^-8 and |l| <= 2^-17.  Of the nine products of two such sums the six with weights down to 2^-16 are formed,
//     a b = ah bh + (ah bm + am bh) + (ah bl + am bm + al bh) + rest,     |rest| = |am bl + al bm + al bl| <= 1.001 2^-24 |a b|, of either sign
// (parts that are cut off, not rounded, leave up to 8 times as much, always of the product's sign; each product is formed by the matrix cores without a rounding and summed in float): a product
// costs six times 32 cycles a step of 16 k instead of 8 times 64 on the float cores.  ah bh has sums of its own, the others share one set, which is added at the end: the large sums are
// rounded once for 16 k.  A bfloat16 number's lowest bit is 2^-133 at least, a float's 2^-149: operands are split 2^16 times as large, exactly, sums divided by 2^32 at the end, so that every
// float has its parts, those below 2^-126 too (which the matrix cores take and give).
// Bound by six products and by the splitting in front of LDS, 13 operations for two entries, which each block does for itself between two barriers (4001 rows of 602 by 1111, gated, with all
// gradients: 453 us on the float cores, 282 so, 114 TFLOP/s as floats count, 292 on a slower card; relative error against 64 bits 1.2e-6 on the float cores, 2.5e-7 so; 8192 rows of 1024 by
// 256 41 us, 105 TFLOP/s; 32768 rows of 1024 by 1024 404 us, 170).  The scale costs 2 to 4 % of that.  Two sets of sums and the pieces on their way take 219 to 242 of the 256 registers that two
// blocks a compute unit leave a lane; LDS would hold more (48 KB of 160 at 128 by 128).
//
// The parts are not all finite where x is not, and from 2^112 on.  Sums that are not finite, as they are of such parts and from 2^96 on, are formed again, by the float cores: those give what
// the inputs do.
#pragma once
#include "matrix_tile.hpp"

namespace csgs {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
constexpr float SPLIT_SCALE = 65536.0f, SPLIT_BACK = 1.0f / 65536.0f / 65536.0f;

template <int R, bool ACROSS, int NT>
struct SplitSide {
    using Layout = TileSide<uint16_t, R, ACROSS, NT, 64>;        // of each of the three planes
    static constexpr int PIECES = Layout::PIECES, BYTES = 3 * Layout::BYTES;

    float held[PIECES][8];
    __device__ CSGS_INLINE void ask(int tid, const Operand &op, int64_t o0, int64_t outer, int64_t k0, int64_t red)
    {
        const float *base = (const float *)op.p;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            int po, pk;
            Layout::piece(tid + i * NT, &po, &pk);
            const int64_t o = o0 + po, k = k0 + pk;
            const int64_t rest = ACROSS ? (k < red ? outer - o : 0) : (o < outer ? red - k : 0);
            const float *from = base + (ACROSS ? k * op.ld + o : o * op.ld + k);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                const int64_t n = rest - 4 * h;
                if (n > 0) load_some(from + 4 * h, n < 4 ? (int)n : 4, x);
#pragma unroll
                for (int e = 0; e < 4; ++e) held[i][4 * h + e] = x[e];
            }
        }
    }
    __device__ CSGS_INLINE void put(int tid, char *lds) const
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            u32x4 plane[3];
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                float x[2] = {held[i][e] * SPLIT_SCALE, held[i][e + 1] * SPLIT_SCALE};
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    plane[q][e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[0], x[1]}), bf16x2));
                    x[0] -= __uint_as_float(plane[q][e / 2] << 16);
                    x[1] -= __uint_as_float(plane[q][e / 2] & 0xFFFF0000u);
                }
            }
#pragma unroll
            for (int q = 0; q < 3; ++q) *(u32x4 *)(lds + q * Layout::BYTES + (tid + i * NT) * 16) = plane[q];
        }
    }
};

template <int BM, int BN, int WM, int WN, bool A_ACROSS, bool B_ACROSS, int NB, int KG>
struct SplitTile : MatrixTile<float, BM, BN, WM, WN, A_ACROSS, B_ACROSS, NB, 128, KG> {
    using Base = MatrixTile<float, BM, BN, WM, WN, A_ACROSS, B_ACROSS, NB, 128, KG>;
    using Base::acc;
    using Base::NT;
    using Base::TM;
    using Base::TN;
    using SideA = SplitSide<BM, A_ACROSS, NT>;
    using SideB = SplitSide<BN, B_ACROSS, NT>;
    static constexpr int BK = 32, STEPS = 2;
    static constexpr int SPLIT_BYTES = SideA::BYTES + NB * SideB::BYTES, LDS_BYTES = Base::larger(KG * SPLIT_BYTES, Base::LDS_BYTES);

    Base second;      // sums of the smaller products; then, where they are asked for, of the float cores

    __device__ CSGS_INLINE void clear()
    {
        Base::clear();
        second.clear();
    }
    __device__ CSGS_INLINE void multiply(const char *lds)
    {
        const int lane = (int)threadIdx.x & (WAVE - 1), wave = Base::my_wave();
        const int m0 = wave / WN * (TM * 32), n0 = wave % WN * (TN * 32);
        each_of<STEPS>([&](auto step) CSGS_INLINE {
            bf16x8 a[3][TM];
            each_of<3 * TM>([&](auto i) CSGS_INLINE { a[i / TM][i % TM] = SideA::Layout::fragment(lds + i / TM * SideA::Layout::BYTES, m0 + 32 * (i % TM), step, lane); });
            each_of<NB * TN>([&](auto j) CSGS_INLINE {
                constexpr int b = j / TN, n = j % TN;
                bf16x8 f[3];
                each_of<3>([&](auto q) CSGS_INLINE {
                    f[q] = SideB::Layout::fragment(lds + SideA::BYTES + b * SideB::BYTES + q * SideB::Layout::BYTES, n0 + 32 * n, step, lane);
                });
                // (small products first)
                each_of<6 * TM>([&](auto i) CSGS_INLINE {
                    constexpr int which = i / TM, m = i % TM;
                    constexpr int pa[6] = {2, 1, 0, 1, 0, 0}, pb[6] = {0, 1, 2, 0, 1, 0};
                    f32x16 &sum = which == 5 ? acc[b][n][m] : second.acc[b][n][m];
                    sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[pb[which]], a[pa[which]][m], sum, 0, 0, 0);
                });
            });
        });
    }
    __device__ CSGS_INLINE void accumulate(char *lds, const Operand &a, const Operand *b, int64_t m0, int64_t rows, int64_t n0, int64_t cols, int64_t k0, int64_t k1)
    {
        SideA sa;
        SideB sb[NB];
        const int tid = Base::my_id(), group = Base::my_group();
        const auto ask = [&](int64_t k) CSGS_INLINE {
            sa.ask(tid, a, m0, rows, k, k1);
            each_of<NB>([&](auto i) CSGS_INLINE { sb[i].ask(tid, b[i], n0, cols, k, k1); });
        };
        if (k0 >= k1) return;
        char *mine = lds + group * SPLIT_BYTES;
        ask(k0 + group * BK);
        for (int64_t k = k0; k < k1; k += KG * BK) {
            __syncthreads();       // (the buffer's last readers are done)
            sa.put(tid, mine);
            each_of<NB>([&](auto i) CSGS_INLINE { sb[i].put(tid, mine + SideA::BYTES + i * SideB::BYTES); });
            __syncthreads();
            if (k + KG * BK < k1) ask(k + (KG + group) * BK);
            multiply(mine);
        }
    }
    static __device__ CSGS_INLINE bool finite(float x) { return fabsf(x) <= 3.4028234e38f; }
    // The sums as a whole; whether one of the block's is not finite.
    __device__ CSGS_INLINE bool settle(char *lds)
    {
        bool bad = false;
        each_of<NB * TN * TM>([&](auto i) CSGS_INLINE { acc[i / (TN * TM)][i / TM % TN][i % TM] += second.acc[i / (TN * TM)][i / TM % TN][i % TM]; });
        Base::join(lds);
        each_of<NB * TN * TM>([&](auto i) CSGS_INLINE {
            f32x16 &x = acc[i / (TN * TM)][i / TM % TN][i % TM];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[r] *= SPLIT_BACK;
                bad |= !finite(x[r]);
            }
        });
        return __syncthreads_or(bad);
    }
    // Sums that are not finite are those of the float cores (the others stay: a row's sums do not depend on other rows).
    template <typename F>
    __device__ CSGS_INLINE void again(char *lds, F sum)
    {
        second.clear();
        sum(second);
        second.join(lds);
        each_of<NB * TN * TM>([&](auto i) CSGS_INLINE {
            f32x16 &x = acc[i / (TN * TM)][i / TM % TN][i % TM];
            const f32x16 y = second.acc[i / (TN * TM)][i / TM % TN][i % TM];
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = finite(x[r]) ? x[r] : y[r];
        });
    }
};

// The tile for operands that start anywhere.
template <typename T, int BM, int BN, int WM, int WN, bool A_ACROSS, bool B_ACROSS, int NB, int KG = 1>
using AnyTile = std::conditional_t<sizeof(T) == 4, SplitTile<BM, BN, WM, WN, A_ACROSS, B_ACROSS, NB, KG>, MatrixTile<T, BM, BN, WM, WN, A_ACROSS, B_ACROSS, NB, 128, KG>>;

}  // namespace csgs
