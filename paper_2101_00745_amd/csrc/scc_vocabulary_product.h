// The matrix product of the vocabulary loss: a tile of BM x BN sums over K per workgroup of four wavefronts, on the matrix cores.
//
// An operand is 16-bit, NP planes of it: one (bf16, or fp16 where HALF), or three, whose sum is a binary32 value (the exact cut of split3; six
// of the nine products are taken).  Its K values are consecutive in memory ("along"), or its rows are ("across": the operand is K x rows
// and is turned on its way out of LDS by ds_read_b64_tr_b16).  Tiles of BK of K go straight into LDS (global_load_lds, 16 bytes a
// lane), three buffers in a ring: while one is multiplied the next is complete and the one after it under way, and one barrier a step is enough.
// A wavefront has a quarter of the tile, a grid of 32 x 32 accumulators.  LDS is read without bank conflicts: in 256 bytes of LDS, which one
// phase of a read covers, 16-byte chunks (along) or 64-byte ones (across) of consecutive rows are exchanged by an exclusive or with the row.
#pragma once
#include "scc_common.h"

namespace scc {
namespace vocabulary {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Operand {
    const uint16_t* at;
    long long plane, ld;            // elements from plane to plane, from row to row (across: from K to K)
    long long last;                 // along: the last row that is read, others read it instead; across: the last chunk's first column
};

template <bool HALF>
__device__ __forceinline__ f32x16 multiply(u32x4 a, u32x4 b, f32x16 c)
{
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
    if constexpr (HALF)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// One operand's tile: R rows of it, BK values of K.
template <int R, int BK, int NP, bool ACROSS>
struct Tile {
    static constexpr int kBytes = R * BK * 2;                           // of a plane
    static constexpr int kLoads = kBytes * NP / 1024;                   // wavefront loads of 64 x 16 bytes
    static constexpr int kPlaneLoads = kBytes / 1024;
    static constexpr int kChunks = (ACROSS ? R : BK) / 8;               // 16-byte chunks of a line in LDS

    // The place in memory of what lane `lane` of wavefront load `i` brings to LDS byte 1024 i + 16 lane, relative to K = 0
    static __device__ __forceinline__ const uint16_t* source(const Operand& o, long long first, int i, int lane)
    {
        const int plane = i / kPlaneLoads, chunk = (i % kPlaneLoads) * 64 + lane;
        const int line = chunk / kChunks, at = chunk % kChunks;
        if constexpr (ACROSS) {
            constexpr int G = kChunks / 4;                              // 64-byte pieces of a line
            const int turned = (((at >> 2) ^ (G >= 4 ? line & 3 : (line >> 1) & 1)) << 2) | (at & 3);
            const long long column = first + turned * 8;
            return o.at + plane * o.plane + line * o.ld + (column < o.last ? column : o.last);
        } else {
            constexpr int kLines = 16 / kChunks;                        // of 256 bytes
            const int turned = at ^ ((line / kLines) & (kChunks - 1));
            const long long row = first + line;
            return o.at + plane * o.plane + (row < o.last ? row : o.last) * o.ld + turned * 8;
        }
    }

    static __device__ __forceinline__ long long step(const Operand& o) { return ACROSS ? BK * o.ld : BK; }

    // 8 values of K of row 32 f + lane % 32 of the wavefront's rows, which begin at a multiple of 32: lanes 0 to 31 the first 8 of 16
    static __device__ __forceinline__ u32x4 fragment(const char* lds, int plane, int first, int f, int kk, int lane)
    {
        if constexpr (ACROSS) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4* lptr;
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
            constexpr int G = kChunks / 4;
            const int q = (lane >> 2) & 3, line = kk * 16 + (lane >> 5) * 8 + q;
            const int piece = (first / 32 + f) ^ (G >= 4 ? q : q >> 1);
            const char* p = lds + plane * kBytes + line * (R * 2) + piece * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
            // four lines further on a line's pieces are exchanged as on this one
            const char* p4 = p + 4 * R * 2;
            const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)p));
            const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)p4));
            return u32x4{a[0], a[1], b[0], b[1]};
        } else {
            constexpr int kLines = 16 / kChunks;
            const int row = first + f * 32 + (lane & 31);
            const int at = (kk * 2 + (lane >> 5)) ^ ((row / kLines) & (kChunks - 1));
            return *(const u32x4*)(lds + plane * kBytes + row * (BK * 2) + at * 16);
        }
    }
};

// BM x BN sums; the wavefront's are 32 FM x 32 FN of them: accumulator register r of lane l holds row 8 (r / 4) + 4 (l / 32) + r % 4 and column l % 32
// of a 32 x 32 block.
template <int BM, int BN, int BK, int NP, bool HALF, bool A_ACROSS, bool B_ACROSS>
struct Product {
    typedef Tile<BM, BK, NP, A_ACROSS> A;
    typedef Tile<BN, BK, NP, B_ACROSS> B;
    static constexpr int kM = BM, kN = BN, kK = BK, kPlanes = NP;
    static constexpr int FM = BM / 64, FN = BN / 64;
    static constexpr int kStage = (A::kBytes + B::kBytes) * NP, kStages = 3, kLds = kStage * kStages;
    static constexpr int kLoadsA = A::kLoads / 4, kLoadsB = B::kLoads / 4, kLoads = kLoadsA + kLoadsB;     // of a wavefront
    static_assert(A::kLoads % 4 == 0 && B::kLoads % 4 == 0 && BM % 64 == 0 && BN % 64 == 0, "the wavefronts load equally much");

    // k: a multiple of BK, from K = begin on
    static __device__ __forceinline__ void run(const Operand& a, const Operand& b, long long row, long long column, long long begin, int steps,
                                               char* lds, f32x16 (&acc)[FM][FN])
    {
        typedef const __attribute__((address_space(1))) void* gptr;
        typedef __attribute__((address_space(3))) void* lptr;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = wave >> 1, wn = wave & 1;
        const uint16_t *from_a[kLoadsA], *from_b[kLoadsB];
#pragma unroll
        for (int i = 0; i < kLoadsA; ++i) from_a[i] = A::source(a, row, wave * kLoadsA + i, lane) + begin / BK * A::step(a);
#pragma unroll
        for (int i = 0; i < kLoadsB; ++i) from_b[i] = B::source(b, column, wave * kLoadsB + i, lane) + begin / BK * B::step(b);
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int n = 0; n < FN; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[m][n][r] = 0.f;
        // the last steps ask for the last tile again, so that the number of loads under way is always the same
        int asked = 0;
        auto request = [&](int stage) {
            char* to = lds + stage * kStage + wave * kLoadsA * 1024;
            const bool more = ++asked < steps;
            const long long next_a = more ? A::step(a) : 0, next_b = more ? B::step(b) : 0;
#pragma unroll
            for (int i = 0; i < kLoadsA; ++i) {
                __builtin_amdgcn_global_load_lds((gptr)from_a[i], (lptr)(to + i * 1024), 16, 0, 0);
                from_a[i] += next_a;
            }
            to = lds + stage * kStage + A::kBytes * NP + wave * kLoadsB * 1024;
#pragma unroll
            for (int i = 0; i < kLoadsB; ++i) {
                __builtin_amdgcn_global_load_lds((gptr)from_b[i], (lptr)(to + i * 1024), 16, 0, 0);
                from_b[i] += next_b;
            }
        };
        request(0);
        request(1);
        int stage = 0;
        for (int k = 0; k < steps; ++k) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
            __builtin_amdgcn_s_barrier();       // this stage is there, and what the one before it held has been read by all
            asm volatile("" ::: "memory");
            request(stage == 0 ? 2 : stage - 1);
            const char* at = lds + stage * kStage;
            stage = stage == 2 ? 0 : stage + 1;
#pragma unroll
            for (int kk = 0; kk < BK / 16; ++kk) {
                u32x4 fa[FM][NP], fb[FN][NP];
#pragma unroll
                for (int p = 0; p < NP; ++p) {
#pragma unroll
                    for (int m = 0; m < FM; ++m) fa[m][p] = A::fragment(at, p, wm * 32 * FM, m, kk, lane);
#pragma unroll
                    for (int n = 0; n < FN; ++n) fb[n][p] = B::fragment(at + A::kBytes * NP, p, wn * 32 * FN, n, kk, lane);
                }
                // three planes: the small products first
#pragma unroll
                for (int sum = NP - 1; sum >= 0; --sum)
#pragma unroll
                    for (int p = sum; p >= 0; --p)
#pragma unroll
                        for (int m = 0; m < FM; ++m)
#pragma unroll
                            for (int n = 0; n < FN; ++n) acc[m][n] = multiply<HALF>(fa[m][p], fb[n][sum - p], acc[m][n]);
            }
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();           // LDS is the caller's again
        asm volatile("" ::: "memory");
    }
};

}  // namespace vocabulary
}  // namespace scc
