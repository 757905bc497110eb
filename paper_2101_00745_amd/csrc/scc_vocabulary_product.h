// The matrix product of the vocabulary loss: a tile of BM x BN sums over K per workgroup, on the matrix cores.
//
// An operand is 16-bit, NP planes of it: one (bf16, or fp16 where HALF), or three, whose sum is a binary32 value (the exact cut of split3; six
// of the nine products are taken).  Its K values are consecutive in memory ("along"), or its rows are ("across": the operand is K x rows
// and is turned on its way out of LDS by ds_read_b64_tr_b16).  Tiles of BK of K go straight into LDS (global_load_lds, 16 bytes a
// lane), into a ring of buffers: while one is multiplied the others are under way, and one barrier a step is enough.  LDS is read without bank conflicts: in 256 bytes of LDS, which one
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

// A read through a restricted pointer: the compiler takes it for one that the loads under way into other buffers of LDS have nothing to do with (they
// have not: the caller has waited for this buffer's).  Without that it waits for all of them before each: 275 instead of 219 us for the
// gradients of 4096 tokens x 512 and a piece of 16128.
__device__ __forceinline__ uint64_t read_turned(const char* __restrict__ p)
{
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lptr;
    return __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)p));
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
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
            constexpr int G = kChunks / 4;
            const int q = (lane >> 2) & 3, line = kk * 16 + (lane >> 5) * 8 + q;
            const int piece = (first / 32 + f) ^ (G >= 4 ? q : q >> 1);
            const char* p = lds + plane * kBytes + line * (R * 2) + piece * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
            // four lines further on a line's pieces are exchanged as on this one
            const char* p4 = p + 4 * R * 2;
            const u32x2 a = __builtin_bit_cast(u32x2, read_turned(p));
            const u32x2 b = __builtin_bit_cast(u32x2, read_turned(p4));
            return u32x4{a[0], a[1], b[0], b[1]};
        } else {
            constexpr int kLines = 16 / kChunks;
            const int row = first + f * 32 + (lane & 31);
            const int at = (kk * 2 + (lane >> 5)) ^ ((row / kLines) & (kChunks - 1));
            return *(const u32x4*)(lds + plane * kBytes + row * (BK * 2) + at * 16);
        }
    }
};

// BM x BN sums by WM x WN wavefronts; a wavefront's are 32 FM x 32 FN of them: accumulator register r of lane l holds row 8 (r / 4) + 4 (l / 32) + r % 4
// and column l % 32 of a 32 x 32 block.  STAGES buffers in LDS.
template <int BM_, int BN_, int WM_, int WN_, int BK_, int STAGES_, int NP_>
struct Form {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = BK_, STAGES = STAGES_, NP = NP_;
};

template <typename F, bool HALF, bool A_ACROSS, bool B_ACROSS>
struct Product {
    static constexpr int kM = F::BM, kN = F::BN, kK = F::BK, kPlanes = F::NP, kWaves = F::WM * F::WN, kThreads = kWaves * 64, kStages = F::STAGES;
    typedef Tile<kM, kK, kPlanes, A_ACROSS> A;
    typedef Tile<kN, kK, kPlanes, B_ACROSS> B;
    static constexpr int FM = kM / F::WM / 32, FN = kN / F::WN / 32;
    static constexpr int kWavesPerSimd = FM * FN > 8 ? 1 : 2;           // accumulators of one fill half of its registers
    static constexpr int kStage = (A::kBytes + B::kBytes) * kPlanes, kLds = kStage * kStages;
    static constexpr int kLoadsA = A::kLoads / kWaves, kLoadsB = B::kLoads / kWaves, kLoads = kLoadsA + kLoadsB;     // of a wavefront
    static_assert(A::kLoads % kWaves == 0 && B::kLoads % kWaves == 0 && kM % (32 * F::WM) == 0 && kN % (32 * F::WN) == 0 && kLds <= 160 * 1024,
                  "the wavefronts load and multiply equally much");

    // What a workgroup multiplies: a tile of rows and columns over `steps` times kK values of K, from K = begin, a multiple of kK, on
    struct Part {
        long long row, column, begin;
        int steps;
    };

    // at(i, part): the workgroup's i'th part, false behind the last one (steps > 0 in all); done(part, acc): its sums.  The loads run on from one part into the next: while
    // done() works on a part's sums the next part's first buffers are under way, so it leaves the kLds bytes alone.
    template <typename At, typename Done>
    static __device__ __forceinline__ void walk(const Operand& a, const Operand& b, char* lds, At&& at, Done&& done)
    {
        typedef const __attribute__((address_space(1))) void* gptr;
        typedef __attribute__((address_space(3))) void* lptr;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = wave / F::WN, wn = wave % F::WN;
        const uint16_t *from_a[kLoadsA], *from_b[kLoadsB];
        Part ahead;
        int asked = 0, left = 0;                // parts that are asked for, steps of the last of them that are not
        if (!at(0, ahead)) return;
        auto begin_part = [&]() {
#pragma unroll
            for (int i = 0; i < kLoadsA; ++i) from_a[i] = A::source(a, ahead.row, wave * kLoadsA + i, lane) + ahead.begin / kK * A::step(a);
#pragma unroll
            for (int i = 0; i < kLoadsB; ++i) from_b[i] = B::source(b, ahead.column, wave * kLoadsB + i, lane) + ahead.begin / kK * B::step(b);
            left = ahead.steps;
            ++asked;
        };
        begin_part();
        // behind the last part its last tile is asked for again, so that the number of loads under way is always the same
        auto request = [&](int stage) {
            char* to = lds + stage * kStage + wave * kLoadsA * 1024;
#pragma unroll
            for (int i = 0; i < kLoadsA; ++i) __builtin_amdgcn_global_load_lds((gptr)from_a[i], (lptr)(to + i * 1024), 16, 0, 0);
            to = lds + stage * kStage + A::kBytes * kPlanes + wave * kLoadsB * 1024;
#pragma unroll
            for (int i = 0; i < kLoadsB; ++i) __builtin_amdgcn_global_load_lds((gptr)from_b[i], (lptr)(to + i * 1024), 16, 0, 0);
            if (--left > 0) {
                const long long next_a = A::step(a), next_b = B::step(b);
#pragma unroll
                for (int i = 0; i < kLoadsA; ++i) from_a[i] += next_a;
#pragma unroll
                for (int i = 0; i < kLoadsB; ++i) from_b[i] += next_b;
            } else if (left == 0 && at(asked, ahead)) {
                begin_part();
            }
        };
        // The fragments of 16 values of K are read while the ones before them are multiplied, the first of a step during the last of the step before: that one's
        // products wait for nothing while the next buffer is waited for and the wavefronts meet.
        constexpr int kParts = kK / 16;
        u32x4 fa[2][FM][kPlanes], fb[2][FN][kPlanes];
        auto read = [&](int to, const char* from, int kk) {
#pragma unroll
            for (int p = 0; p < kPlanes; ++p) {
#pragma unroll
                for (int m = 0; m < FM; ++m) fa[to][m][p] = A::fragment(from, p, wm * 32 * FM, m, kk, lane);
#pragma unroll
                for (int n = 0; n < FN; ++n) fb[to][n][p] = B::fragment(from + A::kBytes * kPlanes, p, wn * 32 * FN, n, kk, lane);
            }
        };
        f32x16 acc[FM][FN];
        auto products = [&](int of) {
            // three planes: the small products first
#pragma unroll
            for (int sum = kPlanes - 1; sum >= 0; --sum)
#pragma unroll
                for (int p = sum; p >= 0; --p)
#pragma unroll
                    for (int m = 0; m < FM; ++m)
#pragma unroll
                        for (int n = 0; n < FN; ++n) acc[m][n] = multiply<HALF>(fa[of][m][p], fb[of][n][sum - p], acc[m][n]);
        };
        // a read after every other product or so, so that neither pipe waits for the other's burst: 155 instead of 161 us for the logits of 4096 tokens x 512 x 32000
        auto interleave = []() {
            constexpr int kReads = kPlanes * (FM * (A_ACROSS ? 2 : 1) + FN * (B_ACROSS ? 2 : 1)), kProducts = FM * FN * (kPlanes == 3 ? 6 : 1);
#pragma unroll
            for (int i = 0; i < kProducts; ++i) {
                const int reads = kReads * (i + 1) / kProducts - kReads * i / kProducts;
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);          // a matrix instruction
                if (reads == 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);      // reads of LDS
                if (reads == 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                if (reads == 3) __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
            }
        };
#pragma unroll
        for (int i = 0; i < kStages; ++i) request(i);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLoads * (kStages - 1)) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read(0, lds, 0);
        int stage = 0;
        Part now, next;
        bool more = at(0, now);
        for (int i = 0; more; ++i) {
            more = at(i + 1, next);
#pragma unroll
            for (int m = 0; m < FM; ++m)
#pragma unroll
                for (int n = 0; n < FN; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[m][n][r] = 0.f;
            for (int k = 0; k < now.steps; ++k) {
                const char* from = lds + stage * kStage;
#pragma unroll
                for (int kk = 0; kk < kParts; ++kk) {
                    if (kk + 1 < kParts) {
                        read((kk + 1) & 1, from, kk + 1);
                    } else if (more || k + 1 < now.steps) {
                        // this wavefront's loads of the next buffer are there and it has read all of this one; then all wavefronts' are and have
                        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLoads * (kStages - 2)) : "memory");
                        __builtin_amdgcn_s_barrier();
                        asm volatile("" ::: "memory");
                        request(stage);
                        stage = stage == kStages - 1 ? 0 : stage + 1;
                        read(0, lds + stage * kStage, 0);
                    }
                    products(kk & 1);
                    interleave();
                }
            }
            done(now, acc);
            now = next;
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();           // nothing is under way to LDS any more
        asm volatile("" ::: "memory");
    }

    // One part; steps may be 0.  LDS is the caller's again afterwards.
    static __device__ __forceinline__ void run(const Operand& a, const Operand& b, const Part& part, char* lds, f32x16 (&sums)[FM][FN])
    {
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int n = 0; n < FN; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) sums[m][n][r] = 0.f;
        walk(
            a, b, lds,
            [&](int i, Part& p) {
                p = part;
                return i == 0 && part.steps > 0;
            },
            [&](const Part&, f32x16 (&acc)[FM][FN]) {
#pragma unroll
                for (int m = 0; m < FM; ++m)
#pragma unroll
                    for (int n = 0; n < FN; ++n) sums[m][n] = acc[m][n];
            });
    }
};

// Barrier for what wavefronts hand each other in LDS; loads and stores of memory go on
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A tile's sums as 16-bit values to memory, rows of it (consecutive sums of a lane) along the lines there.  value(m, n, r): of an accumulator.  In LDS a line of kM values has its 16-byte chunks exchanged by an exclusive or with the line, so that neither the
// writes (32 lines at a time) nor the reads (a line at a time) meet in a bank.
template <typename P>
struct Lines {
    static constexpr int kChunks = P::kM / 8, kBytes = P::kM * P::kN * 2;
    static_assert(kBytes <= P::kLds, "the tile fits where the operands were");

    static __device__ __forceinline__ uint16_t* place(char* lds, int line, int at)
    {
        return (uint16_t*)(lds + line * (P::kM * 2) + (((at >> 3) ^ line) & (kChunks - 1)) * 16 + (at & 7) * 2);
    }

    template <typename V, typename S>
    static __device__ __forceinline__ void store(char* lds, int wm, int wn, V&& value, S&& out)
    {
        typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int n = 0; n < P::FN; ++n) {
            const int line = (wn * P::FN + n) * 32 + (lane & 31);
#pragma unroll
            for (int m = 0; m < P::FM; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const u16x4 v = {value(m, n, 4 * q), value(m, n, 4 * q + 1), value(m, n, 4 * q + 2), value(m, n, 4 * q + 3)};
                    *(u16x4*)place(lds, line, (wm * P::FM + m) * 32 + 8 * q + 4 * (lane >> 5)) = v;
                }
        }
        __syncthreads();
#pragma unroll 4
        for (int i = threadIdx.x; i < P::kN * kChunks; i += P::kThreads) {
            const int line = i / kChunks, chunk = i % kChunks;
            out(line, chunk * 8, *(const u32x4*)place(lds, line, chunk * 8));
        }
    }

    // The same in pieces of 32 lines through a room of kPiece bytes (and another one, where `two`, which saves half of the barriers), for a tile whose operands'
    // buffers are in use.
    static constexpr int kPiece = P::kM * 32 * 2;
    template <bool TWO, typename V, typename S>
    static __device__ __forceinline__ void stream(char* room, int wm, int wn, V&& value, S&& out)
    {
        typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
        constexpr int kColumns = P::kN / 32 / P::FN;
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < kColumns * P::FN; ++i) {
            const int n = i % P::FN;                // of the wavefronts in column i / FN
            char* const lds = room + (TWO ? i & 1 : 0) * kPiece;
            if (wn == i / P::FN) {
                const int line = lane & 31;
#pragma unroll
                for (int m = 0; m < P::FM; ++m)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const u16x4 v = {value(m, n, 4 * q), value(m, n, 4 * q + 1), value(m, n, 4 * q + 2), value(m, n, 4 * q + 3)};
                        *(u16x4*)place(lds, line, (wm * P::FM + m) * 32 + 8 * q + 4 * (lane >> 5)) = v;
                    }
            }
            lds_barrier();
#pragma unroll
            for (int j = 0; j < (32 * kChunks + P::kThreads - 1) / P::kThreads; ++j) {
                const int at = threadIdx.x + j * P::kThreads, line = at / kChunks, chunk = at % kChunks;
                if (32 * kChunks % P::kThreads == 0 || line < 32) out(i * 32 + line, chunk * 8, *(const u32x4*)place(lds, line, chunk * 8));
            }
            if (!TWO) lds_barrier();
        }
        if (TWO) lds_barrier();
    }
};

}  // namespace vocabulary
}  // namespace scc
