// Large products of the gated feed-forward block in bfloat16: tiles of 256 x 256 of 8 waves (and, where these are too few,
// of 128 x 256 of 4, in steps of 32, three of them in LDS).
//
// The inner axis goes by in steps of 64, two of them in LDS (2 x 64 KB).  The data of a step goes from memory to LDS without
// passing registers (16 bytes a lane, whole lines of memory), asked for a step before it is used, so that one barrier a
// step is all the waiting there is: it says that everybody's data of this step has arrived (each wave has waited for its
// own) and that everybody is done with the step whose place is filled next.
// A 16-byte piece of a line goes to a place that is chosen by an exclusive or with bits of the line's number, so that the
// lanes that are served together read from different banks (no conflicts by the counters); memory is read through the
// same permutation, since the lanes of a load write to LDS side by side.
// 8192 x 8192 x 8192: 1260 to 1310 TFLOP/s in all orders of the operands, as the general library's products of this size
// (1290); in steps of 32, four of them in LDS, 1090 to 1190 (lines of 64 bytes are half lines of memory), and 128 x 256
// tiles, two blocks to a compute unit, 990 to 1210.
#pragma once
#include "da_gated_kernels.hip"

namespace daspmm {

// Shape of a block: ROWS x 256 results, STAGES steps of STEP inner positions in LDS, a wave to every 8192 results
template <int ROWS, int STEP, int STAGES> struct WideShape {
    static constexpr int THREADS = ROWS * 2, A_BYTES = ROWS * STEP * 2, B_BYTES = kWideColumns * STEP * 2;
    static constexpr int STAGE = A_BYTES + B_BYTES, LDS = STAGES * STAGE;
    static constexpr int A_PIECES = A_BYTES / 16 / THREADS, B_PIECES = B_BYTES / 16 / THREADS;   // of a thread and step
    static constexpr int LOADS = A_PIECES + B_PIECES;
};

// One operand: OUTER outer positions x STEP inner ones
template <int LAY, int OUTER, int STEP> struct WideTile {
    // piece q of a step (LDS order, 16 bytes): its outer and inner position
    static __device__ __forceinline__ void piece(int q, int* outer, int* inner) {
        if constexpr (LAY == kInner) {                       // OUTER lines of STEP / 8 pieces
            const int line = q / (STEP / 8);
            *outer = line;
            *inner = ((q & (STEP / 8 - 1)) ^ turn(line)) * 8;
        } else {                                             // STEP lines of OUTER / 8 pieces, which stay together in pairs
            const int line = q / (OUTER / 8), at = q % (OUTER / 8);
            *inner = line;
            *outer = (((at >> 1) ^ twist(line)) * 2 + (at & 1)) * 8;
        }
    }
    // A 16-byte read serves 16 lanes at a time: 0-3, 12-15 and 20-27, or 4-11, 16-19 and 28-31, and the same of the upper
    // half.  These turns (0, 2, 3, 1 for fours of lines of 64 bytes, 0 to 7 for pairs of lines of 128) let each of
    // them find its pieces in different banks.
    static __device__ __forceinline__ int turn(int line) {
        if constexpr (STEP == 64) return line >> 1 & 7;
        const int q = line >> 2;
        return ((q ^ q >> 1) & 1) << 1 | (q >> 1 & 1);
    }
    // the 16 lanes of a transposing read take a pair from each of 4 lines, the wave from lines 8 apart
    static __device__ __forceinline__ int twist(int line) { return ((line & 3) | ((line >> 3) & 3) << 2) & (OUTER / 16 - 1); }

    // the lane's part of the fragment of outer positions o .. o + 15, inner ones 32 k and on
    static __device__ __forceinline__ bf16x8 frag(const char* lds, int o, int k) {
        const int i = threadIdx.x & 15, h = (threadIdx.x & 63) >> 4;
        if constexpr (LAY == kInner) {
            const int line = o + i;
            return *reinterpret_cast<const bf16x8*>(lds + line * (STEP * 2) + ((4 * k + h) ^ turn(line)) * 16);
        } else {
            typedef __attribute__((address_space(3))) s16x4* Lds;
            union { s16x4 half[2]; bf16x8 all; } f;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int line = k * 32 + h * 8 + n * 4 + i / 4;
                f.half[n] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (Lds)(lds + line * (OUTER * 2) + ((o / 16) ^ twist(line)) * 32 + (i & 3) * 8));
            }
            return f.all;
        }
    }
};

// Tile of a block: blocks go to the 8 dies of the chip in turn; a die takes neighbouring tiles, four rows of tiles at a time,
// so that what its blocks read at the same time is shared in its cache.
__device__ __forceinline__ void tile_of_block(int block, int tiles_m, int tiles_n, int* bm, int* bn) {
    const int tiles = tiles_m * tiles_n, die = block & 7, k = block >> 3;
    const int at = die * (tiles / 8) + min(die, tiles & 7) + k;
    constexpr int GROUP = 4;
    const int group = at / (GROUP * tiles_n), first = group * GROUP, size = min(GROUP, tiles_m - first);
    const int in = at - group * GROUP * tiles_n;
    *bm = first + in % size;
    *bn = in / size;
}

// 16 bytes a lane from base + offset to LDS: byte `to` of it and on, lane by lane.  Written out because the compiler, which
// knows the builtin of this instruction, waits for all of them before every transposing read; the waits are in the loop.
// Nothing else in these kernels uses m0.
__device__ __forceinline__ void memory_to_lds(const char* base, unsigned offset, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}

// the same for all lanes, for the compiler's knowledge
__device__ __forceinline__ const char* uniform(const char* p) {
    const uint64_t v = (uint64_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (const char*)((uint64_t)hi << 32 | lo);
}

template <int N> __device__ __forceinline__ void wait_for_loads() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// A is one tile; B is one of 256 columns, or one of 128 of each of the two weights whose products the epilogue joins
// (kGate, lines along the outer axis).
// A wave has 128 x 64 results, or 64 x 128 (kGate: 64 x 64 of both), so that 64 columns of a row leave together.
template <int ROWS, int STEP, int STAGES, int ALAY, int BLAY, int EPI>
__global__ __launch_bounds__(ROWS * 2) __attribute__((amdgpu_waves_per_eu(2, 2))) void gated_wide_kernel(GemmArgs<bf16> g)
{
    typedef WideShape<ROWS, STEP, STAGES> S;
    constexpr int MT = EPI == kGate ? 4 : 8, NT = 32 / MT, WN = 16 / NT, WIDTH = EPI == kGate ? kWideColumns / 2 : kWideColumns, THREADS = S::THREADS;
    typedef WideTile<ALAY, ROWS, STEP> TA;
    typedef WideTile<BLAY, WIDTH, STEP> TB;
    static_assert(EPI != kGate || BLAY == kOuter, "the second half of the pieces is the second weight's");
    constexpr int SUBS = EPI == kGate ? 2 : 1, SUB = S::B_PIECES / SUBS;      // weights, pieces of one
    extern __shared__ __attribute__((aligned(16))) char lds[];

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
    const int tiles_n = (g.N + WIDTH - 1) / WIDTH, tiles_m = (g.M + ROWS - 1) / ROWS;
    int bm, bn;
    tile_of_block(blockIdx.x, tiles_m, tiles_n, &bm, &bn);
    const int m0 = bm * ROWS, n0 = bn * WIDTH, batch = blockIdx.z;
    const int tps = (g.K + STEP - 1) / STEP;
    const int t0 = blockIdx.y * g.per, t1 = min(t0 + g.per, tps * g.segments);

    const unsigned lds_at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    // bytes from a step's first element to the thread's pieces; lines past the end are any: their results are not stored
    unsigned aoff[S::A_PIECES], boff[SUB];
#pragma unroll
    for (int i = 0; i < S::A_PIECES; ++i) {
        int outer, inner;
        TA::piece(tid + THREADS * i, &outer, &inner);
        outer = min(outer, g.M - (ALAY == kInner ? 1 : 8) - m0);
        aoff[i] = (unsigned)(ALAY == kInner ? (long)outer * g.lda + inner : (long)inner * g.lda + outer) * 2;
    }
#pragma unroll
    for (int i = 0; i < SUB; ++i) {
        int outer, inner;
        TB::piece(tid + THREADS * i, &outer, &inner);
        outer = min(outer, g.N - (BLAY == kInner ? 1 : 8) - n0);
        boff[i] = (unsigned)(BLAY == kInner ? (long)outer * g.ldb + inner : (long)inner * g.ldb + outer) * 2;
    }
    auto fetch = [&](int t, int stage) {
        const int seg = t >= tps ? 1 : 0, k0 = (t - seg * tps) * STEP;
        const char* A = uniform((const char*)((seg ? g.A[1] : g.A[0]) + (ALAY == kInner ? (long)m0 * g.lda + k0 : (long)k0 * g.lda + m0)));
        const long bat = BLAY == kInner ? (long)n0 * g.ldb + k0 : (long)k0 * g.ldb + n0;
        const char* B[SUBS];
#pragma unroll
        for (int w = 0; w < SUBS; ++w) B[w] = uniform((const char*)(((EPI == kGate ? w : seg + batch) ? g.B[1] : g.B[0]) + bat));
        if (k0 + STEP <= g.K) {
            const unsigned to = lds_at + stage * S::STAGE + wave * 1024;
#pragma unroll
            for (int i = 0; i < S::A_PIECES; ++i) memory_to_lds(A, aoff[i], to + i * THREADS * 16);
#pragma unroll
            for (int w = 0; w < SUBS; ++w)
#pragma unroll
                for (int i = 0; i < SUB; ++i) memory_to_lds(B[w], boff[i], to + S::A_BYTES + (w * SUB + i) * THREADS * 16);
        } else {                                             // the inner axis ends in this step: zeros behind it
            char* const to = lds + stage * S::STAGE + tid * 16;
            int outer, inner;
#pragma unroll
            for (int i = 0; i < S::A_PIECES; ++i) {
                TA::piece(tid + THREADS * i, &outer, &inner);
                const int left = g.K - k0 - inner;
                *(uint4*)(to + i * THREADS * 16) = edge_chunk((const bf16*)(A + aoff[i]), ALAY == kInner ? left : left > 0 ? 8 : 0);
            }
#pragma unroll
            for (int w = 0; w < SUBS; ++w)
#pragma unroll
                for (int i = 0; i < SUB; ++i) {
                    TB::piece(tid + THREADS * i, &outer, &inner);
                    const int left = g.K - k0 - inner;
                    *(uint4*)(to + S::A_BYTES + (w * SUB + i) * THREADS * 16) =
                        edge_chunk((const bf16*)(B[w] + boff[i]), BLAY == kInner ? left : left > 0 ? 8 : 0);
                }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the loop counts on LOADS loads a step, or none on their way
        }
    };
    // first column of the wave's j-th fragment in the result's tile, and its fragment
    auto column = [&](int j) { return EPI == kGate ? wn * (NT / 2) * 16 + j % (NT / 2) * 16 : wn * NT * 16 + j * 16; };
    auto bfrag = [&](const char* buf, int j, int k) {
        return TB::frag(buf + S::A_BYTES + (EPI == kGate && j >= NT / 2 ? S::B_BYTES / 2 : 0), column(j), k);
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    constexpr int AHEAD = STAGES - 1;
    static_assert(AHEAD >= 1 && AHEAD <= 3, "waits below");
#pragma unroll
    for (int s = 0; s < AHEAD; ++s)
        if (t0 + s < t1) fetch(t0 + s, s);
    int stage = 0, filled = AHEAD;
    for (int t = t0; t < t1; ++t) {
        const int left = t1 - 1 - t;
        // the steps after this one may still be on their way
        if (AHEAD == 3 && left >= 2) wait_for_loads<2 * S::LOADS>();
        else if (AHEAD >= 2 && left >= 1) wait_for_loads<S::LOADS>();
        else wait_for_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (left >= AHEAD) {
            fetch(t + AHEAD, filled);
            filled = filled + 1 == STAGES ? 0 : filled + 1;
        }
        const char* buf = lds + stage * S::STAGE;
        stage = stage + 1 == STAGES ? 0 : stage + 1;
#pragma unroll
        for (int k = 0; k < STEP / 32; ++k) {
            bf16x8 a[MT], b[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) b[j] = bfrag(buf, j, k);
#pragma unroll
            for (int i = 0; i < MT; ++i) a[i] = TA::frag(buf, wm * MT * 16 + i * 16, k);
            __builtin_amdgcn_sched_barrier(0);               // all reads are on their way before the first product
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = Mma<bf16>::mul(b[j], a[i], acc[i][j]);
        }
    }
    if (g.splits > 1) {
        part_epilogue<bf16, MT, NT, EPI>(g, acc, m0 + wm * MT * 16, n0, batch, column);
        return;
    }
    __syncthreads();                                         // LDS is free
    constexpr int MINE = S::LDS / (THREADS / 64);
    static_assert(MINE >= 16 * (NT * 16 + 4) * 4, "16 rows of a wave");
    line_epilogue<bf16, MT, NT, EPI>(g, acc, lds + wave * MINE, m0 + wm * MT * 16, n0 + wn * (EPI == kGate ? NT * 8 : NT * 16), batch);
}

}  // namespace daspmm
