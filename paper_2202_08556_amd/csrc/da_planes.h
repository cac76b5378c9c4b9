// Matrices as the matrix cores take them: packed in 16-bit numbers, padded with zeros to multiples of 64 both ways, and
// products of them whose epilogues are those of the operators that use them.
//
// A number is one bf16 (One), one fp16 (Half), or the sum of two fp16 (Halves): the nearest fp16 and what that leaves.  A pair has 22 bits;
// they come times a power of two, for an array or for each of its rows, that takes the largest below 2^15, and the second half of numbers 2^18
// times less begins to lose bits, 2^-25 of the scale.  The product of two pairs is three instructions of 16-bit numbers
// (the fourth, of both second halves, is below the 22 bits) in place of one of 32-bit numbers at a sixteenth of the rate.
//
// Rates: bf16, 4096 x 65536 . 65536 x 2048 1240 TFLOP/s, fp16 1270, pairs, 2048 x 2048 . 2048 x 8192 400 (1190 of single products); the general
// library's 8192^3 in bf16 1276, in float32 154.  Tiles of 256 x 256 have one block to a unit, whose LDS holds two steps of 64 KB; those
// of 128 and 64 have two, and read the next step's fragments while they multiply this one's.
//
// Pairs lie in groups of 32: 32 first halves and 32 second ones along a line, so that 64 bytes of either are 128 in one
// place.
#pragma once
#include "da_layer_common.h"
#include "da_planes_plan.h"

namespace daspmm {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

enum { kAlong = 0, kAcross = 1 };            // a line of memory goes along the inner axis, or across it

constexpr int kPad = 64;
__host__ __device__ inline long padded(long n) { return (n + kPad - 1) / kPad * kPad; }

// Where a packed matrix' numbers are: from a line to the next, and from 64 numbers of a line to the next 64.  Panels of 64 numbers of
// all lines have what a step reads along the lines in one place (4096 x 65536 . 65536 x 2048 bf16, lines of the first operand
// 128 KB apart and in panels: 1149 and 885 us).  The distance of a tile's numbers has to be within 32 bits: more than 2^21 lines lie
// one after the other.
struct Packed {
    long line, group;
};
__host__ __device__ inline Packed packed_lines(long numbers) { return {numbers, 64}; }
__host__ __device__ inline Packed packed(long lines, long n, int N) {
    return lines <= 1 << 21 ? Packed{64, lines * 64} : packed_lines(padded(n) * N);
}

struct One {
    static constexpr int N = 1, STEP = 64;                   // numbers of a value, inner positions of a step
    typedef bf16x8 Frag;
    typedef bf16 Number;
    static __device__ __forceinline__ f32x4 mul(const Frag& a, const Frag& b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
struct Half {
    static constexpr int N = 1, STEP = 64;
    typedef f16x8 Frag;
    typedef _Float16 Number;
    static __device__ __forceinline__ f32x4 mul(const Frag& a, const Frag& b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};
struct Halves {
    static constexpr int N = 2, STEP = 32;
    typedef f16x8 Frag;
    typedef _Float16 Number;
    static __device__ __forceinline__ f32x4 mul(const Frag& a, const Frag& b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};

// Value `at` of a packed line
template <class P> __host__ __device__ __forceinline__ long place(const Packed& l, long line, long at) {
    return line * l.line + at / (64 / P::N) * l.group + at % (64 / P::N);
}
template <class P, class T> __device__ __forceinline__ T* in_line(T* line, long at) { return line + at / (64 / P::N) * 64 + at % (64 / P::N); }

// V neighbouring values whose place is a multiple of V
template <class P, int V> __device__ __forceinline__ void put_values(uint16_t* to, const float (&x)[V]) {
    typedef uint16_t Bits __attribute__((ext_vector_type(V)));
    if constexpr (P::N == 1) {
        Bits b;
#pragma unroll
        for (int i = 0; i < V; ++i) b[i] = __builtin_bit_cast(uint16_t, (typename P::Number)x[i]);
        *reinterpret_cast<Bits*>(to) = b;
    } else {
        Bits first, second;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const _Float16 h = (_Float16)x[i];
            const float rest = x[i] - (float)h;              // exact; of an infinity: none
            first[i] = __builtin_bit_cast(uint16_t, h);
            second[i] = __builtin_bit_cast(uint16_t, (_Float16)(rest == rest ? rest : 0.f));
        }
        *reinterpret_cast<Bits*>(to) = first;
        *reinterpret_cast<Bits*>(to + 32) = second;
    }
}
template <class P, int V> __device__ __forceinline__ void get_values(const uint16_t* from, float (&x)[V]) {
    static_assert(P::N == 2, "pairs");
    typedef uint16_t Bits __attribute__((ext_vector_type(V)));
    const Bits first = *reinterpret_cast<const Bits*>(from), second = *reinterpret_cast<const Bits*>(from + 32);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)first[i]) + (float)__builtin_bit_cast(_Float16, (uint16_t)second[i]);
}

// One operand's part of a step in LDS: OUTER x STEP values, lines of 128 bytes (along) or of OUTER values (across).
// A 16-byte piece of a line goes to a place chosen by an exclusive or with bits of the line's number, so that the lanes that
// are served together read from different banks; memory is read through the same permutation, since the lanes of a load
// write to LDS side by side.
template <class P, int LAY, int OUTER> struct PlaneTile {
    static constexpr int LINE = LAY == kAlong ? 64 : OUTER * P::N;           // numbers
    static constexpr int BYTES = OUTER * 128;
    // piece q in LDS order: which line, and which numbers of it
    static __device__ __forceinline__ void piece(int q, int* line, int* at) {
        if constexpr (LAY == kAlong) {
            *line = q / 8;
            *at = ((q & 7) ^ turn(*line)) * 8;
        } else {
            const int p = q % (LINE / 8);
            *line = q / (LINE / 8);
            *at = (((p >> 1) ^ twist(*line)) * 2 + (p & 1)) * 8;
        }
    }
    static __device__ __forceinline__ int turn(int line) { return line >> 1 & 7; }
    static __device__ __forceinline__ int twist(int line) { return ((line & 3) | ((line >> 3) & 3) << 2) & (LINE / 16 - 1); }

    // the lane's part of the fragment of outer positions o .. o + 15; s: inner positions 32 s and on, or which half
    static __device__ __forceinline__ typename P::Frag frag(const char* lds, int o, int s) {
        const int i = threadIdx.x & 15, h = (threadIdx.x & 63) >> 4;
        if constexpr (LAY == kAlong) {
            const int line = o + i;
            return *reinterpret_cast<const typename P::Frag*>(lds + line * 128 + ((4 * s + h) ^ turn(line)) * 16);
        } else {
            typedef __attribute__((address_space(3))) s16x4* Lds;
            union { s16x4 half[2]; typename P::Frag all; } f;
            const int pair = P::N == 1 ? o / 16 : o / 32 * 4 + s * 2 + (o / 16 & 1);
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int line = (P::N == 1 ? s * 32 : 0) + h * 8 + n * 4 + i / 4;
                f.half[n] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(lds + line * (LINE * 2) + (pair ^ twist(line)) * 32 + (i & 3) * 8));
            }
            return f.all;
        }
    }
};

// Operands of a product: lines of A and B go along or across the inner axis; Ma and Nb are the padded outer extents, K the padded
// inner one.
struct PlaneArgs {
    const uint16_t *A, *B;
    Packed a, b;
    long batch_a, batch_b;       // numbers from one batch to the next
    int Ma, Nb, K;
    int tiles_m, tiles_n;
    const int* rows;             // where not null: so many of the outer positions of A (kBoundM), or of the inner ones (kBoundK), are there
    const int* other;            // kBoundK, where not null and not 0: the first operand is A_other
    const uint16_t* A_other;
    int splits, per;             // parts of the sum, steps of one
    float* part;                 // splits > 1: [batch][tile][split], a tile's sums as its waves hold them
    int* arrived;                // ... [batch][tile], 0: how many of a tile's parts are there
};
enum { kBoundNone = 0, kBoundM = 1, kBoundK = 2 };

// 16 bytes a lane from base + offset to LDS: byte `to` of it and on, lane by lane.  Written out because the compiler, which
// knows the builtin of this instruction, waits for all of them before every transposing read; the waits are in the loop.
// m0 is a reserved register: the compiler keeps nothing in it from one instruction to another, sets it before each use of its own, and
// takes no clobber of it.
__device__ __forceinline__ void line_to_lds(const char* base, unsigned offset, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}
// the same for all lanes, for the compiler's knowledge
__device__ __forceinline__ const char* same_for_all(const char* p) {
    const uint64_t v = (uint64_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (const char*)((uint64_t)hi << 32 | lo);
}
template <int N> __device__ __forceinline__ void wait_for_lines() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// All but the loads of the last `left` steps, MOST at most
template <int LOADS, int MOST> __device__ __forceinline__ void wait_for_steps(int left) {
    if constexpr (MOST == 0) wait_for_lines<0>();
    else if (left >= MOST) wait_for_lines<MOST * LOADS>();
    else wait_for_steps<LOADS, MOST - 1>(left);
}

// Tile of a block: blocks go to the 8 dies of the chip in turn; a die takes neighbouring tiles, four rows of tiles at a time,
// so that what its blocks read at the same time is shared in its cache.
__device__ __forceinline__ void plane_tile(int block, int tiles_m, int tiles_n, int* bm, int* bn) {
    const int tiles = tiles_m * tiles_n, die = block & 7, k = block >> 3;
    const int at = die * (tiles / 8) + min(die, tiles & 7) + k;
    constexpr int GROUP = 4;
    const int group = at / (GROUP * tiles_n), first = group * GROUP, size = min(GROUP, tiles_m - first);
    const int in = at - group * GROUP * tiles_n;
    *bm = first + in % size;
    *bn = in / size;
}
// ... of a symmetric result: tiles with bm <= bn
__device__ __forceinline__ void half_tile(int block, int tiles, int* bm, int* bn) {
    int m = 0;
    while (block >= tiles - m) {
        block -= tiles - m;
        ++m;
    }
    *bm = m;
    *bn = m + block;
}

struct NoColumn {};                          // of an epilogue that asks for nothing

// BM x BN results to a block of WM x WN waves, STAGES steps in LDS, asked for STAGES - 1 steps ahead.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_, bool PIPED_> struct PlaneShape {
    static constexpr bool PIPED = PIPED_;        // two steps' fragments in registers
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
    static constexpr int THREADS = 64 * WM * WN, MT = BM / 16 / WM, NT = BN / 16 / WN;
    static constexpr int STAGE = (BM + BN) * 128, LDS = STAGES * STAGE;
    static constexpr int A_PIECES = BM * 8 / THREADS, B_PIECES = BN * 8 / THREADS, LOADS = A_PIECES + B_PIECES;
    static_assert(BM * 8 % THREADS == 0 && BN * 8 % THREADS == 0, "every thread asks for as many pieces");
    static constexpr int PITCH = (NT * 16 + 4) * 4, MINE = 16 * PITCH;       // 16 rows of a wave on their way out
    static_assert(MINE * WM * WN <= LDS, "all waves' rows");
    static constexpr int OCCUPANCY = LDS > 80 * 1024 ? THREADS / 256 : 2 * THREADS / 256;
};

// E: the epilogue.  epi.tile(...) gets a wave's fragments and its part of LDS if E::kWhole, otherwise epi.four(m, n, x, batch, column) four
// neighbouring results at a time, after their sums are whole; column is epi.column(n), asked for once for all of a lane's rows.  E::kSymmetric: only tiles on and above the diagonal are computed;
// the results of those above it are handed over a second time, turned around.
template <class P, class S, int ALAY, int BLAY, int BOUND, class E>
__global__ __launch_bounds__(S::THREADS) __attribute__((amdgpu_waves_per_eu(S::OCCUPANCY, S::OCCUPANCY))) void plane_kernel(PlaneArgs g, E epi)
{
    typedef PlaneTile<P, ALAY, S::BM> TA;
    typedef PlaneTile<P, BLAY, S::BN> TB;
    constexpr int MT = S::MT, NT = S::NT, THREADS = S::THREADS, STEP = P::STEP;
    extern __shared__ __attribute__((aligned(16))) char lds[];

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / S::WN, wn = wave % S::WN;
    int bm, bn;
    if constexpr (E::kSymmetric) half_tile(blockIdx.x, g.tiles_m, &bm, &bn);
    else plane_tile(blockIdx.x, g.tiles_m, g.tiles_n, &bm, &bn);
    const int m0 = bm * S::BM, n0 = bn * S::BN, batch = blockIdx.z;
    int steps = g.K / STEP;
    if constexpr (BOUND == kBoundM) {
        if (m0 >= *g.rows) return;
    } else if constexpr (BOUND == kBoundK) {
        steps = min(steps, (*g.rows + STEP - 1) / STEP);
    }
    const int t0 = blockIdx.y * g.per, t1 = min(t0 + g.per, steps);
    const uint16_t* first = g.A;
    if constexpr (BOUND == kBoundK) {
        if (g.other && *g.other) first = g.A_other;
    }
    const char* const A = (const char*)(first + batch * g.batch_a);
    const char* const B = (const char*)(g.B + batch * g.batch_b);

    const unsigned lds_at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    // bytes from a step's first number to the thread's pieces; outer positions past the end are any: their results are not stored
    unsigned aoff[S::A_PIECES], boff[S::B_PIECES];
#pragma unroll
    for (int i = 0; i < S::A_PIECES; ++i) {
        int line, at;
        TA::piece(tid + THREADS * i, &line, &at);
        if constexpr (ALAY == kAlong) line = min(line, g.Ma - 1 - m0);
        else at = min(at, (g.Ma - m0) * P::N - 8);
        aoff[i] = (unsigned)((long)line * g.a.line + at / 64 * g.a.group + at % 64) * 2;
    }
#pragma unroll
    for (int i = 0; i < S::B_PIECES; ++i) {
        int line, at;
        TB::piece(tid + THREADS * i, &line, &at);
        if constexpr (BLAY == kAlong) line = min(line, g.Nb - 1 - n0);
        else at = min(at, (g.Nb - n0) * P::N - 8);
        boff[i] = (unsigned)((long)line * g.b.line + at / 64 * g.b.group + at % 64) * 2;
    }
    auto fetch = [&](int t, int stage) {
        static_assert(STEP * P::N == 64 && S::BM * P::N % 64 == 0 && S::BN * P::N % 64 == 0, "whole groups");
        const long k0 = (long)t * STEP;
        const char* a = same_for_all(A + (ALAY == kAlong ? (long)m0 * g.a.line + t * g.a.group : k0 * g.a.line + (long)(m0 * P::N / 64) * g.a.group) * 2);
        const char* b = same_for_all(B + (BLAY == kAlong ? (long)n0 * g.b.line + t * g.b.group : k0 * g.b.line + (long)(n0 * P::N / 64) * g.b.group) * 2);
        const unsigned to = lds_at + stage * S::STAGE + wave * 1024;
#pragma unroll
        for (int i = 0; i < S::A_PIECES; ++i) line_to_lds(a, aoff[i], to + i * THREADS * 16);
#pragma unroll
        for (int i = 0; i < S::B_PIECES; ++i) line_to_lds(b, boff[i], to + TA::BYTES + i * THREADS * 16);
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    typedef typename P::Frag Frag;
    // The fragments of a step: s is inner positions 32 s and on, or which half
    auto afrag = [&](const char* buf, int i, int s) { return TA::frag(buf, (wm * MT + i) * 16, s); };
    auto bfrag = [&](const char* buf, int j, int s) { return TB::frag(buf + TA::BYTES, (wn * NT + j) * 16, s); };
    // columns as the first operand: a lane's four results are neighbours in a row
    auto all = [&](Frag (&x)[MT], Frag (&y)[NT]) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = P::mul(y[j], x[i], acc[i][j]);
    };
    const int steps_here = max(0, t1 - t0);
    if constexpr (S::PIPED) {
        // Fragments of the next step are read while those of this one are multiplied, so a step's place in LDS is free a step earlier.
        struct Step {
            Frag a[2][MT], b[2][NT];
        };
        auto read = [&](const char* buf, Step& f) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
#pragma unroll
                for (int j = 0; j < NT; ++j) f.b[s][j] = bfrag(buf, j, s);
#pragma unroll
                for (int i = 0; i < MT; ++i) f.a[s][i] = afrag(buf, i, s);
            }
        };
        auto multiply = [&](Step& f) {
            all(f.a[0], f.b[0]);
            if constexpr (P::N == 1) {
                all(f.a[1], f.b[1]);
            } else {
                all(f.a[0], f.b[1]);
                all(f.a[1], f.b[0]);
            }
        };
        constexpr int STAGES = S::STAGES;
#pragma unroll
        for (int s = 0; s < STAGES; ++s)
            if (s < steps_here) fetch(t0 + s, s);
        Step one, two;
        int stage = 0;                                       // of step t
        auto next = [&](int at) { return at + 1 == STAGES ? 0 : at + 1; };
        if (steps_here > 0) {
            wait_for_steps<S::LOADS, STAGES - 1>(steps_here - 1);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            read(lds, one);
        }
        auto turn = [&](int t, Step& now, Step& then) {
            if (t + 1 < steps_here) {
                // the steps after the next may still be on their way; this step's fragments are in registers, everybody's behind the barrier
                wait_for_steps<S::LOADS, STAGES - 2>(steps_here - 2 - t);
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                if (t + STAGES < steps_here) fetch(t0 + t + STAGES, stage);
                stage = next(stage);
                read(lds + stage * S::STAGE, then);
            }
            multiply(now);
        };
        for (int t = 0; t < steps_here; t += 2) {
            turn(t, one, two);
            if (t + 1 < steps_here) turn(t + 1, two, one);
        }
    } else {
        constexpr int AHEAD = S::STAGES - 1;
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
            if (s < steps_here) fetch(t0 + s, s);
        int stage = 0, filled = AHEAD;
        for (int t = 0; t < steps_here; ++t) {
            const int left = steps_here - 1 - t;
            wait_for_steps<S::LOADS, AHEAD - 1>(left);       // the steps after this one may still be on their way
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (left >= AHEAD) {
                fetch(t0 + t + AHEAD, filled);
                filled = filled + 1 == S::STAGES ? 0 : filled + 1;
            }
            const char* buf = lds + stage * S::STAGE;
            stage = stage + 1 == S::STAGES ? 0 : stage + 1;
            Frag a[MT], b[NT], c[NT];
            if constexpr (P::N == 1) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
#pragma unroll
                    for (int j = 0; j < NT; ++j) b[j] = bfrag(buf, j, s);
#pragma unroll
                    for (int i = 0; i < MT; ++i) a[i] = afrag(buf, i, s);
                    __builtin_amdgcn_sched_barrier(0);       // all reads are on their way before the first product
                    all(a, b);
                }
            } else {
#pragma unroll
                for (int j = 0; j < NT; ++j) b[j] = bfrag(buf, j, 0);
#pragma unroll
                for (int i = 0; i < MT; ++i) a[i] = afrag(buf, i, 0);
#pragma unroll
                for (int j = 0; j < NT; ++j) c[j] = bfrag(buf, j, 1);
                __builtin_amdgcn_sched_barrier(0);
                all(a, b);
                all(a, c);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const Frag second = afrag(buf, i, 1);
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = P::mul(b[j], second, acc[i][j]);
                }
            }
        }
    }
    const int mw = m0 + wm * MT * 16, nw = n0 + wn * NT * 16, lane = tid & 63, i16 = lane & 15, h = lane >> 4;
    char* const mine = lds + wave * S::MINE;
    if constexpr (E::kWhole) {
        __syncthreads();                                     // LDS is free
        epi.template tile<MT, NT>(acc, mw, nw, bn * S::WN + wn, mine, g.Ma, g.Nb);
    } else {
        // The block that comes last adds a tile's parts, in their order: nobody waits for another.  Parts pass between blocks of
        // different dies, whose caches do not know of each other: they are written and read at the chip's scope (a fence of that
        // scope writes back all that a die's cache holds: 80 us in place of 5).
        if (g.splits > 1) {
            constexpr int PART = S::BM * S::BN / 2, MINE = MT * NT * 128;    // pairs of floats, of a tile and of a wave
            const long tile = (long)batch * gridDim.x + blockIdx.x;
            uint64_t* const part = reinterpret_cast<uint64_t*>(g.part) + tile * g.splits * PART + wave * MINE + lane;
            uint64_t* const to = part + (long)blockIdx.y * PART;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        __hip_atomic_store(to + ((i * NT + j) * 2 + q) * 64,
                                           (uint64_t)__float_as_uint(acc[i][j][2 * q]) | (uint64_t)__float_as_uint(acc[i][j][2 * q + 1]) << 32,
                                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                 // this wave's are there
            __syncthreads();
            int* const last = reinterpret_cast<int*>(lds);
            if (tid == 0) {
                *last = __hip_atomic_fetch_add(g.arrived + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == g.splits - 1;
                if (*last) __hip_atomic_store(g.arrived + tile, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // for the next product
            }
            __syncthreads();
            if (!*last) return;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int k = 0; k < g.splits; ++k)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const uint64_t v = __hip_atomic_load(part + (long)k * PART + ((i * NT + j) * 2 + q) * 64, __ATOMIC_RELAXED,
                                                                 __HIP_MEMORY_SCOPE_AGENT);
                            acc[i][j][2 * q] += __uint_as_float((uint32_t)v);
                            acc[i][j][2 * q + 1] += __uint_as_float((uint32_t)(v >> 32));
                        }
        }
        __syncthreads();                                     // LDS is free
        // Results leave by way of LDS, 16 rows of the wave at a time, so that a store is whole lines
        constexpr int LANES = NT * 4, ROWS = 64 / LANES;
        const int row0 = lane / LANES, col = lane % LANES * 4, n = nw + col;
        const auto column = epi.column(n);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int j = 0; j < NT; ++j) *reinterpret_cast<f32x4*>(mine + i16 * S::PITCH + (j * 16 + h * 4) * 4) = acc[i][j];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");           // LDS serves a wave in order
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int p = 0; p < 16 / ROWS; ++p) {
                const int row = p * ROWS + row0, m = mw + i * 16 + row;
                float x[4];
                load_floats<4>(reinterpret_cast<const float*>(mine + row * S::PITCH) + col, x);
                if (m < g.Ma && n < g.Nb) epi.four(m, n, x, batch, column);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        if constexpr (E::kSymmetric) {
            if (bm == bn) return;
            constexpr int COLS = MT * 16, TURNED = (COLS + 4) * 4, ACROSS = COLS / 4, DOWN = 64 / ACROSS;
            static_assert(16 * TURNED <= S::LDS / (THREADS / 64), "16 turned rows of a wave");
            char* const turned = lds + wave * (S::LDS / (THREADS / 64));
            __syncthreads();                                 // the waves' parts of LDS are others now
#pragma unroll
            for (int j = 0; j < NT; ++j) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) *reinterpret_cast<float*>(turned + (h * 4 + q) * TURNED + (i * 16 + i16) * 4) = acc[i][j][q];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int p = 0; p < 16 / DOWN; ++p) {
                    const int row = p * DOWN + lane / ACROSS, at = lane % ACROSS * 4, m = nw + j * 16 + row, n = mw + at;
                    float x[4];
                    load_floats<4>(reinterpret_cast<const float*>(turned + row * TURNED) + at, x);
                    if (m < g.Nb && n < g.Ma) epi.four(m, n, x, batch, epi.column(n));
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
        }
    }
}

}  // namespace daspmm
