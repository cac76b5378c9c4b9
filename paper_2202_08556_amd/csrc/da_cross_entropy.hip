// Cross entropy of a linear layer on the matrix cores, by pieces of the classes, without keeping logits:
//   z = x w + b,  loss = log sum exp z - z_target;   dz = g (exp(z - log sum exp) - 1 at the target),
//   dx = dz w^T,  dw = x^T dz,  db = sum of dz over the rows
//
// Forward, a tile of z leaves as the maximum and the sum of exponentials of each of its rows in 64 (or fewer) columns; these are
// joined by rows.  Backward, z is computed again a piece of the classes at a time, and leaves as dz, which the other two
// products read: eight operations for each of rows x d x classes instead of six, and nothing of the logits' size is kept.
// Rows that have a target are gathered first (x is packed for the products anyway), and the products stop at their number,
// which only the device knows: rows without one cost nothing and may hold anything.
// db is summed where dz is made, before it is rounded as an operand.
// Where float32 rows differ in size or factor x is packed twice (100000 x 700 x 130: 955 us with one factor, 1080 with one for each row).
// 4096 x 2048 x 65536 bf16, forward and backward: 3940 us, 1120 TFLOP/s; the four products 860 to 1000 each, the more the larger
// their epilogues, w's largest numbers 46 and its packing 120.
#include "da_training.h"

#include "da_ce_few.h"
#include "da_ce_narrow.h"
#include "da_ce_some.h"
#include "da_ce_tall.h"
#include "da_planes_host.h"
#include "da_spmm.h"

#include <type_traits>

namespace daspmm {
namespace {

constexpr int64_t kCeMost = 1 << 22, kCeRowsMost = 1 << 26;
constexpr int kChunks = 1024;                // of the rows, most
constexpr int kJoinBlocks = 1024;
constexpr int64_t kPieceBytes = 512LL << 20;
constexpr float kLog2e = 1.44269504088896f;

// Numbers that the logits are products of, and those of dz and what it is multiplied with: bfloat16 there as fp16, which holds its 8 bits and 11
// of dz (with dz in bfloat16 dw was off by up to 1.5 times what rounding it costs).
template <class T> using PlaneOf = std::conditional_t<std::is_same_v<T, float>, Halves, One>;
template <class T> using GradOf = std::conditional_t<std::is_same_v<T, float>, Halves, Half>;

// What a backward pass reads
struct CeStats {
    int *count, *index, *target;             // rows that have a target: how many, which, and which class
    int* place;                              // of every row in that list; -1: not there
    float* lse;
    int* shift;                              // packed float32: that of a row of x in the list by itself
    uint32_t* maxes;                         // kMaxX and so on
};
constexpr size_t kStatsHead = 32;
size_t stats_bytes(int64_t rows, bool shifts) { return kStatsHead + (shifts ? 5 : 4) * round16((size_t)rows * 4); }
CeStats ce_stats(void* p, int64_t rows) {
    char* c = static_cast<char*>(p);
    const size_t n = round16((size_t)rows * 4);
    auto ints = [&](size_t at) { return reinterpret_cast<int*>(c + at); };
    return {ints(0), ints(kStatsHead), ints(kStatsHead + n), ints(kStatsHead + 2 * n), reinterpret_cast<float*>(c + kStatsHead + 3 * n),
            ints(kStatsHead + 4 * n), reinterpret_cast<uint32_t*>(c + 16)};
}

// Numbers leave for fp16 times a power of two that takes the largest to 2^14 .. 2^15; `shift` is its exponent.  A row of x has that of the
// whole x, or its own where it is more than 2^kNear times smaller, and a row of dz that of its factor: what a row's results are off by
// does not depend on other rows.  w has one (float32), or one for each line, which goes along dx (bfloat16).
// Of x and w: the largest magnitude as bits, and that of the rows' own shifts; and a count of blocks.
enum { kMaxX = 0, kMaxW = 1, kArrived = 2, kRowX = 3, kMaxes = 4 };
constexpr int kNear = 4, kNoShift = -1000, kShiftBias = 512;     // kNoShift: a row of zeros
__device__ __forceinline__ int shift_of(uint32_t bits) {
    const float most = __uint_as_float(bits);
    int e = 15;
    if (most > 0.f) (void)frexpf(most, &e);                  // most < 2^e
    return 15 - e;
}
__device__ __forceinline__ float magnitude(float x) {
    const float a = fabsf(x);
    return a <= 3.402823466e38f ? a : 0.f;                   // infinities and NaN have no part in a scale
}
__device__ __forceinline__ int shift_of_row(const CeStats& st, int m, uint32_t largest) {
    const int own = st.shift[m], all = shift_of(largest);
    return own > all + kNear ? own : all;
}
__device__ __forceinline__ int shift_of_row(const CeStats& st, int m) { return shift_of_row(st, m, st.maxes[kMaxX]); }
// While they are taken the three maxima have kSpread places each, in lines of their own: a thousand blocks that end together and all go to one
// place take 20 us for that
constexpr int kSpread = 16, kApart = 32;
__device__ __forceinline__ uint32_t* spread_at(uint32_t* spread, int which, int block) {
    return spread + ((which == kRowX ? 2 : which) * kSpread + block % kSpread) * kApart;
}
__device__ __forceinline__ uint32_t spread_most(uint32_t* spread, int which) {           // in all lanes
    uint32_t most = *spread_at(spread, which, threadIdx.x);
    for (int d = 1; d < kSpread; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d, 64));
    return most;
}
// whether a row of x has its own
__device__ __forceinline__ bool rows_differ(const CeStats& st) {
    return (int)st.maxes[kRowX] - kShiftBias > shift_of(st.maxes[kMaxX]) + kNear;
}
// lanes to a row of n numbers of so many bytes
__host__ __device__ inline int row_lanes(long n, int size) {
    int lanes = 1;
    while (lanes < 64 && lanes * 16 < n * size) lanes *= 2;
    return lanes;
}
// The largest finite magnitude of a row or line, in all lanes of its team; `lane` of `lanes`, at most a wave
template <class T> __device__ __forceinline__ float most_of(const T* __restrict__ p, long n, int lane, int lanes) {
    constexpr int V = 16 / sizeof(T), U = 4;
    float most = 0.f;
    long c = lane * V;
    for (; c + (U - 1) * lanes * V + V <= n; c += U * lanes * V) {
        float v[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) load_floats<V>(p + c + u * lanes * V, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) most = fmaxf(most, magnitude(v[u][i]));
    }
    for (; c < n; c += lanes * V) {
        if (c + V <= n) {
            float v[V];
            load_floats<V>(p + c, v);
#pragma unroll
            for (int i = 0; i < V; ++i) most = fmaxf(most, magnitude(v[i]));
        } else {
            for (long i = c; i < n; ++i) {
                float one[1];
                load_floats<1>(p + i, one);
                most = fmaxf(most, magnitude(one[0]));
            }
        }
    }
    for (int k = 1; k < lanes; k <<= 1) most = fmaxf(most, __shfl_xor(most, k, 64));
    return most;
}
// ... of several rows at once, whose loads are on their way together
constexpr int kAtOnce = 4;
template <class T>
__device__ __forceinline__ void most_of_rows(const T* const (&p)[kAtOnce], long n, int lane, int lanes, float (&most)[kAtOnce]) {
    constexpr int V = 16 / sizeof(T);
#pragma unroll
    for (int r = 0; r < kAtOnce; ++r) most[r] = 0.f;
    for (long c = lane * V; c < n; c += lanes * V) {
        if (c + V <= n) {
            float v[kAtOnce][V];
#pragma unroll
            for (int r = 0; r < kAtOnce; ++r) load_floats<V>(p[r] + c, v[r]);
#pragma unroll
            for (int r = 0; r < kAtOnce; ++r)
#pragma unroll
                for (int i = 0; i < V; ++i) most[r] = fmaxf(most[r], magnitude(v[r][i]));
        } else {
            for (long i = c; i < n; ++i)
#pragma unroll
                for (int r = 0; r < kAtOnce; ++r) {
                    float one[1];
                    load_floats<1>(p[r] + i, one);
                    most[r] = fmaxf(most[r], magnitude(one[0]));
                }
        }
    }
    for (int k = 1; k < lanes; k <<= 1)
#pragma unroll
        for (int r = 0; r < kAtOnce; ++r) most[r] = fmaxf(most[r], __shfl_xor(most[r], k, 64));
}
// The listed rows of x, a few at once to a team of lanes: f(row, its largest magnitude, whether the lane is the team's first)
template <class T, class F>
__device__ __forceinline__ void each_row_most(const T* __restrict__ x, long ldx, const int* __restrict__ index, int count, long d, int blocks, F&& f) {
    const int lanes = row_lanes(d, sizeof(T)), lane = threadIdx.x & (lanes - 1), teams = 256 / lanes;
    const long step = (long)blocks * teams;
    for (long m = (long)blockIdx.x * teams + threadIdx.x / lanes; m < count; m += kAtOnce * step) {
        const T* p[kAtOnce];
        float most[kAtOnce];
#pragma unroll
        for (int r = 0; r < kAtOnce; ++r) p[r] = x + (long)index[m + r * step < count ? m + r * step : m] * ldx;
        most_of_rows(p, d, lane, lanes, most);
#pragma unroll
        for (int r = 0; r < kAtOnce; ++r)
            if (m + r * step < count) f((int)(m + r * step), most[r], lane == 0);
    }
}

// The gradient of the loss: of the rows, or one factor for all of them
struct Upstream {
    const float* dloss;
    long stride;
    int reduction;
    const int *count, *index;
    __device__ __forceinline__ float all() const { return reduction == DA_LOSS_MEAN ? dloss[0] / (float)max(1, *count) : dloss[0]; }
    __device__ __forceinline__ float row(int m) const { return reduction == DA_LOSS_ROWS ? dloss[index[m] * stride] : all(); }
    // of a row of dz; which numbers it takes to 2^14 .. 2^15 follows from the factor alone, since dz is at most that
    __device__ __forceinline__ int shift(float factor) const { return shift_of(__float_as_uint(magnitude(factor))); }
};

// dw adds rows, so x and dz of a row have to come times the same power of two together, 2^sum: x is packed for it times what dz lacks, a second
// time in float32, and there only where rows of x or of dz have shifts of their own.  sum is the smallest of a row's two shifts
// together: the row that adds most has all its bits, the others theirs from 2^-38 of its numbers on.
struct Joint {
    int sum, differ;
};
struct FactorPart {
    int sum, least, most;        // of some rows: the smallest sum of shifts, the smallest and the largest shift of dz
};
__device__ __forceinline__ FactorPart joined(const FactorPart& a, const FactorPart& b) {
    return {min(a.sum, b.sum), min(a.least, b.least), max(a.most, b.most)};
}
__device__ __forceinline__ FactorPart no_rows() { return {1 << 20, 1 << 20, -(1 << 20)}; }
// all 256 threads' in every thread
__device__ __forceinline__ FactorPart block_joined(FactorPart p) {
    __shared__ FactorPart red[4];
    for (int d = 1; d < 64; d <<= 1) p = joined(p, {__shfl_xor(p.sum, d, 64), __shfl_xor(p.least, d, 64), __shfl_xor(p.most, d, 64)});
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = p;
    __syncthreads();
    return joined(joined(red[0], red[1]), joined(red[2], red[3]));
}
constexpr int kFactorParts = 1024, kLongLine = 2048;
template <class Q> __device__ __forceinline__ Joint joint_of(const CeStats& st, const Upstream& u, const FactorPart* part, int parts) {
    if (Q::N == 2 && u.reduction != DA_LOSS_ROWS) return {shift_of(st.maxes[kMaxX]) + u.shift(u.all()), rows_differ(st)};
    FactorPart p = no_rows();
    for (int k = threadIdx.x; k < parts; k += 256) p = joined(p, part[k]);
    p = block_joined(p);
    if (p.least > p.most) return {0, Q::N == 1};
    const bool differ = Q::N == 1 || rows_differ(st) || p.least != p.most;
    return {differ ? p.sum : shift_of(st.maxes[kMaxX]) + p.least, differ};
}

__device__ __forceinline__ long target_of(const void* t, int wide, long r) {
    return wide ? static_cast<const int64_t*>(t)[r] : (long)static_cast<const int32_t*>(t)[r];
}

// Rows of a chunk that have a target
__global__ __launch_bounds__(256) void ce_count_kernel(const void* __restrict__ target, int wide, long rows, long classes, long chunk,
                                                       int* __restrict__ counts)
{
    __shared__ int red[4];
    const long r0 = blockIdx.x * chunk, r1 = min(r0 + chunk, rows);
    int n = 0;
    for (long r = r0 + threadIdx.x; r < r1; r += 256) {
        const long t = target_of(target, wide, r);
        n += t >= 0 && t < classes;
    }
    n = wave_sum(n, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
    __syncthreads();
    if (threadIdx.x == 0) counts[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

// Lists them in order; the others' losses are 0.  counts: of the chunks, where there are several
__global__ __launch_bounds__(256) void ce_index_kernel(const void* __restrict__ target, int wide, long rows, long classes, long chunk,
                                                       const int* __restrict__ counts, CeStats st, uint32_t* __restrict__ spread,
                                                       float* __restrict__ loss)
{
    __shared__ int red[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int before = 0;
    if (counts) {
        for (int k = tid; k < (int)blockIdx.x; k += 256) before += counts[k];
        before = wave_sum(before, 64);
        if (lane == 0) red[wave] = before;
        __syncthreads();
        before = red[0] + red[1] + red[2] + red[3];
    }
    if (blockIdx.x == 0 && tid < kMaxes) st.maxes[tid] = 0;
    if (blockIdx.x == 0 && tid < 3 * kSpread) spread[tid * kApart] = 0;
    const long r0 = blockIdx.x * chunk, r1 = min(r0 + chunk, rows);
    for (long r = r0 + tid; r - tid < r1; r += 256) {
        const long t = r < r1 ? target_of(target, wide, r) : -1;
        const bool has = t >= 0 && t < classes;
        const uint64_t mask = __ballot(has);
        __syncthreads();                                     // the counts before have been read
        if (lane == 0) red[wave] = __popcll(mask);
        __syncthreads();
        int at = before;
        for (int k = 0; k < wave; ++k) at += red[k];
        if (has) {
            at += __popcll(mask & ((1ull << lane) - 1));
            st.index[at] = (int)r;
            st.target[at] = (int)t;
            st.place[r] = at;
        } else if (r < r1) {
            st.place[r] = -1;
            if (loss) loss[r] = 0.f;
        }
        before += red[0] + red[1] + red[2] + red[3];
    }
    if (r1 == rows && tid == 0) *st.count = before;
}

// The largest of a block's; the order of the blocks does not show
__device__ __forceinline__ void keep_largest(uint32_t most, uint32_t* to) {
    __shared__ uint32_t red[4];
    for (int d = 1; d < 64; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d, 64));
    __syncthreads();                                         // those of a call before have been read
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
        most = max(max(red[0], red[1]), max(red[2], red[3]));
        // most blocks find a larger one there
        if (most > __hip_atomic_load(to, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(to, most);
    }
}
// 4096 x 1024 x 8192: 16 us; 100000 x 700: 56.
// Largest finite magnitudes: blockIdx.y 0 of the rows of x that count, and their shifts, 1 of w
__global__ __launch_bounds__(256) void ce_max_kernel(const float* __restrict__ x, long ldx, CeStats st, long d, const float* __restrict__ w,
                                                     long numbers, uint32_t* __restrict__ spread)
{
    uint32_t most = 0;                                       // of floats that are not negative bits are in order
    if (blockIdx.y == 0) {
        if ((long)blockIdx.x * (256 / row_lanes(d, 4)) >= *st.count) return;
        uint32_t far = 0;
        each_row_most(x, ldx, st.index, *st.count, d, gridDim.x, [&](int m, float here, bool first) {
            const int shift = shift_of(__float_as_uint(here));
            if (first) st.shift[m] = here > 0.f ? shift : kNoShift;
            if (here > 0.f) far = max(far, (uint32_t)(shift + kShiftBias));
            most = max(most, __float_as_uint(here));
        });
        keep_largest(far, spread_at(spread, kRowX, blockIdx.x));
    } else {
        constexpr int U = 4;                                 // pieces of the whole grid on their way
        const long step = (long)gridDim.x * 1024;
        float here = 0.f;
        long c = ((long)blockIdx.x * 256 + threadIdx.x) * 4;
        for (; c + (U - 1) * step + 4 <= numbers; c += U * step) {
            float v[U][4];
#pragma unroll
            for (int u = 0; u < U; ++u) load_floats<4>(w + c + u * step, v[u]);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) here = fmaxf(here, magnitude(v[u][i]));
        }
        for (; c < numbers; c += step)
            for (long i = c; i < min(c + 4, numbers); ++i) here = fmaxf(here, magnitude(w[i]));
        most = __float_as_uint(here);
    }
    keep_largest(most, spread_at(spread, blockIdx.y == 0 ? kMaxX : kMaxW, blockIdx.x));
}

template <class T> __device__ __forceinline__ void store_row(T* p, int left, const float (&x)[4]) {
    if (left >= 4) {
        store_floats<4>(p, x);
    } else {
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            const float one[1] = {x[q]};
            if (q < left) store_floats<1>(p + q, one);
        }
    }
}

// Packs lines of numbers, 8 numbers at a time; lines and their ends are padded with zeros.
template <class T> struct PackJob {
    const T* from;
    long ld, whole, lines;       // lines that there are, and of them to pack
    int n;
    const int *index, *count;    // not null: *count lines of a list, and zeros up to the next multiple of 64
    uint16_t* to;
    Packed layout;
};
// What a backward pass begins with beside that: no parts yet, and 0 in the rows of dx without a target
template <class T> struct BeginJob {
    long rows;
    int d;
    T* dx;
    int* arrived;                // null: forward
    __device__ __forceinline__ void run(const CeStats& st) const {
        if (blockIdx.x == 0)
            for (int k = threadIdx.x; k < kMostParted; k += 256) arrived[k] = 0;
        if (!dx) return;
        const int lane = threadIdx.x & 63;
        for (long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6); r < rows; r += (long)gridDim.x * 4) {
            if (st.place[r] >= 0) continue;
            for (int k = lane * 4; k < d; k += 256) {
                const float zero[4] = {0.f, 0.f, 0.f, 0.f};
                store_row(dx + r * d + k, d - k, zero);
            }
        }
    }
};
// ... and x for dw, and bfloat16's w for dx, both in the numbers of dz; `to` null: not wanted
struct JointJob {
    Upstream u;
    const FactorPart* part;
    int parts;
    const int* shift;            // of the rows of x by themselves
    Joint* joint;
    uint16_t* to;
};
struct LinesJob {
    const int* shift;            // of the lines of w
    uint16_t* to;
};
// blockIdx.y 0: x, 1: w, 2: begin, 3: x for dw, 4: w for dx
template <class T, class P, class Q>
__global__ __launch_bounds__(256) void ce_pack_kernel(CeStats st, uint32_t* __restrict__ spread, PackJob<T> x, PackJob<T> w, BeginJob<T> begin,
                                                      JointJob again, LinesJob lines)
{
    if (blockIdx.y == 2) return begin.run(st);
    uint32_t largest = 0;                                    // of x, or of w
    if constexpr (P::N == 2) {
        if (spread) {                                        // forward: for the kernels after this one, too
            largest = spread_most(spread, blockIdx.y == 1 ? kMaxW : kMaxX);
            const uint32_t row = spread_most(spread, kRowX);
            if (blockIdx.x == 0 && threadIdx.x == 0) {
                st.maxes[blockIdx.y == 1 ? kMaxW : kMaxX] = largest;
                if (blockIdx.y == 0) st.maxes[kRowX] = row;
            }
        } else {
            largest = st.maxes[blockIdx.y == 1 ? kMaxW : kMaxX];
        }
    }
    Joint joint{};
    PackJob<T> j = blockIdx.y == 1 || blockIdx.y == 4 ? w : x;
    if (blockIdx.y == 4) {
        j.lines = j.whole;
        j.to = lines.to;
    }
    if (blockIdx.y == 3) {
        if (!again.to) return;
        joint = joint_of<Q>(st, again.u, again.part, again.parts);
        if (blockIdx.x == 0 && threadIdx.x == 0) *again.joint = joint;
        if (!joint.differ) return;
        j.to = again.to;
    }
    // 16 lines x 128 numbers at a time, four lines to a wave: whole lines of memory on both sides
    const int n = (int)padded(j.n), across = (n + 127) / 128;
    const long there = j.index ? *j.count : j.lines, tiles = (padded(there) / 16) * across;
    for (long k = blockIdx.x; k < tiles; k += gridDim.x) {
        const long line = k / across * 16 + threadIdx.x / 16;
        const int at = (int)(k % across) * 128 + threadIdx.x % 16 * 8;
        if (at >= n) continue;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.f;
        if (line < there) {
            const T* __restrict__ p = j.from + (j.index ? (long)j.index[line] : line) * j.ld + at;
            if (at + 8 <= j.n) {
                load_floats<8>(p, x);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (at + i < j.n) {
                        float one[1];
                        load_floats<1>(p + i, one);
                        x[i] = one[0];
                    }
            }
            if (P::N == 2 && blockIdx.y < 3) {
                const int by = blockIdx.y == 1 ? shift_of(largest) : shift_of_row(st, (int)line, largest);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = ldexpf(x[i], by);
            }
            if (blockIdx.y == 3) {
                // a row that adds nothing to dw, its factor 0 or none, is not in the joint sum: no more than its own shift
                const int own = again.shift[line], by = own == kNoShift ? 0 : min(joint.sum - again.u.shift(again.u.row((int)line)), own);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = ldexpf(x[i], by);
            }
        }
        if (P::N == 1 && blockIdx.y == 4 && line < there) {
            const int by = lines.shift[line];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = ldexpf(x[i], by);
        }
        uint16_t* const to = j.to + place<P>(j.layout, line, at);
        if (blockIdx.y >= 3) put_values<Q, 8>(to, x);
        else put_values<P, 8>(to, x);
    }
}

// ------------------------------------------------------------------------------------------
// Epilogues
// ------------------------------------------------------------------------------------------
template <class P> struct Logits {
    const void* bias;
    int bias_type;
    int classes;
    CeStats st;
    // A wave's logits from its sums: columns nw + 16 j + 4 h and on of row i16 of each 16 (both scales leave as one exponent: neither
    // they nor their product need be floats); -inf behind the last class
    template <int NT> struct Columns {
        int shift;                                           // of w
        float bias[NT][4];
        bool inside;
    };
    template <int NT> __device__ __forceinline__ Columns<NT> columns(int nw) const {
        Columns<NT> c;
        c.shift = P::N == 2 ? shift_of(st.maxes[kMaxW]) : 0;
        c.inside = nw + NT * 16 <= classes;
        const int n = nw + 4 * ((threadIdx.x & 63) >> 4);
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) c.bias[j][q] = bias && n + j * 16 + q < classes ? load_param(bias, bias_type, n + j * 16 + q) : 0.f;
        return c;
    }
    // shift: of the row of x
    template <int NT>
    __device__ __forceinline__ void logits(const f32x4 (&acc)[NT], const Columns<NT>& c, int shift, int nw, float (&z)[NT][4]) const {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                z[j][q] = acc[j][q];
                if constexpr (P::N == 2) z[j][q] = ldexpf(z[j][q], -(shift + c.shift));
            }
        if (bias)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) z[j][q] += c.bias[j][q];
        if (!c.inside) {
            const int n = nw + 4 * ((threadIdx.x & 63) >> 4);
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (n + j * 16 + q >= classes) z[j][q] = -INFINITY;
        }
    }
};

// A row's maximum and sum of exponentials in the columns of a wave
template <class P> struct SumsOut : Logits<P> {
    static constexpr bool kSymmetric = false, kWhole = true;
    float2* part;                // [row][slot]
    int slots;
    float* at_target;            // [row]
    template <int MT, int NT>
    __device__ __forceinline__ void tile(f32x4 (&acc)[MT][NT], int mw, int nw, int slot, char*, int, int) const {
        const int i16 = threadIdx.x & 15, h = (threadIdx.x & 63) >> 4, count = *this->st.count;
        const auto c = this->template columns<NT>(nw);
        int t[MT], shift[MT];                                // of the row; the target from the lane's first column on
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = mw + i * 16 + i16;
            t[i] = (m < count ? this->st.target[m] : -0x40000000) - nw - 4 * h;
            shift[i] = P::N == 2 && m < count ? shift_of_row(this->st, m) : 0;
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = mw + i * 16 + i16;
            float z[NT][4], most = -INFINITY;
            this->logits(acc[i], c, shift[i], nw, z);
            if (__any(t[i] >= 0 && t[i] < NT * 16))
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (t[i] == j * 16 + q) at_target[m] = z[j][q];
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) most = fmaxf(most, z[j][q]);
            most = fmaxf(most, __shfl_xor(most, 16, 64));
            most = fmaxf(most, __shfl_xor(most, 32, 64));
            const float from = most == -INFINITY ? 0.f : most;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) sum += exp2_hw((z[j][q] - from) * kLog2e);
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            if (h == 0 && m < count) part[(long)m * slots + slot] = make_float2(most, sum);
        }
    }
};

// dz of a piece of the classes that begins at `first`; rows behind the last one are 0
template <class P, class Q, bool BIAS> struct GradOut : Logits<P> {
    static constexpr bool kSymmetric = false, kWhole = true;
    Upstream u;
    int first;
    uint16_t* dz;
    Packed lz;
    int* up;                     // what a row of dz comes times, for dx; by the first columns' waves
    float* sums;                 // BIAS: [rows of a wave, one after the other][Nb], what they add to db, in 32 bits
    // 16 rows at a time: a lane makes its numbers of one row, packed as they are in memory, and they leave by way of LDS in whole lines
    template <int MT, int NT>
    __device__ __forceinline__ void tile(f32x4 (&acc)[MT][NT], int mw, int nw, int, char* lds, int Ma, int Nb) const {
        constexpr int BYTES = NT * 32 * P::N, PITCH = BYTES + 16, CHUNKS = BYTES / 16;
        const int lane = threadIdx.x & 63, i16 = lane & 15, h = lane >> 4, count = *this->st.count, n0 = first + nw;
        const auto c = this->template columns<NT>(n0);
        float lse[MT], by[MT], g[MT];
        int t[MT], shift[MT];
        const bool each = u.reduction == DA_LOSS_ROWS;
        const float all = each ? 0.f : u.all();
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = mw + i * 16 + i16;
            const bool there = m < count;
            lse[i] = there ? this->st.lse[m] : 0.f;
            g[i] = there ? each ? u.row(m) : all : 0.f;
            const int s = u.shift(g[i]);
            by[i] = ldexpf(g[i], s);
            if (there && h == 0 && n0 == 0) up[m] = s;
            shift[i] = P::N == 2 && there ? shift_of_row(this->st, m) : 0;
            t[i] = (there ? this->st.target[m] : -0x40000000) - n0 - 4 * h;
        }
        f32x4 sum[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) sum[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            float z[NT][4];
            this->logits(acc[i], c, shift[i], n0, z);
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) z[j][q] = exp2_hw((z[j][q] - lse[i]) * kLog2e);
            if (__any(t[i] >= 0 && t[i] < NT * 16))
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (t[i] == j * 16 + q) z[j][q] -= 1.f;
            const bool there = mw + i * 16 + i16 < count;    // a row that is not may hold anything
            if constexpr (BIAS)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) sum[j][q] += there ? z[j][q] * g[i] : 0.f;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
#pragma unroll
                for (int q = 0; q < 4; ++q) z[j][q] = there && (c.inside || n0 + j * 16 + 4 * h + q < this->classes) ? z[j][q] * by[i] : 0.f;
                put_values<Q, 4>(in_line<Q>(reinterpret_cast<uint16_t*>(lds + i16 * PITCH), j * 16 + 4 * h), z[j]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");           // LDS serves a wave in order
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int p = 0; p < CHUNKS / 4; ++p) {
                const int k = p * 64 + lane, row = k / CHUNKS, at = k % CHUNKS, m = mw + i * 16 + row, n = nw * P::N + at * 8;
                const uint4 line = *reinterpret_cast<const uint4*>(lds + row * PITCH + at * 16);
                if (m < Ma && nw < Nb) *reinterpret_cast<uint4*>(dz + (long)m * lz.line + n / 64 * lz.group + n % 64) = line;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        if (!BIAS || mw >= Ma || nw >= Nb) return;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[j][q] = wave_sum(sum[j][q], 16);
            if (i16 == 0) *reinterpret_cast<f32x4*>(sums + (long)(mw / (MT * 16)) * Nb + nw + j * 16 + 4 * h) = sum[j];
        }
    }
};
// rows of a wave of its tiles
constexpr int grad_rows(int shape) { return shape == 0 ? PlaneLarge::MT * 16 : shape == 1 ? PlaneMiddle::MT * 16 : PlaneSmall::MT * 16; }

// dx, or what the pieces so far give of it
template <class T, class Q> struct InputOut {
    static constexpr bool kSymmetric = false, kWhole = false;
    CeStats st;
    const int* shift;            // of dz's rows
    const float* before;         // dense rows x ldb, packed rows
    float* after;                // where not null: the sum goes here instead of to dx
    long ldb;
    T* dx;
    int d;
    const int* lines;            // bfloat16: shifts of w's
    struct Column {
        int count, down[4];
    };
    __device__ __forceinline__ Column column(int n) const {
        if constexpr (Q::N == 2) {
            const int w = -shift_of(st.maxes[kMaxW]);
            return {*st.count, {w, w, w, w}};
        } else {
            const int4 w = n < d ? *reinterpret_cast<const int4*>(lines + n) : make_int4(0, 0, 0, 0);
            return {*st.count, {-w.x, -w.y, -w.z, -w.w}};
        }
    }
    __device__ __forceinline__ void four(int m, int n, float (&x)[4], int, const Column& c) const {
        if (m >= c.count || n >= d) return;
        const int up = shift[m];
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] = ldexpf(x[q], c.down[q] - up);
        if (before) {
            float u[4];
            load_floats<4>(before + (long)m * ldb + n, u);
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] += u[q];
        }
        if (after) store_floats<4>(after + (long)m * ldb + n, x);
        else store_row(dx + (long)st.index[m] * d + n, d - n, x);
    }
};

template <class T> struct WeightOut {
    static constexpr bool kSymmetric = false, kWhole = false;
    const Joint* joint;
    T* dw;                       // of the piece
    long ldw;
    int d, classes;              // of the piece
    __device__ __forceinline__ int column(int) const { return -joint->sum; }
    __device__ __forceinline__ void four(int m, int n, float (&x)[4], int, int down) const {
        if (m >= d || n >= classes) return;
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] = ldexpf(x[q], down);
        store_row(dw + (long)m * ldw + n, classes - n, x);
    }
};

// ------------------------------------------------------------------------------------------
// Rows
// ------------------------------------------------------------------------------------------
// log sum exp and loss of the rows, P lanes to one; with sums, the loss of all of them
__global__ __launch_bounds__(256) void ce_join_kernel(CeStats st, const float2* __restrict__ part, int slots, int P,
                                                      const float* __restrict__ at_target, float* __restrict__ loss, uint64_t* __restrict__ sums,
                                                      uint32_t* __restrict__ arrived, int mean, float* __restrict__ loss_all)
{
    __shared__ double red[4];
    const int lane = threadIdx.x & (P - 1), count = *st.count, teams = 256 / P;
    double total = 0.0;
    for (long m = (long)blockIdx.x * teams + threadIdx.x / P; m < count; m += (long)gridDim.x * teams) {
        const float2* __restrict__ p = part + m * slots;
        float most = -INFINITY, sum = 0.f;
        for (int k = lane; k < slots; k += P) most = fmaxf(most, p[k].x);
        for (int d = 1; d < P; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
        const float from = most == -INFINITY ? 0.f : most;
        for (int k = lane; k < slots; k += P) sum += p[k].y * exp2_hw((p[k].x - from) * kLog2e);
        sum = wave_sum(sum, P);
        const float lse = most + logf(sum), l = lse - at_target[m];
        if (lane == 0) {
            st.lse[m] = lse;
            if (loss) loss[st.index[m]] = l;
            total += l;
        }
    }
    if (!sums) return;
    // the block that comes last adds the blocks' sums, in their order
    auto block_sum = [&](double v) {
        v = wave_sum(v, 64);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        return (red[0] + red[1]) + (red[2] + red[3]);
    };
    total = block_sum(total);
    __shared__ int last;
    if (threadIdx.x == 0) {
        __hip_atomic_store(sums + blockIdx.x, __builtin_bit_cast(uint64_t, total), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        last = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    total = 0.0;
    for (int k = threadIdx.x; k < (int)gridDim.x; k += 256)
        total += __builtin_bit_cast(double, __hip_atomic_load(sums + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    total = block_sum(total);
    if (threadIdx.x == 0) *loss_all = (float)(mean ? total / max(1, count) : total);
}

// What dz and x have to bring together for dw, by parts of the rows; with bfloat16 the shifts of x's rows are taken first, and beside them
// (blockIdx.y 1) those of w's lines, a line to a wave or, if it is long, to a block
template <class T>
__global__ __launch_bounds__(256) void ce_factor_kernel(CeStats st, Upstream u, const T* __restrict__ x, long ldx, int d, int* __restrict__ shift,
                                                        FactorPart* __restrict__ part, int parts, const T* __restrict__ w, int classes,
                                                        int* __restrict__ lines)
{
    if (blockIdx.y == 1) {
        __shared__ float red[4];
        const bool block = classes > kLongLine;
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, teams = block ? 1 : 4;
        const long per = block ? (classes + 31) / 32 * 8 : classes, c0 = block ? wave * per : 0;             // a wave's quarter of a line
        for (long line = (long)blockIdx.x * teams + (block ? 0 : wave); line < d; line += (long)gridDim.x * teams) {
            float most = most_of(w + line * classes + c0, max(0l, min(per, classes - c0)), lane, 64);
            if (block) {
                __syncthreads();                             // those of the line before have been read
                if (lane == 0) red[wave] = most;
                __syncthreads();
                most = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
            }
            if (lane == 0 && (!block || wave == 0)) lines[line] = shift_of(__float_as_uint(most));
        }
        return;
    }
    if ((int)blockIdx.x >= parts) return;
    const int count = *u.count;
    FactorPart p = no_rows();
    auto add = [&](int m, int own) {
        const float g = magnitude(u.row(m));
        const int t = u.shift(g);
        if (g > 0.f && own != kNoShift) p = joined(p, {own + t, t, t});
    };
    if constexpr (sizeof(T) == 4) {
        for (long m = (long)blockIdx.x * 256 + threadIdx.x; m < count; m += (long)parts * 256) add((int)m, shift[m]);
    } else {
        each_row_most(x, ldx, st.index, count, d, parts, [&](int m, float here, bool first) {
            const int own = here > 0.f ? shift_of(__float_as_uint(here)) : kNoShift;
            if (first) shift[m] = own;
            add(m, own);
        });
    }
    p = block_joined(p);
    if (threadIdx.x == 0) part[blockIdx.x] = p;
}

// db: what the waves' rows add, `per` rows each
__global__ __launch_bounds__(256) void ce_bias_join_kernel(const float* __restrict__ part, const int* __restrict__ count, int per, int Nb,
                                                           int classes, void* db, int type, int first)
{
    __shared__ float red[16][17];
    const int parts = (*count + per - 1) / per, n = blockIdx.x * 16 + (threadIdx.x & 15), k0 = threadIdx.x >> 4;
    float s[4] = {};
    if (n < classes) {
        int k = k0;
        for (; k + 48 < parts; k += 64)
#pragma unroll
            for (int u = 0; u < 4; ++u) s[u] += part[(long)(k + u * 16) * Nb + n];
        for (; k < parts; k += 16) s[0] += part[(long)k * Nb + n];
    }
    red[k0][threadIdx.x & 15] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (threadIdx.x < 16 && n < classes) {
        float t = 0.f;
        for (int i = 0; i < 16; ++i) t += red[i][threadIdx.x];
        store_param(db, type, first + n, t);
    }
}

// ------------------------------------------------------------------------------------------
// Host
// ------------------------------------------------------------------------------------------
int fail(int code, const char* text) { return set_error(code, text); }
int launched(const char* where) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? DA_OK : set_hip_error(e, where);
}

struct CeShape {
    int64_t rows, d, V;
};

// Few classes and inner positions: da_ce_narrow.h
struct NarrowPlan {
    bool taken;
    int NF, KW;                  // fragments of the classes, and of the inner positions to a wave
    int chunk, blocks;
};
NarrowPlan narrow_plan(const CeShape& s, bool backward) {
    NarrowPlan p{};
    if (s.V < 1 || s.V > kNarrowClasses || s.d > kNarrowInner || s.rows < 1) return p;
    const int f = (int)ceil_div(s.V, 16), inner = narrow_inner(s.d);
    p.NF = f <= 4 ? f : f <= 6 ? 6 : 8;
    p.KW = inner <= 64 ? 1 : inner <= 128 ? 2 : 4;
    if (narrow_lds(p.NF, inner, true) > kNarrowLds || p.KW * p.NF > 16) return p;    // of dw, 64 registers at most
    const size_t lds = narrow_lds(p.NF, inner, backward);
    p.taken = true;
    const int64_t cus = compute_units(), resident = cus * std::max<int64_t>(1, std::min<int64_t>(6, (int64_t)(160 * 1024 / (lds + 256))));
    p.chunk = (int)std::max<int64_t>(64, std::min<int64_t>(kNarrowChunk, ceil_div(ceil_div(s.rows, resident), 64) * 64));
    p.blocks = (int)std::min(ceil_div(s.rows, p.chunk), resident);
    return p;
}

// Few classes and more inner positions: da_ce_tall.h
struct TallPlan {
    bool taken;
    int NF, chunk, blocks;       // of the rows
    int parts;                   // of the rows of dw
    int64_t per;
};
TallPlan tall_plan(const CeShape& s) {
    TallPlan p{};
    if (s.V < 1 || s.V > kTallClasses || s.rows <= 16 || s.d < 1) return p;
    p.taken = true;
    p.NF = (int)ceil_div(s.V, 16);
    const int64_t cus = compute_units(), resident = 2 * cus;
    p.chunk = (int)std::max<int64_t>(kTallRows, std::min<int64_t>(kNarrowChunk, ceil_div(ceil_div(s.rows, resident), kTallRows) * kTallRows));
    p.blocks = (int)std::min(ceil_div(s.rows, p.chunk), resident);
    // three blocks to a unit, no fewer than 256 rows to one
    const int64_t parts = std::max<int64_t>(1, std::min(ceil_div(3 * cus, ceil_div(s.d, 64)), ceil_div(s.rows, 256)));
    p.per = ceil_div(ceil_div(s.rows, parts), 64) * 64;
    p.parts = (int)ceil_div(s.rows, p.per);
    return p;
}

// Few rows: da_ce_few.h, and da_ce_some.h
struct FewPlan {
    bool taken;
    int splits, per, across;     // of the lines forward; parts of the classes backward
    int each;                    // classes of a thread in their sums
    int64_t columns, blocks;     // blocks along the classes of the logits and of their sums
};
// In how many parts `steps` of each of so many blocks are taken: the turns on the chip that take least, 4 steps to begin and end a block
int64_t some_parts(int64_t blocks, int64_t steps, int64_t slots) {
    int64_t best = 1, least = INT64_MAX;
    for (int64_t parts = 1; parts <= std::min<int64_t>(1024, steps); parts += std::max<int64_t>(1, parts / 8)) {
        const int64_t time = ceil_div(blocks * parts, slots) * (ceil_div(steps, parts) + 4);
        if (time < least) {
            least = time;
            best = parts;
        }
    }
    return best;
}
FewPlan few_plan(const CeShape& s, int size) {
    FewPlan p{};
    if (s.rows < 1 || s.rows > (size == 4 ? some_rows<float> : some_rows<bf16>) || s.d < 1 || s.V < 1) return p;
    p.taken = true;
    const int64_t cus = compute_units();
    p.each = (int)std::min<int64_t>(16, ceil_div(s.rows * ceil_div(s.V, kFewBlock), 4 * cus));
    p.blocks = ceil_div(s.V, (int64_t)kFewBlock * p.each);
    if (s.rows > kFewRows) {
        const int RF = (int)ceil_div(s.rows, 16);
        p.columns = ceil_div(s.V, kSomeStep);
        p.splits = (int)some_parts(p.columns, ceil_div(s.d, 64), some_logit_blocks(RF) * cus);
        p.per = (int)(ceil_div(ceil_div(s.d, 64), p.splits) * 64);
        p.splits = (int)ceil_div(s.d, p.per);
        p.across = (int)some_parts(ceil_div(s.d, 64), ceil_div(s.V, kSomeStep), some_blocks(RF) * cus);
        return p;
    }
    p.columns = ceil_div(s.V, 64 * 16 / size);
    // four blocks to a unit, no fewer than 32 lines to one
    const int64_t splits = std::max<int64_t>(1, std::min(ceil_div(4 * cus, p.columns), s.d / 32));
    p.per = (int)ceil_div(s.d, splits);
    p.splits = (int)ceil_div(s.d, p.per);
    p.across = (int)std::max<int64_t>(1, std::min(ceil_div(2 * cus, ceil_div(s.d, kFewDown)), ceil_div(s.V, 4 * kFewBlock)));
    return p;
}

struct PiecePlan {
    PlanePlan logits, input, weight;
};
PiecePlan piece_plan(int64_t Ma, int64_t D, int64_t width, int step) {
    const int64_t Vb = padded(width);
    const int halves = step == Halves::STEP;
    return {plane_plan(Ma, Vb, D / step, 1, false, false, halves), plane_plan(Ma, D, Vb / step, 1, false, true, halves),
            plane_plan(D, Vb, Ma / step, 1, false, true, halves)};
}

struct CePlan {
    NarrowPlan narrow, narrow_back;
    FewPlan few;
    TallPlan tall;
    size_t tall_part;
    size_t few_arrived, few_losses, few_sums, few_target, few_dz, few_dx;        // bytes
    int64_t Ma, D, Vb;           // rows, d and classes, padded
    int64_t chunk, chunks;       // of the rows
    PlanePlan logits;
    int slots;
    int64_t piece;               // classes of a piece, a multiple of 64 where there are several
    PiecePlan whole, rest;       // products of a whole piece and of the last one
    size_t spread_at, counts_at, sums_at, target_at, x_at, w_at, part_at, forward;          // bytes
    size_t arrived_at, dz_at, dx_at, bias_at, sum_at, again_at, factor_at, shift_at, wide_at, lines_at, up_at, backward;
    bool shifts() const { return !narrow.taken && !tall.taken && !few.taken && halves; }
    bool halves;
};

int wave_columns(const PlanePlan& p) { return p.shape == 0 ? PlaneLarge::WN : PlaneSmall::WN; }

CePlan make_ce_plan(int dtype, const CeShape& s) {
    CePlan p{};
    p.halves = dtype == DA_F32;
    const int N = dtype == DA_F32 ? 2 : 1, step = N == 2 ? Halves::STEP : One::STEP;
    p.Ma = padded(s.rows);
    p.D = padded(s.d);
    p.Vb = padded(s.V);
    p.chunk = std::max<int64_t>(2048, ceil_div(ceil_div(s.rows, kChunks), 256) * 256);
    p.chunks = std::max<int64_t>(1, ceil_div(s.rows, p.chunk));
    p.logits = plane_plan(p.Ma, p.Vb, p.D / step, 1, false, false, step == Halves::STEP);
    p.slots = p.logits.tiles_n * wave_columns(p.logits);
    p.narrow = narrow_plan(s, false);
    p.narrow_back = narrow_plan(s, true);
    if (p.narrow.taken) {
        p.forward = 16 + (size_t)p.narrow.blocks * 2 * sizeof(double);
        p.backward = 16 + round16((size_t)p.narrow_back.blocks * (s.d + 1) * s.V * sizeof(float));
        return p;
    }
    p.tall = tall_plan(s);
    if (p.tall.taken) {
        p.forward = 16 + (size_t)p.tall.blocks * 2 * sizeof(double);
        p.tall_part = 16 + round16((size_t)s.rows * p.tall.NF * 16 * 4);
        p.backward = p.tall_part + round16((size_t)p.tall.parts * (s.d + 1) * s.V * 4);
        return p;
    }
    size_t at = 16;                                          // Joint, or a count
    auto take = [&](size_t bytes) {
        const size_t from = at;
        at += round16(bytes);
        return from;
    };
    p.few = few_plan(s, dtype == DA_F32 ? 4 : 2);
    if (p.few.taken) {
        (void)take((size_t)p.few.splits * s.rows * p.Vb * 4);
        const size_t both = at;
        p.few_arrived = take((kSomeRows + 1) * kFewApart * 4);
        p.few_losses = take(kSomeRows * sizeof(double));
        p.few_sums = take((size_t)s.rows * p.few.blocks * sizeof(float2));
        p.few_target = take((size_t)s.rows * 4);
        p.forward = at;
        at = both;
        p.few_dz = take((size_t)s.rows * p.Vb * 4);
        p.few_dx = take(p.few.across > 1 ? (size_t)p.few.across * s.rows * s.d * 4 : 0);
        p.backward = at;
        return p;
    }
    p.x_at = take((size_t)p.Ma * p.D * 2 * N);
    p.w_at = take((size_t)p.D * p.Vb * 2 * N);
    const size_t both = at;
    p.spread_at = take(3 * kSpread * kApart * 4);
    p.counts_at = take((size_t)p.chunks * 4);
    p.sums_at = take(kJoinBlocks * sizeof(double));
    p.target_at = take((size_t)p.Ma * 4);
    p.part_at = take((size_t)p.Ma * p.slots * sizeof(float2));
    p.forward = at;

    at = both;
    p.arrived_at = take(kMostParted * sizeof(int));
    p.piece = std::max<int64_t>(1024, kPieceBytes / std::max<int64_t>(1, p.Ma * 2 * N) / 256 * 256);
    if (p.piece >= s.V) p.piece = std::max<int64_t>(s.V, 1);
    const int64_t Pb = padded(p.piece);
    p.dz_at = take((size_t)p.Ma * Pb * 2 * N);
    p.dx_at = take(p.piece < s.V ? (size_t)p.Ma * p.D * 4 : 0);
    size_t sums = 0;
    p.whole = piece_plan(p.Ma, p.D, p.piece, step);
    p.rest = s.V % p.piece ? piece_plan(p.Ma, p.D, s.V % p.piece, step) : p.whole;
    p.bias_at = take((size_t)ceil_div(p.Ma, std::min(grad_rows(p.whole.logits.shape), grad_rows(p.rest.logits.shape))) * Pb * 4);
    for (const PiecePlan& q : {p.whole, p.rest}) sums = std::max({sums, plane_part_bytes(q.input, 1), plane_part_bytes(q.weight, 1)});
    p.sum_at = take(sums);
    p.again_at = take((size_t)p.Ma * p.D * 2 * N);
    p.factor_at = take(kFactorParts * sizeof(FactorPart));
    p.shift_at = take(N == 1 ? (size_t)s.rows * 4 : 0);
    p.up_at = take((size_t)s.rows * 4);
    p.wide_at = take(N == 1 ? (size_t)p.D * p.Vb * 2 : 0);
    p.lines_at = take(N == 1 ? (size_t)p.D * 4 : 0);
    p.backward = at;
    return p;
}

// A call asks for its plan twice, and a program for the same one in every step
const CePlan& ce_plan(int dtype, const CeShape& s) {
    struct Last {
        int dtype = -1, units = 0;
        CeShape s{};
        CePlan p{};
    };
    thread_local Last last;
    const int units = compute_units();
    if (last.dtype != dtype || last.units != units || last.s.rows != s.rows || last.s.d != s.d || last.s.V != s.V) {
        last.p = make_ce_plan(dtype, s);
        last.s = s;
        last.units = units;
        last.dtype = dtype;
    }
    return last.p;
}

int ce_check(int dtype, int64_t rows, int64_t d, int64_t classes) {
    if (dtype != DA_F32 && dtype != DA_BF16) return fail(DA_ERR_UNSUPPORTED, "dtype is neither DA_F32 nor DA_BF16");
    if (rows < 0 || d < 0 || classes < 0) return fail(DA_ERR_INVALID_ARG, "negative size");
    if (rows > kCeRowsMost || d > kCeMost || classes > kCeMost) return fail(DA_ERR_UNSUPPORTED, "size too large");
    // a launch's threads are counted in 32 bits: tiles of 256 x 256 where there are many, and 512 threads to one
    const int64_t m = ceil_div(rows, 256), n = ceil_div(d, 256), v = ceil_div(classes, 256);
    if (std::max({m * v, m * n, n * v}) >= 1 << 23) return fail(DA_ERR_UNSUPPORTED, "size too large");
    return DA_OK;
}

struct CeCall {
    CeShape s;
    CePlan p;
    const void *x, *w, *b;
    int64_t ldx;
    int param_dtype;
    CeStats st;
    char* ws;
    hipStream_t stream;
};

template <class T>
const uint16_t* pack_operands(const CeCall& c, const BeginJob<T>& begin, const JointJob& again, const LinesJob& lines, Packed* lw) {
    typedef PlaneOf<T> P;
    const T* x = static_cast<const T*>(c.x);
    const T* w = static_cast<const T*>(c.w);
    uint32_t* const spread = begin.arrived ? nullptr : reinterpret_cast<uint32_t*>(c.ws + c.p.spread_at);
    if constexpr (P::N == 2) {
        if (!begin.arrived) {                                // kept for the backward pass
            const int64_t most = std::max(ceil_div(c.s.rows, 4), ceil_div(c.s.d * c.s.V, 4096));
            hipLaunchKernelGGL(ce_max_kernel, dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(most, 1024)), 2), dim3(256), 0, c.stream, x,
                               (long)c.ldx, c.st, (long)c.s.d, w, (long)(c.s.d * c.s.V), spread);
        }
    }
    auto job = [&](const T* from, long ld, long lines, int n, const int* index, size_t to) {
        return PackJob<T>{from, ld, lines, lines, n, index, c.st.count, reinterpret_cast<uint16_t*>(c.ws + to), packed(padded(lines), n, P::N)};
    };
    const PackJob<T> jx = job(x, c.ldx, c.s.rows, (int)c.s.d, c.st.index, c.p.x_at), jw = job(w, c.s.V, c.s.d, (int)c.s.V, nullptr, c.p.w_at);
    // a weight of whole pads is read where it is
    const bool direct = P::N == 1 && c.s.d % kPad == 0 && c.s.V % kPad == 0 && reinterpret_cast<uintptr_t>(w) % 16 == 0;
    const int64_t tiles = std::max(c.p.Ma / 16 * ceil_div(c.p.D, 128), direct && !lines.to ? 0 : c.p.D / 16 * ceil_div(c.p.Vb, 128));
    PackJob<T> jw_here = jw;
    if (direct) jw_here.lines = 0;
    if (tiles || begin.arrived)
        hipLaunchKernelGGL((ce_pack_kernel<T, P, GradOf<T>>),
                           dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(tiles, 8192)), lines.to ? 5 : again.to ? 4 : begin.arrived ? 3 : direct ? 1 : 2),
                           dim3(256), 0, c.stream, c.st, spread, jx, jw_here, begin, again, lines);
    *lw = direct ? packed_lines(c.s.V) : jw.layout;
    return direct ? reinterpret_cast<const uint16_t*>(w) : jw.to;
}

template <class P> void fill(Logits<P>& l, const CeCall& c) {
    l.bias = c.b;
    l.bias_type = c.param_dtype;
    l.classes = (int)c.s.V;
    l.st = c.st;
}

// Operands of the logits' product of the classes from `first` on
template <class P> PlaneArgs logits_args(const CeCall& c, const uint16_t* w, const Packed& lw, int64_t first, int64_t width) {
    PlaneArgs g{};
    g.A = reinterpret_cast<const uint16_t*>(c.ws + c.p.x_at);
    g.a = packed(c.p.Ma, c.s.d, P::N);
    g.B = w + place<P>(lw, 0, first);
    g.b = lw;
    g.Ma = (int)c.p.Ma;
    g.Nb = (int)padded(width);
    g.K = (int)c.p.D;
    g.rows = c.st.count;
    return g;
}

template <class T>
void ce_forward(const CeCall& c, const void* target, int target64, int reduction, float* loss) {
    typedef PlaneOf<T> P;
    int* counts = reinterpret_cast<int*>(c.ws + c.p.counts_at);
    const bool several = c.p.chunks > 1;
    if (several)
        hipLaunchKernelGGL(ce_count_kernel, dim3((unsigned)c.p.chunks), dim3(256), 0, c.stream, target, target64, (long)c.s.rows, (long)c.s.V,
                           (long)c.p.chunk, counts);
    float* rows = reduction == DA_LOSS_ROWS ? loss : nullptr;
    hipLaunchKernelGGL(ce_index_kernel, dim3((unsigned)c.p.chunks), dim3(256), 0, c.stream, target, target64, (long)c.s.rows, (long)c.s.V,
                       (long)c.p.chunk, several ? counts : nullptr, c.st,
                       reinterpret_cast<uint32_t*>(c.ws + c.p.spread_at), rows);
    Packed lw{};
    const uint16_t* w = pack_operands<T>(c, BeginJob<T>{}, JointJob{}, LinesJob{}, &lw);
    SumsOut<P> out{};
    fill(out, c);
    out.part = reinterpret_cast<float2*>(c.ws + c.p.part_at);
    out.slots = c.p.slots;
    out.at_target = reinterpret_cast<float*>(c.ws + c.p.target_at);
    plane_product<P, kAlong, kAcross, kBoundM>(logits_args<P>(c, w, lw, 0, c.s.V), out, c.p.logits, 1, nullptr, nullptr, c.stream);
    int lanes = 1;
    while (lanes < 64 && lanes < c.p.slots) lanes *= 2;
    uint64_t* sums = reduction == DA_LOSS_ROWS ? nullptr : reinterpret_cast<uint64_t*>(c.ws + c.p.sums_at);
    const int blocks = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(c.s.rows, 256 / lanes), kJoinBlocks));
    hipLaunchKernelGGL(ce_join_kernel, dim3(blocks), dim3(256), 0, c.stream, c.st, out.part, c.p.slots, lanes, out.at_target, rows, sums,
                       c.st.maxes + kArrived, (int)(reduction == DA_LOSS_MEAN), loss);
}

template <class T>
void ce_backward(const CeCall& c, int reduction, const float* dloss, int64_t stride, T* dx, T* dw, void* db) {
    typedef PlaneOf<T> P;
    typedef GradOf<T> Q;
    int* arrived = reinterpret_cast<int*>(c.ws + c.p.arrived_at);
    Joint* joint = reinterpret_cast<Joint*>(c.ws);
    const Upstream u{dloss, (long)stride, reduction, c.st.count, c.st.index};
    if (c.s.d == 0) dx = dw = nullptr;
    JointJob again{};
    LinesJob lines{};
    FactorPart* factors = reinterpret_cast<FactorPart*>(c.ws + c.p.factor_at);
    int* shift = P::N == 2 ? c.st.shift : reinterpret_cast<int*>(c.ws + c.p.shift_at);
    int* line_shift = reinterpret_cast<int*>(c.ws + c.p.lines_at);
    const int64_t at_once = P::N == 2 ? 256 : 256 / row_lanes(c.s.d, sizeof(T)) * kAtOnce;
    const int parts = dw ? (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(c.s.rows, at_once), kFactorParts)) : 0;
    if (dw && c.s.V > 0) again = JointJob{u, factors, parts, shift, joint, reinterpret_cast<uint16_t*>(c.ws + c.p.again_at)};
    if (P::N == 1 && dx && c.s.V > 0) lines = LinesJob{line_shift, reinterpret_cast<uint16_t*>(c.ws + c.p.wide_at)};
    if ((again.to || lines.to) && (P::N == 1 || reduction == DA_LOSS_ROWS)) {
        const int64_t line_blocks = lines.to ? std::min<int64_t>(ceil_div(c.s.d, c.s.V > kLongLine ? 1 : 4), 4096) : 0;
        hipLaunchKernelGGL((ce_factor_kernel<T>), dim3((unsigned)std::max<int64_t>(parts, line_blocks), lines.to ? 2 : 1), dim3(256), 0, c.stream, c.st,
                           u, static_cast<const T*>(c.x), (long)c.ldx, (int)c.s.d, shift, factors, parts, static_cast<const T*>(c.w), (int)c.s.V,
                           line_shift);
    }
    Packed lw{};
    const uint16_t* w = pack_operands<T>(c, BeginJob<T>{(long)c.s.rows, (int)c.s.d, dx, arrived}, again, lines, &lw);
    if (c.s.V == 0) return;
    uint16_t* dz = reinterpret_cast<uint16_t*>(c.ws + c.p.dz_at);
    float* acc = reinterpret_cast<float*>(c.ws + c.p.dx_at);
    float* part = reinterpret_cast<float*>(c.ws + c.p.sum_at);
    float* bias = reinterpret_cast<float*>(c.ws + c.p.bias_at);
    for (int64_t first = 0; first < c.s.V; first += c.p.piece) {
        const int64_t width = std::min(c.p.piece, c.s.V - first), Vb = padded(width);
        const PiecePlan& q = width == c.p.piece ? c.p.whole : c.p.rest;
        const Packed lz = packed(c.p.Ma, width, P::N);
        int* const up = reinterpret_cast<int*>(c.ws + c.p.up_at);
        auto gradient = [&](auto out) {
            fill(out, c);
            out.u = u;
            out.first = (int)first;
            out.dz = dz;
            out.lz = lz;
            out.up = up;
            out.sums = bias;
            plane_product<P, kAlong, kAcross, kBoundM>(logits_args<P>(c, w, lw, first, width), out, q.logits, 1, nullptr, nullptr, c.stream);
        };
        if (db) gradient(GradOut<P, Q, true>{});
        else gradient(GradOut<P, Q, false>{});
        if (dx) {
            PlaneArgs a{};
            a.A = dz;
            a.a = lz;
            const Packed lb = P::N == 2 ? lw : packed(c.p.D, c.s.V, 1);
            a.B = (P::N == 2 ? w : lines.to) + place<Q>(lb, 0, first);
            a.b = lb;
            a.Ma = (int)c.p.Ma;
            a.Nb = (int)c.p.D;
            a.K = (int)Vb;
            a.rows = c.st.count;
            InputOut<T, Q> out{};
            out.st = c.st;
            out.shift = up;
            out.before = first > 0 ? acc : nullptr;
            out.after = first + width < c.s.V ? acc : nullptr;
            out.ldb = c.p.D;
            out.dx = dx;
            out.d = (int)c.s.d;
            out.lines = line_shift;
            plane_product<Q, kAlong, kAlong, kBoundM>(a, out, q.input, 1, part, arrived, c.stream);
        }
        if (dw) {
            PlaneArgs a{};
            a.A = P::N == 2 ? reinterpret_cast<const uint16_t*>(c.ws + c.p.x_at) : again.to;
            a.a = packed(c.p.Ma, c.s.d, P::N);
            a.B = dz;
            a.b = lz;
            a.Ma = (int)c.p.D;
            a.Nb = (int)Vb;
            a.K = (int)c.p.Ma;
            a.rows = c.st.count;
            a.other = P::N == 2 ? &joint->differ : nullptr;
            a.A_other = again.to;
            const WeightOut<T> out{joint, dw + first, (long)c.s.V, (int)c.s.d, (int)width};
            plane_product<Q, kAcross, kAcross, kBoundK>(a, out, q.weight, 1, part, arrived, c.stream);
        }
        if (db) {
            hipLaunchKernelGGL(ce_bias_join_kernel, dim3((unsigned)ceil_div(width, 16)), dim3(256), 0, c.stream, bias, c.st.count,
                               grad_rows(q.logits.shape), (int)Vb, (int)width, db, c.param_dtype, (int)first);
        }
    }
}

// ... a launch by the fragments that a call has
template <class T, bool BWD> void narrow_launch(const NarrowPlan& p, const NarrowArgs& a, hipStream_t s) {
    const size_t lds = narrow_lds(p.NF, narrow_inner(a.d), BWD);
    auto go = [&](auto k) {
        constexpr auto kernel = decltype(k)::value;
        allow_lds<kernel>(kNarrowLds);
        hipLaunchKernelGGL(kernel, dim3((unsigned)p.blocks), dim3(kNarrowBlock), lds, s, a);
    };
    auto by_inner = [&](auto nf) {
        constexpr int NF = decltype(nf)::value;
        if (!BWD || p.KW == 1) go(std::integral_constant<void (*)(NarrowArgs), ce_narrow_kernel<T, NF, 1, BWD>>());
        else if (p.KW == 2) go(std::integral_constant<void (*)(NarrowArgs), ce_narrow_kernel<T, NF, BWD ? 2 : 1, BWD>>());
        else if constexpr (NF <= 4) go(std::integral_constant<void (*)(NarrowArgs), ce_narrow_kernel<T, NF, BWD ? 4 : 1, BWD>>());
    };
    if (p.NF == 1) by_inner(std::integral_constant<int, 1>());
    else if (p.NF == 2) by_inner(std::integral_constant<int, 2>());
    else if (p.NF == 3) by_inner(std::integral_constant<int, 3>());
    else if (p.NF == 4) by_inner(std::integral_constant<int, 4>());
    else if (p.NF == 6) by_inner(std::integral_constant<int, 6>());
    else by_inner(std::integral_constant<int, 8>());
}

// The statistics of such a call are by row: the class or -1, and log sum exp
NarrowArgs narrow_args(const CeCall& c, const NarrowPlan& p, int reduction) {
    NarrowArgs a{};
    a.x = c.x;
    a.w = c.w;
    a.b = c.b;
    a.ldx = c.ldx;
    a.rows = c.s.rows;
    a.d = (int)c.s.d;
    a.V = (int)c.s.V;
    a.param_type = c.param_dtype;
    a.reduction = reduction;
    a.chunk = p.chunk;
    a.count = c.st.count;
    a.kept_target = c.st.target;
    a.lse = c.st.lse;
    return a;
}
template <class T> void narrow_forward(const CeCall& c, const void* target, int target64, int reduction, float* loss) {
    NarrowArgs a = narrow_args(c, c.p.narrow, reduction);
    a.target = target;
    a.target64 = target64;
    a.loss = loss;
    a.sums = reinterpret_cast<double*>(c.ws + 16);
    narrow_launch<T, false>(c.p.narrow, a, c.stream);
    if (c.p.narrow.blocks > 1) hipLaunchKernelGGL(ce_narrow_total_kernel, dim3(1), dim3(256), 0, c.stream, a, c.p.narrow.blocks);
}
template <class T>
void narrow_backward(const CeCall& c, int reduction, const float* dloss, int64_t stride, void* dx, void* dw, void* db) {
    const NarrowPlan& p = c.p.narrow_back;
    NarrowArgs a = narrow_args(c, p, reduction);
    a.dloss = dloss;
    a.stride = stride;
    a.dx = c.s.d ? dx : nullptr;
    a.dw = c.s.d ? dw : nullptr;
    a.db = db;
    a.part = reinterpret_cast<float*>(c.ws + 16);
    narrow_launch<T, true>(p, a, c.stream);
    const int64_t numbers = (a.dw ? c.s.d * c.s.V : 0) + (db ? c.s.V : 0);
    if (p.blocks > 1 && numbers)
        hipLaunchKernelGGL((ce_narrow_join_kernel<T>), dim3(narrow_join_blocks(numbers)), dim3(256), 0, c.stream, a, p.blocks);
}

template <class F> void by_fragments(int NF, F&& go) {
    if (NF == 1) go(std::integral_constant<int, 1>());
    else if (NF == 2) go(std::integral_constant<int, 2>());
    else if (NF == 3) go(std::integral_constant<int, 3>());
    else go(std::integral_constant<int, 4>());
}
TallArgs tall_args(const CeCall& c, int reduction) {
    NarrowPlan p{};
    p.chunk = c.p.tall.chunk;
    TallArgs a{};
    static_cast<NarrowArgs&>(a) = narrow_args(c, p, reduction);
    return a;
}
template <class T> void tall_forward(const CeCall& c, const void* target, int target64, int reduction, float* loss) {
    TallArgs a = tall_args(c, reduction);
    a.target = target;
    a.target64 = target64;
    a.loss = loss;
    a.sums = reinterpret_cast<double*>(c.ws + 16);
    by_fragments(c.p.tall.NF, [&](auto nf) {
        hipLaunchKernelGGL((ce_tall_kernel<T, decltype(nf)::value, false>), dim3((unsigned)c.p.tall.blocks), dim3(kNarrowBlock), 0, c.stream, a);
    });
    if (c.p.tall.blocks > 1) hipLaunchKernelGGL(ce_narrow_total_kernel, dim3(1), dim3(256), 0, c.stream, static_cast<const NarrowArgs&>(a), c.p.tall.blocks);
}
template <class T> void tall_backward(const CeCall& c, int reduction, const float* dloss, int64_t stride, void* dx, void* dw, void* db) {
    const TallPlan& p = c.p.tall;
    TallArgs a = tall_args(c, reduction);
    a.dloss = dloss;
    a.stride = stride;
    a.dx = dx;
    a.dw = dw;
    a.db = db;
    a.dz = reinterpret_cast<float*>(c.ws + 16);
    a.part = reinterpret_cast<float*>(c.ws + c.p.tall_part);
    a.per = p.per;
    by_fragments(p.NF, [&](auto nf) {
        hipLaunchKernelGGL((ce_tall_kernel<T, decltype(nf)::value, true>), dim3((unsigned)p.blocks), dim3(kNarrowBlock), 0, c.stream, a);
        if (dw || db)
            hipLaunchKernelGGL((ce_tall_weight_kernel<T, decltype(nf)::value>), dim3((unsigned)(dw ? ceil_div(c.s.d, 64) : 1), (unsigned)p.parts),
                               dim3(kNarrowBlock), 0, c.stream, a);
    });
    const int64_t numbers = (dw ? c.s.d * c.s.V : 0) + (db ? c.s.V : 0);
    if (numbers)
        hipLaunchKernelGGL((ce_narrow_join_kernel<T>), dim3(narrow_join_blocks(numbers)), dim3(256), 0, c.stream, static_cast<const NarrowArgs&>(a),
                           p.parts);
}

// ... by the rows that registers are held for
template <class F> void by_rows(int64_t rows, F&& go) {
    if (rows == 1) go(std::integral_constant<int, 1>());
    else if (rows == 2) go(std::integral_constant<int, 2>());
    else go(std::integral_constant<int, 4>());
}
FewArgs few_args(const CeCall& c, int reduction) {
    FewArgs a{};
    a.x = c.x;
    a.w = c.w;
    a.b = c.b;
    a.ldx = c.ldx;
    a.V = c.s.V;
    a.Vp = c.p.Vb;
    a.rows = (int)c.s.rows;
    a.d = (int)c.s.d;
    a.param_type = c.param_dtype;
    a.reduction = reduction;
    a.splits = c.p.few.splits;
    a.per = c.p.few.per;
    a.part = reinterpret_cast<float*>(c.ws + 16);
    a.count = c.st.count;
    a.kept_target = c.st.target;
    a.lse = c.st.lse;
    return a;
}
template <class T, class G> void by_some(int rows, const G& go) {
    if (rows <= 16) return go(std::integral_constant<int, 1>());
    if (some_rows<T> == 32 || rows <= 32) return go(std::integral_constant<int, 2>());
    if constexpr (some_rows<T> > 32) {
        if (rows <= 48) go(std::integral_constant<int, 3>());
        else go(std::integral_constant<int, 4>());
    }
}
template <class T, bool BWD> void few_logits(const CeCall& c, const FewArgs& a) {
    const dim3 grid((unsigned)c.p.few.columns, (unsigned)a.splits), block(kFewBlock);
    if (a.rows > kFewRows)
        by_some<T>(a.rows, [&](auto f) { hipLaunchKernelGGL((ce_some_logits_kernel<T, decltype(f)::value, BWD>), grid, block, 0, c.stream, a); });
    else by_rows(c.s.rows, [&](auto r) { hipLaunchKernelGGL((ce_few_logits_kernel<T, decltype(r)::value, BWD>), grid, block, 0, c.stream, a); });
}
template <class T> void few_forward(const CeCall& c, const void* target, int target64, int reduction, float* loss) {
    FewArgs a = few_args(c, reduction);
    a.target = target;
    a.target64 = target64;
    a.loss = loss;
    a.each = c.p.few.each;
    a.arrived = reinterpret_cast<uint32_t*>(c.ws + c.p.few_arrived);
    a.losses = reinterpret_cast<double*>(c.ws + c.p.few_losses);
    a.sums = reinterpret_cast<float2*>(c.ws + c.p.few_sums);
    a.at_target = reinterpret_cast<float*>(c.ws + c.p.few_target);
    few_logits<T, false>(c, a);
    hipLaunchKernelGGL(ce_few_sums_kernel, dim3((unsigned)c.p.few.blocks, (unsigned)a.rows), dim3(kFewBlock), 0, c.stream, a);
}
template <class T> void few_backward(const CeCall& c, int reduction, const float* dloss, int64_t stride, void* dx, void* dw, void* db) {
    FewArgs a = few_args(c, reduction);
    a.dloss = dloss;
    a.stride = stride;
    a.dx = dx;
    a.dw = dw;
    a.db = db;
    a.dz = reinterpret_cast<float*>(c.ws + c.p.few_dz);
    a.dx_part = reinterpret_cast<float*>(c.ws + c.p.few_dx);
    few_logits<T, true>(c, a);
    if (a.rows > kFewRows) {
        hipLaunchKernelGGL(ce_some_grad_kernel, dim3((unsigned)ceil_div(a.Vp, kFewBlock), (unsigned)a.rows), dim3(kFewBlock), 0, c.stream, a);
        by_some<T>(a.rows, [&](auto f) {
            hipLaunchKernelGGL((ce_some_products_kernel<T, decltype(f)::value>), dim3((unsigned)(dx || dw ? ceil_div(c.s.d, 64) : 1), (unsigned)c.p.few.across),
                               dim3(kFewBlock), 0, c.stream, a);
        });
    } else {
        hipLaunchKernelGGL(ce_few_grad_kernel, dim3((unsigned)ceil_div(a.Vp, kFewBlock)), dim3(kFewBlock), 0, c.stream, a);
        if (!dx && !dw) return;
        by_rows(c.s.rows, [&](auto r) {
            hipLaunchKernelGGL((ce_few_products_kernel<T, decltype(r)::value>), dim3((unsigned)ceil_div(c.s.d, kFewDown), (unsigned)c.p.few.across),
                               dim3(kFewBlock), 0, c.stream, a);
        });
    }
    if (dx && c.p.few.across > 1)
        hipLaunchKernelGGL((ce_few_join_kernel<T>), dim3((unsigned)ceil_div((int64_t)a.rows * a.d, kFewBlock)), dim3(kFewBlock), 0, c.stream, a,
                           c.p.few.across);
}

int ce_call(int dtype, int64_t rows, int64_t d, int64_t classes, const void* x, int64_t ldx, const void* w, const void* b, int param_dtype,
            int reduction, const void* stats, void* workspace, size_t workspace_bytes, bool backward, void* stream, CeCall* c) {
    const int st = ce_check(dtype, rows, d, classes);
    if (st != DA_OK) return st;
    if (b && param_dtype != DA_F32 && param_dtype != DA_BF16) return fail(DA_ERR_UNSUPPORTED, "param_dtype is neither DA_F32 nor DA_BF16");
    if (reduction != DA_LOSS_ROWS && reduction != DA_LOSS_SUM && reduction != DA_LOSS_MEAN) return fail(DA_ERR_INVALID_ARG, "unknown reduction");
    if (ldx < d) return fail(DA_ERR_INVALID_ARG, "leading dimension smaller than the extent it strides over");
    if ((rows > 0 && d > 0 && !x) || (d > 0 && classes > 0 && !w)) return fail(DA_ERR_INVALID_ARG, "null x or w");
    if (!stats || reinterpret_cast<uintptr_t>(stats) % 16 != 0) return fail(DA_ERR_INVALID_ARG, "stats missing or misaligned");
    c->s = CeShape{rows, d, classes};
    c->p = ce_plan(dtype, c->s);
    if (!workspace || workspace_bytes < (backward ? c->p.backward : c->p.forward) || reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
        return fail(DA_ERR_INVALID_ARG, "workspace missing, misaligned or smaller than reported");
    c->x = x;
    c->w = w;
    c->b = b;
    c->ldx = ldx;
    c->param_dtype = param_dtype;
    c->st = ce_stats(const_cast<void*>(stats), rows);
    c->ws = static_cast<char*>(workspace);
    c->stream = (hipStream_t)stream;
    return DA_OK;
}

}  // namespace
}  // namespace daspmm

using namespace daspmm;

extern "C" int da_linear_cross_entropy_sizes(int dtype, int64_t rows, int64_t d, int64_t classes, size_t* stats, size_t* forward_bytes,
                                             size_t* backward_bytes)
{
    if (!stats || !forward_bytes || !backward_bytes) return fail(DA_ERR_INVALID_ARG, "null output");
    const int st = ce_check(dtype, rows, d, classes);
    if (st != DA_OK) return st;
    const CePlan& p = ce_plan(dtype, CeShape{rows, d, classes});
    *stats = stats_bytes(rows, p.shifts());
    *forward_bytes = p.forward;
    *backward_bytes = p.backward;
    return DA_OK;
}

extern "C" int da_linear_cross_entropy(int dtype, int64_t rows, int64_t d, int64_t classes, const void* x, int64_t ldx, const void* w,
                                       const void* b, int param_dtype, const void* target, int target64, int reduction, float* loss,
                                       void* stats, void* workspace, size_t workspace_bytes, void* stream)
{
    CeCall c{};
    const int st = ce_call(dtype, rows, d, classes, x, ldx, w, b, param_dtype, reduction, stats, workspace, workspace_bytes, false, stream, &c);
    if (st != DA_OK) return st;
    if (rows > 0 && !target) return fail(DA_ERR_INVALID_ARG, "null target");
    if (!loss && (rows > 0 || reduction != DA_LOSS_ROWS)) return fail(DA_ERR_INVALID_ARG, "null loss");
    if (c.p.narrow.taken) {
        if (dtype == DA_F32) narrow_forward<float>(c, target, target64, reduction, loss);
        else narrow_forward<bf16>(c, target, target64, reduction, loss);
        return launched("da_linear_cross_entropy launch");
    }
    if (c.p.tall.taken) {
        if (dtype == DA_F32) tall_forward<float>(c, target, target64, reduction, loss);
        else tall_forward<bf16>(c, target, target64, reduction, loss);
        return launched("da_linear_cross_entropy launch");
    }
    if (c.p.few.taken) {
        if (dtype == DA_F32) few_forward<float>(c, target, target64, reduction, loss);
        else few_forward<bf16>(c, target, target64, reduction, loss);
        return launched("da_linear_cross_entropy launch");
    }
    if (dtype == DA_F32) ce_forward<float>(c, target, target64, reduction, loss);
    else ce_forward<bf16>(c, target, target64, reduction, loss);
    return launched("da_linear_cross_entropy launch");
}

extern "C" int da_linear_cross_entropy_backward(int dtype, int64_t rows, int64_t d, int64_t classes, const void* x, int64_t ldx,
                                                const void* w, const void* b, int param_dtype, int reduction, const void* stats,
                                                const float* dloss, int64_t dloss_stride, void* dx, void* dw, void* db, void* workspace,
                                                size_t workspace_bytes, void* stream)
{
    CeCall c{};
    const int st = ce_call(dtype, rows, d, classes, x, ldx, w, b, param_dtype, reduction, stats, workspace, workspace_bytes, true, stream, &c);
    if (st != DA_OK) return st;
    if (dloss_stride < 0) return fail(DA_ERR_INVALID_ARG, "negative stride");
    if (!dloss && (rows > 0 || reduction != DA_LOSS_ROWS)) return fail(DA_ERR_INVALID_ARG, "null dloss");
    if (db && param_dtype != DA_F32 && param_dtype != DA_BF16) return fail(DA_ERR_UNSUPPORTED, "param_dtype is neither DA_F32 nor DA_BF16");
    if (!dx && !dw && !db) return DA_OK;
    if (c.p.narrow.taken) {
        if (dtype == DA_F32) narrow_backward<float>(c, reduction, dloss, dloss_stride, dx, dw, db);
        else narrow_backward<bf16>(c, reduction, dloss, dloss_stride, dx, dw, db);
        return launched("da_linear_cross_entropy_backward launch");
    }
    if (c.p.tall.taken) {
        if (dtype == DA_F32) tall_backward<float>(c, reduction, dloss, dloss_stride, dx, dw, db);
        else tall_backward<bf16>(c, reduction, dloss, dloss_stride, dx, dw, db);
        return launched("da_linear_cross_entropy_backward launch");
    }
    if (c.p.few.taken) {
        if (dtype == DA_F32) few_backward<float>(c, reduction, dloss, dloss_stride, dx, dw, db);
        else few_backward<bf16>(c, reduction, dloss, dloss_stride, dx, dw, db);
        return launched("da_linear_cross_entropy_backward launch");
    }
    if (dtype == DA_F32) ce_backward<float>(c, reduction, dloss, dloss_stride, static_cast<float*>(dx), static_cast<float*>(dw), db);
    else ce_backward<bf16>(c, reduction, dloss, dloss_stride, static_cast<bf16*>(dx), static_cast<bf16*>(dw), db);
    return launched("da_linear_cross_entropy_backward launch");
}
