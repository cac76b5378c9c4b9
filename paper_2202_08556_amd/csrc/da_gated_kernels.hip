// The gated feed-forward block on the matrix cores:
//   u = x Wg, v = x Wu, a = act(u) v, y = a Wd
//   da = dy Wd^T, du = da v act'(u), dv = da act(u), dx = du Wg^T + dv Wu^T, dWg = x^T du, dWu = x^T dv, dWd = a^T dy
// Every line is one product with the rest in its epilogue: both projections share the tile of x and leave as a; du and
// dv leave the product of da; dx is one sum over both pairs.
//
// Operands stay as they are in memory.  A tile of one is either lines of neighbouring inner positions (x, a, dy
// everywhere but in the weights' gradients, the weights in products with their transposes) or lines of neighbouring
// outer ones.  Both are copied to LDS line by line; the second kind is turned around on the way to the registers (for
// bf16 by the transposing LDS read, for float by reading single numbers).
//
// Forward, 8192 x 2048 x 4096 float32: 126 TFLOP/s (the fp32 matrix cores give the general library 154 on large products);
// 2000 x 512 x 2048 bf16, tiles of 128 x 128 and 64 x 64: 285.  A tile's next step waits in registers while this one is
// multiplied; with one block to a compute unit its latency shows, with several they fill each other's gaps.  (Four waves of
// 64 x 64 for a tile of 128 x 128 instead of eight of 32 x 64: 546 us instead of 521 for 100 003 x 64 x 256 float32, both ways.)
#pragma once
#include "da_gated_plan.h"
#include "da_layer_common.h"

namespace daspmm {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

enum { kInner = 0, kOuter = 1 };             // what neighbours in memory

// 16 bytes a lane are a fragment: 8 bf16, one instruction of 16 x 16 x 32, or 4 floats, four of 16 x 16 x 4 (element j
// of all lanes is one instruction: any assignment of inner positions to instructions gives the same sum).
template <class T> struct Mma;
template <> struct Mma<bf16> {
    typedef bf16x8 Frag;
    typedef Pack<uint16_t, 8>::type Memory;                  // at any address that an element may have
    static constexpr int VEC = 8;
    static constexpr int TURNS = 1;                          // instructions that a product of fragments takes
    static __device__ __forceinline__ f32x4 mul(const Frag& a, const Frag& b, f32x4 c, int = 0) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Mma<float> {
    typedef f32x4 Frag;
    typedef Pack<float, 4>::type Memory;
    static constexpr int VEC = 4;
    static constexpr int TURNS = 4;
    static __device__ __forceinline__ f32x4 mul(const Frag& a, const Frag& b, f32x4 c, int turn) {
        return __builtin_amdgcn_mfma_f32_16x16x4f32(a[turn], b[turn], c, 0, 0, 0);
    }
};

template <class T> struct GemmArgs {
    const T* A[2];
    const T* B[2];               // kGate: the second half of a tile's columns; otherwise operands of the second segment or batch
    long lda, ldb;
    int M, N, K;                 // K of one segment
    int segments;                // pairs of operands whose products are summed
    int splits, per;             // parts of the sum and tiles of the inner axis to each
    T* C[2];                     // kStore: by batch; kGate: a; kGateGrad: du, dv
    float *U, *V;                // kGate: written where not null; kGateGrad: read; dense M x N
    float* part;                 // splits > 1: [batch][split][M][N] sums, of u and v side by side for kGate
    int act;
};

// One operand's tile: OUTER outer positions x kLineBytes of the inner axis
template <class T, int LAY, int OUTER> struct Tile {
    static constexpr int VEC = Mma<T>::VEC, BK = kLineBytes / (int)sizeof(T);
    static constexpr int LINES = LAY == kInner ? OUTER : BK;
    static constexpr int CHUNKS = (LAY == kInner ? BK : OUTER) / VEC;         // of 16 bytes in a line
    // padding: 8 or 16 lines of a fragment's read lie in different banks
    static constexpr int PITCH = CHUNKS * 16 + (LAY == kOuter && sizeof(T) == 2 ? 32 : 16);
    static constexpr int BYTES = LINES * PITCH;

    // the fragment of outer positions o .. o + 15 and the step-th half of the inner axis
    static __device__ __forceinline__ typename Mma<T>::Frag frag(const char* lds, int o, int step) {
        const int i = threadIdx.x & 15, h = (threadIdx.x & 63) >> 4;
        if constexpr (LAY == kInner) {
            return *reinterpret_cast<const typename Mma<T>::Frag*>(lds + (o + i) * PITCH + step * 64 + h * 16);
        } else if constexpr (sizeof(T) == 2) {
            // 16 lanes read 4 lines of 16 numbers and get a number of each line
            const char* p = lds + (step * 32 + h * 8 + i / 4) * PITCH + (o + (i & 3) * 4) * 2;
            typedef __attribute__((address_space(3))) s16x4* Lds;
            union { s16x4 half[2]; bf16x8 all; } f;
            f.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)p);
            f.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + 4 * PITCH));
            return f.all;
        } else {
            const char* p = lds + (step * 16 + h * 4) * PITCH + (o + i) * 4;
            f32x4 f;
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = *reinterpret_cast<const float*>(p + j * PITCH);
            return f;
        }
    }
};

template <class T> __device__ __forceinline__ uint4 whole_chunk(const T* p) {
    const auto v = *reinterpret_cast<const typename Mma<T>::Memory*>(p);
    uint4 r;
    __builtin_memcpy(&r, &v, 16);
    return r;
}
// 16 bytes from p on, of which `left` elements are there (none or less: zeros).  Most pieces of a tile at an edge are whole or
// not there at all.
template <class T> __device__ __forceinline__ uint4 edge_chunk(const T* p, int left) {
    constexpr int VEC = Mma<T>::VEC;
    uint4 r = make_uint4(0, 0, 0, 0);
    if (left >= VEC) {
        r = whole_chunk(p);
    } else if (left > 0) {
        T v[VEC] = {};
#pragma unroll
        for (int i = 0; i < VEC - 1; ++i)
            if (i < left) v[i] = p[i];
        __builtin_memcpy(&r, v, 16);
    }
    return r;
}

// Results of a wave, MT x NT fragments from row m0 on, leave by way of LDS (`mine`, the wave's own part), 16 rows at a time:
// a lane's four neighbours in a row and the 16 rows of a fragment would be 64 bytes of each row at a time, and stores of
// parts of lines ran at 2.9 TB/s; this way a store is whole lines.  kGate: the first half of the fragments are u, the
// others v of the same columns.
template <class T, int MT, int NT, int EPI>
__device__ __forceinline__ void line_epilogue(const GemmArgs<T>& g, f32x4 (&acc)[MT][NT], char* mine, int m0, int n0, int batch)
{
    constexpr int COLS = EPI == kGate ? NT * 8 : NT * 16, PITCH = (NT * 16 + 4) * 4;
    constexpr int LANES = COLS / 4, ROWS = 64 / LANES, PASSES = 16 / ROWS;    // lanes of a row, rows at once
    const int lane = threadIdx.x & 63, i16 = lane & 15, h = lane >> 4;
    const int row0 = lane / LANES, col = lane % LANES * 4, n = n0 + col, left = g.N - n;
    float u[2][PASSES][4], v[2][PASSES][4];                  // kGateGrad: of the next 16 rows and of these
    auto load = [&](int i, int to) {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int m = m0 + i * 16 + p * ROWS + row0;
            if (m >= g.M || left <= 0) continue;
            const long at = (long)m * g.N + n;
            if (left >= 4) {
                load_floats<4>(g.U + at, u[to][p]);
                load_floats<4>(g.V + at, v[to][p]);
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    u[to][p][q] = q < left ? g.U[at + q] : 0.f;
                    v[to][p][q] = q < left ? g.V[at + q] : 0.f;
                }
            }
        }
    };
    auto store = [&](auto* p, const float (&x)[4]) {
        if (left >= 4) store_floats<4>(p, x);
        else
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float one[1] = {x[q]};
                if (q < left) store_floats<1>(p + q, one);
            }
    };
    if constexpr (EPI == kGateGrad) load(0, 0);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        if constexpr (EPI == kGateGrad) {
            if (i + 1 < MT) load(i + 1, (i + 1) & 1);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) *reinterpret_cast<f32x4*>(mine + i16 * PITCH + (j * 16 + h * 4) * 4) = acc[i][j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");               // LDS serves a wave in order
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int row = p * ROWS + row0, m = m0 + i * 16 + row;
            float x[4];
            load_floats<4>(reinterpret_cast<const float*>(mine + row * PITCH) + col, x);
            float w[4];
            if constexpr (EPI == kGate) load_floats<4>(reinterpret_cast<const float*>(mine + row * PITCH) + COLS + col, w);
            if (m >= g.M || left <= 0) continue;
            const long at = (long)m * g.N + n;
            if constexpr (EPI == kStore) {
                store((batch ? g.C[1] : g.C[0]) + at, x);
            } else if constexpr (EPI == kGate) {
                if (g.U) {
                    store(g.U + at, x);
                    store(g.V + at, w);
                }
                act_values(g.act, x);
#pragma unroll
                for (int q = 0; q < 4; ++q) x[q] *= w[q];
                store(g.C[0] + at, x);
            } else {
                float (&uu)[4] = u[i & 1][p], (&vv)[4] = v[i & 1][p], slope[4];
                act_both(g.act, uu, slope);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    vv[q] *= x[q] * slope[q];
                    x[q] *= uu[q];
                }
                store(g.C[0] + at, vv);
                store(g.C[1] + at, x);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// A part of a sum: MT x NT fragments of a wave from row m0 on, the j-th at column(j) of the tile that begins at column n0
template <class T, int MT, int NT, int EPI, class F>
__device__ __forceinline__ void part_epilogue(const GemmArgs<T>& g, f32x4 (&acc)[MT][NT], int m0, int n0, int batch, F&& column)
{
    const int i16 = threadIdx.x & 15, h = (threadIdx.x & 63) >> 4;
    const long width = EPI == kGate ? 2L * g.N : g.N;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = m0 + i * 16 + i16;
        if (m >= g.M) continue;
        float* __restrict__ row = g.part + (((long)batch * g.splits + blockIdx.y) * g.M + m) * width;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const bool up = EPI == kGate && j >= NT / 2;
            const int n = n0 + column(up ? j - NT / 2 : j) + 4 * h, left = g.N - n;
            float* __restrict__ p = row + (up ? g.N : 0) + n;
            float x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = acc[i][j][q];
            if (left >= 4) store_floats<4>(p, x);
            else
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (q < left) p[q] = x[q];
        }
    }
}

// MT x NT fragments of 16 x 16 to a wave, WM x WN waves to a block
template <class T, int MT, int NT, int WM, int WN, int ALAY, int BLAY, int EPI>
__global__ __launch_bounds__(64 * WM * WN) void gated_gemm_kernel(GemmArgs<T> g)
{
    constexpr int THREADS = 64 * WM * WN;
    constexpr int BM = 16 * MT * WM, BN = 16 * NT * WN, HALF = BN / 2;
    typedef Tile<T, ALAY, BM> TA;
    typedef Tile<T, BLAY, BN> TB;
    constexpr int VEC = Mma<T>::VEC, BK = TA::BK;
    constexpr int ACHUNKS = TA::LINES * TA::CHUNKS, BCHUNKS = TB::LINES * TB::CHUNKS;
    constexpr int APER = (ACHUNKS + THREADS - 1) / THREADS, BPER = (BCHUNKS + THREADS - 1) / THREADS;   // of a thread
    __shared__ __attribute__((aligned(16))) char lds[2][TA::BYTES + TB::BYTES];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / WN, wn = wave % WN;
    constexpr int WIDTH = EPI == kGate ? HALF : BN;          // columns of the result in a block
    const int tiles_n = (g.N + WIDTH - 1) / WIDTH;
    const int bm = blockIdx.x / tiles_n, bn = blockIdx.x % tiles_n;
    const int m0 = bm * BM, n0 = bn * WIDTH, batch = blockIdx.z;
    const int tps = (g.K + BK - 1) / BK;                     // tiles of a segment
    const int t0 = blockIdx.y * g.per, t1 = min(t0 + g.per, tps * g.segments);
    const bool inside = m0 + BM <= g.M && n0 + WIDTH <= g.N;

    uint4 ra[APER], rb[BPER];
    // Tiles at an edge load from the nearest whole pieces, all in flight together; put() shifts what is there into place and
    // clears what lies past the end of the inner axis.  (Rows and columns past the result's are any: they are not stored.)
    // Lines shorter than a piece go element by element.
    const int a_line = ALAY == kInner ? g.K : g.M, b_line = BLAY == kInner ? g.K : g.N;
    const bool pieces = a_line >= VEC && b_line >= VEC;
    auto place = [&](int LAY, int q, int chunks, int o0, int k0, int* outer, int* inner) {
        const int line = q / chunks, at = q % chunks * VEC;
        *outer = o0 + (LAY == kInner ? line : at);
        *inner = k0 + (LAY == kInner ? at : line);
    };
    auto load = [&](int t) {
        const int seg = t / tps, k0 = (t - seg * tps) * BK;
        const T* __restrict__ A = seg ? g.A[1] : g.A[0];
        const T* __restrict__ B = seg + batch ? g.B[1] : g.B[0];
        // get(layout, operand, its distance of lines, outer and inner position, outer positions) for all pieces: one branch around
        // all loads and none between them, where the compiler would wait
        auto all = [&](auto&& get) {
#pragma unroll
            for (int i = 0; i < APER; ++i) {
                const int q = tid + THREADS * i;
                if (ACHUNKS % THREADS != 0 && q >= ACHUNKS) continue;
                int outer, inner;
                place(ALAY, q, TA::CHUNKS, m0, k0, &outer, &inner);
                ra[i] = get(ALAY, A, g.lda, outer, inner, g.M);
            }
#pragma unroll
            for (int i = 0; i < BPER; ++i) {
                const int q = tid + THREADS * i;
                if (BCHUNKS % THREADS != 0 && q >= BCHUNKS) continue;
                int outer, inner;
                place(BLAY, q, TB::CHUNKS, 0, k0, &outer, &inner);
                const bool up = EPI == kGate && outer >= HALF;
                rb[i] = get(BLAY, up ? g.B[1] : B, g.ldb, n0 + outer - (up ? HALF : 0), inner, g.N);
            }
        };
        auto at = [&](int LAY, const T* W, long ld, int outer, int inner) {
            return LAY == kInner ? W + (long)outer * ld + inner : W + (long)inner * ld + outer;
        };
        if (inside && k0 + BK <= g.K)
            all([&](int LAY, const T* W, long ld, int outer, int inner, int) { return whole_chunk(at(LAY, W, ld, outer, inner)); });
        else if (pieces)
            all([&](int LAY, const T* W, long ld, int outer, int inner, int outers) {
                outer = min(outer, LAY == kInner ? outers - 1 : outers - VEC);
                inner = min(inner, LAY == kInner ? g.K - VEC : g.K - 1);
                return whole_chunk(at(LAY, W, ld, outer, inner));
            });
        else
            all([&](int LAY, const T* W, long ld, int outer, int inner, int outers) {
                const int left = LAY == kInner ? (outer < outers ? g.K - inner : 0) : (inner < g.K ? outers - outer : 0);
                return edge_chunk(at(LAY, W, ld, outer, inner), left);
            });
    };
    auto put = [&](int t, char* buf) {
        const int k0 = t % tps * BK;
        const bool fix = pieces && !(inside && k0 + BK <= g.K);
        auto fixed = [&](int LAY, uint4 x, int outer, int inner, int outers) {
            const int past = LAY == kInner ? inner - (g.K - VEC) : outer - (outers - VEC);      // elements of the piece past the end
            if (past > 0) {
                unsigned __int128 v;
                __builtin_memcpy(&v, &x, 16);
                v = past >= VEC ? 0 : v >> (past * (int)sizeof(T) * 8);
                __builtin_memcpy(&x, &v, 16);
            }
            if (LAY == kOuter && inner >= g.K) x = make_uint4(0, 0, 0, 0);
            return x;
        };
        if (fix) {
#pragma unroll
            for (int i = 0; i < APER; ++i) {
                int outer, inner;
                place(ALAY, tid + THREADS * i, TA::CHUNKS, m0, k0, &outer, &inner);
                ra[i] = fixed(ALAY, ra[i], outer, inner, g.M);
            }
#pragma unroll
            for (int i = 0; i < BPER; ++i) {
                int outer, inner;
                place(BLAY, tid + THREADS * i, TB::CHUNKS, 0, k0, &outer, &inner);
                rb[i] = fixed(BLAY, rb[i], n0 + outer - (EPI == kGate && outer >= HALF ? HALF : 0), inner, g.N);
            }
        }
#pragma unroll
        for (int i = 0; i < APER; ++i) {
            const int q = tid + THREADS * i;
            if (ACHUNKS % THREADS != 0 && q >= ACHUNKS) continue;
            *reinterpret_cast<uint4*>(buf + q / TA::CHUNKS * TA::PITCH + q % TA::CHUNKS * 16) = ra[i];
        }
#pragma unroll
        for (int i = 0; i < BPER; ++i) {
            const int q = tid + THREADS * i;
            if (BCHUNKS % THREADS != 0 && q >= BCHUNKS) continue;
            *reinterpret_cast<uint4*>(buf + TA::BYTES + q / TB::CHUNKS * TB::PITCH + q % TB::CHUNKS * 16) = rb[i];
        }
    };
    // first column of the wave's j-th fragment in the tile; kGate: the first half of them from Wg, the others from Wu
    auto column = [&](int j) {
        return EPI == kGate ? (j < NT / 2 ? wn * (NT / 2) * 16 + j * 16 : HALF + wn * (NT / 2) * 16 + (j - NT / 2) * 16)
                            : wn * NT * 16 + j * 16;
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    if (t0 < t1) {
        load(t0);
        put(t0, lds[0]);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const char* buf = lds[(t - t0) & 1];
        if (t + 1 < t1) load(t + 1);
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            typename Mma<T>::Frag a[MT], b[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i) a[i] = TA::frag(buf, wm * MT * 16 + i * 16, step);
#pragma unroll
            for (int j = 0; j < NT; ++j) b[j] = TB::frag(buf + TA::BYTES, column(j), step);
            // columns as the first operand: a lane's four results are neighbours in a row
#pragma unroll
            for (int k = 0; k < Mma<T>::TURNS; ++k)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = Mma<T>::mul(b[j], a[i], acc[i][j], k);
        }
        if (t + 1 < t1) put(t + 1, lds[(t + 1 - t0) & 1]);
        __syncthreads();
    }

    if (g.splits > 1) {
        part_epilogue<T, MT, NT, EPI>(g, acc, m0 + wm * MT * 16, n0, batch, column);
    } else {
        constexpr int MINE = 16 * (NT * 16 + 4) * 4;         // 16 rows of a wave
        static_assert(MINE * WM * WN <= sizeof(lds), "all waves' rows");
        line_epilogue<T, MT, NT, EPI>(g, acc, lds[0] + wave * MINE, m0 + wm * MT * 16, n0 + column(0), batch);
    }
}

// Sums the parts of a product and does what its epilogue would have done; a thread owns one number.
template <class T, int EPI>
__global__ __launch_bounds__(256) void gated_join_kernel(GemmArgs<T> g)
{
    const long total = (long)g.M * g.N, width = EPI == kGate ? 2L * g.N : g.N;
    const int batch = blockIdx.z;
    for (long at = (long)blockIdx.x * 256 + threadIdx.x; at < total; at += (long)gridDim.x * 256) {
        const long m = at / g.N, n = at % g.N, plane = (long)g.M * width;
        const float* __restrict__ p = g.part + (long)batch * g.splits * plane + m * width + n;
        float x = 0.f, v = 0.f;
        constexpr int U = 4;
        int s = 0;
        float ax[U] = {}, av[U] = {};
        for (; s + U <= g.splits; s += U)
#pragma unroll
            for (int k = 0; k < U; ++k) {
                ax[k] += p[(s + k) * plane];
                if constexpr (EPI == kGate) av[k] += p[(s + k) * plane + g.N];
            }
        for (; s < g.splits; ++s) {
            ax[0] += p[s * plane];
            if constexpr (EPI == kGate) av[0] += p[s * plane + g.N];
        }
        x = (ax[0] + ax[1]) + (ax[2] + ax[3]);
        v = (av[0] + av[1]) + (av[2] + av[3]);
        if constexpr (EPI == kStore) {
            const float one[1] = {x};
            store_floats<1>((batch ? g.C[1] : g.C[0]) + at, one);
        } else if constexpr (EPI == kGate) {
            if (g.U) { g.U[at] = x; g.V[at] = v; }
            float one[1] = {x};
            act_values(g.act, one);
            one[0] *= v;
            store_floats<1>(g.C[0] + at, one);
        } else {
            float u[1] = {g.U[at]}, slope[1];
            act_both(g.act, u, slope);
            const float du[1] = {x * g.V[at] * slope[0]}, dv[1] = {x * u[0]};
            store_floats<1>(g.C[0] + at, du);
            store_floats<1>(g.C[1] + at, dv);
        }
    }
}

}  // namespace daspmm
