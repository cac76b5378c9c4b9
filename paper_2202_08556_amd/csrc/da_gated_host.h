// Products of the gated feed-forward block: operands and launches (da_gated_plan.h cuts them).  Included by one translation unit for
// each type.
#pragma once
#include "da_gated.h"
#include "da_gated_kernels.hip"
#include "da_gated_rows.hip"
#include "da_gated_tiles.hip"
#include "da_gated_plan.h"
#include "da_internal.h"

#include <algorithm>
#include <atomic>
#include <type_traits>

namespace daspmm {
namespace {

// Whether the tiles of 256 x 256 take a product: their loads are of 16 bytes at addresses that are multiples of it
template <int ALAY, int BLAY> bool wide_takes(const GemmArgs<bf16>& g) {
    auto whole = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
    return g.lda % 8 == 0 && g.ldb % 8 == 0 && g.lda < (1 << 22) && g.ldb < (1 << 22) && whole(g.A[0]) && whole(g.A[1]) &&
           whole(g.B[0]) && whole(g.B[1]) && (ALAY == kInner || g.M % 8 == 0) && (BLAY == kInner || g.N % 8 == 0);
}

template <class T, int EPI> void join_parts(const GemmArgs<T>& g, int batches, hipStream_t s) {
    if (g.splits == 1) return;
    const int64_t blocks = std::min<int64_t>(ceil_div((int64_t)g.M * g.N, 256), 16384);
    hipLaunchKernelGGL((gated_join_kernel<T, EPI>), dim3((unsigned)blocks, 1, (unsigned)batches), dim3(256), 0, s, g);
}

template <int ROWS, int STEP, int STAGES, int ALAY, int BLAY, int EPI>
void wide_gemm(GemmArgs<bf16> g, int batches, int splits, hipStream_t s) {
    typedef WideShape<ROWS, STEP, STAGES> S;
    const int64_t width = EPI == kGate ? 2 * (int64_t)g.N : g.N, inner = ceil_div(g.K, STEP) * g.segments;
    g.per = (int)std::max<int64_t>(1, ceil_div(inner, splits));
    g.splits = (int)std::max<int64_t>(1, ceil_div(inner, g.per));
    auto kernel = gated_wide_kernel<ROWS, STEP, STAGES, ALAY, BLAY, EPI>;
    static std::atomic<uint64_t> allowed{0};                 // devices that know how much LDS the kernel takes
    int device = 0;
    (void)hipGetDevice(&device);
    const uint64_t bit = 1ull << (device & 63);
    if (!(allowed.load(std::memory_order_relaxed) & bit) &&
        hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS) == hipSuccess)
        allowed.fetch_or(bit, std::memory_order_relaxed);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(ceil_div(g.M, ROWS) * ceil_div(width, kWideColumns)), (unsigned)g.splits, (unsigned)batches),
                       dim3(S::THREADS), S::LDS, s, g);
    join_parts<bf16, EPI>(g, batches, s);
}

// `part` holds what part_bytes() says of the product
template <class T, int ALAY, int BLAY, int EPI>
void gemm(GemmArgs<T> g, const Product& product, float* part, hipStream_t s) {
    if (product.M == 0 || product.N == 0) return;
    const int batches = product.batches;
    g.M = (int)product.M;
    g.N = (int)product.N;
    g.K = (int)product.K;
    g.segments = product.segments;
    g.part = part;
    if constexpr (std::is_same_v<T, bf16>) {
        const WidePlan w = wide_plan(product);
        if (w.rows && wide_takes<ALAY, BLAY>(g)) {
            if (w.rows == 256) return wide_gemm<256, 64, 2, ALAY, BLAY, EPI>(g, batches, 1, s);
            return wide_gemm<128, 32, 3, ALAY, BLAY, EPI>(g, batches, w.splits, s);
        }
    }
    const GemmPlan p = gemm_plan(product, sizeof(T));
    g.splits = p.splits;
    g.per = p.per;
    const int64_t width = EPI == kGate ? 2 * (int64_t)g.N : g.N;
    const dim3 grid((unsigned)(ceil_div(g.M, p.BM) * ceil_div(width, p.BN)), (unsigned)p.splits, (unsigned)batches);
    auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, g); };
    if (p.BM == 128 && p.BN == 128) go(gated_gemm_kernel<T, 2, 4, 4, 2, ALAY, BLAY, EPI>, 512);
    else if (p.BM == 64 && p.BN == 64) go(gated_gemm_kernel<T, 2, 2, 2, 2, ALAY, BLAY, EPI>, 256);
    else if (p.BM == 16) go(gated_gemm_kernel<T, 1, 2, 1, 4, ALAY, BLAY, EPI>, 256);
    else if (p.BM == 32) go(gated_gemm_kernel<T, 2, 2, 1, 4, ALAY, BLAY, EPI>, 256);
    else if (p.BM == 64) go(gated_gemm_kernel<T, 4, 2, 1, 4, ALAY, BLAY, EPI>, 256);
    if constexpr (EPI != kGate) {
        if (p.BM == 128 && p.BN == 64) go(gated_gemm_kernel<T, 2, 4, 4, 1, ALAY, BLAY, EPI>, 256);
    }
    join_parts<T, EPI>(g, batches, s);
}

// Few rows, forward
struct RowsPlan {
    int LN, splits, per;
    int64_t columns;             // blocks along the columns
};

// Four waves of eight lines each keep a compute unit's share of memory busy: six blocks a unit, no fewer than 32 lines to one.
template <class T> RowsPlan rows_plan(int64_t N, int64_t K) {
    RowsPlan p{};
    const int64_t pieces = ceil_div(N, Mma<T>::VEC);
    p.LN = 1;
    while (p.LN < kRowsBlock && p.LN < pieces) p.LN *= 2;
    if (p.LN > 64) p.LN = 64;                                // a wave a line: 1 KB
    p.columns = std::max<int64_t>(1, ceil_div(pieces, p.LN));
    const int64_t lines = 32 * (kRowsBlock / p.LN) / 4;      // as many blocks' worth for each of the threads along the lines
    int64_t splits = std::min(ceil_div(6 * compute_units(), p.columns), ceil_div(K, std::max<int64_t>(lines, 32)));
    splits = std::min<int64_t>(std::max<int64_t>(splits, 1), 65535);
    p.per = (int)std::max<int64_t>(1, ceil_div(K, splits));
    p.splits = (int)std::max<int64_t>(1, ceil_div(K, p.per));
    return p;
}

template <class T> size_t rows_part_bytes(const GatedShape& s) {
    const RowsPlan a = rows_plan<T>(s.h, s.d), b = rows_plan<T>(s.dout, s.h);
    const size_t u = a.splits > 1 ? (size_t)(a.splits * s.rows * s.h * 2) : 0, y = b.splits > 1 ? (size_t)(b.splits * s.rows * s.dout) : 0;
    return round16(std::max(u, y) * sizeof(float));
}

template <class T, class TX, int EPI> void rows_product(RowsArgs<T> g, const TX* x, int64_t ldx, hipStream_t s) {
    if (g.N == 0) return;
    const RowsPlan p = rows_plan<T>(g.N, g.K);
    g.LN = p.LN;
    g.splits = p.splits;
    g.per = p.per;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)p.columns, (unsigned)p.splits), dim3(kRowsBlock), 0, s, g, x, (long)ldx);
    };
    if (g.rows == 1) go(gated_rows_kernel<T, TX, 1, EPI>);
    else if (g.rows == 2) go(gated_rows_kernel<T, TX, 2, EPI>);
    else if (g.rows <= 4) go(gated_rows_kernel<T, TX, 4, EPI>);
    else go(gated_rows_kernel<T, TX, 8, EPI>);
    if (p.splits > 1)
        hipLaunchKernelGGL((gated_rows_join_kernel<T, EPI>), dim3((unsigned)ceil_div(g.N, 64), (unsigned)g.rows), dim3(kRowsBlock), 0, s, g);
}

}  // namespace

template <class T> size_t gated_forward_bytes(const GatedShape& s) {
    if (s.rows <= kRowsMost) return rows_part_bytes<T>(s) + round16((size_t)(s.rows * s.h) * sizeof(float));
    return std::max(part_bytes(gate_product(s), sizeof(T)), part_bytes(down_product(s), sizeof(T)));
}

template <class T> size_t gated_backward_bytes(const GatedShape& s) {
    return 2 * round16((size_t)(s.rows * s.h) * sizeof(T)) + backward_part_bytes(s, sizeof(T));
}

template <class T> void gated_forward(const GatedCall& c) {
    const int rows = (int)c.s.rows, d = (int)c.s.d, h = (int)c.s.h, dout = (int)c.s.dout;
    if (rows <= kRowsMost) {
        RowsArgs<T> r{};
        float* a32 = reinterpret_cast<float*>(c.workspace + rows_part_bytes<T>(c.s));
        r.W0 = static_cast<const T*>(c.wg);
        r.W1 = static_cast<const T*>(c.wu);
        r.rows = rows;
        r.N = h;
        r.K = d;
        r.part = reinterpret_cast<float*>(c.workspace);
        r.A32 = a32;
        r.C = c.u ? static_cast<T*>(c.a) : nullptr;          // only a backward pass reads it
        r.U = c.u;
        r.V = c.v;
        r.act = c.act;
        rows_product<T, T, kGate>(r, static_cast<const T*>(c.x), c.ldx, c.stream);
        r = RowsArgs<T>{};
        r.W0 = static_cast<const T*>(c.wd);
        r.rows = rows;
        r.N = dout;
        r.K = h;
        r.part = reinterpret_cast<float*>(c.workspace);
        r.C = static_cast<T*>(c.y);
        rows_product<T, float, kStore>(r, a32, h, c.stream);
        return;
    }
    float* part = reinterpret_cast<float*>(c.workspace);
    GemmArgs<T> g{};
    g.A[0] = g.A[1] = static_cast<const T*>(c.x);
    g.B[0] = static_cast<const T*>(c.wg);
    g.B[1] = static_cast<const T*>(c.wu);
    g.lda = c.ldx;
    g.ldb = h;
    g.C[0] = static_cast<T*>(c.a);
    g.U = c.u;
    g.V = c.v;
    g.act = c.act;
    gemm<T, kInner, kOuter, kGate>(g, gate_product(c.s), part, c.stream);

    g = GemmArgs<T>{};
    g.A[0] = g.A[1] = static_cast<const T*>(c.a);
    g.B[0] = g.B[1] = static_cast<const T*>(c.wd);
    g.lda = h;
    g.ldb = dout;
    g.C[0] = static_cast<T*>(c.y);
    gemm<T, kInner, kOuter, kStore>(g, down_product(c.s), part, c.stream);
}

template <class T> void gated_backward(const GatedCall& c) {
    const int h = (int)c.s.h, dout = (int)c.s.dout;
    const size_t hidden = round16((size_t)(c.s.rows * c.s.h) * sizeof(T));
    T* du = reinterpret_cast<T*>(c.workspace);
    T* dv = reinterpret_cast<T*>(c.workspace + hidden);
    float* part = reinterpret_cast<float*>(c.workspace + 2 * hidden);
    GemmArgs<T> g{};
    if (c.dx || c.dwg || c.dwu) {
        g.A[0] = g.A[1] = static_cast<const T*>(c.dy);
        g.B[0] = g.B[1] = static_cast<const T*>(c.wd);
        g.lda = c.ldy;
        g.ldb = dout;
        g.C[0] = du;
        g.C[1] = dv;
        g.U = c.u;
        g.V = c.v;
        g.act = c.act;
        gemm<T, kInner, kInner, kGateGrad>(g, hidden_grad_product(c.s), part, c.stream);
    }
    if (c.dx) {
        g = GemmArgs<T>{};
        g.A[0] = du;
        g.A[1] = dv;
        g.B[0] = static_cast<const T*>(c.wg);
        g.B[1] = static_cast<const T*>(c.wu);
        g.lda = h;
        g.ldb = h;
        g.C[0] = static_cast<T*>(c.dx);
        gemm<T, kInner, kInner, kStore>(g, input_grad_product(c.s), part, c.stream);
    }
    if (c.dwg || c.dwu) {
        const int first = c.dwg ? 0 : 1, batches = c.dwg && c.dwu ? 2 : 1;
        T* const of[2] = {du, dv};
        void* const to[2] = {c.dwg, c.dwu};
        g = GemmArgs<T>{};
        g.A[0] = g.A[1] = static_cast<const T*>(c.x);
        g.B[0] = of[first];
        g.B[1] = dv;
        g.lda = c.ldx;
        g.ldb = h;
        g.C[0] = static_cast<T*>(to[first]);
        g.C[1] = static_cast<T*>(c.dwu);
        gemm<T, kOuter, kOuter, kStore>(g, up_grad_product(c.s, batches), part, c.stream);
    }
    if (c.dwd) {
        g = GemmArgs<T>{};
        g.A[0] = g.A[1] = static_cast<const T*>(c.a);
        g.B[0] = g.B[1] = static_cast<const T*>(c.dy);
        g.lda = h;
        g.ldb = c.ldy;
        g.C[0] = static_cast<T*>(c.dwd);
        gemm<T, kOuter, kOuter, kStore>(g, down_grad_product(c.s), part, c.stream);
    }
}

}  // namespace daspmm
