// Orthogonalised updates by Newton-Schulz steps, X <- a X + (b A + c A^2) X with A = X X^T, on the matrix cores.
//
// All products are of pairs of fp16 halves (da_planes.h): a step multiplies errors of the small singular values by up to
// a, like the values themselves, so what is kept between products keeps 22 bits; bf16 or single fp16 numbers there would be
// off by 1e-2 and 3e-3 of the result where rounding it to bf16 costs 1.7e-3.  That holds for bfloat16, too, from the first step on: with first
// halves there, and X's alone in its product with b A + c A^2, random matrices came out within 1.2 times the rounding, but those of
// numbers of one magnitude, whose roundings are all alike, off by up to 5e-3.
// X is held with the shorter side as rows (a tall matrix is turned around on its way in and out).  A and A^2 are symmetric:
// only tiles on and above the diagonal are computed, and each is written to both of its places.
// 2048 x 8192 bf16, five steps: 1600 us; a step's products 106, 51 and 174.  1187 x 602 float32: 175, of which a kernel's start, its
// first loads from what another die's cache wrote, and its end are some 5 of each launch's 11.
// The scales of X, A and b A + c A^2 follow from how large singular values can be: at most 1 at first (the Frobenius norm
// bounds them), then by the polynomial's extremes, which the host takes.
#include "da_training.h"

#include "da_orth_small.h"
#include "da_planes_host.h"
#include "da_spmm.h"

#include <cmath>

namespace daspmm {
namespace {

constexpr int kNormParts = 512;              // of the norm's sum to a matrix
constexpr int kOrthMost = 1 << 17;

// Sums of squares in 64 bits: the squares of floats neither overflow nor vanish there
template <class T>
__global__ __launch_bounds__(256) void orth_norm_kernel(const T* __restrict__ g, long ldg, long stride, long rows, long cols,
                                                        double* __restrict__ part, int* __restrict__ arrived)
{
    __shared__ double red[4];
    const T* __restrict__ p = g + blockIdx.y * stride;
    if (arrived && blockIdx.x == 0 && blockIdx.y == 0)
        for (int k = threadIdx.x; k < kMostParted; k += 256) arrived[k] = 0;
    // pieces of 1024 columns of a row, a wave's turn each, dealt to all waves of the matrix
    const long across = (cols + 1023) / 1024, all = rows * across, step = (long)gridDim.x * 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double s = 0.0;
    for (long k = (long)blockIdx.x * 4 + wave; k < all; k += step) {
        const long r = k / across, c0 = k % across * 1024;
        const T* __restrict__ row = p + r * ldg;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const long c = c0 + e * 256 + lane * 4;
            float x[4] = {0.f, 0.f, 0.f, 0.f};
            if (c + 4 <= cols) {
                load_floats<4>(row + c, x);
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (c + i < cols) {
                        float one[1];
                        load_floats<1>(row + c + i, one);
                        x[i] = one[0];
                    }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s += (double)x[i] * (double)x[i];
        }
    }
    s = wave_sum(s, 64);
    if (lane == 0) red[wave] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[(long)blockIdx.y * gridDim.x + blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// A tile of 64 x 64 of the packed X = scale g / (|g| + eps), turned around if `tall`
template <class T>
__global__ __launch_bounds__(256) void orth_pack_kernel(const T* __restrict__ g, long ldg, long stride, int rows, int cols, int tall,
                                                        const double* __restrict__ part, int parts, float eps, float scale,
                                                        uint16_t* __restrict__ X, Packed lx, long batch_x)
{
    __shared__ float tile[64][65];
    __shared__ double by;
    const int tid = threadIdx.x;
    if (tid < 64) {
        double s = 0.0;
        for (int k = tid; k < parts; k += 64) s += part[(long)blockIdx.z * parts + k];
        s = wave_sum(s, 64);
        if (tid == 0) by = (double)scale / (sqrt(s) + (double)eps);
    }
    __syncthreads();
    const double f = by;
    const T* __restrict__ p = g + blockIdx.z * stride;
    const int r0 = (tall ? blockIdx.x : blockIdx.y) * 64, c0 = (tall ? blockIdx.y : blockIdx.x) * 64;    // of g
    for (int k = tid; k < 1024; k += 256) {                  // four neighbours in a row of g each
        const int r = r0 + k / 16, c = c0 + k % 16 * 4;
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        if (r < rows) {
            const T* __restrict__ q = p + (long)r * ldg + c;
            if (c + 4 <= cols) {
                load_floats<4>(q, x);
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (c + i < cols) {
                        float one[1];
                        load_floats<1>(q + i, one);
                        x[i] = one[0];
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) tile[k / 16][k % 16 * 4 + i] = (float)((double)x[i] * f);
    }
    __syncthreads();
    uint16_t* __restrict__ out = X + blockIdx.z * batch_x;
    for (int k = tid; k < 1024; k += 256) {
        const int line = k / 16, at = k % 16 * 4;
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = tall ? tile[at + i][line] : tile[line][at + i];
        put_values<Halves, 4>(out + place<Halves>(lx, blockIdx.y * 64 + line, blockIdx.x * 64 + at), x);
    }
}

// The result of a tall matrix: X^T / scale
template <class T>
__global__ __launch_bounds__(256) void orth_turn_kernel(const uint16_t* __restrict__ X, Packed lx, long batch_x, int rows, int cols, float inv,
                                                        T* __restrict__ out)
{
    __shared__ float tile[64][65];
    const int tid = threadIdx.x;
    const uint16_t* __restrict__ in = X + blockIdx.z * batch_x;
    for (int k = tid; k < 1024; k += 256) {
        const int line = k / 16, at = k % 16 * 4;
        float x[4];
        get_values<Halves, 4>(in + place<Halves>(lx, blockIdx.y * 64 + line, blockIdx.x * 64 + at), x);
#pragma unroll
        for (int i = 0; i < 4; ++i) tile[line][at + i] = x[i] * inv;
    }
    __syncthreads();
    T* __restrict__ o = out + (long)blockIdx.z * rows * cols;
    for (int k = tid; k < 4096; k += 256) {
        const int r = blockIdx.x * 64 + k / 64, c = blockIdx.y * 64 + k % 64;
        const float one[1] = {tile[k % 64][k / 64]};
        if (r < rows && c < cols) store_floats<1>(o + (long)r * cols + c, one);
    }
}

// A = X X^T
struct GramOut {
    static constexpr bool kSymmetric = true, kWhole = false;
    uint16_t* A;
    Packed la;
    long batch_a;
    float by;                    // of the product to A's scale
    __device__ __forceinline__ NoColumn column(int) const { return {}; }
    __device__ __forceinline__ void four(int m, int n, float (&x)[4], int batch, NoColumn) const {
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] *= by;
        put_values<Halves, 4>(A + batch * batch_a + place<Halves>(la, m, n), x);
    }
};
// b A + c A^2
struct PolyOut : GramOut {
    const uint16_t* from;        // A, laid out like the result
    float b, c;                  // with the scales
    __device__ __forceinline__ void four(int m, int n, float (&x)[4], int batch, NoColumn) const {
        float a[4];
        get_values<Halves, 4>(from + batch * batch_a + place<Halves>(la, m, n), a);
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] = b * a[q] + c * x[q];
        put_values<Halves, 4>(A + batch * batch_a + place<Halves>(la, m, n), x);
    }
};
// a X + (b A + c A^2) X, packed
struct StepOut {
    static constexpr bool kSymmetric = false, kWhole = false;
    const uint16_t* from;
    uint16_t* to;
    Packed lx;
    long batch_x;
    float a, by;                 // with the scales
    __device__ __forceinline__ NoColumn column(int) const { return {}; }
    __device__ __forceinline__ void value(int m, int n, float (&x)[4], int batch) const {
        float old[4];
        get_values<Halves, 4>(from + batch * batch_x + place<Halves>(lx, m, n), old);
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] = a * old[q] + by * x[q];
    }
    __device__ __forceinline__ void four(int m, int n, float (&x)[4], int batch, NoColumn) const {
        value(m, n, x, batch);
        put_values<Halves, 4>(to + batch * batch_x + place<Halves>(lx, m, n), x);
    }
};
// ... as the result
template <class T> struct LastOut : StepOut {
    T* out;
    int rows, cols;
    __device__ __forceinline__ void four(int m, int n, float (&x)[4], int batch, NoColumn) const {
        if (m >= rows || n >= cols) return;
        value(m, n, x, batch);
        T* __restrict__ p = out + (long)batch * rows * cols + (long)m * cols + n;
        if (n + 4 <= cols) {
            store_floats<4>(p, x);
        } else {
#pragma unroll
            for (int q = 0; q < 3; ++q) {
                const float one[1] = {x[q]};
                if (n + q < cols) store_floats<1>(p + q, one);
            }
        }
    }
};

// No steps: g / (|g| + eps)
template <class T>
__global__ __launch_bounds__(256) void orth_scale_kernel(const T* __restrict__ g, long ldg, long stride, long rows, long cols,
                                                         const double* __restrict__ part, int parts, float eps, T* __restrict__ out)
{
    __shared__ double by;
    if (threadIdx.x < 64) {
        double s = 0.0;
        for (int k = threadIdx.x; k < parts; k += 64) s += part[(long)blockIdx.y * parts + k];
        s = wave_sum(s, 64);
        if (threadIdx.x == 0) by = 1.0 / (sqrt(s) + (double)eps);
    }
    __syncthreads();
    for (long at = (long)blockIdx.x * 256 + threadIdx.x; at < rows * cols; at += (long)gridDim.x * 256) {
        float x[1];
        load_floats<1>(g + blockIdx.y * stride + at / cols * ldg + at % cols, x);
        x[0] = (float)((double)x[0] * by);
        store_floats<1>(out + blockIdx.y * rows * cols + at, x);
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

struct OrthPlan {
    int64_t m, n, Ma, Nb;        // shorter and longer side, padded
    int parts;                   // of a norm
    PlanePlan gram, poly, step;
    size_t X, A, part;           // bytes
    size_t bytes() const { return round16((size_t)parts_bytes) + kMostParted * sizeof(int) + 2 * X + 2 * A + part; }
    size_t parts_bytes;
};

OrthPlan make_orth_plan(int64_t batch, int64_t rows, int64_t cols) {
    OrthPlan p{};
    p.m = std::min(rows, cols);
    p.n = std::max(rows, cols);
    p.Ma = padded(p.m);
    p.Nb = padded(p.n);
    p.parts = (int)std::max<int64_t>(1, std::min<int64_t>(kNormParts, ceil_div(rows * cols, 8192)));
    p.parts_bytes = (size_t)batch * p.parts * sizeof(double);
    const int64_t step = Halves::STEP;
    p.gram = plane_plan(p.Ma, p.Ma, p.Nb / step, batch, true, true, 1);
    p.poly = plane_plan(p.Ma, p.Ma, p.Ma / step, batch, true, true, 1);
    p.step = plane_plan(p.Ma, p.Nb, p.Ma / step, batch, false, true, 1);
    p.X = (size_t)batch * p.Ma * p.Nb * 4;
    p.A = (size_t)batch * p.Ma * p.Ma * 4;
    p.part = std::max({plane_part_bytes(p.gram, batch), plane_part_bytes(p.poly, batch), plane_part_bytes(p.step, batch)});
    return p;
}

// A call asks for its plan twice, and a program for the same one in every step
const OrthPlan& orth_plan(int64_t batch, int64_t rows, int64_t cols) {
    struct Last {
        int units = 0;
        int64_t batch = -1, rows = 0, cols = 0;
        OrthPlan p{};
    };
    thread_local Last last;
    const int units = compute_units();
    if (last.units != units || last.batch != batch || last.rows != rows || last.cols != cols) {
        last.p = make_orth_plan(batch, rows, cols);
        last.batch = batch;
        last.rows = rows;
        last.cols = cols;
        last.units = units;
    }
    return last.p;
}

int orth_check(int dtype, int64_t batch, int64_t rows, int64_t cols, int steps) {
    if (dtype != DA_F32 && dtype != DA_BF16) return fail(DA_ERR_UNSUPPORTED, "dtype is neither DA_F32 nor DA_BF16");
    if (batch < 0 || rows < 0 || cols < 0 || steps < 0) return fail(DA_ERR_INVALID_ARG, "negative size");
    if (rows > kOrthMost || cols > kOrthMost || batch > 65535 || steps > 64) return fail(DA_ERR_UNSUPPORTED, "size too large");
    if (batch * ceil_div(rows, 64) * ceil_div(cols, 64) >= 1LL << 30) return fail(DA_ERR_UNSUPPORTED, "size too large");
    return DA_OK;
}

// Powers of two: bound * the result <= 2^14
float scale_for(double bound) {
    int e = 0;
    std::frexp(std::max(bound, 1e-6), &e);                   // bound <= 2^e
    return (float)std::ldexp(1.0, 14 - e);
}

struct StepScales {
    float X, A, B;
};
// The scales of each step; false where values could leave what is supported.  Extremes on 1025 points of [0, most] are
// within 1e-3 of the polynomial's own; scale_for leaves a factor of four.
bool orth_scales(int steps, const float* c, StepScales* s) {
    double most = 1.0;
    for (int k = 0; k < steps; ++k) {
        const double p = c[3 * k], q = c[3 * k + 1], r = c[3 * k + 2];
        if (!std::isfinite(p) || !std::isfinite(q) || !std::isfinite(r)) return false;
        double next = 0.0, poly = 0.0;
        for (int i = 0; i <= 1024; ++i) {
            const double x = most * i / 1024.0, l = x * x, b = q * l + r * l * l;
            poly = std::max(poly, std::fabs(b));
            next = std::max(next, std::fabs(p * x + b * x));
        }
        s[k] = {scale_for(most), scale_for(most * most), scale_for(poly)};
        if (poly > 4096.0 || next > 128.0) return false;
        most = std::max(next * 1.01, 1e-3);
    }
    s[steps] = {scale_for(most), 1.f, 1.f};
    return true;
}

bool small_takes(int64_t rows, int64_t cols) { return std::min(rows, cols) <= kSmallSide && std::max(rows, cols) <= kSmallLong; }

template <class T>
void orthogonalise_small(int64_t batch, int64_t rows, int64_t cols, const T* g, int64_t ldg, int64_t stride, int steps, const float* c, float eps,
                         T* out, const StepScales* scales, hipStream_t s) {
    SmallArgs a{};
    a.ldg = ldg;
    a.stride = stride;
    a.rows = (int)rows;
    a.cols = (int)cols;
    a.steps = steps;
    a.eps = eps;
    a.first = scales[0].X;
    a.last = 1.f / scales[steps].X;
    for (int k = 0; k < steps; ++k) {
        const float sx = scales[k].X, sa = scales[k].A, sb = scales[k].B, to = scales[k + 1].X;
        a.step[k] = {sa / (sx * sx), c[3 * k + 1] * sb / sa, c[3 * k + 2] * sb / (sa * sa), c[3 * k] * to / sx, to / (sb * sx)};
    }
    const int n = (int)padded(std::max(rows, cols));
    constexpr auto kernel = orth_small_kernel<T>;
    allow_lds<kernel>((int)small_lds(kSmallLong));
    hipLaunchKernelGGL(kernel, dim3((unsigned)batch), dim3(kSmallThreads), small_lds(n), s, g, out, a, n);
}

template <class T>
void orthogonalise(int64_t batch, int64_t rows, int64_t cols, const T* g, int64_t ldg, int64_t stride, int steps, const float* c, float eps,
                   T* out, char* ws, const OrthPlan& p, const StepScales* scales, hipStream_t s) {
    double* norm = reinterpret_cast<double*>(ws);
    ws += round16(p.parts_bytes);
    int* arrived = steps ? reinterpret_cast<int*>(ws) : nullptr;
    ws += kMostParted * sizeof(int);
    uint16_t* X = reinterpret_cast<uint16_t*>(ws);
    uint16_t* Y = reinterpret_cast<uint16_t*>(ws + p.X);
    uint16_t* A = reinterpret_cast<uint16_t*>(ws + 2 * p.X);
    uint16_t* B = reinterpret_cast<uint16_t*>(ws + 2 * p.X + p.A);
    float* part = reinterpret_cast<float*>(ws + 2 * p.X + 2 * p.A);
    const bool tall = rows > cols;
    if (small_takes(rows, cols)) return orthogonalise_small<T>(batch, rows, cols, g, ldg, stride, steps, c, eps, out, scales, s);
    hipLaunchKernelGGL((orth_norm_kernel<T>), dim3((unsigned)p.parts, (unsigned)batch), dim3(256), 0, s, g, (long)ldg, (long)stride,
                       (long)rows, (long)cols, norm, arrived);
    if (steps == 0) {
        hipLaunchKernelGGL((orth_scale_kernel<T>), dim3((unsigned)std::min<int64_t>(ceil_div(rows * cols, 256), 2048), (unsigned)batch),
                           dim3(256), 0, s, g, (long)ldg, (long)stride, (long)rows, (long)cols, norm, p.parts, eps, out);
        return;
    }
    const Packed lx = packed(p.Ma, p.Nb, 2), la = packed(p.Ma, p.Ma, 2);
    const long bx = p.Ma * p.Nb * 2, ba = p.Ma * p.Ma * 2;
    hipLaunchKernelGGL((orth_pack_kernel<T>), dim3((unsigned)(p.Nb / 64), (unsigned)(p.Ma / 64), (unsigned)batch), dim3(256), 0, s, g,
                       (long)ldg, (long)stride, (int)rows, (int)cols, (int)tall, norm, p.parts, eps, scales[0].X, X, lx, bx);
    PlaneArgs gram{}, poly{}, step{};
    gram.a = gram.b = step.b = lx;
    gram.batch_a = gram.batch_b = step.batch_b = bx;
    poly.a = poly.b = step.a = la;
    poly.batch_a = poly.batch_b = step.batch_a = ba;
    gram.Ma = gram.Nb = poly.Ma = poly.Nb = poly.K = step.Ma = step.K = (int)p.Ma;
    gram.K = step.Nb = (int)p.Nb;
    poly.A = poly.B = A;
    step.A = B;
    for (int k = 0; k < steps; ++k) {
        const float sx = scales[k].X, sa = scales[k].A, sb = scales[k].B;
        gram.A = gram.B = step.B = X;
        GramOut first{};
        first.A = A;
        first.la = la;
        first.batch_a = ba;
        first.by = sa / (sx * sx);
        plane_product<Halves, kAlong, kAlong, kBoundNone>(gram, first, p.gram, (int)batch, part, arrived, s);
        PolyOut second{};
        static_cast<GramOut&>(second) = first;
        second.A = B;
        second.from = A;
        second.b = c[3 * k + 1] * sb / sa;
        second.c = c[3 * k + 2] * sb / (sa * sa);
        plane_product<Halves, kAlong, kAlong, kBoundNone>(poly, second, p.poly, (int)batch, part, arrived, s);
        const bool last = k + 1 == steps && !tall;
        const float to = last ? 1.f : scales[k + 1].X;
        const StepOut third{X, Y, lx, bx, c[3 * k] * to / sx, to / (sb * sx)};
        if (last) {
            LastOut<T> l{};
            static_cast<StepOut&>(l) = third;
            l.out = out;
            l.rows = (int)rows;
            l.cols = (int)cols;
            plane_product<Halves, kAlong, kAcross, kBoundNone>(step, l, p.step, (int)batch, part, arrived, s);
        } else {
            plane_product<Halves, kAlong, kAcross, kBoundNone>(step, third, p.step, (int)batch, part, arrived, s);
        }
        std::swap(X, Y);
    }
    if (tall)
        hipLaunchKernelGGL((orth_turn_kernel<T>), dim3((unsigned)(p.Nb / 64), (unsigned)(p.Ma / 64), (unsigned)batch), dim3(256), 0, s, X, lx,
                           bx, (int)rows, (int)cols, 1.f / scales[steps].X, out);
}

}  // namespace
}  // namespace daspmm

using namespace daspmm;

extern "C" int da_orthogonalise_workspace(int dtype, int64_t batch, int64_t rows, int64_t cols, int steps, size_t* bytes)
{
    if (!bytes) return fail(DA_ERR_INVALID_ARG, "null output");
    const int st = orth_check(dtype, batch, rows, cols, steps);
    if (st != DA_OK) return st;
    if (small_takes(rows, cols)) {
        *bytes = 0;
        return DA_OK;
    }
    const OrthPlan& p = orth_plan(batch, rows, cols);
    *bytes = steps == 0 ? round16(p.parts_bytes) : p.bytes();
    return DA_OK;
}

extern "C" int da_orthogonalise(int dtype, int64_t batch, int64_t rows, int64_t cols, const void* g, int64_t ldg, int64_t stride, int steps,
                                const float* coefficients, float eps, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    size_t need = 0;
    const int st = da_orthogonalise_workspace(dtype, batch, rows, cols, steps, &need);
    if (st != DA_OK) return st;
    if (ldg < cols || stride < 0) return fail(DA_ERR_INVALID_ARG, "leading dimension smaller than the extent it strides over");
    if (!(eps >= 0.f)) return fail(DA_ERR_INVALID_ARG, "eps is negative or no number");
    if (steps > 0 && !coefficients) return fail(DA_ERR_INVALID_ARG, "null coefficients");
    StepScales scales[65];
    if (!orth_scales(steps, coefficients, scales)) return fail(DA_ERR_INVALID_ARG, "coefficients with which values could grow too large");
    if (batch == 0 || rows == 0 || cols == 0) return DA_OK;
    if (!g || !out) return fail(DA_ERR_INVALID_ARG, "null g or out");
    if (need && (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 16 != 0))
        return fail(DA_ERR_INVALID_ARG, "workspace missing, misaligned or smaller than reported");
    const OrthPlan p = small_takes(rows, cols) ? OrthPlan{} : orth_plan(batch, rows, cols);
    char* ws = static_cast<char*>(workspace);
    if (dtype == DA_F32)
        orthogonalise<float>(batch, rows, cols, static_cast<const float*>(g), ldg, stride, steps, coefficients, eps, static_cast<float*>(out), ws, p,
                             scales, (hipStream_t)stream);
    else
        orthogonalise<bf16>(batch, rows, cols, static_cast<const bf16*>(g), ldg, stride, steps, coefficients, eps, static_cast<bf16*>(out), ws, p,
                            scales, (hipStream_t)stream);
    return launched("da_orthogonalise launch");
}
