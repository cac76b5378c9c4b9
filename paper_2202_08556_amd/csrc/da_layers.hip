// Host side of include/da_layers.h: argument checks, choice of kernels and launch geometry.
#include "da_layers.h"

#include "da_gated.h"
#include "da_internal.h"
#include "da_norm_kernels.hip"
#include "da_distill_kernels.hip"
#include "da_spmm.h"

#include <algorithm>
#include <numeric>

namespace {

using namespace daspmm;

int fail(int code, const char* text) { return set_error(code, text); }

int launched(const char* where) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? DA_OK : set_hip_error(e, where);
}

bool known_dtype(int d) { return d == DA_F32 || d == DA_BF16; }
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
int pow2_at_least(int64_t x) {
    int p = 1;
    while (p < x) p <<= 1;
    return p;
}

// ------------------------------------------------------------------------------------------
// group norm
// ------------------------------------------------------------------------------------------
// Blocks of a launch: of 2^32 threads and more the high bits are lost.  What takes more is launched in pieces.
constexpr int64_t kMaxBlocks = (1LL << 32) / 1024 - 1;

// launch(first, count) for `all` things, `most` at a time
template <class F> void in_pieces(int64_t all, int64_t most, F&& launch) {
    for (int64_t first = 0; first < all; first += most) launch(first, std::min(most, all - first));
}

// Rows that a thread of a team holds: twice as many cost half of the waves and more than they save
constexpr int norm_held(int V) { return V >= 8 ? 2 : 4; }

struct NormPlan {
    int V;                   // numbers of an access: divides a group
    bool each;               // every row is a sample and a group a few lanes' registers
    int P, E;
    int64_t each_grid;
    int team;                // threads of a team; 0: none
    TeamPlan tp;
    bool split;
    SplitPlan sp;
    int64_t slots;
    // memory
    size_t stats;            // floats
    int64_t col_rows;        // rows of 2 C sums: the first pass's blocks, then the chunks
    size_t forward, table_at, part_at, means_at, backward;  // forward: part, table, stats; backward: sums, part, means, table
};

constexpr int64_t kNormMaxChannels = 1 << 20, kNormMaxGroups = 65535;

int norm_check(int dtype, int64_t rows, int64_t samples, int64_t channels, int64_t groups) {
    if (!known_dtype(dtype)) return fail(DA_ERR_UNSUPPORTED, "dtype is neither DA_F32 nor DA_BF16");
    if (rows < 0 || samples < 0 || channels < 0) return fail(DA_ERR_INVALID_ARG, "negative size");
    if (groups < 1 || channels % groups != 0) return fail(DA_ERR_INVALID_ARG, "channels are no multiple of groups");
    if (rows > INT32_MAX || samples > INT32_MAX || channels > kNormMaxChannels || groups > kNormMaxGroups)
        return fail(DA_ERR_UNSUPPORTED, "size too large");
    return DA_OK;
}

// Which kernels a shape takes.  train: statistics are kept and the backward pass is planned, too.
NormPlan norm_plan(int dtype, int64_t rows, int64_t samples, bool ragged, int64_t C, int64_t G, bool train) {
    NormPlan p{};
    const int64_t cg = C / G, length = ragged || samples == 0 ? 0 : rows / samples;
    const int most = dtype == DA_F32 ? 4 : 8;
    p.V = 1;
    while (p.V < most && cg % (2 * p.V) == 0) p.V *= 2;
    const int64_t cgv = cg / p.V, cus = compute_units();
    int64_t first_rows = 0;

    if (!ragged && length == 1 && cgv * p.V <= 64 * 32) {
        int E = 1;
        while (64 * E < cgv) E *= 2;
        if (E * p.V <= 32) {
            p.each = true;
            p.E = E;
            p.P = pow2_at_least(ceil_div(cgv, E));
            // A lane group that goes on to other rows keeps its group where the launch's lane groups are a multiple of G;
            // where every one of them has a row at most, no more are launched than there are.
            const int64_t per_block = kNormBlock / p.P, m = G / std::gcd(G, per_block);
            p.each_grid = std::min(ceil_div(rows * G, per_block), std::max<int64_t>(m, cus * 8 / m * m));
            first_rows = per_block > G ? p.each_grid : std::min(rows, p.each_grid * per_block / G);
        }
    }
    if (!p.each) {
        const int E = norm_held(p.V);
        const double mean = samples ? (double)rows / (double)samples : 0.0;
        auto tile = [&](int team) { return std::max<int64_t>(1, std::min<int64_t>(team / cgv, G)); };
        auto held = [&](int team) { return cgv > team ? 0 : (team / (tile(team) * cgv)) * (int64_t)E; };
        // A wave or a block of 256 threads takes a sample that its registers hold, and some more that is read again: equal
        // samples up to twice that, ragged ones up to 32768 numbers, since chunks are no longer than the shortest sample
        // that is split and short ones are many blocks with nothing to do.  Longer samples are split.
        // Blocks of 1024 threads take groups too wide for that, and equal samples that are too few to fill the chip, where
        // one launch counts.  (2168 ragged samples of 285 rows x 64 bf16, forward and backward: kernels of 349 us with
        // blocks of 1024 threads for up to 2048 rows, 274 split from 128 rows on, 227 from 512 on.)
        const int64_t blocks = samples * ceil_div(G, tile(1024));
        int64_t longest = 0;
        if (cgv > 256) longest = cgv > 1024 ? 0 : 2 * held(1024);
        else if (!ragged && blocks <= cus && length > 2 * held(256)) longest = held(1024);
        else longest = std::max(2 * held(256), ragged ? 32768 / C : 0);
        if (ragged || length <= longest) {
            if (cgv <= 64 && (ragged ? 2 * mean : mean) <= (double)held(64)) p.team = 64;
            else if (cgv <= 256 && (ragged || length <= 2 * held(256))) p.team = 256;
            else if (cgv <= 1024) p.team = 1024;
        }
        p.split = ragged ? rows > longest : length > longest;
        if (p.team) {
            const int64_t teams = p.team == 64 ? 4 : 1, cap = train ? cus * (p.team == 1024 ? 2 : 8) : 1 << 20;
            p.tp.GT = (int)tile(p.team);
            p.tp.tiles = (int)ceil_div(G, p.tp.GT);
            p.tp.longest = longest;
            p.tp.blocks = std::min({ceil_div(samples, teams), cap, kMaxBlocks / p.tp.tiles});
            first_rows = p.tp.blocks;
        }
        if (p.split) {
            p.sp.longest = longest;
            if (cgv <= kNormBlock) {
                p.sp.gpt = (int)std::min<int64_t>(kNormBlock / cgv, G);
                p.sp.pieces = 1;
                p.sp.TX = (int)(p.sp.gpt * cgv);
                p.sp.tiles = (int)ceil_div(G, p.sp.gpt);
            } else {
                p.sp.gpt = 1;
                p.sp.pieces = (int)ceil_div(cgv, kNormBlock);
                p.sp.TX = kNormBlock;
                p.sp.tiles = (int)G * p.sp.pieces;
            }
            const int64_t TY = kNormBlock / p.sp.TX;
            const int64_t target = std::clamp<int64_t>(rows * C / (cus * 8), ragged ? 32768 : 4096, 65536);
            p.sp.per = ceil_div(std::max<int64_t>(ceil_div(target, C), 1), TY) * TY;
            int64_t chunks, each = 0;
            if (ragged) {
                p.sp.per = longest == 0 ? 1 : std::min(p.sp.per, longest);
                chunks = ceil_div(rows, p.sp.per);
                p.slots = p.sp.per == 1 ? chunks : 2 * chunks;
            } else {
                each = ceil_div(length, p.sp.per);
                chunks = p.slots = samples * each;
            }
            p.sp.each = (int)each;
            p.sp.chunks = (int)chunks;                       // no more than rows
            p.sp.slots = p.slots;
        }
    }
    p.stats = p.each || !(train || p.split) ? 0 : (size_t)(samples * G * 2);
    const size_t parts = p.split ? round16((size_t)(p.slots * G * p.sp.pieces) * sizeof(float2)) : 0;
    const size_t table = p.split && ragged ? (size_t)p.sp.chunks * sizeof(ChunkEntry) : 0;
    p.table_at = parts;
    p.forward = parts + table + (train ? 0 : p.stats * sizeof(float));
    p.col_rows = first_rows + p.sp.chunks;
    p.part_at = round16((size_t)(p.col_rows * 2 * C) * sizeof(float));
    p.means_at = p.part_at + parts;
    const size_t means = p.split ? round16((size_t)(samples * G * 2) * sizeof(float)) : 0;
    p.backward = p.means_at + means + table;
    return p;
}

template <class T, int V, bool BWD>
void launch_each(const NormPlan& p, const NormShape& sh, const T* x, int64_t ldx, const T* dy, int64_t ldy, T* out, float* part,
                 hipStream_t s) {
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)p.each_grid), dim3(kNormBlock), 0, s, sh, p.P, x, (long)ldx, dy, (long)ldy, out,
                           part);
    };
    if (p.E == 1) return go(norm_each_kernel<T, V, 1, BWD>);
    if (p.E == 2) return go(norm_each_kernel<T, V, 2, BWD>);
    if (p.E == 4) return go(norm_each_kernel<T, V, 4, BWD>);
    if constexpr (V <= 4) {
        if (p.E == 8) return go(norm_each_kernel<T, V, 8, BWD>);
    }
    if constexpr (V <= 2) {
        if (p.E == 16) return go(norm_each_kernel<T, V, 16, BWD>);
    }
    if constexpr (V == 1) {
        if (p.E == 32) return go(norm_each_kernel<T, V, 32, BWD>);
    }
}

// Teams and chunks in one launch; teams of 1024 threads, whose blocks no chunk has, in one of their own
template <class T, int V, bool BWD>
void launch_first(const NormPlan& p, const NormShape& sh, const T* x, int64_t ldx, const T* dy, int64_t ldy, T* out, float* stats,
                  float* team_cols, ChunkEntry* table, float2* part, float* cols, hipStream_t s) {
    auto launch = [&](auto kernel, int block, const TeamPlan& tp, int64_t from, int64_t chunks) {
        const int64_t blocks = tp.blocks * tp.tiles + chunks * p.sp.tiles;
        if (blocks)
            hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(block), 0, s, sh, tp, p.sp, (int)from, x, (long)ldx, dy, (long)ldy, out,
                               stats, team_cols, table, part, cols);
    };
    auto go = [&](auto kernel, int block, const TeamPlan& tp, int64_t chunks) {
        if (!chunks) return launch(kernel, block, tp, 0, 0);
        in_pieces(chunks, kMaxBlocks / p.sp.tiles, [&](int64_t from, int64_t count) { launch(kernel, block, from ? TeamPlan{} : tp, from, count); });
    };
    const int64_t chunks = p.split ? p.sp.chunks : 0;
    constexpr int E = norm_held(V);
    if (p.team == 1024) go(norm_first_kernel<T, V, 1024, E, false, BWD>, 1024, p.tp, 0);
    if (p.team == 1024 || !p.team) go(norm_first_kernel<T, V, 256, 0, true, BWD>, 256, TeamPlan{}, chunks);
    else if (p.team == 64 && chunks) go(norm_first_kernel<T, V, 64, E, true, BWD>, 256, p.tp, chunks);
    else if (p.team == 64) go(norm_first_kernel<T, V, 64, E, false, BWD>, 256, p.tp, 0);
    else if (chunks) go(norm_first_kernel<T, V, 256, E, true, BWD>, 256, p.tp, chunks);
    else go(norm_first_kernel<T, V, 256, E, false, BWD>, 256, p.tp, 0);
}

// The last chunks first: the kernel counts down from the last of its own
template <class T, int V, bool BWD>
void launch_apply(const NormPlan& p, const NormShape& sh, const T* x, int64_t ldx, const T* dy, int64_t ldy, const float* stats,
                  const float* means, ChunkEntry* table, T* out, hipStream_t s) {
    in_pieces(p.sp.chunks, kMaxBlocks, [&](int64_t done, int64_t count) {
        hipLaunchKernelGGL((norm_apply_kernel<T, V, BWD>), dim3((unsigned)count, (unsigned)p.sp.tiles), dim3(kNormBlock), 0, s, sh, p.sp,
                           (int)(p.sp.chunks - 1 - done), x, (long)ldx, dy, (long)ldy, stats, means, table, out);
    });
}

template <class T, int V>
void norm_forward(const NormPlan& p, const NormShape& sh, const T* x, int64_t ldx, T* y, float* stats, char* ws, hipStream_t s) {
    const T* none = nullptr;
    if (p.each) return launch_each<T, V, false>(p, sh, x, ldx, none, 0, y, nullptr, s);
    float2* part = reinterpret_cast<float2*>(ws);
    ChunkEntry* table = reinterpret_cast<ChunkEntry*>(ws + p.table_at);
    launch_first<T, V, false>(p, sh, x, ldx, none, 0, y, stats, nullptr, table, part, nullptr, s);
    if (!p.split) return;
    in_pieces(sh.offsets ? p.sp.chunks : sh.samples, kMaxBlocks, [&](int64_t from, int64_t joins) {
        hipLaunchKernelGGL((norm_join_kernel<V>), dim3((unsigned)joins, (unsigned)ceil_div(sh.G, kJoinGroups)), dim3(kJoinBlock), 0, s, sh, p.sp,
                           (int)from, table, part, stats);
    });
    launch_apply<T, V, false>(p, sh, x, ldx, none, 0, stats, nullptr, table, y, s);
}

template <class T, int V>
void norm_backward(const NormPlan& p, const NormShape& sh, const T* x, int64_t ldx, const T* dy, int64_t ldy, const float* stats,
                   T* dx, void* dw, void* db, char* ws, hipStream_t s) {
    float* cols = reinterpret_cast<float*>(ws);
    float2* part = reinterpret_cast<float2*>(ws + p.part_at);
    float* means = reinterpret_cast<float*>(ws + p.means_at);
    ChunkEntry* table = reinterpret_cast<ChunkEntry*>(ws + p.backward - (sh.offsets ? p.sp.chunks * sizeof(ChunkEntry) : 0));
    if (p.each) launch_each<T, V, true>(p, sh, x, ldx, dy, ldy, dx, cols, s);
    else launch_first<T, V, true>(p, sh, x, ldx, dy, ldy, dx, const_cast<float*>(stats), cols, table, part, cols + p.tp.blocks * 2 * sh.C,
                                  s);
    // a join is of kJoinGroups groups of a sample; the sums are part of the first launch
    const int64_t each = ceil_div(sh.G, kJoinGroups), joins = !p.split ? 0 : sh.offsets ? p.sp.chunks : sh.samples, sums = dw || db ? ceil_div(2 * sh.C, 16) : 0;
    auto join = [&](int64_t from, int64_t count) {
        const int64_t more = from ? 0 : sums;
        if (count + more)
            hipLaunchKernelGGL(norm_grad_join_kernel, dim3((unsigned)(count * each + more)), dim3(kJoinBlock), 0, s, sh, p.sp, (int)from,
                               (int)(count * each), table, part, means, cols, (long)p.col_rows, dw, db);
    };
    if (joins) in_pieces(joins, (kMaxBlocks - sums) / each, join);
    else join(0, 0);
    if (p.split) launch_apply<T, V, true>(p, sh, x, ldx, dy, ldy, stats, means, table, dx, s);
}

template <class F> void with_type_and_width(int dtype, int V, F&& f) {
    if (dtype == DA_F32) {
        if (V == 4) f(float{}, std::integral_constant<int, 4>{});
        else if (V == 2) f(float{}, std::integral_constant<int, 2>{});
        else f(float{}, std::integral_constant<int, 1>{});
    } else {
        if (V == 8) f(bf16{}, std::integral_constant<int, 8>{});
        else if (V == 4) f(bf16{}, std::integral_constant<int, 4>{});
        else if (V == 2) f(bf16{}, std::integral_constant<int, 2>{});
        else f(bf16{}, std::integral_constant<int, 1>{});
    }
}

int norm_shape(int dtype, int64_t rows, int64_t samples, const int32_t* offsets, int64_t channels, int64_t groups, const void* x,
               int64_t ldx, const void* w, const void* b, int param_dtype, float eps, int act, NormShape* sh) {
    const int st = norm_check(dtype, rows, samples, channels, groups);
    if (st != DA_OK) return st;
    if (!known_dtype(param_dtype)) return fail(DA_ERR_UNSUPPORTED, "param_dtype is neither DA_F32 nor DA_BF16");
    if (act < 0 || act >= DA_NUM_ACTS) return fail(DA_ERR_INVALID_ARG, "unknown activation");
    if (!(eps >= 0.f)) return fail(DA_ERR_INVALID_ARG, "eps is negative or no number");
    if (ldx < channels) return fail(DA_ERR_INVALID_ARG, "leading dimension smaller than the extent it strides over");
    if (rows > 0 && samples == 0) return fail(DA_ERR_INVALID_ARG, "rows without a sample");
    if (!offsets && samples > 0 && rows % samples != 0) return fail(DA_ERR_INVALID_ARG, "rows are no multiple of samples");
    if (rows > 0 && channels > 0 && !x) return fail(DA_ERR_INVALID_ARG, "null x");
    *sh = NormShape{rows, samples, offsets, samples ? rows / samples : 0, (int)channels, (int)groups, (int)(channels / groups), eps,
                    act, param_dtype, w, b};
    return DA_OK;
}

int workspace_error() {
    return fail(DA_ERR_INVALID_ARG, "workspace missing, misaligned or smaller than reported");
}

}  // namespace

extern "C" int da_group_norm_sizes(int dtype, int64_t rows, int64_t samples, int ragged, int64_t channels, int64_t groups, int train,
                                   size_t* stats_floats, size_t* forward_bytes, size_t* backward_bytes)
{
    if (!stats_floats || !forward_bytes || !backward_bytes) return fail(DA_ERR_INVALID_ARG, "null output");
    const int st = norm_check(dtype, rows, samples, channels, groups);
    if (st != DA_OK) return st;
    *stats_floats = *forward_bytes = *backward_bytes = 0;
    if (channels == 0) return DA_OK;
    const NormPlan p = norm_plan(dtype, rows, samples, ragged != 0, channels, groups, train != 0);
    *stats_floats = train ? p.stats : 0;
    *forward_bytes = p.forward;
    *backward_bytes = p.backward;
    return DA_OK;
}

extern "C" int da_group_norm(int dtype, int64_t rows, int64_t samples, const int32_t* offsets, int64_t channels, int64_t groups,
                             const void* x, int64_t ldx, const void* w, const void* b, int param_dtype, float eps, int act, void* y,
                             float* stats, void* workspace, size_t workspace_bytes, void* stream)
{
    NormShape sh;
    const int st = norm_shape(dtype, rows, samples, offsets, channels, groups, x, ldx, w, b, param_dtype, eps, act, &sh);
    if (st != DA_OK) return st;
    if (rows == 0 || channels == 0) return DA_OK;
    if (!y) return fail(DA_ERR_INVALID_ARG, "null y");
    const NormPlan p = norm_plan(dtype, rows, samples, offsets != nullptr, channels, groups, stats != nullptr);
    if (p.forward && (!workspace || workspace_bytes < p.forward || !aligned16(workspace))) return workspace_error();
    char* ws = static_cast<char*>(workspace);
    float* kept = stats ? stats : p.stats ? reinterpret_cast<float*>(ws + p.forward - p.stats * sizeof(float)) : nullptr;
    with_type_and_width(dtype, p.V, [&](auto t, auto v) {
        using T = decltype(t);
        norm_forward<T, decltype(v)::value>(p, sh, static_cast<const T*>(x), ldx, static_cast<T*>(y), kept, ws, (hipStream_t)stream);
    });
    return launched("da_group_norm launch");
}

extern "C" int da_group_norm_backward(int dtype, int64_t rows, int64_t samples, const int32_t* offsets, int64_t channels,
                                      int64_t groups, const void* x, int64_t ldx, const void* dy, int64_t ldy, const void* w,
                                      const void* b, int param_dtype, float eps, int act, const float* stats, void* dx, void* dw,
                                      void* db, void* workspace, size_t workspace_bytes, void* stream)
{
    NormShape sh;
    const int st = norm_shape(dtype, rows, samples, offsets, channels, groups, x, ldx, w, b, param_dtype, eps, act, &sh);
    if (st != DA_OK) return st;
    if (channels == 0) return DA_OK;
    if (ldy < channels) return fail(DA_ERR_INVALID_ARG, "leading dimension smaller than the extent it strides over");
    if (rows > 0 && (!dy || !dx)) return fail(DA_ERR_INVALID_ARG, "null dy or dx");
    NormPlan p{};
    p.V = 1;                                                 // no rows: dw and db are sums of nothing
    if (rows > 0) p = norm_plan(dtype, rows, samples, offsets != nullptr, channels, groups, true);
    if (p.stats && !stats) return fail(DA_ERR_INVALID_ARG, "null stats");
    if (p.backward && (!workspace || workspace_bytes < p.backward || !aligned16(workspace))) return workspace_error();
    with_type_and_width(dtype, p.V, [&](auto t, auto v) {
        using T = decltype(t);
        norm_backward<T, decltype(v)::value>(p, sh, static_cast<const T*>(x), ldx, static_cast<const T*>(dy), ldy, stats,
                                             static_cast<T*>(dx), dw, db, static_cast<char*>(workspace), (hipStream_t)stream);
    });
    return launched("da_group_norm_backward launch");
}

// ------------------------------------------------------------------------------------------
// distillation
// ------------------------------------------------------------------------------------------
namespace {

constexpr int64_t kDistillMaxClasses = INT32_MAX - (1 << 16);
constexpr size_t kNarrowEntriesBytes = 32 << 10;

struct DistillPlan {
    bool narrow;
    int P, E;
    int64_t pieces, piece;
};

// Rows of up to 2048 classes fit a wave's registers.  Wider ones are cut into pieces where there are too few for the chip.
DistillPlan distill_plan(int dtype, int64_t rows, int64_t classes, int64_t best) {
    DistillPlan p{};
    const int V = dtype == DA_F32 ? 4 : 8;
    const int64_t vecs = ceil_div(classes, V);
    int64_t slots = INT64_MAX;
    for (int E : {1, 2, 3, 4, 8}) {
        if (E * V > 32) continue;
        const int P = pow2_at_least(ceil_div(vecs, E));
        if (P > 64 || (int64_t)P * E >= slots) continue;
        slots = (int64_t)P * E;
        p.P = P;
        p.E = E;
    }
    p.narrow = slots != INT64_MAX && (size_t)(kDistillBlock / p.P) * best * sizeof(Entry) <= kNarrowEntriesBytes;
    const int64_t want = 8 * compute_units();
    p.pieces = std::clamp<int64_t>(ceil_div(want, std::max<int64_t>(rows, 1)), 1, std::max<int64_t>(1, classes / 8192));
    const int64_t turn = 4 * kWideBlock * V;
    p.piece = std::max<int64_t>(1, ceil_div(ceil_div(classes, p.pieces), turn)) * turn;       // no classes: nothing in one piece
    p.pieces = std::max<int64_t>(1, ceil_div(classes, p.piece));
    return p;
}

int distill_check(int dtype, int64_t rows, int64_t classes, int64_t best, const void* z, int64_t ldz, const void* index,
                  const void* top, int top_dtype, float temperature) {
    if (!known_dtype(dtype) || !known_dtype(top_dtype)) return fail(DA_ERR_UNSUPPORTED, "dtype is neither DA_F32 nor DA_BF16");
    if (rows < 0 || classes < 0 || best < 0) return fail(DA_ERR_INVALID_ARG, "negative size");
    if (rows > INT32_MAX || classes > kDistillMaxClasses) return fail(DA_ERR_UNSUPPORTED, "size too large");
    if (best > kDistillMaxBest) return fail(DA_ERR_UNSUPPORTED, "more than 1024 entries to a row");
    if (!(temperature > 0.f) || !(1.f / temperature > 0.f)) return fail(DA_ERR_INVALID_ARG, "temperature is not positive and finite");
    if (ldz < classes) return fail(DA_ERR_INVALID_ARG, "leading dimension smaller than the extent it strides over");
    if (rows > 0 && ((classes > 0 && !z) || (best > 0 && (!index || !top)))) return fail(DA_ERR_INVALID_ARG, "null z, index or top");
    return DA_OK;
}

template <class T, int V, bool BWD>
void launch_narrow(const DistillPlan& p, int64_t rows, const Teacher& te, const T* z, int64_t ldz, float temperature, float* loss,
                   float* stats, const float* dloss, int64_t dloss_stride, T* dz, hipStream_t s) {
    const int64_t per_block = kDistillBlock / p.P;
    const int64_t grid = std::min<int64_t>(ceil_div(rows, per_block), 1 << 20);
    const size_t lds = BWD ? (size_t)per_block * te.best * sizeof(Entry) : 0;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kDistillBlock), lds, s, (long)rows, p.P, te, z, (long)ldz, temperature,
                           loss, stats, dloss, (long)dloss_stride, dz);
    };
    if (p.E == 1) return go(distill_narrow_kernel<T, V, 1, BWD>);
    if (p.E == 2) return go(distill_narrow_kernel<T, V, 2, BWD>);
    if (p.E == 3) return go(distill_narrow_kernel<T, V, 3, BWD>);
    if (p.E == 4) return go(distill_narrow_kernel<T, V, 4, BWD>);
    if constexpr (V == 4) return go(distill_narrow_kernel<T, V, 8, BWD>);
}

template <class T, int V>
void distill_forward(const DistillPlan& p, int64_t rows, const Teacher& te, const T* z, int64_t ldz, float temperature, float* loss,
                     float* stats, float2* part, hipStream_t s) {
    if (p.narrow)
        return launch_narrow<T, V, false>(p, rows, te, z, ldz, temperature, loss, stats, nullptr, 0, nullptr, s);
    hipLaunchKernelGGL((distill_wide_kernel<T, V>), dim3((unsigned)p.pieces, (unsigned)std::min<int64_t>(rows, 65535)),
                       dim3(kWideBlock), 0, s, (long)rows, (long)p.piece, te, z, (long)ldz, temperature, loss, stats, part);
    if (p.pieces > 1)
        hipLaunchKernelGGL((distill_join_kernel<T>), dim3((unsigned)std::min<int64_t>(rows, 65535)), dim3(256), 0, s, (long)rows,
                           (int)p.pieces, te, z, (long)ldz, temperature, loss, stats, part);
}

Teacher teacher(int64_t classes, int64_t best, const void* index, int index64, const void* top, int top_dtype, float temperature) {
    return Teacher{classes, best, index, top, index64, top_dtype, (float)(1.4426950408889634 / (double)temperature)};
}

}  // namespace

extern "C" int da_distill_workspace(int64_t rows, int64_t classes, size_t* bytes)
{
    if (!bytes) return fail(DA_ERR_INVALID_ARG, "null bytes");
    if (rows < 0 || classes < 0) return fail(DA_ERR_INVALID_ARG, "negative size");
    if (rows > INT32_MAX || classes > kDistillMaxClasses) return fail(DA_ERR_UNSUPPORTED, "size too large");
    const int64_t pieces = std::max(distill_plan(DA_F32, rows, classes, 0).pieces, distill_plan(DA_BF16, rows, classes, 0).pieces);
    *bytes = pieces > 1 ? (size_t)(rows * pieces) * sizeof(float2) : 0;
    return DA_OK;
}

extern "C" int da_distill(int dtype, int64_t rows, int64_t classes, int64_t best, const void* z, int64_t ldz, const void* index,
                          int index64, const void* top, int top_dtype, float temperature, float* loss, float* stats,
                          void* workspace, size_t workspace_bytes, void* stream)
{
    const int st = distill_check(dtype, rows, classes, best, z, ldz, index, top, top_dtype, temperature);
    if (st != DA_OK) return st;
    if (rows == 0) return DA_OK;
    if (!loss) return fail(DA_ERR_INVALID_ARG, "null loss");
    const DistillPlan p = distill_plan(dtype, rows, classes, best);
    const size_t need = !p.narrow && p.pieces > 1 ? (size_t)(rows * p.pieces) * sizeof(float2) : 0;
    if (need && (!workspace || workspace_bytes < need || !aligned16(workspace))) return workspace_error();
    const Teacher te = teacher(classes, best, index, index64, top, top_dtype, temperature);
    float2* part = static_cast<float2*>(workspace);
    if (dtype == DA_F32)
        distill_forward<float, 4>(p, rows, te, static_cast<const float*>(z), ldz, temperature, loss, stats, part, (hipStream_t)stream);
    else
        distill_forward<bf16, 8>(p, rows, te, static_cast<const bf16*>(z), ldz, temperature, loss, stats, part, (hipStream_t)stream);
    return launched("da_distill launch");
}

namespace {

template <class T, int V>
void distill_grad(const DistillPlan& p, int64_t rows, const Teacher& te, const void* z, int64_t ldz, float temperature,
                  const float* stats, const float* dloss, int64_t dloss_stride, void* dz, hipStream_t s) {
    const T* zt = static_cast<const T*>(z);
    T* dt = static_cast<T*>(dz);
    if (p.narrow)
        return launch_narrow<T, V, true>(p, rows, te, zt, ldz, temperature, nullptr, const_cast<float*>(stats), dloss, dloss_stride,
                                         dt, s);
    hipLaunchKernelGGL((distill_wide_grad_kernel<T, V>), dim3((unsigned)p.pieces, (unsigned)std::min<int64_t>(rows, 65535)),
                       dim3(kWideBlock), 0, s, (long)rows, (long)p.piece, te, zt, (long)ldz, temperature, stats, dloss,
                       (long)dloss_stride, dt);
}

}  // namespace

extern "C" int da_distill_backward(int dtype, int64_t rows, int64_t classes, int64_t best, const void* z, int64_t ldz,
                                   const void* index, int index64, const void* top, int top_dtype, float temperature,
                                   const float* stats, const float* dloss, int64_t dloss_stride, void* dz, void* stream)
{
    const int st = distill_check(dtype, rows, classes, best, z, ldz, index, top, top_dtype, temperature);
    if (st != DA_OK) return st;
    if (dloss_stride < 0) return fail(DA_ERR_INVALID_ARG, "negative stride");
    if (rows == 0 || classes == 0) return DA_OK;
    if (!stats || !dloss || !dz) return fail(DA_ERR_INVALID_ARG, "null stats, dloss or dz");
    const DistillPlan p = distill_plan(dtype, rows, classes, best);
    const Teacher te = teacher(classes, best, index, index64, top, top_dtype, temperature);
    if (dtype == DA_F32) distill_grad<float, 4>(p, rows, te, z, ldz, temperature, stats, dloss, dloss_stride, dz, (hipStream_t)stream);
    else distill_grad<bf16, 8>(p, rows, te, z, ldz, temperature, stats, dloss, dloss_stride, dz, (hipStream_t)stream);
    return launched("da_distill_backward launch");
}

// ------------------------------------------------------------------------------------------
// gated feed-forward block
// ------------------------------------------------------------------------------------------
namespace {

constexpr int64_t kGatedMax = 1 << 30;                      // the kernels count rows and columns, and those past the end, in 32 bits

int gated_check(int dtype, int64_t rows, int64_t d, int64_t h, int64_t dout) {
    if (!known_dtype(dtype)) return fail(DA_ERR_UNSUPPORTED, "dtype is neither DA_F32 nor DA_BF16");
    if (rows < 0 || d < 0 || h < 0 || dout < 0) return fail(DA_ERR_INVALID_ARG, "negative size");
    const int64_t most = std::max({rows, d, h, dout});
    if (most > kGatedMax) return fail(DA_ERR_UNSUPPORTED, "size too large");
    if (!gated_fits(GatedShape{rows, d, h, dout}, dtype == DA_F32 ? 4 : 2)) return fail(DA_ERR_UNSUPPORTED, "size too large");
    return DA_OK;
}

}  // namespace

extern "C" int da_gated_workspace(int dtype, int64_t rows, int64_t d, int64_t h, int64_t dout, size_t* forward_bytes,
                                  size_t* backward_bytes)
{
    if (!forward_bytes || !backward_bytes) return fail(DA_ERR_INVALID_ARG, "null output");
    const int st = gated_check(dtype, rows, d, h, dout);
    if (st != DA_OK) return st;
    const GatedShape s{rows, d, h, dout};
    *forward_bytes = dtype == DA_F32 ? gated_forward_bytes<float>(s) : gated_forward_bytes<bf16>(s);
    *backward_bytes = dtype == DA_F32 ? gated_backward_bytes<float>(s) : gated_backward_bytes<bf16>(s);
    return DA_OK;
}

extern "C" int da_gated(int dtype, int64_t rows, int64_t d, int64_t h, int64_t dout, const void* x, int64_t ldx, const void* w_gate,
                        const void* w_up, const void* w_down, int act, void* y, float* u, float* v, void* a, void* workspace,
                        size_t workspace_bytes, void* stream)
{
    size_t need = 0, backward = 0;
    const int st = da_gated_workspace(dtype, rows, d, h, dout, &need, &backward);
    if (st != DA_OK) return st;
    if (act < 0 || act >= DA_NUM_ACTS) return fail(DA_ERR_INVALID_ARG, "unknown activation");
    if (ldx < d) return fail(DA_ERR_INVALID_ARG, "leading dimension smaller than the extent it strides over");
    if (rows == 0 || (h == 0 && dout == 0)) return DA_OK;
    if ((d > 0 && (!x || (h > 0 && (!w_gate || !w_up)))) || (h > 0 && (!a || (dout > 0 && !w_down))) || (dout > 0 && !y))
        return fail(DA_ERR_INVALID_ARG, "null x, weight, a or y");
    if (!u != !v) return fail(DA_ERR_INVALID_ARG, "one of u and v is null");
    if (need && (!workspace || workspace_bytes < need || !aligned16(workspace))) return workspace_error();
    GatedCall c{};
    c.s = GatedShape{rows, d, h, dout};
    c.x = x;
    c.wg = w_gate;
    c.wu = w_up;
    c.wd = w_down;
    c.ldx = ldx;
    c.act = act;
    c.u = u;
    c.v = v;
    c.a = a;
    c.y = y;
    c.workspace = static_cast<char*>(workspace);
    c.stream = (hipStream_t)stream;
    if (dtype == DA_F32) gated_forward<float>(c);
    else gated_forward<bf16>(c);
    return launched("da_gated launch");
}

extern "C" int da_gated_backward(int dtype, int64_t rows, int64_t d, int64_t h, int64_t dout, const void* x, int64_t ldx,
                                 const void* dy, int64_t ldy, const void* w_gate, const void* w_up, const void* w_down, int act,
                                 const float* u, const float* v, const void* a, void* dx, void* dw_gate, void* dw_up, void* dw_down,
                                 void* workspace, size_t workspace_bytes, void* stream)
{
    size_t forward = 0, need = 0;
    const int st = da_gated_workspace(dtype, rows, d, h, dout, &forward, &need);
    if (st != DA_OK) return st;
    if (act < 0 || act >= DA_NUM_ACTS) return fail(DA_ERR_INVALID_ARG, "unknown activation");
    if (ldx < d || ldy < dout) return fail(DA_ERR_INVALID_ARG, "leading dimension smaller than the extent it strides over");
    const bool inner = rows > 0 && h > 0;
    if ((rows > 0 && ((d > 0 && !x) || (dout > 0 && !dy))) || (inner && (!u || !v || !a)) ||
        (h > 0 && ((d > 0 && (!w_gate || !w_up)) || (dout > 0 && !w_down))))
        return fail(DA_ERR_INVALID_ARG, "null x, dy, weight, u, v or a");
    if (need && (!workspace || workspace_bytes < need || !aligned16(workspace))) return workspace_error();
    GatedCall c{};
    c.s = GatedShape{rows, d, h, dout};
    c.x = x;
    c.dy = dy;
    c.wg = w_gate;
    c.wu = w_up;
    c.wd = w_down;
    c.ldx = ldx;
    c.ldy = ldy;
    c.act = act;
    c.u = const_cast<float*>(u);
    c.v = const_cast<float*>(v);
    c.a = const_cast<void*>(a);
    c.dx = dx;
    c.dwg = dw_gate;
    c.dwu = dw_up;
    c.dwd = dw_down;
    c.workspace = static_cast<char*>(workspace);
    c.stream = (hipStream_t)stream;
    if (dtype == DA_F32) gated_backward<float>(c);
    else gated_backward<bf16>(c);
    return launched("da_gated_backward launch");
}
