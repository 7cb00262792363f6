// What layer norm and root-mean-square norm share: teams of lanes to a row, and the backward pass.  Internal to the library, for one source file at a time.
//
//   backward  g = dy * weight;  dx = rstd * (g - sum g / n - h * (sum g h) / n) + dsum;  dweight = sum over rows dy * h;  dbias = sum over rows dy
//             with h from the kept 8-bit rows, or (x - mean) * rstd.  CENTRED: false where no mean was taken off, h = x * rstd: no sum g / n, no dbias
#ifndef ADATOPK_NORM_H
#define ADATOPK_NORM_H

#include "stage_ops.h"

// Products and sums are fused where the code says so and nowhere else: the forms of the backward pass give the same bits.
#pragma clang fp contract(off)

namespace {

using namespace adatopk_stage;

constexpr int COMPUTE_UNITS = 256;
constexpr int64_t MAX_COLS = 32768;        // 1024 lanes with four octets each
// Threads of the largest workgroup, by the lanes to a row.
constexpr int threads_of(int lanes) { return lanes < 512 ? 512 : lanes; }

// A row is a team's: L lanes, from an eighth of a wavefront to a whole workgroup.  Sum over them, in a fixed order, in every lane; `scratch`: a place per
// wavefront and value in LDS, the team's own.  Every lane of the workgroup calls it.
template <int L, int N, typename V> __device__ __forceinline__ void team_sum(V (&v)[N], V *scratch) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (L >= 64) {
            v[i] = wave_sum(v[i]);
        } else {
            v[i] += moved<0xB1, 0xF, false>(v[i]);   // the neighbour, the other pair of the quad, the other quad of eight lanes, the other half of sixteen
            v[i] += moved<0x4E, 0xF, false>(v[i]);
            v[i] += moved<0x141, 0xF, false>(v[i]);
            if constexpr (L >= 16) v[i] += moved<0x140, 0xF, false>(v[i]);
            if constexpr (L >= 32) v[i] += __shfl_xor(v[i], 16);
        }
    }
    if constexpr (L > 64) {
        constexpr int W = L / 64;
        const int wave = threadIdx.x / 64 % W;
        __syncthreads();  // the scratch of the sum before has been read
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) scratch[i * W + wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            V t = 0;
#pragma unroll
            for (int w = 0; w < W; ++w) t += scratch[i * W + w];
            v[i] = t;
        }
    }
}
// Up to two octets per lane, the row behind is loaded while one is summed up, and the weights stay in registers; with more, neither: a row is read again.
constexpr bool held(int slots) { return slots <= 2; }
template <typename T> __device__ __forceinline__ void load_weight(const void *p, bool wide, int64_t at, int64_t left, float absent, float (&v)[8]) {
    if (p == nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = absent;
    } else if (wide) {
        unpack(load_row(static_cast<const float *>(p) + at, left, at > 0), v);
    } else {
        unpack(load_row(static_cast<const T *>(p) + at, left, at > 0), v);
    }
}

struct Backward {
    const void *dy, *x, *weight, *dsum;
    const float *mean, *rstd;
    void *dx;
    float *partial;  // [parts][2][cols]: sums of dy * h and of dy over the rows of a workgroup (not CENTRED: [parts][cols], of dy * h)
    float *dweight, *dbias;
    int accumulate;
    int strips, row_groups;  // workgroups on columns, and behind them those on rows
    int64_t strip_rows;      // rows of a strip's workgroup; fewer than all: strips of several shares of the rows, each with a partial sum
    int64_t dy_stride, x_stride, dsum_stride, dx_stride;
    int64_t rows, cols;
    bool wide_weight;
    Act8 act8;
};

// Few rows: workgroups of their own add up the weight's gradient, 32 columns each, from operands that the others read at the same time.  A second read
// of what the caches hold instead of a second launch for the partial sums.  And the widest rows, beside whose own registers the sums have no place: there the
// rows are cut into shares.
constexpr int STRIP = 32;
template <bool CENTRED, typename T, bool KEEP> __device__ __forceinline__ void column_sums(const Backward &f, int group, float *share) {
    constexpr int AT_ONCE = 4;  // rows that a lane has on their way
    const int octet = threadIdx.x % (STRIP / 8), first = threadIdx.x / (STRIP / 8), step = blockDim.x / (STRIP / 8);
    const int strips = static_cast<int>((f.cols + STRIP - 1) / STRIP), strip = group % strips, part = group / strips;
    const int64_t begin = part * f.strip_rows, end = begin + f.strip_rows < f.rows ? begin + f.strip_rows : f.rows;
    const int64_t at = static_cast<int64_t>(strip) * STRIP + octet * 8, left = f.cols - at;
    float sums[2][8] = {};
    for (int64_t base = begin + first; base < end; base += static_cast<int64_t>(step) * AT_ONCE) {
        Raw<T> dy[AT_ONCE], x[KEEP ? 1 : AT_ONCE];
        U2 q[KEEP ? AT_ONCE : 1];
        uint32_t e[KEEP ? AT_ONCE : 1];
        float mean[AT_ONCE], rstd[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int64_t row = base + static_cast<int64_t>(i) * step, n = row < end ? left : 0;
            dy[i] = fetch_row(static_cast<const T *>(f.dy) + row * f.dy_stride + at, n, at > 0);
            if constexpr (KEEP) {
                q[i] = U2{0, 0};
                e[i] = 7;
                if (n > 0) act8_get(f.act8, row, static_cast<int>(at / 8), q[i], e[i]);
            } else {
                x[i] = fetch_row(static_cast<const T *>(f.x) + row * f.x_stride + at, n, at > 0);
                mean[i] = CENTRED && n > 0 ? f.mean[row] : 0.f;
                rstd[i] = n > 0 ? f.rstd[row] : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int64_t n = base + static_cast<int64_t>(i) * step < end ? left : 0;
            float g[8], h[8];
            unpack(settle(dy[i], n, at > 0), g);
            if constexpr (KEEP) {
                values_of(q[i], e[i], h);
            } else {
                unpack(settle(x[i], n, at > 0), h);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[j] = (CENTRED ? h[j] - mean[i] : h[j]) * rstd[i];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sums[0][j] = __builtin_fmaf(g[j], h[j], sums[0][j]);
                if constexpr (CENTRED) sums[1][j] += g[j];
            }
        }
    }
    // the lanes' sums of a column, in a fixed order: a share of them each, then the shares
    constexpr int VALUES = 2 * STRIP;  // (not CENTRED: the second half are zeros, for which there is no place)
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int j = 0; j < 8; ++j) share[first * VALUES + which * STRIP + octet * 8 + j] = sums[which][j];
    __syncthreads();
    const int shares = blockDim.x / VALUES, value = threadIdx.x % VALUES, mine = threadIdx.x / VALUES;
    float t = 0.f;
    for (int k = mine; k < step; k += shares) t += share[k * VALUES + value];
    __syncthreads();
    share[mine * VALUES + value] = t;
    __syncthreads();
    if (threadIdx.x >= VALUES) return;
    t = 0.f;
    for (int k = 0; k < shares; ++k) t += share[k * VALUES + threadIdx.x];
    const int64_t col = static_cast<int64_t>(strip) * STRIP + threadIdx.x % STRIP;
    const bool whole = f.strip_rows >= f.rows;
    float *to = threadIdx.x < STRIP ? f.dweight : CENTRED ? f.dbias : nullptr;
    if (!whole && (CENTRED || threadIdx.x < STRIP)) to = f.partial + (part * static_cast<int64_t>(CENTRED ? 2 : 1) + (threadIdx.x < STRIP ? 0 : 1)) * f.cols;
    if (to != nullptr && col < f.cols) to[col] = t + (whole && f.accumulate != 0 ? to[col] : 0.f);
}

// Rows come round as in the forward pass.  A row's operands stay as they were loaded and are taken apart twice, for the sums and for dx: half the
// registers of keeping them as floats, which the next row's operands take.  KEEP: h comes from the 8-bit rows.
// COLUMNS: the weight's gradient is not added up along with the rows, but, where it is asked for, by workgroups before those of the rows.
// 16384 x 1600 bf16 from 8-bit rows with the residual's gradient: 41.5 us and 4 of the join, 4.1 TB/s; from x without it 39 us, 4.0 TB/s; 32768 x 768 fp32
// 54 us, 5.6 TB/s; 1000 x 1601 fp16 7.7 us.  Without the centre 16384 x 1600 so 34 us and 4.6, 5.4 TB/s; 1000 x 1601 fp16 7.6.  What holds it below the forward pass is registers: the weight's gradient takes 16 for each octet, so a compute
// unit has half the loads on their way.  Two rows ahead instead of one cost more in moves or wavefronts than they hid (57 to 67 us where this took 52).
// 1024 x 20000 bf16: 87 us, 38 without the weight's gradient, whose columns are read a second time in pieces of 64 bytes.
template <bool CENTRED, typename T, int L, int S, bool KEEP, bool COLUMNS> __global__ __launch_bounds__(threads_of(L)) void k_norm_backward(Backward f) {
    constexpr bool HELD = held(S);
    constexpr int R = HELD ? S : 1;  // octets that are held at a time
    constexpr int SUMS = CENTRED ? 2 : 1;
    __shared__ float scratch[threads_of(L) / L][L > 64 ? 2 * (L / 64) : 1];
    if constexpr (COLUMNS) {
        if (static_cast<int>(blockIdx.x) < f.strips) {
            __shared__ float columns[threads_of(L) * 16];
            return column_sums<CENTRED, T, KEEP>(f, static_cast<int>(blockIdx.x), columns);
        }
    }
    const int lane = threadIdx.x % L, team = threadIdx.x / L;
    const int64_t teams = blockDim.x / L, step = f.row_groups * teams;
    const float inverse = 1.f / static_cast<float>(f.cols);
    auto place = [&](int s) {  // (rows that are not held: what is derived from it is not kept from row to row either)
        int l = lane;
        if constexpr (!HELD) asm volatile("" : "+v"(l));
        return (static_cast<int64_t>(s) * L + l) * 8;
    };
    struct Row {
        Raw<T> dy[R], ds[R], x[KEEP ? 1 : R];
        U2 q[KEEP ? R : 1];
        uint32_t e[KEEP ? R : 1];
        float mean, rstd;
    };
    auto scalars = [&](Row &to, int64_t row) {
        to.rstd = row < f.rows ? f.rstd[row] : 0.f;
        to.mean = CENTRED && !KEEP && row < f.rows ? f.mean[row] : 0.f;
    };
    auto fetch = [&](Row &to, int64_t row, int s, int at_slot, bool sum) {
        const int64_t at = place(s), left = row < f.rows ? f.cols - at : 0;
        to.dy[at_slot] = fetch_row(static_cast<const T *>(f.dy) + row * f.dy_stride + at, left, at > 0);
        if constexpr (KEEP) {
            if (left > 0) {
                act8_get(f.act8, row, static_cast<int>(at / 8), to.q[at_slot], to.e[at_slot]);
            } else {
                to.q[at_slot] = U2{0, 0};
                to.e[at_slot] = 7;
            }
        } else {
            to.x[at_slot] = fetch_row(static_cast<const T *>(f.x) + row * f.x_stride + at, left, at > 0);
        }
        if (sum && f.dsum != nullptr) to.ds[at_slot] = fetch_row(static_cast<const T *>(f.dsum) + row * f.dsum_stride + at, left, at > 0);
    };
    auto fetch_all = [&](Row &to, int64_t row) {
        scalars(to, row);
#pragma unroll
        for (int s = 0; s < R; ++s) fetch(to, row, s, s, true);
    };
    float dw[S][8] = {}, db[S][8] = {}, w[R][8];
    auto weights = [&](int s, int to) { load_weight<T>(f.weight, f.wide_weight, place(s), f.cols - place(s), 1.f, w[to]); };
    const int group = static_cast<int>(blockIdx.x) - f.strips;
    int64_t row = group * teams + team;
    Row now;
    if constexpr (HELD) {
        fetch_all(now, row);
#pragma unroll
        for (int s = 0; s < S; ++s) weights(s, s);
    }
    auto take = [&](const Row &from, int s, int slot, int64_t left, float (&g)[8], float (&h)[8]) {
        unpack(settle(from.dy[slot], left, place(s) > 0), g);
        if constexpr (KEEP) {
            values_of(from.q[slot], from.e[slot], h);
        } else {
            unpack(settle(from.x[slot], left, place(s) > 0), h);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = (CENTRED ? h[j] - from.mean : h[j]) * from.rstd;
        }
        // (what lies behind the row is no value: without x there it would count as -mean, and a group that is marked as no number is so in its padding)
        if (left < 8)
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = j < left ? h[j] : 0.f;
    };
    for (; row - team < f.rows; row += step) {  // (the workgroup's teams go round together, one without a row along with the others)
        Row next;
        if constexpr (HELD)
            fetch_all(next, row + step);
        else
            scalars(now, row);
        float sums[SUMS] = {};
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int k = HELD ? s : 0;
            if constexpr (!HELD) {
                fetch(now, row, s, 0, false);
                weights(s, 0);
            }
            float g[8], h[8];
            take(now, s, k, row < f.rows ? f.cols - place(s) : 0, g, h);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (!COLUMNS) {
                    dw[s][j] = __builtin_fmaf(g[j], h[j], dw[s][j]);
                    if constexpr (CENTRED) db[s][j] += g[j];
                }
                g[j] *= w[k][j];
                if constexpr (CENTRED) sums[0] += g[j];
                sums[SUMS - 1] = __builtin_fmaf(g[j], h[j], sums[SUMS - 1]);
            }
        }
        team_sum<L>(sums, scratch[team]);
        const float level = CENTRED ? sums[0] * inverse : 0.f, along = sums[SUMS - 1] * inverse;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int k = HELD ? s : 0;
            if constexpr (!HELD) {
                fetch(now, row, s, 0, true);
                weights(s, 0);
            }
            const int64_t at = place(s), left = row < f.rows ? f.cols - at : 0;
            float g[8], h[8], add[8] = {};
            take(now, s, k, left, g, h);
            if (f.dsum != nullptr) unpack(settle(now.ds[k], left, at > 0), add);
#pragma unroll
            for (int j = 0; j < 8; ++j) add[j] = __builtin_fmaf(now.rstd, __builtin_fmaf(-h[j], along, CENTRED ? __builtin_fmaf(g[j], w[k][j], -level) : g[j] * w[k][j]), add[j]);
            store_row(static_cast<T *>(f.dx) + row * f.dx_stride + at, left, pack<T>(add));
        }
        if constexpr (HELD) now = next;
    }
    if constexpr (COLUMNS) return;
    // n <= 8 neighbouring columns' sums, to the workgroup's place
    auto put = [&](int which, int64_t col, const float *t, int n) {
        typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));
        float *to = f.partial + (group * static_cast<int64_t>(SUMS) + which) * f.cols + col;
#pragma unroll
        for (int j = 0; j < n; j += 4) {
            if (col + j + 4 <= f.cols) {
                *reinterpret_cast<F4 *>(to + j) = F4{t[j], t[j + 1], t[j + 2], t[j + 3]};
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (col + j + i < f.cols) to[j + i] = t[j + i];
            }
        }
    };
    if constexpr (L < threads_of(L)) {  // the teams' shares, in a fixed order
        __shared__ float share[threads_of(L) / L][S * L * 8];
#pragma unroll
        for (int which = 0; which < SUMS; ++which) {
            if (which != 0) __syncthreads();
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int j = 0; j < 8; ++j) share[team][(s * 8 + j) * L + lane] = which == 0 ? dw[s][j] : db[s][j];
            __syncthreads();
            for (int piece = threadIdx.x; piece < 2 * S * L; piece += blockDim.x) {  // four of the eight columns of an octet
                const int octet = piece % (S * L), s = octet / L, l = octet % L, j0 = piece / (S * L) * 4;
                float t[4] = {};
                for (int v = 0; v < teams; ++v)
#pragma unroll
                    for (int j = 0; j < 4; ++j) t[j] += share[v][(s * 8 + j0 + j) * L + l];
                put(which, static_cast<int64_t>(octet) * 8 + j0, t, 4);
            }
        }
    } else {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            put(0, place(s), dw[s], 8);
            if constexpr (CENTRED) put(1, place(s), db[s], 8);
        }
    }
}

// Columns of the partial sums added up, in a fixed order: 32 columns per workgroup, 32 lanes of parts for each.  512 parts of 1600 columns: 4 us, of which
// the launch is most.
__global__ __launch_bounds__(1024) void k_norm_join(const float *partial, int parts, int64_t width, int64_t cols, float *dweight, float *dbias, int accumulate) {
    __shared__ float share[32][33];
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 32 + threadIdx.x % 32;  // column of the sums: cols for the weight and, if width is twice that, for the bias
    const int lane = threadIdx.x / 32;
    float t = 0.f;
    if (i < width) {
#pragma unroll 8
        for (int p = lane; p < parts; p += 32) t += partial[static_cast<int64_t>(p) * width + i];
    }
    share[lane][threadIdx.x % 32] = t;
    __syncthreads();
    if (lane != 0 || i >= width) return;
    t = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) t += share[k][threadIdx.x];
    float *to = i < cols ? dweight : dbias;
    if (to == nullptr) return;
    to += i < cols ? i : i - cols;
    *to = accumulate != 0 ? *to + t : t;
}

// Lanes to a row and octets per lane that hold a row: f is called with L and S as types.
template <int N> using Int = std::integral_constant<int, N>;
//
// The backward pass takes 1025 to 2048 columns with an octet to a lane and two workgroups to a compute unit, whose loads cover one another's sums: 16384 x 1600
// bf16 from 8-bit rows 35.5 us against 39.8 with two octets and one workgroup, from x 39.6 / 42.5, 8192 x 2048 fp32 30.5 / 32.4.  The forward pass takes two
// octets there (21.5 / 23.6), and so does the backward pass with more columns (4096 x 4096 fp32 33.2 / 37.3, 4096 x 8192 bf16 42.0 / 47.0).
template <bool BACKWARD, typename F> void with_shape(int64_t cols, F &&f) {
    if (cols <= 64) return f(Int<8>(), Int<1>());
    if (cols <= 128) return f(Int<16>(), Int<1>());
    if (cols <= 256) return f(Int<32>(), Int<1>());
    if (cols <= 512) return f(Int<64>(), Int<1>());
    if (cols <= 1024) return f(Int<64>(), Int<2>());
    if (BACKWARD && cols > 1024 && cols <= 2048) return f(Int<256>(), Int<1>());
    if (cols <= 2048) return f(Int<128>(), Int<2>());
    if (cols <= 4096) return f(Int<256>(), Int<2>());
    if (cols <= 8192) return f(Int<512>(), Int<2>());
    if (cols <= 16384) return f(Int<512>(), Int<4>());
    return f(Int<1024>(), Int<4>());
}

// Threads and workgroups of a launch: as many rows to a workgroup as it has teams for, but fewer where that would leave compute units without one.
struct Launch {
    int threads, groups;
};
inline Launch launch_of(int64_t rows, int lanes, int groups_per_unit) {
    int threads = threads_of(lanes);
    while (threads > lanes && threads > 64 && rows * lanes < static_cast<int64_t>(COMPUTE_UNITS) * threads) threads /= 2;
    const int teams = threads / lanes;
    const int64_t groups = (rows + teams - 1) / teams, most = static_cast<int64_t>(COMPUTE_UNITS) * groups_per_unit;
    return Launch{threads, static_cast<int>(groups < most ? groups : most)};
}
inline int forward_groups_per_unit(int slots) { return slots == 1 ? 4 : 2; }
// Workgroups of the backward pass to a compute unit: each writes a partial sum, and one octet to a lane leaves registers for two.
inline int groups_per_unit(int slots) { return slots == 1 ? 2 : 1; }
// Of the form with columns apart: whole workgroups, which the columns need, and one to a compute unit, the columns' among them.
inline Launch columns_launch(int64_t rows, int lanes, int64_t cols) {
    const int threads = threads_of(lanes), teams = threads / lanes;
    const int64_t groups = (rows + teams - 1) / teams, strips = (cols + STRIP - 1) / STRIP;
    const int64_t most = strips < COMPUTE_UNITS / 2 ? COMPUTE_UNITS - strips : COMPUTE_UNITS / 2;
    return Launch{threads, static_cast<int>(groups < most ? groups : most)};
}
// Either form, us, columns apart / along with the rows and a second launch: 32 x 768 3.6 / 8.2, 512 x 768 fp32 4.6 / 8.8, 1000 x 1600 bf16 6.4 / 10.7, 1000 x 64 5.4 /
// 7.8, 1000 x 4096 11.6 / 14.7, 512 x 8192 16.1 / 18.4; but 2048 x 1024 8.8 / 9.4, 2048 x 300 12.0 / 7.9, 4096 x 1024 22 / 11, 1024 x 16384 71 / 42: a strip's workgroup
// goes through all rows, and many strips wait for one another.
// The sums of more than 16384 columns do not fit beside the row (with spilled registers 1024 x 20000 bf16 took 178 us where it takes 87).
constexpr int64_t WIDEST = 16384, STRIP_ROWS = 1024;
inline bool by_columns(int64_t rows, int64_t cols) { return cols > WIDEST || (rows <= 4 * COMPUTE_UNITS && rows * cols <= static_cast<int64_t>(1) << 22); }
inline int strip_parts(int64_t rows) {
    const int64_t parts = (rows + STRIP_ROWS - 1) / STRIP_ROWS;
    return static_cast<int>(parts < COMPUTE_UNITS ? parts : COMPUTE_UNITS);
}
inline int64_t parts_at_most(int64_t rows, int64_t cols) {
    int64_t most = 0;
    with_shape<true>(cols, [&](auto, auto slots) { most = static_cast<int64_t>(COMPUTE_UNITS) * groups_per_unit(slots()); });
    return rows < most ? rows : most;
}

inline bool weights_ok(const void *p, adatopk_dtype wdt) { return pointer_ok_or_null(p, static_cast<size_t>(elem_size(wdt))); }

// The launches of a backward pass; arguments have been looked at.
template <bool CENTRED> void launch_backward(Backward f, adatopk_dtype dt, hipStream_t st) {
    const bool weights = f.dweight != nullptr || (CENTRED && f.dbias != nullptr);
    int parts = 0;
    if (f.rows > 0) {
        with_type(dt, [&](auto *null) {
            using T = std::remove_pointer_t<decltype(null)>;
            with_shape<true>(f.cols, [&](auto lanes, auto slots) {
                constexpr int L = decltype(lanes)::value, S = decltype(slots)::value;
                constexpr bool APART = static_cast<int64_t>(L) * S * 8 > WIDEST;  // (no size would come to the other form)
                const bool keep = f.act8.q != nullptr;
                const auto together = keep ? k_norm_backward<CENTRED, T, L, S, true, APART> : k_norm_backward<CENTRED, T, L, S, false, APART>;
                const auto apart = keep ? k_norm_backward<CENTRED, T, L, S, true, true> : k_norm_backward<CENTRED, T, L, S, false, true>;
                const bool columns = !weights || by_columns(f.rows, f.cols);
                const Launch l = !columns ? launch_of(f.rows, L, groups_per_unit(S)) : weights ? columns_launch(f.rows, L, f.cols) : launch_of(f.rows, L, 2);
                const int shares = strip_parts(f.rows), strips = columns && weights ? static_cast<int>((f.cols + STRIP - 1) / STRIP) * shares : 0;
                f.strip_rows = (f.rows + shares - 1) / shares;
                parts = columns ? static_cast<int>((f.rows + f.strip_rows - 1) / f.strip_rows) : l.groups;
                const auto launch = [&](int row_groups, int strip_groups) {
                    f.row_groups = row_groups;
                    f.strips = strip_groups;
                    hipLaunchKernelGGL(columns ? apart : together, dim3(static_cast<unsigned>(row_groups + strip_groups)), dim3(static_cast<unsigned>(l.threads)), 0,
                                       st, f);
                };
                if (strips != 0 && f.dx == f.dy) {  // the columns before the rows overwrite what they read
                    launch(0, strips);
                    launch(l.groups, 0);
                } else {
                    launch(l.groups, strips);
                }
            });
        });
    }
    if (weights && parts != 1) {  // (no rows: the sums are zero.  A matrix whose columns are not apart is always several workgroups')
        const int64_t width = (CENTRED ? 2 : 1) * f.cols;
        hipLaunchKernelGGL(k_norm_join, dim3(static_cast<unsigned>((width + 31) / 32)), dim3(1024), 0, st, f.partial, parts, width, f.cols, f.dweight, f.dbias,
                           f.accumulate);
    }
}

}  // namespace
#endif
