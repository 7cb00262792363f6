// A weight matrix changed by its orthogonalised gradient, as the optimiser Muon does.
//
//   m = mu m + g;  u = m, or g + mu m;  X = u / (|u| + eps);  in each step A = X X^T, B = a I + b A + c A A, X = B X;  w = decay w + scale X
//
// with the Frobenius norm and a, b, c = 3.4445, -4.7750, 2.0315, which take singular values from 0 ... 1 to 0.7 ... 1.2 in five steps.  X is taken with its shorter side
// first (transposed where that is the other).  A step is three products of matrices whose rows lie along the sum: A from X twice, A A from A twice since A is
// symmetric, and X from B and X transposed, so each step writes X both ways; of A and B half the tiles are computed and written twice.
//
// Small singular values grow 3.4-fold in each step, and so does what a rounding of X leaves in their directions: with X in bf16 the result is some 2 to 7 % off, in
// one fp16 1e-3 to 6e-3, in two fp16 4e-7 to 8e-6, like fp32 (512 to 1000 rows, of noise and of low rank with noise).  So everything between the steps is two fp16,
// h + l, times 2^14 (A and X stay within 1.5, X's singular values within 1.21: nothing overflows, and l keeps its bits down to 2^-17) or, for B, whose diagonal
// reaches 3.45, 2^13.  Products are three of the matrix instruction's, sums fp32; |u| is a 64-bit sum.
#include <hip/hip_runtime.h>

#include "row_tiles.h"

// Products and sums are fused where the code says so and nowhere else.
#pragma clang fp contract(off)

namespace {

using namespace adatopk_stage;

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float ONE = 16384.f, ONE_OF_B = 8192.f;  // what 1 is held as

// A matrix of pairs: rows of 128 bytes for 32 elements, 32 h and then their l, padded with zeros.
struct Pairs {
    uint8_t *at;
    int64_t pitch;
};
constexpr int64_t padded(int64_t n) { return (n + 31) / 32 * 32; }
inline size_t pairs_bytes(int64_t rows, int64_t cols) { return adatopk_internal::align_up(static_cast<size_t>(rows) * static_cast<size_t>(padded(cols)) * 4, 256); }

__device__ __forceinline__ uint8_t *octet_of(const Pairs &p, int64_t row, int64_t col) { return p.at + row * p.pitch + col / 32 * 128 + col % 32 * 2; }
// Eight elements of a row from col on, a multiple of eight; those from `limit` on are zeros, and what lies behind its padding is left alone.
__device__ __forceinline__ void put_pairs(const Pairs &p, int64_t row, int64_t col, int64_t limit, const float (&v)[8]) {
    if (col >= padded(limit)) return;
    float h[8], l[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float t = col + j < limit ? v[j] : 0.f;
        h[j] = static_cast<float>(static_cast<_Float16>(t));
        l[j] = t - h[j];
    }
    uint8_t *const to = octet_of(p, row, col);
    *reinterpret_cast<U4 *>(to) = pack<F16>(h).w[0];
    *reinterpret_cast<U4 *>(to + 64) = pack<F16>(l).w[0];
}
__device__ __forceinline__ void get_pairs(const Pairs &p, int64_t row, int64_t col, float (&v)[8]) {
    const uint8_t *const from = octet_of(p, row, col);
    float l[8];
    unpack(Raw<F16>{{*reinterpret_cast<const U4 *>(from)}}, v);
    unpack(Raw<F16>{{*reinterpret_cast<const U4 *>(from + 64)}}, l);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += l[j];
}

// ---- before the steps
struct Start {
    const void *grad;
    float *momentum;
    int64_t grad_stride, rows, cols;
    float mu;
    int nesterov;
    double *squares;  // of a workgroup each
    int parts;
    float eps;
    Pairs straight, across;  // rows x cols, cols x rows
};
// u of an octet, from the gradient and the momentum as it is before (BEFORE) or after the step.
template <typename G, bool BEFORE> __device__ __forceinline__ void direction(const Start &f, int64_t row, int64_t col, float (&u)[8]) {
    const int64_t left = f.cols - col;
    unpack(load_row(static_cast<const G *>(f.grad) + row * f.grad_stride + col, left, col > 0), u);
    if (f.momentum == nullptr) return;
    float *const at = f.momentum + row * f.cols + col;
    float m[8];
    // (a row's last octet by itself: what stands before it is another lane's, which may be writing it)
    unpack(load_row(at, left, false), m);
    if constexpr (BEFORE) {
#pragma unroll
        for (int j = 0; j < 8; ++j) m[j] = __builtin_fmaf(f.mu, m[j], u[j]);
        store_row(at, left, pack<float>(m));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = f.nesterov != 0 ? __builtin_fmaf(f.mu, m[j], u[j]) : m[j];
}

// The momentum's step and the sum of u's squares.
constexpr int MIX_GROUPS = 1024;
template <typename G> __global__ __launch_bounds__(256) void k_muon_mix(Start f, Divisor per_row, uint32_t octets) {
    __shared__ double share[4];
    double sum = 0.0;
    for (uint32_t t = blockIdx.x * 256u + threadIdx.x; t < octets; t += gridDim.x * 256u) {
        const uint32_t row = per_row.quotient(t);
        float u[8];
        direction<G, true>(f, row, (t - row * per_row.d) * static_cast<int64_t>(8), u);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const double d = static_cast<double>(u[j]);
            sum = __builtin_fma(d, d, sum);
        }
    }
    sum = wave_sum(sum);
    if (threadIdx.x % 64 == 0) share[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0) f.squares[blockIdx.x] = ((share[0] + share[1]) + share[2]) + share[3];
}

// X's first pairs, both ways, in tiles of 64 x 64.
template <typename G> __global__ __launch_bounds__(256) void k_muon_start(Start f, int tiles_across) {
    __shared__ double share[4];
    __shared__ float tile[64][65];
    double sum = 0.0;
    for (int i = threadIdx.x; i < f.parts; i += 256) sum += f.squares[i];
    sum = wave_sum(sum);
    if (threadIdx.x % 64 == 0) share[threadIdx.x / 64] = sum;
    __syncthreads();
    const double factor = static_cast<double>(ONE) / (__builtin_sqrt(((share[0] + share[1]) + share[2]) + share[3]) + static_cast<double>(f.eps));
    const int64_t row0 = static_cast<int64_t>(blockIdx.x / tiles_across) * 64, col0 = static_cast<int64_t>(blockIdx.x % tiles_across) * 64;
    const int octet = threadIdx.x % 8;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = threadIdx.x / 8 + 32 * i;
        const int64_t row = row0 + r, col = col0 + octet * 8;
        float v[8] = {};
        if (row < f.rows && col < f.cols) direction<G, false>(f, row, col, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = static_cast<float>(static_cast<double>(v[j]) * factor);
            if (row >= f.rows || col + j >= f.cols) v[j] = 0.f;  // (of what is not there nothing, whatever the factor)
            tile[r][octet * 8 + j] = v[j];
        }
        if (row < f.rows) put_pairs(f.straight, row, col, f.cols, v);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = threadIdx.x / 8 + 32 * i;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = tile[octet * 8 + j][c];
        if (col0 + c < f.cols) put_pairs(f.across, col0 + c, row0 + octet * 8, f.rows, v);
    }
}

// ---- the steps' products
enum Mode { GRAM, POLY, NEXT, LAST, SHARE };  // A = X X^T; B = a I + b A + c A A; X = B X; w = decay w + scale B X; partial sums of A = X X^T
struct Product {
    Pairs a, b;             // operands: the result's [j][i], i of a's rows and j of b's
    int64_t rows_a, rows_b;
    int slices;             // of the whole sum
    int tiles_a, tiles_b, slices_per_split;
    Pairs by_j, by_i;       // the result as pairs, [j][i] and [i][j]
    Pairs gram;             // POLY: A
    float *partial;         // SHARE: [split][rows][rows]
    void *w;
    int64_t w_stride;
    float scale, decay;
};
struct Source {
    uint64_t a, b;
    int64_t pitch_a, pitch_b, left_a, left_b;
    __device__ __forceinline__ uint64_t at_a(int t) const { return a + static_cast<uint64_t>(t) * SLICE; }
    __device__ __forceinline__ uint64_t at_b(int t) const { return b + static_cast<uint64_t>(t) * SLICE; }
};

template <Mode MODE, typename T, typename Tile, int PER_CU> __global__ __launch_bounds__(Tile::NT, PER_CU * Tile::WAVES / 4) void k_muon_product(Product f) {
    constexpr int MI = Tile::MI, NI = Tile::NI;
    constexpr int PITCH = MI * 32 + 4;  // floats from one j's results to the next in LDS
    constexpr int RESULTS = Tile::WAVES * 32 * PITCH * 4;
    constexpr bool SYMMETRIC = MODE == GRAM || MODE == POLY;
    __shared__ __attribute__((aligned(16))) char lds[Tile::LDS > RESULTS ? Tile::LDS : RESULTS];
    int b = place(blockIdx.x, gridDim.x), part = 0, tile_a, tile_b;
    if constexpr (SYMMETRIC) {  // tiles on and to one side of the diagonal: row b has b + 1
        tile_b = static_cast<int>((__builtin_sqrtf(8.f * static_cast<float>(b) + 1.f) - 1.f) * 0.5f);
        while (tile_b * (tile_b + 1) / 2 > b) --tile_b;
        while ((tile_b + 1) * (tile_b + 2) / 2 <= b) ++tile_b;
        tile_a = b - tile_b * (tile_b + 1) / 2;
    } else {
        part = b / (f.tiles_a * f.tiles_b);
        tile_at(b - part * f.tiles_a * f.tiles_b, f.tiles_a, f.tiles_b, tile_a, tile_b);
    }
    const int64_t a0 = static_cast<int64_t>(tile_a) * Tile::BM, b0 = static_cast<int64_t>(tile_b) * Tile::BN;
    const int first = part * f.slices_per_split, slices = f.slices - first < f.slices_per_split ? f.slices - first : f.slices_per_split;
    const Source source{reinterpret_cast<uint64_t>(f.a.at + a0 * f.a.pitch + first * static_cast<int64_t>(SLICE)),
                        reinterpret_cast<uint64_t>(f.b.at + b0 * f.b.pitch + first * static_cast<int64_t>(SLICE)), f.a.pitch, f.b.pitch,
                        f.rows_a - a0 < Tile::BM ? f.rows_a - a0 : Tile::BM, f.rows_b - b0 < Tile::BN ? f.rows_b - b0 : Tile::BN};
    F16v acc[MI][NI] = {};
    Tile::run(lds, source, slices, acc);
    __syncthreads();  // the buffers have been read

    // Results through LDS, 32 j of a wavefront at a time: rows of either matrix are written sixteen bytes and more at a time.
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wm = wave / Tile::WN, wn = wave % Tile::WN;
    float *const mine = reinterpret_cast<float *>(lds) + wave * 32 * PITCH;
    constexpr int OCTETS = MI * 4, AT_ONCE = 64 / OCTETS;
    const int octet = lane % OCTETS, line = lane / OCTETS;
    const int64_t i_at = a0 + wm * (Tile::BM / Tile::WM);
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int64_t j_at = b0 + wn * (Tile::BN / Tile::WN) + n * 32;
#pragma unroll
        for (int m = 0; m < MI; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                typedef float F4 __attribute__((ext_vector_type(4)));
                *reinterpret_cast<F4 *>(mine + lane % 32 * PITCH + m * 32 + q * 8 + lane / 32 * 4) =
                    F4{acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]};
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int k = 0; k < 32; k += AT_ONCE) {
            const int64_t j = j_at + k + line, i = i_at + octet * 8;
            U4 *const at = reinterpret_cast<U4 *>(mine + (k + line) * PITCH + octet * 8);
            float v[8];
            unpack(Raw<float>{{at[0], at[1]}}, v);
            if (j >= f.rows_b) continue;
            if constexpr (MODE == GRAM) {
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] *= 1.f / ONE;
                put_pairs(f.by_j, j, i, f.rows_a, v);
            } else if constexpr (MODE == POLY) {
                float gram[8] = {};
                if (i < padded(f.rows_a)) get_pairs(f.gram, j, i, gram);
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    v[x] = __builtin_fmaf(v[x], NS_C * (ONE_OF_B / ONE / ONE), gram[x] * (NS_B * (ONE_OF_B / ONE)));
                    if (i + x == j) v[x] += NS_A * ONE_OF_B;
                }
                put_pairs(f.by_j, j, i, f.rows_a, v);
                if (tile_a != tile_b) {
                    const Raw<float> r = pack<float>(v);
                    at[0] = r.w[0];
                    at[1] = r.w[1];
                }
            } else if constexpr (MODE == NEXT) {
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] *= 1.f / ONE_OF_B;
                put_pairs(f.by_j, j, i, f.rows_a, v);
            } else if constexpr (MODE == SHARE) {
                if (i < f.rows_a) store_row(f.partial + (part * f.rows_b + j) * f.rows_a + i, f.rows_a - i, Raw<float>{{at[0], at[1]}});
            } else {
                if (i >= f.rows_a) continue;
                T *const to = static_cast<T *>(f.w) + j * f.w_stride + i;
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] *= f.scale * (1.f / ONE / ONE_OF_B);
                if (f.decay != 0.f) {
                    float old[8];
                    unpack(load_row(to, f.rows_a - i, false), old);
#pragma unroll
                    for (int x = 0; x < 8; ++x) v[x] = __builtin_fmaf(f.decay, old[x], v[x]);
                }
                store_row(to, f.rows_a - i, pack<T>(v));
            }
        }
        if constexpr (MODE == LAST || MODE == SHARE) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            continue;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (!SYMMETRIC || tile_a != tile_b) {
#pragma unroll
            for (int k = 0; k < 2 * MI; ++k) {  // an octet of j for an i
                const int item = k * 64 + lane, i = item % (MI * 32), eight = item / (MI * 32) * 8;
                float v[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] = mine[(eight + x) * PITCH + i];
                if (i_at + i >= f.rows_a) continue;
                if constexpr (MODE != POLY)
#pragma unroll
                    for (int x = 0; x < 8; ++x) v[x] *= MODE == GRAM ? 1.f / ONE : 1.f / ONE_OF_B;
                put_pairs(f.by_i, i_at + i, j_at + eight, f.rows_b, v);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// The shares of A added up in order.
__global__ __launch_bounds__(256) void k_muon_join(const float *partial, int split, int64_t n, Pairs to, Divisor per_row, uint32_t octets) {
    const uint32_t t = blockIdx.x * 256u + threadIdx.x;
    if (t >= octets) return;
    const uint32_t row = per_row.quotient(t);
    const int64_t col = (t - row * per_row.d) * static_cast<int64_t>(8);
    float v[8] = {};
    for (int s = 0; s < split; ++s) {
        float p[8];
        unpack(load_row(partial + (s * n + row) * n + col, n - col, col > 0), p);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += p[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= 1.f / ONE;
    put_pairs(to, row, col, n, v);
}

using Large = RowTile<PAIRS, 256, 256, 2, 2, 2>;
using Middle = RowTile<PAIRS, 128, 128, 2, 2, 2>;
using Small = RowTile<PAIRS, 64, 64, 2, 2, 3>;

// Which tile, and for the product of X with itself how many shares of the sum.
struct Choice {
    int side, split, per;
};
constexpr int SPLIT_MAX = 32;
Choice choice_of(int64_t rows_a, int64_t rows_b, int64_t sum, bool symmetric, bool shares) {
    Choice best{0, 1, 0};
    double least = 0;
    const int slices = static_cast<int>(padded(sum) / 32);
    for (const int side : {256, 128, 64}) {
        const int64_t a = (rows_a + side - 1) / side, b = (rows_b + side - 1) / side;
        const int units = side == 256 ? 256 : side == 128 ? 512 : 768;
        const double step = side == 256 ? 1.6 : side == 128 ? 0.9 : 0.35, beside = side == 256 ? 10. : side == 128 ? 6. : 4.;
        for (int split = 1; split <= (shares ? SPLIT_MAX : 1) && split <= slices; ++split) {
            const int per = (slices + split - 1) / split;
            if ((slices + per - 1) / per != split) continue;
            const int64_t tiles = (symmetric && split == 1 ? a * (a + 1) / 2 : a * b) * split;
            const double rounds = static_cast<double>((tiles + units - 1) / units);
            const double cost = rounds * (beside + step * per) + (split == 1 ? 0. : 4. + 0.4e-6 * 4. * split * static_cast<double>(rows_a * rows_b));
            if (best.side == 0 || cost < least) {
                least = cost;
                best = Choice{side, split, per};
            }
        }
    }
    return best;
}

template <Mode MODE, typename T> void launch_product(Product f, int side, int split, hipStream_t st) {
    f.tiles_a = static_cast<int>((f.rows_a + side - 1) / side);
    f.tiles_b = static_cast<int>((f.rows_b + side - 1) / side);
    const int64_t tiles = MODE == GRAM || MODE == POLY ? static_cast<int64_t>(f.tiles_a) * (f.tiles_a + 1) / 2 : static_cast<int64_t>(f.tiles_a) * f.tiles_b * split;
    const dim3 groups(static_cast<unsigned>(tiles));
    if (side == 256)
        hipLaunchKernelGGL((k_muon_product<MODE, T, Large, 1>), groups, dim3(Large::NT), 0, st, f);
    else if (side == 128)
        hipLaunchKernelGGL((k_muon_product<MODE, T, Middle, 2>), groups, dim3(Middle::NT), 0, st, f);
    else
        hipLaunchKernelGGL((k_muon_product<MODE, T, Small, 3>), groups, dim3(Small::NT), 0, st, f);
}

constexpr int64_t MAX_SIDE = 1 << 16, MAX_STEPS = 64;
bool update_ok(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 0 && rows <= MAX_SIDE && cols <= MAX_SIDE && rows * cols < (static_cast<int64_t>(1) << 31); }

// The workspace: X and, twice, X transposed; A, B; partial sums.
struct Workspace {
    size_t x, xt[2], gram, poly, squares, shares, bytes;
    Choice for_gram;
};
Workspace workspace_of(int64_t less, int64_t more) {
    Workspace w{};
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += adatopk_internal::align_up(bytes, 256);
        return here;
    };
    w.x = take(pairs_bytes(less, more));
    w.xt[0] = take(pairs_bytes(more, less));
    w.xt[1] = take(pairs_bytes(more, less));
    w.gram = take(pairs_bytes(less, less));
    w.poly = take(pairs_bytes(less, less));
    w.squares = take(MIX_GROUPS * sizeof(double));
    w.for_gram = choice_of(less, less, more, true, true);
    w.shares = take(w.for_gram.split == 1 ? 0 : static_cast<size_t>(w.for_gram.split) * static_cast<size_t>(less) * static_cast<size_t>(less) * sizeof(float));
    w.bytes = at;
    return w;
}

}  // namespace

extern "C" {

size_t adatopk_muon_update_workspace_bytes(int64_t rows, int64_t cols) {
    if (!update_ok(rows, cols) || rows == 0 || cols == 0) return 0;
    return workspace_of(rows < cols ? rows : cols, rows < cols ? cols : rows).bytes;
}

adatopk_status adatopk_muon_update(const void *grad, int64_t grad_stride, adatopk_dtype grad_dt, float *momentum, float mu, int32_t nesterov, int64_t rows,
                                   int64_t cols, int32_t steps, float eps, void *w, int64_t w_stride, adatopk_dtype dt, float scale, float decay,
                                   void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!dtype_ok(grad_dt) || !dtype_ok(dt) || !update_ok(rows, cols) || steps < 1 || steps > MAX_STEPS || !(eps >= 0.f)) return ADATOPK_EINVAL;
    if (rows == 0 || cols == 0) return ADATOPK_OK;
    if (!matrix_ok(grad, grad_stride, rows, cols, grad_dt) || !matrix_ok(w, w_stride, rows, cols, dt) || !pointer_ok_or_null(momentum, 4) || !pointer_ok(workspace, 256))
        return ADATOPK_EINVAL;
    const bool wide = rows <= cols;
    const int64_t less = wide ? rows : cols, more = wide ? cols : rows;
    const Workspace at = workspace_of(less, more);
    if (workspace_bytes < at.bytes) return ADATOPK_EWORKSPACE;
    uint8_t *const base = static_cast<uint8_t *>(workspace);
    const auto pairs = [&](size_t where, int64_t of) { return Pairs{base + where, padded(of) * 4}; };
    const Pairs x = pairs(at.x, more), gram = pairs(at.gram, less), poly = pairs(at.poly, less);
    Pairs xt = pairs(at.xt[0], less), xt_next = pairs(at.xt[1], less);
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);

    const int64_t per_row = (cols + 7) / 8, octets = rows * per_row;
    const unsigned mix = static_cast<unsigned>((octets + 255) / 256 < MIX_GROUPS ? (octets + 255) / 256 : MIX_GROUPS);
    const Start start{grad, momentum, grad_stride, rows, cols, mu, nesterov, reinterpret_cast<double *>(base + at.squares), static_cast<int>(mix), eps,
                      wide ? x : xt, wide ? xt : x};
    const int64_t across = (cols + 63) / 64, tiles = across * ((rows + 63) / 64);
    with_type(grad_dt, [&](auto *null) {
        using G = std::remove_pointer_t<decltype(null)>;
        hipLaunchKernelGGL(k_muon_mix<G>, dim3(mix), dim3(256), 0, st, start, Divisor(static_cast<uint32_t>(per_row)), static_cast<uint32_t>(octets));
        hipLaunchKernelGGL(k_muon_start<G>, dim3(static_cast<unsigned>(tiles)), dim3(256), 0, st, start, static_cast<int>(across));
    });

    const int along = static_cast<int>(padded(more) / 32), side = static_cast<int>(padded(less) / 32);
    const int poly_tile = choice_of(less, less, less, true, false).side, next_tile = choice_of(less, more, less, false, false).side;
    for (int step = 0; step < steps; ++step) {
        Product p{};
        p.a = p.b = x;
        p.rows_a = p.rows_b = less;
        p.slices = along;
        p.slices_per_split = at.for_gram.per;
        p.by_j = p.by_i = gram;
        if (at.for_gram.split == 1) {
            launch_product<GRAM, float>(p, at.for_gram.side, 1, st);
        } else {
            p.partial = reinterpret_cast<float *>(base + at.shares);
            launch_product<SHARE, float>(p, at.for_gram.side, at.for_gram.split, st);
            const int64_t row_octets = padded(less) / 8;
            const uint32_t all = static_cast<uint32_t>(less * row_octets);
            hipLaunchKernelGGL(k_muon_join, dim3((all + 255) / 256), dim3(256), 0, st, p.partial, at.for_gram.split, less, gram,
                               Divisor(static_cast<uint32_t>(row_octets)), all);
        }
        p.a = p.b = p.gram = gram;
        p.slices = p.slices_per_split = side;
        p.by_j = p.by_i = poly;
        launch_product<POLY, float>(p, poly_tile, 1, st);
        if (step + 1 < steps) {
            p.a = poly;
            p.b = xt;
            p.rows_b = more;
            p.by_j = xt_next;
            p.by_i = x;
            launch_product<NEXT, float>(p, next_tile, 1, st);
            const Pairs t = xt;
            xt = xt_next;
            xt_next = t;
        } else {  // w's rows along the first operand
            p.a = wide ? xt : poly;
            p.b = wide ? poly : xt;
            p.rows_a = cols;
            p.rows_b = rows;
            p.w = w;
            p.w_stride = w_stride;
            p.scale = scale;
            p.decay = decay;
            with_type(dt, [&](auto *null) {
                using T = std::remove_pointer_t<decltype(null)>;
                launch_product<LAST, T>(p, next_tile, 1, st);
            });
        }
    }
    return launched();
}

}  // extern "C"
