// A weight matrix changed by its orthogonalised gradient, as the optimiser Muon does.
//
//   m = mu m + g;  u = m, or g + mu m;  X = u / (|u| + eps);  in each step A = X X^T, B = a I + b A + c A A, X = B X;  w = decay w + scale X
//
// with the Frobenius norm and a, b, c = 3.4445, -4.7750, 2.0315, which take singular values from 0 ... 1 to 0.7 ... 1.2 in five steps.  X is taken with its shorter side
// first (transposed where that is the other).  A step is three products of matrices whose rows lie along the sum: A from X twice, A A from A twice since A is
// symmetric, and X from B and X transposed, so each step writes X both ways; of A and B half the tiles are computed and written twice.
//
// Small singular values grow 3.4-fold in each step, and so does what a rounding of X leaves in their directions: with X in bf16 the result is some 2 to 7 % off, in
// one fp16 1e-3 to 6e-3 (512 to 1000 rows, of noise and of low rank with noise; 2-norm of the error, relative), in two fp16 2e-7 to 7e-6, like fp32 (256 to 1600
// rows, few rows with all else nothing among them).  So everything between the steps is two fp16, h + l, times 2^14 (A and X stay within 1.5, X's singular values
// within 1.21: nothing overflows, and l keeps its bits down to 2^-17) or, for B, whose diagonal reaches 3.45, 2^13.  Products are three of the matrix instruction's, sums
// fp32; |u| is a 64-bit sum.
//
// Coarse steps, where the caller asks for them and w has 16 bits.  With B X = a X + (b A + c A A) X only the first term matters where singular values are small: a step
// whose a X is added in the full 22 bits and whose products are of the h alone leaves errors of some 2^-12 in directions that are large.  So they are the first ones, two
// for fp16 and three for bf16, as far as three (two) others come behind; counted from the end, updates of more than five steps had them where singular values are near 1, and
// noise was 4e-3 off after eight steps instead of 2e-5 (512 x 1024, fp16).  How much of them the steps behind level is the gradient's affair: five steps are 5e-6 off in fp16 on noise of
// 1600 rows, but 3e-3 where five rows are all there is; in bf16, whose last product is of the h alone too, 5e-4 to 4e-3.  That is more than w's own rounding (2e-4 and
// 1.7e-3 in the 2-norm), so nobody gets it unasked.  With fewer than 256 rows less is levelled and products are not what takes the time: there all steps take the full 22 bits.
//
// Measured, five steps, us, and with coarse steps for bf16 and fp16 weights: 768 x 768 168 (140, 155); 1024 x 4096 372 (258, 317); 1600 x 6400 921 (613, 781); 4096 x 4096 3885
// (2200, 3057).  Of the largest the matrix unit's share at a library product's rate is 3.2 ms (1.5, 2.4).  What bounds the rest: a B X writes X twice at the end of its one
// round of tiles, with nothing to cover it; small matrices' products are 10 us each whatever they compute, start, six slices' latency and end, and each needs the
// one before.
#include <hip/hip_runtime.h>

#ifdef ADATOPK_MEASURE_BUILD
#include "adatopk_measure.h"
#endif
#include "row_tiles.h"

// Products and sums are fused where the code says so and nowhere else.
#pragma clang fp contract(off)

namespace {

using namespace adatopk_stage;

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float ONE = 16384.f, ONE_OF_B = 8192.f;  // what 1 is held as

// A matrix of pairs: rows of 2^run h and then their l, and so on, padded with zeros.  Runs of 32 where products take both (128 bytes are 32 elements), of 64 where
// they take the h alone (128 bytes are 64, and the other half of no line is fetched with them).
struct Pairs {
    uint8_t *at;
    int64_t pitch;
    int run;
    bool halves;  // only h are written: nobody reads the l
};
constexpr int run_for(bool high) { return high ? 6 : 5; }
constexpr int64_t padded(int64_t n) { return (n + 63) / 64 * 64; }
inline size_t pairs_bytes(int64_t rows, int64_t cols) { return adatopk_internal::align_up(static_cast<size_t>(rows) * static_cast<size_t>(padded(cols)) * 4, 256); }

__device__ __forceinline__ uint8_t *octet_of(const Pairs &p, int64_t row, int64_t col) {
    return p.at + row * p.pitch + ((col >> p.run) << (p.run + 2)) + (col & ((1 << p.run) - 1)) * 2;
}
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
    if (!p.halves) *reinterpret_cast<U4 *>(to + (2 << p.run)) = pack<F16>(l).w[0];
}
__device__ __forceinline__ Raw<float> fetch_pairs(const Pairs &p, int64_t row, int64_t col) {
    const uint8_t *const from = octet_of(p, row, col);
    return Raw<float>{{*reinterpret_cast<const U4 *>(from), *reinterpret_cast<const U4 *>(from + (2 << p.run))}};
}
__device__ __forceinline__ void unpack_pairs(const Raw<float> &pairs, float (&v)[8]) {
    float l[8];
    unpack(Raw<F16>{{pairs.w[0]}}, v);
    unpack(Raw<F16>{{pairs.w[1]}}, l);
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
enum Mode { GRAM, POLY, NEXT, LAST, SHARE };  // A = X X^T; B = a I + b A + c A A; X = B X; w = decay w + scale B X; partial sums of X X^T or A A
struct Product {
    Pairs a, b;             // operands: the result's [j][i], i of a's rows and j of b's
    int64_t rows_a, rows_b;
    int slices;             // of the whole sum
    int tiles_a, tiles_b, tiles, slices_per_split;
    Pairs by_j, by_i;       // the result as pairs, [j][i] and [i][j]
    Pairs gram;             // POLY: A
    Pairs old_by_j, old_by_i;  // NEXT from the h alone: X as it was
    float diagonal;         // POLY: a, or nothing where X a is added apart
    float *partial;         // SHARE: [share][tile on and to one side of the diagonal][j][i], whole tiles
    void *w;
    int64_t w_stride;
    float scale, decay;
};
struct Source {
    uint64_t a, b;
    int64_t pitch_a, pitch_b, left_a, left_b;
};

// Tiles on and to one side of the diagonal, row by row: row b has b + 1.
__device__ __forceinline__ void tile_below(int tile, int &a, int &b) {
    b = static_cast<int>((__builtin_sqrtf(8.f * static_cast<float>(tile) + 1.f) - 1.f) * 0.5f);
    while (b * (b + 1) / 2 > tile) --b;
    while ((b + 1) * (b + 2) / 2 <= tile) ++b;
    a = tile - b * (b + 1) / 2;
}
// B's elements from A's and A A's, both as they are held: i and the seven behind it of row j.
__device__ __forceinline__ void polynomial(const Product &f, int64_t j, int64_t i, float (&v)[8]) {
    float gram[8] = {};
    if (j < f.rows_b && i < padded(f.rows_a)) unpack_pairs(fetch_pairs(f.gram, j, i), gram);
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        v[x] = __builtin_fmaf(v[x], NS_C * (ONE_OF_B / ONE / ONE), gram[x] * (NS_B * (ONE_OF_B / ONE)));
        if (i + x == j) v[x] += f.diagonal * ONE_OF_B;
    }
}

template <Mode MODE, typename T, typename Tile, int PER_CU> __global__ __launch_bounds__(Tile::NT, PER_CU * Tile::NT / 256) void k_muon_product(Product f) {
    constexpr int MI = Tile::MI, NI = Tile::NI;
    constexpr int PITCH = MI * 32 + 4;  // floats from one j's results to the next in LDS
    constexpr int RESULTS = Tile::WAVES * 32 * PITCH * 4;
    static_assert(Tile::ALONG == 1 || Tile::BN * PITCH * 4 <= Tile::GROUP_LDS, "a group's results fit its buffers");
    constexpr bool SYMMETRIC = MODE == GRAM || MODE == POLY || MODE == SHARE;
    __shared__ __attribute__((aligned(16))) char lds[Tile::LDS > RESULTS ? Tile::LDS : RESULTS];
    int b = place(blockIdx.x, gridDim.x), part = 0, tile_a, tile_b;
    if constexpr (SYMMETRIC) {
        part = b / f.tiles;
        b -= part * f.tiles;
        tile_below(b, tile_a, tile_b);
    } else {
        tile_at(b, f.tiles_a, f.tiles_b, tile_a, tile_b);
    }
    const int64_t a0 = static_cast<int64_t>(tile_a) * Tile::BM, b0 = static_cast<int64_t>(tile_b) * Tile::BN;
    const int first = part * f.slices_per_split, slices = f.slices - first < f.slices_per_split ? f.slices - first : f.slices_per_split;
    const Source source{reinterpret_cast<uint64_t>(f.a.at + a0 * f.a.pitch + first * static_cast<int64_t>(Tile::STRIDE)),
                        reinterpret_cast<uint64_t>(f.b.at + b0 * f.b.pitch + first * static_cast<int64_t>(Tile::STRIDE)), f.a.pitch, f.b.pitch,
                        f.rows_a - a0 < Tile::BM ? f.rows_a - a0 : Tile::BM, f.rows_b - b0 < Tile::BN ? f.rows_b - b0 : Tile::BN};
    F16v acc[MI][NI] = {};
    Tile::run(lds, source, slices, acc);
    __syncthreads();  // the buffers have been read

    // What eight results are added to: X as it was, or w.
    constexpr bool TO_X = MODE == NEXT && Tile::FORM == HIGH, TO_W = MODE == LAST;
    const auto before = [&](int64_t j, int64_t i) {
        if constexpr (TO_W) {
            return fetch_row(static_cast<const T *>(f.w) + j * f.w_stride + i, f.decay != 0.f && j < f.rows_b ? f.rows_a - i : 0, false);
        } else {
            Raw<float> old{};
            if (TO_X && j < f.rows_b && i < padded(f.rows_a)) old = fetch_pairs(f.old_by_j, j, i);
            return old;
        }
    };
    // Eight results of a j, i and the seven behind it: what becomes of them, and there they are for the other way of writing them.
    const auto finish = [&](int64_t j, int64_t i, float (&v)[8], const auto &before) {
        if constexpr (MODE == GRAM || MODE == NEXT) {
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x] *= MODE == GRAM ? 1.f / ONE : 1.f / ONE_OF_B;
            if constexpr (TO_X) {
                float old[8];
                unpack_pairs(before, old);
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] = __builtin_fmaf(NS_A, old[x], v[x]);
            }
            if (j < f.rows_b) put_pairs(f.by_j, j, i, f.rows_a, v);
        } else if constexpr (MODE == POLY) {
            polynomial(f, j, i, v);
            if (j < f.rows_b) put_pairs(f.by_j, j, i, f.rows_a, v);
        } else if constexpr (MODE == SHARE) {
            float *const to = f.partial + ((static_cast<int64_t>(part) * f.tiles + b) * Tile::BN + (j - b0)) * Tile::BM + (i - a0);
            store_row(to, 8, pack<float>(v));
        } else if (j < f.rows_b && i < f.rows_a) {
            T *const to = static_cast<T *>(f.w) + j * f.w_stride + i;
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x] *= f.scale * (1.f / ONE / ONE_OF_B);
            if (f.decay != 0.f) {
                float old[8];
                unpack(before, old);
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] = __builtin_fmaf(f.decay, old[x], v[x]);
            }
            store_row(to, f.rows_a - i, pack<T>(v));
        }
    };
    const bool both = MODE == NEXT || (MODE != SHARE && SYMMETRIC && tile_a != tile_b);  // whether [i][j] is written too

    // Results through LDS: rows of either matrix are written sixteen bytes and more at a time.
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wm = wave % Tile::WAVES / Tile::WN, wn = wave % Tile::WN;
    const auto lay = [&](float *to, int n) {  // a wavefront's results of 32 j
#pragma unroll
        for (int m = 0; m < MI; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                typedef float F4 __attribute__((ext_vector_type(4)));
                *reinterpret_cast<F4 *>(to + lane % 32 * PITCH + m * 32 + q * 8 + lane / 32 * 4) =
                    F4{acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]};
            }
    };
    constexpr int OCTETS = MI * 4;
    if constexpr (Tile::ALONG > 1) {  // the groups' sums, added up in their order; the workgroup goes through the tile together
        constexpr int STEP = Tile::GROUP_LDS / 4;  // floats from one group's to the next
        float *const sums = reinterpret_cast<float *>(lds);
#pragma unroll
        for (int n = 0; n < NI; ++n) lay(sums + wave * STEP + n * 32 * PITCH, n);
        __syncthreads();
#pragma unroll 2
        for (int item = threadIdx.x; item < Tile::BN * OCTETS; item += Tile::NT) {
            const int j = item / OCTETS, i = item % OCTETS * 8;
            float v[8] = {};
#pragma unroll
            for (int g = 0; g < Tile::ALONG; ++g) {
                const U4 *const at = reinterpret_cast<const U4 *>(sums + g * STEP + j * PITCH + i);
                float t[8];
                unpack(Raw<float>{{at[0], at[1]}}, t);
#pragma unroll
                for (int x = 0; x < 8; ++x) v[x] += t[x];
            }
            finish(b0 + j, a0 + i, v, before(b0 + j, a0 + i));
            if (both) {
                const Raw<float> r = pack<float>(v);
                U4 *const at = reinterpret_cast<U4 *>(sums + j * PITCH + i);
                at[0] = r.w[0];
                at[1] = r.w[1];
            }
        }
        if constexpr (MODE == LAST || MODE == SHARE) return;
        if (!both) return;
        __syncthreads();
#pragma unroll 2
        for (int item = threadIdx.x; item < Tile::BM * (Tile::BN / 8); item += Tile::NT) {
            const int i = item / 4 % Tile::BM, eight = (item / 4 / Tile::BM * 4 + item % 4) * 8;
            float v[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x] = sums[(eight + x) * PITCH + i];
            if (a0 + i < f.rows_a) put_pairs(f.by_i, a0 + i, b0 + eight, f.rows_b, v);
        }
    } else {
        const auto together = [] {  // (a wavefront's lanes read what others of them have written)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
        float *const mine = reinterpret_cast<float *>(lds) + wave * 32 * PITCH;
        const int64_t i_at = a0 + wm * (Tile::BM / Tile::WM), j_first = b0 + wn * (Tile::BN / Tile::WN);
        // What the next 32 j's results are added to is asked for while the last ones' are written.
        constexpr int ITEMS = OCTETS / 2, TOGETHER = TO_X || TO_W ? ITEMS : 2;
        decltype(before(0, 0)) old[TO_X || TO_W ? ITEMS : 1];
        const auto ask = [&](int n) {
            if constexpr (TO_X || TO_W)
#pragma unroll
                for (int k = 0; k < ITEMS; ++k) old[k] = before(j_first + n * 32 + (lane + 64 * k) / OCTETS, i_at + (lane + 64 * k) % OCTETS * 8);
        };
        ask(0);
#pragma unroll
        for (int n = 0; n < NI; ++n) {
            const int64_t j_at = j_first + n * 32;
            lay(mine, n);
            together();
#pragma unroll TOGETHER
            for (int which = 0; which < ITEMS; ++which) {
                const int item = lane + 64 * which, k = item / OCTETS, octet = item % OCTETS;
                U4 *const at = reinterpret_cast<U4 *>(mine + k * PITCH + octet * 8);
                float v[8];
                unpack(Raw<float>{{at[0], at[1]}}, v);
                finish(j_at + k, i_at + octet * 8, v, old[TO_X || TO_W ? which : 0]);
                if (both) {
                    const Raw<float> r = pack<float>(v);
                    at[0] = r.w[0];
                    at[1] = r.w[1];
                }
            }
            together();
            if (n + 1 < NI) ask(n + 1);
            if constexpr (MODE != LAST && MODE != SHARE) {
                if (both) {
#pragma unroll 2
                    for (int item = lane; item < MI * 128; item += 64) {  // an octet of j for an i; four lanes write 64 bytes of h, then of l
                        const int i = item / 4, eight = item % 4 * 8;
                        float v[8];
#pragma unroll
                        for (int x = 0; x < 8; ++x) v[x] = mine[(eight + x) * PITCH + i];
                        if (i_at + i < f.rows_a) put_pairs(f.by_i, i_at + i, j_at + eight, f.rows_b, v);
                    }
                    together();
                }
            }
        }
    }
}

// The shares of a symmetric product added up in order, 64 x 64 of a tile per workgroup, and what becomes of them (MODE: GRAM or POLY).
template <Mode MODE> __global__ __launch_bounds__(256) void k_muon_join(Product f, int split, int side) {
    __shared__ float tile[64][65];
    const int per = side / 64, b = blockIdx.x / (per * per), sub = blockIdx.x % (per * per);
    int tile_a, tile_b;
    tile_below(b, tile_a, tile_b);
    const int64_t i0 = sub % per * 64, j0 = sub / per * 64, a0 = static_cast<int64_t>(tile_a) * side + i0, b0 = static_cast<int64_t>(tile_b) * side + j0;
    const bool both = tile_a != tile_b;
    const int octet = threadIdx.x % 8;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int line = threadIdx.x / 8 + 32 * n;
        const float *from = f.partial + (static_cast<int64_t>(b) * side + j0 + line) * side + i0 + octet * 8;
        float v[8] = {};
#pragma unroll 4
        for (int s = 0; s < split; ++s) {
            float t[8];
            unpack(load_octet(from + static_cast<int64_t>(s) * f.tiles * side * side), t);
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x] += t[x];
        }
        if constexpr (MODE == GRAM) {
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x] *= 1.f / ONE;
        } else {
            polynomial(f, b0 + line, a0 + octet * 8, v);
        }
        if (b0 + line < f.rows_b) put_pairs(f.by_j, b0 + line, a0 + octet * 8, f.rows_a, v);
        if (both)
#pragma unroll
            for (int x = 0; x < 8; ++x) tile[line][octet * 8 + x] = v[x];
    }
    if (!both) return;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int line = threadIdx.x / 8 + 32 * n;
        float v[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] = tile[octet * 8 + x][line];
        if (a0 + line < f.rows_a) put_pairs(f.by_i, a0 + line, b0 + octet * 8, f.rows_b, v);
    }
}

// Tiles that there are kernels for.
enum Shape { SHAPE_256, SHAPE_192, SHAPE_160, SHAPE_128, SHAPE_64, SHAPES };
constexpr int SHAPE_BM[SHAPES] = {256, 192, 160, 128, 64}, SHAPE_BN[SHAPES] = {256, 256, 256, 128, 64}, SHAPE_SLOTS[SHAPES] = {256, 256, 256, 512, 768};
template <Kind KIND> struct Tiles {
    using Of256 = RowTile<KIND, 256, 256, 2, 4, 2>;
    using Of192 = RowTile<KIND, 192, 256, 2, 4, 2>;
    using Of160 = RowTile<KIND, 160, 256, 1, 4, 2>;
    using Of128 = RowTile<KIND, 128, 128, 2, 2, 2>;
    using Of64 = RowTile<KIND, 64, 64, 2, 2, 3>;
    using Deep64 = RowTile<KIND, 64, 64, 1, 1, 2, 4>;  // where every tile has a compute unit to itself
};

// Which tile, whether the operands change places (then i is the second one's row), and for symmetric products how many shares of the sum.
struct Choice {
    Shape shape;
    bool high, turned;
    int split, per;
};
constexpr int SPLIT_MAX = 16;
// us: of a slice on a full chip, from pairs (32 elements) and from the h alone (64), and what a workgroup takes beside its slices.  Measured on 1600 x 6400: X = B X
// from pairs 129, 115, 104, 115, 135 us by tile, from the h alone 83, 72, 74, 74, 75, written as w 59, 50, 51, 57, 68; X X^T from pairs (with the join) 80, -, -,
// 68, 82, from the h alone 48, -, -, 38, 46; A A 45, -, -, 35, 30 and 28, -, -, 26, 22.  (64 from pairs .76 for .72 after 1024 x 4096 fp32: 400 us, 367 with tiles of 128.  At other
// sizes the choice follows from these costs and has not been measured against the others.)
constexpr double STEP[2][SHAPES] = {{2.3, 2.05, 1.85, 1.45, 0.76}, {2.0, 1.95, 2.1, 1.5, 1.1}}, BESIDE[SHAPES] = {14., 12., 11., 8., 5.};
constexpr double DEEP_STEP = 0.17;  // of Deep64
enum Writes { HALF, X, X_AS_IT_LIES, W };  // a symmetric matrix; X, either operand first or the first one; w
Choice choice_of(int64_t rows_a, int64_t rows_b, int64_t sum, Writes writes, bool high) {
    const bool symmetric = writes == HALF, x = writes == X || writes == X_AS_IT_LIES;
    Choice best{SHAPES, high, false, 1, 0};
    double least = 0;
    const int slices = static_cast<int>(padded(sum) / (high ? 64 : 32));
    for (int t = 0; t < SHAPES; ++t)
        for (int turned = 0; turned < (writes == X && SHAPE_BM[t] != SHAPE_BN[t] ? 2 : 1); ++turned) {
            if (symmetric && SHAPE_BM[t] != SHAPE_BN[t]) continue;
            // X's tiles have to reach to the end of its last 64, whose zeros they write
            if (x && padded(turned ? rows_b : rows_a) > ((turned ? rows_b : rows_a) + SHAPE_BM[t] - 1) / SHAPE_BM[t] * SHAPE_BM[t]) continue;
            const int64_t a = ((turned ? rows_b : rows_a) + SHAPE_BM[t] - 1) / SHAPE_BM[t], b = ((turned ? rows_a : rows_b) + SHAPE_BN[t] - 1) / SHAPE_BN[t];
            for (int split = 1; split <= (symmetric ? SPLIT_MAX : 1) && split <= slices; ++split) {
                const int per = (slices + split - 1) / split;
                if ((slices + per - 1) / per != split) continue;
                const int64_t tiles = (symmetric ? a * (a + 1) / 2 : a * b) * split;
                const bool deep = t == SHAPE_64 && tiles <= 256;
                if (symmetric && high && t == SHAPE_64 && split == 1 && !deep) continue;  // never the least over the sizes that there are: no kernel
                const double filled = static_cast<double>(tiles) / SHAPE_SLOTS[t];
                // workgroups that share a compute unit slow one another down, and their rounds run into one another
                const bool shared = SHAPE_SLOTS[t] > 256;
                const double rounds = shared ? (filled < 1. ? 1. : 1.1 * filled) : static_cast<double>((tiles + SHAPE_SLOTS[t] - 1) / SHAPE_SLOTS[t]);
                const double step = deep ? DEEP_STEP : STEP[high][t] * (shared && filled < 1. ? 0.5 + 0.5 * filled : 1.);
                const double join = split == 1 ? 0. : 4. + 0.17e-6 * 4. * static_cast<double>(tiles) * SHAPE_BM[t] * SHAPE_BN[t];
                const double cost = rounds * (BESIDE[t] + step * per) + join;
                if (best.shape == SHAPES || cost < least) {
                    least = cost;
                    best = Choice{static_cast<Shape>(t), high, turned != 0, split, per};
                }
            }
        }
    return best;
}

template <Mode MODE, typename T, Kind KIND> void launch_product(Product f, const Choice &c, hipStream_t st) {
    using Of = Tiles<KIND>;
    if (c.turned) {
        const Pairs a = f.a, by_j = f.by_j;
        const int64_t rows_a = f.rows_a;
        f.a = f.b;
        f.b = a;
        f.rows_a = f.rows_b;
        f.rows_b = rows_a;
        f.by_j = f.by_i;
        f.by_i = by_j;
        f.old_by_j = f.old_by_i;
    }
    constexpr bool SYMMETRIC = MODE != NEXT && MODE != LAST;
    f.tiles_a = static_cast<int>((f.rows_a + SHAPE_BM[c.shape] - 1) / SHAPE_BM[c.shape]);
    f.tiles_b = static_cast<int>((f.rows_b + SHAPE_BN[c.shape] - 1) / SHAPE_BN[c.shape]);
    f.tiles = SYMMETRIC ? f.tiles_a * (f.tiles_a + 1) / 2 : f.tiles_a * f.tiles_b;
    f.slices /= KIND == HIGH ? 2 : 1;
    f.slices_per_split = c.per;
    const int64_t all = static_cast<int64_t>(f.tiles) * c.split;
    const dim3 groups(static_cast<unsigned>(all));
    if (c.shape == SHAPE_64 && all <= 256) {
        hipLaunchKernelGGL((k_muon_product<MODE, T, typename Of::Deep64, 1>), groups, dim3(Of::Deep64::NT), 0, st, f);
    } else if (c.shape == SHAPE_64) {
        if constexpr (KIND != HIGH || (MODE != GRAM && MODE != POLY))
            hipLaunchKernelGGL((k_muon_product<MODE, T, typename Of::Of64, 3>), groups, dim3(Of::Of64::NT), 0, st, f);
    } else if (c.shape == SHAPE_128) {
        hipLaunchKernelGGL((k_muon_product<MODE, T, typename Of::Of128, 2>), groups, dim3(Of::Of128::NT), 0, st, f);
    } else if (c.shape == SHAPE_256) {
        hipLaunchKernelGGL((k_muon_product<MODE, T, typename Of::Of256, 1>), groups, dim3(Of::Of256::NT), 0, st, f);
    } else if constexpr (!SYMMETRIC) {
        if (c.shape == SHAPE_192)
            hipLaunchKernelGGL((k_muon_product<MODE, T, typename Of::Of192, 1>), groups, dim3(Of::Of192::NT), 0, st, f);
        else
            hipLaunchKernelGGL((k_muon_product<MODE, T, typename Of::Of160, 1>), groups, dim3(Of::Of160::NT), 0, st, f);
    }
}
// A A's polynomial or X X^T, whole or in shares.
template <Mode MODE> void launch_symmetric(Product f, const Choice &c, hipStream_t st) {
    if (c.split == 1) return c.high ? launch_product<MODE, float, HIGH>(f, c, st) : launch_product<MODE, float, PAIRS>(f, c, st);
    c.high ? launch_product<SHARE, float, HIGH>(f, c, st) : launch_product<SHARE, float, PAIRS>(f, c, st);
    const int side = SHAPE_BM[c.shape], along = static_cast<int>((f.rows_a + side - 1) / side);
    f.tiles = along * (along + 1) / 2;
    hipLaunchKernelGGL(k_muon_join<MODE>, dim3(static_cast<unsigned>(f.tiles * (side / 64) * (side / 64))), dim3(256), 0, st, f, c.split, side);
}
size_t shares_bytes(const Choice &c, int64_t rows) {
    const size_t side = static_cast<size_t>(SHAPE_BM[c.shape]), along = (static_cast<size_t>(rows) + side - 1) / side;
    return c.split == 1 ? 0 : static_cast<size_t>(c.split) * (along * (along + 1) / 2) * side * side * sizeof(float);
}

constexpr int64_t MAX_SIDE = 1 << 16, MAX_STEPS = 64, COARSE_FROM = 256;
bool update_ok(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 0 && rows <= MAX_SIDE && cols <= MAX_SIDE && rows * cols < (static_cast<int64_t>(1) << 31); }

// The workspace: X and, twice, X transposed; A, B; partial sums.
struct Workspace {
    size_t x, xt[2], gram, poly, squares, shares, bytes;
    Choice gram_of[2], poly_of[2];  // of the pairs, of their h alone
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
    size_t most = 0;
    for (int high = 0; high < 2; ++high) {
        w.gram_of[high] = choice_of(less, less, more, HALF, high != 0);
        w.poly_of[high] = choice_of(less, less, less, HALF, high != 0);
        for (const Choice &c : {w.gram_of[high], w.poly_of[high]})
            if (const size_t bytes = shares_bytes(c, less); bytes > most) most = bytes;
    }
    w.shares = take(most);
    w.bytes = at;
    return w;
}

// `coarse_too`: products of some steps in 11 bits where w has 16.
adatopk_status update(const void *grad, int64_t grad_stride, adatopk_dtype grad_dt, float *momentum, float mu, int32_t nesterov, int64_t rows, int64_t cols, int32_t steps,
                      float eps, void *w, int64_t w_stride, adatopk_dtype dt, float scale, float decay, void *workspace, size_t workspace_bytes, void *hip_stream,
                      bool coarse_too) {
    if (!dtype_ok(grad_dt) || !dtype_ok(dt) || !update_ok(rows, cols) || steps < 1 || steps > MAX_STEPS || !(eps >= 0.f)) return ADATOPK_EINVAL;
    if (rows == 0 || cols == 0) return ADATOPK_OK;
    if (!matrix_ok(grad, grad_stride, rows, cols, grad_dt) || !matrix_ok(w, w_stride, rows, cols, dt) || !pointer_ok_or_null(momentum, 4) || !pointer_ok(workspace, 256))
        return ADATOPK_EINVAL;
    const bool wide = rows <= cols;
    const int64_t less = wide ? rows : cols, more = wide ? cols : rows;
    const Workspace at = workspace_of(less, more);
    if (workspace_bytes < at.bytes) return ADATOPK_EWORKSPACE;
    uint8_t *const base = static_cast<uint8_t *>(workspace);
    // Where the caller asks for it and w is of 16 bits: products of 11 bits in the first steps, while singular values are small, and in bf16's last.
    const bool coarser = coarse_too && dt != ADATOPK_F32 && less >= COARSE_FROM, coarse_end = coarser && dt == ADATOPK_BF16;
    const int first = !coarser ? 0 : dt == ADATOPK_F16 ? 2 : 3, fine = dt == ADATOPK_F16 ? 3 : 2;
    const auto high_at = [&](int step) { return (step < first && steps - step > fine) || (coarse_end && step + 1 == steps); };
    const auto pairs = [&](size_t where, int64_t of) { return Pairs{base + where, padded(of) * 4, run_for(high_at(0)), false}; };
    Pairs x = pairs(at.x, more), gram = pairs(at.gram, less), poly = pairs(at.poly, less);
    Pairs xt = pairs(at.xt[0], less), xt_next = pairs(at.xt[1], less);
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);

    const Choice next = choice_of(less, more, less, X, false), next_coarse = choice_of(less, more, less, X, true);
    // (X's runs change: turned, it would be read and written in place in two orders)
    const Choice next_changing = choice_of(less, more, less, X_AS_IT_LIES, true);
    const Choice last = choice_of(cols, rows, less, W, coarse_end);
    // X as `step` reads it: its l by products from pairs, and one of the two X by a coarse step, which adds to it.
    const auto coarse_of = [&](int step) -> const Choice & { return high_at(step + 1) ? next_coarse : next_changing; };
    const auto as_read_at = [&](int step, Pairs &rows_first, Pairs &turned) {
        rows_first.run = turned.run = run_for(high_at(step));
        rows_first.halves = high_at(step) && (step + 1 == steps || !coarse_of(step).turned);
        turned.halves = high_at(step) && (step + 1 == steps || coarse_of(step).turned);
    };
    as_read_at(0, x, xt);

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
    for (int step = 0; step < steps; ++step) {
        const bool high = high_at(step);
        x.run = xt.run = gram.run = poly.run = run_for(high);
        poly.halves = high;
        Product p{};
        p.partial = reinterpret_cast<float *>(base + at.shares);
        p.a = p.b = x;
        p.rows_a = p.rows_b = less;
        p.slices = along;
        p.by_j = p.by_i = gram;
        launch_symmetric<GRAM>(p, at.gram_of[high], st);
        p.a = p.b = p.gram = gram;
        p.slices = side;
        p.by_j = p.by_i = poly;
        const bool coarse = high && step + 1 < steps;
        p.diagonal = coarse ? 0.f : NS_A;
        launch_symmetric<POLY>(p, at.poly_of[high], st);
        if (step + 1 < steps) {
            p.a = poly;
            p.b = xt;
            p.rows_b = more;
            p.by_j = xt_next;
            p.by_i = x;
            as_read_at(step + 1, p.by_i, p.by_j);
            p.old_by_j = xt;
            p.old_by_i = x;
            if (coarse)
                launch_product<NEXT, float, HIGH>(p, coarse_of(step), st);
            else
                launch_product<NEXT, float, PAIRS>(p, next, st);
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
                if constexpr (__is_same(T, Bf16)) {
                    if (coarse_end) return launch_product<LAST, T, HIGH>(p, last, st);
                }
                launch_product<LAST, T, PAIRS>(p, last, st);
            });
        }
    }
    return launched();
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
    return update(grad, grad_stride, grad_dt, momentum, mu, nesterov, rows, cols, steps, eps, w, w_stride, dt, scale, decay, workspace, workspace_bytes, hip_stream, false);
}

adatopk_status adatopk_muon_update_coarse(const void *grad, int64_t grad_stride, adatopk_dtype grad_dt, float *momentum, float mu, int32_t nesterov, int64_t rows,
                                          int64_t cols, int32_t steps, float eps, void *w, int64_t w_stride, adatopk_dtype dt, float scale, float decay,
                                          void *workspace, size_t workspace_bytes, void *hip_stream) {
    return update(grad, grad_stride, grad_dt, momentum, mu, nesterov, rows, cols, steps, eps, w, w_stride, dt, scale, decay, workspace, workspace_bytes, hip_stream, true);
}

#ifdef ADATOPK_MEASURE_BUILD
adatopk_status adatopk_measure_muon_update_cut(int64_t rows, int64_t cols, int32_t *out) {
    if (!update_ok(rows, cols) || rows == 0 || cols == 0) return ADATOPK_EINVAL;
    const int64_t less = rows < cols ? rows : cols, more = rows < cols ? cols : rows;
    for (int high = 0; high < 2; ++high) {
        const Choice four[] = {choice_of(less, less, more, HALF, high != 0), choice_of(less, less, less, HALF, high != 0),
                               choice_of(less, more, less, X, high != 0), choice_of(cols, rows, less, W, high != 0)};
        for (int k = 0; k < 4; ++k) {
            const Choice &c = four[k];
            const int64_t ra = k < 2 ? less : k == 3 ? cols : c.turned ? more : less, rb = k < 2 ? less : k == 3 ? rows : c.turned ? less : more;
            const int64_t a = (ra + SHAPE_BM[c.shape] - 1) / SHAPE_BM[c.shape], b = (rb + SHAPE_BN[c.shape] - 1) / SHAPE_BN[c.shape];
            const bool deep = c.shape == SHAPE_64 && (k < 2 ? a * (a + 1) / 2 : a * b) * c.split <= 256;
            int32_t *const to = out + (high * 4 + k) * 3;
            to[0] = SHAPE_BM[c.shape];
            to[1] = SHAPE_BN[c.shape];
            to[2] = c.split + (deep ? 64 : 0);
        }
    }
    return ADATOPK_OK;
}
adatopk_status adatopk_measure_muon_update_next_cut(int64_t rows, int64_t cols, int32_t *out) {
    if (!update_ok(rows, cols) || rows == 0 || cols == 0) return ADATOPK_EINVAL;
    const int64_t less = rows < cols ? rows : cols, more = rows < cols ? cols : rows;
    const Choice three[] = {choice_of(less, more, less, X, false), choice_of(less, more, less, X, true), choice_of(less, more, less, X_AS_IT_LIES, true)};
    for (int k = 0; k < 3; ++k) {
        const Choice &c = three[k];
        const int64_t a = ((c.turned ? more : less) + SHAPE_BM[c.shape] - 1) / SHAPE_BM[c.shape], b = ((c.turned ? less : more) + SHAPE_BN[c.shape] - 1) / SHAPE_BN[c.shape];
        out[4 * k] = SHAPE_BM[c.shape];
        out[4 * k + 1] = SHAPE_BN[c.shape];
        out[4 * k + 2] = c.shape == SHAPE_64 && a * b <= 256 ? 1 : 0;
        out[4 * k + 3] = c.turned ? 1 : 0;
    }
    return ADATOPK_OK;
}
#endif

}  // extern "C"
