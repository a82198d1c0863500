// What the operators that are made of matrix products over weights share (cross_entropy.hip, linear.hip): operands laid out for the tiles of
// mfma_tile.h, the two products of a backward pass, sums of shares of k, and when places are done with tiles of two lengths.
#pragma once

#include "loose.h"
#include "mfma_tile.h"

#include <type_traits>
#include <utility>

namespace dol {

constexpr int kUnits = 256;                             // compute units of the chip
constexpr int kLds = 160 * 1024;                        // of each

// Tiles of x w^T (Big, Small, Tiny), and of the two products that the result's gradient goes into in Q planes (..X: of x's, ..W: of w's).
template <int P, int Q>
struct Shapes;
template <>
struct Shapes<1, 1> {       // bf16
    using Big = MfmaTile<bf16x8, 1, 1, kRows, kRows, 256, 256, 64, 2, 4, 2>;
    using Small = MfmaTile<bf16x8, 1, 1, kRows, kRows, 128, 128, 64, 4, 2, 2>;
    using BigX = MfmaTile<bf16x8, 1, 1, kCols, kRows, 256, 256, 64, 2, 4, 2>;
    using BigW = MfmaTile<bf16x8, 1, 1, kCols, kCols, 256, 256, 64, 2, 4, 2>;
    using SmallX = MfmaTile<bf16x8, 1, 1, kCols, kRows, 128, 128, 64, 4, 2, 2>;
    using SmallW = MfmaTile<bf16x8, 1, 1, kCols, kCols, 128, 128, 64, 4, 2, 2>;
    using Tiny = MfmaTile<bf16x8, 1, 1, kRows, kRows, 64, 64, 64, 4, 1, 3>;
    using TinyX = MfmaTile<bf16x8, 1, 1, kCols, kRows, 64, 64, 64, 4, 1, 3>;
    using TinyW = MfmaTile<bf16x8, 1, 1, kCols, kCols, 64, 64, 64, 4, 1, 3>;
};
template <>
struct Shapes<1, 2> : Shapes<1, 1> {
    using BigX = MfmaTile<bf16x8, 1, 2, kCols, kRows, 128, 128, 32, 4, 2, 2>;
    using BigW = MfmaTile<bf16x8, 1, 2, kCols, kCols, 128, 128, 32, 4, 2, 2>;
    using SmallX = BigX;
    using SmallW = BigW;
    using TinyX = MfmaTile<bf16x8, 1, 2, kCols, kRows, 64, 64, 64, 4, 1, 3>;
    using TinyW = MfmaTile<bf16x8, 1, 2, kCols, kCols, 64, 64, 64, 4, 1, 3>;
};
template <>
struct Shapes<3, 3> {       // float
    using Big = MfmaTile<bf16x8, 3, 3, kRows, kRows, 128, 256, 32, 2, 4, 2>;
    using Small = MfmaTile<bf16x8, 3, 3, kRows, kRows, 128, 128, 32, 4, 2, 2>;
    using BigX = MfmaTile<bf16x8, 3, 3, kCols, kRows, 128, 256, 32, 2, 4, 2>;
    using BigW = MfmaTile<bf16x8, 3, 3, kCols, kCols, 128, 256, 32, 2, 4, 2>;
    using SmallX = MfmaTile<bf16x8, 3, 3, kCols, kRows, 128, 128, 32, 4, 2, 2>;
    using SmallW = MfmaTile<bf16x8, 3, 3, kCols, kCols, 128, 128, 32, 4, 2, 2>;
    using Tiny = MfmaTile<bf16x8, 3, 3, kRows, kRows, 64, 64, 64, 4, 1, 3>;
    using TinyX = MfmaTile<bf16x8, 3, 3, kCols, kRows, 64, 64, 64, 4, 1, 3>;
    using TinyW = MfmaTile<bf16x8, 3, 3, kCols, kCols, 64, 64, 64, 4, 1, 3>;
};

template <int P>
struct Source { using T = float; };
template <>
struct Source<1> { using T = __bf16; };

// Plane k of N.
template <int N>
__device__ __forceinline__ uint32_t plane_of(int k, float &x) { return N > 1 && k == 0 ? take_first_plane(x) : take_plane<__bf16>(x); }

__device__ __forceinline__ bool kept_row(int32_t target, int32_t classes) { return target >= 0 && target < classes; }

// ---------------------------------------------------------------- operands laid out

// A matrix laid out for the tiles: out[p][r][0..kp) = planes of src[r][0..cols), zeros behind and in rows past the source's.  Rows that do
// not count (if target and lse are given) are taken as zeros, whatever they hold.
struct Pack {
    const void *src;
    int64_t ld, rows;
    int32_t cols;
    const int32_t *target;
    const float *lse;
    int32_t classes;
    uint16_t *out;
    int64_t out_rows, kp, out_ld;
    unsigned blocks;            // none where the matrix is read as it is
};

// Plane k of three, an infinity as 1, 0 and itself with its sign: of its products with another number's planes (none of the dropped ones among them) the
// one with that number's first plane is infinite, or NaN beside a zero, and the others are finite or the same infinity, as the product of the two is.  (With
// itself as the plane that plane_of gives it, it meets what is left of the other number, whose sign may be another: NaN.)
__device__ __forceinline__ uint32_t plane_or_infinity(int k, float &x)
{
    if (!__builtin_isinf(x)) return plane_of<3>(k, x);
    const uint32_t sign = __float_as_uint(x) >> 16 & 0x8000;
    return k == 0 ? sign | 0x3F80 : k == 1 ? 0 : sign | 0x7F80;
}

// This workgroup's share (of 256 threads, eight elements to each at a time).  INF: products with infinities are infinities.
template <typename S, int P, bool INF = false>
__device__ __forceinline__ void pack_rows(const Pack &p, unsigned block)
{
    const int64_t per = p.kp / 8, all = p.out_rows * per;
    for (int64_t t = static_cast<int64_t>(block) * 256 + threadIdx.x; t < all; t += static_cast<int64_t>(p.blocks) * 256) {
        const int64_t r = t / per;
        const int c = static_cast<int>(t - r * per) * 8;
        const bool in = r < p.rows && (!p.target || (kept_row(p.target[r], p.classes) && p.lse[r] != -INFINITY));
        const S *from = static_cast<const S *>(p.src) + r * p.ld + c;
        float v[8];
        constexpr int V = kLooseElements<S>;
#pragma unroll
        for (int h = 0; h < 8 / V; ++h) {
            const Loose<S> q = loose_load_end(from + h * V, in ? p.cols - c - h * V : 0, c + h * V);
#pragma unroll
            for (int k = 0; k < V; ++k) v[h * V + k] = loose_get(q, k);
        }
#pragma unroll
        for (int q = 0; q < P; ++q) {
            u32x4 w;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                auto plane = [&](float &x) { return INF && P == 3 ? plane_or_infinity(q, x) : plane_of<P>(q, x); };
                const uint32_t lo = plane(v[2 * k]), hi = plane(v[2 * k + 1]);
                w[k] = lo | hi << 16;
            }
            *reinterpret_cast<u32x4 *>(p.out + (q * p.out_rows + r) * p.out_ld + c) = w;
        }
    }
}

// ---------------------------------------------------------------- the products of a backward pass

// One set of tiles of the launch that follows: out[n][m] = sum_k a[k][m] b(n, k), k in `splits` shares.  Rows of a tile are elements of x or w,
// which lie side by side in `out` too.
struct Product {
    Planes a, b;
    int32_t M, N;               // columns of out, rows of out
    int32_t wide, tall;         // what a and b have of them in memory
    int32_t tm, tn, splits, steps;
    int64_t k, have;            // that count, and that there are of operands which lie across k
    float *part;                // [splits][N][part_ld], or null: out is written
    int64_t part_ld;
    bool add;                   // to what part holds
    void *out;
    int64_t out_ld;
};

template <typename T, typename O>
__device__ __forceinline__ void product_tile(const Product &p, int id, char *smem)
{
    const int tiles = p.tm * p.tn, split = id / tiles;
    int mt, nt;
    tile_of(id - split * tiles, p.tm, p.tn, 4, mt, nt);
    const int s0 = static_cast<int>(static_cast<int64_t>(p.steps) * split / p.splits), s1 = static_cast<int>(static_cast<int64_t>(p.steps) * (split + 1) / p.splits);
    const int64_t k0 = static_cast<int64_t>(s0) * T::BK;
    f32x4 acc[T::MI][T::NI];
    T::clear(acc);
    T::run(p.a, static_cast<int64_t>(mt) * T::BM, p.wide, p.b, static_cast<int64_t>(nt) * T::BN, p.tall, k0, s1 - s0, smem, acc, p.have - k0);
#pragma unroll
    for (int j = 0; j < T::NI; ++j) {
        const int n = nt * T::BN + T::col_of(j);
        if (n >= p.N) continue;
#pragma unroll
        for (int i = 0; i < T::MI; ++i) {
            const int m = mt * T::BM + T::row_of(i);
            if (m >= p.M) continue;
            if (p.part) {       // (its rows are filled up to whole fours)
                f32x4 *to = reinterpret_cast<f32x4 *>(p.part + (static_cast<int64_t>(split) * p.N + n) * p.part_ld + m);
                *to = p.add ? *to + acc[i][j] : acc[i][j];
            } else
                store4(static_cast<O *>(p.out) + n * p.out_ld + m, acc[i][j], p.M - m);
        }
    }
}

// ---------------------------------------------------------------- sums of shares

// out[m][n] = the sum of its parts, in an order that the sizes fix.
struct Sum {
    const float *part;
    int32_t M, N, splits;       // rows, columns
    int64_t part_ld;
    void *out;
    int64_t out_ld;
    bool shared;                // four threads to four columns, each for a quarter of the parts
    unsigned blocks;            // none where nothing is to be summed
};

template <typename O>
__device__ __forceinline__ void sum_parts(const Sum &s, unsigned block)
{
    __shared__ f32x4 red[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t per = (s.N + 3) / 4, all = s.M * per;
    const int each = s.shared ? 64 : 256, at = s.shared ? lane : threadIdx.x;
    for (int64_t first = static_cast<int64_t>(block) * each; first < all; first += static_cast<int64_t>(s.blocks) * each) {
        const int64_t t = first + at, m = t / per;
        const bool in = t < all;
        const int n = static_cast<int>(t - m * per) * 4;
        f32x4 v = {0, 0, 0, 0};
        if (in)
#pragma unroll 8
            for (int k = s.shared ? wave : 0; k < s.splits; k += s.shared ? 4 : 1) v += *reinterpret_cast<const f32x4 *>(s.part + (static_cast<int64_t>(k) * s.M + m) * s.part_ld + n);
        if (s.shared) {
            red[wave][lane] = v;
            __syncthreads();
            v = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
            __syncthreads();
            if (wave != 0) continue;
        }
        if (in) store4(static_cast<O *>(s.out) + m * s.out_ld + n, v, s.N - n);
    }
}

// ---------------------------------------------------------------- host side

constexpr int32_t kMostRows = 1 << 22;      // of either operand: a lane's offsets into a tile of dl fit 32 bits
constexpr int32_t kMostWidth = 1 << 20;     // of a row: 64 columns to a workgroup of a grid's second dimension

inline bool direct(const dol_matrix *m)            // can be read by the tiles as it is
{
    return m->dtype == DOL_BF16 && m->cols % 64 == 0 && m->ld % 8 == 0 && m->ld <= kMostRows && !(reinterpret_cast<uintptr_t>(m->data) & 15);
}

inline int32_t tiles(int64_t n, int t) { return static_cast<int32_t>((n + t - 1) / t); }
inline unsigned blocks(int64_t n) { return static_cast<unsigned>((n + 255) / 256); }

// Launches have less than 2^32 threads: workgroups of what is done element by element, at most (each then takes several pieces in turn).
constexpr int64_t kMostBlocks = 1 << 15;

// When `slots` places, each of which takes the next one as it becomes free, are done with n1 pieces of work of length a and then n2 of
// length b.
inline double done(int64_t n1, double a, int64_t n2, double b, int64_t slots)
{
    const int64_t late = n1 % slots;                    // so many places are free one a later than the others
    double soon = n1 / slots * a, then = soon + a;
    double end = late ? then : soon;
    while (n2 > 0) {
        if (late == 0 || soon <= then) soon += b, n2 -= slots - late, end = std::max(end, soon);
        else then += b, n2 -= late, end = std::max(end, then);
    }
    return end;
}

template <typename T>
struct Type { using Tile = T; };

template <typename B, typename S, typename T, typename F>
auto by_size(int size, B big, S small, T tiny, F f) { return size == 2 ? f(big) : size == 1 ? f(small) : f(tiny); }

// Rows with contiguous k as the tiles read them: the matrix itself, or `out`, its planes in rows of kp elements (out_rows of them).
template <int P>
Pack pack_of(const dol_matrix *m, const int32_t *target, const float *lse, int32_t classes, uint16_t *out, int64_t out_rows, int64_t kp, int64_t ld, Planes *p)
{
    if (!out) {
        *p = Planes{static_cast<const uint16_t *>(m->data), m->ld, 0};
        return Pack{};
    }
    *p = Planes{out, ld, out_rows * ld};
    return Pack{m->data, m->ld, m->rows, m->cols, target, lse, classes, out, out_rows, kp, ld, blocks(std::min(out_rows * (kp / 8), kMostBlocks * 256))};
}

// (few parts are read as fast by a thread each; a loop over many of them waits for every load)
inline Sum make_sum(const float *part, int32_t M, int32_t N, int32_t splits, int64_t part_ld, void *out, int64_t out_ld)
{
    const bool shared = splits >= 16;
    const int64_t n = int64_t(M) * ((N + 3) / 4);
    return Sum{part, M, N, splits, part_ld, out, out_ld, shared, static_cast<unsigned>(std::min((n + (shared ? 63 : 255)) / (shared ? 64 : 256), kMostBlocks))};
}

inline Sum sum_of(const Product &p)
{
    if (!p.part) return Sum{};
    return make_sum(p.part, p.N, p.M, p.splits, p.part_ld, p.out, p.out_ld);
}

}  // namespace dol
