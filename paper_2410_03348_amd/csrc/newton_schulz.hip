// An update's orthogonalisation by Newton-Schulz products: X = G / (|G| + eps), then `steps` times
//   A = X X^T,   B = b A + c A A,   X <- a X + B X
// so that every singular value s of X becomes s (a + b s^2 + c s^4); a matrix taller than wide is taken as its transpose.
//
// X lies one way, as wide rows: A's tiles read it along k, X's own across k (mfma_tile.h); A and B are symmetric.  Numbers lie as fp16
// times a power of two that their bounds allow: singular values stay below a bound known beforehand, and no element is above them.
// float: two planes each, 22 bits, three products: as exact as 32-bit sums of 32-bit numbers (an error of a step's X grows with the
// steps after it, up to a^steps = 485 times for directions whose singular value is near 0, so there is nothing to spare).
// bf16: one plane and one product; X alone keeps its second plane, which a X adds.  The result is off by 1.2e-3 to 2e-3 before it is
// rounded to bf16, which itself takes 1.7e-3 (2.0e-3 to 2.6e-3 together); with X's second plane left out as well by up to 3.3e-3.
#include "mfma_tile.h"

#include <cmath>
#include <cstdio>

namespace dol {
namespace {

constexpr int kNormParts = 1024;    // workgroups that share a matrix's sum of squares, at most
constexpr int kUnits = 256;

// Tiles of the symmetric products, of B X with X's columns as the tile's rows, and (for a tall result) as its columns.
template <int P>
struct Shapes;
template <>
struct Shapes<1> {
    template <Order A, Order B>
    using Big = MfmaTile<f16x8, 1, 1, A, B, 256, 256, 64, 2, 4, 2>;
    template <Order A, Order B>
    using Mid = MfmaTile<f16x8, 1, 1, A, B, 128, 128, 64, 4, 2, 2>;
    template <Order A, Order B>
    using Small = MfmaTile<f16x8, 1, 1, A, B, 64, 64, 64, 4, 1, 3, 2>;
};
template <>
struct Shapes<2> {
    template <Order A, Order B>
    using Big = MfmaTile<f16x8, 2, 2, A, B, 256, 256, 32, 2, 4, 2>;
    template <Order A, Order B>
    using Mid = MfmaTile<f16x8, 2, 2, A, B, 128, 128, 64, 2, 2, 2, 2>;
    template <Order A, Order B>
    using Small = MfmaTile<f16x8, 2, 2, A, B, 64, 64, 64, 4, 1, 3, 2>;
};

// Powers of two that X, A and B are stored times.
struct Scales {
    int x, a, b;
};

// ---------------------------------------------------------------- norm and first layout

// Sums of squares in 64 bits: no float overflows there, and none that counts underflows.  4096 x 4096 of bf16 in 8.2 us, 4.1 TB/s.
template <typename S>
__global__ void __launch_bounds__(256) ns_norm_kernel(const S *g, int64_t ld, int64_t stride, int32_t rows, int32_t cols, double *part)
{
    __shared__ double red[4];
    const S *src = g + blockIdx.y * stride;
    double s = 0.0;
    const int64_t n = static_cast<int64_t>(rows) * cols;
    constexpr int E = 16 / sizeof(S);
    if (ld == cols && n % E == 0 && (reinterpret_cast<uintptr_t>(src) & 15) == 0) {
        struct alignas(16) Piece { S v[E]; };
#pragma unroll 4
        for (int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; t < n / E; t += static_cast<int64_t>(gridDim.x) * 256) {
            const Piece q = reinterpret_cast<const Piece *>(src)[t];
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const double v = static_cast<float>(q.v[k]);
                s = __builtin_fma(v, v, s);
            }
        }
    } else {
        for (int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; t < n; t += static_cast<int64_t>(gridDim.x) * 256) {
            const int64_t r = t / cols;
            const double v = static_cast<float>(src[r * ld + (t - r * cols)]);
            s = __builtin_fma(v, v, s);
        }
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// X [mp][np] in two planes, from g (transposed where it is taller than wide); a tile of 64 x 64 to a workgroup.  Bytes bound it where there are
// many: 4096 x 4096 of bf16 in 32.8 us, 3.1 TB/s; 1000 x 777 of float takes 11, waits for the load, the norm's parts and the stores.
template <typename S>
__global__ void __launch_bounds__(256) ns_first_kernel(const S *g, int64_t ld, int64_t stride, int32_t rows, int32_t cols, bool tall, const double *part, int parts,
                                                       float eps, int scale, uint16_t *x, int32_t mp, int32_t np)
{
    __shared__ float tile[64][65];
    __shared__ double total;
    const S *src = g + blockIdx.z * stride;
    const int32_t r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;     // in g
    const int cx = threadIdx.x & 63, cy = threadIdx.x >> 6;
    float in[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) in[k] = r0 + k * 4 + cy < rows && c0 + cx < cols ? static_cast<float>(src[static_cast<int64_t>(r0 + k * 4 + cy) * ld + c0 + cx]) : 0.0f;
    if (threadIdx.x < 64) {
        double s = 0.0;
        for (int k = threadIdx.x; k < parts; k += 64) s += part[static_cast<int64_t>(blockIdx.z) * parts + k];
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
        if (threadIdx.x == 0) total = s;
    }
    __syncthreads();
    const double f = ldexp(1.0, scale) / (sqrt(total) + static_cast<double>(eps));
#pragma unroll
    for (int k = 0; k < 16; ++k) tile[k * 4 + cy][cx] = static_cast<float>(static_cast<double>(in[k]) * f);
    __syncthreads();
    const int64_t plane = static_cast<int64_t>(mp) * np;
    uint16_t *dst = x + blockIdx.z * 2 * plane;
    const int q = threadIdx.x & 7;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int k = (threadIdx.x >> 3) + h * 32;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tall ? tile[q * 8 + e][k] : tile[k][q * 8 + e];
        uint16_t *to = dst + (tall ? static_cast<int64_t>(c0 + k) * np + r0 + q * 8 : static_cast<int64_t>(r0 + k) * np + c0 + q * 8);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t lo = take_plane<_Float16>(v[2 * e]), hi = take_plane<_Float16>(v[2 * e + 1]);
                w[e] = lo | hi << 16;
            }
            *reinterpret_cast<u32x4 *>(to + p * plane) = w;
        }
    }
}

// ---------------------------------------------------------------- the products

__device__ __forceinline__ float half_of(uint32_t bits) { return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(bits))); }

// Four neighbouring elements of `planes` planes.
__device__ __forceinline__ f32x4 read4(const uint16_t *p, int64_t plane, int planes)
{
    f32x4 v = {0, 0, 0, 0};
    for (int k = planes - 1; k >= 0; --k) {     // the small plane first
        const u32x2 w = *reinterpret_cast<const u32x2 *>(p + k * plane);
        v += f32x4{half_of(w[0]), half_of(w[0] >> 16), half_of(w[1]), half_of(w[1] >> 16)};
    }
    return v;
}

// Four neighbouring elements to P planes.
template <int P>
__device__ __forceinline__ void write4(uint16_t *to, int64_t plane, f32x4 v)
{
#pragma unroll
    for (int p = 0; p < P; ++p) {
        float r[4] = {v[0], v[1], v[2], v[3]};
        u32x2 w;
        const uint32_t w0 = take_plane<_Float16>(r[0]), w1 = take_plane<_Float16>(r[1]), w2 = take_plane<_Float16>(r[2]), w3 = take_plane<_Float16>(r[3]);
        w[0] = w0 | w1 << 16, w[1] = w2 | w3 << 16;
        *reinterpret_cast<u32x2 *>(to + p * plane) = w;
        v = f32x4{r[0], r[1], r[2], r[3]};
    }
}

// A symmetric product of rows: with POLY B = b A + c A A from A, else A = X X^T.  Only tiles on and below the diagonal are computed, and
// written to both sides.  alpha scales the product, beta (POLY) what A holds.  Its tiles seldom fill the chip: bf16 4096 x 4096 105 us, 136 of
// 256 x 256 for 256 units (128 x 128 ones come out even, but load twice as much), float 777 rows 12.5 us, 91 of 64 x 64.
template <typename T, bool POLY>
__global__ void __launch_bounds__(T::NT, 2) ns_symmetric_kernel(const uint16_t *in, int64_t in_stride, int64_t ld, int64_t plane, int32_t mp, int steps, float alpha, float beta,
                                                                uint16_t *out, int64_t out_stride, int64_t out_plane)
{
    extern __shared__ __align__(128) char smem[];
    const int id = xcd_contiguous(blockIdx.x, gridDim.x);
    int mt = static_cast<int>((__builtin_sqrtf(8.0f * id + 1.0f) - 1.0f) * 0.5f);
    while (mt * (mt + 1) / 2 > id) --mt;
    while ((mt + 1) * (mt + 2) / 2 <= id) ++mt;
    const int nt = id - mt * (mt + 1) / 2;
    const uint16_t *src = in + blockIdx.y * in_stride;
    uint16_t *dst = out + blockIdx.y * out_stride;
    const int64_t m0 = mt * T::BM, n = nt * T::BN + T::col_of();
    f32x4 early[4];         // small tiles have the registers to ask for A beforehand
    if (POLY && T::MI == 1 && T::first_set())
#pragma unroll
        for (int e = 0; e < 4; ++e) early[e] = read4(src + (m0 + T::row_of(0) + e) * mp + n, plane, T::PA);
    f32x4 acc[T::MI][T::NI];
    T::clear(acc);
    const Planes p{src, ld, plane};
    T::run(p, m0, mp, p, nt * T::BN, mp, 0, steps, smem, acc);
    T::join(acc, smem);
    if (!T::first_set()) return;
#pragma unroll
    for (int i = 0; i < T::MI; ++i) {
        const int64_t m = m0 + T::row_of(i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f32x4 v = {acc[i][0][e], acc[i][1][e], acc[i][2][e], acc[i][3][e]}, old = {0, 0, 0, 0};
            if constexpr (POLY && T::MI == 1) old = early[e];
            else if constexpr (POLY) old = read4(src + (m + e) * mp + n, plane, T::PA);
#pragma unroll
            for (int j = 0; j < T::NI; ++j) acc[i][j][e] = v[j] = POLY ? __builtin_fmaf(beta, old[j], alpha * v[j]) : alpha * v[j];
            write4<T::PA>(dst + (m + e) * mp + n, out_plane, v);
        }
        if (mt != nt)
#pragma unroll
            for (int j = 0; j < T::NI; ++j) write4<T::PA>(dst + (n + j) * mp + m, out_plane, acc[i][j]);
    }
}

// X' = alpha (B X) + beta X, X' [mp][np] in two planes, or (out) the result.  TURN: a tile's columns are X's columns and out is tall.
// Loads into LDS bound it, and in bf16 with 256 x 256 tiles the registers: the operand that lies across k keeps its addresses beside 224 registers of sums
// and halves, so that 22 are spilled (TURN: 67).  bf16 4096 x 4096 148 us, 929 TFLOP/s, where such a loop alone does 1 256; float 1000 x 777 16 us.
struct Apply {
    const uint16_t *x, *b;
    int64_t x_stride, b_stride;
    int32_t mp, np;
    float alpha, beta;
    uint16_t *to;
    void *out;
    int64_t out_ld, out_stride;
    int32_t out_rows, out_cols;
};

template <typename T, typename O, bool TURN>
__global__ void __launch_bounds__(T::NT, 2) ns_apply_kernel(Apply p)
{
    extern __shared__ __align__(128) char smem[];
    const int tm = (TURN ? p.mp : p.np) / T::BM, tn = (TURN ? p.np : p.mp) / T::BN;
    int mt, nt;
    tile_of(xcd_contiguous(blockIdx.x, gridDim.x), tm, tn, 4, mt, nt);
    const int64_t z = blockIdx.y, plane = static_cast<int64_t>(p.mp) * p.np;
    const uint16_t *x = p.x + z * p.x_stride;
    const Planes px{x, p.np, plane}, pb{p.b + z * p.b_stride, p.mp, static_cast<int64_t>(p.mp) * p.mp};
    f32x4 acc[T::MI][T::NI];        // begins with beta / alpha X: read while the first operands are on their way
    const float begin = p.beta / p.alpha;
    T::clear(acc);
    if (T::first_set())
#pragma unroll
        for (int i = 0; i < T::MI; ++i)
#pragma unroll
            for (int j = 0; j < T::NI; ++j) {
                const int64_t m = static_cast<int64_t>(mt) * T::BM + T::row_of(i), n = static_cast<int64_t>(nt) * T::BN + T::col_of(j);
                if constexpr (TURN) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = begin * (half_of(x[plane + (m + e) * p.np + n]) + half_of(x[(m + e) * p.np + n]));
                } else
                    acc[i][j] = begin * read4(x + n * p.np + m, plane, 2);
            }
    T::run(TURN ? pb : px, mt * T::BM, TURN ? p.mp : p.np, TURN ? px : pb, nt * T::BN, TURN ? p.np : p.mp, 0, p.mp / T::BK, smem, acc, p.mp);
    T::join(acc, smem);
    if (!T::first_set()) return;
    const bool vec = p.out_ld % 4 == 0 && (reinterpret_cast<uintptr_t>(static_cast<O *>(p.out) + z * p.out_stride) & (4 * sizeof(O) - 1)) == 0;
#pragma unroll
    for (int i = 0; i < T::MI; ++i) {
        const int64_t m = static_cast<int64_t>(mt) * T::BM + T::row_of(i);      // four rows of the tile from here: neighbours in memory
#pragma unroll
        for (int j = 0; j < T::NI; ++j) {
            const int64_t n = static_cast<int64_t>(nt) * T::BN + T::col_of(j);
            const f32x4 v = p.alpha * acc[i][j];
            if (TURN || p.out) {
                if (n < p.out_rows && m < p.out_cols)
                    store4(static_cast<O *>(p.out) + z * p.out_stride + n * p.out_ld + m, v, static_cast<int>(p.out_cols - m), vec);
            } else
                write4<2>(p.to + z * p.x_stride + n * p.np + m, plane, v);
        }
    }
}

// ---------------------------------------------------------------- small matrices

// A whole matrix in the LDS of one workgroup, all steps in one launch, in 32 bits throughout (v_mfma_f32_16x16x4: lane l gives element
// (l & 15, l >> 4) of a 16 x 4 operand and gets rows 4 (l >> 4) .. + 3 of column l & 15).  A chain of 15 dependent products bounds it: 10 x 128 in
// 16 us, 32 x 500 in 56.
constexpr int kSmallWaves = 16, kSmallSide = 64;
constexpr size_t kSmallLds = 150 * 1024;

struct SmallShape {
    int mp, np, ldx, lda, slices;       // filled up to 16; rows an odd number of fours apart; shares of X X^T's k
    size_t floats() const { return static_cast<size_t>(mp) * ldx + static_cast<size_t>(2) * mp * lda + static_cast<size_t>(slices) * mp * mp; }
};

__host__ __device__ inline SmallShape small_shape(int m, int n)
{
    SmallShape s;
    s.mp = (m + 15) / 16 * 16, s.np = (n + 15) / 16 * 16;
    s.ldx = s.np + 4, s.lda = s.mp + 4, s.slices = kSmallWaves / (s.mp / 16);
    return s;
}

template <typename S>
__global__ void __launch_bounds__(kSmallWaves * 64) ns_small_kernel(const S *g, int64_t ld, int64_t stride, int32_t rows, int32_t cols, int32_t steps, float ka, float kb,
                                                                   float kc, float eps, S *out, int64_t out_ld, int64_t out_stride)
{
    extern __shared__ __align__(16) float lds[];
    __shared__ double red[kSmallWaves];
    constexpr int NT = kSmallWaves * 64;
    const bool tall = rows > cols;
    const int m = tall ? cols : rows, n = tall ? rows : cols;
    const SmallShape s = small_shape(m, n);
    float *X = lds, *A = X + s.mp * s.ldx, *B = A + s.mp * s.lda, *part = B + s.mp * s.lda;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r16 = lane & 15, k4 = lane >> 4, row_tiles = s.mp / 16;
    const S *src = g + blockIdx.x * stride;
    for (int t = tid; t < s.mp * s.ldx; t += NT) X[t] = 0.0f;
    __syncthreads();
    double sum = 0.0;
    for (int t = tid; t < rows * cols; t += NT) {
        const int r = t / cols, c = t - r * cols;
        const float v = static_cast<float>(src[r * ld + c]);
        X[(tall ? c : r) * s.ldx + (tall ? r : c)] = v;
        sum = __builtin_fma(static_cast<double>(v), static_cast<double>(v), sum);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if (lane == 0) red[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int k = 0; k < kSmallWaves; ++k) sum += red[k];
    const double f = 1.0 / (sqrt(sum) + static_cast<double>(eps));
    for (int t = tid; t < s.mp * s.ldx; t += NT) X[t] = static_cast<float>(static_cast<double>(X[t]) * f);
    __syncthreads();
    for (int step = 0; step < steps; ++step) {
        // X X^T: a wavefront takes a row of its tiles over a share of k
        const int tr = wave % row_tiles, slice = wave / row_tiles;
        if (slice < s.slices) {
            f32x4 acc[kSmallSide / 16] = {};
            const int q = s.np / 4, k0 = q * slice / s.slices, k1 = q * (slice + 1) / s.slices;
            for (int k = k0; k < k1; ++k) {
                const float a = X[(tr * 16 + r16) * s.ldx + k * 4 + k4];
#pragma unroll
                for (int j = 0; j < kSmallSide / 16; ++j)
                    if (j < row_tiles) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, X[(j * 16 + r16) * s.ldx + k * 4 + k4], acc[j], 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < kSmallSide / 16; ++j)
                if (j < row_tiles)
#pragma unroll
                    for (int e = 0; e < 4; ++e) part[(slice * s.mp + tr * 16 + k4 * 4 + e) * s.mp + j * 16 + r16] = acc[j][e];
        }
        __syncthreads();
        for (int t = tid; t < s.mp * s.mp; t += NT) {
            float v = 0.0f;
            for (int k = 0; k < s.slices; ++k) v += part[k * s.mp * s.mp + t];
            A[t / s.mp * s.lda + t % s.mp] = v;
        }
        __syncthreads();
        for (int t = wave; t < row_tiles * row_tiles; t += kSmallWaves) {
            const int i = t / row_tiles, j = t % row_tiles;
            f32x4 acc = {};
            for (int k = 0; k < s.mp / 4; ++k)
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(A[(i * 16 + r16) * s.lda + k * 4 + k4], A[(j * 16 + r16) * s.lda + k * 4 + k4], acc, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = (i * 16 + k4 * 4 + e) * s.lda + j * 16 + r16;
                B[at] = kb * A[at] + kc * acc[e];
            }
        }
        __syncthreads();
        // a X + B X: a wavefront's sixteen columns depend on these columns alone
        for (int j = wave; j < s.np / 16; j += kSmallWaves) {
            f32x4 acc[kSmallSide / 16] = {};
            for (int k = 0; k < s.mp / 4; ++k) {
                const float x = X[(k * 4 + k4) * s.ldx + j * 16 + r16];
#pragma unroll
                for (int i = 0; i < kSmallSide / 16; ++i)
                    if (i < row_tiles) acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(B[(i * 16 + r16) * s.lda + k * 4 + k4], x, acc[i], 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < kSmallSide / 16; ++i)
                if (i < row_tiles)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float &x = X[(i * 16 + k4 * 4 + e) * s.ldx + j * 16 + r16];
                        x = ka * x + acc[i][e];
                    }
        }
        __syncthreads();
    }
    S *dst = out + blockIdx.x * out_stride;
    for (int t = tid; t < rows * cols; t += NT) {
        const int r = t / cols, c = t - r * cols;
        dst[r * out_ld + c] = static_cast<S>(X[(tall ? c : r) * s.ldx + (tall ? r : c)]);
    }
}

// ---------------------------------------------------------------- host side

// One launch of one workgroup to a matrix against seventeen that share each matrix's tiles out.  us, one / seventeen: float 32 x 500 56 / 76,
// 48 x 250 61 / 68, 64 x 128 63 / 63; bf16 32 x 500 57 / 62, 48 x 250 61 / 58, 64 x 128 63 / 54, where 32 bits throughout are what is left.
bool small(const dol_matrix *g)
{
    const int64_t m = std::min(g->rows, g->cols), n = std::max(g->rows, g->cols);
    if (m > kSmallSide || n > 4096) return false;
    const SmallShape s = small_shape(static_cast<int>(m), static_cast<int>(n));
    return s.floats() * 4 <= kSmallLds && int64_t(s.mp) * s.mp * s.np <= 600000;
}

struct Layout {
    bool tall;
    int32_t m, n, mp, np;           // the wide orientation, and filled up
    double *part;
    uint16_t *x[2], *a, *b;
    int64_t bytes;
};

Layout lay_out(const dol_matrix *g, int32_t batch, int planes, void *workspace)
{
    Layout L{};
    L.tall = g->rows > g->cols;
    L.m = L.tall ? g->cols : g->rows, L.n = L.tall ? g->rows : g->cols;
    // rows and columns are filled up with zeros, which stay zeros
    auto pad = [](int32_t v) { return static_cast<int32_t>(round_up(v, v > 1920 ? 256 : v > 256 ? 128 : 64)); };
    L.mp = pad(L.m), L.np = pad(L.n);
    Carver c(workspace);
    const int64_t x = 2 * int64_t(L.mp) * L.np * batch, a = planes * int64_t(L.mp) * L.mp * batch;
    L.part = c.take<double>(int64_t(kNormParts) * batch);
    for (int k = 0; k < 2; ++k) L.x[k] = c.take<uint16_t>(x);
    L.a = c.take<uint16_t>(a), L.b = c.take<uint16_t>(a);
    L.bytes = c.used;
    return L;
}

// The greatest |s (a + b s^2 + c s^4)| (of_x) or |b s^2 + c s^4| over 0 <= s <= most, from the ends and where the derivative vanishes.
double bound_of(const float *k, double most, bool of_x)
{
    const double a = of_x ? k[0] : 0.0, b = k[1], c = k[2];
    auto value = [&](double s) { return std::fabs(of_x ? s * (a + s * s * (b + s * s * c)) : s * s * (b + s * s * c)); };
    double top = value(most);
    auto at = [&](double s2) {
        if (s2 > 0.0 && s2 < most * most) top = std::max(top, value(std::sqrt(s2)));
    };
    if (of_x) {             // 5 c t^2 + 3 b t + a = 0, t = s^2
        const double q = 9.0 * b * b - 20.0 * a * c;
        if (c != 0.0 && q >= 0.0) at((-3.0 * b + std::sqrt(q)) / (10.0 * c)), at((-3.0 * b - std::sqrt(q)) / (10.0 * c));
        if (b != 0.0) at(-a / (3.0 * b));
    } else if (c != 0.0)
        at(-b / (2.0 * c));
    return top;
}

// Which tiles the symmetric products (half) or B X take: 2 is 256 x 256, 1 is 128 x 128, 0 is 64 x 64.
// The largest that fill the chip well enough: larger ones load less for what they do, and loads bound them all.  Of 256 x 256
// half a chip (float 4096 x 4096 takes 4.52 ms so and 4.77 with 128 x 128, bf16 1.67 and 1.87).  Of 128 x 128 from these numbers on,
// beside 64 x 64, us: float 1400 x 1500 400 / 486, 2000 x 2000 797 / 1 150, 1280 x 2500 423 / 592, but with 66 symmetric ones
// 599 / 400; bf16 1792 x 1792 312 / 372, 1280 x 2500 263 / 301, but with 192 of them for B X 246 / 230 and with 136 symmetric 433 / 399.
int size_of(int planes, int64_t rows, int64_t cols, bool half, int32_t batch)
{
    auto many = [&](int t) { return rows % t || cols % t ? 0 : (half ? rows / t * (rows / t + 1) / 2 : rows / t * (cols / t)) * batch; };
    return many(256) >= kUnits / 2 ? 2 : many(128) >= (planes == 1 ? 193 : half ? 100 : 128) ? 1 : 0;
}

template <typename K>
dol_status ready(K kernel, int lds)
{
    DOL_HIP(allow_dynamic_lds(reinterpret_cast<const void *>(kernel), lds));
    return DOL_OK;
}

template <typename T>
dol_status symmetric(const Layout &L, int32_t batch, bool poly, int k, float alpha, float beta, hipStream_t st)
{
    const int t = L.mp / T::BM;
    const dim3 grid(static_cast<unsigned>(t * (t + 1) / 2), static_cast<unsigned>(batch));
    const int64_t plane = int64_t(L.mp) * L.mp;
    if (poly) {
        if (dol_status s = ready(ns_symmetric_kernel<T, true>, T::LDS)) return s;
        ns_symmetric_kernel<T, true><<<grid, T::NT, T::LDS, st>>>(L.a, T::PA * plane, L.mp, plane, L.mp, L.mp / T::BK, alpha, beta, L.b, T::PA * plane, plane);
    } else {
        const int64_t xplane = int64_t(L.mp) * L.np;
        if (dol_status s = ready(ns_symmetric_kernel<T, false>, T::LDS)) return s;
        ns_symmetric_kernel<T, false><<<grid, T::NT, T::LDS, st>>>(L.x[k], 2 * xplane, L.np, xplane, L.mp, L.np / T::BK, alpha, beta, L.a, T::PA * plane, plane);
    }
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <typename T, typename O, bool TURN>
dol_status apply(const Layout &L, int32_t batch, int k, bool last, float alpha, float beta, const dol_matrix *out, int64_t out_stride, hipStream_t st)
{
    Apply p{};
    p.x = L.x[k], p.b = L.b, p.x_stride = 2 * int64_t(L.mp) * L.np, p.b_stride = T::PA * int64_t(L.mp) * L.mp;
    p.mp = L.mp, p.np = L.np, p.alpha = alpha, p.beta = beta, p.to = L.x[k ^ 1];
    if (last) p.out = out->data, p.out_ld = out->ld, p.out_stride = out_stride, p.out_rows = out->rows, p.out_cols = out->cols;
    if (dol_status s = ready(ns_apply_kernel<T, O, TURN>, T::LDS)) return s;
    const int rows = TURN ? L.mp : L.np, cols = TURN ? L.np : L.mp;
    ns_apply_kernel<T, O, TURN><<<dim3(static_cast<unsigned>(rows / T::BM * (cols / T::BN)), static_cast<unsigned>(batch)), T::NT, T::LDS, st>>>(p);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <typename S>
dol_status newton_schulz_small(const dol_matrix *g, int64_t g_stride, const dol_matrix *out, int64_t out_stride, int32_t batch, int32_t steps, const float *k, float eps,
                               hipStream_t st)
{
    const SmallShape s = small_shape(std::min(g->rows, g->cols), std::max(g->rows, g->cols));
    if (dol_status e = ready(ns_small_kernel<S>, kSmallLds)) return e;
    ns_small_kernel<S><<<batch, kSmallWaves * 64, s.floats() * 4, st>>>(static_cast<const S *>(g->data), g->ld, g_stride, g->rows, g->cols, steps, k[0], k[1], k[2], eps,
                                                                        static_cast<S *>(out->data), out->ld, out_stride);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <int P, typename S>
dol_status newton_schulz(const Layout &L, const dol_matrix *g, int64_t g_stride, const dol_matrix *out, int64_t out_stride, int32_t batch, int32_t steps,
                         const float *k, float eps, Scales e, hipStream_t st)
{
    using Z = Shapes<P>;
    const int parts = static_cast<int>(std::min<int64_t>(kNormParts, (int64_t(g->rows) * g->cols + 4095) / 4096));
    ns_norm_kernel<S><<<dim3(parts, batch), 256, 0, st>>>(static_cast<const S *>(g->data), g->ld, g_stride, g->rows, g->cols, L.part);
    DOL_HIP(hipGetLastError());
    const int32_t gr = L.tall ? L.np : L.mp, gc = L.tall ? L.mp : L.np;
    ns_first_kernel<S><<<dim3(gr / 64, gc / 64, batch), 256, 0, st>>>(static_cast<const S *>(g->data), g->ld, g_stride, g->rows, g->cols, L.tall, L.part, parts, eps, e.x, L.x[0],
                                                                      L.mp, L.np);
    DOL_HIP(hipGetLastError());
    auto two = [](int n) { return std::ldexp(1.0f, n); };
    for (int32_t t = 0; t < steps; ++t) {
        const int from = t & 1;
        for (int poly = 0; poly < 2; ++poly) {
            const float alpha = poly ? k[2] * two(e.b - 2 * e.a) : two(e.a - 2 * e.x), beta = poly ? k[1] * two(e.b - e.a) : 0.0f;
            const int size = size_of(P, L.mp, L.mp, true, batch);
            if (dol_status s = size == 2   ? symmetric<typename Z::template Big<kRows, kRows>>(L, batch, poly, from, alpha, beta, st)
                               : size == 1 ? symmetric<typename Z::template Mid<kRows, kRows>>(L, batch, poly, from, alpha, beta, st)
                                           : symmetric<typename Z::template Small<kRows, kRows>>(L, batch, poly, from, alpha, beta, st))
                return s;
        }
        const bool last = t == steps - 1;
        const float alpha = last ? two(-e.b - e.x) : two(-e.b), beta = last ? k[0] * two(-e.x) : k[0];
        const int size = size_of(P, L.mp, L.np, false, batch);
        if (last && L.tall) {
            if (dol_status s = size == 2   ? apply<typename Z::template Big<kRows, kCols>, S, true>(L, batch, from, last, alpha, beta, out, out_stride, st)
                               : size == 1 ? apply<typename Z::template Mid<kRows, kCols>, S, true>(L, batch, from, last, alpha, beta, out, out_stride, st)
                                           : apply<typename Z::template Small<kRows, kCols>, S, true>(L, batch, from, last, alpha, beta, out, out_stride, st))
                return s;
        } else {
            if (dol_status s = size == 2   ? apply<typename Z::template Big<kCols, kRows>, S, false>(L, batch, from, last, alpha, beta, out, out_stride, st)
                               : size == 1 ? apply<typename Z::template Mid<kCols, kRows>, S, false>(L, batch, from, last, alpha, beta, out, out_stride, st)
                                           : apply<typename Z::template Small<kCols, kRows>, S, false>(L, batch, from, last, alpha, beta, out, out_stride, st))
                return s;
        }
    }
    return DOL_OK;
}

constexpr int32_t kMostSide = 1 << 20;      // 64 rows to a workgroup of a grid's second dimension, a lane's offsets in 32 bits
constexpr int32_t kMostBatch = 65535;

dol_status check_operand(const dol_matrix *m, int64_t stride, int32_t batch, const char *name)
{
    if (!m) return check_matrix(m, name);
    dol_matrix one = *m;
    if (batch == 0) one.rows = 0;       // no matrix, no data
    if (dol_status s = check_matrix(&one, name)) return s;
    if (batch > 1 && stride < 0) return fail(DOL_ESHAPE, "%s's matrices are %lld elements apart", name, static_cast<long long>(stride));
    return DOL_OK;
}

}  // namespace
}  // namespace dol

using namespace dol;

extern "C" {

dol_status dol_newton_schulz_workspace(const dol_matrix *g, int32_t batch, int64_t *bytes)
{
    if (dol_status s = check_operand(g, 0, batch, "g")) return s;
    if (!bytes) return fail(DOL_EINVAL, "bytes is NULL");
    if (batch < 0) return fail(DOL_ESHAPE, "batch = %d", batch);
    if (batch > kMostBatch || g->rows > kMostSide || g->cols > kMostSide)
        return fail(DOL_EUNSUPPORTED, "%d matrices of %d x %d: more than %d, or a side above %d", batch, g->rows, g->cols, kMostBatch, kMostSide);
    *bytes = batch == 0 || g->rows == 0 || g->cols == 0 || small(g) ? 0 : lay_out(g, batch, g->dtype == DOL_BF16 ? 1 : 2, nullptr).bytes;
    return DOL_OK;
}

const char *dol_newton_schulz_kernel(const dol_matrix *g, int32_t batch)
{
    static thread_local char name[64];
    int64_t needs = 0;
    if (dol_newton_schulz_workspace(g, batch, &needs) != DOL_OK || batch == 0 || g->rows == 0 || g->cols == 0) return "";
    if (small(g)) return "ns_small_kernel";
    const int planes = g->dtype == DOL_BF16 ? 1 : 2;
    const Layout L = lay_out(g, batch, planes, nullptr);
    const int side[] = {64, 128, 256}, a = side[size_of(planes, L.mp, L.mp, true, batch)], b = side[size_of(planes, L.mp, L.np, false, batch)];
    snprintf(name, sizeof name, "ns_symmetric_kernel %dx%d, ns_apply_kernel %dx%d", a, a, b, b);
    return name;
}

dol_status dol_newton_schulz(const dol_matrix *g, int64_t g_stride, const dol_matrix *out, int64_t out_stride, int32_t batch, int32_t steps,
                             const float *coefficients, float eps, void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    int64_t needs = 0;
    if (dol_status s = dol_newton_schulz_workspace(g, batch, &needs)) return s;
    if (dol_status s = check_operand(g, g_stride, batch, "g")) return s;
    if (dol_status s = check_operand(out, out_stride, batch, "out")) return s;
    if (g->dtype != out->dtype) return fail(DOL_EINVAL, "g and out are of different types");
    if (g->rows != out->rows || g->cols != out->cols) return fail(DOL_ESHAPE, "g is %d x %d, out %d x %d", g->rows, g->cols, out->rows, out->cols);
    if (batch > 1 && !apart(out->rows, out->ld, batch, out_stride, out->cols)) return fail(DOL_ESHAPE, "out's matrices overlap: %lld elements apart", static_cast<long long>(out_stride));
    if (steps < 1 || steps > 64) return fail(DOL_EINVAL, "%d steps, not 1 to 64", steps);
    if (!coefficients) return fail(DOL_EINVAL, "coefficients is NULL");
    if (!(eps >= 0.0f)) return fail(DOL_EINVAL, "eps = %g is not a number of at least 0", static_cast<double>(eps));
    // how far singular values, and elements of B, can get
    double x = 1.0, xs = 1.0, bs = 0.0;
    for (int32_t t = 0; t < steps; ++t) {
        bs = std::max(bs, bound_of(coefficients, x, false));
        x = bound_of(coefficients, x, true);
        if (t < steps - 1) xs = std::max(xs, x);
        if (!(x <= 64.0 && bs <= 64.0))
            return fail(DOL_EUNSUPPORTED, "with coefficients %g, %g, %g singular values can pass 64 by step %d", static_cast<double>(coefficients[0]),
                        static_cast<double>(coefficients[1]), static_cast<double>(coefficients[2]), t + 1);
    }
    if (batch == 0 || g->rows == 0 || g->cols == 0) return DOL_OK;
    if (dol_status s = check_workspace(workspace, workspace_bytes, needs)) return s;
    // half of fp16's range is kept for what rounding adds
    auto room = [](double most) { return 15 - static_cast<int>(std::ceil(std::log2(std::max(most, 1.0)))); };
    const Scales e{room(xs), room(xs * xs), room(bs)};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool bf = g->dtype == DOL_BF16;
    if (small(g))
        return bf ? newton_schulz_small<__bf16>(g, g_stride, out, out_stride, batch, steps, coefficients, eps, st)
                  : newton_schulz_small<float>(g, g_stride, out, out_stride, batch, steps, coefficients, eps, st);
    const Layout L = lay_out(g, batch, bf ? 1 : 2, workspace);
    return bf ? newton_schulz<1, __bf16>(L, g, g_stride, out, out_stride, batch, steps, coefficients, eps, e, st)
              : newton_schulz<2, float>(L, g, g_stride, out, out_stride, batch, steps, coefficients, eps, e, st);
}

}  // extern "C"
