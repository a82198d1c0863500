// Softmax cross entropy of a linear layer over many classes, and its gradients, without the logits ever in memory.
//
//   l[i, v]    = x[i] . w[v] + bias[v]
//   lse[i]     = log sum_v exp l[i, v],     loss[i] = lse[i] - l[i, target[i]]
//   dl[i, v]   = grad_loss[i] (exp(l[i, v] - lse[i]) - [v = target[i]])
//   grad_x     = dl w,     grad_w = dl^T x,     grad_bias[v] = sum_i dl[i, v]
//
// Forward: a tile of logits stays in the registers that the matrix cores leave it in; of each row it gives the largest logit and the
// sum of the exponentials below it, which a second kernel joins over the tiles.
// Backward: the classes are taken in pieces.  A piece's logits are computed once more, dl is rounded for the matrix cores and written
// both ways round (a few tens of MB that the next launch reads), and grad_x and grad_w are two sets of tiles of one launch.
// Everything is a product of rows with contiguous k (mfma_tile.h), so x and w are also laid out transposed, once a call.
#include "mfma_tile.h"

#include <cfloat>

namespace dol {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kFar = 1e38f;       // logits further from 0 (a bias of the type's lowest value) have no finite l log2e
constexpr int kPad = 256;                               // rows and classes of a piece are filled up to a multiple of this
constexpr int64_t kPieceBytes = int64_t(256) << 20;     // of dl both ways round (see pieces_of)
constexpr int kUnits = 256;                             // compute units of the chip

template <int P>
struct Shapes;
template <>
struct Shapes<1> {      // bf16
    using Big = MfmaTile<bf16x8, 1, 256, 256, 64, 2, 4, 2>;
    using Small = MfmaTile<bf16x8, 1, 128, 128, 64, 2, 2, 2>;
};
template <>
struct Shapes<3> {      // float
    using Big = MfmaTile<bf16x8, 3, 128, 256, 32, 2, 4, 2>;
    using Small = MfmaTile<bf16x8, 3, 128, 128, 32, 2, 2, 2>;
};

template <int P>
struct Source { using T = float; };
template <>
struct Source<1> { using T = __bf16; };

__device__ __forceinline__ bool kept_row(int32_t target, int32_t classes) { return target >= 0 && target < classes; }

// ---------------------------------------------------------------- layouts for the matrix cores

// out[p][r][0..kp) = planes of src[r][0..cols), zeros behind; eight elements to a thread.
template <typename S, int P>
__global__ void __launch_bounds__(256) xent_pack_rows_kernel(const S *src, int64_t ld, int64_t rows, int32_t cols, uint16_t *out, int64_t kp)
{
    const int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, per = kp / 8;
    if (t >= rows * per) return;
    const int64_t r = t / per;
    const int c = static_cast<int>(t - r * per) * 8;
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = c + k < cols ? static_cast<float>(src[r * ld + c + k]) : 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        u32x4 w;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t lo = take_plane<__bf16>(v[2 * k]), hi = take_plane<__bf16>(v[2 * k + 1]);
            w[k] = lo | hi << 16;
        }
        *reinterpret_cast<u32x4 *>(out + (p * rows + r) * kp + c) = w;
    }
}

// out[p][c][0..rp) = planes of src[0..rows)[c], zeros behind; a tile of 64 x 64 to a workgroup.  Rows whose target (if given) names no
// class count as zeros, whatever they hold.
template <typename S, int P>
__global__ void __launch_bounds__(256) xent_pack_cols_kernel(const S *src, int64_t ld, int64_t rows, int32_t cols, const int32_t *target, int32_t classes,
                                                             uint16_t *out, int64_t rp)
{
    __shared__ float tile[64][65];
    const int64_t r0 = static_cast<int64_t>(blockIdx.x) * 64;
    const int32_t c0 = static_cast<int32_t>(blockIdx.y) * 64;
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
#pragma unroll 4
    for (int k = y; k < 64; k += 4) {
        const int64_t r = r0 + k;
        const bool in = r < rows && c0 + x < cols && (!target || kept_row(target[r], classes));
        tile[k][x] = in ? static_cast<float>(src[r * ld + c0 + x]) : 0.0f;
    }
    __syncthreads();
    const int q = threadIdx.x & 7;
    for (int c = threadIdx.x >> 3; c < 64 && c0 + c < cols; c += 32) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = tile[q * 8 + k][c];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            u32x4 w;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t lo = take_plane<__bf16>(v[2 * k]), hi = take_plane<__bf16>(v[2 * k + 1]);
                w[k] = lo | hi << 16;
            }
            *reinterpret_cast<u32x4 *>(out + (static_cast<int64_t>(p) * cols + c0 + c) * rp + r0 + q * 8) = w;
        }
    }
}

// ---------------------------------------------------------------- forward

// Rows of a tile are classes, its columns samples.  part[(WM * class tile + wavefront row) * n_pad + sample] = (top, sum of exp(l - top))
// over these classes, top the largest logit among them; at[sample] = l of the target.
// The exponentials are taken as 2^(l log2e - c), c = top log2e rounded: one multiply-add a logit.  What c lost is the same factor in all of
// them, and divided out of the sum as the top's own term: that is 1 to the bit, and a row whose other classes vanish has lse = top.
template <typename T>
__global__ void __launch_bounds__(T::NT, 2) xent_sums_kernel(Planes w, Planes x, int32_t classes, int32_t rows, int steps, const float *bias, const int32_t *target,
                                                             float2 *part, int64_t n_pad, float *at)
{
    extern __shared__ __align__(128) char smem[];
    const int tm = (classes + T::BM - 1) / T::BM, tn = (rows + T::BN - 1) / T::BN;
    int mt, nt;
    tile_of(xcd_contiguous(blockIdx.x, gridDim.x), tm, tn, 4, mt, nt);
    f32x4 acc[T::MI][T::NI];
    T::run(w, static_cast<int64_t>(mt) * T::BM, classes, x, static_cast<int64_t>(nt) * T::BN, rows, 0, steps, smem, acc);
    const int m0 = mt * T::BM, n0 = nt * T::BN + T::col_of();
    if (bias || m0 + T::BM > classes) {
#pragma unroll
        for (int i = 0; i < T::MI; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int m = m0 + T::row_of(i) + e;
                const float b = m >= classes ? -INFINITY : bias ? bias[m] : 0.0f;
#pragma unroll
                for (int j = 0; j < T::NI; ++j) acc[i][j][e] = m >= classes ? -INFINITY : acc[i][j][e] + b;
            }
    }
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < T::NI; ++j) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < T::MI; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, acc[i][j][e]);
        top = with_lane32<MaxOp>(with_lane16<MaxOp>(top));
        float sum = 0.0f;
        if (__builtin_fabsf(top) <= kFar) {
            const float c = top * kLog2e;
#pragma unroll
            for (int i = 0; i < T::MI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][e], kLog2e, -c));
            sum = with_lane32<AddOp>(with_lane16<AddOp>(sum)) / __builtin_amdgcn_exp2f(__builtin_fmaf(top, kLog2e, -c));
        } else {
#pragma unroll
            for (int i = 0; i < T::MI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float l = acc[i][j][e];
                    sum += l == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((l - top) * kLog2e);
                }
            sum = with_lane32<AddOp>(with_lane16<AddOp>(sum));
        }
        const int n = n0 + j;
        if (n < rows && lane < 16) part[static_cast<int64_t>(mt * T::WM + (threadIdx.x >> 6) / T::WN) * n_pad + n] = make_float2(top, sum);
        const int t = n < rows ? target[n] - m0 - T::row_of(0) : -1;       // the target's row, from this lane's first
        if (t >= 0 && (t & 15) < 4 && t < T::TM) {
            float l = 0.0f;
#pragma unroll
            for (int i = 0; i < T::MI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) l = t == i * 16 + e ? acc[i][j][e] : l;
            at[n] = l;
        }
    }
}

// Joins the parts of a sample: sixty-four samples to a workgroup, a quarter of the parts to each of its wavefronts.
__global__ void __launch_bounds__(256) xent_join_kernel(const float2 *part, int parts, int64_t n_pad, int32_t rows, int32_t classes, const int32_t *target,
                                                        const float *at, float *loss, float *lse)
{
    __shared__ float2 red[4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 64 + lane;
    float top = -INFINITY, s = 0.0f;
    auto join = [&](float2 p) {
        if (p.y == 0.0f) return;                    // no logit above -inf
        const float to = fmaxf(top, p.x);
        s = (s == 0.0f ? 0.0f : s * __builtin_amdgcn_exp2f((top - to) * kLog2e)) + p.y * __builtin_amdgcn_exp2f((p.x - to) * kLog2e);
        top = to;
    };
    if (n < rows)
        for (int k = w; k < parts; k += 4) join(part[k * n_pad + n]);
    red[w][lane] = make_float2(top, s);
    __syncthreads();
    if (w != 0 || n >= rows) return;
    for (int k = 1; k < 4; ++k) join(red[k][lane]);
    const float lg = kLn2 * log2f(s);
    lse[n] = s == 0.0f ? -INFINITY : top + lg;
    // (a row without any class left has lse = -inf and, by this rule, loss = +inf)
    loss[n] = !kept_row(target[n], classes) ? 0.0f : s == 0.0f ? INFINITY : lg + (top - at[n]);
}

// ---------------------------------------------------------------- backward

// dl of one piece of classes, rounded to P planes: dl[p][sample][class of the piece] and dlt[p][class of the piece][sample], both filled up
// with zeros to kPad.  bias_part[(nt * WN + wavefront column) * piece + class] = sums of the unrounded dl (if asked for).
template <typename T>
__global__ void __launch_bounds__(T::NT, 2) xent_dlogits_kernel(Planes w, Planes x, int32_t classes, int32_t rows, int steps, int32_t first, int32_t piece,
                                                                const float *bias, const int32_t *target, const float *lse, const float *grad_loss,
                                                                uint16_t *dl, uint16_t *dlt, int64_t n_pad, float *bias_part)
{
    extern __shared__ __align__(128) char smem[];
    const int tm = piece / T::BM, tn = static_cast<int>(n_pad / T::BN);
    int mt, nt;
    tile_of(xcd_contiguous(blockIdx.x, gridDim.x), tm, tn, 4, mt, nt);
    f32x4 acc[T::MI][T::NI];
    const int m0 = first + mt * T::BM;
    // (a tile that lies wholly past the last class or sample repeats the last row; all of it is masked below)
    T::run(w, min(m0, classes - 1), classes, x, min(nt * T::BN, rows - 1), rows, 0, steps, smem, acc);
    const int n0 = nt * T::BN + T::col_of();
    float off[T::NI], scale[T::NI], own[T::NI];
    bool kept[T::NI];
    int at[T::NI];
    bool hit = false, far = false;
#pragma unroll
    for (int j = 0; j < T::NI; ++j) {
        const int n = n0 + j;
        const int32_t t = n < rows ? target[n] : -1;
        const float z = n < rows ? lse[n] : 0.0f;
        kept[j] = kept_row(t, classes) && z != -INFINITY;
        const float g = kept[j] ? grad_loss[n] : 0.0f;
        off[j] = kept[j] ? z : 0.0f;
        scale[j] = g;
        far |= !(__builtin_fabsf(off[j]) <= kFar);
        // the target's own exp(l - lse) - 1 is small where the network is right: not taken as a difference
        at[j] = kept[j] ? t - m0 - T::row_of(0) : -1;
        own[j] = 0.0f;
        if (at[j] >= 0 && at[j] < T::TM && (at[j] & 15) < 4) {
            hit = true;
            float l = 0.0f;
#pragma unroll
            for (int i = 0; i < T::MI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) l = at[j] == i * 16 + e ? acc[i][j][e] : l;
            own[j] = g * expm1f((bias ? l + bias[t] : l) - z);
        }
    }
    auto fill = [&](auto exponential) {
#pragma unroll
        for (int i = 0; i < T::MI; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int m = m0 + T::row_of(i) + e;
                const bool in = m < classes;
                const float b = bias && in ? bias[m] : 0.0f;
#pragma unroll
                for (int j = 0; j < T::NI; ++j) {
                    const float p = exponential(acc[i][j][e] + b, j);
                    acc[i][j][e] = in && kept[j] ? p : 0.0f;
                }
            }
    };
    if (!__any(far)) {
#pragma unroll
        for (int j = 0; j < T::NI; ++j) {
            // exp(l - lse) = 2^(l log2e - off) 2^(-rest): what lse log2e loses to rounding goes into the factor of the row
            const float z = off[j];
            off[j] = z * kLog2e;
            scale[j] *= __builtin_amdgcn_exp2f(-__builtin_fmaf(z, kLog2e, -off[j]));
        }
        fill([&](float l, int j) { return __builtin_amdgcn_exp2f(__builtin_fmaf(l, kLog2e, -off[j])) * scale[j]; });
    } else
        fill([&](float l, int j) { return __builtin_amdgcn_exp2f((l - off[j]) * kLog2e) * scale[j]; });
    if (hit)
#pragma unroll
        for (int j = 0; j < T::NI; ++j)
#pragma unroll
            for (int i = 0; i < T::MI; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = at[j] == i * 16 + e ? own[j] : acc[i][j][e];
    if (bias_part) {
        float *to = bias_part + static_cast<int64_t>(nt * T::WN + (threadIdx.x >> 6) % T::WN) * piece + mt * T::BM;
#pragma unroll
        for (int i = 0; i < T::MI; ++i) {
            f32x4 s;
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = reduce16<AddOp>((acc[i][0][e] + acc[i][1][e]) + (acc[i][2][e] + acc[i][3][e]));
            if ((threadIdx.x & 15) == 0) *reinterpret_cast<f32x4 *>(to + T::row_of(i)) = s;
        }
    }
#pragma unroll 1
    for (int p = 0; p < T::P; ++p) {
        uint16_t *to = dlt + (static_cast<int64_t>(p) * piece + mt * T::BM) * n_pad + n0;
#pragma unroll
        for (int i = 0; i < T::MI; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                u32x2 v;
                v[0] = bits16<__bf16>(acc[i][0][e]) | bits16<__bf16>(acc[i][1][e]) << 16;
                v[1] = bits16<__bf16>(acc[i][2][e]) | bits16<__bf16>(acc[i][3][e]) << 16;
                *reinterpret_cast<u32x2 *>(to + (T::row_of(i) + e) * n_pad) = v;
            }
        T::store_transposed(smem, dl + (p * n_pad + static_cast<int64_t>(nt) * T::BN) * piece + mt * T::BM, piece, T::BN,
                            [&](int i, int j, int e) { float v = acc[i][j][e]; const uint32_t b = take_plane<__bf16>(v); acc[i][j][e] = v; return b; });
    }
}

// One set of tiles of the launch that follows: out = a b^T over `steps` steps, in `splits` shares of the steps.
struct Product {
    Planes a, b;
    int32_t M, N;               // rows of out, columns of out
    int32_t tm, tn, splits, steps;
    float *part;                // [splits][M][part_ld], or null: out is written
    int64_t part_ld;
    bool add;                   // to what part holds
    void *out;
    int64_t out_ld;
};

template <typename T, typename O>
__global__ void __launch_bounds__(T::NT, 2) xent_products_kernel(Product p0, Product p1)
{
    extern __shared__ __align__(128) char smem[];
    int id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int first = p0.tm * p0.tn * p0.splits;
    const Product &p = id < first ? p0 : p1;
    if (id >= first) id -= first;
    const int tiles = p.tm * p.tn, split = id / tiles;
    int mt, nt;
    tile_of(id - split * tiles, p.tm, p.tn, 8, mt, nt);
    const int s0 = static_cast<int>(static_cast<int64_t>(p.steps) * split / p.splits), s1 = static_cast<int>(static_cast<int64_t>(p.steps) * (split + 1) / p.splits);
    f32x4 acc[T::MI][T::NI];
    T::run(p.a, static_cast<int64_t>(mt) * T::BM, p.M, p.b, static_cast<int64_t>(nt) * T::BN, p.N, static_cast<int64_t>(s0) * T::BK, s1 - s0, smem, acc);
    const int n = nt * T::BN + T::col_of(), left = p.N - n;
    const bool vec = p.out_ld % 4 == 0 && (reinterpret_cast<uintptr_t>(p.out) & (4 * sizeof(O) - 1)) == 0;
#pragma unroll
    for (int i = 0; i < T::MI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int m = mt * T::BM + T::row_of(i) + e;
            if (m >= p.M || left <= 0) continue;
            f32x4 v = {acc[i][0][e], acc[i][1][e], acc[i][2][e], acc[i][3][e]};
            if (p.part) {       // (its rows are filled up to whole fours)
                f32x4 *to = reinterpret_cast<f32x4 *>(p.part + (static_cast<int64_t>(split) * p.M + m) * p.part_ld + n);
                *to = p.add ? *to + v : v;
            } else
                store4(static_cast<O *>(p.out) + m * p.out_ld + n, v, left, vec);
        }
}

// out = the sum of the parts in their order, for one set or two; four columns to a thread.
struct Sum {
    const float *part;
    int32_t M, N, splits;
    int64_t part_ld;
    void *out;
    int64_t out_ld;
};

template <typename O>
__global__ void __launch_bounds__(256) xent_sum_parts_kernel(Sum s)
{
    const int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, per = (s.N + 3) / 4;
    if (t >= s.M * per) return;
    const int64_t m = t / per;
    const int n = static_cast<int>(t - m * per) * 4;
    f32x4 v = {0, 0, 0, 0};
    for (int k = 0; k < s.splits; ++k) v += *reinterpret_cast<const f32x4 *>(s.part + (static_cast<int64_t>(k) * s.M + m) * s.part_ld + n);
    const bool vec = s.out_ld % 4 == 0 && (reinterpret_cast<uintptr_t>(s.out) & (4 * sizeof(O) - 1)) == 0;
    store4(static_cast<O *>(s.out) + m * s.out_ld + n, v, s.N - n, vec);
}

__global__ void __launch_bounds__(256) xent_bias_kernel(const float *part, int parts, int32_t piece, int32_t n, float *out)
{
    const int v = blockIdx.x * 256 + threadIdx.x;
    if (v >= n) return;
    float s = 0.0f;
    for (int k = 0; k < parts; ++k) s += part[static_cast<int64_t>(k) * piece + v];
    out[v] = s;
}

template <typename O>
__global__ void __launch_bounds__(256) xent_zero_kernel(O *out, int64_t ld, int64_t rows, int32_t cols)
{
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; t < rows * cols; t += static_cast<int64_t>(gridDim.x) * 256)
        out[t / cols * ld + t % cols] = static_cast<O>(0.0f);
}

// ---------------------------------------------------------------- host side

constexpr int32_t kMostRows = 1 << 22;      // of either operand: a lane's offsets into a tile of dl fit 32 bits
constexpr int32_t kMostWidth = 1 << 20;     // of a row: 64 columns to a workgroup of a grid's second dimension

bool direct(const dol_matrix *m)            // can be read by the tiles as it is
{
    return m->dtype == DOL_BF16 && m->cols % 64 == 0 && m->ld % 8 == 0 && m->ld <= kMostRows && !(reinterpret_cast<uintptr_t>(m->data) & 15);
}

struct Layout {
    int32_t rows, width, classes;
    int64_t kp, n_pad, v_pad;               // width, rows and classes as they are laid out
    int32_t piece, pieces;
    bool big;                               // tiles of logits
    uint16_t *xp, *wp, *xt, *wt, *dl, *dlt;
    float2 *part;
    float *at, *bias_part, *part_x, *part_w;
    bool big_products;
    int32_t splits_x, splits_w;
    int64_t part_ld;
    int64_t bytes;
};

int32_t tiles(int64_t n, int t) { return static_cast<int32_t>((n + t - 1) / t); }

template <int P>
Layout lay_out(const dol_matrix *x, const dol_matrix *w, bool backward, void *workspace)
{
    using Big = typename Shapes<P>::Big;
    using Small = typename Shapes<P>::Small;
    Layout L{};
    L.rows = x->rows, L.width = x->cols, L.classes = w->rows;
    L.kp = round_up(L.width, 64), L.n_pad = round_up(L.rows, kPad);
    // Tiles of 256 x 256 (float 128 x 256) do more with what they load; smaller ones fill the chip sooner.
    L.big = int64_t(tiles(L.classes, Big::BM)) * tiles(L.rows, Big::BN) >= kUnits * 3 / 4;
    Carver c(workspace);
    if (!direct(x)) L.xp = c.take<uint16_t>(P * int64_t(L.rows) * L.kp);
    if (!direct(w)) L.wp = c.take<uint16_t>(P * int64_t(L.classes) * L.kp);
    if (!backward) {
        const int parts = L.big ? tiles(L.classes, Big::BM) * Big::WM : tiles(L.classes, Small::BM) * Small::WM;
        L.part = c.take<float2>(int64_t(parts) * L.n_pad);
        L.at = c.take<float>(L.rows);
        L.bytes = c.used;
        return L;
    }
    const int64_t most = std::max<int64_t>(kPad, kPieceBytes / (4 * P * L.n_pad) / kPad * kPad);
    L.pieces = static_cast<int32_t>((L.classes + most - 1) / most);
    L.piece = static_cast<int32_t>(round_up((L.classes + L.pieces - 1) / L.pieces, kPad));
    L.pieces = tiles(L.classes, L.piece);
    L.v_pad = int64_t(L.pieces) * L.piece;
    L.xt = c.take<uint16_t>(P * int64_t(L.width) * L.n_pad);
    L.wt = c.take<uint16_t>(P * int64_t(L.width) * L.v_pad);
    L.dl = c.take<uint16_t>(P * L.n_pad * L.piece);
    L.dlt = c.take<uint16_t>(P * L.n_pad * L.piece);
    L.bias_part = c.take<float>(L.n_pad / 64 * L.piece);
    // Both products of a piece share a launch: their k is split so that the launch has a workgroup of equal length for every place there
    // is, of at least 256 elements of k.
    const int64_t kx = L.piece, kw = L.n_pad;
    auto total = [&](int bm, int bn) { return (int64_t(tiles(L.rows, bm)) * kx + int64_t(tiles(std::min(L.piece, L.classes), bm)) * kw) * tiles(L.width, bn); };
    L.big_products = total(Big::BM, Big::BN) / kUnits >= 1024;
    const int64_t share = std::max<int64_t>(256, L.big_products ? total(Big::BM, Big::BN) / kUnits : total(Small::BM, Small::BN) / (2 * kUnits));
    L.splits_x = static_cast<int32_t>(std::max<int64_t>(1, (kx + share / 2) / share));
    L.splits_w = static_cast<int32_t>(std::max<int64_t>(1, (kw + share / 2) / share));
    L.part_ld = round_up(L.width, 4);
    if (L.splits_x > 1 || L.pieces > 1) L.part_x = c.take<float>(int64_t(L.splits_x) * L.rows * L.part_ld);
    if (L.splits_w > 1) L.part_w = c.take<float>(int64_t(L.splits_w) * std::min(L.piece, L.classes) * L.part_ld);
    L.bytes = c.used;
    return L;
}

unsigned blocks(int64_t n) { return static_cast<unsigned>((n + 255) / 256); }

template <int P>
dol_status pack(const dol_matrix *m, uint16_t *out, int64_t kp, Planes *p, hipStream_t st)
{
    using S = typename Source<P>::T;
    if (!out) {
        *p = Planes{static_cast<const uint16_t *>(m->data), m->ld, 0};
        return DOL_OK;
    }
    xent_pack_rows_kernel<S, P><<<blocks(m->rows * (kp / 8)), 256, 0, st>>>(static_cast<const S *>(m->data), m->ld, m->rows, m->cols, out, kp);
    DOL_HIP(hipGetLastError());
    *p = Planes{out, kp, m->rows * kp};
    return DOL_OK;
}

template <typename T>
dol_status launch_sums(const Layout &L, Planes w, Planes x, const float *bias, const int32_t *target, float *loss, float *lse, hipStream_t st)
{
    DOL_HIP(allow_dynamic_lds(reinterpret_cast<const void *>(xent_sums_kernel<T>), T::LDS));
    const int tm = tiles(L.classes, T::BM), tn = tiles(L.rows, T::BN);
    xent_sums_kernel<T><<<tm * tn, T::NT, T::LDS, st>>>(w, x, L.classes, L.rows, static_cast<int>(L.kp / T::BK), bias, target, L.part, L.n_pad, L.at);
    DOL_HIP(hipGetLastError());
    xent_join_kernel<<<tiles(L.rows, 64), 256, 0, st>>>(L.part, tm * T::WM, L.n_pad, L.rows, L.classes, target, L.at, loss, lse);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <int P>
dol_status forward(const Layout &L, const dol_matrix *x, const dol_matrix *w, const float *bias, const int32_t *target, float *loss, float *lse, hipStream_t st)
{
    Planes xp, wp;
    if (dol_status s = pack<P>(x, L.xp, L.kp, &xp, st)) return s;
    if (dol_status s = pack<P>(w, L.wp, L.kp, &wp, st)) return s;
    return L.big ? launch_sums<typename Shapes<P>::Big>(L, wp, xp, bias, target, loss, lse, st)
                 : launch_sums<typename Shapes<P>::Small>(L, wp, xp, bias, target, loss, lse, st);
}

template <typename T>
dol_status launch_dlogits(const Layout &L, Planes w, Planes x, int32_t first, const float *bias, const int32_t *target, const float *lse,
                          const float *grad_loss, float *grad_bias, hipStream_t st)
{
    DOL_HIP(allow_dynamic_lds(reinterpret_cast<const void *>(xent_dlogits_kernel<T>), T::LDS));
    const int tm = L.piece / T::BM, tn = static_cast<int>(L.n_pad / T::BN);
    xent_dlogits_kernel<T><<<tm * tn, T::NT, T::LDS, st>>>(w, x, L.classes, L.rows, static_cast<int>(L.kp / T::BK), first, L.piece, bias, target, lse, grad_loss,
                                                           L.dl, L.dlt, L.n_pad, grad_bias ? L.bias_part : nullptr);
    DOL_HIP(hipGetLastError());
    if (grad_bias) {
        const int32_t n = std::min(L.piece, L.classes - first);
        xent_bias_kernel<<<blocks(n), 256, 0, st>>>(L.bias_part, tn * T::WN, L.piece, n, grad_bias + first);
        DOL_HIP(hipGetLastError());
    }
    return DOL_OK;
}

template <typename T, typename O>
dol_status launch_products(Product a, Product b, hipStream_t st)
{
    DOL_HIP(allow_dynamic_lds(reinterpret_cast<const void *>(xent_products_kernel<T, O>), T::LDS));
    for (Product *p : {&a, &b})
        if (p->M > 0) p->tm = tiles(p->M, T::BM), p->tn = tiles(p->N, T::BN), p->steps /= T::BK;
    const int n = a.tm * a.tn * a.splits + b.tm * b.tn * b.splits;
    if (n == 0) return DOL_OK;
    xent_products_kernel<T, O><<<n, T::NT, T::LDS, st>>>(a, b);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <typename O>
dol_status sum_parts(const Product &p, hipStream_t st)
{
    const Sum s{p.part, p.M, p.N, p.splits, p.part_ld, p.out, p.out_ld};
    xent_sum_parts_kernel<O><<<blocks(int64_t(p.M) * ((p.N + 3) / 4)), 256, 0, st>>>(s);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <int P>
dol_status reverse(const Layout &L, const dol_matrix *x, const dol_matrix *w, const float *bias, const int32_t *target, const float *lse,
                   const float *grad_loss, const dol_matrix *grad_x, const dol_matrix *grad_w, float *grad_bias, hipStream_t st)
{
    using S = typename Source<P>::T;
    using Big = typename Shapes<P>::Big;
    using Small = typename Shapes<P>::Small;
    Planes xp, wp;
    if (dol_status s = pack<P>(x, L.xp, L.kp, &xp, st)) return s;
    if (dol_status s = pack<P>(w, L.wp, L.kp, &wp, st)) return s;
    if (grad_w) {
        xent_pack_cols_kernel<S, P><<<dim3(static_cast<unsigned>(L.n_pad / 64), tiles(L.width, 64)), 256, 0, st>>>(
            static_cast<const S *>(x->data), x->ld, L.rows, L.width, target, L.classes, L.xt, L.n_pad);
        DOL_HIP(hipGetLastError());
    }
    if (grad_x) {
        xent_pack_cols_kernel<S, P><<<dim3(static_cast<unsigned>(L.v_pad / 64), tiles(L.width, 64)), 256, 0, st>>>(
            static_cast<const S *>(w->data), w->ld, L.classes, L.width, nullptr, 0, L.wt, L.v_pad);
        DOL_HIP(hipGetLastError());
    }
    for (int32_t k = 0; k < L.pieces; ++k) {
        const int32_t first = k * L.piece, n = std::min(L.piece, L.classes - first);
        if (dol_status s = L.big ? launch_dlogits<Big>(L, wp, xp, first, bias, target, lse, grad_loss, grad_bias, st)
                                 : launch_dlogits<Small>(L, wp, xp, first, bias, target, lse, grad_loss, grad_bias, st))
            return s;
        Product a{}, b{};
        if (grad_x) {
            a.a = Planes{L.dl, L.piece, L.n_pad * L.piece}, a.b = Planes{L.wt + first, L.v_pad, L.width * L.v_pad};
            a.M = L.rows, a.N = L.width, a.splits = L.splits_x, a.steps = L.piece;
            a.part = L.part_x, a.part_ld = L.part_ld, a.add = k > 0, a.out = grad_x->data, a.out_ld = grad_x->ld;
        }
        if (grad_w) {
            b.a = Planes{L.dlt, L.n_pad, L.n_pad * L.piece}, b.b = Planes{L.xt, L.n_pad, L.width * L.n_pad};
            b.M = n, b.N = L.width, b.splits = L.splits_w, b.steps = static_cast<int32_t>(L.n_pad);
            b.part = L.part_w, b.part_ld = L.part_ld, b.out = static_cast<S *>(grad_w->data) + first * grad_w->ld, b.out_ld = grad_w->ld;
        }
        if (dol_status s = L.big_products ? launch_products<Big, S>(a, b, st) : launch_products<Small, S>(a, b, st)) return s;
        if (b.part)
            if (dol_status s = sum_parts<S>(b, st)) return s;
        if (a.part && k == L.pieces - 1)
            if (dol_status s = sum_parts<S>(a, st)) return s;
    }
    return DOL_OK;
}

template <typename S>
dol_status zero(const dol_matrix *m, hipStream_t st)
{
    if (!m || m->rows == 0) return DOL_OK;
    xent_zero_kernel<S><<<std::min(blocks(int64_t(m->rows) * m->cols), 4096u), 256, 0, st>>>(static_cast<S *>(m->data), m->ld, m->rows, m->cols);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

dol_status check_operands(const dol_matrix *x, const dol_matrix *w)
{
    if (dol_status s = check_matrix(x, "x")) return s;
    if (dol_status s = check_matrix(w, "weight")) return s;
    if (x->dtype != w->dtype) return fail(DOL_EINVAL, "x and weight are of different types");
    if (x->cols != w->cols) return fail(DOL_ESHAPE, "x has %d columns, weight %d", x->cols, w->cols);
    if (w->rows < 1 || w->cols < 1) return fail(DOL_ESHAPE, "%d classes of %d elements: there has to be one of each", w->rows, w->cols);
    if (x->rows > kMostRows || w->rows > kMostRows || w->cols > kMostWidth)
        return fail(DOL_EUNSUPPORTED, "%d rows, %d classes of %d elements: more than %d, or %d elements", x->rows, w->rows, w->cols, kMostRows, kMostWidth);
    return DOL_OK;
}

}  // namespace

dol_status check_matrix(const dol_matrix *m, const char *name)
{
    if (!m) return fail(DOL_EINVAL, "%s is NULL", name);
    if (m->dtype != DOL_F32 && m->dtype != DOL_BF16) return fail(DOL_EINVAL, "%s has unknown type %d", name, m->dtype);
    if (m->rows < 0 || m->cols < 0) return fail(DOL_ESHAPE, "%s is %d x %d", name, m->rows, m->cols);
    if (m->ld < m->cols) return fail(DOL_ESHAPE, "%s.ld = %lld smaller than its %d columns", name, static_cast<long long>(m->ld), m->cols);
    if (m->rows > 0 && m->cols > 0) {
        if (!m->data) return fail(DOL_EINVAL, "%s.data is NULL", name);
        if (reinterpret_cast<uintptr_t>(m->data) & (m->dtype == DOL_F32 ? 3 : 1)) return fail(DOL_EINVAL, "%s.data is not aligned to its elements", name);
    }
    return DOL_OK;
}

dol_status check_workspace(const void *workspace, int64_t has, int64_t needs)
{
    if (needs > 0 && !workspace) return fail(DOL_EINVAL, "workspace is NULL, the call needs %lld bytes", static_cast<long long>(needs));
    if (has < needs) return fail(DOL_EINVAL, "the workspace has %lld bytes, the call needs %lld", static_cast<long long>(has), static_cast<long long>(needs));
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return fail(DOL_EINVAL, "the workspace is not aligned to 256 bytes");
    return DOL_OK;
}

}  // namespace dol

using namespace dol;

extern "C" {

dol_status dol_cross_entropy_workspace(const dol_matrix *x, const dol_matrix *weight, int32_t backward, int64_t *bytes)
{
    if (dol_status s = check_operands(x, weight)) return s;
    if (!bytes) return fail(DOL_EINVAL, "bytes is NULL");
    *bytes = x->rows == 0 ? 0 : (x->dtype == DOL_BF16 ? lay_out<1>(x, weight, backward, nullptr) : lay_out<3>(x, weight, backward, nullptr)).bytes;
    return DOL_OK;
}

dol_status dol_cross_entropy(const dol_matrix *x, const dol_matrix *weight, const float *bias, const int32_t *target, float *loss, float *lse,
                             void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    if (dol_status s = check_operands(x, weight)) return s;
    if (x->rows == 0) return DOL_OK;
    if (!target || !loss || !lse) return fail(DOL_EINVAL, "target, loss or lse is NULL");
    const bool bf = x->dtype == DOL_BF16;
    const Layout L = bf ? lay_out<1>(x, weight, false, workspace) : lay_out<3>(x, weight, false, workspace);
    if (dol_status s = check_workspace(workspace, workspace_bytes, L.bytes)) return s;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return bf ? forward<1>(L, x, weight, bias, target, loss, lse, st) : forward<3>(L, x, weight, bias, target, loss, lse, st);
}

dol_status dol_cross_entropy_backward(const dol_matrix *x, const dol_matrix *weight, const float *bias, const int32_t *target, const float *lse,
                                      const float *grad_loss, const dol_matrix *grad_x, const dol_matrix *grad_weight, float *grad_bias,
                                      void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    if (dol_status s = check_operands(x, weight)) return s;
    for (const auto &g : {std::make_pair(grad_x, x), std::make_pair(grad_weight, weight)}) {
        if (!g.first) continue;
        const char *name = g.second == x ? "grad_x" : "grad_weight";
        if (dol_status s = check_matrix(g.first, name)) return s;
        if (g.first->dtype != x->dtype) return fail(DOL_EINVAL, "%s is of another type than x", name);
        if (g.first->rows != g.second->rows || g.first->cols != g.second->cols)
            return fail(DOL_ESHAPE, "%s is %d x %d, not %d x %d", name, g.first->rows, g.first->cols, g.second->rows, g.second->cols);
    }
    if (!grad_x && !grad_weight && !grad_bias) return fail(DOL_EINVAL, "no gradient is asked for");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool bf = x->dtype == DOL_BF16;
    if (x->rows == 0) {                     // sums over no rows
        if (dol_status s = bf ? zero<__bf16>(grad_weight, st) : zero<float>(grad_weight, st)) return s;
        const dol_matrix b{DOL_F32, 1, weight->rows, weight->rows, grad_bias};
        return grad_bias ? zero<float>(&b, st) : DOL_OK;
    }
    if (!target || !lse || !grad_loss) return fail(DOL_EINVAL, "target, lse or grad_loss is NULL");
    const Layout L = bf ? lay_out<1>(x, weight, true, workspace) : lay_out<3>(x, weight, true, workspace);
    if (dol_status s = check_workspace(workspace, workspace_bytes, L.bytes)) return s;
    return bf ? reverse<1>(L, x, weight, bias, target, lse, grad_loss, grad_x, grad_weight, grad_bias, st)
              : reverse<3>(L, x, weight, bias, target, lse, grad_loss, grad_x, grad_weight, grad_bias, st);
}

}  // extern "C"
