// Softmax cross entropy of a linear layer over many classes, and its gradients, without the logits ever in memory.
//
//   l[i, v]    = x[i] . w[v] + bias[v]
//   lse[i]     = log sum_v exp l[i, v],     loss[i] = lse[i] - l[i, target[i]]
//   dl[i, v]   = grad_loss[i] (exp(l[i, v] - lse[i]) - [v = target[i]])
//   grad_x     = dl w,     grad_w = dl^T x,     grad_bias[v] = sum_i dl[i, v]
//
// Forward: a tile of logits stays in the registers that the matrix cores leave it in; of each row it gives the largest logit and the
// sum of the exponentials below it, which a second kernel joins over the tiles.
// Backward: the classes are taken in pieces.  A piece's logits are computed once more, dl is rounded for the matrix cores and written (a
// hundred MB or so that the next launch reads), and grad_x and grad_w are two sets of tiles of one launch, which read dl, x and w as they
// lie, along rows or across them (mfma_tile.h).
// A few classes, whose logits a workgroup holds, have a form of their own (xent_few_kernel).
#include "mfma_products.h"

#include <cstdio>

namespace dol {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
// Logits further from 0 (masks of -1e10, of the type's lowest value) are subtracted from each other before they are multiplied by log2e: what
// rounding takes from l log2e, 2^-24 of it, is an exponent of its own, 1/16 here and 512 at 1e10.
constexpr float kFar = 1e6f;
constexpr int kPad = 256;                               // rows and classes of a piece are filled up to a multiple of this
constexpr int64_t kMostPieceBytes = int64_t(192) << 20; // of dl

// ---------------------------------------------------------------- layouts for the matrix cores

// Two of them in one launch, eight elements to a thread.  Bytes bound it: 8 192 x 1 024 of bf16 in 9.5 us, 3.5 TB/s.
template <typename S, int P>
__global__ void __launch_bounds__(256) xent_pack_kernel(Pack p0, Pack p1)
{
    if (blockIdx.x < p0.blocks) pack_rows<S, P>(p0, blockIdx.x);
    else pack_rows<S, P>(p1, blockIdx.x - p0.blocks);
}

// ---------------------------------------------------------------- forward

// Rows of a tile are classes, its columns samples.  part[(WM * class tile + wavefront row) * n_pad + sample] = (top, sum of exp(l - top))
// over these classes, top the largest logit among them; at[sample] = l of the target.
// The exponentials are taken as 2^(l log2e - c), c = top log2e rounded: one multiply-add a logit.  What c lost is the same factor in all of
// them, and divided out of the sum as the top's own term: that is 1 to the bit, and a row whose other classes vanish has lse = top.
// The product bounds it: 8 192 x 1 024 into 65 535 in bf16 927 to 970 us, 1 133 to 1 186 TFLOP/s.
template <typename T>
__global__ void __launch_bounds__(T::NT, 2) xent_sums_kernel(Planes w, Planes x, int32_t classes, int32_t rows, int steps, const float *bias, const int32_t *target,
                                                             float2 *part, int64_t n_pad, float *at)
{
    extern __shared__ __align__(128) char smem[];
    const int tm = (classes + T::BM - 1) / T::BM, tn = (rows + T::BN - 1) / T::BN;
    int mt, nt;
    tile_of(xcd_contiguous(blockIdx.x, gridDim.x), tm, tn, 4, mt, nt);
    f32x4 acc[T::MI][T::NI];
    T::clear(acc);
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
                    sum += l == -INFINITY ? 0.0f : l == top ? 1.0f : __builtin_amdgcn_exp2f((l - top) * kLog2e);      // (inf - inf is NaN)
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

// Joins the parts of a sample: sixty-four samples to a workgroup, a share of the parts to each of its wavefronts.  Waits for its loads: 512
// parts of 8 192 samples in 18.6 us, 16 of 4 096 in 4.5.
constexpr int kJoinWaves = 16;
__global__ void __launch_bounds__(kJoinWaves * 64) xent_join_kernel(const float2 *part, int parts, int64_t n_pad, int32_t rows, int32_t classes, const int32_t *target,
                                                                    const float *at, float *loss, float *lse)
{
    __shared__ float2 red[kJoinWaves][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 64 + lane;
    float top = -INFINITY, s = 0.0f;
    auto join = [&](float2 p) {
        if (p.y == 0.0f) return;                    // no logit above -inf
        const float to = fmaxf(top, p.x);
        auto scale = [&](float from) { return from == to ? 1.0f : __builtin_amdgcn_exp2f((from - to) * kLog2e); };        // (inf - inf is NaN)
        s = (s == 0.0f ? 0.0f : s * scale(top)) + p.y * scale(p.x);
        top = to;
    };
    if (n < rows)
#pragma unroll 4
        for (int k = w; k < parts; k += kJoinWaves) join(part[k * n_pad + n]);
    red[w][lane] = make_float2(top, s);
    __syncthreads();
    if (w != 0 || n >= rows) return;
    for (int k = 1; k < min(parts, kJoinWaves); ++k) join(red[k][lane]);
    const float lg = kLn2 * log2f(s);
    lse[n] = s == 0.0f ? -INFINITY : top + lg;
    // (a row without any class left has lse = -inf and, by this rule, loss = +inf)
    loss[n] = !kept_row(target[n], classes) ? 0.0f : s == 0.0f ? INFINITY : lg + (top - at[n]);
}

// ---------------------------------------------------------------- backward

// dl of one piece of classes in Q planes: dl[q][sample][class of the piece] (rows ld apart), zeros in the samples and classes that there are not.  Rows of a
// tile are samples, columns classes.  bias_part[(mt * WM + wavefront row) * piece + class] = sums of the unrounded dl (if asked for).
// The product bounds it, and the exponentials and stores behind it: 8 192 x 1 024 into 65 535 in bf16 1 132 us in all, 972 TFLOP/s.
template <typename T, int Q>
__global__ void __launch_bounds__(T::NT, 2) xent_dlogits_kernel(Planes x, Planes w, int32_t rows, int32_t classes, int steps, int32_t first, int32_t piece, int64_t ld,
                                                                const float *bias, const int32_t *target, const float *lse, const float *grad_loss,
                                                                uint16_t *dl, int64_t n_pad, float *bias_part)
{
    extern __shared__ __align__(128) char smem[];
    const int tm = static_cast<int>(n_pad / T::BM), tn = piece / T::BN;
    int mt, nt;
    tile_of(xcd_contiguous(blockIdx.x, gridDim.x), tm, tn, 8, mt, nt);
    f32x4 acc[T::MI][T::NI];
    T::clear(acc);
    const int m0 = mt * T::BM, n0 = first + nt * T::BN;
    // (a tile that lies wholly past the last sample or class repeats the last row; it comes out as zeros all the same)
    T::run(x, min(m0, rows - 1), rows, w, min(n0, classes - 1), classes, 0, steps, smem, acc);
    // What a row of the tile needs.  exp(l - lse) = 2^(l log2e - off) 2^(-rest): what lse log2e loses to rounding goes into the row's factor.
    // A row that does not count has off = inf and factor 0, which leaves 0 of any finite logit; what a bias or weight that is not finite leaves
    // is taken away beside the rows that are far.
    enum { kNear, kFarRow, kNoRow };
    struct Row {
        float off, factor;
        int32_t target, kind;
    };
    Row *info = reinterpret_cast<Row *>(smem);
    lds_barrier();
    for (int r = threadIdx.x; r < T::BM; r += T::NT) {
        const int m = m0 + r;
        Row q{INFINITY, 0.0f, -1, kNoRow};
        if (m < rows) {
            const int32_t t = target[m];
            const float z = lse[m];
            if (kept_row(t, classes) && z != -INFINITY) {
                const float g = grad_loss[m];
                q.kind = __builtin_fabsf(z) <= kFar ? kNear : kFarRow;
                q.off = z * kLog2e;
                q.factor = g * __builtin_amdgcn_exp2f(-__builtin_fmaf(z, kLog2e, -q.off));
                q.target = t;
            }
        }
        info[r] = q;
    }
    lds_barrier();
    const int n = n0 + T::col_of();
    float b[T::NI], sum[T::NI];
#pragma unroll
    for (int j = 0; j < T::NI; ++j) b[j] = n + j >= classes ? -INFINITY : bias ? bias[n + j] : 0.0f, sum[j] = 0.0f;
    uint16_t *to = dl + m0 * ld + nt * T::BN + T::col_of();
#pragma unroll
    for (int i = 0; i < T::MI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = T::row_of(i) + e;
            const Row q = info[r];
            float l[T::NI], v[T::NI];
#pragma unroll
            for (int j = 0; j < T::NI; ++j) {
                l[j] = acc[i][j][e] + b[j];
                v[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(l[j], kLog2e, -q.off)) * q.factor;
            }
            if (static_cast<uint32_t>(q.target - n) < T::NI || q.kind != kNear) {
                if (q.kind == kNoRow) {
#pragma unroll
                    for (int j = 0; j < T::NI; ++j) v[j] = 0.0f;
                } else {
                    const float z = lse[m0 + r], g = grad_loss[m0 + r];
#pragma unroll
                    for (int j = 0; j < T::NI; ++j) {
                        if (q.kind == kFarRow) v[j] = __builtin_amdgcn_exp2f((l[j] - z) * kLog2e) * g;
                        // the target's own exp(l - lse) - 1 is small where the network is right: not taken as a difference
                        if (q.target == n + j) v[j] = g * expm1f(l[j] - z);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < T::NI; ++j) sum[j] += v[j];
#pragma unroll
            for (int p = 0; p < Q; ++p) {
                u32x2 out;
                const uint32_t w0 = plane_of<Q>(p, v[0]), w1 = plane_of<Q>(p, v[1]), w2 = plane_of<Q>(p, v[2]), w3 = plane_of<Q>(p, v[3]);
                out[0] = w0 | w1 << 16, out[1] = w2 | w3 << 16;
                *reinterpret_cast<u32x2 *>(to + (p * n_pad + r) * ld) = out;
            }
        }
    if (bias_part) {
        f32x4 s;
#pragma unroll
        for (int j = 0; j < T::NI; ++j) s[j] = with_lane32<AddOp>(with_lane16<AddOp>(sum[j]));
        if ((threadIdx.x & 63) < 16)
            *reinterpret_cast<f32x4 *>(bias_part + static_cast<int64_t>(mt * T::WM + (threadIdx.x >> 6) / T::WN) * piece + nt * T::BN + T::col_of()) = s;
    }
}

// grad_x's tiles (TX: dl along its rows) and grad_w's (TW: dl across them), in one launch since each alone seldom fills the chip.  Loads into
// LDS bound it: 8 192 x 1 024 into 65 535 in bf16 1 821 to 1 890 us in all, 1 163 to 1 207 TFLOP/s; float 1 000 x 300 into 5 003 51 us, 700 TFLOP/s of
// planes.  (256 x 256 in bf16 has 4 registers more than there are, which it spills.)
template <typename TX, typename TW, typename O>
__global__ void __launch_bounds__(TX::NT, 2) xent_products_kernel(Product px, Product pw)
{
    static_assert(TX::LDS == TW::LDS && TX::NT == TW::NT, "one launch");
    extern __shared__ __align__(128) char smem[];
    // each XCD gets an eighth of both, which are of different lengths
    const int first = px.tm * px.tn * px.splits, id = blockIdx.x;
    if (id < first) product_tile<TX, O>(px, xcd_contiguous(id, first), smem);
    else product_tile<TW, O>(pw, xcd_contiguous(id - first, gridDim.x - first), smem);
}

// Up to three sums in one launch: of grad_x's, of grad_w's and of grad_bias's parts (one row of classes).
template <typename O>
__global__ void __launch_bounds__(256) xent_finish_kernel(Sum x, Sum w, Sum bias)
{
    unsigned block = blockIdx.x;
    if (block < x.blocks) return sum_parts<O>(x, block);
    block -= x.blocks;
    if (block < w.blocks) return sum_parts<O>(w, block);
    sum_parts<float>(bias, block - w.blocks);
}

// ---------------------------------------------------------------- few classes

// A head over a handful of classes is all launches: everything of 16 samples is done by one workgroup, forward in one launch, backward in
// one and the sums over the workgroups.  Logits from the matrix cores (float as it is, v_mfma_f32_16x16x4; lane l: class l & 15 or sample
// l & 15, and gets classes 4 (l >> 4) .. + 3 of sample l & 15), each of the four wavefronts over its share of the width, the first of which
// joins them; both gradients from vector multiply-adds, a thread to a column: a row of dl is the same for all threads, and never rounded.
// Waits bound it, a load's or a join's after the other: float 64 x 128 into 10 classes 3.6 us forward and 10.6 + 3.5 backward.
constexpr int kFewRows16 = 16;

template <typename S, int VT, bool BACK>
__global__ void __launch_bounds__(256) xent_few_kernel(const S *x, int64_t ldx, const S *w, int64_t ldw, int32_t rows, int32_t width, int32_t classes, bool vec,
                                                       const float *bias, const int32_t *target, float *loss, float *lse, const float *grad_loss, S *gx, int64_t ldgx,
                                                       float *part, int64_t part_ld, float *bias_part)
{
    __shared__ f32x4 red[4][VT][64];
    __shared__ float dl[BACK ? VT * 16 : 1][kFewRows16];        // transposed: a class to a row
    __shared__ bool counts[kFewRows16];
    constexpr int E = 16 / sizeof(S);                           // elements that a lane loads at a time
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, c4 = lane >> 4;
    const int64_t r0 = static_cast<int64_t>(blockIdx.x) * kFewRows16;
    const int here = static_cast<int>(min(static_cast<int64_t>(kFewRows16), rows - r0));
    struct alignas(16) Piece { S e[E]; };
    auto load = [&](const S *row, int k) {
        if (vec && k + E <= width) return *reinterpret_cast<const Piece *>(row + k);
        Piece p;
#pragma unroll
        for (int e = 0; e < E; ++e) p.e[e] = k + e < width ? row[k + e] : static_cast<S>(0.0f);
        return p;
    };
    {
        const S *row = x + min(r0 + r16, static_cast<int64_t>(rows) - 1) * ldx;
        f32x4 acc[VT];
#pragma unroll
        for (int t = 0; t < VT; ++t) acc[t] = f32x4{0, 0, 0, 0};
        for (int k = wave * 4 * E; k < width; k += 16 * E) {
            const Piece px = load(row, k + c4 * E);
#pragma unroll
            for (int t = 0; t < VT; ++t) {
                const Piece pw = load(w + static_cast<int64_t>(min(t * 16 + r16, classes - 1)) * ldw, k + c4 * E);
                if constexpr (sizeof(S) == 4) {
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(pw.e[e], px.e[e], acc[t], 0, 0, 0);
                } else
                    acc[t] = Mfma<bf16x8>::go(__builtin_bit_cast(bf16x8, pw), __builtin_bit_cast(bf16x8, px), acc[t]);
            }
        }
#pragma unroll
        for (int t = 0; t < VT; ++t) red[wave][t][lane] = acc[t];
    }
    __syncthreads();
    if (wave == 0) {
        const int64_t n = r0 + r16;
        const int32_t goal = n < rows ? target[n] : -1;
        f32x4 acc[VT];
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < VT; ++t) {
            acc[t] = (red[0][t][lane] + red[1][t][lane]) + (red[2][t][lane] + red[3][t][lane]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int v = t * 16 + c4 * 4 + e;
                acc[t][e] = v >= classes ? -INFINITY : bias ? acc[t][e] + bias[v] : acc[t][e];
                top = fmaxf(top, acc[t][e]);
            }
        }
        if constexpr (!BACK) {
            top = with_lane32<MaxOp>(with_lane16<MaxOp>(top));
            // the largest logit's own term is one: kept apart, what the others add to it is not rounded away
            float ones = 0.0f, rest = 0.0f, at = 0.0f;
#pragma unroll
            for (int t = 0; t < VT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float l = acc[t][e];
                    ones += l == top ? 1.0f : 0.0f;
                    rest += l == top || l == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((l - top) * kLog2e);
                    at += goal == t * 16 + c4 * 4 + e ? l : 0.0f;
                }
            ones = with_lane32<AddOp>(with_lane16<AddOp>(ones)), rest = with_lane32<AddOp>(with_lane16<AddOp>(rest)), at = with_lane32<AddOp>(with_lane16<AddOp>(at));
            if (n < rows && c4 == 0) {
                const float lg = log1pf(ones - 1.0f + rest);
                const bool none = top == -INFINITY && rest == 0.0f;     // (a NaN is no largest logit either, but then rest is NaN)
                lse[n] = none ? top : top + lg;
                loss[n] = !kept_row(goal, classes) ? 0.0f : none ? INFINITY : lg + (top - at);
            }
        } else {
            const float z = n < rows ? lse[n] : 0.0f;
            const bool kept = kept_row(goal, classes) && z != -INFINITY;
            const float g = kept ? grad_loss[n] : 0.0f;
#pragma unroll
            for (int t = 0; t < VT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int v = t * 16 + c4 * 4 + e;
                    const float d = acc[t][e] - z, p = v == goal ? expm1f(d) : __builtin_amdgcn_exp2f(d * kLog2e);
                    dl[v][r16] = kept && v < classes ? p * g : 0.0f;
                }
            if (c4 == 0) counts[r16] = kept;
        }
    }
    if constexpr (BACK) {
        __syncthreads();
        for (int d = threadIdx.x; (gx || part) && d < width; d += 256) {
            asm volatile("" ::: "memory");      // (dl is read from shared memory for every column: it does not fit into the registers)
            float wv[VT * 16], gw[VT * 16], xv[16], gr[16] = {};
#pragma unroll
            for (int v = 0; v < VT * 16; ++v) wv[v] = v < classes ? static_cast<float>(w[v * ldw + d]) : 0.0f, gw[v] = 0.0f;
#pragma unroll
            for (int k = 0; k < 16; ++k) xv[k] = k < here && counts[k] ? static_cast<float>(x[(r0 + k) * ldx + d]) : 0.0f;
#pragma unroll
            for (int v = 0; v < VT * 16; ++v)
                if (v < classes)
#pragma unroll
                    for (int k = 0; k < 16; k += 4) {
                        const f32x4 q = *reinterpret_cast<const f32x4 *>(&dl[v][k]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) gr[k + e] = __builtin_fmaf(q[e], wv[v], gr[k + e]), gw[v] = __builtin_fmaf(q[e], xv[k + e], gw[v]);
                    }
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (gx && k < here) gx[(r0 + k) * ldgx + d] = static_cast<S>(gr[k]);
            if (part)
#pragma unroll
                for (int v = 0; v < VT * 16; ++v)
                    if (v < classes) part[(static_cast<int64_t>(blockIdx.x) * classes + v) * part_ld + d] = gw[v];
        }
        if (bias_part && static_cast<int>(threadIdx.x) < classes) {
            float s = 0.0f;
            for (int r = 0; r < here; ++r) s += dl[threadIdx.x][r];
            bias_part[static_cast<int64_t>(blockIdx.x) * ((classes + 3) & ~3) + threadIdx.x] = s;
        }
    }
}

template <typename O>
__global__ void __launch_bounds__(256) xent_zero_kernel(O *out, int64_t ld, int64_t rows, int32_t cols)
{
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; t < rows * cols; t += static_cast<int64_t>(gridDim.x) * 256)
        out[t / cols * ld + t % cols] = static_cast<O>(0.0f);
}

// ---------------------------------------------------------------- host side

struct Layout {
    int32_t rows, width, classes;
    int64_t kp, n_pad;                      // width and rows as they are laid out
    int32_t piece, pieces;
    int64_t ldk, ldl;                       // from row to row of what is laid out, and of dl
    int32_t size;                           // 2, 1, 0: of the logits' tiles
    uint16_t *xp, *wp, *dl;
    float2 *part;
    float *at, *bias_part, *part_x, *part_w;
    int32_t product_size;                   // and of the products'
    int32_t splits_x, splits_w;
    int64_t part_ld;
    bool few;                               // classes: the form of its own
    int64_t bytes;
};

// A thread of the form for few classes holds a column of w and of its gradient, and each 16 samples leave a part of grad_w.  Forward and
// backward, us, so / in general: float 64 x 128 into 10 classes 16 / 35, 1 000 x 256 into 32 30 / 58, 64 x 1 024 into 32 68 / 94,
// 16 384 x 256 into 10 51 / 100; bf16 64 x 128 into 10 16 / 24, 8 192 x 1 024 into 8 61 / 63, 64 x 1 024 into 32 (not taken) 68 / 37.
bool few_classes(const dol_matrix *x, const dol_matrix *w)
{
    return w->rows <= 32 && int64_t(w->rows) * w->cols <= (x->dtype == DOL_F32 ? 32768 : 8192) && x->rows <= 16384;
}

// Tiles of 64 x 64 below so many of 128 x 128 (of logits) or k of a place with them (of the products).  Forward and backward, us, 64 x 64 /
// 128 x 128 in both: float 64 x 128 x 360 35 / 50, 100 x 100 x 1 000 33 / 50; bf16 26 / 32, 28 / 36.  Logits alone: float 300 x 256 x 3 000 (72
// tiles) 66 / 70, bf16 50 x 512 x 20 000 (157) 85 / 70.  Products alone: float 300 x 256 x 3 000 (126) 70 / 66, 2 000 x 128 x 2 000 (250) 71 / 65;
// bf16 300 x 256 x 3 000 36 / 40, 8 192 x 64 x 500 (253) 35 / 42, 700 x 700 x 7 000 105 / 93.
constexpr int kTiny = 128;
template <int P>
constexpr int kTinyProducts = P == 3 ? 64 : 256;

// What a tile takes beside its products, in k, and what an element of a sum and a piece's launches take, in a tile's area times k (some 2.2 G of
// which a unit does in a millisecond with one product of planes, at the rates above: a piece's launches some 7.6 us).
constexpr double kAround = 160, kSumWeight = 6, kLaunchWeight = 256 * 256 * 256;

template <int P, int Q>
Layout lay_out(const dol_matrix *x, const dol_matrix *w, bool backward, void *workspace)
{
    using S = Shapes<P, Q>;
    Layout L{};
    L.rows = x->rows, L.width = x->cols, L.classes = w->rows;
    L.part_ld = round_up(L.width, 4);
    L.few = few_classes(x, w);
    if (L.few) {
        Carver c(workspace);
        L.splits_w = tiles(L.rows, kFewRows16);
        // (the same for both passes, though only the backward one writes it)
        L.part_w = c.take<float>(int64_t(L.splits_w) * L.classes * L.part_ld);
        L.bias_part = c.take<float>(int64_t(L.splits_w) * round_up(L.classes, 4));
        L.bytes = c.used;
        return L;
    }
    L.kp = round_up(L.width, 64), L.n_pad = round_up(L.rows, kPad), L.ldk = spread(L.kp);
    // Tiles of 256 x 256 (float 128 x 256) do more with what they load; smaller ones (128 x 128, 64 x 64) fill the chip sooner.  Forward and backward, us,
    // large / small: bf16 with 64 of the large ones 76 / 57, 128 67 / 58, 1 280 895 / 950; float with 128 167 / 141, 160 142 / 155.
    L.size = int64_t(tiles(L.classes, S::Big::BM)) * tiles(L.rows, S::Big::BN) >= (P == 3 ? 160 : 192) ? 2
             : int64_t(tiles(L.classes, S::Small::BM)) * tiles(L.rows, S::Small::BN) >= kTiny              ? 1
                                                                                                            : 0;
    Carver c(workspace);
    if (backward || !direct(x)) L.xp = c.take<uint16_t>(P * (backward ? L.n_pad : L.rows) * L.ldk);
    if (!direct(w)) L.wp = c.take<uint16_t>(P * int64_t(L.classes) * L.ldk);
    if (!backward) {
        const int parts = by_size(L.size, Type<typename S::Big>(), Type<typename S::Small>(), Type<typename S::Tiny>(),
                                  [&](auto z) { return tiles(L.classes, decltype(z)::Tile::BM) * decltype(z)::Tile::WM; });
        L.part = c.take<float2>(int64_t(parts) * L.n_pad);
        L.at = c.take<float>(L.rows);
        L.bytes = c.used;
        return L;
    }
    // Large tiles where a place's k with them is long, or (float) can be split evenly.  us, large / small: bf16 4 096 x 512 x 1 024 (a place's
    // k 256) 65 / 57; float 1 000 x 300 x 5 003 (469) 141 / 155, 4 096 x 512 x 1 024 (512) 131 / 141, 500 x 300 x 20 000 (931, longer than
    // grad_w's) 311 / 293, 300 x 200 x 3 000 (75) 84 / 75.
    const int64_t most = std::max<int64_t>(kPad, kMostPieceBytes / (2 * Q * L.n_pad) / kPad * kPad), one = std::min<int64_t>(L.classes, most);
    const int64_t place = (tiles(L.rows, S::BigX::BN) * one + tiles(one, S::BigX::BN) * int64_t(L.rows)) * tiles(L.width, S::BigX::BM) / kUnits;
    const bool big = place >= 1024 || (P == 3 && place >= 384 && std::min<int64_t>(one, L.rows) >= 2 * place);
    const int64_t small = (tiles(L.rows, S::SmallX::BN) * one + tiles(one, S::SmallX::BN) * int64_t(L.rows)) * tiles(L.width, S::SmallX::BM);
    L.product_size = big ? 2 : small >= kTinyProducts<P> * kUnits ? 1 : 0;
    // Pieces and shares so that the launches' workgroups come out even on the places there are.  Beside pieces of 128 MB and shares of one
    // place's k, us, now / then: float 4 096 x 512 x 30 000 2 702 / 3 420, 2 000 x 256 x 60 000 1 562 / 1 957, 8 192 x 1 024 x 10 000 3 525 / 3 859;
    // bf16 8 192 x 256 x 20 000 515 / 637, 1 000 x 512 x 20 000 148 / 167, 4 000 x 1 000 x 30 000 1 030 / 1 022.  Pieces of up to 256 MB: bf16
    // 8 192 x 1 024 x 65 535 4 025 / 3 890, 8 192 x 256 x 20 000 508 / 515; of up to 128 MB: float 4 096 x 512 x 30 000 3 367.
    int bm = 0, bn = 0, lds = 0, pm = 0, pn = 0, plds = 0;
    by_size(L.size, Type<typename S::Big>(), Type<typename S::Small>(), Type<typename S::Tiny>(), [&](auto z) {
        using T = typename decltype(z)::Tile;
        bm = T::BM, bn = T::BN, lds = T::LDS;
    });
    by_size(L.product_size, Type<typename S::BigX>(), Type<typename S::SmallX>(), Type<typename S::TinyX>(), [&](auto z) {
        using T = typename decltype(z)::Tile;
        pm = T::BM, pn = T::BN, plds = T::LDS;
    });
    const int64_t places = kUnits * std::max(1, kLds / lds), product_places = kUnits * std::max(1, kLds / plds);
    const int64_t fewest = (L.classes + most - 1) / most, spare = fewest == 1 ? 1 : std::min<int64_t>(fewest + 12, 4 * fewest);
    constexpr double kProducts = P == 3 ? 6 : Q;        // of planes
    double best = 0.0;
    for (int64_t pieces = fewest; pieces <= spare; ++pieces) {
        const int64_t piece = round_up((L.classes + pieces - 1) / pieces, kPad), n = std::min<int64_t>(piece, L.classes);
        if (pieces > fewest && tiles(L.classes, piece) != pieces) continue;
        // areas of tiles times their k, the same for both launches
        const double logits = done(L.n_pad / bm * (piece / bn), L.kp + kAround, 0, 0.0, places) * bm * bn * (places / kUnits);
        const int64_t tx = tiles(L.width, pm) * int64_t(tiles(L.rows, pn)), tw = tiles(L.width, pm) * int64_t(tiles(n, pn));
        const int64_t even = (tx * n + tw * L.rows) / product_places;
        for (int q = 6; q <= 20; ++q) {
            const int64_t share = std::max<int64_t>(256, even * q / 10), sx = std::max<int64_t>(1, (n + share / 2) / share), sw = std::max<int64_t>(1, (L.rows + share / 2) / share);
            const double sums = (sx > 1 ? double(sx) * L.rows : 0.0) + (sw > 1 ? double(sw) * n : 0.0);
            const double products = done(tx * sx, double(n) / sx + kAround, tw * sw, double(L.rows) / sw + kAround, product_places) * pm * pn * (product_places / kUnits) +
                                    sums * L.width * kSumWeight / kProducts;
            const double all = pieces * (logits + products + kLaunchWeight / kProducts);
            if (best == 0.0 || all < best)
                best = all, L.piece = static_cast<int32_t>(piece), L.pieces = static_cast<int32_t>(tiles(L.classes, piece)), L.splits_x = static_cast<int32_t>(sx), L.splits_w = static_cast<int32_t>(sw);
        }
    }
    const int32_t n = std::min(L.piece, L.classes);
    L.ldl = spread(L.piece);
    L.dl = c.take<uint16_t>(Q * L.n_pad * L.ldl);
    L.bias_part = c.take<float>(L.n_pad / 16 * L.piece);
    if (L.splits_x > 1 || L.pieces > 1) L.part_x = c.take<float>(int64_t(L.splits_x) * L.rows * L.part_ld);
    if (L.splits_w > 1) L.part_w = c.take<float>(int64_t(L.splits_w) * n * L.part_ld);
    L.bytes = c.used;
    return L;
}

// dl in bf16 is off by 2^-9 or so in every term of a gradient.  Sums over many rows average that out; with few rows, where the products
// cost little, a second plane takes it away.  Forward and backward, us, two planes / one: 64 x 128 x 360 31 / 27, 500 x 512 x 1 000 46 / 41,
// 512 x 256 x 20 000 107 / 87, 4 096 x 512 x 1 024 69 / 57; gradients of 64 x 128 x 360 off by 1e-5 / 2.8e-3 before they are rounded.
constexpr int32_t kFewRows = 512;

template <typename F>
auto with_planes(const dol_matrix *x, F f)
{
    if (x->dtype == DOL_F32) return f(std::integral_constant<int, 3>(), std::integral_constant<int, 3>());
    if (x->rows <= kFewRows) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
    return f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
}

template <int P>
dol_status launch_pack(const Pack &a, const Pack &b, hipStream_t st)
{
    if (a.blocks + b.blocks == 0) return DOL_OK;
    xent_pack_kernel<typename Source<P>::T, P><<<a.blocks + b.blocks, 256, 0, st>>>(a, b);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <typename O>
dol_status launch_finish(const Sum &x, const Sum &w, const Sum &bias, hipStream_t st)
{
    const unsigned n = x.blocks + w.blocks + bias.blocks;
    if (n == 0) return DOL_OK;
    xent_finish_kernel<O><<<n, 256, 0, st>>>(x, w, bias);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <typename S, bool BACK>
dol_status launch_few(const Layout &L, const dol_matrix *x, const dol_matrix *w, const float *bias, const int32_t *target, float *loss, float *lse, const float *grad_loss,
                      const dol_matrix *gx, const dol_matrix *gw, float *grad_bias, hipStream_t st)
{
    constexpr int64_t E = 16 / sizeof(S);
    const bool vec = x->ld % E == 0 && w->ld % E == 0 && !((reinterpret_cast<uintptr_t>(x->data) | reinterpret_cast<uintptr_t>(w->data)) & 15);
    auto go = [&](auto vt) {
        xent_few_kernel<S, vt.value, BACK><<<L.splits_w, 256, 0, st>>>(static_cast<const S *>(x->data), x->ld, static_cast<const S *>(w->data), w->ld, L.rows, L.width, L.classes, vec,
                                                                      bias, target, loss, lse, grad_loss, gx ? static_cast<S *>(gx->data) : nullptr, gx ? gx->ld : 0,
                                                                      gw ? L.part_w : nullptr, L.part_ld, grad_bias ? L.bias_part : nullptr);
    };
    if (L.classes <= 16) go(std::integral_constant<int, 1>());
    else go(std::integral_constant<int, 2>());
    DOL_HIP(hipGetLastError());
    if (!BACK) return DOL_OK;
    Sum sw{}, sb{};
    if (gw) sw = make_sum(L.part_w, L.classes, L.width, L.splits_w, L.part_ld, gw->data, gw->ld);
    if (grad_bias) sb = make_sum(L.bias_part, 1, L.classes, L.splits_w, round_up(L.classes, 4), grad_bias, L.classes);
    return launch_finish<S>(Sum{}, sw, sb, st);
}

template <typename T>
dol_status launch_sums(const Layout &L, Planes w, Planes x, const float *bias, const int32_t *target, float *loss, float *lse, hipStream_t st)
{
    DOL_HIP(allow_dynamic_lds(reinterpret_cast<const void *>(xent_sums_kernel<T>), T::LDS));
    const int tm = tiles(L.classes, T::BM), tn = tiles(L.rows, T::BN);
    const int most = std::max(1, INT32_MAX / T::NT / tm);       // tiles of samples that a launch has the threads for
    for (int t = 0; t < tn; t += most) {
        const int64_t n = int64_t(t) * T::BN;
        xent_sums_kernel<T><<<tm * std::min(most, tn - t), T::NT, T::LDS, st>>>(w, Planes{x.data + n * x.ld, x.ld, x.plane}, L.classes,
                                                                               static_cast<int32_t>(std::min<int64_t>(L.rows - n, int64_t(most) * T::BN)),
                                                                               static_cast<int>(L.kp / T::BK), bias, target + n, L.part + n, L.n_pad, L.at + n);
        DOL_HIP(hipGetLastError());
    }
    xent_join_kernel<<<tiles(L.rows, 64), kJoinWaves * 64, 0, st>>>(L.part, tm * T::WM, L.n_pad, L.rows, L.classes, target, L.at, loss, lse);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <int P, int Q>
dol_status forward(const Layout &L, const dol_matrix *x, const dol_matrix *w, const float *bias, const int32_t *target, float *loss, float *lse, hipStream_t st)
{
    if (L.few) return launch_few<typename Source<P>::T, false>(L, x, w, bias, target, loss, lse, nullptr, nullptr, nullptr, nullptr, st);
    Planes xp, wp;
    const Pack a = pack_of<P>(x, nullptr, nullptr, 0, L.xp, L.rows, L.kp, L.ldk, &xp), b = pack_of<P>(w, nullptr, nullptr, 0, L.wp, L.classes, L.kp, L.ldk, &wp);
    if (dol_status s = launch_pack<P>(a, b, st)) return s;
    using Z = Shapes<P, Q>;
    return by_size(L.size, Type<typename Z::Big>(), Type<typename Z::Small>(), Type<typename Z::Tiny>(),
                   [&](auto z) { return launch_sums<typename decltype(z)::Tile>(L, wp, xp, bias, target, loss, lse, st); });
}

template <typename T, int Q>
dol_status launch_dlogits(const Layout &L, Planes x, Planes w, int32_t first, const float *bias, const int32_t *target, const float *lse,
                          const float *grad_loss, float *grad_bias, Sum *bias_parts, hipStream_t st)
{
    DOL_HIP(allow_dynamic_lds(reinterpret_cast<const void *>(xent_dlogits_kernel<T, Q>), T::LDS));
    const int tm = static_cast<int>(L.n_pad / T::BM), tn = L.piece / T::BN;
    xent_dlogits_kernel<T, Q><<<tm * tn, T::NT, T::LDS, st>>>(x, w, L.rows, L.classes, static_cast<int>(L.kp / T::BK), first, L.piece, L.ldl, bias, target, lse, grad_loss, L.dl,
                                                              L.n_pad, grad_bias ? L.bias_part : nullptr);
    DOL_HIP(hipGetLastError());
    *bias_parts = grad_bias ? make_sum(L.bias_part, 1, std::min(L.piece, L.classes - first), tm * T::WM, L.piece, grad_bias + first, L.classes) : Sum{};
    return DOL_OK;
}

template <typename TX, typename TW, typename O>
dol_status launch_products(Product x, Product w, hipStream_t st)
{
    DOL_HIP(allow_dynamic_lds(reinterpret_cast<const void *>(xent_products_kernel<TX, TW, O>), TX::LDS));
    for (Product *p : {&x, &w})
        if (p->M > 0) p->tm = tiles(p->M, TX::BM), p->tn = tiles(p->N, TX::BN), p->steps = tiles(p->k, TX::BK);
    const int n = x.tm * x.tn * x.splits + w.tm * w.tn * w.splits;
    if (n == 0) return DOL_OK;
    xent_products_kernel<TX, TW, O><<<n, TX::NT, TX::LDS, st>>>(x, w);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <int P, int Q>
dol_status reverse(const Layout &L, const dol_matrix *x, const dol_matrix *w, const float *bias, const int32_t *target, const float *lse,
                   const float *grad_loss, const dol_matrix *grad_x, const dol_matrix *grad_w, float *grad_bias, hipStream_t st)
{
    using S = typename Source<P>::T;
    using Z = Shapes<P, Q>;
    if (L.few) return launch_few<S, true>(L, x, w, bias, target, nullptr, const_cast<float *>(lse), grad_loss, grad_x, grad_w, grad_bias, st);
    Planes xp, wp;
    // x is always laid out, with zeros in the rows that do not count: as k of grad_w they would meet dl's zeros with whatever they hold
    const Pack lx = pack_of<P>(x, target, lse, L.classes, L.xp, L.n_pad, L.kp, L.ldk, &xp), lw = pack_of<P>(w, nullptr, nullptr, 0, L.wp, L.classes, L.kp, L.ldk, &wp);
    if (dol_status s = launch_pack<P>(lx, lw, st)) return s;
    for (int32_t k = 0; k < L.pieces; ++k) {
        const int32_t first = k * L.piece, n = std::min(L.piece, L.classes - first);
        Sum sb{};
        if (dol_status s = by_size(L.size, Type<typename Z::Big>(), Type<typename Z::Small>(), Type<typename Z::Tiny>(), [&](auto z) {
                return launch_dlogits<typename decltype(z)::Tile, Q>(L, xp, wp, first, bias, target, lse, grad_loss, grad_bias, &sb, st);
            }))
            return s;
        const Planes dl{L.dl, L.ldl, L.n_pad * L.ldl};
        Product a{}, b{};
        if (grad_x) {
            a.a = Planes{wp.data + first * wp.ld, wp.ld, wp.plane}, a.b = dl;
            a.M = L.width, a.N = L.rows, a.wide = static_cast<int32_t>(L.kp), a.tall = static_cast<int32_t>(L.n_pad), a.splits = L.splits_x, a.k = a.have = n;
            a.part = L.part_x, a.part_ld = L.part_ld, a.add = k > 0, a.out = grad_x->data, a.out_ld = grad_x->ld;
        }
        if (grad_w) {
            b.a = xp, b.b = dl;
            b.M = L.width, b.N = n, b.wide = static_cast<int32_t>(L.kp), b.tall = L.piece, b.splits = L.splits_w, b.k = L.rows, b.have = L.n_pad;
            b.part = L.part_w, b.part_ld = L.part_ld, b.out = static_cast<S *>(grad_w->data) + first * grad_w->ld, b.out_ld = grad_w->ld;
        }
        if (dol_status s = L.product_size == 2   ? launch_products<typename Z::BigX, typename Z::BigW, S>(a, b, st)
                           : L.product_size == 1 ? launch_products<typename Z::SmallX, typename Z::SmallW, S>(a, b, st)
                                                 : launch_products<typename Z::TinyX, typename Z::TinyW, S>(a, b, st))
            return s;
        if (dol_status s = launch_finish<S>(k == L.pieces - 1 ? sum_of(a) : Sum{}, sum_of(b), sb, st)) return s;
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
    *bytes = 0;
    if (x->rows > 0) *bytes = with_planes(x, [&](auto p, auto q) { return lay_out<p.value, q.value>(x, weight, backward, nullptr); }).bytes;
    return DOL_OK;
}

const char *dol_cross_entropy_kernel(const dol_matrix *x, const dol_matrix *weight, int32_t backward)
{
    static thread_local char name[96];
    if (check_operands(x, weight) != DOL_OK || x->rows == 0) return "";
    if (few_classes(x, weight)) return "xent_few_kernel";
    with_planes(x, [&](auto p, auto q) {
        using Z = Shapes<p.value, q.value>;
        const Layout L = lay_out<p.value, q.value>(x, weight, backward, nullptr);
        auto at = [&](const char *kernel, int have, auto z) {
            using T = typename decltype(z)::Tile;
            return snprintf(name + have, sizeof name - have, "%s%s %dx%dx%d", have ? ", " : "", kernel, T::BM, T::BN, T::BK);
        };
        const int n = by_size(L.size, Type<typename Z::Big>(), Type<typename Z::Small>(), Type<typename Z::Tiny>(),
                              [&](auto z) { return at(backward ? "xent_dlogits_kernel" : "xent_sums_kernel", 0, z); });
        if (backward) by_size(L.product_size, Type<typename Z::BigX>(), Type<typename Z::SmallX>(), Type<typename Z::TinyX>(), [&](auto z) { return at("xent_products_kernel", n, z); });
    });
    return name;
}

dol_status dol_cross_entropy(const dol_matrix *x, const dol_matrix *weight, const float *bias, const int32_t *target, float *loss, float *lse,
                             void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    if (dol_status s = check_operands(x, weight)) return s;
    if (x->rows == 0) return DOL_OK;
    if (!target || !loss || !lse) return fail(DOL_EINVAL, "target, loss or lse is NULL");
    return with_planes(x, [&](auto p, auto q) {
        const Layout L = lay_out<p.value, q.value>(x, weight, false, workspace);
        if (dol_status s = check_workspace(workspace, workspace_bytes, L.bytes)) return s;
        return forward<p.value, q.value>(L, x, weight, bias, target, loss, lse, static_cast<hipStream_t>(hip_stream));
    });
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
    if (x->rows == 0) {                     // sums over no rows
        if (dol_status s = x->dtype == DOL_BF16 ? zero<__bf16>(grad_weight, st) : zero<float>(grad_weight, st)) return s;
        const dol_matrix b{DOL_F32, 1, weight->rows, weight->rows, grad_bias};
        return grad_bias ? zero<float>(&b, st) : DOL_OK;
    }
    if (!target || !lse || !grad_loss) return fail(DOL_EINVAL, "target, lse or grad_loss is NULL");
    return with_planes(x, [&](auto p, auto q) {
        const Layout L = lay_out<p.value, q.value>(x, weight, true, workspace);
        if (dol_status s = check_workspace(workspace, workspace_bytes, L.bytes)) return s;
        return reverse<p.value, q.value>(L, x, weight, bias, target, lse, grad_loss, grad_x, grad_weight, grad_bias, st);
    });
}

}  // extern "C"
