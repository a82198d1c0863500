// A linear layer with what follows it, and its gradients.
//
//   z = x w^T + bias,   y = act(z) + residual
//   dz = grad_y act'(z),   grad_x = dz w,   grad_w = dz^T x,   grad_bias[o] = sum_i dz[i, o]
//
// A tile of z stays in the registers that the matrix cores leave it in, and y (and z, where the gradients need it) is written from there.  Few
// tiles share out their k, and a second launch adds up the shares and does the rest.  Few rows are no work for tiles: weights go straight from memory into
// the operands of the matrix cores, and their bytes bound the call.  Forward (linear_few_kernel) that is up to 16 rows in bf16 and 64 in float, and up to 256 of
// a layer with few weights, which sets of 16 to 64 rows then read again; grad_x (linear_few_back_kernel) up to 64 rows of a layer with many weights.
// Backward: dz is rounded for the matrix cores and written, with its sums over rows beside it, and grad_x and grad_w are two sets of tiles
// of one launch (mfma_products.h).
#include "activation.h"
#include "loose.h"
#include "mfma_products.h"

#include <cstdio>

namespace dol {
namespace {

// What a call leaves of z.
struct Result {
    const float *bias;
    const void *residual;
    int64_t residual_ld;
    void *y, *z;
    int64_t y_ld, z_ld;
    int16_t *rest;              // [rows][cols]
    int32_t rows, cols, act;
};

// What rounding z to bf16 leaves, in a float's steps (whose bits count them across powers of two as well): -32768 .. 32768, the last of which, where z lies
// half way and the lower neighbour is even, is taken for 32767.  With it z is a float again, and sums of act'(z) in 32 bits are not off by 2^-9 a term.
__device__ __forceinline__ uint32_t rest_of(float z)
{
    const int r = static_cast<int>(__float_as_uint(z) - (bits16<__bf16>(z) << 16));
    return __builtin_isfinite(z) ? static_cast<uint32_t>(min(r, 32767)) & 0xFFFF : 0;
}

__device__ __forceinline__ void store_rest(int16_t *to, f32x4 z)
{
    struct __attribute__((packed, aligned(2))) Words { uint32_t w[2]; };
    *reinterpret_cast<Words *>(to) = Words{{rest_of(z[0]) | rest_of(z[1]) << 16, rest_of(z[2]) | rest_of(z[3]) << 16}};
}

__device__ __forceinline__ float with_rest(float z, uint32_t rest) { return __uint_as_float(__float_as_uint(z) + static_cast<uint32_t>(static_cast<int16_t>(rest))); }

// The bias of columns c .. c + 3, asked for early: behind the products it would be one more wait.
__device__ __forceinline__ f32x4 bias_of(const Result &o, int c)
{
    f32x4 b = {0, 0, 0, 0};
    if (o.bias)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + k < o.cols) b[k] = o.bias[c + k];
    return b;
}

// Columns c .. c + 3 of row r of z without its bias to what the call leaves; those of them that are there.
template <typename S, typename A>
__device__ __forceinline__ void leave(const Result &o, A, int64_t r, int c, f32x4 bias, f32x4 z)
{
    const int n = o.cols - c;
    S *y = static_cast<S *>(o.y) + r * o.y_ld + c;
    z += bias;
    if (o.z) {
        store4(static_cast<S *>(o.z) + r * o.z_ld + c, z, n);
        if (sizeof(S) == 2 && o.rest) {
            int16_t *to = o.rest + r * o.cols + c;
            if (n >= 4) store_rest(to, z);
            else
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (k < n) to[k] = static_cast<int16_t>(rest_of(z[k]));
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) z[k] = act_of<A::value, false>(z[k], nullptr);
    if (o.residual) {
        const S *from = static_cast<const S *>(o.residual) + r * o.residual_ld + c;
        if (n >= 4) {
            const Four<S> q = *reinterpret_cast<const Four<S> *>(from);
#pragma unroll
            for (int k = 0; k < 4; ++k) z[k] += static_cast<float>(q.e[k]);
        } else
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < n) z[k] += static_cast<float>(from[k]);
    }
    store4(y, z, n);
}

// ---------------------------------------------------------------- tiles

struct Tiles {
    int32_t tm, tn, splits, steps;
    float *part;                // [splits][rows][part_ld], or null: one share
    int64_t part_ld;
};

// A whole tile to what the call leaves, from its row m0 and this lane's column c on.  The residual of the next rows is asked for before these rows' results
// are written: it may lie in their place, and no load passes a store.
template <int ACT, typename S, typename T>
__device__ __forceinline__ void leave_whole(const Result &o, int64_t m0, int c, const f32x4 (&acc)[T::MI][T::NI])
{
    const f32x4 b = bias_of(o, c);
    const int64_t first = m0 + T::row_of(0);
    const S *from = static_cast<const S *>(o.residual) + first * o.residual_ld + c;
    Four<S> next[4];
    auto ask = [&](int i) {
        if (o.residual)
#pragma unroll
            for (int e = 0; e < 4; ++e) next[e] = *reinterpret_cast<const Four<S> *>(from + (i * 16 + e) * o.residual_ld);
    };
    ask(0);
#pragma unroll
    for (int i = 0; i < T::MI; ++i) {
        Four<S> r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = next[e];
        if (i + 1 < T::MI) ask(i + 1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t row = first + i * 16 + e;
            f32x4 z = f32x4{acc[i][0][e], acc[i][1][e], acc[i][2][e], acc[i][3][e]} + b;
            if (o.z) store4(static_cast<S *>(o.z) + row * o.z_ld + c, z, 4);
            if (sizeof(S) == 2 && o.rest)
                store_rest(o.rest + row * o.cols + c, z);
#pragma unroll
            for (int k = 0; k < 4; ++k) z[k] = act_of<ACT, false>(z[k], nullptr);
            if (o.residual)
#pragma unroll
                for (int k = 0; k < 4; ++k) z[k] += static_cast<float>(r[e].e[k]);
            store4(static_cast<S *>(o.y) + row * o.y_ld + c, z, 4);
        }
    }
}

template <typename T, typename S, int ACT>
__global__ void __launch_bounds__(T::NT, 2) linear_tiles_kernel(Planes x, Planes w, Tiles g, Result o)
{
    extern __shared__ __align__(128) char smem[];
    const int id = xcd_contiguous(blockIdx.x, gridDim.x), each = g.tm * g.tn, split = id / each;
    int mt, nt;
    tile_of(id - split * each, g.tm, g.tn, 8, mt, nt);
    const int s0 = static_cast<int>(static_cast<int64_t>(g.steps) * split / g.splits), s1 = static_cast<int>(static_cast<int64_t>(g.steps) * (split + 1) / g.splits);
    f32x4 acc[T::MI][T::NI];
    T::clear(acc);
    const int m0 = mt * T::BM, n0 = nt * T::BN;
    T::run(x, m0, o.rows, w, n0, o.cols, static_cast<int64_t>(s0) * T::BK, s1 - s0, smem, acc);
    const int c = n0 + T::col_of();
    if (!g.part && m0 + T::BM <= o.rows && n0 + T::BN <= o.cols) return leave_whole<ACT, S, T>(o, m0, c, acc);
    if (c >= o.cols) return;
    const f32x4 b = bias_of(o, c);
#pragma unroll
    for (int i = 0; i < T::MI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t r = m0 + T::row_of(i) + e;
            const f32x4 z{acc[i][0][e], acc[i][1][e], acc[i][2][e], acc[i][3][e]};
            if (r >= o.rows) continue;
            if (g.part) *reinterpret_cast<f32x4 *>(g.part + (split * static_cast<int64_t>(o.rows) + r) * g.part_ld + c) = z;
            else leave<S>(o, Act<ACT>(), r, c, b, z);
        }
}

// The shares of k added up, in their order, and what follows.
template <typename S>
__global__ void __launch_bounds__(256) linear_join_kernel(const float *part, int64_t part_ld, int splits, Result o)
{
    const int64_t per = (o.cols + 3) / 4, all = o.rows * per;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; t < all; t += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t r = t / per;
        const int c = static_cast<int>(t - r * per) * 4;
        const f32x4 b = bias_of(o, c);
        f32x4 z = {0, 0, 0, 0};
#pragma unroll 8
        for (int k = 0; k < splits; ++k) z += *reinterpret_cast<const f32x4 *>(part + (static_cast<int64_t>(k) * o.rows + r) * part_ld + c);
        with_act(o.act, [&](auto a) { leave<S>(o, a, r, c, b, z); });
    }
}

// ---------------------------------------------------------------- few rows

// 16 M outs and 16 R rows to a workgroup, whose wavefronts share out its k.  A lane loads 32 neighbouring bytes of rows of w (l & 15) and of x, four
// lanes a line of 128; which of a product's k these are does not matter, as long as both operands agree.  float as it is, by v_mfma_f32_16x16x4.
constexpr int few_waves(int n) { return n < 8 ? 16 : 8; }       // at most, for n sums of 16 x 16, which all lie in LDS at the end

template <typename S, int R, int M>
__global__ void __launch_bounds__(few_waves(R * M) * 64) linear_few_kernel(const S *x, int64_t ldx, const S *w, int64_t ldw, int32_t width, int32_t each, int32_t groups, int32_t sets,
                                                                    float *part, int64_t part_ld, Result o)
{
    constexpr int V = kLooseElements<S>, STEP = 8 * V;       // k of a step: two vectors to each of four lanes
    constexpr int N = R * M, W = few_waves(N);
    __shared__ f32x4 red[W][N][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int group = blockIdx.x % groups, set = blockIdx.x / groups % sets, split = blockIdx.x / groups / sets, row0 = set * (16 * R), out0 = group * (16 * M);
    const int64_t k0 = static_cast<int64_t>(split * waves + wave) * each, k1 = min(k0 + each, static_cast<int64_t>(width));
    const S *from_w[M], *from_x[R];
    f32x4 acc[M][R], bias[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
        from_w[m] = w + min(out0 + m * 16 + (lane & 15), o.cols - 1) * ldw;
        bias[m] = bias_of(o, out0 + m * 16 + (lane >> 4) * 4);
#pragma unroll
        for (int r = 0; r < R; ++r) acc[m][r] = f32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int r = 0; r < R; ++r) from_x[r] = x + min(row0 + r * 16 + (lane & 15), o.rows - 1) * ldx;
    auto products = [&](const Loose<S> (&a)[M][2], const Loose<S> (&b)[R][2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (sizeof(S) == 2) {
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int r = 0; r < R; ++r) acc[m][r] = Mfma<bf16x8>::go(__builtin_bit_cast(bf16x8, a[m][h]), __builtin_bit_cast(bf16x8, b[r][h]), acc[m][r]);
            } else
#pragma unroll
                for (int e = 0; e < V; ++e)
#pragma unroll
                    for (int m = 0; m < M; ++m)
#pragma unroll
                        for (int r = 0; r < R; ++r) acc[m][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(loose_get(a[m][h], e), loose_get(b[r][h], e), acc[m][r], 0, 0, 0);
        }
    };
    int64_t k = k0 + (lane >> 4) * (2 * V);
    constexpr int U = N == 1 ? 4 : 2;
    const int64_t whole = k0 + (k1 > k0 ? (k1 - k0) / (U * STEP) * (U * STEP) : 0);
    for (int64_t at = k0; at < whole; at += U * STEP, k += U * STEP) {
        Loose<S> a[U][M][2], b[U][R][2];
#pragma unroll
        for (int q = 0; q < U; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int m = 0; m < M; ++m) a[q][m][h] = *reinterpret_cast<const Loose<S> *>(from_w[m] + k + q * STEP + h * V);
#pragma unroll
                for (int r = 0; r < R; ++r) b[q][r][h] = *reinterpret_cast<const Loose<S> *>(from_x[r] + k + q * STEP + h * V);
            }
#pragma unroll
        for (int q = 0; q < U; ++q) products(a[q], b[q]);
    }
    for (int64_t at = max(whole, k0); at < k1; at += STEP, k += STEP) {
        Loose<S> a[M][2], b[R][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int left = static_cast<int>(k1 - k) - h * V, before = static_cast<int>(k) + h * V;
#pragma unroll
            for (int m = 0; m < M; ++m) a[m][h] = loose_load_end(from_w[m] + k + h * V, left, before);
#pragma unroll
            for (int r = 0; r < R; ++r) b[r][h] = loose_load_end(from_x[r] + k + h * V, left, before);
        }
        products(a, b);
    }
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int r = 0; r < R; ++r) red[wave][m * R + r][lane] = acc[m][r];
    lds_barrier();
#pragma unroll
    for (int q = 0; q < N; ++q) {
        if (q % waves != wave) continue;
        f32x4 z = red[0][q][lane];
#pragma unroll
        for (int t = 1; t < W; ++t)
            if (t < waves) z += red[t][q][lane];
        const int64_t r = row0 + q % R * 16 + (lane & 15);
        const int c = out0 + q / R * 16 + (lane >> 4) * 4;
        if (r >= o.rows || c >= o.cols) continue;
        if (part) *reinterpret_cast<f32x4 *>(part + (split * static_cast<int64_t>(o.rows) + r) * part_ld + c) = z;
        else with_act(o.act, [&](auto a) { leave<S>(o, a, r, c, bias[q / R], z); });
    }
}

// ---------------------------------------------------------------- backward

// x and w laid out, where the tiles cannot read them as they are.
template <typename S, int P>
__global__ void __launch_bounds__(256) linear_pack_kernel(Pack p0, Pack p1)
{
    if (blockIdx.x < p0.blocks) pack_rows<S, P, true>(p0, blockIdx.x);
    else pack_rows<S, P, true>(p1, blockIdx.x - p0.blocks);
}

// dz in Q planes, zeros behind its columns and in rows past the last, and its sums over rows.
struct Slope {
    const void *grad_y, *z;
    int64_t grad_ld, z_ld;
    const int16_t *rest;
    int32_t rows, cols, act;
    uint16_t *dz;               // null: only the sums
    float *flat;                // dz as it is, at the same distances, where not null
    int64_t out_rows, out_cols, ld, plane;      // as they are laid out
    float *part;                // [chunks][part_cols], null: only dz
    int32_t part_cols;
    int32_t chunk;              // rows of a workgroup
    int32_t wide;               // workgroups side by side
    bool narrow;                // of 64 columns, or of 256
    unsigned blocks;            // none where dz is grad_y as it is
};

// LANES threads of eight columns by 256 / LANES rows at a time.
template <typename S, int Q, int LANES>
__device__ __forceinline__ void slope_rows(const Slope &p, unsigned block, float *red)
{
    constexpr int V = kLooseElements<S>, H = 8 / V, ROWS = 256 / LANES, WIDE = LANES * 8;
    // what a row's eight columns are read for; kAhead rows are asked for before the first of them is worked on
    struct Row {
        Loose<S> g[H], z[H];
        Loose<__bf16> rest;
    };
    constexpr int kAhead = sizeof(S) == 2 ? 4 : 2;
    const int lane = threadIdx.x % LANES, row = threadIdx.x / LANES;
    const int64_t chunk = block / p.wide, column = static_cast<int64_t>(block % p.wide) * WIDE, c = column + lane * 8, n = p.cols - c;
    const int64_t r0 = chunk * p.chunk + row, r1 = min((chunk + 1) * p.chunk, p.out_rows);
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
    with_act(p.act, [&](auto a) {
        constexpr bool ACT = decltype(a)::value != DOL_ACT_NONE;
        const bool rests = ACT && sizeof(S) == 2 && p.rest;
        for (int64_t first = r0; first < r1 && c < p.out_cols; first += ROWS * kAhead) {
            Row q[kAhead];
            // (one branch for all loads: each is waited for at a branch's end; where a vector is not all there the row's last one, shifted)
            if (p.cols >= 8) {
#pragma unroll
                for (int t = 0; t < kAhead; ++t) {
                    const int64_t r = min(first + ROWS * t, static_cast<int64_t>(p.rows) - 1);
#pragma unroll
                    for (int h = 0; h < H; ++h) {
                        const int64_t at = min(c + h * V, static_cast<int64_t>(p.cols) - V);
                        q[t].g[h] = *reinterpret_cast<const Loose<S> *>(static_cast<const S *>(p.grad_y) + r * p.grad_ld + at);
                        if (ACT) q[t].z[h] = *reinterpret_cast<const Loose<S> *>(static_cast<const S *>(p.z) + r * p.z_ld + at);
                    }
                    if (rests) q[t].rest = *reinterpret_cast<const Loose<__bf16> *>(p.rest + r * p.cols + min(c, static_cast<int64_t>(p.cols) - 8));
                }
                if (n < 8 || first + ROWS * (kAhead - 1) >= p.rows)
#pragma unroll
                    for (int t = 0; t < kAhead; ++t) {
                        const int left = first + ROWS * t < p.rows ? static_cast<int>(n) : 0;
#pragma unroll
                        for (int h = 0; h < H; ++h)
                            if (left - h * V < V) {
                                q[t].g[h] = loose_from(q[t].g[h], V - (left - h * V));
                                if (ACT) q[t].z[h] = loose_from(q[t].z[h], V - (left - h * V));
                            }
                        if (rests && left < 8) q[t].rest = loose_from(q[t].rest, 8 - left);
                    }
            } else
#pragma unroll
                for (int t = 0; t < kAhead; ++t) {
                    const int64_t r = first + ROWS * t;
                    const int left = r < p.rows ? static_cast<int>(n) : 0, before = static_cast<int>(c);
#pragma unroll
                    for (int h = 0; h < H; ++h) {
                        q[t].g[h] = loose_load_end(static_cast<const S *>(p.grad_y) + r * p.grad_ld + c + h * V, left - h * V, before + h * V);
                        if (ACT) q[t].z[h] = loose_load_end(static_cast<const S *>(p.z) + r * p.z_ld + c + h * V, left - h * V, before + h * V);
                    }
                    if (rests) q[t].rest = loose_load_end(reinterpret_cast<const __bf16 *>(p.rest) + r * p.cols + c, left, before);
                }
#pragma unroll
            for (int t = 0; t < kAhead; ++t) {
                const int64_t r = first + ROWS * t;
                if (r >= r1) break;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] = loose_get(q[t].g[e / V], e % V);
                    if constexpr (ACT) {
                        float z = loose_get(q[t].z[e / V], e % V), slope;
                        if (rests) z = with_rest(z, q[t].rest.w[e >> 1] >> (e & 1) * 16);
                        act_of<decltype(a)::value, true>(z, &slope);
                        v[e] *= slope;
                    }
                    sum[e] += v[e];
                }
                if (p.flat) {
                    *reinterpret_cast<f32x4 *>(p.flat + r * p.ld + c) = f32x4{v[0], v[1], v[2], v[3]};
                    *reinterpret_cast<f32x4 *>(p.flat + r * p.ld + c + 4) = f32x4{v[4], v[5], v[6], v[7]};
                }
                if (p.dz)
#pragma unroll
                    for (int s = 0; s < Q; ++s) {
                        u32x4 o;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t lo = plane_of<Q>(s, v[2 * k]), hi = plane_of<Q>(s, v[2 * k + 1]);
                            o[k] = lo | hi << 16;
                        }
                        *reinterpret_cast<u32x4 *>(p.dz + s * p.plane + r * p.ld + c) = o;
                    }
            }
        }
    });
    if (!p.part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) red[row * WIDE + lane * 8 + e] = sum[e];
    __syncthreads();
    if (threadIdx.x >= WIDE) return;
    const int64_t at = column + threadIdx.x;
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < ROWS; ++k) s += red[k * WIDE + threadIdx.x];
    if (at < p.part_cols) p.part[chunk * p.part_cols + at] = s;
}

// All that a backward pass does before its products, in one launch.
template <typename S, int P, int Q>
__global__ void __launch_bounds__(256) linear_slope_kernel(Slope p, Pack x, Pack w)
{
    unsigned block = blockIdx.x;
    __shared__ float red[2048];
    if (block < p.blocks) return p.narrow ? slope_rows<S, Q, 8>(p, block, red) : slope_rows<S, Q, 32>(p, block, red);
    block -= p.blocks;
    if (block < x.blocks) return pack_rows<S, P>(x, block);
    pack_rows<S, P>(w, block - x.blocks);
}

// grad_x of few rows: w is read once, as it lies, at any alignment.  A lane reads a vector of each of 8 (float: 4) neighbouring rows of w, which are k, and
// exchanges their columns in registers: column j of its vector is a row of the j-th product's first operand.  dz is the second one (float: as it is, by
// v_mfma_f32_16x16x4).  The wavefronts of a workgroup share out k.
constexpr int kBackWaves = 8;

template <typename S, int R, int Q>
__global__ void __launch_bounds__(kBackWaves * 64) linear_few_back_kernel(const S *w, int64_t ldw, int32_t out, int32_t width, const uint16_t *dz, const float *flat, int64_t ldo,
                                                                          int64_t plane, int32_t rows, int32_t each, int32_t groups, int32_t sets, float *part, int64_t part_ld,
                                                                          S *grad_x, int64_t grad_ld)
{
    constexpr int J = kLooseElements<S>, COLS = 16 * J, STEP = 4 * J;
    __shared__ __align__(16) float red[kBackWaves][J][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, kq = lane >> 4;
    const int group = blockIdx.x % groups, set = blockIdx.x / groups % sets, split = blockIdx.x / groups / sets, row0 = set * (16 * R);
    const int c = group * COLS + i * J, n = width - c;
    const int64_t k0 = static_cast<int64_t>(split * kBackWaves + wave) * each, k1 = min(k0 + each, static_cast<int64_t>(out));
    f32x4 acc[J][R];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[j][r] = f32x4{0, 0, 0, 0};
    for (int64_t k = k0; k < k1; k += STEP) {
        Loose<S> v[J];
        if (width >= J) {       // (all loads at once; past the end of a row its last vector, shifted, and past the last row zeros)
            const S *from = w + min(c, width - J);
            if (k + STEP <= out)
#pragma unroll
                for (int t = 0; t < J; ++t) v[t] = *reinterpret_cast<const Loose<S> *>(from + (k + kq * J + t) * ldw);
            else {
#pragma unroll
                for (int t = 0; t < J; ++t) v[t] = *reinterpret_cast<const Loose<S> *>(from + min(k + kq * J + t, static_cast<int64_t>(out) - 1) * ldw);
#pragma unroll
                for (int t = 0; t < J; ++t)
                    if (k + kq * J + t >= out) v[t] = Loose<S>{};
            }
            if (n < J)
#pragma unroll
                for (int t = 0; t < J; ++t) v[t] = loose_from(v[t], J - n);
        } else
#pragma unroll
            for (int t = 0; t < J; ++t) v[t] = loose_load(w + (k + kq * J + t) * ldw + c, k + kq * J + t < out ? n : 0);
        if constexpr (sizeof(S) == 2) {
            bf16x8 b[R][Q];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int q = 0; q < Q; ++q) b[r][q] = *reinterpret_cast<const bf16x8 *>(dz + q * plane + (row0 + r * 16 + i) * ldo + k + kq * 8);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                u32x4 f;
#pragma unroll
                for (int t = 0; t < 4; ++t) f[t] = __builtin_amdgcn_perm(v[2 * t + 1].w[j / 2], v[2 * t].w[j / 2], j & 1 ? 0x07060302 : 0x05040100);
#pragma unroll
                for (int q = Q - 1; q >= 0; --q)
#pragma unroll
                    for (int r = 0; r < R; ++r) acc[j][r] = Mfma<bf16x8>::go(__builtin_bit_cast(bf16x8, f), b[r][q], acc[j][r]);
            }
        } else {
            f32x4 b[R];
#pragma unroll
            for (int r = 0; r < R; ++r) b[r] = *reinterpret_cast<const f32x4 *>(flat + (row0 + r * 16 + i) * ldo + k + kq * 4);
#pragma unroll
            for (int t = 0; t < J; ++t)
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int r = 0; r < R; ++r) acc[j][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(loose_get(v[t], j), b[r][t], acc[j][r], 0, 0, 0);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (r > 0) lds_barrier();
#pragma unroll
        for (int j = 0; j < J; ++j) *reinterpret_cast<f32x4 *>(&red[wave][j][lane * 4]) = acc[j][r];
        lds_barrier();
        // element e of lane l's sums: row l & 15 of x, columns (4 (l >> 4) + e) J .. + J - 1; a thread takes four of them
        const int at = threadIdx.x & 255, first = threadIdx.x / 256 * 4, l = at >> 2, e = at & 3;
        const int row = row0 + r * 16 + (l & 15), column = group * COLS + ((l >> 4) * 4 + e) * J + first;
        if (first < J && row < rows && column < width) {
            f32x4 v = {0, 0, 0, 0};
#pragma unroll
            for (int q = 0; q < kBackWaves; ++q)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += red[q][(first + j) % J][at];
            if (part) *reinterpret_cast<f32x4 *>(part + (static_cast<int64_t>(split) * rows + row) * part_ld + column) = v;
            else store4(grad_x + row * grad_ld + column, v, width - column);
        }
    }
}

template <typename TX, typename TW, typename O>
__global__ void __launch_bounds__(TX::NT, 2) linear_products_kernel(Product px, Product pw)
{
    static_assert(TX::LDS == TW::LDS && TX::NT == TW::NT, "one launch");
    extern __shared__ __align__(128) char smem[];
    // each XCD gets an eighth of both, which are of different lengths
    const int first = px.tm * px.tn * px.splits, id = blockIdx.x;
    if (id < first) product_tile<TX, O>(px, xcd_contiguous(id, first), smem);
    else product_tile<TW, O>(pw, xcd_contiguous(id - first, gridDim.x - first), smem);
}

// Up to three sums in one launch: of grad_x's, of grad_w's and of grad_bias's parts.
template <typename O>
__global__ void __launch_bounds__(256) linear_finish_kernel(Sum x, Sum w, Sum bias)
{
    unsigned block = blockIdx.x;
    if (block < x.blocks) return sum_parts<O>(x, block);
    block -= x.blocks;
    if (block < w.blocks) return sum_parts<O>(w, block);
    sum_parts<float>(bias, block - w.blocks);
}

template <typename O>
__global__ void __launch_bounds__(256) linear_zero_kernel(O *out, int64_t ld, int64_t rows, int32_t cols)
{
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; t < rows * cols; t += static_cast<int64_t>(gridDim.x) * 256)
        out[t / cols * ld + t % cols] = static_cast<O>(0.0f);
}

// ---------------------------------------------------------------- host side

// linear_few_kernel or tiles, us: bf16 1 x 4 096 x 16 384 23 / 25, 16 x 4 096 x 4 096 11 / 12, 32 x 4 096 x 4 096 17 / 12 (not taken), but 16 x 4 096 x 16 384 33 / 28,
// which a rule that goes by rows takes all the same; float, whose tiles want their operands in planes, 16 x 4 096 x 4 096 18 / 55, 64 x 4 096 x 4 096 39 / 50,
// 128 x 1 509 x 12 939 107 / 78 (not taken).  Few weights are launches and waits, of which it has fewer: 128 x 1 568 x 128 6 / 14, float 8 / 14, 256 x 300 x 2 000
// 7 / 11, float 10 / 15.
constexpr int64_t kSmallWeights = 1 << 20;
// linear_few_back_kernel or tiles, us of a backward pass: bf16 1 x 4 096 x 4 096 30 / 39, 16 x 1 509 x 12 939 46 / 62, 64 x 4 096 x 16 384 126 / 222, 128 x 4 096 x 4 096
// 54 / 45 (not taken), but 50 x 1 509 x 12 939 63 / 60, which is taken all the same; float 1 x 4 096 x 4 096 45 / 83, 64 x 1 509 x 12 939 99 / 126, 128 x 4 096 x 4 096
// 111 / 101 (not taken); few weights (not taken) 16 x 1 568 x 128 15 / 12, 64 x 300 x 2 000 23 / 16.
constexpr int32_t kMostFewBack = 64;
constexpr int64_t kFewBackWeights = 1 << 22;

// What tiles take, in elements of a result times k, some 2.35 G of which the chip does in a millisecond with one product of planes in the large tiles
// (256 x 256; float 128 x 256, six products).  A tile takes kAround k more than it has, and two on a unit twice as long as one.  Smaller ones load more for what they multiply, by kSlower; adding up
// shares costs kSumWeight an element of each and a launch kLaunchWeight, both in terms of one product.  us, as chosen / others, a pass one way without z: forward, bf16
// 4 096 x 1 024 x 4 096 42 (256 x 256) / 45 (128 x 128), 2 000 x 2 048 x 2 048 26 (128 x 128) / 58 (256 x 256) / 32 (64 x 64), 1 000 x 777 x 1 501 15 (64 x 64) / 21
// (128 x 128 in two shares), float 1 000 x 777 x 1 501 32 (128 x 128 in two shares) / 41 (64 x 64) / 47 (128 x 128); backward, bf16 4 096 x 1 024 x 4 096 105 (128 x 128)
// / 116 (256 x 256 in two shares each) / 134 (256 x 256), 8 192 x 4 096 x 4 096 490 (256 x 256) / 576 (128 x 128), float 300 x 300 x 300 16 (64 x 64 in three shares) / 19 (in one).
constexpr double kAround = 160, kSumWeight = 2.5, kLaunchWeight = 7e6;
template <int P, int Q>
constexpr double kSlower[3] = {P == 3 ? 3.0 : 2.2, P == 3 ? 1.33 : Q == 2 ? 1.0 : 1.16, 1.0};
template <int P, int Q>
constexpr int kProducts = P == 3 ? 6 : Q;

// A forward pass.
struct Layout {
    int few, few_outs;                      // 16 rows and outs to R and M of linear_few_kernel; 0: tiles
    int32_t waves, each, groups, sets;      // few: wavefronts of a workgroup, k of each, workgroups to outs and to rows
    int size;                               // 2, 1, 0: of the tiles
    Tiles tiles;
    int64_t kp, ldk;                        // width as it is laid out, and from row to row
    uint16_t *xp, *wp;
    int64_t bytes;
};

template <int P>
Layout lay_out(const dol_matrix *x, const dol_matrix *w, void *workspace)
{
    using Z = Shapes<P, P>;
    Layout L{};
    Carver c(workspace);
    const int32_t rows = x->rows, width = x->cols, out = w->rows;
    L.tiles.part_ld = round_up(out, 4), L.tiles.splits = 1;
    const int64_t weights = int64_t(out) * width;
    if (rows <= 16 || (P == 3 && rows <= 64) || (weights <= kSmallWeights && rows <= 256)) {
        // (rows of their own for a workgroup read the weights again, which costs nothing where the chip is not full)
        L.few = rows <= 16 || P == 1 || tiles(out, 16) * tiles(rows, 16) <= 2 * kUnits ? 1 : rows <= 32 ? 2 : 4;
        L.few_outs = L.few > 1 && tiles(out, 128 / L.few) >= kUnits / 2 ? 8 / L.few : 1;
        L.groups = tiles(out, 16 * L.few_outs);
        L.sets = tiles(rows, 16 * L.few);
        const int32_t shares = std::min(tiles(width, 128), std::max(4, 4096 / (L.groups * L.sets)));
        const int most = few_waves(L.few * L.few_outs);
        L.waves = std::min(shares, most), L.tiles.splits = tiles(shares, most);
        L.each = static_cast<int32_t>(round_up(tiles(width, L.waves * L.tiles.splits), 64));
    } else {
        L.kp = round_up(width, 64), L.ldk = spread(L.kp);
        double best = 0.0;
        auto consider = [&](int size, auto z) {
            using T = typename decltype(z)::Tile;
            const int32_t tm = tiles(rows, T::BM), tn = tiles(out, T::BN), steps = static_cast<int32_t>(L.kp / T::BK);
            for (int32_t n = 1; n <= std::min(16, std::max(1, steps / 2)); ++n) {
                const double all = done(int64_t(tm) * tn * n, double(width) / n + kAround, 0, 0.0, kUnits) * T::BM * T::BN * kSlower<P, P>[size] +
                                   (n > 1 ? (kSumWeight * n * rows * out + kLaunchWeight) / kProducts<P, P> : 0.0);
                if (best == 0.0 || all < best) best = all, L.size = size, L.tiles.tm = tm, L.tiles.tn = tn, L.tiles.steps = steps, L.tiles.splits = n;
            }
        };
        consider(2, Type<typename Z::Big>()), consider(1, Type<typename Z::Small>()), consider(0, Type<typename Z::Tiny>());
        if (!direct(x)) L.xp = c.take<uint16_t>(P * int64_t(rows) * L.ldk);
        if (!direct(w)) L.wp = c.take<uint16_t>(P * int64_t(out) * L.ldk);
    }
    if (L.tiles.splits > 1) L.tiles.part = c.take<float>(int64_t(L.tiles.splits) * rows * L.tiles.part_ld);
    L.bytes = c.used;
    return L;
}

constexpr int kOneChunk = 64;

// A backward pass.
struct Back {
    int64_t kp, ldk, ko, ldo, n_pad;        // width, out and rows as they are laid out
    uint16_t *xp, *wp, *dz;
    bool x_direct;
    int few;                                // 16 rows to R of linear_few_back_kernel, 0: tiles for grad_x as for grad_w
    int32_t few_each, few_groups, few_sets; // k of a wavefront, workgroups to columns and to rows
    float *flat;
    int size, splits_x, splits_w;
    float *part_x, *part_w, *bias_part;
    int64_t part_ld;
    int32_t chunk, chunks;
    int64_t bytes;
};

template <int P, int Q>
Back lay_back(const dol_matrix *x, const dol_matrix *w, void *workspace)
{
    using Z = Shapes<P, Q>;
    Back L{};
    Carver c(workspace);
    const int32_t rows = x->rows, width = x->cols, out = w->rows;
    L.kp = round_up(width, 64), L.ldk = spread(L.kp), L.ko = round_up(out, 64), L.ldo = spread(L.ko), L.n_pad = round_up(rows, 64);
    L.part_ld = round_up(width, 4);
    // (k of grad_w: rows past the last have to be zeros in both operands)
    L.x_direct = direct(x) && rows % 64 == 0;
    if (!L.x_direct) L.xp = c.take<uint16_t>(P * L.n_pad * L.ldk);
    if (rows <= kMostFewBack && int64_t(out) * width >= kFewBackWeights) {
        constexpr int J = P == 3 ? 4 : 8;
        L.few = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
        L.few_groups = tiles(width, 16 * J), L.few_sets = tiles(rows, 16 * L.few);
        const int32_t splits = std::max(1, std::min(tiles(out, kBackWaves * 8 * J), 384 / (L.few_groups * L.few_sets)));
        L.few_each = static_cast<int32_t>(round_up(tiles(out, kBackWaves * splits), 4 * J));
        if (P == 3) L.flat = c.take<float>(L.n_pad * L.ldo);
    } else if (!direct(w)) L.wp = c.take<uint16_t>(P * int64_t(out) * L.ldk);
    L.dz = c.take<uint16_t>(Q * L.n_pad * L.ldo);
    // (few rows are one chunk, whose sums are grad_bias)
    L.chunk = rows <= kOneChunk ? kOneChunk : static_cast<int32_t>(std::max<int64_t>(8, std::min<int64_t>(64, round_up(tiles(L.n_pad * tiles(L.ko, 256), 1024), 8))));
    L.chunks = tiles(L.n_pad, L.chunk);
    L.bias_part = c.take<float>(L.chunks * L.ko);
    // shares of k so that the workgroups of both products come out even on the units
    double best = 0.0;
    auto consider = [&](int size, auto z) {
        using T = typename decltype(z)::Tile;
        const int64_t tx = L.few ? 0 : int64_t(tiles(width, T::BM)) * tiles(rows, T::BN), tw = int64_t(tiles(width, T::BM)) * tiles(out, T::BN);
        const int64_t even = (tx * out + tw * rows) / kUnits;
        for (int q = 6; q <= 20; ++q) {
            const int64_t share = std::max<int64_t>(96, even * q / 10), sx = L.few ? 1 : std::max<int64_t>(1, (out + share / 2) / share), sw = std::max<int64_t>(1, (rows + share / 2) / share);
            const double sums = (sx > 1 ? double(sx) * rows : 0.0) + (sw > 1 ? double(sw) * out : 0.0);
            const double all = done(tx * sx, double(out) / sx + kAround, tw * sw, double(rows) / sw + kAround, kUnits) * T::BM * T::BN * kSlower<P, Q>[size] +
                               (sums * width * kSumWeight + (sums > 0.0 && L.chunks == 1 ? kLaunchWeight : 0.0)) / kProducts<P, Q>;
            if (best == 0.0 || all < best) best = all, L.size = size, L.splits_x = static_cast<int>(sx), L.splits_w = static_cast<int>(sw);
        }
    };
    consider(2, Type<typename Z::BigX>()), consider(1, Type<typename Z::SmallX>()), consider(0, Type<typename Z::TinyX>());
    if (L.few) L.splits_x = tiles(out, kBackWaves * L.few_each);
    if (L.splits_x > 1) L.part_x = c.take<float>(int64_t(L.splits_x) * rows * L.part_ld);
    if (L.splits_w > 1) L.part_w = c.take<float>(int64_t(L.splits_w) * out * L.part_ld);
    L.bytes = c.used;
    return L;
}

// dz rounded to bf16 is off by up to 2^-8 of each number, which adds to grad_x and grad_weight about as much error as their own rounding does: 2.4e-3 in the norm
// in all where it is 1.7e-3, whatever the sizes.  A second plane takes it away, and is a second product: with few rows, where the products cost little, it is
// taken; above, it would double the largest launch.
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
    linear_pack_kernel<typename Source<P>::T, P><<<a.blocks + b.blocks, 256, 0, st>>>(a, b);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <typename S>
dol_status launch_join(const Layout &L, const Result &o, hipStream_t st)
{
    if (L.tiles.splits == 1) return DOL_OK;
    const int64_t n = int64_t(o.rows) * tiles(o.cols, 4);
    linear_join_kernel<S><<<blocks(std::min(n, kMostBlocks * 256)), 256, 0, st>>>(L.tiles.part, L.tiles.part_ld, L.tiles.splits, o);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <int P>
dol_status forward(const Layout &L, const dol_matrix *x, const dol_matrix *w, const Result &o, hipStream_t st)
{
    using S = typename Source<P>::T;
    if (L.few) {
        using std::integral_constant;
        auto go = [&](auto r, auto m) {
            linear_few_kernel<S, r.value, m.value><<<L.groups * L.sets * L.tiles.splits, L.waves * 64, 0, st>>>(static_cast<const S *>(x->data), x->ld, static_cast<const S *>(w->data),
                                                                                                            w->ld, x->cols, L.each, L.groups, L.sets, L.tiles.part, L.tiles.part_ld, o);
            DOL_HIP(hipGetLastError());
            return DOL_OK;
        };
        const integral_constant<int, 1> one;
        dol_status s = DOL_OK;
        if (L.few == 1) s = go(one, one);
        else if constexpr (P == 3) {
            const integral_constant<int, 2> two;
            const integral_constant<int, 4> four;
            s = L.few == 2 ? L.few_outs == 1 ? go(two, one) : go(two, four) : L.few_outs == 1 ? go(four, one) : go(four, two);
        }
        if (s) return s;
        return launch_join<S>(L, o, st);
    }
    Planes xp, wp;
    const Pack a = pack_of<P>(x, nullptr, nullptr, 0, L.xp, x->rows, L.kp, L.ldk, &xp), b = pack_of<P>(w, nullptr, nullptr, 0, L.wp, w->rows, L.kp, L.ldk, &wp);
    if (dol_status s = launch_pack<P>(a, b, st)) return s;
    using Z = Shapes<P, P>;
    if (dol_status s = by_size(L.size, Type<typename Z::Big>(), Type<typename Z::Small>(), Type<typename Z::Tiny>(), [&](auto z) {
            using T = typename decltype(z)::Tile;
            auto go = [&](auto a) {
                const auto kernel = linear_tiles_kernel<T, S, a.value>;
                DOL_HIP(allow_dynamic_lds(reinterpret_cast<const void *>(kernel), T::LDS));
                kernel<<<L.tiles.tm * L.tiles.tn * L.tiles.splits, T::NT, T::LDS, st>>>(xp, wp, L.tiles, o);
                DOL_HIP(hipGetLastError());
                return DOL_OK;
            };
            return L.tiles.splits > 1 || o.act == DOL_ACT_NONE ? go(Act<DOL_ACT_NONE>())
                   : o.act == DOL_ACT_RELU                     ? go(Act<DOL_ACT_RELU>())
                   : o.act == DOL_ACT_SILU                     ? go(Act<DOL_ACT_SILU>())
                                                               : go(Act<DOL_ACT_GELU>());
        }))
        return s;
    return launch_join<S>(L, o, st);
}

template <typename TX, typename TW, typename O>
dol_status launch_products(Product x, Product w, hipStream_t st)
{
    DOL_HIP(allow_dynamic_lds(reinterpret_cast<const void *>(linear_products_kernel<TX, TW, O>), TX::LDS));
    for (Product *p : {&x, &w})
        if (p->M > 0) p->tm = tiles(p->M, TX::BM), p->tn = tiles(p->N, TX::BN), p->steps = tiles(p->k, TX::BK);
    const int n = x.tm * x.tn * x.splits + w.tm * w.tn * w.splits;
    if (n == 0) return DOL_OK;
    linear_products_kernel<TX, TW, O><<<n, TX::NT, TX::LDS, st>>>(x, w);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <int P, int Q>
dol_status reverse(const Back &L, const dol_matrix *x, const dol_matrix *w, int act, const dol_matrix *z, const int16_t *rest, const dol_matrix *grad_y,
                   const dol_matrix *grad_x, const dol_matrix *grad_w, float *grad_bias, hipStream_t st)
{
    using S = typename Source<P>::T;
    using Z = Shapes<P, Q>;
    Planes xp{}, wp{}, dz{L.dz, L.ldo, L.n_pad * L.ldo};
    Pack lx{}, lw{};
    if (grad_w) lx = pack_of<P>(x, nullptr, nullptr, 0, L.xp, L.n_pad, L.kp, L.ldk, &xp);
    if (grad_x && !L.few) lw = pack_of<P>(w, nullptr, nullptr, 0, L.wp, w->rows, L.kp, L.ldk, &wp);
    // dz is grad_y itself where the tiles can read that (in one plane)
    const bool as_it_is = Q == 1 && !L.few && act == DOL_ACT_NONE && direct(grad_y) && x->rows % 64 == 0, write = !as_it_is && (grad_x || grad_w);
    if (as_it_is) dz = Planes{static_cast<const uint16_t *>(grad_y->data), grad_y->ld, 0};
    Slope p{};
    if (write || grad_bias) {
        const bool narrow = L.chunks == 1;
        const int32_t wide = tiles(L.ko, narrow ? 64 : 256);
        p = Slope{grad_y->data, z ? z->data : nullptr, grad_y->ld, z ? z->ld : 0, rest, x->rows, w->rows, act, write ? L.dz : nullptr, write && grad_x ? L.flat : nullptr, L.n_pad, L.ko, L.ldo, L.n_pad * L.ldo,
                  grad_bias ? L.chunks == 1 ? grad_bias : L.bias_part : nullptr, L.chunks == 1 ? w->rows : static_cast<int32_t>(L.ko), L.chunk, wide,
                  narrow, static_cast<unsigned>(wide * L.chunks)};
    }
    if (const unsigned n = p.blocks + lx.blocks + lw.blocks) {
        linear_slope_kernel<S, P, Q><<<n, 256, 0, st>>>(p, lx, lw);
        DOL_HIP(hipGetLastError());
    }
    Product a{}, b{};
    Sum sx{};
    if (grad_x && L.few) {
        auto go = [&](auto r) {
            // (in bf16 only ever of two planes, since these are few rows)
            linear_few_back_kernel<S, r.value, 2><<<L.few_groups * L.few_sets * L.splits_x, kBackWaves * 64, 0, st>>>(
                static_cast<const S *>(w->data), w->ld, w->rows, w->cols, L.dz, L.flat, L.ldo, L.n_pad * L.ldo, x->rows, L.few_each, L.few_groups, L.few_sets, L.part_x, L.part_ld,
                static_cast<S *>(grad_x->data), grad_x->ld);
            DOL_HIP(hipGetLastError());
            return DOL_OK;
        };
        if (dol_status s = L.few == 1 ? go(std::integral_constant<int, 1>())
                           : L.few == 2 ? go(std::integral_constant<int, 2>())
                                        : go(std::integral_constant<int, 4>()))
            return s;
        if (L.part_x) sx = make_sum(L.part_x, x->rows, x->cols, L.splits_x, L.part_ld, grad_x->data, grad_x->ld);
    } else if (grad_x) {
        a.a = wp, a.b = dz;
        a.M = x->cols, a.N = x->rows, a.wide = static_cast<int32_t>(L.kp), a.tall = x->rows, a.splits = L.splits_x, a.k = a.have = w->rows;
        a.part = L.part_x, a.part_ld = L.part_ld, a.out = grad_x->data, a.out_ld = grad_x->ld;
    }
    if (grad_w) {
        b.a = xp, b.b = dz;
        b.M = x->cols, b.N = w->rows, b.wide = static_cast<int32_t>(L.kp), b.tall = static_cast<int32_t>(L.ko), b.splits = L.splits_w, b.k = x->rows, b.have = L.n_pad;
        b.part = L.part_w, b.part_ld = L.part_ld, b.out = grad_w->data, b.out_ld = grad_w->ld;
    }
    if (dol_status s = L.size == 2   ? launch_products<typename Z::BigX, typename Z::BigW, S>(a, b, st)
                       : L.size == 1 ? launch_products<typename Z::SmallX, typename Z::SmallW, S>(a, b, st)
                                     : launch_products<typename Z::TinyX, typename Z::TinyW, S>(a, b, st))
        return s;
    if (!L.few) sx = sum_of(a);
    const Sum sw = sum_of(b), sb = grad_bias && L.chunks > 1 ? make_sum(L.bias_part, 1, w->rows, L.chunks, L.ko, grad_bias, w->rows) : Sum{};
    const unsigned n = sx.blocks + sw.blocks + sb.blocks;
    if (n == 0) return DOL_OK;
    linear_finish_kernel<S><<<n, 256, 0, st>>>(sx, sw, sb);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <typename S>
dol_status zero(const dol_matrix *m, hipStream_t st)
{
    if (!m || m->rows == 0) return DOL_OK;
    linear_zero_kernel<S><<<std::min(blocks(int64_t(m->rows) * m->cols), 4096u), 256, 0, st>>>(static_cast<S *>(m->data), m->ld, m->rows, m->cols);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

dol_status check_operands(const dol_matrix *x, const dol_matrix *w)
{
    if (dol_status s = check_matrix(x, "x")) return s;
    if (dol_status s = check_matrix(w, "weight")) return s;
    if (x->dtype != w->dtype) return fail(DOL_EINVAL, "x and weight are of different types");
    if (x->cols != w->cols) return fail(DOL_ESHAPE, "x has %d columns, weight %d", x->cols, w->cols);
    if (w->rows < 1 || w->cols < 1) return fail(DOL_ESHAPE, "weight is %d x %d: there has to be one out of one element", w->rows, w->cols);
    if (x->rows > kMostRows || w->rows > kMostRows || w->cols > kMostWidth)
        return fail(DOL_EUNSUPPORTED, "%d rows, %d outs of %d elements: more than %d, or %d elements", x->rows, w->rows, w->cols, kMostRows, kMostWidth);
    return DOL_OK;
}

dol_status check_as(const dol_matrix *m, int32_t rows, int32_t cols, int32_t dtype, const char *name)
{
    if (!m) return DOL_OK;
    if (dol_status s = check_matrix(m, name)) return s;
    if (m->dtype != dtype) return fail(DOL_EINVAL, "%s is of another type than x", name);
    if (m->rows != rows || m->cols != cols) return fail(DOL_ESHAPE, "%s is %d x %d, not %d x %d", name, m->rows, m->cols, rows, cols);
    return DOL_OK;
}

}  // namespace
}  // namespace dol

using namespace dol;

extern "C" {

dol_status dol_linear_workspace(const dol_matrix *x, const dol_matrix *weight, int32_t backward, int64_t *bytes)
{
    if (dol_status s = check_operands(x, weight)) return s;
    if (!bytes) return fail(DOL_EINVAL, "bytes is NULL");
    *bytes = 0;
    if (x->rows > 0)
        *bytes = with_planes(x, [&](auto p, auto q) { return backward ? lay_back<p.value, q.value>(x, weight, nullptr).bytes : lay_out<p.value>(x, weight, nullptr).bytes; });
    return DOL_OK;
}

const char *dol_linear_kernel(const dol_matrix *x, const dol_matrix *weight, int32_t backward)
{
    static thread_local char name[64];
    if (check_operands(x, weight) != DOL_OK || x->rows == 0) return "";
    with_planes(x, [&](auto p, auto q) {
        using Z = Shapes<p.value, q.value>;
        auto at = [&](const char *kernel, auto z) {
            using T = typename decltype(z)::Tile;
            return snprintf(name, sizeof name, "%s %dx%dx%d", kernel, T::BM, T::BN, T::BK);
        };
        if (backward) {
            const Back L = lay_back<p.value, q.value>(x, weight, nullptr);
            if (L.few) return snprintf(name, sizeof name, "linear_few_back_kernel %d", 16 * L.few);
            return by_size(L.size, Type<typename Z::BigX>(), Type<typename Z::SmallX>(), Type<typename Z::TinyX>(), [&](auto z) { return at("linear_products_kernel", z); });
        }
        const Layout L = lay_out<p.value>(x, weight, nullptr);
        if (L.few) return snprintf(name, sizeof name, "linear_few_kernel %dx%d", 16 * L.few, 16 * L.few_outs);
        using F = Shapes<p.value, p.value>;
        return by_size(L.size, Type<typename F::Big>(), Type<typename F::Small>(), Type<typename F::Tiny>(), [&](auto z) { return at("linear_tiles_kernel", z); });
    });
    return name;
}

dol_status dol_linear(const dol_matrix *x, const dol_matrix *weight, const float *bias, int32_t act, const dol_matrix *residual, const dol_matrix *y, const dol_matrix *z,
                      int16_t *z_rest, void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    if (dol_status s = check_operands(x, weight)) return s;
    if (act < DOL_ACT_NONE || act > DOL_ACT_GELU) return fail(DOL_EINVAL, "unknown activation function %d", act);
    if (!y) return fail(DOL_EINVAL, "y is NULL");
    for (const auto &m : {std::make_pair(residual, "residual"), std::make_pair(y, "y"), std::make_pair(z, "z")})
        if (dol_status s = check_as(m.first, x->rows, weight->rows, x->dtype, m.second)) return s;
    if (z_rest && (!z || x->dtype != DOL_BF16)) return fail(DOL_EINVAL, "z_rest without z in bf16");
    const Span bias_(bias, weight->rows * sizeof(float)), rest(z_rest, static_cast<uint64_t>(x->rows) * weight->rows * sizeof(int16_t));
    for (const Span &m : {Span(x), Span(weight), Span(z), bias_, rest})
        if (meet(y, m)) return fail(DOL_EINVAL, "y is x, weight, z or another operand, or lies over part of it");
    for (const Span &m : {Span(x), Span(weight), Span(residual), bias_, rest})
        if (meet(z, m)) return fail(DOL_EINVAL, "z is x, weight, the residual or another operand, or lies over part of it");
    for (const Span &m : {Span(x), Span(weight), Span(residual), bias_})
        if (meet(rest, m)) return fail(DOL_EINVAL, "z_rest lies over an operand");
    if (cross(y, residual)) return fail(DOL_EINVAL, "y lies over the residual, but not each row over its own");
    if (x->rows == 0) return DOL_OK;
    Result o{};
    o.bias = bias, o.act = act, o.rows = x->rows, o.cols = weight->rows, o.y = y->data, o.y_ld = y->ld, o.rest = z_rest;
    if (residual) o.residual = residual->data, o.residual_ld = residual->ld;
    if (z) o.z = z->data, o.z_ld = z->ld;
    auto go = [&](auto p) {
        const Layout L = lay_out<p.value>(x, weight, workspace);
        if (dol_status s = check_workspace(workspace, workspace_bytes, L.bytes)) return s;
        return forward<p.value>(L, x, weight, o, static_cast<hipStream_t>(hip_stream));
    };
    return x->dtype == DOL_F32 ? go(std::integral_constant<int, 3>()) : go(std::integral_constant<int, 1>());
}

dol_status dol_linear_backward(const dol_matrix *x, const dol_matrix *weight, int32_t act, const dol_matrix *z, const int16_t *z_rest, const dol_matrix *grad_y,
                               const dol_matrix *grad_x, const dol_matrix *grad_weight, float *grad_bias, void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    if (dol_status s = check_operands(x, weight)) return s;
    if (act < DOL_ACT_NONE || act > DOL_ACT_GELU) return fail(DOL_EINVAL, "unknown activation function %d", act);
    if (!grad_y) return fail(DOL_EINVAL, "grad_y is NULL");
    if (act == DOL_ACT_NONE) z = nullptr, z_rest = nullptr;
    else if (!z) return fail(DOL_EINVAL, "z is NULL");
    if (z_rest && x->dtype != DOL_BF16) return fail(DOL_EINVAL, "z_rest without z in bf16");
    for (const auto &m : {std::make_pair(z, "z"), std::make_pair(grad_y, "grad_y")})
        if (dol_status s = check_as(m.first, x->rows, weight->rows, x->dtype, m.second)) return s;
    if (dol_status s = check_as(grad_x, x->rows, x->cols, x->dtype, "grad_x")) return s;
    if (dol_status s = check_as(grad_weight, weight->rows, weight->cols, x->dtype, "grad_weight")) return s;
    if (!grad_x && !grad_weight && !grad_bias) return fail(DOL_EINVAL, "no gradient is asked for");
    const Span bias(grad_bias, weight->rows * sizeof(float)), rest(z_rest, static_cast<uint64_t>(x->rows) * weight->rows * sizeof(int16_t));
    for (const Span &m : {Span(x), Span(weight), Span(z), Span(grad_y), rest}) {
        if (meet(grad_x, m) || meet(grad_weight, m)) return fail(DOL_EINVAL, "grad_x or grad_weight is x, weight, z or grad_y, or lies over part of it");
        if (meet(bias, m)) return fail(DOL_EINVAL, "grad_bias lies over an operand");
    }
    if (meet(grad_x, grad_weight) || meet(grad_x, bias) || meet(grad_weight, bias)) return fail(DOL_EINVAL, "grad_x, grad_weight and grad_bias lie over each other");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (x->rows == 0) {                     // sums over no rows
        if (dol_status s = x->dtype == DOL_BF16 ? zero<__bf16>(grad_weight, st) : zero<float>(grad_weight, st)) return s;
        const dol_matrix b{DOL_F32, 1, weight->rows, weight->rows, grad_bias};
        return grad_bias ? zero<float>(&b, st) : DOL_OK;
    }
    return with_planes(x, [&](auto p, auto q) {
        const Back L = lay_back<p.value, q.value>(x, weight, workspace);
        if (dol_status s = check_workspace(workspace, workspace_bytes, L.bytes)) return s;
        return reverse<p.value, q.value>(L, x, weight, act, z, z_rest, grad_y, grad_x, grad_weight, grad_bias, st);
    });
}

}  // extern "C"
