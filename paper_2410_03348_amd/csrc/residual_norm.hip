// Where one block of a network ends and the next begins, and its gradients.  rms(v) = 1 / sqrt(mean of a row's v^2 + eps).
//
//   uhat = u rms(u), v = gamma_u uhat   (or v = u),   h = x + scale gate v,   hhat = h rms(h),   y = gamma_y hhat
//   a = gamma_y dy,   m1 = mean(a hhat),   dh = grad_h + rms(h) (a - hhat m1) = grad_x
//   k = scale gate gamma_u,   m2 = mean(k dh uhat),   grad_u = rms(u) (k dh - uhat m2)   (or scale gate dh)
//   grad_gate = scale sum dh v,   grad_gamma_u = sum scale gate dh uhat,   grad_gamma_y = sum dy hhat   over rows
//
// Memory bounds it: four tensors forward, six backward.  A row lies in the registers of a group of 4 to 1 024 threads, each with one or two
// vectors of 16 bytes, and is read once.  Backward one round of sums is enough: with dh put into it, mean(k dh uhat) is
//   sum k uhat (grad_h + rms(h) a) - rms(h) m1 sum k uhat hhat,
// three sums that need nothing of each other.  Sums over rows stay in registers while a group goes down its rows; a workgroup leaves one part of
// each, which a second launch adds up in the order of the rows.  Rows too long for that are read twice (wide_*).
#include "internal.h"
#include "loose.h"
#include "wave_util.h"

#include <type_traits>
#include <utility>

namespace dol {
namespace {

constexpr int kThreads = 256;           // of a workgroup, where a row does not take more
constexpr int kWideThreads = 1024;
constexpr int kFewPoints = 32;          // rows to a set, below which a group takes all rows of its sets by itself
constexpr int kUnits = 256;             // compute units of the chip
constexpr int64_t kMostBlocks = 1 << 20;        // of a launch, which has less than 2^32 threads

template <typename S>
struct Mat {
    S *p;
    int64_t ld;
    __device__ S *at(int64_t r, int c) const { return p + r * ld + c; }
};

template <typename S>
struct Args {
    Mat<const S> x, u, gate, grad_h, grad_y;
    Mat<S> out_h, out_y, grad_x, grad_u, grad_gate;
    const float *gamma_u, *gamma_y;
    float *rstd_u, *rstd_h;             // written forward, read backward
    int32_t rows, cols, norm_u, each;   // each: a gate for every row; else rows come in `sets` of `points`, a gate (or none) to a set
    int64_t sets, points;
    float scale, eps, per_cols;
    int64_t chunk, chunks;              // backward: rows that a workgroup takes, and how many such a set is
    float *part_y, *part_u, *part_gate; // [workgroups][cols], null where not asked for
    float2 *row;                        // wide: m1 and m2 of each row
    __device__ int64_t gate_of(int64_t r) const { return each || !gate.p ? r : r / points; }
};

template <int G>
__device__ __forceinline__ float group_sum(float x)
{
    static_assert(G >= 4 && G <= 64, "lanes of one wavefront");
    x += dpp<0xB1>(x);
    x += dpp<0x4E>(x);
    if constexpr (G >= 8) x += dpp<0x141>(x);
    if constexpr (G >= 16) x += dpp<0x140>(x);
    if constexpr (G >= 32) x = with_lane16<AddOp>(x);
    if constexpr (G >= 64) x = with_lane32<AddOp>(x);
    return x;
}

// Sums of N numbers over a group of G threads, in all of them.  `red` is N numbers for each wavefront, not used again before another barrier.
template <int G, int N>
__device__ __forceinline__ void group_sums(float (&x)[N], float *red)
{
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = group_sum<G < 64 ? G : 64>(x[n]);
    if constexpr (G > 64) {
        constexpr int W = G / 64;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) red[wave * N + n] = x[n];
        lds_barrier();
        const float *mine = red + wave / W * W * N;
#pragma unroll
        for (int n = 0; n < N; ++n) x[n] = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
            for (int n = 0; n < N; ++n) x[n] += mine[w * N + n];
    }
}

// n of a vector's values from p, `other` where there is no tensor.
template <typename S, int V>
__device__ __forceinline__ void get(float (&x)[V], const S *p, bool given, int n, float other)
{
    if (!given) {
#pragma unroll
        for (int k = 0; k < V; ++k) x[k] = other;
        return;
    }
    if constexpr (sizeof(S) == 4 && V == 8) {
        const Loose<float> a = loose_load(p, n), b = loose_load(p + 4, n - 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = loose_get(a, k), x[4 + k] = loose_get(b, k);
    } else {
        const Loose<S> a = loose_load(p, n);
#pragma unroll
        for (int k = 0; k < V; ++k) x[k] = loose_get(a, k);
    }
}

template <typename S, int V>
__device__ __forceinline__ void put(S *p, const float (&x)[V], int n)
{
    Loose<S> v;
    loose_set(v, x);
    loose_store(p, v, n);
}

__device__ __forceinline__ float rms(float squares, float per_cols, float eps) { return 1.0f / __builtin_amdgcn_sqrtf(__builtin_fmaf(squares, per_cols, eps)); }

// ---------------------------------------------------------------- forward

template <typename S, int G, int NV>
__global__ void __launch_bounds__(G > kThreads ? G : kThreads) residual_norm_kernel(Args<S> a)
{
    constexpr int V = kLooseElements<S>, T = G > kThreads ? G : kThreads, R = T / G;
    __shared__ float red[2][T / 64];
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * R; first < a.rows; first += static_cast<int64_t>(gridDim.x) * R) {
        const int64_t r = first + group;
        const bool in = r < a.rows;
        const int64_t g = in ? a.gate_of(r) : 0;
        float h[NV][V], k[NV][V], x[NV][V];
        float s[1] = {0.0f};
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int c = (q * G + lane) * V, n = in ? a.cols - c : 0;
            get(x[q], a.x.at(r, c), a.x.p, n, 0.0f);
            get(h[q], a.u.at(r, c), true, n, 0.0f);
            get(k[q], a.gate.at(g, c), a.gate.p, n, 1.0f);
            float gamma[V];
            get(gamma, a.gamma_u + c, a.norm_u && a.gamma_u, n, 1.0f);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                s[0] = __builtin_fmaf(h[q][e], h[q][e], s[0]);
                h[q][e] *= gamma[e], k[q][e] *= a.scale;
            }
        }
        float rstd = 1.0f;
        if (a.norm_u) {
            group_sums<G, 1>(s, red[0]);
            rstd = rms(s[0], a.per_cols, a.eps);
            if (a.rstd_u && in && lane == 0) a.rstd_u[r] = rstd;
        }
        s[0] = 0.0f;
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                h[q][e] = __builtin_fmaf(k[q][e], h[q][e] * rstd, x[q][e]);
                s[0] = __builtin_fmaf(h[q][e], h[q][e], s[0]);
            }
        if (a.out_y.p) {
            group_sums<G, 1>(s, red[1]);
            rstd = rms(s[0], a.per_cols, a.eps);
            if (a.rstd_h && in && lane == 0) a.rstd_h[r] = rstd;
        }
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int c = (q * G + lane) * V, n = in ? a.cols - c : 0;
            if (n <= 0) continue;
            if (a.out_h.p) put(a.out_h.at(r, c), h[q], n);
            if (!a.out_y.p) continue;
            float gamma[V];
            get(gamma, a.gamma_y + c, a.gamma_y, n, 1.0f);
#pragma unroll
            for (int e = 0; e < V; ++e) h[q][e] = h[q][e] * rstd * gamma[e];
            put(a.out_y.at(r, c), h[q], n);
        }
        if constexpr (G > 64) lds_barrier();            // (red is written again)
    }
}

// ---------------------------------------------------------------- backward

// What a vector of a row leaves, and what it adds to the sums over rows.
template <typename S, int V>
struct Piece {
    float h[V], u[V], gy[V], gh[V];             // hhat, uhat (or u), grad_y, grad_h
    // gate: times scale.  h is made again from x and u: as it was rounded it would be off by 2^-9 in every term of grad_gamma_y.
    __device__ void read(const Args<S> &a, int64_t r, int c, int n, const float (&gamma_u)[V], const float (&gate)[V], float rstd_u, float rstd_h)
    {
        get(h, a.x.at(r, c), a.x.p && a.grad_y.p, n, 0.0f);
        get(u, a.u.at(r, c), true, n, 0.0f);
        get(gy, a.grad_y.at(r, c), a.grad_y.p, n, 0.0f);
        get(gh, a.grad_h.at(r, c), a.grad_h.p, n, 0.0f);
#pragma unroll
        for (int e = 0; e < V; ++e) u[e] *= rstd_u, h[e] = __builtin_fmaf(gate[e], gamma_u[e] * u[e], h[e]) * rstd_h;
    }
    __device__ void sums(float (&s)[3], const float (&gamma_u)[V], const float (&gamma_y)[V], const float (&gate)[V], float rstd_h) const
    {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float ay = gamma_y[e] * gy[e], ku = gate[e] * gamma_u[e] * u[e];
            s[0] = __builtin_fmaf(ay, h[e], s[0]);
            s[1] = __builtin_fmaf(ku, __builtin_fmaf(rstd_h, ay, gh[e]), s[1]);
            s[2] = __builtin_fmaf(ku, h[e], s[2]);
        }
    }
    __device__ void leave(const Args<S> &a, int64_t r, int c, int n, const float (&gamma_u)[V], const float (&gamma_y)[V], const float (&gate)[V], float rstd_u,
                          float rstd_h, float m1, float m2, bool own_gate, float (&sum_y)[V], float (&sum_u)[V], float (&sum_gate)[V]) const
    {
        float dh[V], du[V], dg[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            dh[e] = __builtin_fmaf(rstd_h, __builtin_fmaf(-h[e], m1, gamma_y[e] * gy[e]), gh[e]);
            const float dv = gate[e] * dh[e], t = dh[e] * u[e];
            du[e] = a.norm_u ? rstd_u * __builtin_fmaf(-u[e], m2, gamma_u[e] * dv) : dv;
            dg[e] = a.scale * gamma_u[e] * t;
            sum_y[e] = __builtin_fmaf(gy[e], h[e], sum_y[e]);
            sum_u[e] = __builtin_fmaf(gate[e], t, sum_u[e]);
            sum_gate[e] += dg[e];
        }
        if (n <= 0) return;
        if (a.grad_x.p) put(a.grad_x.at(r, c), dh, n);
        if (a.grad_u.p) put(a.grad_u.at(r, c), du, n);
        if (own_gate) put(a.grad_gate.at(r, c), dg, n);
    }
};

// The sums of a workgroup's groups over their rows, in the order of the groups, to to[c].
template <int G, int NV, int V, int R>
__device__ __forceinline__ void leave_part(const float (&sum)[NV][V], float *to, int cols, float *buf)
{
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    if constexpr (R == 1) {
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int c = (q * G + lane) * V + e;
                if (c < cols) to[c] = sum[q][e];
            }
    } else {
        constexpr int W = G * NV * V;
        lds_barrier();
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < V; ++e) buf[group * W + (q * G + lane) * V + e] = sum[q][e];
        lds_barrier();
        for (int c = threadIdx.x; c < cols; c += R * G) {
            float s = 0.0f;
            for (int g = 0; g < R; ++g) s += buf[g * W + c];
            to[c] = s;
        }
    }
}

// WHOLE: a group takes all rows of its sets; else a workgroup takes a chunk of the rows of one set.
template <typename S, int G, int NV, bool WHOLE>
__global__ void __launch_bounds__(G > kThreads ? G : kThreads) residual_norm_backward_kernel(Args<S> a)
{
    constexpr int V = kLooseElements<S>, T = G > kThreads ? G : kThreads, R = T / G;
    __shared__ float red[2][3 * (T / 64)];
    __shared__ float buf[R > 1 ? T * NV * V : 1];
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    const bool own_gate = a.grad_gate.p && a.each;
    const int64_t set = WHOLE ? 0 : blockIdx.x / a.chunks, r0 = WHOLE ? 0 : set * a.points + blockIdx.x % a.chunks * a.chunk;
    const int64_t r1 = WHOLE ? 0 : min(r0 + a.chunk, (set + 1) * a.points);
    const int64_t sets = WHOLE ? (a.sets + static_cast<int64_t>(gridDim.x) * R - 1) / (static_cast<int64_t>(gridDim.x) * R) : 1;
    float sum_y[NV][V], sum_u[NV][V], sum_gate[NV][V], gamma_y[NV][V], gamma_u[NV][V];
#pragma unroll
    for (int q = 0; q < NV; ++q) {
        const int c = (q * G + lane) * V, n = a.cols - c;
        get(gamma_y[q], a.gamma_y + c, a.gamma_y, n, 1.0f);
        get(gamma_u[q], a.gamma_u + c, a.norm_u && a.gamma_u, n, 1.0f);
#pragma unroll
        for (int e = 0; e < V; ++e) sum_y[q][e] = sum_u[q][e] = sum_gate[q][e] = 0.0f;
    }
    int turn = 0;
    for (int64_t t = 0; t < sets; ++t) {
        const int64_t mine = (t * gridDim.x + blockIdx.x) * R + group;          // WHOLE: this group's set
        const int64_t count = WHOLE ? a.points : (r1 - r0 + R - 1) / R;
        for (int64_t k = 0; k < count; ++k) {
            const int64_t r = WHOLE ? mine * a.points + k : r0 + k * R + group;
            const bool in = WHOLE ? mine < a.sets : r < r1;
            const int64_t g = WHOLE ? mine : a.each ? r : set;
            const float rstd_u = a.norm_u && in ? a.rstd_u[r] : 1.0f, rstd_h = a.grad_y.p && in ? a.rstd_h[r] : 0.0f;
            Piece<S, V> p[NV];
            float gate[NV][V], s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                const int c = (q * G + lane) * V, n = in ? a.cols - c : 0;
                get(gate[q], a.gate.at(g, c), a.gate.p, n, 1.0f);
#pragma unroll
                for (int e = 0; e < V; ++e) gate[q][e] *= a.scale;
                p[q].read(a, r, c, n, gamma_u[q], gate[q], rstd_u, rstd_h);
                p[q].sums(s, gamma_u[q], gamma_y[q], gate[q], rstd_h);
            }
            group_sums<G, 3>(s, red[turn]);
            turn ^= 1;
            const float m1 = s[0] * a.per_cols, m2 = __builtin_fmaf(-rstd_h * m1, s[2], s[1]) * a.per_cols;
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                const int c = (q * G + lane) * V, n = in ? a.cols - c : 0;
                p[q].leave(a, r, c, n, gamma_u[q], gamma_y[q], gate[q], rstd_u, rstd_h, m1, m2, own_gate, sum_y[q], sum_u[q], sum_gate[q]);
            }
        }
        if (WHOLE && a.grad_gate.p) {
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                const int c = (q * G + lane) * V, n = mine < a.sets ? a.cols - c : 0;
                if (n > 0) put(a.grad_gate.at(mine, c), sum_gate[q], n);
#pragma unroll
                for (int e = 0; e < V; ++e) sum_gate[q][e] = 0.0f;
            }
        }
    }
    const int64_t at = static_cast<int64_t>(blockIdx.x) * a.cols;
    if (a.part_y) leave_part<G, NV, V, R>(sum_y, a.part_y + at, a.cols, buf);
    if (a.part_u) leave_part<G, NV, V, R>(sum_u, a.part_u + at, a.cols, buf);
    if (!WHOLE && a.part_gate) leave_part<G, NV, V, R>(sum_gate, a.part_gate + at, a.cols, buf);
}

// ---------------------------------------------------------------- wide rows

// A workgroup to a row, which it goes through three times; all is written in the last one, since h and y may lie on x and u.
template <typename S>
__global__ void __launch_bounds__(kWideThreads) residual_norm_wide_kernel(Args<S> a)
{
    constexpr int V = kLooseElements<S>;
    __shared__ float red[2][kWideThreads / 64];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const int64_t g = a.gate_of(r);
        float rstd_u = 1.0f, rstd_h = 0.0f, s[1] = {0.0f};
        auto stream = [&](int c, int n, float (&h)[V]) {        // h of the vector at c
            float x[V], k[V], gamma[V];
            get(x, a.x.at(r, c), a.x.p, n, 0.0f);
            get(h, a.u.at(r, c), true, n, 0.0f);
            get(k, a.gate.at(g, c), a.gate.p, n, 1.0f);
            get(gamma, a.gamma_u + c, a.norm_u && a.gamma_u, n, 1.0f);
#pragma unroll
            for (int e = 0; e < V; ++e) h[e] = __builtin_fmaf(k[e] * a.scale, h[e] * gamma[e] * rstd_u, x[e]);
        };
        if (a.norm_u) {
            for (int c = threadIdx.x * V; c < a.cols; c += kWideThreads * V) {
                float u[V];
                get(u, a.u.at(r, c), true, a.cols - c, 0.0f);
#pragma unroll
                for (int e = 0; e < V; ++e) s[0] = __builtin_fmaf(u[e], u[e], s[0]);
            }
            group_sums<kWideThreads, 1>(s, red[0]);
            rstd_u = rms(s[0], a.per_cols, a.eps);
            s[0] = 0.0f;
        }
        if (a.out_y.p) {
            for (int c = threadIdx.x * V; c < a.cols; c += kWideThreads * V) {
                float h[V];
                stream(c, a.cols - c, h);
#pragma unroll
                for (int e = 0; e < V; ++e) s[0] = __builtin_fmaf(h[e], h[e], s[0]);
            }
            group_sums<kWideThreads, 1>(s, red[1]);
            rstd_h = rms(s[0], a.per_cols, a.eps);
        }
        if (threadIdx.x == 0) {
            if (a.norm_u && a.rstd_u) a.rstd_u[r] = rstd_u;
            if (a.out_y.p && a.rstd_h) a.rstd_h[r] = rstd_h;
        }
        for (int c = threadIdx.x * V; c < a.cols; c += kWideThreads * V) {
            const int n = a.cols - c;
            float h[V], gamma[V];
            stream(c, n, h);
            if (a.out_h.p) put(a.out_h.at(r, c), h, n);
            if (!a.out_y.p) continue;
            get(gamma, a.gamma_y + c, a.gamma_y, n, 1.0f);
#pragma unroll
            for (int e = 0; e < V; ++e) h[e] = h[e] * rstd_h * gamma[e];
            put(a.out_y.at(r, c), h, n);
        }
        lds_barrier();          // (red is written again)
    }
}

// m1 and m2 of each row.
template <typename S>
__global__ void __launch_bounds__(kWideThreads) residual_norm_wide_rows_kernel(Args<S> a)
{
    constexpr int V = kLooseElements<S>;
    __shared__ float red[3 * (kWideThreads / 64)];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const int64_t g = a.gate_of(r);
        const float rstd_u = a.norm_u ? a.rstd_u[r] : 1.0f, rstd_h = a.grad_y.p ? a.rstd_h[r] : 0.0f;
        float s[3] = {0.0f, 0.0f, 0.0f};
        for (int c = threadIdx.x * V; c < a.cols; c += kWideThreads * V) {
            const int n = a.cols - c;
            Piece<S, V> p;
            float gate[V], gamma_u[V], gamma_y[V];
            get(gate, a.gate.at(g, c), a.gate.p, n, 1.0f);
            get(gamma_y, a.gamma_y + c, a.gamma_y, n, 1.0f);
            get(gamma_u, a.gamma_u + c, a.norm_u && a.gamma_u, n, 1.0f);
#pragma unroll
            for (int e = 0; e < V; ++e) gate[e] *= a.scale;
            p.read(a, r, c, n, gamma_u, gate, rstd_u, rstd_h);
            p.sums(s, gamma_u, gamma_y, gate, rstd_h);
        }
        group_sums<kWideThreads, 3>(s, red);
        const float m1 = s[0] * a.per_cols;
        if (threadIdx.x == 0) a.row[r] = make_float2(m1, __builtin_fmaf(-rstd_h * m1, s[2], s[1]) * a.per_cols);
        lds_barrier();
    }
}

// A workgroup takes kThreads vectors of the columns of a chunk of one set's rows.
template <typename S>
__global__ void __launch_bounds__(kThreads) residual_norm_wide_map_kernel(Args<S> a, int stripes)
{
    constexpr int V = kLooseElements<S>;
    const int64_t block = blockIdx.x / stripes, set = block / a.chunks, r0 = set * a.points + block % a.chunks * a.chunk, r1 = min(r0 + a.chunk, (set + 1) * a.points);
    const int c = (static_cast<int>(blockIdx.x % stripes) * kThreads + threadIdx.x) * V, n = a.cols - c;
    if (n <= 0) return;
    const bool own_gate = a.grad_gate.p && a.each;
    float sum_y[V], sum_u[V], sum_gate[V], gamma_y[V], gamma_u[V];
    get(gamma_y, a.gamma_y + c, a.gamma_y, n, 1.0f);
    get(gamma_u, a.gamma_u + c, a.norm_u && a.gamma_u, n, 1.0f);
#pragma unroll
    for (int e = 0; e < V; ++e) sum_y[e] = sum_u[e] = sum_gate[e] = 0.0f;
    for (int64_t r = r0; r < r1; ++r) {
        const int64_t g = a.each ? r : set;
        const float rstd_u = a.norm_u ? a.rstd_u[r] : 1.0f, rstd_h = a.grad_y.p ? a.rstd_h[r] : 0.0f;
        const float2 m = a.row[r];
        Piece<S, V> p;
        float gate[V];
        get(gate, a.gate.at(g, c), a.gate.p, n, 1.0f);
#pragma unroll
        for (int e = 0; e < V; ++e) gate[e] *= a.scale;
        p.read(a, r, c, n, gamma_u, gate, rstd_u, rstd_h);
        p.leave(a, r, c, n, gamma_u, gamma_y, gate, rstd_u, rstd_h, m.x, m.y, own_gate, sum_y, sum_u, sum_gate);
    }
    const int64_t at = block * a.cols + c;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        if (e >= n) break;
        if (a.part_y) a.part_y[at + e] = sum_y[e];
        if (a.part_u) a.part_u[at + e] = sum_u[e];
        if (a.part_gate) a.part_gate[at + e] = sum_gate[e];
    }
}

// ---------------------------------------------------------------- sums of the parts

// Up to three sums over the workgroups' parts: grad_gamma_y's, grad_gamma_u's, and each gate's.
template <typename S>
struct Sums {
    const float *part_y, *part_u, *part_gate;
    float *grad_gamma_y, *grad_gamma_u;
    Mat<S> grad_gate;
    int64_t parts, per_gate;            // parts in all, and of a gate
    int32_t cols;
};

// 64 columns by 16 shares of the parts to a workgroup; a share's parts lie 16 apart.
template <typename S>
__global__ void __launch_bounds__(1024) residual_norm_sums_kernel(Sums<S> s, int64_t jobs)
{
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t wide = (s.cols + 63) / 64;
    for (int64_t j = blockIdx.x; j < jobs; j += gridDim.x) {
        int64_t what = j / wide;
        const int c = static_cast<int>(j % wide) * 64 + lane;
        const float *from = nullptr;
        float *to = nullptr;
        if (s.part_y && what-- == 0) from = s.part_y, to = s.grad_gamma_y;
        else if (s.part_u && what-- == 0) from = s.part_u, to = s.grad_gamma_u;
        const int64_t first = from ? 0 : what * s.per_gate, n = from ? s.parts : s.per_gate;
        if (!from) from = s.part_gate;
        float v = 0.0f;
        if (c < s.cols)
#pragma unroll 4
            for (int64_t k = wave; k < n; k += 16) v += from[(first + k) * s.cols + c];
        red[wave][lane] = v;
        __syncthreads();
        if (wave == 0 && c < s.cols) {
            float t = 0.0f;
#pragma unroll
            for (int w = 0; w < 16; ++w) t += red[w][lane];
            if (to) to[c] = t;
            else *s.grad_gate.at(what, c) = static_cast<S>(t);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- host side

constexpr int32_t kMostCols = 1 << 24;

// Threads to a row and vectors of each; 0 threads: a row too long for registers.
struct Form {
    int threads, vectors;
};

Form form_of(int32_t cols, int32_t dtype)
{
    const int v = dtype == DOL_F32 ? 4 : 8;
    const int64_t n = (static_cast<int64_t>(cols) + v - 1) / v;
    for (const Form f : {Form{4, 1}, Form{8, 1}, Form{16, 1}, Form{32, 1}, Form{64, 1}, Form{64, 2}, Form{128, 2}, Form{256, 2}, Form{512, 2}, Form{1024, 2}})
        if (n <= f.threads * f.vectors) return f;
    return Form{0, 0};
}

// f(threads to a row, vectors) with both as types.
template <typename F>
dol_status with_form(Form form, F f)
{
    using std::integral_constant;
    const integral_constant<int, 1> one;
    const integral_constant<int, 2> two;
    switch (form.threads) {
    case 4: return f(integral_constant<int, 4>(), one);
    case 8: return f(integral_constant<int, 8>(), one);
    case 16: return f(integral_constant<int, 16>(), one);
    case 32: return f(integral_constant<int, 32>(), one);
    case 64: return form.vectors == 1 ? f(integral_constant<int, 64>(), one) : f(integral_constant<int, 64>(), two);
    case 128: return f(integral_constant<int, 128>(), two);
    case 256: return f(integral_constant<int, 256>(), two);
    case 512: return f(integral_constant<int, 512>(), two);
    default: return f(integral_constant<int, 1024>(), two);
    }
}

// How the rows of a backward pass are dealt out.
struct Plan {
    Form form;
    bool each, whole;                   // a gate for every row; a group takes all rows of its sets
    int64_t sets, points, chunk, chunks, blocks;
    float *part_y, *part_u, *part_gate;
    float2 *row;
    int64_t bytes;
};

Plan plan_of(const dol_matrix *u, const dol_matrix *gate, void *workspace)
{
    Plan p{};
    p.form = form_of(u->cols, u->dtype);
    p.each = gate && gate->rows == u->rows;
    p.sets = gate && !p.each ? gate->rows : 1, p.points = u->rows / p.sets;
    const int groups = p.form.threads && p.form.threads < kThreads ? kThreads / p.form.threads : 1;
    p.whole = p.sets > 1 && p.form.threads && (p.points < kFewPoints || p.sets > kMostBlocks);
    if (p.whole) p.blocks = std::min<int64_t>((p.sets + groups - 1) / groups, 2 * kUnits);
    else {
        const int64_t wanted = std::max<int64_t>(1, 2 * kUnits / p.sets), most = std::max<int64_t>(1, p.points / (4 * groups));
        p.chunks = std::min(wanted, most);
        p.chunk = (p.points + p.chunks - 1) / p.chunks;
        p.chunks = (p.points + p.chunk - 1) / p.chunk;
        p.blocks = p.sets * p.chunks;
    }
    Carver c(workspace);
    p.part_y = c.take<float>(p.blocks * u->cols), p.part_u = c.take<float>(p.blocks * u->cols);
    if (gate && !p.each && !p.whole) p.part_gate = c.take<float>(p.blocks * u->cols);
    if (!p.form.threads) p.row = c.take<float2>(u->rows);
    p.bytes = c.used;
    return p;
}

dol_status check_like(const dol_matrix *m, const dol_matrix *u, const char *name)
{
    if (!m) return DOL_OK;
    if (dol_status s = check_matrix(m, name)) return s;
    if (m->dtype != u->dtype) return fail(DOL_EINVAL, "%s is of another type than u", name);
    if (m->rows != u->rows || m->cols != u->cols) return fail(DOL_ESHAPE, "%s is %d x %d, not %d x %d", name, m->rows, m->cols, u->rows, u->cols);
    return DOL_OK;
}

dol_status check_call(const dol_matrix *u, const dol_matrix *gate)
{
    if (dol_status s = check_matrix(u, "u")) return s;
    if (u->cols < 1) return fail(DOL_ESHAPE, "u has no columns");
    if (u->cols > kMostCols) return fail(DOL_EUNSUPPORTED, "u has %d columns, more than %d", u->cols, kMostCols);
    if (!gate) return DOL_OK;
    if (dol_status s = check_matrix(gate, "gate")) return s;
    if (gate->dtype != u->dtype) return fail(DOL_EINVAL, "gate is of another type than u");
    if (gate->cols != u->cols) return fail(DOL_ESHAPE, "gate has %d columns, u %d", gate->cols, u->cols);
    if (gate->rows < 1 ? u->rows > 0 : u->rows % gate->rows != 0) return fail(DOL_ESHAPE, "%d gates do not divide %d rows", gate->rows, u->rows);
    return DOL_OK;
}

template <typename S>
Mat<const S> in_of(const dol_matrix *m) { return m ? Mat<const S>{static_cast<const S *>(m->data), m->ld} : Mat<const S>{nullptr, 0}; }
template <typename S>
Mat<S> out_of(const dol_matrix *m) { return m ? Mat<S>{static_cast<S *>(m->data), m->ld} : Mat<S>{nullptr, 0}; }

template <typename S>
Args<S> args_of(const dol_matrix *u, int32_t norm_u, const float *gamma_u, const dol_matrix *gate, float scale, const float *gamma_y)
{
    Args<S> a{};
    a.u = in_of<S>(u), a.gate = in_of<S>(gate), a.gamma_u = gamma_u, a.gamma_y = gamma_y;
    a.rows = u->rows, a.cols = u->cols, a.norm_u = norm_u != 0, a.scale = scale, a.per_cols = 1.0f / static_cast<float>(u->cols);
    a.each = gate && gate->rows == u->rows, a.sets = gate && !a.each ? gate->rows : 1, a.points = u->rows / a.sets;
    return a;
}

template <typename S>
dol_status forward(const Args<S> &a, Form form, hipStream_t st)
{
    if (!form.threads) {
        residual_norm_wide_kernel<S><<<static_cast<unsigned>(std::min<int64_t>(a.rows, kMostBlocks)), kWideThreads, 0, st>>>(a);
        DOL_HIP(hipGetLastError());
        return DOL_OK;
    }
    return with_form(form, [&](auto g, auto nv) {
        constexpr int T = std::max<int>(g.value, kThreads), R = T / g.value;
        residual_norm_kernel<S, g.value, nv.value><<<static_cast<unsigned>(std::min<int64_t>((static_cast<int64_t>(a.rows) + R - 1) / R, kMostBlocks)), T, 0, st>>>(a);
        DOL_HIP(hipGetLastError());
        return DOL_OK;
    });
}

template <typename S>
dol_status reverse(const Plan &p, Args<S> a, float *grad_gamma_u, const dol_matrix *grad_gate, float *grad_gamma_y, hipStream_t st)
{
    a.chunk = p.chunk, a.chunks = p.chunks, a.row = p.row, a.grad_gate = out_of<S>(grad_gate);
    a.part_y = grad_gamma_y ? p.part_y : nullptr, a.part_u = grad_gamma_u ? p.part_u : nullptr, a.part_gate = grad_gate ? p.part_gate : nullptr;
    if (p.form.threads) {
        const dol_status s = with_form(p.form, [&](auto g, auto nv) {
            constexpr int T = std::max<int>(g.value, kThreads);
            if (p.whole) residual_norm_backward_kernel<S, g.value, nv.value, true><<<static_cast<unsigned>(p.blocks), T, 0, st>>>(a);
            else residual_norm_backward_kernel<S, g.value, nv.value, false><<<static_cast<unsigned>(p.blocks), T, 0, st>>>(a);
            DOL_HIP(hipGetLastError());
            return DOL_OK;
        });
        if (s) return s;
    } else {
        residual_norm_wide_rows_kernel<S><<<static_cast<unsigned>(std::min<int64_t>(a.rows, kMostBlocks)), kWideThreads, 0, st>>>(a);
        DOL_HIP(hipGetLastError());
        const int stripes = (a.cols + kThreads * kLooseElements<S> - 1) / (kThreads * kLooseElements<S>);
        residual_norm_wide_map_kernel<S><<<static_cast<unsigned>(p.blocks * stripes), kThreads, 0, st>>>(a, stripes);
        DOL_HIP(hipGetLastError());
    }
    const Sums<S> s{a.part_y, a.part_u, a.part_gate, grad_gamma_y, grad_gamma_u, a.grad_gate, p.blocks, p.chunks, a.cols};
    const int64_t jobs = (a.cols + 63) / 64 * ((a.part_y != nullptr) + (a.part_u != nullptr) + (a.part_gate ? p.sets : 0));
    if (jobs == 0) return DOL_OK;
    residual_norm_sums_kernel<S><<<static_cast<unsigned>(std::min(jobs, kMostBlocks)), 1024, 0, st>>>(s, jobs);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

__global__ void __launch_bounds__(kThreads) residual_norm_zero_kernel(float *a, float *b, int32_t n)
{
    const int t = blockIdx.x * kThreads + threadIdx.x;
    if (t >= n) return;
    if (a) a[t] = 0.0f;
    if (b) b[t] = 0.0f;
}

}  // namespace
}  // namespace dol

using namespace dol;

extern "C" {

dol_status dol_residual_norm(const dol_matrix *x, const dol_matrix *u, int32_t norm_u, const float *gamma_u, const dol_matrix *gate, float scale,
                             const float *gamma_y, float eps, const dol_matrix *h, const dol_matrix *y, float *rstd_u, float *rstd_h, void *hip_stream)
{
    if (dol_status s = check_call(u, gate)) return s;
    for (const auto &m : {std::make_pair(x, "x"), std::make_pair(h, "h"), std::make_pair(y, "y")})
        if (dol_status s = check_like(m.first, u, m.second)) return s;
    if (!h && !y) return fail(DOL_EINVAL, "neither h nor y is asked for");
    if (gamma_u && !norm_u) return fail(DOL_EINVAL, "gamma_u without norm_u");
    if (!(eps >= 0.0f)) return fail(DOL_EINVAL, "eps = %g is not a number of at least 0", static_cast<double>(eps));
    if (u->rows == 0) return DOL_OK;
    auto go = [&](auto type) {
        using S = decltype(type);
        Args<S> a = args_of<S>(u, norm_u, gamma_u, gate, scale, gamma_y);
        a.x = in_of<S>(x), a.out_h = out_of<S>(h), a.out_y = out_of<S>(y), a.eps = eps, a.rstd_u = rstd_u, a.rstd_h = rstd_h;
        return forward<S>(a, form_of(u->cols, u->dtype), static_cast<hipStream_t>(hip_stream));
    };
    return u->dtype == DOL_F32 ? go(0.0f) : go(static_cast<__bf16>(0.0f));
}

dol_status dol_residual_norm_workspace(const dol_matrix *u, const dol_matrix *gate, int64_t *bytes)
{
    if (dol_status s = check_call(u, gate)) return s;
    if (!bytes) return fail(DOL_EINVAL, "bytes is NULL");
    *bytes = u->rows ? plan_of(u, gate, nullptr).bytes : 0;
    return DOL_OK;
}

dol_status dol_residual_norm_backward(const dol_matrix *x, const dol_matrix *u, int32_t norm_u, const float *gamma_u, const dol_matrix *gate, float scale,
                                      const float *gamma_y, const float *rstd_u, const float *rstd_h, const dol_matrix *grad_h, const dol_matrix *grad_y,
                                      const dol_matrix *grad_x, const dol_matrix *grad_u, float *grad_gamma_u, const dol_matrix *grad_gate, float *grad_gamma_y,
                                      void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    if (dol_status s = check_call(u, gate)) return s;
    for (const auto &m : {std::make_pair(x, "x"), std::make_pair(grad_h, "grad_h"), std::make_pair(grad_y, "grad_y"), std::make_pair(grad_x, "grad_x"),
                          std::make_pair(grad_u, "grad_u")})
        if (dol_status s = check_like(m.first, u, m.second)) return s;
    if (!grad_x && !grad_u && !grad_gamma_u && !grad_gate && !grad_gamma_y) return fail(DOL_EINVAL, "no gradient is asked for");
    if ((gamma_u || grad_gamma_u) && !norm_u) return fail(DOL_EINVAL, "gamma_u or grad_gamma_u without norm_u");
    if (grad_gate) {
        if (!gate) return fail(DOL_EINVAL, "grad_gate without gate");
        if (dol_status s = check_matrix(grad_gate, "grad_gate")) return s;
        if (grad_gate->dtype != u->dtype) return fail(DOL_EINVAL, "grad_gate is of another type than u");
        if (grad_gate->rows != gate->rows || grad_gate->cols != gate->cols)
            return fail(DOL_ESHAPE, "grad_gate is %d x %d, not %d x %d", grad_gate->rows, grad_gate->cols, gate->rows, gate->cols);
    }
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (u->rows == 0) {                     // sums over nothing
        if (grad_gate && grad_gate->rows > 0) return fail(DOL_ESHAPE, "%d gates for no rows", grad_gate->rows);
        residual_norm_zero_kernel<<<(u->cols + kThreads - 1) / kThreads, kThreads, 0, st>>>(grad_gamma_u, grad_gamma_y, u->cols);
        DOL_HIP(hipGetLastError());
        return DOL_OK;
    }
    if (norm_u && !rstd_u) return fail(DOL_EINVAL, "rstd_u is NULL");
    if (grad_y && !rstd_h) return fail(DOL_EINVAL, "rstd_h is NULL");
    auto go = [&](auto type) {
        using S = decltype(type);
        const Plan p = plan_of(u, gate, workspace);
        if (dol_status s = check_workspace(workspace, workspace_bytes, p.bytes)) return s;
        Args<S> a = args_of<S>(u, norm_u, gamma_u, gate, scale, gamma_y);
        a.x = in_of<S>(x), a.grad_h = in_of<S>(grad_h), a.grad_y = in_of<S>(grad_y), a.grad_x = out_of<S>(grad_x), a.grad_u = out_of<S>(grad_u);
        a.rstd_u = const_cast<float *>(rstd_u), a.rstd_h = const_cast<float *>(rstd_h);
        return reverse<S>(p, a, grad_gamma_u, grad_gate, grad_gamma_y, st);
    };
    return u->dtype == DOL_F32 ? go(0.0f) : go(static_cast<__bf16>(0.0f));
}

}  // extern "C"
