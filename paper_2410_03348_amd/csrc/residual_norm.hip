// Where one block of a network ends and the next begins, and its gradients.  rms(v) = 1 / sqrt(mean of a row's v^2 + eps).
//
//   uhat = u rms(u), v = gamma_u uhat   (or v = u),   h = x + scale gate v,   hhat = h rms(h),   y = gamma_y hhat
//   a = gamma_y dy,   m1 = mean(a hhat),   dh = grad_h + rms(h) (a - hhat m1) = grad_x
//   k = scale gate gamma_u,   m2 = mean(k dh uhat),   grad_u = rms(u) (k dh - uhat m2)   (or scale gate dh)
//   grad_gate = scale sum dh v,   grad_gamma_u = sum scale gate dh uhat,   grad_gamma_y = sum dy hhat   over rows
//
// Memory bounds it: four tensors forward, six backward.  A row lies in the registers of a group of 4 to 1 024 threads, eight columns to
// each, and is read once; memory gives it as fast as some 40 instructions an element take, so that rstd's stay out of all that is done by element.
// Backward one round of sums is enough: with dh put into it and t = gate gamma_u u, the sum of k dh uhat is scale rms(u) times
//   sum t grad_h + rms(h) sum t a - rms(h)^2 m1 sum t h,
// sums that need nothing of each other.  Sums over rows stay in registers while a group goes down its rows; a workgroup leaves one part of
// each, which a second launch adds up in the order of the rows.  Rows too long for that are read twice (wide_*).
#include "internal.h"
#include "loose.h"
#include "wave_util.h"

#include <type_traits>
#include <utility>

namespace dol {
namespace {

constexpr int kEight = 8;               // columns of a thread: one vector of bf16, or two of float
// Columns from one of a thread's vectors to the next in a row of G threads: each load is of neighbouring vectors (of float, whose vectors in a thread
// side by side leave half of every line to the next load: 8 192 x 2 048 forward 73 us, 56 so, backward 95 and 88).
template <typename S, int G>
constexpr int kApart = sizeof(S) == 4 ? 4 * G : 4;
constexpr int kThreads = 256;
constexpr int kWideThreads = 1024;
// Groups of G threads, a row to each, that make a workgroup, forward and backward.
template <int G>
constexpr int kGroups = G < kThreads ? kThreads / G : 1;
// Wavefronts to a SIMD that the forward kernel's registers leave room for, and the workgroups of the chip that are.  More of them than that would be a second
// round of fewer: bf16 8 192 x 4 096 58 us with four to a unit, of which three fit, 52 with three.
template <typename S, int G>
constexpr int kForwardWaves = G == 4 ? 4 : sizeof(S) == 4 || G < 64 ? 5 : G <= 384 ? 7 : G <= 768 ? 6 : 4;
template <typename S, int G>
constexpr int kForwardBlocks = 256 * (kForwardWaves<S, G> * 4 / ((G * kGroups<G> + 63) / 64) > 0 ? kForwardWaves<S, G> * 4 / ((G * kGroups<G> + 63) / 64) : 1);
// Backward fewer workgroups leave fewer parts, but they have to fill a unit.  Both ways, us, four to a unit / two / one: bf16 39 574 x 361 90 / 104 / 134,
// 900 x 20 x 300 with a gate to each sample 42 / 42 / 61, float 31 360 x 32 20 / 20 / 21, bf16 16 384 x 1 000 85 / 77 / 87, 8 192 x 1 500 85 / 73 / 67, 8 192 x 4 096
// 165 / 152 / 143.
constexpr int back_groups(int threads) { return threads == 0 ? 1 : threads <= 64 ? kThreads / threads : threads == 128 ? 4 : 1024 / threads; }
constexpr int back_blocks(int threads) { return threads <= 64 ? 4 : threads == 128 ? 2 : 1; }    // to a unit
template <int G>
constexpr int kBackGroups = back_groups(G);
constexpr int kUnits = 256;             // compute units of the chip
constexpr int kNoRow = -(1 << 20);      // in place of the columns that are left of a row, where there is no row
constexpr int64_t kMostBlocks = 1 << 20;        // of a launch, which has less than 2^32 threads

template <typename S>
struct Mat {
    S *p;
    int64_t ld;
    // (a row's address is the same for the wavefronts of one row; its columns are an offset of 32 bits to it)
    __device__ S *at(int64_t r, int c) const
    {
        using B = std::conditional_t<std::is_const_v<S>, const char, char>;
        return reinterpret_cast<S *>(reinterpret_cast<B *>(p + r * ld) + static_cast<uint32_t>(c) * static_cast<uint32_t>(sizeof(S)));
    }
};

template <typename S>
struct Args {
    Mat<const S> x, u, gate, grad_h, grad_y;
    Mat<S> out_h, out_y, grad_x, grad_u, grad_gate;
    const float *gamma_u, *gamma_y;
    float *rstd_u, *rstd_h;             // written forward, read backward
    int32_t rows, cols, norm_u;
    bool given_h;                       // backward: x is h itself
    int32_t each;                       // a gate for every row; else rows come in `sets` of `points`, a gate (or none) to a set
    int64_t sets, points;
    float scale, eps, per_cols;
    int64_t chunk, chunks;              // backward: rows that a workgroup takes, and how many such a set is
    float *part_y, *part_u, *part_gate; // [workgroups][cols], null where not asked for
    float2 *row;                        // wide: what the sums over each row give
    __device__ int64_t gate_of(int64_t r) const { return each || !gate.p ? r : static_cast<uint32_t>(r) / static_cast<uint32_t>(points); }
};

// A group's number in its workgroup: the same for a whole wavefront where that is one group's, so that rows' addresses are.
template <int G>
__device__ __forceinline__ int group_of()
{
    const int g = threadIdx.x / G;
    return G >= 64 ? __builtin_amdgcn_readfirstlane(g) : g;
}

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
        static_assert(W <= 16 && N <= 4, "a row of 16 lanes to a number");
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        float *mine = red + wave / W * (W * N);
        if (lane == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) mine[n * W + wave % W] = x[n];
        lds_barrier();
        // lanes 16 n .. + 15 add up the n-th (read one after the other they would take a register each)
        const float v = group_sum<16>((lane & 15) < W && (lane >> 4) < N ? mine[(lane >> 4) * W + (lane & 15)] : 0.0f);
#pragma unroll
        for (int n = 0; n < N; ++n) x[n] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 16 * n));
    }
}

// A thread's eight elements as memory has them, vectors D apart.
template <typename S, int D>
struct Eight {
    static constexpr int V = kLooseElements<S>, H = kEight / V, kSpan = (H - 1) * D + V;
    static constexpr int column(int e) { return e / V * D + e % V; }
    Loose<S> v[H];
    // The row's, of at least a vector, from column c on; where a vector is not all there the row's last one, so that all threads load at once, and cut() does
    // the rest (behind a branch for those threads each load is waited for by itself: bf16 39 574 x 361 both ways 90 us, 110 so).
    __device__ void all(const Mat<const S> &m, int64_t r, int c, int cols)
    {
#pragma unroll
        for (int h = 0; h < H; ++h) v[h] = *reinterpret_cast<const Loose<S> *>(m.at(r, min(c + h * D, cols - V)));
    }
    __device__ void cut(int n)
    {
#pragma unroll
        for (int h = 0; h < H; ++h) {
            if (n - h * D < V) v[h] = loose_from(v[h], V - (n - h * D));
            __builtin_amdgcn_sched_barrier(0);      // (one vector's numbers in registers at a time)
        }
    }
    // those of them that are in the n columns from column c on, zeros behind
    __device__ void some(const S *p, int n, int c)
    {
#pragma unroll
        for (int h = 0; h < H; ++h) v[h] = loose_load_end(p + h * D, n - h * D, c + h * D);
    }
    // `other` in all of them, where there is no tensor (and what was loaded for it is another's)
    __device__ void only(bool given, float other)
    {
        const uint32_t bits = __float_as_uint(other), w = sizeof(S) == 4 ? bits : bits >> 16 | (bits & 0xFFFF0000u);
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[h].w[k] = given ? v[h].w[k] : w;
    }
    __device__ float get(int e) const { return loose_get(v[e / V], e % V); }
    // elements 2 k and 2 k + 1
    __device__ void set(int k, float x0, float x1)
    {
        if constexpr (sizeof(S) == 4) v[k / 2].w[k % 2 * 2] = __float_as_uint(x0), v[k / 2].w[k % 2 * 2 + 1] = __float_as_uint(x1);
        else v[0].w[k] = __builtin_bit_cast(uint16_t, static_cast<S>(x0)) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<S>(x1))) << 16;
    }
    __device__ void store(S *p, int n) const
    {
#pragma unroll
        for (int h = 0; h < H; ++h) loose_store(p + h * D, v[h], n - h * D);
    }
    // Nothing that was computed of it before is kept for what comes after: unpacked it would take two to four times its registers.
    __device__ void again()
    {
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t w = v[h].w[k];
                asm("" : "+v"(w));
                v[h].w[k] = w;
            }
    }
};

template <int D, typename S>
__device__ __forceinline__ void put(S *p, const float (&x)[kEight], int n)
{
    constexpr int V = kLooseElements<S>;
#pragma unroll
    for (int h = 0; h < kEight / V; ++h) {
        float part[V];
#pragma unroll
        for (int e = 0; e < V; ++e) part[e] = x[h * V + e];
        Loose<S> v;
        loose_set(v, part);
        loose_store(p + h * D, v, n - h * D);
    }
}

// Factors of eight columns, 1 where there are none.
template <int D>
__device__ __forceinline__ void factors(float (&x)[kEight], const float *p, int n, int c)
{
#pragma unroll
    for (int e = 0; e < kEight; ++e) x[e] = 1.0f;
    if (!p) return;
    Eight<float, D> v;
    v.some(p + c, n, c);
#pragma unroll
    for (int e = 0; e < kEight; ++e) x[e] = v.get(e);
}

__device__ __forceinline__ float rms(float squares, float per_cols, float eps) { return 1.0f / __builtin_amdgcn_sqrtf(__builtin_fmaf(squares, per_cols, eps)); }

// Both factors of a thread's eight columns, in registers, or (G threads to a row) in LDS: beside three sums over rows and a row of five tensors there are
// no registers left for them.
template <int D>
struct InRegisters {
    float u[kEight], y[kEight];
    template <typename S>
    __device__ InRegisters(const Args<S> &a, int c, int n, void *)
    {
        factors<D>(u, a.gamma_u, n, c);
        factors<D>(y, a.gamma_y, n, c);
    }
    __device__ void get(int k, float (&gu)[2], float (&gy)[2]) const { gu[0] = u[2 * k], gu[1] = u[2 * k + 1], gy[0] = y[2 * k], gy[1] = y[2 * k + 1]; }
};

template <int G, int D>
struct InLds {
    struct alignas(16) Pair { float u[2], y[2]; };
    const Pair *at;             // [4][G]: a wavefront's reads are next to each other
    template <typename S>
    __device__ InLds(const Args<S> &a, int c, int n, void *lds) : at(static_cast<const Pair *>(lds) + c / kLooseElements<S>)
    {
        float u[kEight], y[kEight];
        factors<D>(u, a.gamma_u, n, c);
        factors<D>(y, a.gamma_y, n, c);
        // (the groups of a workgroup write the same)
#pragma unroll
        for (int k = 0; k < kEight / 2; ++k) static_cast<Pair *>(lds)[k * G + c / kLooseElements<S>] = Pair{{u[2 * k], u[2 * k + 1]}, {y[2 * k], y[2 * k + 1]}};
        lds_barrier();
    }
    __device__ void get(int k, float (&gu)[2], float (&gy)[2]) const
    {
        const Pair p = at[k * G];
        gu[0] = p.u[0], gu[1] = p.u[1], gy[0] = p.y[0], gy[1] = p.y[1];
    }
};

template <int G>
constexpr int kGammaLds = G >= 64 ? 2 * G * kEight * 4 : 0;

// What a row's eight columns are read for; FEW: a row may have less than a vector.
template <typename S, int D, bool FEW>
struct Columns {
    Eight<S, D> x, u, gate;
    // n columns of row r of x and u, and g of gate, from c on.  (One branch for all of them, and none for a tensor that is not there: a load behind a branch of its
    // own is waited for at its end.)
    __device__ void load(const Args<S> &a, int64_t r, int64_t g, int c, int n)
    {
        const Mat<const S> mx = a.x.p ? a.x : a.u, mg = a.gate.p ? a.gate : a.u;
        if (!a.gate.p) g = r;
        if (FEW && a.cols < Eight<S, D>::V) x.some(mx.at(r, c), n, c), u.some(a.u.at(r, c), n, c), gate.some(mg.at(g, c), n, c);
        else if (n != kNoRow) x.all(mx, r, c, a.cols), u.all(a.u, r, c, a.cols), gate.all(mg, g, c, a.cols);
    }
    // Before they are used, as late as can be: nothing of it is done before the loads are there.
    __device__ void ready(const Args<S> &a, int n)
    {
        if ((!FEW || a.cols >= Eight<S, D>::V) && n < Eight<S, D>::kSpan) x.cut(n), u.cut(n), gate.cut(n);
        x.only(a.x.p, 0.0f), gate.only(a.gate.p, 1.0f);
    }
    // gate gamma_u u of column e, and h, of which it is scale rstd_u
    __device__ float part(int e, float gamma_u) const { return gate.get(e) * (gamma_u * u.get(e)); }
    __device__ float stream(int e, float gamma_u, float f) const { return __builtin_fmaf(f, part(e, gamma_u), x.get(e)); }
};

// ---------------------------------------------------------------- forward

// Bytes bound it: bf16 8 192 x 4 096, a gate to 1 024 rows, 48 us, 5.6 TB/s.
template <typename S, int G>
__global__ void __launch_bounds__(G * kGroups<G>, (kForwardWaves<S, G>)) residual_norm_kernel(Args<S> a)
{
    constexpr int R = kGroups<G>, D = kApart<S, G>;
    __shared__ float red[2][(G * R + 63) / 64];
    const int lane = threadIdx.x % G, group = group_of<G>(), c = lane * kLooseElements<S>;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * R;
    float gamma_u[kEight], gamma_y[kEight];
    factors<D>(gamma_u, a.gamma_u, a.cols - c, c);
    factors<D>(gamma_y, a.gamma_y, a.cols - c, c);
    Columns<S, D, (G == 4)> q;
    auto fetch = [&](int64_t r) { q.load(a, r, r < a.rows ? a.gate_of(r) : 0, c, r < a.rows ? a.cols - c : kNoRow); };
    fetch(static_cast<int64_t>(blockIdx.x) * R + group);
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * R; first < a.rows; first += stride) {
        const int64_t r = first + group;
        const bool in = r < a.rows;
        const int n = in ? a.cols - c : kNoRow;
        float h[kEight], s[1] = {0.0f}, rstd = 1.0f;
        Columns<S, D, (G == 4)> p = q;
        fetch(r + stride);
        p.ready(a, n);
        if (a.norm_u) {
#pragma unroll
            for (int e = 0; e < kEight; ++e) s[0] = __builtin_fmaf(p.u.get(e), p.u.get(e), s[0]);
            group_sums<G, 1>(s, red[0]);
            rstd = rms(s[0], a.per_cols, a.eps);
            if (a.rstd_u && in && lane == 0) a.rstd_u[r] = rstd;
            s[0] = 0.0f;
        }
        const float f = a.scale * rstd;
#pragma unroll
        for (int e = 0; e < kEight; ++e) {
            h[e] = p.stream(e, gamma_u[e], f);
            s[0] = __builtin_fmaf(h[e], h[e], s[0]);
        }
        if (a.out_h.p && n > 0) put<D>(a.out_h.at(r, c), h, n);
        if (a.out_y.p) {
            group_sums<G, 1>(s, red[1]);
            rstd = rms(s[0], a.per_cols, a.eps);
            if (a.rstd_h && in && lane == 0) a.rstd_h[r] = rstd;
#pragma unroll
            for (int e = 0; e < kEight; ++e) h[e] = h[e] * rstd * gamma_y[e];
            if (n > 0) put<D>(a.out_y.at(r, c), h, n);
        }
        if constexpr (G > 64) lds_barrier();            // (red is written again)
    }
}

// ---------------------------------------------------------------- backward

// Eight columns of a row.  h is made again from x and u: as it was rounded to bf16 it would be off by 2^-9 in every term of grad_gamma_y.  Where the caller has only
// h (given_h), that is what x holds, and nothing of u goes into it.
template <typename S, int D, bool FEW>
struct Piece {
    Columns<S, D, FEW> p;
    Eight<S, D> gy, gh;
    __device__ void load(const Args<S> &a, int64_t r, int64_t g, int c, int n)
    {
        const Mat<const S> mx = a.x.p ? a.x : a.u, mg = a.gate.p ? a.gate : a.u, my = a.grad_y.p ? a.grad_y : a.u, mh = a.grad_h.p ? a.grad_h : a.u;
        if (!a.gate.p) g = r;
        if (FEW && a.cols < Eight<S, D>::V)
            p.x.some(mx.at(r, c), n, c), p.u.some(a.u.at(r, c), n, c), p.gate.some(mg.at(g, c), n, c), gy.some(my.at(r, c), n, c), gh.some(mh.at(r, c), n, c);
        else
            p.x.all(mx, r, c, a.cols), p.u.all(a.u, r, c, a.cols), p.gate.all(mg, g, c, a.cols), gy.all(my, r, c, a.cols), gh.all(mh, r, c, a.cols);
        p.ready(a, n);
        if ((!FEW || a.cols >= Eight<S, D>::V) && n < Eight<S, D>::kSpan) gy.cut(n), gh.cut(n);
        gy.only(a.grad_y.p, 0.0f), gh.only(a.grad_h.p, 0.0f);
    }
    __device__ void again() { p.x.again(), p.u.again(), p.gate.again(), gy.again(), gh.again(); }
    // What a row is multiplied with; sums() adds up four products of eight columns, which with rstd's left out of them are two instructions each.
    struct Factors {
        float f, rstd_h;                        // scale rstd_u
        float in_h;                             // f, or 0 where h is given: what the block's part is in h
        float kh, kv;                           // after the sums, of hhat and of v = scale uhat: rstd_h m1, and rstd_u m2 / scale
        __device__ Factors(const Args<S> &a, float rstd_u, float rstd) : f(a.scale * rstd_u), rstd_h(rstd), in_h(a.given_h ? 0.0f : f), kh(0.0f), kv(0.0f) {}
        __device__ void join(const float (&s)[4], bool norm_u, float rstd_u, float per_cols)
        {
            kh = rstd_h * (rstd_h * (s[0] * per_cols));
            // (a sum before the rstd that its numbers go with: rstd's by themselves multiply out of a float's range long before any square does)
            kv = norm_u ? rstd_u * (rstd_u * (per_cols * __builtin_fmaf(rstd_h, s[2], __builtin_fmaf(-kh, rstd_h * s[3], s[1])))) : 0.0f;
        }
    };
    template <typename F>
    __device__ void sums(float (&s)[4], const F &gamma, const Factors &m) const
    {
#pragma unroll
        for (int k = 0; k < kEight / 2; ++k) {
            float gamma_u[2], gamma_y[2];
            gamma.get(k, gamma_u, gamma_y);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int e = 2 * k + q;
                const float t = p.part(e, gamma_u[q]), h = __builtin_fmaf(m.in_h, t, p.x.get(e)), ay = gamma_y[q] * gy.get(e);
                s[0] = __builtin_fmaf(ay, h, s[0]);
                s[1] = __builtin_fmaf(t, gh.get(e), s[1]);
                s[2] = __builtin_fmaf(t, ay, s[2]);
                s[3] = __builtin_fmaf(t, h, s[3]);
            }
            __builtin_amdgcn_sched_barrier(0);      // (two columns' numbers in registers, not eight)
        }
    }
    // sum_y and sum_t add up dy hhat and scale dh uhat (times the gate, where each row has its own).
    template <typename F>
    __device__ void leave(const Args<S> &a, int64_t r, int c, int n, const F &gamma, const Factors &m, float (&sum_y)[kEight], float (&sum_t)[kEight]) const
    {
        Eight<S, D> ox, ou, og;
#pragma unroll
        for (int k = 0; k < kEight / 2; ++k) {
            float dh[2], du[2], dg[2], gamma_u[2], gamma_y[2];
            gamma.get(k, gamma_u, gamma_y);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int e = 2 * k + q;
                const float u = p.u.get(e), gate = p.gate.get(e), h = p.stream(e, gamma_u[q], m.in_h), g = gy.get(e);
                const float hhat = h * m.rstd_h;
                dh[q] = __builtin_fmaf(m.rstd_h, gamma_y[q] * g, __builtin_fmaf(-m.kh, hhat, gh.get(e)));
                const float dv = gate * dh[q], v = m.f * u;
                du[q] = __builtin_fmaf(m.f, gamma_u[q] * dv, -(m.kv * v));
                dg[q] = gamma_u[q] * (dh[q] * v);
                sum_y[e] = __builtin_fmaf(g, hhat, sum_y[e]);
                sum_t[e] = __builtin_fmaf(a.each ? dv : dh[q], v, sum_t[e]);
            }
            ox.set(k, dh[0], dh[1]), ou.set(k, du[0], du[1]), og.set(k, dg[0], dg[1]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (n <= 0) return;
        if (a.grad_x.p) ox.store(a.grad_x.at(r, c), n);
        if (a.grad_u.p) ou.store(a.grad_u.at(r, c), n);
        if (a.each && a.grad_gate.p) og.store(a.grad_gate.at(r, c), n);
    }
};

// Of a set's sums of scale dh uhat: grad_gate's, times gamma_u, and grad_gamma_u's, times the gate (which a row of its own has multiplied already).
template <int D, typename S, typename F>
__device__ __forceinline__ void spread_sums(const Args<S> &a, int64_t set, int c, const F &gamma, const float (&sum_t)[kEight], float (&to_gate)[kEight], float (&to_u)[kEight])
{
    Eight<S, D> gate{};
    const bool given = a.gate.p && !a.each;
    if (given) gate.some(a.gate.at(set, c), a.cols - c, c);
#pragma unroll
    for (int k = 0; k < kEight / 2; ++k) {
        float gamma_u[2], gamma_y[2];
        gamma.get(k, gamma_u, gamma_y);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int e = 2 * k + q;
            to_gate[e] = gamma_u[q] * sum_t[e], to_u[e] = given ? gate.get(e) * sum_t[e] : sum_t[e];
        }
    }
}

// The sums of a workgroup's groups over their rows, in the order of the groups, to to[c].
template <typename S, int G, int R, typename O>
__device__ __forceinline__ void leave_part(const float (&sum)[kEight], O *to, int cols, float *buf)
{
    using E = Eight<S, kApart<S, G>>;
    const int first = threadIdx.x % G * E::V, group = threadIdx.x / G;
    if constexpr (R == 1) {
#pragma unroll
        for (int e = 0; e < kEight; ++e)
            if (first + E::column(e) < cols) to[first + E::column(e)] = static_cast<O>(sum[e]);
    } else {
        lds_barrier();
#pragma unroll
        for (int e = 0; e < kEight; ++e) buf[group * G * kEight + first + E::column(e)] = sum[e];
        lds_barrier();
        for (int c = threadIdx.x; c < cols; c += R * G) {
            float s = 0.0f;
            for (int g = 0; g < R; ++g) s += buf[g * G * kEight + c];
            to[c] = static_cast<O>(s);
        }
    }
}

// WHOLE: a group takes all rows of its sets; else a workgroup takes a chunk of the rows of one set.
// Bytes bound it: bf16 8 192 x 4 096, a gate to 1 024 rows, 92 us, 4.4 TB/s.  (With the next row asked for ahead, as forward, it had registers for one row on a
// unit at a time instead of two: 116 us, 99 at that time without.)
template <typename S, int G, bool WHOLE>
__global__ void __launch_bounds__(G * kBackGroups<G>, G < 64 ? 2 : 4) residual_norm_backward_kernel(Args<S> a)
{
    constexpr int R = kBackGroups<G>, D = kApart<S, G>;
    __shared__ float red[2][4 * ((G * R + 63) / 64)];
    __shared__ float buf[R > 1 ? G * R * kEight : 1];
    const int lane = threadIdx.x % G, group = group_of<G>(), c = lane * kLooseElements<S>;
    // rows of this group: `count` of each of `turns` sets (WHOLE), or `count` of the chunk, R apart
    const int64_t set = WHOLE ? 0 : blockIdx.x / static_cast<unsigned>(a.chunks);
    const int64_t r0 = WHOLE ? 0 : set * a.points + (blockIdx.x - set * a.chunks) * a.chunk, r1 = WHOLE ? 0 : min(r0 + a.chunk, (set + 1) * a.points);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * R, mine = static_cast<int64_t>(blockIdx.x) * R + group;
    const int64_t turns = WHOLE ? (a.sets + stride - 1) / stride : 1, count = WHOLE ? a.points : (r1 - r0 + R - 1) / R;
    extern __shared__ __align__(16) char gammas[];
    const std::conditional_t<(kGammaLds<G> > 0), InLds<G, D>, InRegisters<D>> gamma(a, c, a.cols - c, gammas);
    float sum_y[kEight], sum_t[kEight], sum_u[kEight], gates[kEight];
#pragma unroll
    for (int e = 0; e < kEight; ++e) sum_y[e] = sum_t[e] = sum_u[e] = 0.0f;
    struct Row {
        Piece<S, D, (G == 4)> p;
        int64_t r;
        int n;
        float rstd_u, rstd_h;
    };
    auto fetch = [&](Row &q, int64_t t, int64_t k) {
        const int64_t m = mine + t * stride;
        const bool in = WHOLE ? m < a.sets : r0 + k * R + group < r1;       // (else row 0 is read, and none of it kept)
        q.r = !in ? 0 : WHOLE ? m * a.points + k : r0 + k * R + group;
        q.n = in ? a.cols - c : kNoRow;
        q.p.load(a, q.r, WHOLE ? in ? m : 0 : a.each ? q.r : set, c, q.n);
        q.rstd_u = a.norm_u && in ? a.rstd_u[q.r] : 1.0f, q.rstd_h = a.grad_y.p && in ? a.rstd_h[q.r] : 0.0f;
    };
    int turn = 0;
    for (int64_t t = 0; t < turns; ++t) {
        for (int64_t k = 0; k < count; ++k) {
            Row now;
            fetch(now, t, k);
            typename Piece<S, D, (G == 4)>::Factors m(a, now.rstd_u, now.rstd_h);
            float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            now.p.sums(s, gamma, m);
            group_sums<G, 4>(s, red[turn]);
            turn ^= 1;
            m.join(s, a.norm_u, now.rstd_u, a.per_cols);
            now.p.again();
            now.p.leave(a, now.r, c, now.n, gamma, m, sum_y, sum_t);
        }
        if constexpr (WHOLE) {
            const int64_t m = mine + t * stride;
            if (m < a.sets) {
                float to_u[kEight];
                spread_sums<D>(a, m, c, gamma, sum_t, gates, to_u);
                if (a.grad_gate.p && c < a.cols) put<D>(a.grad_gate.at(m, c), gates, a.cols - c);
#pragma unroll
                for (int e = 0; e < kEight; ++e) sum_u[e] += to_u[e], sum_t[e] = 0.0f;
            }
        }
    }
    if constexpr (!WHOLE) spread_sums<D>(a, set, c, gamma, sum_t, gates, sum_u);
    const int64_t at = static_cast<int64_t>(blockIdx.x) * a.cols;
    if (a.part_y) leave_part<S, G, R>(sum_y, a.part_y + at, a.cols, buf);
    if (a.part_u) leave_part<S, G, R>(sum_u, a.part_u + at, a.cols, buf);
    if (WHOLE || a.each || !a.grad_gate.p) return;
    if (a.part_gate) leave_part<S, G, R>(gates, a.part_gate + at, a.cols, buf);
    else leave_part<S, G, R>(gates, a.grad_gate.at(set, 0), a.cols, buf);             // (a set is one chunk)
}

// ---------------------------------------------------------------- wide rows

// A workgroup to a row, which it goes through three times; all is written in the last one, since h and y may lie on x and u.
template <typename S>
__global__ void __launch_bounds__(kWideThreads) residual_norm_wide_kernel(Args<S> a)
{
    constexpr int D = kApart<S, kWideThreads>, V = kLooseElements<S>;
    __shared__ float red[2][kWideThreads / 64];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const int64_t g = a.gate_of(r);
        float rstd_u = 1.0f, rstd_h = 0.0f, s[1] = {0.0f};
        auto stream = [&](int c, int n, float (&h)[kEight]) {
            Columns<S, D, false> p;
            float gamma_u[kEight];
            p.load(a, r, g, c, n);
            p.ready(a, n);
            factors<D>(gamma_u, a.gamma_u, n, c);
#pragma unroll
            for (int e = 0; e < kEight; ++e) h[e] = p.stream(e, gamma_u[e], a.scale * rstd_u);
        };
        if (a.norm_u) {
            for (int c = threadIdx.x * V; c < a.cols; c += kWideThreads * kEight) {
                Eight<S, D> u;
                u.some(a.u.at(r, c), a.cols - c, c);
#pragma unroll
                for (int e = 0; e < kEight; ++e) s[0] = __builtin_fmaf(u.get(e), u.get(e), s[0]);
            }
            group_sums<kWideThreads, 1>(s, red[0]);
            rstd_u = rms(s[0], a.per_cols, a.eps);
            s[0] = 0.0f;
        }
        if (a.out_y.p) {
            for (int c = threadIdx.x * V; c < a.cols; c += kWideThreads * kEight) {
                float h[kEight];
                stream(c, a.cols - c, h);
#pragma unroll
                for (int e = 0; e < kEight; ++e) s[0] = __builtin_fmaf(h[e], h[e], s[0]);
            }
            group_sums<kWideThreads, 1>(s, red[1]);
            rstd_h = rms(s[0], a.per_cols, a.eps);
        }
        if (threadIdx.x == 0) {
            if (a.norm_u && a.rstd_u) a.rstd_u[r] = rstd_u;
            if (a.out_y.p && a.rstd_h) a.rstd_h[r] = rstd_h;
        }
        for (int c = threadIdx.x * V; c < a.cols; c += kWideThreads * kEight) {
            const int n = a.cols - c;
            float h[kEight], gamma_y[kEight];
            stream(c, n, h);
            if (a.out_h.p) put<D>(a.out_h.at(r, c), h, n);
            if (!a.out_y.p) continue;
            factors<D>(gamma_y, a.gamma_y, n, c);
#pragma unroll
            for (int e = 0; e < kEight; ++e) h[e] = h[e] * rstd_h * gamma_y[e];
            put<D>(a.out_y.at(r, c), h, n);
        }
        lds_barrier();          // (red is written again)
    }
}

// What a row's sums give (Factors) for each row.
template <typename S>
__global__ void __launch_bounds__(kWideThreads) residual_norm_wide_rows_kernel(Args<S> a)
{
    constexpr int D = kApart<S, kWideThreads>, V = kLooseElements<S>;
    __shared__ float red[4 * (kWideThreads / 64)];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const int64_t g = a.gate_of(r);
        const float rstd_u = a.norm_u ? a.rstd_u[r] : 1.0f, rstd_h = a.grad_y.p ? a.rstd_h[r] : 0.0f;
        typename Piece<S, D, false>::Factors m(a, rstd_u, rstd_h);
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int c = threadIdx.x * V; c < a.cols; c += kWideThreads * kEight) {
            const int n = a.cols - c;
            Piece<S, D, false> p;
            p.load(a, r, g, c, n);
            p.sums(s, InRegisters<D>(a, c, n, nullptr), m);
        }
        group_sums<kWideThreads, 4>(s, red);
        m.join(s, a.norm_u, rstd_u, a.per_cols);
        if (threadIdx.x == 0) a.row[r] = make_float2(m.kh, m.kv);
        lds_barrier();
    }
}

// A workgroup takes eight columns a thread of a chunk of one set's rows.
template <typename S>
__global__ void __launch_bounds__(kThreads) residual_norm_wide_map_kernel(Args<S> a, int stripes)
{
    constexpr int D = kApart<S, kThreads>;
    const int64_t block = blockIdx.x / stripes, set = block / a.chunks, r0 = set * a.points + block % a.chunks * a.chunk, r1 = min(r0 + a.chunk, (set + 1) * a.points);
    const int c = static_cast<int>(blockIdx.x % stripes) * (kThreads * kEight) + threadIdx.x * kLooseElements<S>, n = a.cols - c;
    if (n <= 0) return;
    const InRegisters<D> gamma(a, c, n, nullptr);
    float sum_y[kEight], sum_t[kEight], sum_u[kEight], gates[kEight];
#pragma unroll
    for (int e = 0; e < kEight; ++e) sum_y[e] = sum_t[e] = 0.0f;
    for (int64_t r = r0; r < r1; ++r) {
        const float rstd_u = a.norm_u ? a.rstd_u[r] : 1.0f, rstd_h = a.grad_y.p ? a.rstd_h[r] : 0.0f;
        typename Piece<S, D, false>::Factors m(a, rstd_u, rstd_h);
        m.kh = a.row[r].x, m.kv = a.row[r].y;
        Piece<S, D, false> p;
        p.load(a, r, a.each ? r : set, c, n);
        p.leave(a, r, c, n, gamma, m, sum_y, sum_t);
    }
    spread_sums<D>(a, set, c, gamma, sum_t, gates, sum_u);
    const int64_t at = block * a.cols + c;
#pragma unroll
    for (int e = 0; e < kEight; ++e) {
        const int k = Eight<S, D>::column(e);
        if (k >= n) break;
        if (a.part_y) a.part_y[at + k] = sum_y[e];
        if (a.part_u) a.part_u[at + k] = sum_u[e];
        if (a.part_gate) a.part_gate[at + k] = gates[e];
        else if (!a.each && a.grad_gate.p) *a.grad_gate.at(set, c + k) = static_cast<S>(gates[e]);         // (a set is one chunk)
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

// 64 columns by 16 shares of the parts to a workgroup; a share's parts lie 16 apart.  Gates of few parts are a wavefront's each, behind those.
template <typename S>
__global__ void __launch_bounds__(1024) residual_norm_sums_kernel(Sums<S> s, int64_t shared, int64_t alone)
{
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t wide = (s.cols + 63) / 64;
    for (int64_t j = blockIdx.x; j < shared + (alone + 15) / 16; j += gridDim.x) {
        if (j >= shared) {
            const int64_t q = (j - shared) * 16 + wave, g = q / wide;
            const int c = static_cast<int>(q % wide) * 64 + lane;
            if (q >= alone || c >= s.cols) continue;
            float v = 0.0f;
#pragma unroll 4
            for (int64_t k = 0; k < s.per_gate; ++k) v += s.part_gate[(g * s.per_gate + k) * s.cols + c];
            *s.grad_gate.at(g, c) = static_cast<S>(v);
            continue;
        }
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

// Threads to a row, eight columns to each; 0: a row too long for registers.
int threads_of(int32_t cols)
{
    const int n = (cols + kEight - 1) / kEight;
    for (int g : {4, 8, 16, 32, 64, 128, 192, 256, 384, 512, 768, 1024})
        if (n <= g) return g;
    return 0;
}

// f(threads to a row) with them as a type.
template <typename F>
dol_status with_threads(int threads, F f)
{
    using std::integral_constant;
    switch (threads) {
    case 4: return f(integral_constant<int, 4>());
    case 8: return f(integral_constant<int, 8>());
    case 16: return f(integral_constant<int, 16>());
    case 32: return f(integral_constant<int, 32>());
    case 64: return f(integral_constant<int, 64>());
    case 128: return f(integral_constant<int, 128>());
    case 192: return f(integral_constant<int, 192>());
    case 256: return f(integral_constant<int, 256>());
    case 384: return f(integral_constant<int, 384>());
    case 512: return f(integral_constant<int, 512>());
    case 768: return f(integral_constant<int, 768>());
    default: return f(integral_constant<int, 1024>());
    }
}

// Workgroups side by side of residual_norm_wide_map_kernel.
int stripes_of(int32_t cols) { return (cols + kThreads * kEight - 1) / (kThreads * kEight); }

// How the rows of a backward pass are dealt out.
struct Plan {
    int threads;                        // to a row
    bool each, whole;                   // a gate for every row; a group takes all rows of its sets
    int64_t sets, points, chunk, chunks, blocks;
    float *part_y, *part_u, *part_gate;
    float2 *row;
    int64_t bytes;
};

Plan plan_of(const dol_matrix *u, const dol_matrix *gate, void *workspace)
{
    Plan p{};
    p.threads = threads_of(u->cols);
    p.each = gate && gate->rows == u->rows;
    p.sets = gate && !p.each ? gate->rows : 1, p.points = u->rows / p.sets;
    const int groups = back_groups(p.threads);
    // (rows too long for registers: as many of kThreads as lie side by side)
    const int64_t most_blocks = p.threads ? back_blocks(p.threads) * kUnits : std::max(1, 4 * kUnits / stripes_of(u->cols));
    // As chunks of a set's rows to workgroups, or as whole sets to groups: what takes fewer rows in a row, where leaving a chunk's parts takes as long as three
    // rows.  Both ways, us, chunks / whole: bf16 900 x 20 x 300 42 / 61, 2 000 x 30 x 300 119 / 131, 4 000 x 10 x 1 024 217 / 182, 8 000 x 40 x 96 193 / 167,
    // 100 000 x 3 x 16 1 127 / 50, float 3 000 x 3 x 2 048 239 / 172, 128 x 50 x 7 463 425 / 564.
    const int64_t wanted = std::max<int64_t>(1, most_blocks / p.sets), most = std::max<int64_t>(1, p.points / groups);
    p.chunks = std::min(wanted, most);
    p.chunk = (p.points + p.chunks - 1) / p.chunks;
    p.chunks = (p.points + p.chunk - 1) / p.chunk;
    p.blocks = p.sets * p.chunks;
    const int64_t by_chunk = (p.blocks + most_blocks - 1) / most_blocks * ((p.chunk + groups - 1) / groups + 3);
    const int64_t by_set = (p.sets + most_blocks * groups - 1) / (most_blocks * groups) * p.points;
    p.whole = p.sets > 1 && p.threads && (by_set < by_chunk || p.blocks > kMostBlocks);
    if (p.whole) p.blocks = std::min<int64_t>((p.sets + groups - 1) / groups, most_blocks);
    Carver c(workspace);
    p.part_y = c.take<float>(p.blocks * u->cols), p.part_u = c.take<float>(p.blocks * u->cols);
    if (gate && !p.each && !p.whole && p.chunks > 1) p.part_gate = c.take<float>(p.blocks * u->cols);
    if (!p.threads) p.row = c.take<float2>(u->rows);
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
dol_status forward(const Args<S> &a, int threads, hipStream_t st)
{
    if (!threads) {
        residual_norm_wide_kernel<S><<<static_cast<unsigned>(std::min<int64_t>(a.rows, kMostBlocks)), kWideThreads, 0, st>>>(a);
        DOL_HIP(hipGetLastError());
        return DOL_OK;
    }
    return with_threads(threads, [&](auto g) {
        constexpr int G = g.value, R = kGroups<G>;
        residual_norm_kernel<S, G><<<static_cast<unsigned>(std::min<int64_t>((static_cast<int64_t>(a.rows) + R - 1) / R, kForwardBlocks<S, G>)), G * R, 0, st>>>(a);
        DOL_HIP(hipGetLastError());
        return DOL_OK;
    });
}

template <typename S>
dol_status reverse(const Plan &p, Args<S> a, float *grad_gamma_u, const dol_matrix *grad_gate, float *grad_gamma_y, hipStream_t st)
{
    a.chunk = p.chunk, a.chunks = p.chunks, a.row = p.row, a.grad_gate = out_of<S>(grad_gate);
    a.part_y = grad_gamma_y ? p.part_y : nullptr, a.part_u = grad_gamma_u ? p.part_u : nullptr, a.part_gate = grad_gate ? p.part_gate : nullptr;
    if (p.threads) {
        const dol_status s = with_threads(p.threads, [&](auto g) {
            constexpr int G = g.value, T = G * kBackGroups<G>, LDS = kGammaLds<G>;
            const auto kernel = p.whole ? residual_norm_backward_kernel<S, G, true> : residual_norm_backward_kernel<S, G, false>;
            if (LDS >= 32 * 1024) DOL_HIP(allow_dynamic_lds(reinterpret_cast<const void *>(kernel), LDS));
            kernel<<<static_cast<unsigned>(p.blocks), T, LDS, st>>>(a);
            DOL_HIP(hipGetLastError());
            return DOL_OK;
        });
        if (s) return s;
    } else {
        residual_norm_wide_rows_kernel<S><<<static_cast<unsigned>(std::min<int64_t>(a.rows, kMostBlocks)), kWideThreads, 0, st>>>(a);
        DOL_HIP(hipGetLastError());
        const int stripes = stripes_of(a.cols);
        residual_norm_wide_map_kernel<S><<<static_cast<unsigned>(p.blocks * stripes), kThreads, 0, st>>>(a, stripes);
        DOL_HIP(hipGetLastError());
    }
    const Sums<S> s{a.part_y, a.part_u, a.part_gate, grad_gamma_y, grad_gamma_u, a.grad_gate, p.blocks, p.chunks, a.cols};
    const int64_t wide = (a.cols + 63) / 64, gates = a.part_gate ? p.sets : 0;
    const bool few = p.chunks < 64;         // parts of a gate
    const int64_t shared = wide * ((a.part_y != nullptr) + (a.part_u != nullptr) + (few ? 0 : gates)), alone = few ? wide * gates : 0, jobs = shared + (alone + 15) / 16;
    if (jobs == 0) return DOL_OK;
    residual_norm_sums_kernel<S><<<static_cast<unsigned>(std::min(jobs, kMostBlocks)), 1024, 0, st>>>(s, shared, alone);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

// Sums over no rows.
template <typename S>
__global__ void __launch_bounds__(kThreads) residual_norm_zero_kernel(float *a, float *b, Mat<S> gates, int64_t count, int32_t n)
{
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (t < n) {
        if (a) a[t] = 0.0f;
        if (b) b[t] = 0.0f;
    }
    for (int64_t k = t; k < count * n; k += static_cast<int64_t>(gridDim.x) * kThreads) *gates.at(k / n, static_cast<int>(k % n)) = static_cast<S>(0.0f);
}

dol_status backward(bool given_h, const dol_matrix *x, const dol_matrix *u, int32_t norm_u, const float *gamma_u, const dol_matrix *gate, float scale,
                    const float *gamma_y, const float *rstd_u, const float *rstd_h, const dol_matrix *grad_h, const dol_matrix *grad_y,
                    const dol_matrix *grad_x, const dol_matrix *grad_u, float *grad_gamma_u, const dol_matrix *grad_gate, float *grad_gamma_y,
                    void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    if (dol_status s = check_call(u, gate)) return s;
    for (const auto &m : {std::make_pair(x, given_h ? "h" : "x"), std::make_pair(grad_h, "grad_h"), std::make_pair(grad_y, "grad_y"), std::make_pair(grad_x, "grad_x"),
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
        for (const dol_matrix *m : {x, u, gate, grad_h, grad_y, grad_x, grad_u})
            if (meet(grad_gate, m)) return fail(DOL_EINVAL, "grad_gate is another operand's or result's memory");
    }
    if (meet(grad_x, grad_u) || meet(grad_x, gate) || meet(grad_u, gate)) return fail(DOL_EINVAL, "two of grad_x, grad_u and gate are the same, or lie over each other");
    for (const dol_matrix *m : {x, u, grad_h, grad_y})
        if (cross(grad_x, m) || cross(grad_u, m)) return fail(DOL_EINVAL, "grad_x or grad_u lies over an operand, but not each row over its own");
    const uint64_t per_row = u->rows * sizeof(float), per_col = u->cols * sizeof(float);
    const Span sums_u(grad_gamma_u, per_col), sums_y(grad_gamma_y, per_col);
    for (const Span &m : {Span(gamma_u, per_col), Span(gamma_y, per_col), Span(norm_u ? rstd_u : nullptr, per_row), Span(grad_y ? rstd_h : nullptr, per_row), sums_u, sums_y})
        if (meet(grad_x, m) || meet(grad_u, m) || meet(grad_gate, m)) return fail(DOL_EINVAL, "grad_x, grad_u or grad_gate lies over a vector of the call");
    for (const dol_matrix *m : {x, u, gate, grad_h, grad_y})
        if (meet(sums_u, m) || meet(sums_y, m)) return fail(DOL_EINVAL, "grad_gamma_u or grad_gamma_y lies over an operand");
    if (meet(sums_u, sums_y)) return fail(DOL_EINVAL, "grad_gamma_u and grad_gamma_y lie over each other");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (u->rows == 0) {
        auto zero = [&](auto type) {
            using S = decltype(type);
            const int64_t gates = grad_gate ? grad_gate->rows : 0, blocks = (std::max<int64_t>(gates, 1) * u->cols + kThreads - 1) / kThreads;
            residual_norm_zero_kernel<S><<<static_cast<unsigned>(std::min<int64_t>(blocks, kMostCols / kThreads)), kThreads, 0, st>>>(grad_gamma_u, grad_gamma_y, out_of<S>(grad_gate), gates, u->cols);
            DOL_HIP(hipGetLastError());
            return DOL_OK;
        };
        return u->dtype == DOL_F32 ? zero(0.0f) : zero(static_cast<__bf16>(0.0f));
    }
    if (norm_u && !rstd_u) return fail(DOL_EINVAL, "rstd_u is NULL");
    if (grad_y && !rstd_h) return fail(DOL_EINVAL, "rstd_h is NULL");
    if (grad_y && given_h && !x) return fail(DOL_EINVAL, "h is NULL");
    auto go = [&](auto type) {
        using S = decltype(type);
        const Plan p = plan_of(u, gate, workspace);
        if (dol_status s = check_workspace(workspace, workspace_bytes, p.bytes)) return s;
        Args<S> a = args_of<S>(u, norm_u, gamma_u, gate, scale, gamma_y);
        a.given_h = given_h, a.x = in_of<S>(x), a.grad_h = in_of<S>(grad_h), a.grad_y = in_of<S>(grad_y), a.grad_x = out_of<S>(grad_x), a.grad_u = out_of<S>(grad_u);
        a.rstd_u = const_cast<float *>(rstd_u), a.rstd_h = const_cast<float *>(rstd_h);
        return reverse<S>(p, a, grad_gamma_u, grad_gate, grad_gamma_y, st);
    };
    return u->dtype == DOL_F32 ? go(0.0f) : go(static_cast<__bf16>(0.0f));
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
    if (meet(h, y) || meet(h, gate) || meet(y, gate)) return fail(DOL_EINVAL, "two of h, y and gate are the same, or lie over each other");
    for (const dol_matrix *m : {x, u})
        if (cross(h, m) || cross(y, m)) return fail(DOL_EINVAL, "h or y lies over x or u, but not each row over its own");
    const uint64_t per_row = u->rows * sizeof(float), per_col = u->cols * sizeof(float);
    const Span of_u(norm_u ? rstd_u : nullptr, per_row), of_h(y ? rstd_h : nullptr, per_row);
    for (const Span &m : {Span(gamma_u, per_col), Span(gamma_y, per_col), of_u, of_h})
        if (meet(h, m) || meet(y, m)) return fail(DOL_EINVAL, "h or y lies over a vector of the call");
    for (const Span &m : {Span(x), Span(u), Span(gate), Span(gamma_u, per_col), Span(gamma_y, per_col)})
        if (meet(of_u, m) || meet(of_h, m)) return fail(DOL_EINVAL, "rstd_u or rstd_h lies over an operand");
    if (meet(of_u, of_h)) return fail(DOL_EINVAL, "rstd_u and rstd_h lie over each other");
    if (gamma_u && !norm_u) return fail(DOL_EINVAL, "gamma_u without norm_u");
    if (!(eps >= 0.0f)) return fail(DOL_EINVAL, "eps = %g is not a number of at least 0", static_cast<double>(eps));
    if (u->rows == 0) return DOL_OK;
    auto go = [&](auto type) {
        using S = decltype(type);
        Args<S> a = args_of<S>(u, norm_u, gamma_u, gate, scale, gamma_y);
        a.x = in_of<S>(x), a.out_h = out_of<S>(h), a.out_y = out_of<S>(y), a.eps = eps, a.rstd_u = rstd_u, a.rstd_h = rstd_h;
        return forward<S>(a, threads_of(u->cols), static_cast<hipStream_t>(hip_stream));
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
    return backward(false, x, u, norm_u, gamma_u, gate, scale, gamma_y, rstd_u, rstd_h, grad_h, grad_y, grad_x, grad_u, grad_gamma_u, grad_gate, grad_gamma_y, workspace,
                    workspace_bytes, hip_stream);
}

dol_status dol_residual_norm_backward_from_h(const dol_matrix *h, const dol_matrix *u, int32_t norm_u, const float *gamma_u, const dol_matrix *gate, float scale,
                                             const float *gamma_y, const float *rstd_u, const float *rstd_h, const dol_matrix *grad_h, const dol_matrix *grad_y,
                                             const dol_matrix *grad_x, const dol_matrix *grad_u, float *grad_gamma_u, const dol_matrix *grad_gate, float *grad_gamma_y,
                                             void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    return backward(true, h, u, norm_u, gamma_u, gate, scale, gamma_y, rstd_u, rstd_h, grad_h, grad_y, grad_x, grad_u, grad_gamma_u, grad_gate, grad_gamma_y, workspace,
                    workspace_bytes, hip_stream);
}

}  // extern "C"
