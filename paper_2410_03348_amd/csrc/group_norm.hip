// Group norm over channels-last activations x[sample][point][channel], followed by an activation function, and its gradients.
//
//   mean, var over the points and the channels of a group,   rstd = 1 / sqrt(var + eps)
//   xhat = (x - mean) rstd,   z = gamma xhat + beta,   y = act(z)
//   dz = dy act'(z),   grad_beta[c] = sum dz,   grad_gamma[c] = sum dz xhat
//   grad_x = rstd (gamma dz - c1 - xhat c2),   c1, c2 the group's means of gamma dz and of gamma dz xhat
//
// Memory bounds all of it: 2 tensors forward, 3 backward.  Where a slab of a sample (all points of some whole groups) fits the
// registers of a workgroup it is read once: sums of deviations from the mean itself, not of squares, and backward dz is kept while its
// sums are made (group_norm_slab_*).  Larger groups are shared out over the points: a launch for the sums, one that joins them, and one
// that reads x again (group_norm_part_*, group_norm_finish_*, group_norm_map_*).
// A thread keeps to its few neighbouring channels, so that sums over points stay in registers until the points are done.
#include "activation.h"
#include "internal.h"
#include "wave_util.h"

namespace dol {
namespace {

constexpr int kFewVecs = 4, kForwardVecs = 16, kBackwardVecs = 8;       // vectors that a thread of a slab holds (x; x and dz)
constexpr size_t kSlabLds = 128 * 1024;
constexpr int kSlabThreads = 1024, kSlabThreadsBack = 512;      // at most, so that what a thread holds stays in registers
constexpr int kUnits = 256;

// V neighbouring channels as memory has them: a thread that holds many keeps them so, and unpacks one where it is used.
template <typename T, int V>
struct alignas(V * sizeof(T)) Vec {
    static constexpr int WORDS = V * sizeof(T) / 4;
    uint32_t w[WORDS];
    __device__ float get(int v) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[v]);
        else return __uint_as_float(v & 1 ? w[v >> 1] & 0xFFFF0000u : w[v >> 1] << 16);
    }
    __device__ void set(const float (&x)[V])
    {
#pragma unroll
        for (int k = 0; k < WORDS; ++k) {
            if constexpr (sizeof(T) == 4) w[k] = __float_as_uint(x[k]);
            else w[k] = __builtin_bit_cast(uint16_t, static_cast<T>(x[2 * k])) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<T>(x[2 * k + 1]))) << 16;
        }
    }
};
template <>
struct Vec<__bf16, 1> {
    uint16_t w;
    __device__ float get(int) const { return __uint_as_float(static_cast<uint32_t>(w) << 16); }
    __device__ void set(const float (&x)[1]) { w = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x[0])); }
};

struct Shape {
    int32_t batch, points, channels, groups, per;       // per: channels of a group
    int32_t slice, slices;                              // channels that a workgroup takes; how many such
    int32_t lanes, rows;                                // threads to a point of the slice; points that a workgroup takes at a time
    float count, per_lanes, per_per, per_count;         // a group's elements; reciprocals of lanes, per and count
    int32_t chunk, chunks;                              // points that a workgroup of the shared-out form takes; how many such
};

struct Tensor {
    void *data;
    int64_t ld_batch, ld_point;
    template <typename T>
    __device__ T *at(int64_t b, int64_t p, int64_t c) const { return static_cast<T *>(data) + b * ld_batch + p * ld_point + c; }
};

// t / count to the last bit or so: the product with the reciprocal, and what it is off by.
__device__ __forceinline__ float mean_of(float t, const Shape &s)
{
    const float m = t * s.per_count;
    return __builtin_fmaf(__builtin_fmaf(-m, s.count, t), s.per_count, m);
}

__device__ __forceinline__ float rstd_of(float var, float eps) { return 1.0f / __builtin_amdgcn_sqrtf(var + eps); }

// ---------------------------------------------------------------- sums over the threads of a workgroup

// A workgroup of a small tensor runs its code once, and waits for every line of it: divisions are made of the host's reciprocals, and
// the sums are loops (written out they took 3 400 of a workgroup's 16 800 clocks at 784 x 4 floats, each of the two).

// Where a thread stands in a slab or a chunk: `lanes` threads of V channels make a row of the slice, `rows` such rows the workgroup.
struct Place {
    int rows, lane, row;
    bool in;
};

// floor(x / d) for x below 8192 and r = 1 / d rounded: (x + 1/2) / d is at least 1 / (2 d) from the next whole number.
__device__ __forceinline__ int small_quotient(int x, float r) { return static_cast<int>((static_cast<float>(x) + 0.5f) * r); }

__device__ __forceinline__ Place place_of(const Shape &s)
{
    Place p;
    p.rows = s.rows, p.row = small_quotient(threadIdx.x, s.per_lanes);
    p.lane = threadIdx.x - p.row * s.lanes, p.in = p.row < p.rows;
    return p;
}

__device__ __forceinline__ float sum_of_wave(float x) { return with_lane32<AddOp>(reduce32<AddOp>(x)); }

// Threads' values of their channels, for Q quantities, to buf[q * size + row * pitch + channel], pitch odd.
template <int V, int Q>
__device__ __forceinline__ void put_rows(const float (&s)[Q][V], const Place &p, int pitch, float *buf)
{
    if (p.in)
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int v = 0; v < V; ++v) buf[(q * p.rows + p.row) * pitch + p.lane * V + v] = s[q][v];
    lds_barrier();
}

// The sum of a block of rows x columns values (below 8192), taken by a wavefront; the same in all lanes.
__device__ __forceinline__ float sum_block(const float *buf, int rows, int pitch, int columns, float per_columns)
{
    float t = 0.0f;
#pragma unroll 4
    for (int e = threadIdx.x & 63; e < rows * columns; e += 64) {
        const int r = small_quotient(e, per_columns);
        t += buf[r * pitch + e - r * columns];
    }
    return sum_of_wave(t);
}

// The group, from the slice's first, of each of the channels lane * V ..
template <int V>
__device__ __forceinline__ void groups_of(int (&g)[V], const Place &p, const Shape &s)
{
    int at = small_quotient(p.lane * V, s.per_per), rest = p.lane * V - at * s.per;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        g[v] = at;
        if (++rest == s.per) rest = 0, ++at;
    }
}

// ---------------------------------------------------------------- slabs

// A slab is read once, and kept.  Bytes bound it where there are many slabs: bf16 128 x 1024 x 256 28.9 us, 4.6 TB/s; small ones take a load,
// two rounds of sums and the stores one after the other, float 64 x 784 x 32 8.9 us.
template <typename T, int V, int K>
__global__ void __launch_bounds__(kSlabThreads) group_norm_slab_forward_kernel(Shape s, Tensor x, const float *gamma, const float *beta, float eps, int act, Tensor y,
                                                                              float *mean, float *rstd)
{
    extern __shared__ __align__(16) float lds[];
    const unsigned id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int b = id / s.slices, sl = id - b * s.slices, c0 = sl * s.slice, groups = s.groups / s.slices, pitch = s.slice | 1;
    const int64_t g0 = static_cast<int64_t>(b) * s.groups + sl * groups;
    const Place p = place_of(s);
    float *gmean = lds, *grstd = gmean + groups, *buf = grstd + groups;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const T *src = x.at<T>(b, p.row, c0 + p.lane * V);
    const int64_t step = p.rows * x.ld_point;
    const int left = p.in ? s.points - p.row : 0;           // vector k is there where k * rows < left
    Vec<T, V> in[K];
    float sum[1][V] = {}, f[V], o[V];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k * p.rows < left) in[k] = *reinterpret_cast<const Vec<T, V> *>(src + k * step);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = c0 + p.lane * V + v;
        f[v] = p.in && gamma ? gamma[c] : 1.0f, o[v] = p.in && beta ? beta[c] : 0.0f;
    }
    int gi[V];
    groups_of(gi, p, s);
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k * p.rows < left)
#pragma unroll
            for (int v = 0; v < V; ++v) sum[0][v] += in[k].get(v);
    put_rows<V, 1>(sum, p, pitch, buf);
#pragma unroll 1
    for (int g = wave; g < groups; g += waves) gmean[g] = mean_of(sum_block(buf + g * s.per, p.rows, pitch, s.per, s.per_per), s);
    lds_barrier();
    float m[V], sq[1][V] = {};
#pragma unroll
    for (int v = 0; v < V; ++v) m[v] = p.in ? gmean[gi[v]] : 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k * p.rows < left)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float d = in[k].get(v) - m[v];
                sq[0][v] = __builtin_fmaf(d, d, sq[0][v]);
            }
    put_rows<V, 1>(sq, p, pitch, buf);
#pragma unroll 1
    for (int g = wave; g < groups; g += waves) {
        const float r = rstd_of(sum_block(buf + g * s.per, p.rows, pitch, s.per, s.per_per) * s.per_count, eps);
        grstd[g] = r;
        if (mean && (threadIdx.x & 63) == 0) mean[g0 + g] = gmean[g];
        if (rstd && (threadIdx.x & 63) == 0) rstd[g0 + g] = r;
    }
    lds_barrier();
    if (left <= 0) return;
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] *= grstd[gi[v]];
    T *dst = y.at<T>(b, p.row, c0 + p.lane * V);
    const int64_t out_step = p.rows * y.ld_point;
    with_act(act, [&](auto A) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k * p.rows < left) {
                Vec<T, V> out;
                float z[V];
#pragma unroll
                for (int v = 0; v < V; ++v) z[v] = act_of<decltype(A)::value, false>(__builtin_fmaf(in[k].get(v) - m[v], f[v], o[v]), nullptr);
                out.set(z);
                *reinterpret_cast<Vec<T, V> *>(dst + k * out_step) = out;
            }
    });
}

// sums[2][batch][channels]: of dz and of dz xhat over the sample's points.  With eight vectors to a thread one workgroup is all that a unit
// holds, and loads wait for the stores before: bf16 128 x 1024 x 256 68.7 us, 2.9 TB/s; with four two.
template <typename T, int V, int K>
__global__ void __launch_bounds__(kSlabThreadsBack, K == kFewVecs ? 4 : 2) group_norm_slab_backward_kernel(Shape s, Tensor x, const float *gamma, const float *beta, const float *mean, const float *rstd,
                                                                               Tensor dy, int act, Tensor dx, float *sums_out)
{
    extern __shared__ __align__(16) float lds[];
    const unsigned id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int b = id / s.slices, sl = id - b * s.slices, c0 = sl * s.slice, groups = s.groups / s.slices, pitch = s.slice | 1;
    const int64_t g0 = static_cast<int64_t>(b) * s.groups + sl * groups;
    const Place p = place_of(s);
    float *sums = lds, *c12 = sums + 2 * s.slice, *buf = c12 + 2 * groups;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const T *src = x.at<T>(b, p.row, c0 + p.lane * V), *up = dy.at<T>(b, p.row, c0 + p.lane * V);
    const int64_t step = p.rows * x.ld_point, up_step = p.rows * dy.ld_point;
    const int left = p.in ? s.points - p.row : 0;
    Vec<T, V> in[K], gr[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k * p.rows < left) {
            in[k] = *reinterpret_cast<const Vec<T, V> *>(src + k * step);
            gr[k] = *reinterpret_cast<const Vec<T, V> *>(up + k * up_step);
        }
    float m[V], f[V], sum[2][V] = {}, dz[K][V];
    if (p.in) {
        int gi[V];
        groups_of(gi, p, s);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float r = rstd[g0 + gi[v]];
            m[v] = mean[g0 + gi[v]], f[v] = gamma ? r * gamma[c0 + p.lane * V + v] : r;
        }
    }
    {
        float o[V];         // z = (x - m) f + o
        if (p.in)
#pragma unroll
            for (int v = 0; v < V; ++v) o[v] = beta ? beta[c0 + p.lane * V + v] : 0.0f;
        with_act(act, [&](auto A) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (k * p.rows < left)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const float d = in[k].get(v) - m[v];
                        float slope;
                        act_of<decltype(A)::value, true>(__builtin_fmaf(d, f[v], o[v]), &slope);
                        dz[k][v] = gr[k].get(v) * slope;
                        sum[0][v] += dz[k][v], sum[1][v] = __builtin_fmaf(dz[k][v], d, sum[1][v]);
                    }
        });
    }
    // (what a later part needs of rstd and the groups it reads and works out again: registers decide how many workgroups a unit takes)
    if (p.in) {             // of dz xhat
        int gi[V];
        groups_of(gi, p, s);
#pragma unroll
        for (int v = 0; v < V; ++v) sum[1][v] *= rstd[g0 + gi[v]];
    }
    put_rows<V, 2>(sum, p, pitch, buf);
    // A wavefront to a sum, or a thread: some 170 clocks each and 28 a row.
    const int threads = blockDim.x;
    if (p.rows * ((2 * s.slice + threads - 1) / threads) > 6 * ((2 * s.slice + waves - 1) / waves)) {
#pragma unroll 1
        for (int t = wave; t < 2 * s.slice; t += waves) {
            const int q = t >= s.slice;
            sums[t] = sum_block(buf + q * p.rows * pitch + t - q * s.slice, p.rows, pitch, 1, 1.0f);
        }
    } else
#pragma unroll 1
        for (int t = threadIdx.x; t < 2 * s.slice; t += blockDim.x) {
            const int q = t >= s.slice;
            const float *from = buf + q * p.rows * pitch + t - q * s.slice;
            float a = 0.0f;
#pragma unroll 4
            for (int k = 0; k < p.rows; ++k) a += from[k * pitch];
            sums[t] = a;
        }
    lds_barrier();
    if (sums_out)
#pragma unroll 1
        for (int t = threadIdx.x; t < 2 * s.slice; t += blockDim.x) {
            const int q = t >= s.slice;
            sums_out[(static_cast<int64_t>(q) * s.batch + b) * s.channels + c0 + t - q * s.slice] = sums[t];
        }
    if (!dx.data) return;
#pragma unroll 1
    for (int t = wave; t < 2 * groups; t += waves) {
        const int q = t >= groups, ch = (t - q * groups) * s.per;
        float a = 0.0f;
        for (int c = threadIdx.x & 63; c < s.per; c += 64) a = __builtin_fmaf(sums[q * s.slice + ch + c], gamma ? gamma[c0 + ch + c] : 1.0f, a);
        c12[t] = sum_of_wave(a) * s.per_count;
    }
    lds_barrier();
    if (left <= 0) return;
    T *dst = dx.at<T>(b, p.row, c0 + p.lane * V);
    const int64_t out_step = p.rows * dx.ld_point;
    float k1[V], k2[V];     // rstd c1, rstd^2 c2
    int gi[V];
    groups_of(gi, p, s);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float r = rstd[g0 + gi[v]];
        k1[v] = r * c12[gi[v]], k2[v] = r * r * c12[groups + gi[v]];
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k * p.rows < left) {
            Vec<T, V> out;
            float g[V];
#pragma unroll
            for (int v = 0; v < V; ++v) g[v] = __builtin_fmaf(f[v], dz[k][v], -__builtin_fmaf(in[k].get(v) - m[v], k2[v], k1[v]));
            out.set(g);
            *reinterpret_cast<Vec<T, V> *>(dst + k * out_step) = out;
        }
}

// grad_beta (blockIdx.y 0) and grad_gamma = the samples' sums added up; sixteen channels to a workgroup, every sixty-fourth sample to a thread.
__global__ void __launch_bounds__(1024) group_norm_params_kernel(const float *sums, int32_t batch, int32_t channels, float *grad_gamma, float *grad_beta)
{
    __shared__ float red[64][17];
    float *out = blockIdx.y ? grad_gamma : grad_beta;
    if (!out) return;
    const int lane = threadIdx.x & 15, row = threadIdx.x >> 4, c = blockIdx.x * 16 + lane;
    const float *from = sums + static_cast<int64_t>(blockIdx.y) * batch * channels + c;
    float s = 0.0f;
    if (c < channels)
#pragma unroll 8
        for (int b = row; b < batch; b += 64) s += from[static_cast<int64_t>(b) * channels];
    red[row][lane] = s;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    s = 0.0f;               // a lane sixteen of them, and the four lanes of a channel meet
#pragma unroll
    for (int k = 0; k < 16; ++k) s += red[row * 16 + k][lane];
    s = with_lane32<AddOp>(with_lane16<AddOp>(s));
    if (row == 0 && c < channels) out[c] = s;
}

// ---------------------------------------------------------------- groups shared out over their points

constexpr int kPartThreads = 256, kPartLanes = 64;   // threads of a workgroup, the most of them to a point
constexpr int kBlock = 8;                           // points whose own mean a thread takes before it joins them

// Mean and sum of squared deviations of n more values joined to those of `have` values.
__device__ __forceinline__ void join(float &mean, float &m2, float have, float mean2, float m22, float n)
{
    const float all = have + n, d = mean2 - mean, f = n / all;
    mean = __builtin_fmaf(d, f, mean);
    m2 = m2 + m22 + d * d * have * f;
}

// part[batch][chunks][channels] = (mean, squared deviations) of a channel's points in a chunk.  Bytes bound it: bf16 16 x 65536 x 128 64 us, 4.2 TB/s.
template <typename T, int V>
__global__ void __launch_bounds__(kPartThreads) group_norm_part_forward_kernel(Shape s, Tensor x, float2 *part)
{
    __shared__ float red[2][kPartThreads * V];
    __shared__ float counts[kPartThreads];
    const int b = blockIdx.z, c0 = blockIdx.y * s.slice, width = min(s.slice, s.channels - c0);
    const Place p = place_of(s);
    const int64_t first = static_cast<int64_t>(blockIdx.x) * s.chunk, end = min(first + s.chunk, static_cast<int64_t>(s.points));
    const bool in = p.in && p.lane * V < width;
    float mean[V] = {}, m2[V] = {}, have = 0.0f;
    if (in) {
        const T *src = x.at<T>(b, 0, c0 + p.lane * V);
        for (int64_t pt = first + p.row; pt < end; pt += static_cast<int64_t>(kBlock) * p.rows) {
            Vec<T, V> v[kBlock];
            const int n = static_cast<int>(min(static_cast<int64_t>(kBlock), (end - pt + p.rows - 1) / p.rows));
#pragma unroll
            for (int k = 0; k < kBlock; ++k)
                if (k < n) v[k] = *reinterpret_cast<const Vec<T, V> *>(src + (pt + static_cast<int64_t>(k) * p.rows) * x.ld_point);
            const float fn = static_cast<float>(n), rn = 1.0f / fn;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float sum = 0.0f, sq = 0.0f;
#pragma unroll
                for (int k = 0; k < kBlock; ++k) sum += k < n ? v[k].get(e) : 0.0f;
                const float own = sum * rn;
#pragma unroll
                for (int k = 0; k < kBlock; ++k) {
                    const float d = k < n ? v[k].get(e) - own : 0.0f;
                    sq = __builtin_fmaf(d, d, sq);
                }
                join(mean[e], m2[e], have, own, sq, fn);
            }
            have += fn;
        }
    }
    if (p.in && p.lane == 0) counts[p.row] = have;
    if (p.in)
#pragma unroll
        for (int e = 0; e < V; ++e) red[0][p.row * s.slice + p.lane * V + e] = mean[e], red[1][p.row * s.slice + p.lane * V + e] = m2[e];
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += kPartThreads) {
        float m = 0.0f, q = 0.0f, n = 0.0f;
        for (int r = 0; r < p.rows; ++r)
            if (counts[r] > 0.0f) {
                join(m, q, n, red[0][r * s.slice + c], red[1][r * s.slice + c], counts[r]);
                n += counts[r];
            }
        part[(static_cast<int64_t>(b) * s.chunks + blockIdx.x) * s.channels + c0 + c] = make_float2(m, q);
    }
}

// A group's mean and rstd from its parts.
__global__ void __launch_bounds__(256) group_norm_finish_forward_kernel(Shape s, const float2 *part, float eps, float *mean, float *rstd, float *mean_out, float *rstd_out)
{
    __shared__ float red[4];
    const int64_t b = blockIdx.y, g = blockIdx.x, at = b * s.groups + g;
    const float2 *p = part + b * s.chunks * s.channels + g * s.per;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    auto points_of = [&](int k) { return static_cast<float>(min(s.chunk, s.points - k * s.chunk)); };
    auto all = [&](float v) {
        v = sum_of_wave(v);
        lds_barrier();
        if (lane == 0) red[w] = v;
        lds_barrier();
        return (red[0] + red[1]) + (red[2] + red[3]);
    };
    float t = 0.0f;
    const int n = s.chunks * s.per;
    for (int k = threadIdx.x; k < n; k += 256) t += p[static_cast<int64_t>(k / s.per) * s.channels + k % s.per].x * points_of(k / s.per);
    const float m = mean_of(all(t), s);
    t = 0.0f;
    for (int k = threadIdx.x; k < n; k += 256) {
        const float2 q = p[static_cast<int64_t>(k / s.per) * s.channels + k % s.per];
        t += __builtin_fmaf((q.x - m) * (q.x - m), points_of(k / s.per), q.y);
    }
    const float r = rstd_of(all(t) * s.per_count, eps);
    if (threadIdx.x == 0) {
        mean[at] = m, rstd[at] = r;
        if (mean_out) mean_out[at] = m;
        if (rstd_out) rstd_out[at] = r;
    }
}

// y, or grad_x (BACKWARD; c12: a group's c1 and c2), of a chunk.  The last chunk first: what the sums read last may still be in cache.
// bf16 16 x 65536 x 128 in 101 us, 5.3 TB/s, the rate of a copy.
template <typename T, int V, bool BACKWARD>
__global__ void __launch_bounds__(kPartThreads) group_norm_map_kernel(Shape s, Tensor x, Tensor dy, const float *gamma, const float *beta, const float *mean, const float *rstd,
                                                                      const float2 *c12, int act, Tensor out)
{
    const int b = s.batch - 1 - blockIdx.z, c0 = blockIdx.y * s.slice, width = min(s.slice, s.channels - c0);
    const Place p = place_of(s);
    if (!p.in || p.lane * V >= width) return;
    float m[V], r[V], ga[V], be[V], c1[V], c2[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = c0 + p.lane * V + v;
        const int64_t g = static_cast<int64_t>(b) * s.groups + c / s.per;
        m[v] = mean[g], r[v] = rstd[g], ga[v] = gamma ? gamma[c] : 1.0f, be[v] = beta ? beta[c] : 0.0f;
        if (BACKWARD) c1[v] = c12[g].x, c2[v] = c12[g].y;
        else ga[v] *= r[v];
    }
    const int64_t first = static_cast<int64_t>(s.chunks - 1 - blockIdx.x) * s.chunk, end = min(first + s.chunk, static_cast<int64_t>(s.points));
    const T *src = x.at<T>(b, 0, c0 + p.lane * V), *up = BACKWARD ? dy.at<T>(b, 0, c0 + p.lane * V) : nullptr;
    T *dst = out.at<T>(b, 0, c0 + p.lane * V);
    with_act(act, [&](auto A) {
#pragma unroll 4
        for (int64_t pt = first + p.row; pt < end; pt += p.rows) {
            const Vec<T, V> in = *reinterpret_cast<const Vec<T, V> *>(src + pt * x.ld_point);
            Vec<T, V> gr, packed;
            float o[V];
            if (BACKWARD) gr = *reinterpret_cast<const Vec<T, V> *>(up + pt * dy.ld_point);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float d = in.get(v) - m[v];
                if (BACKWARD) {
                    const float xh = d * r[v];
                    float slope;
                    act_of<decltype(A)::value, true>(__builtin_fmaf(ga[v], xh, be[v]), &slope);
                    o[v] = r[v] * __builtin_fmaf(ga[v], gr.get(v) * slope, -__builtin_fmaf(xh, c2[v], c1[v]));
                } else
                    o[v] = act_of<decltype(A)::value, false>(__builtin_fmaf(d, ga[v], be[v]), nullptr);
            }
            packed.set(o);
            *reinterpret_cast<Vec<T, V> *>(dst + pt * out.ld_point) = packed;
        }
    });
}

// part[batch][chunks][channels] = sums of dz and of dz xhat over a channel's points in a chunk.
template <typename T, int V>
__global__ void __launch_bounds__(kPartThreads) group_norm_part_backward_kernel(Shape s, Tensor x, Tensor dy, const float *gamma, const float *beta, const float *mean,
                                                                                const float *rstd, int act, float2 *part)
{
    __shared__ float buf[2 * kPartThreads * (V + 1)];
    const int b = blockIdx.z, c0 = blockIdx.y * s.slice, width = min(s.slice, s.channels - c0);
    const Place p = place_of(s);
    const int64_t first = static_cast<int64_t>(blockIdx.x) * s.chunk, end = min(first + s.chunk, static_cast<int64_t>(s.points));
    float sum[2][V] = {};
    if (p.in && p.lane * V < width) {
        float m[V], r[V], ga[V], be[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = c0 + p.lane * V + v;
            const int64_t g = static_cast<int64_t>(b) * s.groups + c / s.per;
            m[v] = mean[g], r[v] = rstd[g], ga[v] = gamma ? gamma[c] : 1.0f, be[v] = beta ? beta[c] : 0.0f;
        }
        const T *src = x.at<T>(b, 0, c0 + p.lane * V), *up = dy.at<T>(b, 0, c0 + p.lane * V);
        with_act(act, [&](auto A) {
#pragma unroll 4
            for (int64_t pt = first + p.row; pt < end; pt += p.rows) {
                const Vec<T, V> in = *reinterpret_cast<const Vec<T, V> *>(src + pt * x.ld_point), gr = *reinterpret_cast<const Vec<T, V> *>(up + pt * dy.ld_point);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float xh = (in.get(v) - m[v]) * r[v];
                    float slope;
                    act_of<decltype(A)::value, true>(__builtin_fmaf(ga[v], xh, be[v]), &slope);
                    const float dz = gr.get(v) * slope;
                    sum[0][v] += dz, sum[1][v] = __builtin_fmaf(dz, xh, sum[1][v]);
                }
            }
        });
    }
    const int pitch = s.slice | 1;
    put_rows<V, 2>(sum, p, pitch, buf);
    for (int c = threadIdx.x; c < width; c += kPartThreads) {
        float a[2] = {0.0f, 0.0f};
#pragma unroll 4
        for (int k = 0; k < p.rows; ++k) a[0] += buf[k * pitch + c], a[1] += buf[(p.rows + k) * pitch + c];
        part[(static_cast<int64_t>(b) * s.chunks + blockIdx.x) * s.channels + c0 + c] = make_float2(a[0], a[1]);
    }
}

// Joins a group's parts: its channels' sums over the sample (sums as group_norm_slab_backward_kernel leaves them) and c1, c2.
__global__ void __launch_bounds__(256) group_norm_finish_backward_kernel(Shape s, const float2 *part, const float *gamma, float *sums, float2 *c12)
{
    __shared__ float red[2][4];
    const int64_t b = blockIdx.y, g = blockIdx.x, at = b * s.groups + g;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    float c1 = 0.0f, c2 = 0.0f;
    for (int c = w; c < s.per; c += 4) {            // a wavefront to a channel, a lane to every sixty-fourth chunk
        const int64_t ch = g * s.per + c;
        float t = 0.0f, u = 0.0f;
        for (int k = lane; k < s.chunks; k += 64) {
            const float2 q = part[(b * s.chunks + k) * s.channels + ch];
            t += q.x, u += q.y;
        }
        t = sum_of_wave(t), u = sum_of_wave(u);
        const float ga = gamma ? gamma[ch] : 1.0f;
        c1 = __builtin_fmaf(t, ga, c1), c2 = __builtin_fmaf(u, ga, c2);
        if (lane == 0) sums[b * s.channels + ch] = t, sums[(s.batch + b) * s.channels + ch] = u;
    }
    if (lane == 0) red[0][w] = c1, red[1][w] = c2;
    __syncthreads();
    if (threadIdx.x == 0) {
        c12[at] = make_float2(((red[0][0] + red[0][1]) + (red[0][2] + red[0][3])) * s.per_count, ((red[1][0] + red[1][1]) + (red[1][2] + red[1][3])) * s.per_count);
    }
}

__global__ void __launch_bounds__(256) group_norm_zero_kernel(float *a, float *b, int32_t n)
{
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t < n && a) a[t] = 0.0f;
    if (t < n && b) b[t] = 0.0f;
}

// ---------------------------------------------------------------- host side

dol_status check_activations(const dol_activations *t, const dol_activations *like, const char *name)
{
    if (!t) return fail(DOL_EINVAL, "%s is NULL", name);
    if (t->dtype != DOL_F32 && t->dtype != DOL_BF16) return fail(DOL_EINVAL, "%s has unknown type %d", name, t->dtype);
    if (t->batch < 0 || t->points < 0 || t->channels < 0) return fail(DOL_ESHAPE, "%s is %d x %d x %d", name, t->batch, t->points, t->channels);
    if (like && t->dtype != like->dtype) return fail(DOL_EINVAL, "%s is of another type than x", name);
    if (like && (t->batch != like->batch || t->points != like->points || t->channels != like->channels))
        return fail(DOL_ESHAPE, "%s is %d x %d x %d, x is %d x %d x %d", name, t->batch, t->points, t->channels, like->batch, like->points, like->channels);
    if (t->ld_point < t->channels) return fail(DOL_ESHAPE, "%s.ld_point = %lld smaller than its %d channels", name, static_cast<long long>(t->ld_point), t->channels);
    if (t->points > 0 && t->batch > 1 && !apart(t->points, t->ld_point, t->batch, t->ld_batch, t->channels))
        return fail(DOL_ESHAPE, "%s.ld_batch = %lld: samples overlap", name, static_cast<long long>(t->ld_batch));
    if (t->batch > 0 && t->points > 0 && t->channels > 0) {
        if (!t->data) return fail(DOL_EINVAL, "%s.data is NULL", name);
        if (reinterpret_cast<uintptr_t>(t->data) & (t->dtype == DOL_F32 ? 3 : 1)) return fail(DOL_EINVAL, "%s.data is not aligned to its elements", name);
    }
    return DOL_OK;
}

dol_status check_call(const dol_activations *x, int32_t groups, int32_t act)
{
    if (dol_status s = check_activations(x, nullptr, "x")) return s;
    if (groups < 1 || x->channels % groups != 0) return fail(DOL_ESHAPE, "%d channels in %d groups", x->channels, groups);
    if (act < DOL_ACT_NONE || act > DOL_ACT_GELU) return fail(DOL_EINVAL, "unknown activation function %d", act);
    if (x->batch > 65535 || x->channels > 1 << 20 || int64_t(x->batch) * x->channels > INT32_MAX)
        return fail(DOL_EUNSUPPORTED, "%d samples of %d channels: more than 65535, %d, or 2^31 of both", x->batch, x->channels, 1 << 20);
    return DOL_OK;
}

// The most neighbouring channels that every tensor of the call can be read and written by at a time.
int vector_of(const dol_activations *x, const dol_activations *a, const dol_activations *b)
{
    const int e = x->dtype == DOL_F32 ? 4 : 2;
    int v = 16 / e;
    for (const dol_activations *t : {x, a, b}) {
        if (!t || !t->data) continue;
        while (v > 1 && (t->ld_point % v || (t->batch > 1 && t->ld_batch % v) || t->channels % v || reinterpret_cast<uintptr_t>(t->data) % (v * e))) v /= 2;
    }
    return v;
}

struct Plan {
    Shape s;
    int vec, vecs, threads;         // vecs: that a thread of a slab holds; threads: 0 where groups are shared out
    size_t lds;
};

Plan plan_of(const dol_activations *x, int32_t groups, int vec, bool backward)
{
    Plan p{};
    p.vec = vec;
    Shape &s = p.s;
    s.batch = x->batch, s.points = x->points, s.channels = x->channels, s.groups = groups, s.per = x->channels / groups;
    const int e = x->dtype == DOL_F32 ? 4 : 2;
    // A slab is a set of whole groups, in whole vectors, of at least 16 bytes to a point.  Wider ones are taken up to 64 bytes while there
    // are two workgroups to a compute unit, and beyond while there are four.  (A line of memory is then shared by slabs of one sample, which
    // run on one XCD, at the same time.)
    // Backward, eight vectors of x and of dy to a thread leave a unit one workgroup, which loads, computes and stores in turn: taken only
    // where slabs would else be narrower than 64 bytes.  Forward and backward, four / eight vectors, us: bf16 512 x 256 x 256 120 / 145,
    // 512 x 512 x 64 61 / 69, float 512 x 256 x 256 162 / 194, but bf16 128 x 1024 x 256 (32 bytes in four) 125 / 118, float 184 / 172.
    for (int k = 1; k <= groups; ++k) {
        const int64_t slice = int64_t(k) * s.per, lanes = slice / vec;
        if (groups % k || slice % vec || (slice * e < 16 && k < groups)) continue;
        int vecs = kFewVecs;
        int64_t threads = round_up((int64_t(s.points) + vecs - 1) / vecs * lanes, 64);
        if (threads > kSlabThreads / 2) {
            if (backward && p.threads && int64_t(s.slice) * e >= 64) break;
            vecs = backward ? kBackwardVecs : kForwardVecs;
            threads = round_up((int64_t(s.points) + vecs - 1) / vecs * lanes, 64);
            if (threads > (backward ? kSlabThreadsBack : kSlabThreads)) break;
        }
        const int64_t workgroups = int64_t(s.batch) * (groups / k);
        if (workgroups * threads >> 32) continue;               // (a launch has less than 2^32 threads)
        if (p.threads && !(workgroups >= 4 * kUnits || (int64_t(s.slice) * e < 64 && workgroups >= 2 * kUnits))) break;
        p.vecs = vecs, p.threads = static_cast<int>(threads), s.slice = static_cast<int32_t>(slice), s.slices = groups / k;
    }
    s.per_per = 1.0f / static_cast<float>(s.per), s.count = static_cast<float>(s.points) * static_cast<float>(s.per), s.per_count = 1.0f / s.count;
    auto place = [&](int threads) { s.lanes = s.slice / vec, s.rows = threads / s.lanes, s.per_lanes = 1.0f / static_cast<float>(s.lanes); };
    if (p.threads) {
        place(p.threads);
        const size_t q = backward ? 2 : 1;
        p.lds = 4 * (q * s.slice + 2 * (s.slice / s.per) + q * p.threads * (vec + 1));
        return p;
    }
    s.slice = std::min<int32_t>(s.channels, kPartLanes * vec);
    s.slices = (s.channels + s.slice - 1) / s.slice;
    place(kPartThreads);
    // eight workgroups to a compute unit, if that leaves a thread sixteen points
    const int64_t want = std::max<int64_t>(1, 8 * kUnits / (int64_t(s.batch) * s.slices)), rows = s.rows;
    s.chunks = static_cast<int32_t>(std::min(want, (s.points + rows * 16 - 1) / (rows * 16)));
    s.chunk = static_cast<int32_t>((int64_t(s.points) + s.chunks - 1) / s.chunks);
    s.chunks = static_cast<int32_t>((int64_t(s.points) + s.chunk - 1) / s.chunk);
    return p;
}

struct Space {
    float2 *part, *c12;
    float *mean, *rstd, *sums;
    int64_t bytes;
};

Space space_of(const Plan &p, bool backward, void *workspace)
{
    Space w{};
    Carver c(workspace);
    const Shape &s = p.s;
    if (!p.threads) w.part = c.take<float2>(int64_t(s.batch) * s.chunks * s.channels);
    if (backward) w.sums = c.take<float>(2 * int64_t(s.batch) * s.channels);
    if (!p.threads && backward) w.c12 = c.take<float2>(int64_t(s.batch) * s.groups);
    if (!p.threads && !backward) w.mean = c.take<float>(int64_t(s.batch) * s.groups), w.rstd = c.take<float>(int64_t(s.batch) * s.groups);
    w.bytes = c.used;
    return w;
}

Tensor tensor_of(const dol_activations *t) { return t ? Tensor{t->data, t->ld_batch, t->ld_point} : Tensor{}; }

template <typename T, int V, int K>
dol_status slab_forward(const Plan &p, const dol_activations *x, const float *gamma, const float *beta, float eps, int act, const dol_activations *y, float *mean, float *rstd,
                        hipStream_t st)
{
    DOL_HIP(allow_dynamic_lds(reinterpret_cast<const void *>(group_norm_slab_forward_kernel<T, V, K>), kSlabLds));
    group_norm_slab_forward_kernel<T, V, K><<<p.s.batch * p.s.slices, p.threads, p.lds, st>>>(p.s, tensor_of(x), gamma, beta, eps, act, tensor_of(y), mean, rstd);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <typename T, int V, int K>
dol_status slab_backward(const Plan &p, const dol_activations *x, const float *gamma, const float *beta, const float *mean, const float *rstd, const dol_activations *dy, int act,
                         const dol_activations *dx, float *sums, hipStream_t st)
{
    DOL_HIP(allow_dynamic_lds(reinterpret_cast<const void *>(group_norm_slab_backward_kernel<T, V, K>), kSlabLds));
    group_norm_slab_backward_kernel<T, V, K><<<p.s.batch * p.s.slices, p.threads, p.lds, st>>>(p.s, tensor_of(x), gamma, beta, mean, rstd, tensor_of(dy), act, tensor_of(dx), sums);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <typename T, int V>
dol_status forward(const Plan &p, const Space &w, const dol_activations *x, const float *gamma, const float *beta, float eps, int act, const dol_activations *y, float *mean,
                   float *rstd, hipStream_t st)
{
    if (p.threads)
        return p.vecs == kFewVecs ? slab_forward<T, V, kFewVecs>(p, x, gamma, beta, eps, act, y, mean, rstd, st)
                                  : slab_forward<T, V, kForwardVecs>(p, x, gamma, beta, eps, act, y, mean, rstd, st);
    const Shape &s = p.s;
    const dim3 grid(s.chunks, s.slices, s.batch);
    group_norm_part_forward_kernel<T, V><<<grid, kPartThreads, 0, st>>>(s, tensor_of(x), w.part);
    DOL_HIP(hipGetLastError());
    group_norm_finish_forward_kernel<<<dim3(s.groups, s.batch), 256, 0, st>>>(s, w.part, eps, w.mean, w.rstd, mean, rstd);
    DOL_HIP(hipGetLastError());
    group_norm_map_kernel<T, V, false><<<grid, kPartThreads, 0, st>>>(s, tensor_of(x), Tensor{}, gamma, beta, w.mean, w.rstd, nullptr, act, tensor_of(y));
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

template <typename T, int V>
dol_status reverse(const Plan &p, const Space &w, const dol_activations *x, const float *gamma, const float *beta, const float *mean, const float *rstd, const dol_activations *dy,
                   int act, const dol_activations *dx, float *grad_gamma, float *grad_beta, hipStream_t st)
{
    const Shape &s = p.s;
    const bool params = grad_gamma || grad_beta;
    if (p.threads) {
        if (dol_status e = p.vecs == kFewVecs ? slab_backward<T, V, kFewVecs>(p, x, gamma, beta, mean, rstd, dy, act, dx, params ? w.sums : nullptr, st)
                                              : slab_backward<T, V, kBackwardVecs>(p, x, gamma, beta, mean, rstd, dy, act, dx, params ? w.sums : nullptr, st))
            return e;
    } else {
        const dim3 grid(s.chunks, s.slices, s.batch);
        group_norm_part_backward_kernel<T, V><<<grid, kPartThreads, 0, st>>>(s, tensor_of(x), tensor_of(dy), gamma, beta, mean, rstd, act, w.part);
        DOL_HIP(hipGetLastError());
        group_norm_finish_backward_kernel<<<dim3(s.groups, s.batch), 256, 0, st>>>(s, w.part, gamma, w.sums, w.c12);
        DOL_HIP(hipGetLastError());
        if (dx) {
            group_norm_map_kernel<T, V, true><<<grid, kPartThreads, 0, st>>>(s, tensor_of(x), tensor_of(dy), gamma, beta, mean, rstd, w.c12, act, tensor_of(dx));
            DOL_HIP(hipGetLastError());
        }
    }
    if (params) {
        group_norm_params_kernel<<<dim3((s.channels + 15) / 16, 2), 1024, 0, st>>>(w.sums, s.batch, s.channels, grad_gamma, grad_beta);
        DOL_HIP(hipGetLastError());
    }
    return DOL_OK;
}

// f<T, V>(args) for the type and the vector width of the plan
#define DOL_GN_DISPATCH(f, dtype, vec, ...)                              \
    (dtype == DOL_F32 ? (vec == 4   ? f<float, 4>(__VA_ARGS__)           \
                         : vec == 2 ? f<float, 2>(__VA_ARGS__)           \
                                    : f<float, 1>(__VA_ARGS__))          \
                      : (vec == 8   ? f<__bf16, 8>(__VA_ARGS__)          \
                         : vec == 4 ? f<__bf16, 4>(__VA_ARGS__)          \
                         : vec == 2 ? f<__bf16, 2>(__VA_ARGS__)          \
                                    : f<__bf16, 1>(__VA_ARGS__)))

bool empty(const dol_activations *x) { return x->batch == 0 || x->points == 0 || x->channels == 0; }

}  // namespace
}  // namespace dol

using namespace dol;

extern "C" {

dol_status dol_group_norm_workspace(const dol_activations *x, int32_t groups, int32_t backward, int64_t *bytes)
{
    if (dol_status s = check_call(x, groups, DOL_ACT_NONE)) return s;
    if (!bytes) return fail(DOL_EINVAL, "bytes is NULL");
    *bytes = 0;
    if (!empty(x))      // whichever vectors the call's tensors allow
        for (int vec = 16 / (x->dtype == DOL_F32 ? 4 : 2); vec >= 1; vec /= 2)
            if (x->channels % vec == 0) *bytes = std::max(*bytes, space_of(plan_of(x, groups, vec, backward), backward, nullptr).bytes);
    return DOL_OK;
}

dol_status dol_group_norm(const dol_activations *x, int32_t groups, const float *gamma, const float *beta, float eps, int32_t act, const dol_activations *y, float *mean,
                          float *rstd, void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    if (dol_status s = check_call(x, groups, act)) return s;
    if (dol_status s = check_activations(y, x, "y")) return s;
    if (!(eps >= 0.0f)) return fail(DOL_EINVAL, "eps = %g is not a number of at least 0", static_cast<double>(eps));
    if (empty(x)) return DOL_OK;
    const Plan p = plan_of(x, groups, vector_of(x, y, nullptr), false);
    const Space w = space_of(p, false, workspace);
    if (dol_status s = check_workspace(workspace, workspace_bytes, w.bytes)) return s;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return DOL_GN_DISPATCH(forward, x->dtype, p.vec, p, w, x, gamma, beta, eps, act, y, mean, rstd, st);
}

dol_status dol_group_norm_backward(const dol_activations *x, int32_t groups, const float *gamma, const float *beta, int32_t act, const float *mean, const float *rstd,
                                   const dol_activations *grad_y, const dol_activations *grad_x, float *grad_gamma, float *grad_beta, void *workspace,
                                   int64_t workspace_bytes, void *hip_stream)
{
    if (dol_status s = check_call(x, groups, act)) return s;
    if (dol_status s = check_activations(grad_y, x, "grad_y")) return s;
    if (grad_x)
        if (dol_status s = check_activations(grad_x, x, "grad_x")) return s;
    if (!grad_x && !grad_gamma && !grad_beta) return fail(DOL_EINVAL, "no gradient is asked for");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (empty(x)) {                         // sums over nothing
        if (x->channels == 0) return DOL_OK;
        group_norm_zero_kernel<<<(x->channels + 255) / 256, 256, 0, st>>>(grad_gamma, grad_beta, x->channels);
        DOL_HIP(hipGetLastError());
        return DOL_OK;
    }
    if (!mean || !rstd) return fail(DOL_EINVAL, "mean or rstd is NULL");
    const Plan p = plan_of(x, groups, vector_of(x, grad_y, grad_x), true);
    const Space w = space_of(p, true, workspace);
    if (dol_status s = check_workspace(workspace, workspace_bytes, w.bytes)) return s;
    return DOL_GN_DISPATCH(reverse, x->dtype, p.vec, p, w, x, gamma, beta, mean, rstd, grad_y, act, grad_x, grad_gamma, grad_beta, st);
}

}  // extern "C"
