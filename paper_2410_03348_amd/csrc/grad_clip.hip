// The norm over all gradients of a network together, and the gradients clipped by it.
//
//   norm = sqrt(sum over all buffers and elements of g^2),   coef = min(1, max_norm / (norm + eps)),   out = coef g
//
// Memory bounds it: every gradient is read for the norm, and read and written for the result.  Squares and sums are in 64 bits, so that no
// gradient's square is too large or too small for them; a converted element and its multiply-add cost less than its bytes.
// A list's buffers are cut into chunks, whose table lies on the device.  One launch sums squares, a part for each workgroup; the next has every
// workgroup add up all parts, in the same order, rather than wait for a launch that does.  A small network's gradients are held by one workgroup,
// in one launch.
#include "internal.h"
#include "loose.h"
#include "wave_util.h"

#include <cmath>
#include <mutex>

namespace dol {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kChunk = 8192;        // elements
constexpr int kMostParts = 2048;        // workgroups of a launch: eight of four wavefronts to a unit
constexpr int kSmallThreads = 1024, kSmallEach = 4;             // chunks that a wavefront holds
constexpr int64_t kSmallChunk = 1024;
constexpr int kSmallChunks = kSmallThreads / kWave * kSmallEach;

struct Chunk {
    void *data;
    int32_t n, bf16;
};

}  // namespace
}  // namespace dol

struct dol_tensor_list {
    int device = 0;
    std::vector<int32_t> dtype;
    std::vector<int64_t> size;
    std::vector<void *> data;
    std::vector<int32_t> by_address;    // buffers that hold something, by their first byte
    bool overlaps = false;              // two of them share memory
    int32_t chunks = 0;
    bool small = false;                 // chunks of kSmallChunk, kSmallChunks at most
    dol::DevArray<dol::Chunk> table;
};

namespace dol {
namespace {

// The sum over the workgroup, in every thread; `red` has a place for each wavefront.
template <int THREADS>
__device__ __forceinline__ double sum_of_block(double x, double *red)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) x += __shfl_xor(x, d, kWave);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w) s += red[w];
    return s;
}

// This thread's share of a chunk: its vectors one after the other, f(elements, how many, where they are).
template <typename S, int THREADS, typename F>
__device__ __forceinline__ void each_vector(const S *p, int n, F f)
{
    constexpr int V = kLooseElements<S>;
#pragma unroll 4
    for (int k = threadIdx.x * V; k < n; k += THREADS * V) f(loose_load_end(p + k, n - k, k), n - k, k);
}

template <typename S>
__device__ __forceinline__ void add_vector(const Loose<S> &v, double (&sum)[2])
{
#pragma unroll
    for (int k = 0; k < kLooseElements<S>; ++k) {
        const double x = loose_get(v, k);
        sum[k & 1] = __builtin_fma(x, x, sum[k & 1]);
    }
}

template <typename S>
__device__ __forceinline__ void scale_vector(const Loose<S> &v, float coef, S *to, int n)
{
    float x[kLooseElements<S>];
#pragma unroll
    for (int k = 0; k < kLooseElements<S>; ++k) x[k] = loose_get(v, k) * coef;
    Loose<S> r;
    loose_set(r, x);
    loose_store(to, r, n);
}

template <typename S, int THREADS>
__device__ __forceinline__ void add_squares(const void *data, int n, double (&sum)[2])
{
    each_vector<S, THREADS>(static_cast<const S *>(data), n, [&](const Loose<S> &v, int, int) { add_vector(v, sum); });
}

template <typename S, int THREADS>
__device__ __forceinline__ void scale_chunk(const void *data, void *out, int n, float coef)
{
    S *to = static_cast<S *>(out);
    each_vector<S, THREADS>(static_cast<const S *>(data), n, [&](const Loose<S> &v, int left, int at) { scale_vector(v, coef, to + at, left); });
}

__global__ void __launch_bounds__(kThreads) grad_squares_kernel(const Chunk *table, int chunks, double *part)
{
    __shared__ double red[kThreads / kWave];
    double sum[2] = {0.0, 0.0};
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const Chunk k = table[c];
        if (k.bf16) add_squares<__bf16, kThreads>(k.data, k.n, sum);
        else add_squares<float, kThreads>(k.data, k.n, sum);
    }
    const double s = sum_of_block<kThreads>(sum[0] + sum[1], red);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The sum of all parts, in every thread of the workgroup.
__device__ __forceinline__ double sum_of_parts(const double *part, int parts, double *red)
{
    double s = 0.0;
    for (int k = threadIdx.x; k < parts; k += kThreads) s += part[k];
    return sum_of_block<kThreads>(s, red);
}

__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const double *part, int parts, float *norm)
{
    __shared__ double red[kThreads / kWave];
    const double s = sum_of_parts(part, parts, red);
    if (threadIdx.x == 0) *norm = static_cast<float>(sqrt(s));
}

// (not fminf, which would take 1 for NaN)
__device__ __forceinline__ float coef_of(double norm, double max_norm, double eps)
{
    const double r = max_norm / (norm + eps);
    return r > 1.0 ? 1.0f : static_cast<float>(r);
}

// Chunks are taken from the last on: those that the launch before read last may still be in the caches.
__global__ void __launch_bounds__(kThreads) grad_scale_kernel(const Chunk *table, const Chunk *out, int chunks, const double *part, int parts, double max_norm,
                                                              double eps, float *norm, float *coef)
{
    __shared__ double red[kThreads / kWave];
    const double all = sqrt(sum_of_parts(part, parts, red));
    const float c = coef_of(all, max_norm, eps);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = static_cast<float>(all), *coef = c;
    if (c == 1.0f && table == out) return;
    for (int q = chunks - 1 - blockIdx.x; q >= 0; q -= gridDim.x) {
        const Chunk k = table[q];
        void *to = out[q].data;
        if (k.bf16) scale_chunk<__bf16, kThreads>(k.data, to, k.n, c);
        else scale_chunk<float, kThreads>(k.data, to, k.n, c);
    }
}

// All of it for a list of few chunks, which the wavefronts hold as they lie: coef and out null, only the norm.  5 buffers of 16 234
// floats in all 7.0 us from Python, 10 by the two launches of longer lists.
__global__ void __launch_bounds__(kSmallThreads) grad_small_kernel(const Chunk *table, const Chunk *out, int chunks, double max_norm, double eps, float *norm, float *coef)
{
    __shared__ double red[kSmallThreads / kWave];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int W = kSmallThreads / kWave;
    Chunk chunk[kSmallEach];
    Loose<float> v[kSmallEach][4];              // 1 024 numbers of a float's or (the first two) bf16's vectors
    static_assert(kSmallChunk == 4 * 64 * 4, "a float chunk");
#pragma unroll
    for (int q = 0; q < kSmallEach; ++q) chunk[q] = wave + q * W < chunks ? table[wave + q * W] : Chunk{nullptr, 0, 0};
#pragma unroll
    for (int q = 0; q < kSmallEach; ++q)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = (k * 64 + lane) * (chunk[q].bf16 ? 8 : 4), n = chunk[q].n - at;
            if (chunk[q].bf16) v[q][k] = __builtin_bit_cast(Loose<float>, loose_load_end(static_cast<const __bf16 *>(chunk[q].data) + at, n, at));
            else v[q][k] = loose_load_end(static_cast<const float *>(chunk[q].data) + at, n, at);
        }
    double sum[2] = {0.0, 0.0};
#pragma unroll
    for (int q = 0; q < kSmallEach; ++q)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (chunk[q].bf16) add_vector(__builtin_bit_cast(Loose<__bf16>, v[q][k]), sum);
            else add_vector(v[q][k], sum);
        }
    const double all = sqrt(sum_of_block<kSmallThreads>(sum[0] + sum[1], red));
    if (threadIdx.x == 0) *norm = static_cast<float>(all);
    if (!coef) return;
    const float c = coef_of(all, max_norm, eps);
    if (threadIdx.x == 0) *coef = c;
    if (c == 1.0f && table == out) return;
#pragma unroll
    for (int q = 0; q < kSmallEach; ++q) {
        if (chunk[q].n == 0) continue;
        void *to = out[wave + q * W].data;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = (k * 64 + lane) * (chunk[q].bf16 ? 8 : 4), n = chunk[q].n - at;
            if (n <= 0) continue;
            if (chunk[q].bf16) scale_vector(__builtin_bit_cast(Loose<__bf16>, v[q][k]), c, static_cast<__bf16 *>(to) + at, n);
            else scale_vector(v[q][k], c, static_cast<float *>(to) + at, n);
        }
    }
}

int parts_of(const dol_tensor_list *l) { return std::min(l->chunks, kMostParts); }

dol_status check_list(const dol_tensor_list *l, const char *name)
{
    if (!l) return fail(DOL_EINVAL, "%s is NULL", name);
    int device = 0;
    DOL_HIP(hipGetDevice(&device));
    if (device != l->device) return fail(DOL_EINVAL, "%s was made on device %d, the current one is %d", name, l->device, device);
    return DOL_OK;
}

const char *end_of(const dol_tensor_list *l, int32_t t) { return static_cast<const char *>(l->data[t]) + l->size[t] * (l->dtype[t] == DOL_F32 ? 4 : 2); }

// Whether a buffer of one list shares memory with another than its own, which is the whole of it, of the other list.
bool crossed(const dol_tensor_list *a, const dol_tensor_list *b)
{
    size_t i = 0, j = 0;
    while (i < a->by_address.size() && j < b->by_address.size()) {
        const int32_t s = a->by_address[i], t = b->by_address[j];
        const char *sb = static_cast<const char *>(a->data[s]), *tb = static_cast<const char *>(b->data[t]), *se = end_of(a, s), *te = end_of(b, t);
        if (sb < te && tb < se && (s != t || sb != tb)) return true;
        if (se <= te) ++i;
        else ++j;
    }
    return false;
}

dol_status sum_squares(const dol_tensor_list *l, double *part, hipStream_t st)
{
    grad_squares_kernel<<<parts_of(l), kThreads, 0, st>>>(l->table.ptr, l->chunks, part);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

}  // namespace
}  // namespace dol

using namespace dol;

extern "C" {

dol_status dol_tensor_list_create(int32_t count, const int32_t *dtype, const int64_t *size, void *const *data, dol_tensor_list **list)
{
    if (!list) return fail(DOL_EINVAL, "list is NULL");
    *list = nullptr;
    if (count < 0) return fail(DOL_EINVAL, "count = %d is negative", count);
    if (count > 0 && (!dtype || !size || !data)) return fail(DOL_EINVAL, "dtype, size or data is NULL");
    int64_t chunks = 0, small = 0;
    for (int32_t t = 0; t < count; ++t) {
        if (dtype[t] != DOL_F32 && dtype[t] != DOL_BF16) return fail(DOL_EINVAL, "buffer %d has unknown type %d", t, dtype[t]);
        if (size[t] < 0) return fail(DOL_ESHAPE, "buffer %d has %lld elements", t, static_cast<long long>(size[t]));
        if (size[t] == 0) continue;
        if (!data[t]) return fail(DOL_EINVAL, "buffer %d is NULL", t);
        if (reinterpret_cast<uintptr_t>(data[t]) & (dtype[t] == DOL_F32 ? 3 : 1)) return fail(DOL_EINVAL, "buffer %d is not aligned to its elements", t);
        const int64_t n = size[t] / kChunk + (size[t] % kChunk != 0);
        if (n > INT32_MAX - chunks) return fail(DOL_EUNSUPPORTED, "the buffers have more than %lld elements", static_cast<long long>(kChunk) * INT32_MAX);
        chunks += n;
        small = std::min<int64_t>(small + size[t] / kSmallChunk + (size[t] % kSmallChunk != 0), INT32_MAX);
    }
    const bool few = small <= kSmallChunks;
    const int64_t each = few ? kSmallChunk : kChunk;
    if (few) chunks = small;
    try {
        auto l = std::make_unique<dol_tensor_list>();
        DOL_HIP(hipGetDevice(&l->device));
        l->chunks = static_cast<int32_t>(chunks), l->small = few;
        l->dtype.assign(dtype, dtype + count), l->size.assign(size, size + count), l->data.assign(data, data + count);
        std::vector<Chunk> table;
        table.reserve(chunks);
        for (int32_t t = 0; t < count; ++t) {
            if (size[t] == 0) continue;
            l->by_address.push_back(t);
            for (int64_t at = 0; at < size[t]; at += each)
                table.push_back(Chunk{static_cast<char *>(data[t]) + at * (dtype[t] == DOL_F32 ? 4 : 2), static_cast<int32_t>(std::min(each, size[t] - at)), dtype[t] == DOL_BF16});
        }
        std::sort(l->by_address.begin(), l->by_address.end(), [&](int32_t a, int32_t b) { return std::less<void *>()(data[a], data[b]); });
        for (size_t k = 1; k < l->by_address.size(); ++k)
            if (end_of(l.get(), l->by_address[k - 1]) > static_cast<const char *>(data[l->by_address[k]])) l->overlaps = true;
        if (l->table.upload(table) != hipSuccess) return fail(DOL_ENOMEM, "no memory for a list of %d buffers", count);
        *list = l.release();
    } catch (const std::bad_alloc &) {
        return fail(DOL_ENOMEM, "no memory for a list of %d buffers", count);
    }
    return DOL_OK;
}

void dol_tensor_list_destroy(dol_tensor_list *list) { delete list; }

dol_status dol_grad_norm_workspace(const dol_tensor_list *grads, int64_t *bytes)
{
    if (!grads) return fail(DOL_EINVAL, "grads is NULL");
    if (!bytes) return fail(DOL_EINVAL, "bytes is NULL");
    *bytes = grads->small ? 0 : round_up(parts_of(grads) * static_cast<int64_t>(sizeof(double)), 256);
    return DOL_OK;
}

dol_status dol_grad_norm(const dol_tensor_list *grads, float *norm, void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    if (dol_status s = check_list(grads, "grads")) return s;
    if (!norm) return fail(DOL_EINVAL, "norm is NULL");
    int64_t need = 0;
    if (dol_status s = dol_grad_norm_workspace(grads, &need)) return s;
    if (dol_status s = check_workspace(workspace, workspace_bytes, need)) return s;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (grads->small) {
        grad_small_kernel<<<1, kSmallThreads, 0, st>>>(grads->table.ptr, nullptr, grads->chunks, 0.0, 0.0, norm, nullptr);
        DOL_HIP(hipGetLastError());
        return DOL_OK;
    }
    double *part = static_cast<double *>(workspace);
    if (dol_status s = sum_squares(grads, part, st)) return s;
    grad_norm_kernel<<<1, kThreads, 0, st>>>(part, parts_of(grads), norm);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

dol_status dol_clip_grads(const dol_tensor_list *grads, const dol_tensor_list *out, double max_norm, double eps, float *norm, float *coef, void *workspace,
                          int64_t workspace_bytes, void *hip_stream)
{
    if (dol_status s = check_list(grads, "grads")) return s;
    if (dol_status s = check_list(out, "out")) return s;
    if (!norm || !coef) return fail(DOL_EINVAL, "norm or coef is NULL");
    if (!(max_norm >= 0.0)) return fail(DOL_EINVAL, "max_norm = %g is not a number of at least 0", max_norm);
    if (!(eps >= 0.0)) return fail(DOL_EINVAL, "eps = %g is not a number of at least 0", eps);
    if (out != grads && (out->dtype != grads->dtype || out->size != grads->size)) return fail(DOL_ESHAPE, "grads and out differ in their buffers' number, types or sizes");
    if (grads->overlaps) return fail(DOL_EINVAL, "two buffers of grads share memory");
    if (out->overlaps) return fail(DOL_EINVAL, "two buffers of out share memory");
    if (out != grads && crossed(grads, out)) return fail(DOL_EINVAL, "a buffer of grads shares memory with another one of out");
    int64_t need = 0;
    if (dol_status s = dol_grad_norm_workspace(grads, &need)) return s;
    if (dol_status s = check_workspace(workspace, workspace_bytes, need)) return s;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (grads->small) {
        grad_small_kernel<<<1, kSmallThreads, 0, st>>>(grads->table.ptr, out->table.ptr, grads->chunks, max_norm, eps, norm, coef);
        DOL_HIP(hipGetLastError());
        return DOL_OK;
    }
    double *part = static_cast<double *>(workspace);
    if (dol_status s = sum_squares(grads, part, st)) return s;
    grad_scale_kernel<<<parts_of(grads), kThreads, 0, st>>>(grads->table.ptr, out->table.ptr, grads->chunks, part, parts_of(grads), max_norm, eps, norm, coef);
    DOL_HIP(hipGetLastError());
    return DOL_OK;
}

}  // extern "C"
