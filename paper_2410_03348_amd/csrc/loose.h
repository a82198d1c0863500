// Vectors of 16 bytes of a tensor whose elements alone are aligned (rows of odd lengths, views into a buffer of many tensors): one load or
// store all the same, which global memory takes at any address.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace dol {

template <typename S>
struct __attribute__((packed, aligned(sizeof(S)))) Loose {
    uint32_t w[4];
};

// Elements of a vector.
template <typename S>
constexpr int kLooseElements = 16 / static_cast<int>(sizeof(S));

template <typename S>
__device__ __forceinline__ float loose_get(const Loose<S> &v, int k)
{
    if constexpr (sizeof(S) == 4) return __uint_as_float(v.w[k]);
    else return __uint_as_float(k & 1 ? v.w[k >> 1] & 0xFFFF0000u : v.w[k >> 1] << 16);
}

template <typename S>
__device__ __forceinline__ void loose_set(Loose<S> &v, const float (&x)[kLooseElements<S>])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(S) == 4) v.w[k] = __float_as_uint(x[k]);
        else v.w[k] = __builtin_bit_cast(uint16_t, static_cast<S>(x[2 * k])) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<S>(x[2 * k + 1]))) << 16;
    }
}

// The first n elements at p (a vector's at most), zeros behind them; n may be below 1.
template <typename S>
__device__ __forceinline__ Loose<S> loose_load(const S *p, int64_t n)
{
    constexpr int V = kLooseElements<S>;
    if (n >= V) return *reinterpret_cast<const Loose<S> *>(p);
    Loose<S> v{};
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (k < n) {
            if constexpr (sizeof(S) == 4) v.w[k] = __builtin_bit_cast(uint32_t, p[k]);
            else v.w[k >> 1] |= static_cast<uint32_t>(__builtin_bit_cast(uint16_t, p[k])) << (k & 1) * 16;
        }
    return v;
}

// v's elements from the k-th on (k > 0), zeros behind them.
template <typename S>
__device__ __forceinline__ Loose<S> loose_from(const Loose<S> &v, int k)
{
    const int bytes = k * static_cast<int>(sizeof(S));
    Loose<S> r = v;
    // (by eight, four and two of them: one shift of the whole would hold twice the registers)
    if (bytes & 8) r.w[0] = r.w[2], r.w[1] = r.w[3], r.w[2] = r.w[3] = 0;
    if (bytes & 4) r.w[0] = r.w[1], r.w[1] = r.w[2], r.w[2] = r.w[3], r.w[3] = 0;
    if (sizeof(S) == 2 && (bytes & 2))
        r.w[0] = r.w[0] >> 16 | r.w[1] << 16, r.w[1] = r.w[1] >> 16 | r.w[2] << 16, r.w[2] = r.w[2] >> 16 | r.w[3] << 16, r.w[3] >>= 16;
    if (bytes >= 16) r.w[0] = r.w[1] = r.w[2] = r.w[3] = 0;
    return r;
}

// The first n elements at p where `before` elements of the row lie before it: the row's last vector, shifted, is one load, where one of each element would
// wait for the one before it.
template <typename S>
__device__ __forceinline__ Loose<S> loose_load_end(const S *p, int n, int before)
{
    constexpr int V = kLooseElements<S>;
    if (n >= V) return *reinterpret_cast<const Loose<S> *>(p);
    if (n <= 0) return Loose<S>{};
    if (before + n < V) return loose_load(p, n);
    return loose_from(*reinterpret_cast<const Loose<S> *>(p - (V - n)), V - n);
}

template <typename S>
__device__ __forceinline__ void loose_store(S *p, const Loose<S> &v, int64_t n)
{
    constexpr int V = kLooseElements<S>;
    if (n >= V) {
        *reinterpret_cast<Loose<S> *>(p) = v;
        return;
    }
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (k < n) {
            if constexpr (sizeof(S) == 4) p[k] = __builtin_bit_cast(S, v.w[k]);
            else p[k] = __builtin_bit_cast(S, static_cast<uint16_t>(v.w[k >> 1] >> (k & 1) * 16));
        }
}

}  // namespace dol
