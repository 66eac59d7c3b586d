// Rows of channels, whatever their width and wherever they begin: a thread takes VEC adjacent channels of one.
//
// The memory instructions take any address, so that neither strides nor odd widths send a row through them value by value.  (Norm, 8,192 rows of 4,095 channels
// in bf16: one by one 85 us, so 47, of 4,096 channels 40; with 8 bits and a scale for every 128 of them 174, 48 and 42.)
#pragma once
#include "cawn_ops.hpp"

namespace cawn {
namespace ops {

// Adjacent elements wherever they begin: the memory instructions take any address.
template <typename T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Loose { T v[N]; };

// N adjacent elements, 16 bytes an access at most
template <typename T, int N> __device__ inline void read_n(const T *p, float (&x)[N])
{
    constexpr int W = N * sizeof(T) <= 16 ? N : 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < N; i += W) {
        const Loose<T, W> a = *reinterpret_cast<const Loose<T, W> *>(p + i);
#pragma unroll
        for (int j = 0; j < W; ++j) x[i + j] = (float)a.v[j];
    }
}
// ... all but the first `skip`
template <typename T, int N> __device__ inline void write_n(T *p, const float (&x)[N], int skip)
{
    constexpr int W = N * sizeof(T) <= 16 ? N : 16 / sizeof(T);
    if (skip) {
#pragma unroll
        for (int i = 1; i < N; ++i)
            if (i >= skip) p[i] = (T)x[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < N; i += W) {
        Loose<T, W> a;
#pragma unroll
        for (int j = 0; j < W; ++j) a.v[j] = (T)x[i + j];
        *reinterpret_cast<Loose<T, W> *>(p + i) = a;
    }
}

// A thread's VEC channels of a row.  TAIL: rows are no multiple of VEC, and the last unit ends with the row: its first `skip` channels are the unit's before
// it, are left out of sums and not written.
template <int VEC, bool TAIL> struct Unit {
    int c, at, skip;        // first channel read; first channel that is its own, c + skip, if the unit exists
    bool in;
    __device__ Unit() {}
    __device__ Unit(int u, int C) : at(u * VEC), in(at < C)
    {
        c = TAIL ? min(at, C - VEC) : in ? at : 0;
        skip = TAIL ? min(at - c, VEC) : 0;
    }
    // what is not its own, 0
    __device__ inline void own(float (&x)[VEC], bool live) const
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[i] = live && (!TAIL || i >= skip) ? x[i] : 0.f;
    }
};

} // namespace ops
} // namespace cawn
