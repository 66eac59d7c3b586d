// Dropout joined with the residual addition; the mask is a function of the element's number and is never stored.
//
// Philox-4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011): ten rounds of two 32 x 32 -> 64 bit products turn the 128-bit counter
// (number of the block of four elements, 0) under a 64-bit key into four random words.
//
// Bound by memory: 65,536 x 768 in bf16, forward and backward, 0.50 GB in 100 us, 5.0 TB/s (a large copy reaches 5.2); 1,021 x 97 in fp32 8 us,
// two launches.
#include "cawn_ops.hpp"

using namespace cawn::ops;

namespace {

struct DropArgs {
    const void *x, *residual;
    void *y;
    const uint64_t *rng;
    long long rows, cols, xs, rs, ys;
    uint32_t threshold;
    int all;                // p = 1: nothing is kept
    float scale;
};

__device__ inline void philox(uint64_t block, uint32_t k0, uint32_t k1, uint32_t (&w)[4])
{
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = 0, c3 = 0;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    w[0] = c0, w[1] = c1, w[2] = c2, w[3] = c3;
}

// A thread's unit is VEC adjacent elements of a row that begin on a multiple of four: VEC / 4 blocks.
template <typename T, int VEC, bool RES> __global__ __launch_bounds__(256) void dropout_units(const DropArgs a)
{
    const long long per_row = (a.cols + VEC - 1) / VEC, n = a.rows * per_row;
    const uint64_t seed = a.rng[0], offset = a.rng[1];
    for (long long u = (long long)blockIdx.x * 256 + threadIdx.x; u < n; u += (long long)gridDim.x * 256) {
        const long long r = a.rows == 1 ? 0 : u / per_row, c = (u - r * per_row) * VEC;
        const T *x = (const T *)a.x + r * a.xs + c;
        const T *res = RES ? (const T *)a.residual + r * a.rs + c : nullptr;
        T *y = (T *)a.y + r * a.ys + c;
        const uint64_t block = offset + (uint64_t)(r * a.cols + c) / 4;
        float xv[VEC], rv[VEC];
        const bool whole = c + VEC <= a.cols;
        if (whole) {
            load_n<T, VEC>(x, xv);
            if (RES) load_n<T, VEC>(res, rv);
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                xv[i] = c + i < a.cols ? (float)x[i] : 0.f;
                if (RES) rv[i] = c + i < a.cols ? (float)res[i] : 0.f;
            }
        }
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) {
            uint32_t w[4];
            philox(block + q, (uint32_t)seed, (uint32_t)(seed >> 32), w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float kept = !a.all && w[i] >= a.threshold ? xv[4 * q + i] * a.scale : 0.f;
                xv[4 * q + i] = RES ? rv[4 * q + i] + kept : kept;
            }
        }
        if (whole) store_n<T, VEC>(y, xv);
        else {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (c + i < a.cols) y[i] = (T)xv[i];
        }
    }
}

// Rows that no unit may begin in (their length or stride is no multiple of the unit, or their address is not aligned): a thread
// takes one block of four elements, wherever its rows end.  (65,536 x 768 in bf16, which the units take in 99 us, in 204.)
template <typename T, bool RES> __global__ __launch_bounds__(256) void dropout_elements(const DropArgs a)
{
    const long long n = a.rows * a.cols, blocks = (n + 3) / 4;
    const uint64_t seed = a.rng[0], offset = a.rng[1];
    for (long long u = (long long)blockIdx.x * 256 + threadIdx.x; u < blocks; u += (long long)gridDim.x * 256) {
        uint32_t w[4];
        philox(offset + (uint64_t)u, (uint32_t)seed, (uint32_t)(seed >> 32), w);
        long long r = 4 * u / a.cols, c = 4 * u - r * a.cols;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (4 * u + i < n) {
                const float kept = !a.all && w[i] >= a.threshold ? (float)((const T *)a.x)[r * a.xs + c] * a.scale : 0.f;
                ((T *)a.y)[r * a.ys + c] = (T)(RES ? (float)((const T *)a.residual)[r * a.rs + c] + kept : kept);
            }
            if (++c == a.cols) c = 0, ++r;
        }
    }
}

template <typename T> int launch(DropArgs a, bool res, hipStream_t s)
{
    constexpr int VEC = 16 / sizeof(T);
    // dense rows are one row: units then begin anywhere in it
    if (a.xs == a.cols && a.ys == a.cols && (!res || a.rs == a.cols)) {
        a.cols *= a.rows, a.rows = 1;
        a.xs = a.ys = a.rs = 0;
    }
    const bool units = (a.rows == 1 || (a.cols % VEC == 0 && a.xs % VEC == 0 && a.ys % VEC == 0 && (!res || a.rs % VEC == 0))) &&
                       aligned_to(a.x, 16) && aligned_to(a.y, 16) && (!res || aligned_to(a.residual, 16));
    const long long n = units ? a.rows * ceil_div(a.cols, VEC) : ceil_div(a.rows * a.cols, 4);
    const long long blocks = ceil_div(n, 256);
    const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)));
    if (units) {
        if (res) hipLaunchKernelGGL((dropout_units<T, VEC, true>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((dropout_units<T, VEC, false>), grid, dim3(256), 0, s, a);
    } else {
        if (res) hipLaunchKernelGGL((dropout_elements<T, true>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((dropout_elements<T, false>), grid, dim3(256), 0, s, a);
    }
    return launched();
}

int check_and_launch(const cawn_dropout_desc *d, const void *x, const void *residual, const uint64_t *rng, void *y, long long xs, long long ys, void *stream)
{
    if (!d || d->rows < 0 || d->cols < 0 || !(d->p >= 0.0 && d->p <= 1.0) || (d->bf16 & ~1)) return CAWN_EINVAL;
    if (d->rows > 0 && d->cols > (1LL << 60) / d->rows) return CAWN_EUNSUPPORTED;
    DropArgs a{x, residual, y, rng, d->rows, d->cols, xs ? xs : d->cols, d->residual_stride ? d->residual_stride : d->cols, ys ? ys : d->cols, 0, 0, 0.f};
    if (d->rows > 1 && (a.xs < a.cols || a.ys < a.cols || (residual && a.rs < a.cols))) return CAWN_EINVAL;
    if (d->rows == 0 || d->cols == 0) return CAWN_OK;
    if (!x || !rng || !y) return CAWN_EINVAL;
    if (!aligned_to(rng, 8) || !aligned_to(x, d->bf16 ? 2 : 4) || !aligned_to(y, d->bf16 ? 2 : 4) || !aligned_to(residual, d->bf16 ? 2 : 4)) return CAWN_EINVAL;
    a.all = d->p >= 1.0;
    a.threshold = a.all ? 0u : (uint32_t)(d->p * 4294967296.0);
    a.scale = a.all ? 0.f : (float)(1.0 / (1.0 - d->p));
    return d->bf16 ? launch<bf16>(a, residual != nullptr, (hipStream_t)stream) : launch<float>(a, residual != nullptr, (hipStream_t)stream);
}

} // namespace

extern "C" {

int cawn_dropout_add_fwd(const cawn_dropout_desc *d, const void *x, const void *residual, const uint64_t *rng, void *y, void *stream)
{
    return check_and_launch(d, x, residual, rng, y, d ? d->x_stride : 0, d ? d->y_stride : 0, stream);
}

int cawn_dropout_add_bwd(const cawn_dropout_desc *d, const void *dy, const uint64_t *rng, void *dx, void *stream)
{
    return check_and_launch(d, dy, nullptr, rng, dx, d ? d->y_stride : 0, d ? d->x_stride : 0, stream);
}

} // extern "C"
