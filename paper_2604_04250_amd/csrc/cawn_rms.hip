// Root-mean-square norm joined with the residual addition in front of it, forward and backward, its output in 8 bits among them.
//
// Forward: h = x + residual, rounded to h's type; y = w h rstd, rstd = 1 / sqrt(mean h^2 + eps); q = e4m3(y / scale), scale = max |y| / 448 over a block.
// Backward: hh = h rstd, t = w dy, dr = dh + rstd (t - hh avg(t hh)), dw = sum dy hh.
//
// A row is in registers from its one read to its write: a run of 4 to 64 lanes holds it, or a workgroup of 256 to 1,024; the longest, beyond 16,384 channels, are
// read again.  Bound by memory: 65,536 rows of 768 channels in bf16 with an fp32 residual forward 115 us (5.2 TB/s), backward 155 (5.2); 32,768 rows of 4,096 with
// 8 bits and a scale for 128 channels 172 (5.5).  Wide rows of an odd width begin between the 16 bytes of an access: 4,096 rows of 12,001 channels in bf16 forward 114,
// backward 160 (3.4, 3.1), of 12,000 84 and 111.  A few rows are a launch: 4 of 768 4.6.
// The sum of squares is plain: all of its terms have one sign.
#include "cawn_rows.hpp"
#include "cawn_sums.hpp"

using namespace cawn::ops;

namespace {

struct RmsArgs {
    const void *x, *res, *dy, *dh;
    const float *w, *rstd_in;
    void *h, *y, *dx, *dres;
    uint8_t *q;
    float *scales, *rstd, *part;
    long long rows, xs, rs, ys;
    int C, block, blocks;       // channels of a scale, scales of a row
    int lpr, rpw;               // lanes of a row, rows that a workgroup has at once
    int lpb;                    // lanes that share a scale (a power of two up to 64, within a row's), 0: by way of LDS
    float eps;
};

constexpr float E4M3_MAX = 448.f;

__device__ inline float nan_max(float a, float b) { return a >= b || a != a ? a : b; }      // a NaN stays
template <bool MAX> __device__ inline float two(float a, float b) { return MAX ? nan_max(a, b) : a + b; }

// sum or maximum over the run of `lanes` (a power of two) adjacent lanes, in every one of them
template <bool MAX> __device__ inline float over_run(float v, int lanes)
{
    for (int m = lanes >> 1; m > 0; m >>= 1) v = two<MAX>(v, __shfl_xor(v, m));
    return v;
}

// ... over a row: its run of lanes, or the workgroup
template <bool WIDE, bool MAX> __device__ inline float over_row(float v, int lpr, float *sh)
{
    v = over_run<MAX>(v, WIDE ? 64 : lpr);
    if (!WIDE) return v;
    __syncthreads();                // (what the last call left has been read)
    if (threadIdx.x % 64 == 0) sh[threadIdx.x / 64] = v;
    __syncthreads();
    v = sh[0];
    for (int i = 1; i < (int)blockDim.x / 64; ++i) v = two<MAX>(v, sh[i]);
    return v;
}

// four values as e4m3, rounded to nearest even
__device__ inline uint32_t e4m3_4(float a, float b, float c, float d)
{
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

// Scale of a block whose largest magnitude is m; 0 for one of zeros, or of values so small that the scale would lose its digits.
__device__ inline float scale_of(float m) { return m < E4M3_MAX * 1.17549435e-38f ? 0.f : m / E4M3_MAX; }

// VEC values y of the type's 8 bits
template <int VEC> __device__ inline void write_q(uint8_t *q, const float (&y)[VEC], float scale, int skip)
{
    float v[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = scale == 0.f ? 0.f : y[i] / scale;
    if constexpr (VEC == 1) *q = (uint8_t)(e4m3_4(v[0], 0.f, 0.f, 0.f) & 0xff);
    else {
        Loose<uint32_t, VEC / 4> b;
#pragma unroll
        for (int i = 0; i < VEC; i += 4) b.v[i / 4] = e4m3_4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        if (skip) {
#pragma unroll
            for (int i = 1; i < VEC; ++i)
                if (i >= skip) q[i] = (uint8_t)(b.v[i / 4] >> i % 4 * 8);
        } else *reinterpret_cast<Loose<uint8_t, VEC> *>(q) = __builtin_bit_cast(Loose<uint8_t, VEC>, b);
    }
}

template <int VEC> __device__ inline void read_w(const RmsArgs &a, int c, float (&w)[VEC])
{
    if (a.w) read_n<float, VEC>(a.w + c, w);
    else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) w[i] = 1.f;
    }
}

// VEC values of h, as they are kept
template <typename X, typename R, int VEC> __device__ inline void read_h(const RmsArgs &a, long long r, int c, float (&h)[VEC])
{
    read_n<X, VEC>((const X *)a.x + r * a.xs + c, h);
    if (a.res) {
        float v[VEC];
        read_n<R, VEC>((const R *)a.res + r * a.rs + c, v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) h[i] += v[i];
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) h[i] = (float)(R)h[i];
}

template <int VEC> __device__ inline float largest(const float (&y)[VEC])
{
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < VEC; ++i) m = nan_max(fabsf(y[i]), m);
    return m;
}

// X, R: types of x, y and of the residual stream.  WIDE: a row is the workgroup's.
template <typename X, typename R, int VEC, bool TAIL, int NIT, bool WIDE, int THREADS> __global__ __launch_bounds__(THREADS) void rms_forward(const RmsArgs a)
{
    __shared__ float sh[WIDE ? THREADS / 64 : 1];
    __shared__ uint32_t most[THREADS * NIT * VEC / 16 + 256];     // maxima of the blocks, as the bits of values without a sign
    const int run = WIDE ? 0 : threadIdx.x / a.lpr, lane = WIDE ? threadIdx.x : threadIdx.x % a.lpr;
    const int step = WIDE ? THREADS : a.lpr;
    float w[NIT][VEC];
    Unit<VEC, TAIL> u[NIT];
#pragma unroll
    for (int n = 0; n < NIT; ++n) {
        u[n] = Unit<VEC, TAIL>(n * step + lane, a.C);
        read_w<VEC>(a, u[n].c, w[n]);
    }
    const long long stride = (long long)gridDim.x * a.rpw;
    const float inv = 1.f / (float)a.C;
    // (all runs of a workgroup go round equally often: there are barriers inside)
    for (long long r0 = (long long)blockIdx.x * a.rpw; r0 < a.rows; r0 += stride) {
        const bool live = r0 + run < a.rows;
        const long long r = live ? r0 + run : r0;
        float h[NIT][VEC], s = 0.f;
#pragma unroll
        for (int n = 0; n < NIT; ++n) {
            read_h<X, R, VEC>(a, r, u[n].c, h[n]);
            u[n].own(h[n], u[n].in);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s = fmaf(h[n][i], h[n][i], s);
        }
        const float rstd = 1.f / sqrtf(over_row<WIDE, false>(s, a.lpr, sh) * inv + a.eps);
        if (live && lane == 0 && a.rstd) a.rstd[r] = rstd;
#pragma unroll
        for (int n = 0; n < NIT; ++n) {
            if (live && u[n].in && a.h) write_n<R, VEC>((R *)a.h + r * a.rs + u[n].c, h[n], u[n].skip);
#pragma unroll
            for (int i = 0; i < VEC; ++i) h[n][i] = h[n][i] * rstd * w[n][i];
            if (live && u[n].in && a.y) write_n<X, VEC>((X *)a.y + r * a.ys + u[n].c, h[n], u[n].skip);
        }
        if (!a.q) continue;
        float m[NIT];
#pragma unroll
        for (int n = 0; n < NIT; ++n) {
            u[n].own(h[n], u[n].in);       // (0 times an infinite weight or rstd is none)
            m[n] = largest<VEC>(h[n]);
        }
        if (a.block == 0) {
            float t = m[0];
#pragma unroll
            for (int n = 1; n < NIT; ++n) t = nan_max(m[n], t);
            t = over_row<WIDE, true>(t, a.lpr, sh);
#pragma unroll
            for (int n = 0; n < NIT; ++n) m[n] = t;
        } else if (a.lpb > 0) {
#pragma unroll
            for (int n = 0; n < NIT; ++n) m[n] = over_run<true>(m[n], a.lpb);
        } else {
            __syncthreads();
            for (int i = threadIdx.x; i < a.blocks * a.rpw; i += THREADS) most[i] = 0;
            __syncthreads();
#pragma unroll
            for (int n = 0; n < NIT; ++n) {
                // (a block is a multiple of 16 channels: of VEC)
                if (u[n].in && live) atomicMax(&most[run * a.blocks + u[n].at / a.block], __float_as_uint(m[n]) & 0x7fffffffu);
            }
            __syncthreads();
#pragma unroll
            for (int n = 0; n < NIT; ++n) {
                if (u[n].in && live) m[n] = __uint_as_float(most[run * a.blocks + u[n].at / a.block]);
            }
        }
#pragma unroll
        for (int n = 0; n < NIT; ++n) {
            if (!live || !u[n].in) continue;
            const float scale = scale_of(m[n]);
            const int j = a.block ? u[n].at / a.block : 0;
            if (u[n].at == j * a.block) a.scales[r * a.blocks + j] = scale;
            write_q<VEC>(a.q + r * a.ys + u[n].c, h[n], scale, u[n].skip);
        }
    }
}

// Rows that no workgroup's registers hold: read twice, three times where 8 bits are asked for.
template <typename X, typename R, int VEC, bool TAIL> __global__ __launch_bounds__(1024) void rms_forward_long(const RmsArgs a)
{
    __shared__ float sh[16];
    __shared__ uint32_t most[2048];
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
        float s = 0.f;
        for (Unit<VEC, TAIL> u(threadIdx.x, a.C); u.in; u = Unit<VEC, TAIL>(u.at / VEC + 1024, a.C)) {
            float h[VEC];
            read_h<X, R, VEC>(a, r, u.c, h);
            u.own(h, true);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s = fmaf(h[i], h[i], s);
        }
        const float rstd = 1.f / sqrtf(over_row<true, false>(s, 0, sh) / (float)a.C + a.eps);
        if (threadIdx.x == 0 && a.rstd) a.rstd[r] = rstd;
        const int per = a.block ? a.block : a.C;
        float whole = 0.f;
        // (h or y may lie where x or the residual did: nothing is written before the last reading, and there by the thread that has read it)
        auto norm = [&](const Unit<VEC, TAIL> &u, float(&h)[VEC]) {
            float w[VEC];
            read_w<VEC>(a, u.c, w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) h[i] = h[i] * rstd * w[i];
            u.own(h, true);
        };
        if (a.q) {
            __syncthreads();
            for (int i = threadIdx.x; i < a.blocks; i += 1024) most[i] = 0;
            __syncthreads();
            for (Unit<VEC, TAIL> u(threadIdx.x, a.C); u.in; u = Unit<VEC, TAIL>(u.at / VEC + 1024, a.C)) {
                float h[VEC];
                read_h<X, R, VEC>(a, r, u.c, h);
                norm(u, h);
                const float m = largest<VEC>(h);
                if (a.block) atomicMax(&most[u.at / per], __float_as_uint(m) & 0x7fffffffu);
                else whole = nan_max(m, whole);
            }
            __syncthreads();
            if (!a.block) whole = over_row<true, true>(whole, 0, sh);
        }
        for (Unit<VEC, TAIL> u(threadIdx.x, a.C); u.in; u = Unit<VEC, TAIL>(u.at / VEC + 1024, a.C)) {
            float h[VEC];
            read_h<X, R, VEC>(a, r, u.c, h);
            if (a.h) write_n<R, VEC>((R *)a.h + r * a.rs + u.c, h, u.skip);
            norm(u, h);
            if (a.y) write_n<X, VEC>((X *)a.y + r * a.ys + u.c, h, u.skip);
            if (a.q) {
                const float scale = scale_of(a.block ? __uint_as_float(most[u.at / per]) : whole);
                if (u.at % per == 0) a.scales[r * a.blocks + u.at / per] = scale;
                write_q<VEC>(a.q + r * a.ys + u.c, h, scale, u.skip);
            }
        }
    }
}

// VEC values of hh and of t = w dy
template <typename X, typename R, int VEC> __device__ inline void read_back(const RmsArgs &a, long long r, int c, float rstd, float (&h)[VEC], float (&t)[VEC])
{
    read_n<R, VEC>((const R *)a.x + r * a.rs + c, h);
    read_n<X, VEC>((const X *)a.dy + r * a.ys + c, t);
#pragma unroll
    for (int i = 0; i < VEC; ++i) h[i] *= rstd;
}

// dr of VEC values, into dx and dresidual
template <typename X, typename R, int VEC> __device__ inline void write_back(const RmsArgs &a, long long r, int c, float rstd, float s, const float (&h)[VEC], const float (&t)[VEC],
                                                                                int skip)
{
    float d[VEC];
    if (a.dh) read_n<R, VEC>((const R *)a.dh + r * a.rs + c, d);
#pragma unroll
    for (int i = 0; i < VEC; ++i) d[i] = fmaf(rstd, fmaf(-h[i], s, t[i]), a.dh ? d[i] : 0.f);
    if (a.dx) write_n<X, VEC>((X *)a.dx + r * a.xs + c, d, skip);
    if (a.dres) write_n<R, VEC>((R *)a.dres + r * a.rs + c, d, skip);
}

template <typename X, typename R, int VEC, bool TAIL, int NIT, bool WIDE, int THREADS> __global__ __launch_bounds__(THREADS) void rms_backward(const RmsArgs a)
{
    __shared__ float sh[WIDE ? THREADS / 64 : THREADS * NIT * VEC];
    const int run = WIDE ? 0 : threadIdx.x / a.lpr, lane = WIDE ? threadIdx.x : threadIdx.x % a.lpr;
    const int step = WIDE ? THREADS : a.lpr;
    float w[NIT][VEC], sw[NIT][VEC];
    Unit<VEC, TAIL> u[NIT];
#pragma unroll
    for (int n = 0; n < NIT; ++n) {
        u[n] = Unit<VEC, TAIL>(n * step + lane, a.C);
        read_w<VEC>(a, u[n].c, w[n]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) sw[n][i] = 0.f;
    }
    const long long stride = (long long)gridDim.x * a.rpw;
    const float inv = 1.f / (float)a.C;
    for (long long r0 = (long long)blockIdx.x * a.rpw; r0 < a.rows; r0 += stride) {
        const bool live = r0 + run < a.rows;
        const long long r = live ? r0 + run : r0;
        const float rstd = a.rstd_in[r];
        float h[NIT][VEC], t[NIT][VEC], s = 0.f;
#pragma unroll
        for (int n = 0; n < NIT; ++n) {
            read_back<X, R, VEC>(a, r, u[n].c, rstd, h[n], t[n]);
            u[n].own(h[n], u[n].in && live);
            u[n].own(t[n], u[n].in && live);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                sw[n][i] = fmaf(t[n][i], h[n][i], sw[n][i]);
                t[n][i] *= w[n][i];
                s = fmaf(t[n][i], h[n][i], s);
            }
        }
        s = over_row<WIDE, false>(s, a.lpr, sh) * inv;
        if (!live || (!a.dx && !a.dres)) continue;      // (the row's lanes all, and no barrier is left out: a workgroup's row is live)
#pragma unroll
        for (int n = 0; n < NIT; ++n)
            if (u[n].in) write_back<X, R, VEC>(a, r, u[n].c, rstd, s, h[n], t[n], u[n].skip);
    }
    if (!a.part) return;
    float *out = a.part + (long long)blockIdx.x * a.C;
    if (!WIDE) {
        float sums[NIT * VEC];
#pragma unroll
        for (int i = 0; i < NIT * VEC; ++i) sums[i] = sw[i / VEC][i % VEC];
        over_runs<THREADS>(sums, a.rpw, a.lpr, sh);
        if (run) return;
#pragma unroll
        for (int i = 0; i < NIT * VEC; ++i) sw[i / VEC][i % VEC] = sums[i];
    }
#pragma unroll
    for (int n = 0; n < NIT; ++n) {
        if (u[n].in) write_n<float, VEC>(out + u[n].c, sw[n], u[n].skip);
    }
}

// Rows that no workgroup's registers hold: read twice, the sums of dweight in the workspace.
template <typename X, typename R, int VEC, bool TAIL> __global__ __launch_bounds__(1024) void rms_backward_long(const RmsArgs a)
{
    __shared__ float sh[16];
    float *part = a.part ? a.part + (long long)blockIdx.x * a.C : nullptr;
    bool first = true;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x, first = false) {
        const float rstd = a.rstd_in[r];
        float s = 0.f;
        for (Unit<VEC, TAIL> u(threadIdx.x, a.C); u.in; u = Unit<VEC, TAIL>(u.at / VEC + 1024, a.C)) {
            float h[VEC], t[VEC], w[VEC], sum[VEC];
            read_back<X, R, VEC>(a, r, u.c, rstd, h, t);
            read_w<VEC>(a, u.c, w);
            if (part && !first) read_n<float, VEC>(part + u.c, sum);
#pragma unroll
            for (int i = 0; i < VEC; ++i) h[i] *= t[i], t[i] = h[i] * w[i];
            u.own(t, true);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s += t[i], sum[i] = first ? h[i] : sum[i] + h[i];
            if (part) write_n<float, VEC>(part + u.c, sum, u.skip);         // (the thread's own columns)
        }
        s = over_row<true, false>(s, 0, sh) / (float)a.C;
        if (!a.dx && !a.dres) continue;
        for (Unit<VEC, TAIL> u(threadIdx.x, a.C); u.in; u = Unit<VEC, TAIL>(u.at / VEC + 1024, a.C)) {
            float h[VEC], t[VEC], w[VEC];
            read_back<X, R, VEC>(a, r, u.c, rstd, h, t);
            read_w<VEC>(a, u.c, w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) t[i] *= w[i];
            write_back<X, R, VEC>(a, r, u.c, rstd, s, h, t, u.skip);
        }
    }
}

struct Plain {
    float *out;
    __device__ float *operator()(long long c) const { return out + c; }
};

// ---------------------------------------------------------------------------------------------- host
struct Plan {
    RmsArgs a;
    int vec, nit, threads;
    bool wide, held;            // a row is a workgroup's; it is in registers
    long long blocks;
};

int plan_of(const cawn_rms_desc *d, bool bwd, Plan *p)
{
    if (!d || d->rows < 0 || d->C <= 0 || (d->bf16 & ~1) || (d->residual_bf16 & ~1) || d->block < 0 || d->block % 16) return CAWN_EINVAL;
    if (d->C > 32768) return CAWN_EUNSUPPORTED;
    RmsArgs &a = p->a;
    a = RmsArgs{};
    a.rows = d->rows, a.C = d->C, a.eps = d->eps;
    a.xs = d->x_stride ? d->x_stride : a.C, a.rs = d->residual_stride ? d->residual_stride : a.C, a.ys = d->y_stride ? d->y_stride : a.C;
    if (a.xs < a.C || a.rs < a.C || a.ys < a.C) return CAWN_EINVAL;
    a.block = d->block >= d->C ? 0 : d->block;
    a.blocks = a.block ? (int)ceil_div(a.C, a.block) : 1;
    const int most = d->bf16 ? 8 : 4;
    p->vec = a.C >= most ? most : 1;
    const int units = (int)ceil_div(a.C, p->vec);
    p->wide = units > 192;
    p->held = true;
    if (!p->wide) {
        // the run of lanes that has fewest to spare
        int best = 1 << 30;
        for (int nit = 1; nit <= 3; ++nit)
            for (int lanes = 4; lanes <= 64; lanes *= 2)
                if (lanes * nit >= units && lanes * nit < best) best = lanes * nit, a.lpr = lanes, p->nit = nit;
        p->threads = 256;
        a.rpw = 256 / a.lpr;
    } else {        // 16 values a thread at most
        const int top = 16 / p->vec;
        p->threads = units <= 256 * top ? 256 : units <= 512 * top ? 512 : 1024;
        p->held = units <= 1024 * top;
        a.lpr = p->threads, a.rpw = 1;
        const int nit = (int)ceil_div(units, p->threads);
        p->nit = nit <= 1 ? 1 : nit <= 2 ? 2 : 4;
    }
    a.lpb = 0;
    if (a.block) {
        const int lanes = a.block / p->vec;
        if ((lanes & (lanes - 1)) == 0 && lanes <= 64 && lanes <= a.lpr) a.lpb = lanes;
    }
    // Workgroups: forward as many as rows are, up to 16,384; backward, where each leaves a row of sums for dweight, those that are there at once, three a CU.
    // (32,768 rows of 4,096 channels, 8 bits, on 2,048, 4,096, 8,192, 32,768: 205, 193, 174, 174 us; forward and backward of 65,536 of 768 channels, bf16 with
    // an fp32 residual, the latter on 384, 512, 768, 1,024, 2,048: 291, 273, 275, 290, 284.)
    const long long all = ceil_div(a.rows, a.rpw), there = bwd ? 768 : 16384;
    p->blocks = all < there ? all : there;
    return CAWN_OK;
}

template <typename X, typename R, int VEC, bool TAIL, int NIT, bool WIDE, int THREADS> void go(const Plan &p, bool bwd, hipStream_t s)
{
    if (bwd) hipLaunchKernelGGL((rms_backward<X, R, VEC, TAIL, NIT, WIDE, THREADS>), dim3((unsigned)p.blocks), dim3(THREADS), 0, s, p.a);
    else hipLaunchKernelGGL((rms_forward<X, R, VEC, TAIL, NIT, WIDE, THREADS>), dim3((unsigned)p.blocks), dim3(THREADS), 0, s, p.a);
}

template <typename X, typename R, int VEC, bool TAIL, int THREADS> void go_wide(const Plan &p, bool bwd, hipStream_t s)
{
    if (p.nit == 1) go<X, R, VEC, TAIL, 1, true, THREADS>(p, bwd, s);
    else if (p.nit == 2) go<X, R, VEC, TAIL, 2, true, THREADS>(p, bwd, s);
    else go<X, R, VEC, TAIL, 16 / VEC, true, THREADS>(p, bwd, s);
}

template <typename X, typename R, int VEC, bool TAIL> int launch(const Plan &p, bool bwd, hipStream_t s)
{
    if (!p.wide) {
        if (p.nit == 1) go<X, R, VEC, TAIL, 1, false, 256>(p, bwd, s);
        else if (p.nit == 2) go<X, R, VEC, TAIL, 2, false, 256>(p, bwd, s);
        else go<X, R, VEC, TAIL, 3, false, 256>(p, bwd, s);
    } else if (!p.held) {
        if (bwd) hipLaunchKernelGGL((rms_backward_long<X, R, VEC, TAIL>), dim3((unsigned)p.blocks), dim3(1024), 0, s, p.a);
        else hipLaunchKernelGGL((rms_forward_long<X, R, VEC, TAIL>), dim3((unsigned)p.blocks), dim3(1024), 0, s, p.a);
    } else if (p.threads == 256) go_wide<X, R, VEC, TAIL, 256>(p, bwd, s);
    else if (p.threads == 512) go_wide<X, R, VEC, TAIL, 512>(p, bwd, s);
    else go_wide<X, R, VEC, TAIL, 1024>(p, bwd, s);
    return launched();
}

template <typename X, typename R, int VEC> int launch_tail(const Plan &p, bool bwd, hipStream_t s)
{
    if (p.vec == 1) {           // fewer channels than VEC
        go<X, R, 1, false, 1, false, 256>(p, bwd, s);
        return launched();
    }
    return p.a.C % VEC ? launch<X, R, VEC, true>(p, bwd, s) : launch<X, R, VEC, false>(p, bwd, s);
}

int run(const cawn_rms_desc *d, const Plan &p, bool bwd, hipStream_t s)
{
    if (d->bf16) return d->residual_bf16 ? launch_tail<bf16, bf16, 8>(p, bwd, s) : launch_tail<bf16, float, 8>(p, bwd, s);
    return d->residual_bf16 ? launch_tail<float, bf16, 4>(p, bwd, s) : launch_tail<float, float, 4>(p, bwd, s);
}

} // namespace

extern "C" {

size_t cawn_rms_norm_add_workspace_bytes(const cawn_rms_desc *d)
{
    Plan p;
    if (plan_of(d, true, &p) != CAWN_OK) return 0;
    const size_t bytes = (size_t)p.blocks * p.a.C * 4;
    return bytes > 256 ? bytes : 256;
}

int cawn_rms_norm_add_fwd(const cawn_rms_desc *d, const void *x, const void *residual, const float *weight, void *h, void *y, void *q, float *scales, float *rstd,
                          void *stream)
{
    Plan p;
    if (int r = plan_of(d, false, &p)) return r;
    const size_t e = d->bf16 ? 2 : 4, f = d->residual_bf16 ? 2 : 4;
    if (!aligned_to(x, e) || !aligned_to(y, e) || !aligned_to(residual, f) || !aligned_to(h, f) || !aligned_to(weight, 4) || !aligned_to(scales, 4) || !aligned_to(rstd, 4))
        return CAWN_EINVAL;
    if ((y == nullptr && q == nullptr) || (q == nullptr) != (scales == nullptr)) return CAWN_EINVAL;
    if (d->rows == 0) return CAWN_OK;
    if (!x) return CAWN_EINVAL;
    p.a.x = x, p.a.res = residual, p.a.w = weight, p.a.h = h, p.a.y = y, p.a.q = (uint8_t *)q, p.a.scales = scales, p.a.rstd = rstd;
    return run(d, p, false, (hipStream_t)stream);
}

int cawn_rms_norm_add_bwd(const cawn_rms_desc *d, const void *h, const float *weight, const float *rstd, const void *dy, const void *dh, void *dx, void *dresidual,
                          float *dweight, void *workspace, size_t workspace_bytes, void *stream)
{
    Plan p;
    if (int r = plan_of(d, true, &p)) return r;
    const size_t e = d->bf16 ? 2 : 4, f = d->residual_bf16 ? 2 : 4;
    if (!aligned_to(h, f) || !aligned_to(dh, f) || !aligned_to(dresidual, f) || !aligned_to(dy, e) || !aligned_to(dx, e) || !aligned_to(weight, 4) || !aligned_to(rstd, 4) ||
        !aligned_to(dweight, 4)) return CAWN_EINVAL;
    hipStream_t s = (hipStream_t)stream;
    if (d->rows == 0) {
        if (dweight && !d->accumulate_param_grads) launch_sums(nullptr, 0, d->C, Plain{dweight}, 0, s);     // the sum over nothing
        return launched();
    }
    if (!h || !rstd || !dy) return CAWN_EINVAL;
    if (!dx && !dresidual && !dweight) return CAWN_OK;
    if (dweight && (!workspace || workspace_bytes < (size_t)p.blocks * p.a.C * 4 || !aligned_to(workspace, 256))) return CAWN_EWORKSPACE;
    p.a.x = h, p.a.w = weight, p.a.rstd_in = rstd, p.a.dy = dy, p.a.dh = dh, p.a.dx = dx, p.a.dres = dresidual, p.a.part = dweight ? (float *)workspace : nullptr;
    if (int r = run(d, p, true, s)) return r;
    if (dweight) launch_sums(p.a.part, p.blocks, p.a.C, Plain{dweight}, d->accumulate_param_grads, s);
    return launched();
}

} // extern "C"
