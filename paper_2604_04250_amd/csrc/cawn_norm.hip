// Group norm with an activation, channels last, forward and backward.
//
// Forward: mean and variance over a group's values, y = act(w xh + b), xh = (x - mean) rstd.
// Backward: dz = dy act'(z), t = w dz, dx = rstd (t - avg(t) - xh avg(t xh)), dw = sum dz xh, db = sum dz.
//
// Two forms, by T:
//   T = 1 (a token's heads, each by itself): a run of 4 to 64 lanes holds a group in registers from the one read to the write; the
//     variance is that of the centred values.  Bytes: x in, y out (backward: x, dy in, dx out).
//   T > 1, or a group too wide for 64 lanes' registers: a workgroup sums a run of tokens over its channels, a second kernel joins
//     the sums and applies them: x is read twice.  A thread's sums are of x less its own first value over 64 tokens at most; these, threads and
//     workgroups are joined as (count, mean, sum of squares about it), means within a run as differences from its first value: neither a
//     mean of many deviations, a first value that is far off nor a long clip costs the variance its digits.
// Both are bound by memory.  Measured, forward and backward: 65,536 tokens of 12 heads of 64 in bf16 116 us for 0.50 GB (4.3 TB/s; a large copy
// reaches 5.2); 8 x 8,191 tokens of 12 groups of 64 in fp32 346 us for 1.6 GB with the second reads (4.7 TB/s).
// Parameter gradients: every workgroup keeps its channels' sums over the rows it takes and leaves them in the workspace; a last
// kernel adds these in a fixed order.
#include "cawn_ops.hpp"

using namespace cawn::ops;

namespace {

struct NormArgs {
    const void *x, *dy;
    const float *w, *b;
    float *stats;
    void *y, *dx;
    float *part;            // T > 1: sums of a group's part
    float *colpart;         // [rows][2][C]: a workgroup's share of dweight, dbias
    int B, T, C, G, cg, act;
    float eps;
    long long xsb, xst, ysb, yst;
    // geometry
    int lpg, gb, rb, gblocks, rblocks;               // T = 1: lanes of a group; groups and rows of a workgroup; their numbers of workgroups
    int cb, slots, ncb, splits, bblocks, t_run;      // T > 1: channels and groups of a workgroup, its column blocks, runs of tokens, rows at a time
};

// (v_rcp_f32 is good to one unit in the last place; a division takes ten instructions, and these kernels have about as many to spare
// per value as memory leaves them)
__device__ inline float sigmoid_f(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

// The normal distribution function (1 + erf(z / sqrt 2)) / 2 and its density's exponential, which serves the slope too.  The smaller tail
// is e^{-z^2/2} times a polynomial in t = 1 / (1 + 0.31 |z|) without a constant term (the form of Abramowitz and Stegun 7.1.26), fitted to erfc(|z| / sqrt 2) e^{z^2/2} / 2
// for |z| <= 14.5, where the exponential ends, so that the largest relative error is least: 1.6e-7, 4.6e-7 in fp32.
__device__ inline float normal_f(float z, float &e)
{
    e = __expf(-0.5f * z * z);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.31f, fabsf(z), 1.f));
    float p = fmaf(0.0358705036f, t, -0.14173086f);
    p = fmaf(p, t, 0.155298099f);
    p = fmaf(p, t, -0.0151287308f);
    p = fmaf(p, t, 0.110237502f);
    p = fmaf(p, t, 0.107729688f);
    p = fmaf(p, t, 0.124067478f);
    p = fmaf(p, t, 0.123656407f);
    const float tail = p * t * e;
    return z < 0.f ? tail : 1.f - tail;
}

__device__ inline float act_f(float z, int act)
{
    float e;
    if (act == 1) return z * sigmoid_f(z);
    if (act == 2) return z * normal_f(z, e);
    return z;
}

__device__ inline float act_slope(float z, int act)
{
    if (act == 1) {
        const float s = sigmoid_f(z);
        return s * fmaf(z, 1.f - s, 1.f);
    }
    if (act == 2) {
        float e;
        const float n = normal_f(z, e);
        return fmaf(z * 0.3989422804014327f, e, n);
    }
    return 1.f;
}

// sum over the run of `lanes` (a power of two) adjacent lanes, in every one of them
__device__ inline float run_sum(float v, int lanes)
{
    for (int m = lanes >> 1; m > 0; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

template <int VEC> __device__ inline void params(const float *p, int c, float missing, float (&v)[VEC])
{
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = p ? p[c + i] : missing;
}

// ---------------------------------------------------------------------------------------------- T = 1
template <typename T, int VEC, int NIT, bool BWD> __global__ __launch_bounds__(256) void group_norm_rows(const NormArgs a)
{
    const int sub = threadIdx.x / a.lpg, lane = threadIdx.x % a.lpg, gi = sub % a.gb, ri = sub / a.gb;
    const int g = (blockIdx.x % a.gblocks) * a.gb + gi, first = (blockIdx.x / a.gblocks) * a.rb + ri;
    const bool mine = ri < a.rb && g < a.G;
    const int c0 = (mine ? g : 0) * a.cg;
    float w[NIT][VEC], bias[NIT][VEC], sw[BWD ? NIT : 1][VEC], sb[BWD ? NIT : 1][VEC];
    bool in[NIT];
#pragma unroll
    for (int n = 0; n < NIT; ++n) {
        const int c = (n * a.lpg + lane) * VEC;
        in[n] = mine && c < a.cg;
        params<VEC>(in[n] ? a.w : nullptr, c0 + c, 1.f, w[n]);
        params<VEC>(in[n] ? a.b : nullptr, c0 + c, 0.f, bias[n]);
        if (BWD) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) sw[n][i] = sb[n][i] = 0.f;
        }
    }
    const float inv = 1.f / (float)a.cg;
    // a row's values travel while the one before is worked on
    Pack<T, VEC> xn[NIT], dn[BWD ? NIT : 1];
    float mn = 0.f, sn = 0.f;
    auto fetch = [&](long long r) {
#pragma unroll
        for (int n = 0; n < NIT; ++n) {
            const int c = c0 + (in[n] ? (n * a.lpg + lane) * VEC : 0);
            xn[n] = *reinterpret_cast<const Pack<T, VEC> *>((const T *)a.x + r * a.xsb + c);
            if (BWD) dn[n] = *reinterpret_cast<const Pack<T, VEC> *>((const T *)a.dy + r * a.ysb + c);
        }
        if (BWD) mn = a.stats[(r * a.G + (mine ? g : 0)) * 2], sn = a.stats[(r * a.G + (mine ? g : 0)) * 2 + 1];
    };
    const long long stride = (long long)a.rblocks * a.rb;
    if (first < a.B) fetch(first);
    for (long long r = first; r < a.B; r += stride) {
        const bool live = mine;
        float x[NIT][VEC], d[BWD ? NIT : 1][VEC];
        float s = 0.f;
        const float m0 = mn, s0 = sn;
#pragma unroll
        for (int n = 0; n < NIT; ++n) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                x[n][i] = in[n] ? (float)xn[n].v[i] : 0.f;
                if (BWD) d[n][i] = in[n] ? (float)dn[n].v[i] : 0.f;
                s += x[n][i];
            }
        }
        fetch(r + stride < a.B ? r + stride : r);
        float mean, rstd;
        if (BWD) {
            mean = live ? m0 : 0.f;
            rstd = live ? s0 : 0.f;
        } else {
            mean = run_sum(s, a.lpg) * inv;
            float q = 0.f;
#pragma unroll
            for (int n = 0; n < NIT; ++n)
#pragma unroll
                for (int i = 0; i < VEC; ++i) q = in[n] ? fmaf(x[n][i] - mean, x[n][i] - mean, q) : q;
            rstd = 1.f / sqrtf(run_sum(q, a.lpg) * inv + a.eps);
            if (a.stats && live && lane == 0) a.stats[(r * a.G + g) * 2] = mean, a.stats[(r * a.G + g) * 2 + 1] = rstd;
        }
        if (!BWD) {
#pragma unroll
            for (int n = 0; n < NIT; ++n) {
                if (!in[n]) continue;
#pragma unroll
                for (int i = 0; i < VEC; ++i) x[n][i] = act_f(fmaf((x[n][i] - mean) * rstd, w[n][i], bias[n][i]), a.act);
                store_n<T, VEC>((T *)a.y + r * a.ysb + c0 + (n * a.lpg + lane) * VEC, x[n]);
            }
        } else {
            float m1 = 0.f, m2 = 0.f;
#pragma unroll
            for (int n = 0; n < NIT; ++n)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float xh = (x[n][i] - mean) * rstd;
                    // (lanes without values hold zeros: dy and so dz are 0 there)
                    const float dz = d[n][i] * act_slope(fmaf(xh, w[n][i], bias[n][i]), a.act);
                    sw[n][i] = fmaf(dz, xh, sw[n][i]);
                    sb[n][i] += dz;
                    x[n][i] = xh;
                    d[n][i] = dz * w[n][i];
                    m1 += d[n][i];
                    m2 = fmaf(d[n][i], xh, m2);
                }
            m1 = run_sum(m1, a.lpg) * inv;
            m2 = run_sum(m2, a.lpg) * inv;
            if (a.dx) {
#pragma unroll
                for (int n = 0; n < NIT; ++n) {
                    if (!in[n]) continue;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) x[n][i] = rstd * (d[n][i] - m1 - x[n][i] * m2);
                    store_n<T, VEC>((T *)a.dx + r * a.xsb + c0 + (n * a.lpg + lane) * VEC, x[n]);
                }
            }
        }
    }
    if (BWD && a.colpart) {
        // the workgroup's rows of one channel, in the order of its runs of lanes
        __shared__ float sh[256 * VEC * NIT];
        float *out = a.colpart + (long long)(blockIdx.x / a.gblocks) * 2 * a.C;
        for (int which = 0; which < 2; ++which, out += a.C) {
            __syncthreads();
#pragma unroll
            for (int n = 0; n < NIT; ++n)
#pragma unroll
                for (int i = 0; i < VEC; ++i) sh[(sub * NIT + n) * a.lpg * VEC + lane * VEC + i] = which ? sb[n][i] : sw[n][i];
            __syncthreads();
            if (mine && ri == 0) {
#pragma unroll
                for (int n = 0; n < NIT; ++n) {
                    if (!in[n]) continue;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        float v = 0.f;
                        for (int q = 0; q < a.rb; ++q) v += sh[((q * a.gb + gi) * NIT + n) * a.lpg * VEC + lane * VEC + i];
                        out[c0 + (n * a.lpg + lane) * VEC + i] = v;
                    }
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- T > 1
// A workgroup: a.cb adjacent channels (whole groups, or a piece of one), a run of tokens, rows bblk, bblk + bblocks, ...
// WHAT 0: mean and sum of squares about it -> part;  1: y;  2: sums of t and t xh -> part, column sums -> colpart;  3: dx
constexpr int FOLD = 64;        // tokens of a thread's plain sums; a sum of 8,192 squares of bf16 values is off by 1e-5, and always upwards
template <typename T, int VEC, int WHAT> __global__ __launch_bounds__(256) void group_norm_runs(const NormArgs a)
{
    __shared__ float sh[2][256 * (WHAT == 2 ? VEC : 1)];
    __shared__ float stat[256][4];
    const int units = a.cb / VEC, per = (int)blockDim.x / units, rp = threadIdx.x / units, unit = threadIdx.x % units;
    // (the second pass goes backwards: what the first read last is still in the memory-side cache)
    const int blk = WHAT == 1 || WHAT == 3 ? gridDim.x - 1 - blockIdx.x : blockIdx.x, cblk = blk % a.ncb, split = blk / a.ncb % a.splits, bblk = blk / a.ncb / a.splits;
    const bool mine = rp < per;
    const int c = cblk * a.cb + unit * VEC;                             // the thread's channels
    const int per_group = a.cg > a.cb ? a.cg / a.cb : 1;                // workgroups side by side that share a group
    const int slot = a.cg > a.cb ? 0 : unit * VEC / a.cg, g = c / a.cg;
    const int su = a.cg > a.cb ? units : a.cg / VEC;                    // units of a slot
    // (rows and tokens without a sign: T and B go up to 2^31 - 1, and a step or two beyond the last of them has to stay above it)
    const uint32_t t0 = (uint32_t)split * a.t_run, t1 = min((uint32_t)a.T, t0 + a.t_run);
    float w[VEC], bias[VEC], sw[VEC], sb[VEC];
    params<VEC>(mine ? a.w : nullptr, c, 1.f, w);
    params<VEC>(mine ? a.b : nullptr, c, 0.f, bias);
#pragma unroll
    for (int i = 0; i < VEC; ++i) sw[i] = sb[i] = 0.f;
    const double n = (double)a.T * a.cg;
    // (n1, a1, a2) and (n2, b1, b2), counts, means and squares about them, into the first
    auto join = [](float n1, float &a1, float &a2, float n2, float b1, float b2) {
        if (n2 == 0.f) return;
        const float off = b1 - a1, part = n2 / (n1 + n2);
        a1 = fmaf(off, part, a1);
        a2 += b2 + off * off * (n1 * part);
    };
    for (uint32_t b = bblk; b < (uint32_t)a.B; b += a.bblocks) {
        const T *xb = (const T *)a.x + b * a.xsb + c;
        float p0 = 0.f, p1 = 0.f;       // WHAT 1..3: mean, rstd
        float m1 = 0.f, m2 = 0.f;
        if (WHAT == 1 || WHAT == 3) {
            // join the parts of this workgroup's groups: 16 lanes for each slot
            __syncthreads();
            for (int s = threadIdx.x / 16; s < a.slots; s += (int)blockDim.x / 16) {
                const int gs = a.cg > a.cb ? g : cblk * a.slots + s;
                double s1 = 0.0, s2 = 0.0;
                const double about = WHAT == 1 ? (double)a.part[(((long long)b * a.splits * a.ncb + (a.cg > a.cb ? gs * per_group : cblk)) * a.slots + s) * 2] : 0.0;
                const double wide = a.cg > a.cb ? a.cb : a.cg;      // channels of a part
                for (int j = threadIdx.x % 16; j < a.splits * per_group; j += 16) {
                    const int sp = j / per_group, cbk = a.cg > a.cb ? gs * per_group + j % per_group : cblk;
                    const float *p = a.part + ((((long long)b * a.splits + sp) * a.ncb + cbk) * a.slots + s) * 2;
                    if (WHAT == 1) {        // its mean and squares, seen from the first part's mean
                        const double values = (double)(min((uint32_t)a.T, (uint32_t)(sp + 1) * a.t_run) - (uint32_t)sp * a.t_run) * wide, off = (double)p[0] - about;
                        s1 += values * off;
                        s2 += (double)p[1] + values * off * off;
                    } else s1 += p[0], s2 += p[1];
                }
                for (int m = 8; m > 0; m >>= 1) s1 += __shfl_xor(s1, m), s2 += __shfl_xor(s2, m);
                s1 /= n, s2 /= n;
                if (threadIdx.x % 16 == 0) {
                    if (WHAT == 1) {
                        const double var = s2 - s1 * s1;
                        stat[s][0] = (float)(about + s1);
                        stat[s][1] = (float)(1.0 / sqrt((var > 0.0 || var != var ? var : 0.0) + (double)a.eps));
                        const bool one = a.cg > a.cb ? cblk % per_group == 0 : true;
                        if (a.stats && split == 0 && one) {
                            a.stats[((long long)b * a.G + gs) * 2] = stat[s][0];
                            a.stats[((long long)b * a.G + gs) * 2 + 1] = stat[s][1];
                        }
                    } else {
                        stat[s][2] = (float)s1;
                        stat[s][3] = (float)s2;
                    }
                }
            }
            __syncthreads();
            if (WHAT == 1) p0 = stat[slot][0], p1 = stat[slot][1];
            else m1 = stat[slot][2], m2 = stat[slot][3];
        }
        if (WHAT >= 2 && mine) {
            p0 = a.stats[((long long)b * a.G + g) * 2];
            p1 = a.stats[((long long)b * a.G + g) * 2 + 1];
        }
        float s1 = 0.f, s2 = 0.f, shift = 0.f;
        float counted = 0.f, mean = 0.f, about = 0.f;           // WHAT 0: values folded so far, their mean less the shift, squares about it
        if (mine) {
            // two tokens ahead (behind the last, the last again)
            Pack<T, VEC> xa[2], da[2];
            const T *db = WHAT >= 2 ? (const T *)a.dy + b * a.ysb + c : nullptr;
            auto fetch = [&](int e, uint32_t t) {
                t = min(t, t1 - 1);
                xa[e] = *reinterpret_cast<const Pack<T, VEC> *>(xb + t * a.xst);
                if (WHAT >= 2) da[e] = *reinterpret_cast<const Pack<T, VEC> *>(db + t * a.yst);
            };
            fetch(0, t0 + rp);
            fetch(1, t0 + rp + per);
            if (WHAT == 0) shift = (float)xa[0].v[0];
            int fold = FOLD;
            for (uint32_t t = t0 + rp; t < t1; t += per) {
                float x[VEC], d[VEC];
                const Pack<T, VEC> x0 = xa[0], d0 = da[0];
                xa[0] = xa[1], da[0] = da[1];
                fetch(1, t + 2 * per);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    x[i] = (float)x0.v[i];
                    if (WHAT >= 2) d[i] = (float)d0.v[i];
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    if (WHAT == 0) {
                        const float v = x[i] - shift;
                        s1 += v;
                        s2 = fmaf(v, v, s2);
                    } else {
                        const float xh = (x[i] - p0) * p1;
                        const float z = fmaf(xh, w[i], bias[i]);
                        if (WHAT == 1) x[i] = act_f(z, a.act);
                        else {
                            const float dz = d[i] * act_slope(z, a.act), u = dz * w[i];
                            if (WHAT == 2) {
                                sw[i] = fmaf(dz, xh, sw[i]);
                                sb[i] += dz;
                                s1 += u;
                                s2 = fmaf(u, xh, s2);
                            } else x[i] = p1 * (u - m1 - xh * m2);
                        }
                    }
                }
                if (WHAT == 1) store_n<T, VEC>((T *)a.y + b * a.ysb + t * a.yst + c, x);
                if (WHAT == 3) store_n<T, VEC>((T *)a.dx + b * a.xsb + t * a.xst + c, x);
                if (WHAT == 0 && (--fold == 0 || t + per >= t1)) {
                    const float values = (float)((FOLD - fold) * VEC), avg = s1 / values;
                    join(counted, mean, about, values, avg, fmaxf(fmaf(-s1, avg, s2), 0.f) + 0.f * s2);        // (an infinity or NaN stays one)
                    counted += values;
                    s1 = s2 = 0.f, fold = FOLD;
                }
            }
        }
        if (WHAT == 0 || WHAT == 2) {
            // over the token phases of a unit, then over a slot's units
            auto values = [&](uint32_t phase) { return t0 + phase < t1 ? (float)((t1 - t0 - phase + per - 1) / per * VEC) : 0.f; };
            // the run's first value of the group
            const float ref = WHAT == 0 && mine ? (float)*((const T *)a.x + b * a.xsb + t0 * a.xst + (a.cg > a.cb ? cblk * a.cb : g * a.cg)) : 0.f;
            if (WHAT == 0 && mine && counted > 0.f) s1 = shift - ref + mean, s2 = about;
            __syncthreads();
            sh[0][threadIdx.x] = s1, sh[1][threadIdx.x] = s2;
            __syncthreads();
            if (rp == 0) {
                float have = values(0);
                for (int q = 1; q < per; ++q) {
                    if (WHAT == 0) {
                        join(have, s1, s2, values(q), sh[0][q * units + unit], sh[1][q * units + unit]);
                        have += values(q);
                    } else s1 += sh[0][q * units + unit], s2 += sh[1][q * units + unit];
                }
                sh[0][unit] = s1, sh[1][unit] = s2;
                if (WHAT == 0 && unit % su == 0) stat[slot][0] = ref;
            }
            __syncthreads();
            if ((int)threadIdx.x < a.slots) {
                float v1 = 0.f, v2 = 0.f, have = 0.f;
                const float each = (float)(t1 - t0) * VEC;
                for (int q = 0; q < su; ++q) {
                    const float u1 = sh[0][threadIdx.x * su + q], u2 = sh[1][threadIdx.x * su + q];
                    if (WHAT == 0) {
                        join(have, v1, v2, each, u1, u2);
                        have += each;
                    } else v1 += u1, v2 += u2;
                }
                if (WHAT == 0) v1 += stat[threadIdx.x][0];
                float *p = a.part + ((((long long)b * a.splits + split) * a.ncb + cblk) * a.slots + threadIdx.x) * 2;
                p[0] = v1, p[1] = v2;
            }
        }
    }
    if (WHAT == 2 && a.colpart) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            sh[0][threadIdx.x * VEC + i] = sw[i];
            sh[1][threadIdx.x * VEC + i] = sb[i];
        }
        __syncthreads();
        if (rp == 0) {
            float *out = a.colpart + ((long long)bblk * a.splits + split) * 2 * a.C;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float v1 = 0.f, v2 = 0.f;
                for (int q = 0; q < per; ++q) v1 += sh[0][(q * units + unit) * VEC + i], v2 += sh[1][(q * units + unit) * VEC + i];
                out[c + i] = v1;
                out[(long long)a.C + c + i] = v2;
            }
        }
    }
}

// dweight, dbias: the sums of `rows` rows of [2][C], in a fixed order: 16 columns by 64 runs of rows a workgroup
__global__ __launch_bounds__(1024) void group_norm_columns(const float *part, int rows, int C, float *dw, float *db, int accumulate)
{
    __shared__ float sh[64][17];
    const int col = threadIdx.x % 16, run = threadIdx.x / 16;
    const long long c = (long long)blockIdx.x * 16 + col;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < 2LL * C) {
        for (int r = run; r < rows; r += 256) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += r + 64 * e < rows ? part[(long long)(r + 64 * e) * 2 * C + c] : 0.f;
        }
    }
    sh[run][col] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (run == 0 && c < 2LL * C) {
        float v = 0.f;
        for (int q = 0; q < 64; ++q) v += sh[q][col];
        float *out = c < C ? dw : db;
        const long long at = c < C ? c : c - C;
        if (out) out[at] = accumulate ? out[at] + v : v;
    }
}

// ---------------------------------------------------------------------------------------------- host
struct Plan {
    NormArgs a;
    bool rows;              // the T = 1 form
    int vec, nit;
    long long blocks, colrows;
    int threads;            // whole waves of those that have work
    size_t part_bytes, bytes;
};

// The geometry must not depend on pointers: the workspace is sized without them.  Unaligned calls take vec = 1.
bool plan_of(const cawn_norm_desc *d, bool wide, bool bwd, Plan *p)
{
    if (!d || d->B < 0 || d->T < 0 || d->C <= 0 || d->groups <= 0 || d->C % d->groups || d->act < 0 || d->act > 2 || (d->bf16 & ~1)) return false;
    NormArgs &a = p->a;
    a = NormArgs{};
    a.B = d->B, a.T = d->T, a.C = d->C, a.G = d->groups, a.cg = d->C / d->groups, a.act = d->act, a.eps = d->eps;
    a.xst = d->x_stride_t ? d->x_stride_t : d->C, a.yst = d->y_stride_t ? d->y_stride_t : d->C;
    a.xsb = d->x_stride_b ? d->x_stride_b : a.xst * d->T, a.ysb = d->y_stride_b ? d->y_stride_b : a.yst * d->T;
    if (a.xst < a.C || a.yst < a.C) return false;
    const int most = d->bf16 ? 8 : 4;
    const bool fits = a.cg % most == 0 && a.xst % most == 0 && a.xsb % most == 0 && a.yst % most == 0 && a.ysb % most == 0;
    // 16 bytes an access, or single values where rows or groups do not begin on them (65,536 tokens of 12 heads of 64 in bf16, both directions:
    // 117 us, 376; 8 x 8,191 of 12 groups of 64 in fp32: 345 us, 497)
    p->vec = wide && fits ? most : 1;
    const long long lanes = ceil_div(a.cg, p->vec);
    // groups in registers where a run of lanes holds one (the first shape above: 117 us, 534 with sums joined by a second kernel)
    p->rows = a.T == 1 && lanes <= 64 * 4;
    const long long cap = 33554432LL / (8LL * a.C) > 64 ? 33554432LL / (8LL * a.C) : 64;      // rows of parameter sums: 32 MiB of them
    if (p->rows) {
        a.lpg = 1;
        while (a.lpg < 64 && a.lpg < lanes) a.lpg *= 2;
        const long long nit = ceil_div(lanes, a.lpg);
        p->nit = nit <= 1 ? 1 : nit <= 2 ? 2 : 4;
        const int subs = 256 / a.lpg;
        a.gb = a.G < subs ? a.G : subs;
        a.rb = subs / a.gb;
        a.gblocks = (int)ceil_div(a.G, a.gb);
        p->threads = (a.lpg * a.gb * a.rb + 63) / 64 * 64;
        long long rblocks = ceil_div(a.B, a.rb);
        // as many as are there at once, eight or (backward) six to a CU: a second round would be half empty (65,536 tokens of 12 heads of 64 in
        // bf16, forward and backward, the latter on 2,048, 1,536, 1,024: 125, 117, 134 us; forward alone 44, on 1,024 57 us)
        const int groups = bwd ? 1536 : 2048;
        long long want = groups / a.gblocks > 1 ? groups / a.gblocks : 1;
        if (want > cap) want = cap;
        a.rblocks = (int)(rblocks < want ? rblocks : want);
        p->blocks = (long long)a.rblocks * a.gblocks;
        p->colrows = a.rblocks;
        p->part_bytes = 0;
    } else {
        const int top = 256 * p->vec;
        if (a.cg <= top) {
            a.slots = top / a.cg < a.G ? top / a.cg : a.G;
            while (a.G % a.slots) --a.slots;
            a.cb = a.slots * a.cg;
        } else {                            // the widest piece of a group that divides it
            int units = 256;
            while (a.cg / p->vec % units) --units;
            a.slots = 1;
            a.cb = units * p->vec;
        }
        a.ncb = a.C / a.cb;
        const int per = 256 / (a.cb / p->vec);
        p->threads = (a.cb / p->vec * per + 63) / 64 * 64;
        // (8 x 8,191 tokens of 12 groups of 64 in fp32, both directions, backward on 2,048, 1,024: 366, 345 us: every
        // workgroup leaves column sums)
        const int groups = bwd ? 1024 : 2048;
        long long bb = groups / a.ncb > 1 ? groups / a.ncb : 1;
        if (bb > cap) bb = cap;
        a.bblocks = (int)(a.B < bb ? a.B : bb);
        long long splits = a.bblocks > 0 ? bb / a.bblocks : 1;
        const long long useful = ceil_div(a.T, 4LL * per);          // a thread takes four tokens at least
        if (splits > useful) splits = useful;
        if (splits > 512) splits = 512;                             // all parts are joined by everyone (one row of 16,384 x 768, fp32, both
                                                                    // directions, parts up to 1,024, 512, 256: 131, 120, 153 us)
        if (splits < 1) splits = 1;
        a.t_run = (int)ceil_div(a.T, splits);
        if (a.t_run < 1) a.t_run = 1;
        a.splits = (int)(a.T > 0 ? ceil_div(a.T, a.t_run) : 1);
        p->blocks = (long long)a.bblocks * a.splits * a.ncb;
        p->colrows = (long long)a.bblocks * a.splits;
        p->part_bytes = ((size_t)a.B * a.splits * a.ncb * a.slots * 8 + 255) / 256 * 256;
    }
    p->bytes = p->part_bytes + (size_t)p->colrows * 8 * a.C;
    return true;
}

template <typename T, int VEC, bool BWD> void launch_rows(const Plan &p, hipStream_t s)
{
    const dim3 grid((unsigned)p.blocks);
    switch (p.nit) {
    case 1: hipLaunchKernelGGL((group_norm_rows<T, VEC, 1, BWD>), grid, dim3(p.threads), 0, s, p.a); break;
    case 2: hipLaunchKernelGGL((group_norm_rows<T, VEC, 2, BWD>), grid, dim3(p.threads), 0, s, p.a); break;
    default: hipLaunchKernelGGL((group_norm_rows<T, VEC, 4, BWD>), grid, dim3(p.threads), 0, s, p.a); break;
    }
}

template <typename T, int VEC> int launch(const Plan &p, bool bwd, float *dw, float *db, int accumulate, hipStream_t s)
{
    const dim3 grid((unsigned)p.blocks), nt(p.threads);
    if (p.rows) {
        if (bwd) launch_rows<T, VEC, true>(p, s);
        else launch_rows<T, VEC, false>(p, s);
    } else if (!bwd) {
        hipLaunchKernelGGL((group_norm_runs<T, VEC, 0>), grid, nt, 0, s, p.a);
        hipLaunchKernelGGL((group_norm_runs<T, VEC, 1>), grid, nt, 0, s, p.a);
    } else {
        hipLaunchKernelGGL((group_norm_runs<T, VEC, 2>), grid, nt, 0, s, p.a);
        if (p.a.dx) hipLaunchKernelGGL((group_norm_runs<T, VEC, 3>), grid, nt, 0, s, p.a);
    }
    if (p.a.colpart) hipLaunchKernelGGL(group_norm_columns, dim3((unsigned)ceil_div(2LL * p.a.C, 16)), dim3(1024), 0, s, p.a.colpart, (int)p.colrows, p.a.C, dw, db, accumulate);
    return launched();
}

int run(const cawn_norm_desc *d, bool bwd, const void *x, const float *w, const float *b, void *y, float *stats, const void *dy, void *dx, float *dw, float *db,
        void *ws, size_t bytes, void *stream)
{
    Plan p;
    if (!plan_of(d, true, bwd, &p) || !aligned_to(stats, 4) || !aligned_to(dw, 4) || !aligned_to(db, 4)) return CAWN_EINVAL;
    hipStream_t s = (hipStream_t)stream;
    const bool grads = bwd && (dw || db);
    if (d->B == 0 || d->T == 0) {
        if (grads && !d->accumulate_param_grads)        // the sums over nothing
            hipLaunchKernelGGL(group_norm_columns, dim3((unsigned)ceil_div(2LL * p.a.C, 16)), dim3(1024), 0, s, nullptr, 0, p.a.C, dw, db, 0);
        return launched();
    }
    if (!x || (bwd ? !dy || !stats : !y)) return CAWN_EINVAL;
    const size_t e = d->bf16 ? 2 : 4;
    if (!aligned_to(x, e) || !aligned_to(y, e) || !aligned_to(dy, e) || !aligned_to(dx, e) || !aligned_to(w, 4) || !aligned_to(b, 4)) return CAWN_EINVAL;
    if (!aligned_to(x, 16) || !aligned_to(y, 16) || !aligned_to(dy, 16) || !aligned_to(dx, 16)) plan_of(d, false, bwd, &p);
    const size_t need = p.part_bytes + (grads ? (size_t)p.colrows * 8 * p.a.C : 0);
    if (need > 0 && (!ws || bytes < need || !aligned_to(ws, 256))) return CAWN_EWORKSPACE;
    if (p.blocks > 0x7fffffffLL) return CAWN_EUNSUPPORTED;
    p.a.x = x, p.a.w = w, p.a.b = b, p.a.y = y, p.a.stats = stats, p.a.dy = dy, p.a.dx = dx;
    p.a.part = (float *)ws;
    p.a.colpart = grads ? (float *)((char *)ws + p.part_bytes) : nullptr;
    if (bwd && !dx && !grads) return CAWN_OK;
    const int acc = d->accumulate_param_grads;
    if (d->bf16) return p.vec == 8 ? launch<bf16, 8>(p, bwd, dw, db, acc, s) : launch<bf16, 1>(p, bwd, dw, db, acc, s);
    return p.vec == 4 ? launch<float, 4>(p, bwd, dw, db, acc, s) : launch<float, 1>(p, bwd, dw, db, acc, s);
}

} // namespace

extern "C" {

size_t cawn_group_norm_workspace_bytes(const cawn_norm_desc *d)
{
    size_t most = 0;
    for (int i = 0; i < 4; ++i) {
        Plan p;
        if (!plan_of(d, i & 1, i & 2, &p)) return 0;
        most = most > p.bytes ? most : p.bytes;
    }
    return most;
}

int cawn_group_norm_fwd(const cawn_norm_desc *d, const void *x, const float *weight, const float *bias, void *y, float *stats, void *workspace, size_t workspace_bytes, void *stream)
{
    return run(d, false, x, weight, bias, y, stats, nullptr, nullptr, nullptr, nullptr, workspace, workspace_bytes, stream);
}

int cawn_group_norm_bwd(const cawn_norm_desc *d, const void *x, const float *weight, const float *bias, const float *stats, const void *dy, void *dx, float *dweight,
                        float *dbias, void *workspace, size_t workspace_bytes, void *stream)
{
    return run(d, true, x, weight, bias, nullptr, const_cast<float *>(stats), dy, dx, dweight, dbias, workspace, workspace_bytes, stream);
}

} // extern "C"
