// Selective state space scan by tiles of 16 tokens, backward.
//
//     g = dy SiLU(z);  dS[t] = C[t] g[t] + exp(delta[t+1] A) dS[t+1];  h[t] = exp(delta[t] A) dS[t];  p[t] = h[t] S[t-1]
//     dC[t] = sum over channels g S[t];  dB[t] = sum over channels u dS[t];  du = sum over states B dS;  ddelta = sum over states A p + x du
//     dA = sum over tokens delta p;  dx = delta du + D g;  dz = dy SiLU'(z) y;  dD = sum x g;  ddt = ddelta softplus'(dt + bias)
//
// As the forward, from the last token to the first: what a segment makes of no gradient from behind it, the chain over the segments, and all segments
// with what reaches their end.  A tile's states are made again from those kept before it, two states of a channel at a time for its 16 tokens, which then
// stay in registers for the way back.  The sums over channels go through a tree of lanes that halves the values as it halves the lanes (64 values in 129
// instructions, one by one they would take 384); a workgroup adds up its waves, and what the workgroups leave is added in their order.
// Bound by instruction issue: 8 x 8,192 tokens of 768 channels of 16 states in bf16 163 us for what segments hand on, 567 for the gradients (341 instructions a
// token of a wave, vector units busy for 88 % of the time), the chain 13, the sums 14.
#include "cawn_select.hpp"

namespace cawn {
namespace select {

__device__ inline float dsilu(float z, float &silu)
{
    const float f = sigmoid_f(z);
    silu = z * f;
    return f * fmaf(z, 1.f - f, 1.f);
}

// What a segment hands on where nothing reaches its end, and its sum of delta.
template <typename T, int NP, int NB> __global__ __launch_bounds__(NB > 1 ? 64 * NB : 256) void select_back(const Args a)
{
    constexpr int NPT = NP * NB, AHEAD = 2;
    const Place p = place_of<(NB > 1)>(a);
    if (!p.there) return;
    const int n = __builtin_amdgcn_readfirstlane(row_length(a, p.b));
    const int t0 = p.seg * a.seg_tiles * TILE, t1 = min(n, t0 + a.seg_tiles * TILE);
    if (t0 >= t1 || t0 == 0) return;        // (the chain ends behind the first)
    const T *dp = (const T *)a.dt + p.b * a.dsb + p.base, *dyp = (const T *)a.dy + p.b * a.ysb + p.base, *zp = a.z ? (const T *)a.z + p.b * a.zsb + p.base : nullptr;
    const uint32_t at = p.bytes<T>();
    auto step = [](long long stride) { return (uint32_t)stride * (uint32_t)sizeof(T); };
    uint32_t dr[RUN], yr[RUN], zr[RUN];
    auto fetch = [&](int t) {
        if (t < t0) {
            no_run<RUN>(dr), no_run<RUN>(yr), no_run<RUN>(zr);
            return;
        }
        const int left = t1 - t;
        load_run<T, RUN>(dp + t * a.dst, step(a.dst), left, at, dr);
        load_run<T, RUN>(dyp + t * a.yst, step(a.yst), left, at, yr);
        if (zp) load_run<T, RUN>(zp + t * a.zst, step(a.zst), left, at, zr);
        else no_run<RUN>(zr);
    };
    const int last = (t1 - 1) / RUN * RUN;
    fetch(last);
    float A[NP], h[NP], total = 0.f;
    load_rates<NP>(a, p, A);
#pragma unroll
    for (int i = 0; i < NP; ++i) h[i] = 0.f;
    const float bias = a.bias ? a.bias[p.ch] : 0.f;
    for (int t = last; t >= t0; t -= RUN) {
        const int left = t1 - t;
        const float *tile = a.bc + (((long long)p.b * a.tiles + t / TILE) * a.G + p.g) * NPT * 2 * TILE + p.blk * NP * 2 * TILE + t % TILE;
        Scalars<RUN> Cq[NP];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) Cq[s] = bc_run<RUN>(tile, s, 1);
        float delta[RUN], g[RUN];
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            delta[i] = value<T>(dr[i]) + bias;
            g[i] = value<T>(yr[i]);
        }
        if (a.softplus) {
#pragma unroll
            for (int i = 0; i < RUN; ++i) delta[i] = softplus_f(delta[i]);
        }
        if (zp) {
#pragma unroll
            for (int i = 0; i < RUN; ++i) {
                const float z = value<T>(zr[i]);
                g[i] *= z * sigmoid_f(z);
            }
        }
        if (left < RUN) {
#pragma unroll
            for (int i = 0; i < RUN; ++i) {
                delta[i] = i < left ? delta[i] : 0.f;
                g[i] = i < left ? g[i] : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < RUN; ++i) total += delta[i];
        fetch(t - RUN);
#pragma unroll
        for (int s = 0; s < NP; ++s) {
#pragma unroll
            for (int i = RUN - 1; i >= 0; --i) {
                h[s] = factor(delta[i], A[s]) * fmaf(Cq[s][i], g[i], h[s]);
                if (i == RUN - 1 && s + AHEAD < NP) {      // (as in the forward)
                    __builtin_amdgcn_sched_barrier(0);
                    Cq[s + AHEAD < NP ? s + AHEAD : 0] = bc_run<RUN>(tile, s + AHEAD, 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    const long long seg = (long long)p.b * a.segments + p.seg;
    store_states<NP>(a.seg_b + (seg * a.Dp + p.pad) * NPT + p.blk * NP, h);
    if (p.blk == 0) a.seg_g[seg * a.Dp + p.pad] = total;
}

template <int CTRL> __device__ inline float from_lane(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false)); }

// Sums over lanes by a tree that halves the values as it halves the lanes: of two values one remains, summed over pairs of lanes, the first in the lanes
// without a bit of the lane's number, the second in those with it.
//
// Four values, by bits 3 and 2: the lanes of a bit are banks of a row, which an addition may leave out, so that two instructions make one value of two (with
// selections it takes three).  Whoever writes a register that is read across lanes has to be two instructions away: the s_nops; no lane is idle here.
__device__ inline float four(float a0, float a1, float b0, float b1)
{
    float s, t, r;
    asm("s_nop 1\n\t"
        "v_add_f32_dpp %0, %3, %3 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
        "v_add_f32_dpp %1, %5, %5 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
        "v_add_f32_dpp %0, %4, %4 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "v_add_f32_dpp %1, %6, %6 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "s_nop 0\n\t"
        "v_add_f32_dpp %2, %0, %0 row_half_mirror row_mask:0xf bank_mask:0x5\n\t"
        "v_add_f32_dpp %2, %1, %1 row_half_mirror row_mask:0xf bank_mask:0xa\n\t"
        "s_nop 1"
        : "=&v"(s), "=&v"(t), "=&v"(r)
        : "v"(a0), "v"(a1), "v"(b0), "v"(b1));
    return r;
}

// Two values, by bit 5, 4, 1, 0 for level 0 to 3.
__device__ inline float two_values(int level, float first, float second, int lane)
{
    if (level == 0) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(first), __float_as_uint(second), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (level == 1) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(first), __float_as_uint(second), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    const bool bit = lane & (level == 2 ? 2 : 1);
    const float keep = bit ? second : first, give = bit ? first : second;
    return keep + (level == 2 ? from_lane<0x4e>(give) : from_lane<0xb1>(give));         // quad_perm 2,3,0,1 and 1,0,3,2
}

// 64 values, four at a time: value i is then in the lane whose bits 3, 2, 5, 4, 1, 0 are i's bits 0 to 5.
struct LaneSums {
    float held[4];
    __device__ inline float push(int group, float a0, float a1, float b0, float b1, int lane)
    {
        float v = four(a0, a1, b0, b1);
#pragma unroll
        for (int level = 0; level < 4; ++level) {
            if (!(group >> level & 1)) {
                held[level] = v;
                return v;
            }
            v = two_values(level, held[level], v, lane);
        }
        return v;
    }
};

template <typename T, int NP, int NB> __global__ __launch_bounds__(NB > 1 ? 64 * NB : 256) __attribute__((amdgpu_waves_per_eu(2, 2))) void select_gradients(const Args a)
{
    constexpr bool MULTI = NB > 1;
    constexpr int NPT = NP * NB, WAVES = MULTI ? NB : 4;
    __shared__ float carry[WAVES][NP][3][64];       // of each state: h from behind, dA, A
    __shared__ float stage[2][MULTI ? 1 : WAVES][TILE][2][NP];
    __shared__ float xch[MULTI ? NB : 1][TILE][64];
    const Place p = place_of<MULTI>(a);
    const int n = __builtin_amdgcn_readfirstlane(row_length(a, p.b)), w = MULTI ? p.blk : __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int t0 = p.seg * a.seg_tiles * TILE, t1 = min(n, t0 + a.seg_tiles * TILE), end = min(a.L, t0 + a.seg_tiles * TILE);
    const long long seg = (long long)p.b * a.segments + p.seg, user = (long long)p.b * a.D + p.ch;
    const bool whole = (p.cb + 1) * (MULTI ? 1 : a.wide) * 64 <= a.cg;       // every lane of the workgroup has a channel
    float(*mine)[3][64] = carry[w];
    {
        float A[NP], h[NP];
        load_rates<NP>(a, p, A);
#pragma unroll
        for (int i = 0; i < NP; ++i) h[i] = 0.f;
        if (a.segments > 1) {
            if (t0 < t1 || (p.seg == 0 && n == 0)) load_states<NP>(a.seg_s + (seg * a.Dp + p.pad) * NPT + p.blk * NP, h);
        } else if (a.dstate_out) load_user<NP>(a.dstate_out, a, user, p.blk * NP, h);
#pragma unroll
        for (int i = 0; i < NP; ++i) mine[i][0][p.lane] = h[i], mine[i][1][p.lane] = 0.f, mine[i][2][p.lane] = A[i];
    }
    const float bias = a.bias ? a.bias[p.ch] : 0.f, Dk = a.Dk ? a.Dk[p.ch] : 0.f;
    const T *xp = (const T *)a.x + p.b * a.xsb + p.base, *dp = (const T *)a.dt + p.b * a.dsb + p.base, *dyp = (const T *)a.dy + p.b * a.ysb + p.base;
    const T *zp = a.z ? (const T *)a.z + p.b * a.zsb + p.base : nullptr;
    T *dxp = a.dx ? (T *)a.dx + p.b * a.xsb + p.base : nullptr, *ddp = a.ddt ? (T *)a.ddt + p.b * a.dsb + p.base : nullptr;
    T *dzp = a.dz ? (T *)a.dz + p.b * a.zsb + p.base : nullptr;
    const uint32_t at = p.bytes<T>();
    auto step = [](long long stride) { return (uint32_t)stride * (uint32_t)sizeof(T); };
    uint32_t xr[TILE], xn[TILE], dr[TILE], yr[TILE], zr[TILE];
    auto fetch = [&](int t) {
        if (t < t0) {
            no_run<TILE>(dr), no_run<TILE>(xn), no_run<TILE>(yr), no_run<TILE>(zr);
            return;
        }
        const int left = t1 - t;
        load_run<T, TILE>(dp + t * a.dst, step(a.dst), left, at, dr);
        load_run<T, TILE>(xp + t * a.xst, step(a.xst), left, at, xn);
        load_run<T, TILE>(dyp + t * a.yst, step(a.yst), left, at, yr);
        if (zp) load_run<T, TILE>(zp + t * a.zst, step(a.zst), left, at, zr);
        else no_run<TILE>(zr);
    };
    const int last = t1 > t0 ? (t1 - 1) / TILE * TILE : t0 - 1;
    fetch(last);
    const float first = MULTI && p.blk > 0 ? 0.f : Dk;          // (one wave adds D x to y)
    float sumD = 0.f, sumb = 0.f;
    int buf = 0;
    for (int t = last; t >= t0; t -= TILE) {
        const int left = t1 - t;
        const long long bt = (long long)p.b * a.tiles + t / TILE;
        const float *tile = a.bc + (bt * a.G + p.g) * NPT * 2 * TILE + p.blk * NP * 2 * TILE;
        const float *ck = a.ck + (bt * a.Dp + p.pad) * NPT + p.blk * NP;
        // a state's B, C, begin, h, dA and A, each asked for while the state before is worked on
        Scalars<TILE> Bv[2], Cv[2];
        float before[2], h[2], dA[2], A[2];
        auto ask = [&](int j, int s) {
            Bv[j] = bc_run<TILE>(tile, s, 0), Cv[j] = bc_run<TILE>(tile, s, 1);
            before[j] = ck[s];
            h[j] = mine[s][0][p.lane], dA[j] = mine[s][1][p.lane], A[j] = mine[s][2][p.lane];
        };
        ask(0, 0);
        // (one stream after the other, so that what has been read makes room for what comes of it)
        float delta[TILE], slope[TILE], u[TILE], g[TILE], q[TILE], du[TILE], dd[TILE], y[TILE];
#pragma unroll
        for (int i = 0; i < TILE; ++i) delta[i] = value<T>(dr[i]) + bias, slope[i] = 1.f;
        if (a.softplus) {
#pragma unroll
            for (int i = 0; i < TILE; ++i) {
                slope[i] = sigmoid_f(delta[i]);
                delta[i] = softplus_f(delta[i]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TILE; ++i) g[i] = value<T>(yr[i]), q[i] = 0.f;
        if (zp) {
#pragma unroll
            for (int i = 0; i < TILE; ++i) {
                float silu;
                const float ds = dsilu(value<T>(zr[i]), silu);
                q[i] = g[i] * ds;
                g[i] *= silu;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TILE; ++i) {
            if (!MULTI) xr[i] = xn[i];
            const float x = value<T>(xn[i]);
            u[i] = delta[i] * x;
            y[i] = first * x;
        }
        if (left < TILE) {          // behind the last token nothing is added anywhere
#pragma unroll
            for (int i = 0; i < TILE; ++i) {
                delta[i] = i < left ? delta[i] : 0.f;
                u[i] = i < left ? u[i] : 0.f;
                g[i] = i < left ? g[i] : 0.f;
            }
        }
        if (!whole) {               // ... nor where there is no channel
#pragma unroll
            for (int i = 0; i < TILE; ++i) {
                u[i] = p.on ? u[i] : 0.f;
                g[i] = p.on ? g[i] : 0.f;
            }
        }
        if (!MULTI) {
            stay<TILE>(slope);
            stay<TILE>(q);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TILE; ++i) du[i] = dd[i] = 0.f;
#pragma unroll 1
        for (int s = 0; s < NP; s += 2) {
            LaneSums sums;
            float all = 0.f;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float S[TILE], e[TILE];
#pragma unroll
                for (int i = 0; i < TILE; ++i) {
                    e[i] = factor(delta[i], A[j]);
                    S[i] = fmaf(e[i], i ? S[i ? i - 1 : 0] : before[j], u[i] * Bv[j][i]);
                    y[i] = fmaf(Cv[j][i], S[i], y[i]);
                    if (i == 0) {       // (the wait for this state's is over)
                        __builtin_amdgcn_sched_barrier(0);
                        ask(1 - j, j ? min(s + 2, NP - 2) : s + 1);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                const float Af = fmaxf(A[j], -3.4028235e38f);       // (where the rate is minus infinity p is 0, and so is its share)
                // (token pairs: their four products' sums are begun together)
                float ub[2], gc[2];
#pragma unroll
                for (int i = TILE - 1; i >= 0; --i) {
                    const float dS = fmaf(Cv[j][i], g[i], h[j]);
                    du[i] = fmaf(Bv[j][i], dS, du[i]);
                    h[j] = e[i] * dS;
                    const float pr = h[j] * (i ? S[i ? i - 1 : 0] : before[j]);
                    dd[i] = fmaf(Af, pr, dd[i]);
                    dA[j] = fmaf(delta[i], pr, dA[j]);
                    ub[i & 1] = u[i] * dS, gc[i & 1] = g[i] * S[i];
                    if ((i & 1) == 0) all = sums.push((j * TILE + TILE - 2 - i) / 2, ub[1], gc[1], ub[0], gc[0], p.lane);
                }
                mine[s + j][0][p.lane] = h[j], mine[s + j][1][p.lane] = dA[j];
            }
            // value 2 (16 j + 15 - i) + which
            const int which = p.lane >> 3 & 1, j = p.lane & 1;
            const int i = TILE - 1 - ((p.lane >> 2 & 1) | (p.lane >> 4 & 2) | (p.lane >> 2 & 4) | (p.lane << 2 & 8));
            if (MULTI) {
                if (a.part_bc) a.part_bc[((((bt * TILE + i) * a.G + p.g) * a.parts + p.cb) * 2 + which) * NPT + p.blk * NP + s + j] = all;
            } else stage[buf][MULTI ? 0 : w][i][which][s + j] = all;
        }
        stay<TILE>(du);
        stay<TILE>(dd);
        stay<TILE>(y);
        fetch(t - TILE);
        if (!MULTI && a.part_bc) {
            __syncthreads();
            for (int k = threadIdx.x; k < TILE * 2 * NP; k += blockDim.x) {
                const int i = k / (2 * NP), at = k % (2 * NP);
                float v = 0.f;
                for (int m = 0; m < a.wide; ++m) v += stage[buf][MULTI ? 0 : m][i][at / NP][at % NP];
                a.part_bc[(((bt * TILE + i) * a.G + p.g) * a.parts + p.cb) * 2 * NPT + at] = v;
            }
            buf ^= 1;
        }
        // (dd becomes the gradient of dt, du that of x, y that of z)
        auto finish = [&](bool there, float x, float delta, float slope, float g, float q, float &du, float &dd, float &y) {
            dd = fmaf(du, x, dd * LN2) * slope;
            du = fmaf(du, delta, Dk * g);
            y *= q;
            if (there) {
                sumD = fmaf(g, x, sumD);
                sumb += dd;
            }
        };
        if constexpr (!MULTI) {
#pragma unroll
            for (int i = 0; i < TILE; ++i) finish(i < left, value<T>(xr[i]), delta[i], slope[i], g[i], q[i], du[i], dd[i], y[i]);
            if (p.on) {
                if (dxp) store_run<T, TILE>(dxp + t * a.xst, step(a.xst), left, at, [&](int i) { return du[i]; });
                if (ddp) store_run<T, TILE>(ddp + t * a.dst, step(a.dst), left, at, [&](int i) { return dd[i]; });
                if (dzp) store_run<T, TILE>(dzp + t * a.zst, step(a.zst), left, at, [&](int i) { return y[i]; });
            }
        } else {
            // the waves' shares of du, dd and y are added up; wave i % NB goes on with token i, whose streams it reads again
            constexpr int OWN = TILE / NB;
            float duo[OWN], ddo[OWN], yo[OWN];
            auto exchange = [&](const float(&v)[TILE], float(&own)[OWN]) {
#pragma unroll
                for (int i = 0; i < TILE; ++i) xch[p.blk][i][p.lane] = v[i];
                __syncthreads();
#pragma unroll
                for (int k = 0; k < OWN; ++k) {
                    own[k] = 0.f;
#pragma unroll
                    for (int m = 0; m < NB; ++m) own[k] += xch[m][k * NB + p.blk][p.lane];
                }
                __syncthreads();
            };
            exchange(du, duo);
            exchange(dd, ddo);
            exchange(y, yo);
            const auto xs = rows_at(xp + t * a.xst), ds = rows_at(dp + t * a.dst), ys = rows_at(dyp + t * a.yst), zs = rows_at(zp ? zp + t * a.zst : nullptr);
            float x[OWN], d[OWN], g1[OWN], z[OWN];
#pragma unroll
            for (int k = 0; k < OWN; ++k) {
                const uint32_t i = min(k * NB + p.blk, left - 1);
                x[k] = value<T>(load_at<T>(xs, at, i * step(a.xst))), d[k] = value<T>(load_at<T>(ds, at, i * step(a.dst)));
                g1[k] = value<T>(load_at<T>(ys, at, i * step(a.yst))), z[k] = zp ? value<T>(load_at<T>(zs, at, i * step(a.zst))) : 0.f;
            }
#pragma unroll
            for (int k = 0; k < OWN; ++k) {
                const int i = k * NB + p.blk;
                const bool there = i < left && p.on;
                const float v = d[k] + bias;
                float silu = 1.f, q1 = 0.f;
                if (zp) q1 = g1[k] * dsilu(z[k], silu);
                finish(there, x[k], a.softplus ? softplus_f(v) : v, a.softplus ? sigmoid_f(v) : 1.f, there ? g1[k] * silu : 0.f, q1, duo[k], ddo[k], yo[k]);
                if (!there) continue;
                if (dxp) store_at<T>(rows_at(dxp + (t + i) * a.xst), at, 0, duo[k]);
                if (ddp) store_at<T>(rows_at(ddp + (t + i) * a.dst), at, 0, ddo[k]);
                if (dzp) store_at<T>(rows_at(dzp + (t + i) * a.zst), at, 0, yo[k]);
            }
        }
    }
    if (p.on && p.blk == 0) {
        for (int t = max(t0, n); t < end; ++t) {
            if (dxp) store_at<T>(rows_at(dxp + t * a.xst), at, 0, 0.f);
            if (ddp) store_at<T>(rows_at(ddp + t * a.dst), at, 0, 0.f);
            if (dzp) store_at<T>(rows_at(dzp + t * a.zst), at, 0, 0.f);
        }
    }
    if (!p.there) return;
    float h[NP], dA[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) h[i] = mine[i][0][p.lane], dA[i] = mine[i][1][p.lane];
    if (a.part_a) {         // a row: [Dp][NPT] of A, [Dp] of D, [Dp] of the bias
        float *out = a.part_a + seg * a.Dp * (NPT + 2);
        store_states<NP>(out + p.pad * NPT + p.blk * NP, dA);
        if (MULTI) {        // (the waves' tokens)
            xch[MULTI ? p.blk : 0][0][p.lane] = sumD, xch[MULTI ? p.blk : 0][1][p.lane] = sumb;
            __syncthreads();
            sumD = sumb = 0.f;
#pragma unroll
            for (int m = 0; m < NB; ++m) sumD += xch[MULTI ? m : 0][0][p.lane], sumb += xch[MULTI ? m : 0][1][p.lane];
        }
        if (p.blk == 0) {
            out += (long long)a.Dp * NPT + p.pad;
            out[0] = sumD, out[a.Dp] = sumb;
        }
    }
    if (p.on && a.dstate_in && p.seg == 0) store_user<NP>(a.dstate_in, a, user, p.blk * NP, h);
}

// What the workgroups left, in their order: the first `bc` workgroups dB and dC, four states a thread, from workgroup `from` of these sums on; the others the
// parameters' gradients.  (A launch counts its threads in 32 bits.  Workgroups that go round take 65 registers for 46 and are one a CU: 6.6 us for 5.0 in a call of
// few rows, 16.2 for 14.8 at 8 x 8,192 tokens; what is beyond BC_BLOCKS is a launch more.)
constexpr long long BC_BLOCKS = 1 << 12;

template <typename T> __global__ __launch_bounds__(1024) void select_bc_sums(const Args a, const long long from, const unsigned bc, const ParamSums sums, const int accumulate)
{
    const int NPT = a.NP * a.NB, per = 2 * NPT;
    if (blockIdx.x >= bc) {
        sum_columns(blockIdx.x - bc, a.part_a, (long long)a.B * a.segments, (long long)a.Dp * (NPT + 2), sums, accumulate);
        return;
    }
    const long long id = (from + blockIdx.x) * 1024 + threadIdx.x;
    const int at = (int)(id % (per / 4)) * 4, which = at / NPT, n = at % NPT;
    const long long rest = id / (per / 4), g = rest % a.G, bt = rest / a.G, b = bt / a.L, t = bt - b * a.L;
    if (b >= a.B || n >= a.N) return;
    T *out = (T *)(which ? a.dC : a.dB);
    if (!out) return;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (t < row_length(a, (int)b)) {
        const float *p = a.part_bc + (((b * a.tiles * TILE + t) * a.G + g) * a.parts) * per + at;
        for (int k = 0; k < a.parts; ++k) v += *reinterpret_cast<const f32x4 *>(p + (long long)k * per);
    }
    out += b * a.bsb + t * a.bst + g * a.N + n;
    if (n + 4 <= a.N && ((uintptr_t)out & (4 * sizeof(T) - 1)) == 0) {
        const float x[4] = {v[0], v[1], v[2], v[3]};
        store_n<T, 4>(out, x);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n + j < a.N) out[j] = (T)v[j];
    }
}

int launch_bc_sums(const Args &a, bool bf16_, const ParamSums &sums, int accumulate, hipStream_t s)
{
    const int NPT = a.NP * a.NB;
    const long long cols = (long long)a.Dp * (NPT + 2), columns = ceil_div(cols, SUM_COLS);
    const bool apart = a.part_a && columns > SUM_BLOCKS;            // (a launch of their own goes round)
    if (apart) launch_sums(a.part_a, (long long)a.B * a.segments, cols, sums, accumulate, s);
    unsigned pa = a.part_a && !apart ? (unsigned)columns : 0;
    const long long all = a.part_bc ? ceil_div((long long)a.B * a.L * a.G * 2 * NPT / 4, 1024) : 0;
    for (long long from = 0; from < all || pa > 0; from += BC_BLOCKS, pa = 0) {
        const unsigned bc = (unsigned)(all - from < BC_BLOCKS ? all - from : BC_BLOCKS);
        if (bf16_) hipLaunchKernelGGL(select_bc_sums<bf16>, dim3(bc + pa), dim3(1024), 0, s, a, from, bc, sums, accumulate);
        else hipLaunchKernelGGL(select_bc_sums<float>, dim3(bc + pa), dim3(1024), 0, s, a, from, bc, sums, accumulate);
    }
    return launched();
}

template <typename T, int NP, int NB> static void launch_np(const Args &a, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)a.B * a.segments * a.G * a.cbg)), block(64 * (NB > 1 ? NB : a.wide));
    if (a.segments > 1) {
        hipLaunchKernelGGL((select_back<T, NP, NB>), grid, block, 0, s, a);
        launch_join(a, true, s);
    }
    hipLaunchKernelGGL((select_gradients<T, NP, NB>), grid, block, 0, s, a);
}

template <typename T> static int launch(const Args &a, hipStream_t s)
{
    by_states(a, [&](auto np, auto nb) { launch_np<T, decltype(np)::value, decltype(nb)::value>(a, s); });
    return launched();
}

int launch_backward(const Args &a, bool bf16_, hipStream_t s) { return bf16_ ? launch<bf16>(a, s) : launch<float>(a, s); }

} // namespace select
} // namespace cawn
