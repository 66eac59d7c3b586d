// Selective state space scan by tiles of 16 tokens, backward.
//
//     g = dy SiLU(z);  dS[t] = C[t] g[t] + exp(delta[t+1] A) dS[t+1];  h[t] = exp(delta[t] A) dS[t];  p[t] = h[t] S[t-1]
//     dC[t] = sum over channels g S[t];  dB[t] = sum over channels u dS[t];  du = sum over states B dS;  ddelta = sum over states A p + x du
//     dA = sum over tokens delta p;  dx = delta du + D g;  dz = dy SiLU'(z) y;  dD = sum x g;  ddt = ddelta softplus'(dt + bias)
//
// As the forward, from the last token to the first: what a segment makes of no gradient from behind it, the chain over the segments, and all segments
// with what reaches their end.  A tile's states are made again from those kept before it, two states of a channel at a time for its 16 tokens, which then
// stay in registers for the way back.  The sums over channels go through a tree of lanes that halves the values as it halves the lanes (64 values in 141
// instructions, one by one they would take 384); a workgroup adds up its waves, and what the workgroups leave is added in their order.
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
    constexpr int NPT = NP * NB;
    const Place p = place_of<(NB > 1)>(a);
    if (!p.there) return;
    const int n = row_length(a, p.b);
    const long long t0 = (long long)p.seg * a.seg_tiles * TILE, t1 = min((long long)n, t0 + (long long)a.seg_tiles * TILE);
    if (t0 >= t1) return;
    float A[NP], h[NP], total = 0.f;
    load_rates<NP>(a, p, A);
#pragma unroll
    for (int i = 0; i < NP; ++i) h[i] = 0.f;
    const float bias = a.bias ? a.bias[p.ch] : 0.f;
    const T *dp = (const T *)a.dt + p.b * a.dsb + p.ch, *dyp = (const T *)a.dy + p.b * a.ysb + p.ch;
    const T *zp = a.z ? (const T *)a.z + p.b * a.zsb + p.ch : nullptr;
    for (long long t = (t1 - 1) / TILE * TILE; t >= t0; t -= TILE) {
        const int left = (int)min(t1 - t, (long long)TILE);
        const float *tile = a.bc + (((long long)p.b * a.tiles + t / TILE) * a.G + p.g) * NPT * 2 * TILE + p.blk * NP * 2 * TILE;
        float delta[TILE], g[TILE];
        T zr[TILE];
#pragma unroll
        for (int i = 0; i < TILE; ++i) {
            const long long at = t + min(i, left - 1);
            delta[i] = (float)dp[at * a.dst] + bias;
            g[i] = (float)dyp[at * a.yst];
            zr[i] = zp ? zp[at * a.zst] : (T)0.f;
        }
#pragma unroll
        for (int i = 0; i < TILE; ++i) {
            if (a.softplus) delta[i] = softplus_f(delta[i]);
            const float z = (float)zr[i];
            if (zp) g[i] *= z * sigmoid_f(z);
            delta[i] = i < left ? delta[i] : 0.f;
            g[i] = i < left ? g[i] : 0.f;
            total += delta[i];
        }
        f32x16 Cn = bc_tile(tile, 0, 1);
#pragma unroll
        for (int s = 0; s < NP; ++s) {
            const f32x16 Cv = Cn;
#pragma unroll
            for (int i = TILE - 1; i >= 0; --i) {
                h[s] = factor(delta[i], A[s]) * fmaf(Cv[i], g[i], h[s]);
                if (i == TILE - 1 && s + 1 < NP) {      // (as in the forward)
                    __builtin_amdgcn_sched_barrier(0);
                    Cn = bc_tile(tile, s + 1, 1);
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

// Two values a lane become one, each summed over pairs of lanes: the lanes without the level's bit (32, 16, 8, .. for level 0, 1, 2, ..) keep the first.
__device__ inline float merge(int level, float first, float second, int lane)
{
    if (level == 0) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(first), __float_as_uint(second), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (level == 1) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(first), __float_as_uint(second), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    const bool bit = lane & (32 >> level);
    const float keep = bit ? second : first, give = bit ? first : second;
    if (level == 2) return keep + from_lane<0x128>(give);           // row_ror:8
    if (level == 3) return keep + from_lane<0x141>(give);           // row_half_mirror: lane i from 7 - i
    if (level == 4) return keep + from_lane<0x4e>(give);            // quad_perm 2,3,0,1
    return keep + from_lane<0xb1>(give);                            // quad_perm 1,0,3,2
}

// Sums of 64 values over the 64 lanes, given one by one: the i-th is then in the lane whose number is i's six bits turned round.
struct LaneSums {
    float held[6];
    __device__ inline float push(int i, float v, int lane)
    {
#pragma unroll
        for (int level = 0; level < 6; ++level) {
            if (!(i >> level & 1)) {
                held[level] = v;
                return v;
            }
            v = merge(level, held[level], v, lane);
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
    const int n = row_length(a, p.b), w = MULTI ? p.blk : __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const long long t0 = (long long)p.seg * a.seg_tiles * TILE, t1 = min((long long)n, t0 + (long long)a.seg_tiles * TILE), end = min((long long)a.L, t0 + (long long)a.seg_tiles * TILE);
    const long long seg = (long long)p.b * a.segments + p.seg, user = (long long)p.b * a.D + p.ch;
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
    const T *xp = (const T *)a.x + p.b * a.xsb + p.ch, *dp = (const T *)a.dt + p.b * a.dsb + p.ch, *dyp = (const T *)a.dy + p.b * a.ysb + p.ch;
    const T *zp = a.z ? (const T *)a.z + p.b * a.zsb + p.ch : nullptr;
    T *dxp = a.dx ? (T *)a.dx + p.b * a.xsb + p.ch : nullptr, *ddp = a.ddt ? (T *)a.ddt + p.b * a.dsb + p.ch : nullptr;
    T *dzp = a.dz ? (T *)a.dz + p.b * a.zsb + p.ch : nullptr;
    float sumD = 0.f, sumb = 0.f;
    int buf = 0;
    for (long long t = t1 > t0 ? (t1 - 1) / TILE * TILE : t0 - 1; t >= t0; t -= TILE) {
        const int left = (int)min(t1 - t, (long long)TILE);
        const long long bt = (long long)p.b * a.tiles + t / TILE;
        const float *tile = a.bc + (bt * a.G + p.g) * NPT * 2 * TILE + p.blk * NP * 2 * TILE;
        const float *ck = a.ck + (bt * a.Dp + p.pad) * NPT + p.blk * NP;
        float delta[TILE], slope[TILE], u[TILE], g[TILE], q[TILE], du[TILE], dd[TILE], y[TILE];
#pragma unroll
        for (int i = 0; i < TILE; ++i) {
            const long long at = t + min(i, left - 1);
            delta[i] = (float)dp[at * a.dst] + bias;
            u[i] = (float)xp[at * a.xst];
            g[i] = (float)dyp[at * a.yst];
            q[i] = zp ? (float)zp[at * a.zst] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < TILE; ++i) {
            slope[i] = 1.f;
            if (a.softplus) {
                slope[i] = sigmoid_f(delta[i]);
                delta[i] = softplus_f(delta[i]);
            }
            if (zp) {
                float silu;
                const float ds = dsilu(q[i], silu);
                q[i] = g[i] * ds;
                g[i] *= silu;
            }
            // (behind the last token, and where there is no channel, nothing is added anywhere)
            delta[i] = i < left ? delta[i] : 0.f;
            y[i] = Dk * u[i];
            u[i] = i < left && p.on ? delta[i] * u[i] : 0.f;
            g[i] = i < left && p.on ? g[i] : 0.f;
            du[i] = dd[i] = 0.f;
        }
        if (MULTI && p.blk > 0) {
#pragma unroll
            for (int i = 0; i < TILE; ++i) y[i] = 0.f;
        }
#pragma unroll 1
        for (int s = 0; s < NP; s += 2) {
            f32x16 Bv[2], Cv[2];
            float S[2][TILE], e[2][MULTI ? 1 : TILE], before[2], h[2], dA[2], A[2], Af[2];     // (a channel's factors are made again where registers are short)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                Bv[j] = bc_tile(tile, s + j, 0), Cv[j] = bc_tile(tile, s + j, 1);
                before[j] = ck[s + j];
                h[j] = mine[s + j][0][p.lane], dA[j] = mine[s + j][1][p.lane], A[j] = mine[s + j][2][p.lane];
                Af[j] = fmaxf(A[j], -3.4028235e38f);        // (where the rate is minus infinity p is 0, and so is its share)
            }
#pragma unroll
            for (int i = 0; i < TILE; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float f = factor(delta[i], A[j]);
                    if (!MULTI) e[j][MULTI ? 0 : i] = f;
                    S[j][i] = fmaf(f, i ? S[j][i ? i - 1 : 0] : before[j], u[i] * Bv[j][i]);
                    y[i] = fmaf(Cv[j][i], S[j][i], y[i]);
                }
            LaneSums sums;
            float all = 0.f;
#pragma unroll
            for (int i = TILE - 1; i >= 0; --i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int k = ((TILE - 1 - i) * 2 + j) * 2;
                    const float dS = fmaf(Cv[j][i], g[i], h[j]);
                    du[i] = fmaf(Bv[j][i], dS, du[i]);
                    h[j] = (MULTI ? factor(delta[i], A[j]) : e[j][MULTI ? 0 : i]) * dS;
                    const float pr = h[j] * (i ? S[j][i ? i - 1 : 0] : before[j]);
                    dd[i] = fmaf(Af[j], pr, dd[i]);
                    dA[j] = fmaf(delta[i], pr, dA[j]);
                    sums.push(k, u[i] * dS, p.lane);
                    all = sums.push(k + 1, g[i] * S[j][i], p.lane);
                }
#pragma unroll
            for (int j = 0; j < 2; ++j) mine[s + j][0][p.lane] = h[j], mine[s + j][1][p.lane] = dA[j];
            const int which = p.lane >> 5 & 1, j = p.lane >> 4 & 1;
            const int i = TILE - 1 - ((p.lane >> 3 & 1) | (p.lane >> 1 & 2) | (p.lane << 1 & 4) | (p.lane << 3 & 8));
            if (MULTI) {
                if (a.part_bc) a.part_bc[((((bt * TILE + i) * a.G + p.g) * a.parts + p.cb) * 2 + which) * NPT + p.blk * NP + s + j] = all;
            } else stage[buf][MULTI ? 0 : w][i][which][s + j] = all;
        }
        stay<TILE>(du);
        stay<TILE>(dd);
        stay<TILE>(y);
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
        if (MULTI) {        // the waves' shares of du, dd and y; wave i % NB goes on with token i
            auto exchange = [&](float(&v)[TILE]) {
#pragma unroll
                for (int i = 0; i < TILE; ++i) xch[MULTI ? p.blk : 0][i][p.lane] = v[i];
                __syncthreads();
#pragma unroll
                for (int i = 0; i < TILE; ++i) {
                    if (i % NB != p.blk) continue;
                    v[i] = 0.f;
#pragma unroll
                    for (int k = 0; k < NB; ++k) v[i] += xch[MULTI ? k : 0][i][p.lane];
                }
                __syncthreads();
            };
            exchange(du);
            exchange(dd);
            if (dzp) exchange(y);
        }
#pragma unroll
        for (int i = 0; i < TILE; ++i) {
            if (i >= left || (MULTI && i % NB != p.blk)) continue;
            const long long at = t + i;
            const float x = (float)xp[at * a.xst];
            const float dv = fmaf(du[i], x, dd[i] * LN2) * slope[i];
            sumD = fmaf(g[i], x, sumD);
            if (p.on) {
                sumb += dv;
                if (dxp) dxp[at * a.xst] = (T)fmaf(du[i], delta[i], Dk * g[i]);
                if (ddp) ddp[at * a.dst] = (T)dv;
                if (dzp) dzp[at * a.zst] = (T)(q[i] * y[i]);
            }
        }
    }
    if (p.on && p.blk == 0) {
        for (long long t = max(t0, (long long)n); t < end; ++t) {
            if (dxp) dxp[t * a.xst] = (T)0.f;
            if (ddp) ddp[t * a.dst] = (T)0.f;
            if (dzp) dzp[t * a.zst] = (T)0.f;
        }
    }
    if (!p.there) return;
    float h[NP], dA[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) h[i] = mine[i][0][p.lane], dA[i] = mine[i][1][p.lane];
    if (a.part_a) store_states<NP>(a.part_a + (seg * a.Dp + p.pad) * NPT + p.blk * NP, dA);
    if (a.part_d) {
        float *out = a.part_d + ((seg * NB + p.blk) * 2) * a.Dp + p.pad;
        out[0] = sumD, out[a.Dp] = sumb;
    }
    if (p.on && a.dstate_in && p.seg == 0) store_user<NP>(a.dstate_in, a, user, p.blk * NP, h);
}

// dB and dC: the workgroups' sums, in their order.
template <typename T> __global__ __launch_bounds__(256) void select_bc_sums(const Args a)
{
    const int NPT = a.NP * a.NB;
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int per = 2 * NPT, at = (int)(id % per), which = at / NPT, n = at % NPT;
    const long long rest = id / per, g = rest % a.G, bt = rest / a.G, b = bt / a.L, t = bt - b * a.L;
    if (b >= a.B || n >= a.N) return;
    T *out = (T *)(which ? a.dC : a.dB);
    if (!out) return;
    float v = 0.f;
    if (t < row_length(a, (int)b)) {
        const float *p = a.part_bc + (((b * a.tiles * TILE + t) * a.G + g) * a.parts) * per + at;
        for (int k = 0; k < a.parts; ++k) v += p[(long long)k * per];
    }
    out[b * a.bsb + t * a.bst + g * a.N + n] = (T)v;
}

int launch_bc_sums(const Args &a, bool bf16_, hipStream_t s)
{
    const dim3 grid((unsigned)ceil_div((long long)a.B * a.L * a.G * 2 * a.NP * a.NB, 256));
    if (a.L == 0) return CAWN_OK;
    if (bf16_) hipLaunchKernelGGL(select_bc_sums<bf16>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(select_bc_sums<float>, grid, dim3(256), 0, s, a);
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
    if (a.NB == 8) launch_np<T, 16, 8>(a, s);
    else if (a.NB == 4) launch_np<T, 16, 4>(a, s);
    else if (a.NB == 2) launch_np<T, 16, 2>(a, s);
    else if (a.NP == 16) launch_np<T, 16, 1>(a, s);
    else if (a.NP == 8) launch_np<T, 8, 1>(a, s);
    else launch_np<T, 4, 1>(a, s);
    return launched();
}

int launch_backward(const Args &a, bool bf16_, hipStream_t s) { return bf16_ ? launch<bf16>(a, s) : launch<float>(a, s); }

} // namespace select
} // namespace cawn
