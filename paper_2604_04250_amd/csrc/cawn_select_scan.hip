// Selective state space scan by tiles of 16 tokens, forward.
//
// Four launches: B and C as the kernels read them; what each segment of a row makes of a zero state (its last states and the sum of delta: the
// product of its factors is exp(A sum delta)); the chain over the segments; and all segments from their true states.  The second costs each state's
// exponential and update twice, so that a few rows of many channels fill the chip; one segment does without it and the chain.
// What bounds it: instruction issue.  A token's state costs a product, an exponential (two issue slots), a product and two sums (without y one), 24 (20) cycles
// of a SIMD a wave, and a token 27 (15) instructions more for softplus, the gate, conversions and memory.  2 x 32,768 tokens of 4,096 channels of 16 states in
// bf16: 703 us without y, 904 with it, vector units busy for 99 % of both; the chain 18, B and C 9.
// Runs of eight tokens: with 16 the registers of two more waves a SIMD are gone (the same call 1,673 us for 1,579).
#include "cawn_select.hpp"

namespace cawn {
namespace select {

// bc[b][tile][g][n][which][token of the tile]; zeros where there is no token or state.  A workgroup takes a tile of a group, read along the states and
// written along the tokens; beyond PREPARE_BLOCKS of them the workgroups go round.
constexpr long long PREPARE_BLOCKS = 1 << 16;

template <typename T> __global__ __launch_bounds__(256) void select_prepare(const Args a)
{
    __shared__ float sh[2][TILE][N_MAX + 1];
    const int npt = a.NP * a.NB;
    for (unsigned at = blockIdx.x, all = (unsigned)a.B * a.tiles * a.G; at < all; at += gridDim.x) {
        if (at != blockIdx.x) __syncthreads();      // (the tile before has been written)
        const unsigned bt = at / (unsigned)a.G, row = bt / (unsigned)a.tiles;
        const long long b = row, t = (long long)(bt - row * a.tiles) * TILE;
        const int g = (int)(at - bt * a.G), left = row_length(a, (int)row) - (int)t;
        for (int i = threadIdx.x; i < 2 * TILE * npt; i += 256) {
            const int n = i % npt, tt = i / npt % TILE, which = i / npt / TILE;
            sh[which][tt][n] = n < a.N && tt < left ? (float)((const T *)(which ? a.Cm : a.Bm))[b * a.bsb + (t + tt) * a.bst + (long long)g * a.N + n] : 0.f;
        }
        __syncthreads();
        float *out = a.bc + (long long)at * npt * 2 * TILE;
        for (int i = threadIdx.x; i < 2 * TILE * npt; i += 256) out[i] = sh[i / TILE % 2][i % TILE][i / TILE / 2];
    }
}

// RUN tokens at a time, the next ones' streams on their way meanwhile.  NB waves share a channel's states: of a run's tokens each has every NB-th for its own,
// makes their delta and u for all, and their y from all shares (67 tokens of 15 rows of 284 channels of 128 states 45 us, each wave all of them 56;
// 4 x 2,048 of 1,024 of 24 110, 117).
template <typename T, int NP, int NB, bool SUMMARY> __global__ __launch_bounds__(NB > 1 ? 64 * NB : 256) void select_scan(const Args a)
{
    constexpr bool MULTI = NB > 1;
    constexpr bool SHARE = NB > 2 || (MULTI && !SUMMARY);              // (two waves without a barrier for y are better off without one for delta)
    constexpr int NPT = NP * NB, AHEAD = 2, OWN = SHARE ? RUN / NB : RUN;
    __shared__ float ys[2][MULTI && !SUMMARY ? NB : 1][RUN][64];        // the waves' shares of y
    __shared__ float2 shared[2][SHARE ? RUN : 1][64];                   // delta and u (two buffers: a wave may be a run ahead of another)
    const Place p = place_of<MULTI>(a);
    if (!MULTI && !p.there) return;
    const int n = __builtin_amdgcn_readfirstlane(row_length(a, p.b));
    const int t0 = p.seg * a.seg_tiles * TILE, t1 = min(n, t0 + a.seg_tiles * TILE), end = min(a.L, t0 + a.seg_tiles * TILE);
    if (SUMMARY && (t0 >= t1 || t1 == n)) return;       // (the chain ends before it)
    const long long sat = (((long long)p.b * a.segments + p.seg) * a.Dp + p.pad) * NPT + p.blk * NP;
    const long long user = (long long)p.b * a.D + p.ch;
    const T *xp = (const T *)a.x + p.b * a.xsb + p.base + t0 * a.xst, *dp = (const T *)a.dt + p.b * a.dsb + p.base + t0 * a.dst;
    const T *zp = !SUMMARY && a.z ? (const T *)a.z + p.b * a.zsb + p.base + t0 * a.zst : nullptr;
    const uint32_t at = p.bytes<T>();
    auto step = [](long long stride) { return (uint32_t)stride * (uint32_t)sizeof(T); };
    uint32_t xr[OWN], dr[OWN], zr[SUMMARY ? 1 : OWN];
    auto load_own = [&](const T *row, long long stride, int left, uint32_t(&v)[OWN]) {
        if constexpr (!SHARE) load_run<T, RUN>(row, step(stride), left, at, v);
        else {
            const auto r = rows_at(row);
#pragma unroll
            for (int k = 0; k < OWN; ++k) v[k] = load_at<T>(r, at, (uint32_t)min(k * NB + p.blk, left - 1) * step(stride));
        }
    };
    auto fetch = [&](int t) {
        const int left = t1 - t;
        if (left > 0) {
            load_own(dp, a.dst, left, dr);
            load_own(xp, a.xst, left, xr);
            dp += RUN * a.dst, xp += RUN * a.xst;
        } else no_run<OWN>(dr), no_run<OWN>(xr);
    };
    fetch(t0);
    float A[NP], S[NP], total = 0.f;
    load_rates<NP>(a, p, A);
#pragma unroll
    for (int i = 0; i < NP; ++i) S[i] = 0.f;
    if (!SUMMARY) {
        if (a.segments > 1) {
            if (t0 < t1 || (p.seg == 0 && n == 0)) load_states<NP>(a.seg_s + sat, S);
        } else if (a.state_in) load_user<NP>(a.state_in, a, user, p.blk * NP, S);
    }
    const float bias = a.bias ? a.bias[p.ch] : 0.f, Dk = a.Dk ? a.Dk[p.ch] : 0.f;
    T *yp = SUMMARY ? nullptr : (T *)a.y + p.b * a.ysb + p.base + t0 * a.yst;
    int buf = 0;
    // the wave's own tokens: delta, u and x
    float delta_own[OWN], u_own[OWN], x_own[OWN];
    auto begin = [&](int left) {
#pragma unroll
        for (int k = 0; k < OWN; ++k) {
            delta_own[k] = value<T>(dr[k]) + bias, u_own[k] = value<T>(xr[k]);
            x_own[k] = u_own[k];
        }
        if (a.softplus) {
#pragma unroll
            for (int k = 0; k < OWN; ++k) delta_own[k] = softplus_f(delta_own[k]);
        }
#pragma unroll
        for (int k = 0; k < OWN; ++k) u_own[k] *= delta_own[k];
        if (left < RUN) {           // behind the last token nothing changes
#pragma unroll
            for (int k = 0; k < OWN; ++k) {
                const bool there = k * NB + p.blk < left;
                delta_own[k] = there ? delta_own[k] : 0.f;
                u_own[k] = there ? u_own[k] : 0.f;
            }
        }
    };
    auto hand_out = [&](int to) {
#pragma unroll
        for (int k = 0; k < OWN; ++k) shared[to][SHARE ? k * NB + p.blk : 0][p.lane] = make_float2(delta_own[k], u_own[k]);
    };
    if (SHARE && t0 < t1) {
        begin(t1 - t0);
        hand_out(0);
        fetch(t0 + RUN);
        __syncthreads();
    }
    for (int t = t0; t < t1; t += RUN) {
        const int left = t1 - t;
        const float *tile = a.bc + (((long long)p.b * a.tiles + t / TILE) * a.G + p.g) * NPT * 2 * TILE + p.blk * NP * 2 * TILE + t % TILE;
        if (!SUMMARY && a.ck && p.there && t % TILE == 0) store_states<NP>(a.ck + (((long long)p.b * a.tiles + t / TILE) * a.Dp + p.pad) * NPT + p.blk * NP, S);
        Scalars<RUN> Bq[NP], Cq[NP];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            Bq[s] = bc_run<RUN>(tile, s, 0);
            if (!SUMMARY) Cq[s] = bc_run<RUN>(tile, s, 1);
        }
        float delta[RUN], u[RUN], y[SUMMARY ? 1 : RUN], x[OWN];
        if constexpr (!SHARE) {
#pragma unroll
            for (int i = 0; i < RUN; ++i) {
                delta[i] = value<T>(dr[i]) + bias, u[i] = value<T>(xr[i]);
                if constexpr (!SUMMARY) y[i] = Dk * u[i];
            }
            if (a.softplus) {
#pragma unroll
                for (int i = 0; i < RUN; ++i) delta[i] = softplus_f(delta[i]);
            }
#pragma unroll
            for (int i = 0; i < RUN; ++i) u[i] *= delta[i];
            if (left < RUN) {
#pragma unroll
                for (int i = 0; i < RUN; ++i) {
                    delta[i] = i < left ? delta[i] : 0.f;
                    u[i] = i < left ? u[i] : 0.f;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < RUN; ++i) {
                const float2 v = shared[buf][SHARE ? i : 0][p.lane];
                delta[i] = v.x, u[i] = v.y;
                if constexpr (!SUMMARY) y[i] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < OWN; ++k) x[k] = x_own[k];
        }
        if constexpr (SUMMARY) {
#pragma unroll
            for (int i = 0; i < RUN; ++i) total += delta[i];
        } else {
            if (zp) {
                load_own(zp, a.zst, left, zr);
                zp += RUN * a.zst;
            } else no_run<OWN>(zr);
        }
        if (!SHARE) fetch(t + RUN);
        // (B and C of the state after next are asked for behind the first token of this one, whose wait would be for them too; without the fences the
        // compiler asks for all at once and keeps them in lanes of vector registers)
#pragma unroll
        for (int s = 0; s < NP; ++s) {
#pragma unroll
            for (int i = 0; i < RUN; ++i) {
                S[s] = fmaf(factor(delta[i], A[s]), S[s], u[i] * Bq[s][i]);
                if constexpr (!SUMMARY) y[i] = fmaf(Cq[s][i], S[s], y[i]);
                if (i == 0 && s + AHEAD < NP) {
                    __builtin_amdgcn_sched_barrier(0);
                    Bq[s + AHEAD < NP ? s + AHEAD : 0] = bc_run<RUN>(tile, s + AHEAD, 0);
                    if constexpr (!SUMMARY) Cq[s + AHEAD < NP ? s + AHEAD : 0] = bc_run<RUN>(tile, s + AHEAD, 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (!SUMMARY) stay<RUN>(y);
        if (SHARE) {
            if (t + RUN < t1) {
                begin(left - RUN);
                hand_out(buf ^ 1);
            }
            fetch(t + 2 * RUN);
            if constexpr (!SUMMARY) {
#pragma unroll
                for (int i = 0; i < RUN; ++i) ys[buf][MULTI ? p.blk : 0][i][p.lane] = y[i];
            }
            __syncthreads();
        }
        if constexpr (!SUMMARY) {
            if constexpr (MULTI) {
#pragma unroll
                for (int k = 0; k < OWN; ++k) {
                    y[k] = Dk * x[k];
#pragma unroll
                    for (int m = 0; m < NB; ++m) y[k] += ys[buf][MULTI ? m : 0][k * NB + p.blk][p.lane];
                }
            }
            if (zp) {
#pragma unroll
                for (int k = 0; k < OWN; ++k) {
                    const float z = value<T>(zr[k]);
                    y[k] *= z * sigmoid_f(z);
                }
            }
            if (p.on) {
                if (!MULTI) store_run<T, RUN>(yp, step(a.yst), left, at, [&](int i) { return y[i]; });
                else {
#pragma unroll
                    for (int k = 0; k < OWN; ++k)
                        if (k * NB + p.blk < left) store_at<T>(rows_at(yp + (k * NB + p.blk) * a.yst), at, 0, y[k]);
                }
            }
            yp += RUN * a.yst;
        }
        buf ^= 1;
    }
    if (SUMMARY) {
        store_states<NP>(a.seg_b + sat, S);
        if (p.blk == 0) a.seg_g[((long long)p.b * a.segments + p.seg) * a.Dp + p.pad] = total;
        return;
    }
    if (p.on && p.blk == 0)
        for (int t = max(t0, n); t < end; ++t) store_at<T>(rows_at((T *)a.y + p.b * a.ysb + p.base + t * a.yst), at, 0, 0.f);
    // the segment of the row's last token, or of a row without any the first
    if (p.on && a.state_out && (n == 0 ? p.seg == 0 : t0 < t1 && t1 == n)) store_user<NP>(a.state_out, a, user, p.blk * NP, S);
}

// The chain over the segments.  Forward: their states at the begin; backward: what reaches their end, from the last that a row has to the first.
// The links are cut into RUNS runs of up to LINKS, which are joined first: no link's loads wait for another link.  Where the runs are many the workgroups are larger,
// so that a run's threads read 128 bytes side by side (the call of 4,096 tokens of 768 channels 47.4 us, with 64 bytes 49.4).
template <bool REV, int RUNS, int LINKS, int THREADS> __global__ __launch_bounds__(THREADS) void select_join(const Args a)
{
    constexpr int WIDE = THREADS / RUNS;            // states side by side
    __shared__ float2 sh[RUNS][WIDE];
    const int NPT = a.NP * a.NB, e = threadIdx.x % WIDE, run = threadIdx.x / WIDE;
    const long long per = (long long)a.Dp * NPT, groups = per / WIDE, b = blockIdx.x / groups, i = (blockIdx.x - b * groups) * WIDE + e, pad = i / NPT;
    const int s = (int)(i - pad * NPT), g = (int)(pad / 64 / a.cpg), in = (int)(pad - (long long)g * a.cpg * 64);
    const bool on = in < a.cg && s < a.N;
    const long long ch = (long long)g * a.cg + in;
    const int seg_tokens = a.seg_tiles * TILE, live = (__builtin_amdgcn_readfirstlane(row_length(a, (int)b)) + seg_tokens - 1) / seg_tokens;
    // link k leads from the k-th segment to the next
    const int links = live > 0 ? live - 1 : 0, first = run * LINKS;
    const long long seg0 = b * a.segments + (REV ? (live > 0 ? live - 1 : 0) : 0), to = REV ? -1 : 1;
    float gs[LINKS], bs[LINKS];
#pragma unroll
    for (int j = 0; j < LINKS; ++j) {           // (behind the last, the last again: a load behind a branch would be waited for by itself)
        const long long seg = seg0 + to * max(min(first + j, links - 1), 0);
        gs[j] = a.seg_g[seg * a.Dp + pad], bs[j] = a.seg_b[seg * per + i];
    }
    const float A = on ? rate(a.A[ch * a.N + s]) : 0.f;
    const float *begin = REV ? a.dstate_out : a.state_in;
    float S = on && begin ? begin[(b * a.D + ch) * a.N + s] : 0.f;
    float product = 1.f, from_zero = 0.f;
#pragma unroll
    for (int j = 0; j < LINKS; ++j) {
        const bool link = first + j < links;
        gs[j] = factor(link ? gs[j] : 0.f, A), bs[j] = link ? bs[j] : 0.f;          // (no link: 1 and 0)
        from_zero = fmaf(gs[j], from_zero, bs[j]);
        product *= gs[j];
    }
    if (RUNS > 1) {
        sh[run][e] = make_float2(product, from_zero);
        __syncthreads();
        for (int r = 0; r < run; ++r) S = fmaf(sh[r][e].x, S, sh[r][e].y);
    }
    if (run == 0) a.seg_s[seg0 * per + i] = S;
#pragma unroll
    for (int j = 0; j < LINKS; ++j) {           // a link writes the segment behind it
        S = fmaf(gs[j], S, bs[j]);
        if (first + j < links) a.seg_s[(seg0 + to * (first + j + 1)) * per + i] = S;
    }
}

template <bool REV, int RUNS, int LINKS, int THREADS> static void go_join(const Args &a, hipStream_t s)
{
    hipLaunchKernelGGL((select_join<REV, RUNS, LINKS, THREADS>), dim3((unsigned)((long long)a.B * a.Dp * a.NP * a.NB * RUNS / THREADS)), dim3(THREADS), 0, s, a);
}

template <bool REV> static void join(const Args &a, hipStream_t s)
{
    const int links = a.segments - 1;
    if (links <= 4) go_join<REV, 1, 4, 256>(a, s);
    else if (links <= 16) go_join<REV, 4, 4, 256>(a, s);
    else if (links <= 32) go_join<REV, 4, 8, 256>(a, s);
    else if (links <= 64) go_join<REV, 4, 16, 512>(a, s);
    else if (links <= 128) go_join<REV, 16, 8, 512>(a, s);
    else go_join<REV, 16, 16, 512>(a, s);
}

int launch_join(const Args &a, bool reverse, hipStream_t s)
{
    reverse ? join<true>(a, s) : join<false>(a, s);
    return launched();
}

template <typename T, int NP, int NB> static void launch_np(const Args &a, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)a.B * a.segments * a.G * a.cbg)), block(64 * (NB > 1 ? NB : a.wide));
    if (a.segments > 1) {
        hipLaunchKernelGGL((select_scan<T, NP, NB, true>), grid, block, 0, s, a);
        launch_join(a, false, s);
    }
    hipLaunchKernelGGL((select_scan<T, NP, NB, false>), grid, block, 0, s, a);
}

template <typename T> static int launch(const Args &a, hipStream_t s)
{
    const long long all = (long long)a.B * a.tiles * a.G;
    if (all > 0) {
        hipLaunchKernelGGL((select_prepare<T>), dim3((unsigned)(all < PREPARE_BLOCKS ? all : PREPARE_BLOCKS)), dim3(256), 0, s, a);
        if (int r = launched()) return r;           // (without B and C the scan would write over y and the state what is none)
    }
    by_states(a, [&](auto np, auto nb) { launch_np<T, decltype(np)::value, decltype(nb)::value>(a, s); });
    return launched();
}

int launch_forward(const Args &a, bool bf16_, hipStream_t s) { return bf16_ ? launch<bf16>(a, s) : launch<float>(a, s); }

} // namespace select
} // namespace cawn
