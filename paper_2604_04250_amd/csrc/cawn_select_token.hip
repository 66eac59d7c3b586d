// Selective state space scan, token by token: single tokens of a decoding step and calls of a few tokens.
//
// A lane owns four or eight adjacent states of a channel for the whole call, a run of LPC lanes the channel: the state is read and written 16 bytes at a time
// in the order it lies in, and the run adds up its share of y.  Bound by the state's bytes, in and out, and for one row by a launch: 128 rows of 4,096 channels
// of 16 states, an eighth of the slots unused, 15 us (4.4 TB/s of 67 MB), one row of 768 channels 3.7.
#include "cawn_select.hpp"

namespace cawn {
namespace select {

// W adjacent values of B or C (16 bytes at a time at most where VEC, else one by one and those that there are)
template <typename T, int W, bool VEC> __device__ inline void load_some(const T *p, int n0, int N, T (&v)[W])
{
    if (VEC) {
#pragma unroll
        for (int i = 0; i < W; i += 4) {
            const Pack<T, 4> x = *reinterpret_cast<const Pack<T, 4> *>(p + min(n0 + i, N - 4));
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i + j] = x.v[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = p[min(n0 + j, N - 1)];
    }
}

// LPC lanes to a channel, W states to a lane
template <typename T, int LPC, int W, bool VEC> __global__ __launch_bounds__(256) void select_tokens(const Args a)
{
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x, at = id / LPC, bl = at / a.D;
    const int q = (int)(id % LPC), n0 = q * W;
    if (bl >= a.B) return;      // (whole runs of lanes)
    const int b = (int)bl, ch = (int)(at - bl * a.D), g = ch / a.cg;
    const bool in_place = !a.state_out || a.state_out == a.state_in;
    const long long sat = at * a.N;
    float S[W], A[W];
    auto load_state = [&] {
        load_some<float, W, VEC>(a.state_in + sat, n0, a.N, S);
    };
#pragma unroll
    for (int j = 0; j < W; ++j) S[j] = 0.f;
    if (a.state_in && !in_place) load_state();      // (before the row's length is known)
    load_some<float, W, VEC>(a.A + (long long)ch * a.N, n0, a.N, A);
    const float bias = a.bias ? a.bias[ch] : 0.f, Dk = a.Dk ? a.Dk[ch] : 0.f;
    const int n = row_length(a, b);
    if (a.state_in && in_place && n > 0) load_state();          // (nothing is asked of an unused slot's state in its place)
    const T *xp = (const T *)a.x + b * a.xsb + ch, *dp = (const T *)a.dt + b * a.dsb + ch;
    const T *zp = a.z ? (const T *)a.z + b * a.zsb + ch : nullptr;
    const T *Bp = (const T *)a.Bm + b * a.bsb + (long long)g * a.N, *Cp = (const T *)a.Cm + b * a.bsb + (long long)g * a.N;
    T xn = (T)0.f, dn = (T)0.f, zn = (T)0.f, Bn[W], Cn[W];
    auto fetch = [&](int t) {
        xn = xp[t * a.xst], dn = dp[t * a.dst];
        if (zp) zn = zp[t * a.zst];
        load_some<T, W, VEC>(Bp + t * a.bst, n0, a.N, Bn);
        load_some<T, W, VEC>(Cp + t * a.bst, n0, a.N, Cn);
    };
    if (n > 0) fetch(0);
#pragma unroll
    for (int j = 0; j < W; ++j) A[j] = rate(A[j]);
    T *yp = (T *)a.y + b * a.ysb + ch;
    for (int t = 0; t < n; ++t) {
        const float x = (float)xn, v = (float)dn + bias, z = (float)zn;
        float Bv[W], Cv[W];
#pragma unroll
        for (int j = 0; j < W; ++j) Bv[j] = n0 + j < a.N ? (float)Bn[j] : 0.f, Cv[j] = n0 + j < a.N ? (float)Cn[j] : 0.f;
        if (t + 1 < n) fetch(t + 1);
        const float delta = a.softplus ? softplus_f(v) : v, u = delta * x;
        float y = 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            S[j] = fmaf(factor(delta, A[j]), S[j], u * Bv[j]);
            y = fmaf(Cv[j], n0 + j < a.N ? S[j] : 0.f, y);
        }
#pragma unroll
        for (int m = 1; m < LPC; m <<= 1) y += __shfl_xor(y, m);
        y = fmaf(Dk, x, y);
        if (zp) y *= z * sigmoid_f(z);
        if (q == 0) yp[t * a.yst] = (T)y;
    }
    for (int t = n; t < a.L; ++t)           // tokens that the row does not have
        if (q == 0) yp[t * a.yst] = (T)0.f;
    if (!a.state_out || (in_place && n == 0 && a.state_in)) return;
#pragma unroll
    for (int i = 0; i < W; i += VEC ? 4 : 1) {
        if constexpr (VEC) {
            const float v[4] = {S[i], S[i + 1], S[i + 2], S[i + 3]};
            if (n0 + i < a.N) store_n<float, 4>(a.state_out + sat + n0 + i, v);
        } else if (n0 + i < a.N) a.state_out[sat + n0 + i] = S[i];
    }
}

template <typename T> static int launch(const Args &a, hipStream_t s)
{
    const int w = token_states(a), lpc = token_lanes(a);
    const bool vec4 = a.N % 4 == 0 && aligned_to(a.state_in, 16) && aligned_to(a.state_out, 16) && aligned_to(a.A, 16) && a.bst % 4 == 0 && a.bsb % 4 == 0 &&
                      aligned_to(a.Bm, 4 * sizeof(T)) && aligned_to(a.Cm, 4 * sizeof(T));
    const dim3 grid((unsigned)ceil_div((long long)a.B * a.D * lpc, 256));
#define CAWN_TOKENS(LPC, W)                                                                                        \
    case LPC:                                                                                                   \
        if (vec4) hipLaunchKernelGGL((select_tokens<T, LPC, W, true>), grid, dim3(256), 0, s, a);                \
        else hipLaunchKernelGGL((select_tokens<T, LPC, W, false>), grid, dim3(256), 0, s, a);                    \
        break;
    if (w == 8) switch (lpc) {
        CAWN_TOKENS(1, 8)
        CAWN_TOKENS(2, 8)
        CAWN_TOKENS(4, 8)
        CAWN_TOKENS(8, 8)
        CAWN_TOKENS(16, 8)
    }
    else switch (lpc) {
        CAWN_TOKENS(1, 4)
        CAWN_TOKENS(2, 4)
        CAWN_TOKENS(4, 4)
        CAWN_TOKENS(8, 4)
        CAWN_TOKENS(16, 4)
        CAWN_TOKENS(32, 4)
    }
#undef CAWN_TOKENS
    return launched();
}

int launch_token(const Args &a, bool bf16_, hipStream_t s) { return bf16_ ? launch<bf16>(a, s) : launch<float>(a, s); }

} // namespace select
} // namespace cawn
