// Selective state space scan, token by token: single tokens of a decoding step and calls of a few tokens.
//
// A lane owns four adjacent states of a channel for the whole call, a run of LPC lanes the channel: the state is read and written 16 bytes a lane in
// the order it lies in, and the run adds up its share of y.  Bound by the state's bytes, in and out, and for one row by a launch.
#include "cawn_select.hpp"

namespace cawn {
namespace select {

template <typename T, int LPC, bool VEC4> __global__ __launch_bounds__(256) void select_tokens(const Args a)
{
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x, at = id / LPC, bl = at / a.D;
    const int q = (int)(id % LPC), n0 = q * 4;
    if (bl >= a.B) return;      // (whole runs of lanes)
    const int b = (int)bl, ch = (int)(at - bl * a.D), n = row_length(a, b), g = ch / a.cg;
    const bool idle = n == 0 && (!a.state_out || a.state_out == a.state_in);    // nothing is asked of the state
    const long long sat = at * a.N + n0;
    const T *xp = (const T *)a.x + b * a.xsb + ch, *dp = (const T *)a.dt + b * a.dsb + ch;
    const T *zp = a.z ? (const T *)a.z + b * a.zsb + ch : nullptr;
    const T *Bp = (const T *)a.Bm + b * a.bsb + (long long)g * a.N, *Cp = (const T *)a.Cm + b * a.bsb + (long long)g * a.N;
    T xn = (T)0.f, dn = (T)0.f, zn = (T)0.f, Bn[4], Cn[4];
    auto fetch = [&](int t) {
        xn = xp[t * a.xst], dn = dp[t * a.dst];
        if (zp) zn = zp[t * a.zst];
#pragma unroll
        for (int j = 0; j < 4; ++j) Bn[j] = Bp[t * a.bst + min(n0 + j, a.N - 1)], Cn[j] = Cp[t * a.bst + min(n0 + j, a.N - 1)];
    };
    if (n > 0) fetch(0);
    float S[4] = {}, A[4];
    if (VEC4) {
        if (a.state_in && !idle && n0 < a.N) load_n<float, 4>(a.state_in + sat, S);
        load_n<float, 4>(a.A + (long long)ch * a.N + min(n0, a.N - 4), A);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            S[j] = a.state_in && !idle && n0 + j < a.N ? a.state_in[sat + j] : 0.f;
            A[j] = a.A[(long long)ch * a.N + min(n0 + j, a.N - 1)];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) A[j] = rate(A[j]);
    const float bias = a.bias ? a.bias[ch] : 0.f, Dk = a.Dk ? a.Dk[ch] : 0.f;
    T *yp = (T *)a.y + b * a.ysb + ch;
    for (int t = 0; t < n; ++t) {
        const float x = (float)xn, v = (float)dn + bias, z = (float)zn;
        float Bv[4], Cv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) Bv[j] = n0 + j < a.N ? (float)Bn[j] : 0.f, Cv[j] = n0 + j < a.N ? (float)Cn[j] : 0.f;
        if (t + 1 < n) fetch(t + 1);
        const float delta = a.softplus ? softplus_f(v) : v, u = delta * x;
        float y = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            S[j] = fmaf(factor(delta, A[j]), S[j], u * Bv[j]);
            y = fmaf(Cv[j], S[j], y);
        }
#pragma unroll
        for (int m = 1; m < LPC; m <<= 1) y += __shfl_xor(y, m);
        y = fmaf(Dk, x, y);
        if (zp) y *= z * sigmoid_f(z);
        if (q == 0) yp[t * a.yst] = (T)y;
    }
    for (int t = n; t < a.L; ++t)           // tokens that the row does not have
        if (q == 0) yp[t * a.yst] = (T)0.f;
    if (!a.state_out || idle) return;
    if (VEC4) {
        if (n0 < a.N) store_n<float, 4>(a.state_out + sat, S);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n0 + j < a.N) a.state_out[sat + j] = S[j];
    }
}

template <typename T> static int launch(const Args &a, hipStream_t s)
{
    int lpc = 1;
    while (lpc * 4 < a.N) lpc *= 2;
    const bool vec4 = a.N % 4 == 0 && aligned_to(a.state_in, 16) && aligned_to(a.state_out, 16) && aligned_to(a.A, 16);
    const long long blocks = ceil_div((long long)a.B * a.D * lpc, 256);
    if (blocks > 0x7fffffffLL) return CAWN_EUNSUPPORTED;
    const dim3 grid((unsigned)blocks);
#define CAWN_TOKENS(LPC)                                                                                        \
    case LPC:                                                                                                   \
        if (vec4) hipLaunchKernelGGL((select_tokens<T, LPC, true>), grid, dim3(256), 0, s, a);                   \
        else hipLaunchKernelGGL((select_tokens<T, LPC, false>), grid, dim3(256), 0, s, a);                       \
        break;
    switch (lpc) {
        CAWN_TOKENS(1)
        CAWN_TOKENS(2)
        CAWN_TOKENS(4)
        CAWN_TOKENS(8)
        CAWN_TOKENS(16)
        CAWN_TOKENS(32)
    }
#undef CAWN_TOKENS
    return launched();
}

int launch_token(const Args &a, bool bf16_, hipStream_t s) { return bf16_ ? launch<bf16>(a, s) : launch<float>(a, s); }

} // namespace select
} // namespace cawn
