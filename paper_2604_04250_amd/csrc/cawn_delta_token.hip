// Gated delta rule, token by token: single tokens of a decoding step and calls of a few tokens.
//
// A wave owns VS columns of one head's state (all K rows of them, in registers) for the whole call.  Per token it needs two products
// of the decayed state with vectors, r^T k and r^T q; with them
//     u = beta (v - r^T k),   o = scale (r^T q + (k.q) u),   S = r + k u^T,
// so one reduction over the rows serves both, and the squares of k and q for their norm ride along in it.  The norms' factors are
// applied behind the sums.  What bounds it: the state's bytes, in and out (K V 8 bytes a head), and for a few heads the latency of
// load, reduction and store.
#include "cawn_delta.hpp"

namespace cawn {
namespace delta {

template <typename T, int KP, int VS, bool VEC4> __global__ __launch_bounds__(64) void delta_tokens(const Args a)
{
    constexpr int CL = VS / 4, RG = 64 / CL, NR = KP / RG;      // lanes of a row, rows at a time, rows of a lane
    const int blk = blockIdx.x, slab = blk % a.slabs, h = blk / a.slabs % a.H, b = blk / a.slabs / a.H;
    const int lane = threadIdx.x, v0 = slab * VS + (lane % CL) * 4, r0 = (lane / CL) * NR;
    const int n = row_length(a, b), hk = h / (a.H / a.Hk);
    const long long sbase = ((long long)b * a.H + h) * a.K * a.V;
    float S[NR][4];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const long long at = sbase + (long long)(r0 + i) * a.V + v0;
        if (VEC4 && a.state_in && r0 + i < a.K && v0 < a.V) load_n<float, 4>(a.state_in + at, S[i]);
        else {
#pragma unroll
            for (int j = 0; j < 4; ++j) S[i][j] = a.state_in && r0 + i < a.K && v0 + j < a.V ? a.state_in[at + j] : 0.f;
        }
    }
    for (int t = 0; t < n; ++t) {
        const T *kp = (const T *)a.k + b * a.qsb + t * a.qst + (long long)hk * a.K, *qp = (const T *)a.q + b * a.qsb + t * a.qst + (long long)hk * a.K;
        const T *vp = (const T *)a.v + b * a.vsb + t * a.vst + (long long)h * a.V;
        const long long gate = ((long long)b * a.L + t) * a.H + h;
        const float alpha = expf(fmaxf(a.decay[gate], DECAY_MIN)), beta = a.beta[gate], bad = a.decay[gate];
        float v[4], k[NR], q[NR], sk[4] = {0.f, 0.f, 0.f, 0.f}, sq[4] = {0.f, 0.f, 0.f, 0.f}, kk = 0.f, qq = 0.f, kq = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = v0 + j < a.V ? (float)vp[v0 + j] : 0.f;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            k[i] = r0 + i < a.K ? (float)kp[r0 + i] : 0.f;
            q[i] = r0 + i < a.K ? (float)qp[r0 + i] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            kk = fmaf(k[i], k[i], kk), qq = fmaf(q[i], q[i], qq), kq = fmaf(k[i], q[i], kq);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sk[j] = fmaf(k[i], S[i][j], sk[j]);
                sq[j] = fmaf(q[i], S[i][j], sq[j]);
            }
        }
#pragma unroll
        for (int m = CL; m < 64; m <<= 1) {
            kk += __shfl_xor(kk, m), qq += __shfl_xor(qq, m), kq += __shfl_xor(kq, m);
#pragma unroll
            for (int j = 0; j < 4; ++j) sk[j] += __shfl_xor(sk[j], m), sq[j] += __shfl_xor(sq[j], m);
        }
        const float rk = a.norm ? 1.f / sqrtf(kk + a.eps) : 1.f, rq = a.norm ? 1.f / sqrtf(qq + a.eps) : 1.f;
        const float f = bad != bad ? bad : alpha;       // (fmaxf drops a NaN)
        float u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = beta * (v[j] - f * rk * sk[j]);
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) S[i][j] = fmaf(rk * k[i], u[j], f * S[i][j]);
        if (lane < CL) {
            T *op = (T *)a.o + b * a.osb + t * a.ost + (long long)h * a.V;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (v0 + j < a.V) op[v0 + j] = (T)(a.scale * rq * (f * sq[j] + rk * kq * u[j]));
        }
    }
    for (int t = n; t < a.L; ++t) {         // tokens that the row does not have
        if (lane < CL) {
            T *op = (T *)a.o + b * a.osb + t * a.ost + (long long)h * a.V;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (v0 + j < a.V) op[v0 + j] = (T)0.f;
        }
    }
    if (a.state_out && !(n == 0 && a.state_out == a.state_in)) {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const long long at = sbase + (long long)(r0 + i) * a.V + v0;
            if (VEC4 && r0 + i < a.K && v0 < a.V) store_n<float, 4>(a.state_out + at, S[i]);
            else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (r0 + i < a.K && v0 + j < a.V) a.state_out[at + j] = S[i][j];
            }
        }
    }
}

template <typename T, int VS> static void launch_vs(Args a, hipStream_t s)
{
    a.slabs = (int)ceil_div(a.V, VS);
    const dim3 grid((unsigned)((long long)a.B * a.H * a.slabs));
#define CAWN_TOKENS(KP)                                                                                                        \
    if (a.vec4) hipLaunchKernelGGL((delta_tokens<T, KP, VS, true>), grid, dim3(64), 0, s, a);                                   \
    else hipLaunchKernelGGL((delta_tokens<T, KP, VS, false>), grid, dim3(64), 0, s, a);
    if (a.K <= 32) { CAWN_TOKENS(32) }
    else if (a.K <= 64) { CAWN_TOKENS(64) }
    else { CAWN_TOKENS(128) }
#undef CAWN_TOKENS
}

int launch_token(const Args &a, bool bf16_, hipStream_t s)
{
    // narrow slabs where wide ones would leave compute units without a wave; wide ones read whole 128-byte lines
    const bool narrow = (long long)a.B * a.H * ceil_div(a.V, 32) < 1024;
    if ((long long)a.B * a.H * ceil_div(a.V, 16) > 0x7fffffffLL) return CAWN_EUNSUPPORTED;
    if (bf16_) narrow ? launch_vs<bf16, 16>(a, s) : launch_vs<bf16, 32>(a, s);
    else narrow ? launch_vs<float, 16>(a, s) : launch_vs<float, 32>(a, s);
    return launched();
}

} // namespace delta
} // namespace cawn
