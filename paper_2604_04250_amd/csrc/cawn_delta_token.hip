// Gated delta rule, token by token: single tokens of a decoding step and calls of a few tokens.
//
// A workgroup owns VS columns of one head's state (all K rows of them, in registers) for the whole call.  Per token it needs two products
// of the decayed state with vectors, r^T k and r^T q; with them
//     u = beta (v - r^T k),   o = scale (r^T q + (k.q) u),   S = r + k u^T,
// so one reduction over the rows serves both, and the squares of k and q for their norm ride along in it.  The norms' factors are
// applied behind the sums.  What bounds it: the state's bytes, in and out (K V 8 bytes a head), and for a few heads the latency of
// load, reduction and store.  Measured: one token of 128 rows of 32 heads of 128 x 128 (537 MB of state) in 101 us, 5.3 TB/s; one row of 12
// heads of 64 in 5 us, the time of a launch.
#include "cawn_delta.hpp"

namespace cawn {
namespace delta {

// N adjacent elements in as few accesses as 16 bytes allow; p aligned to them
template <typename T, int N> __device__ inline void load_raw(const T *p, T (&x)[N])
{
    constexpr int W = N * sizeof(T) <= 16 ? N : 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < N; i += W) {
        const Pack<T, W> y = *reinterpret_cast<const Pack<T, W> *>(p + i);
#pragma unroll
        for (int j = 0; j < W; ++j) x[i + j] = y.v[j];
    }
}

// NW waves share the rows; VS columns, four a lane
template <typename T, int KP, int VS, int NW, bool VEC4> __global__ __launch_bounds__(64 * NW) void delta_tokens(const Args a)
{
    constexpr int CL = VS / 4, RG = 64 / CL, NR = KP / (RG * NW);      // lanes of a row, rows of a wave at a time, rows of a lane
    static_assert(NR >= 1, "rows");
    __shared__ float sums[2][NW][CL][12];
    const int blk = blockIdx.x, slab = blk % a.slabs, h = blk / a.slabs % a.H, b = blk / a.slabs / a.H;
    const int w = threadIdx.x / 64, lane = threadIdx.x % 64, v0 = slab * VS + (lane % CL) * 4, r0 = (w * RG + lane / CL) * NR;
    const int n = row_length(a, b), hk = h / (a.H / a.Hk);
    const long long sbase = ((long long)b * a.H + h) * a.K * a.V;
    const bool idle = n == 0 && (!a.state_out || a.state_out == a.state_in);    // nothing is asked of the state
    // A token's inputs.  What is not there is loaded from where something is and dropped where it is used: a load behind a lane's branch, or
    // one converted at once, would be waited for by itself
    T kn[NR], qn[NR], vn[4];
    float decay, beta;
    auto fetch = [&](int t) {
        const T *kp = (const T *)a.k + b * a.qsb + t * a.qst + (long long)hk * a.K, *qp = (const T *)a.q + b * a.qsb + t * a.qst + (long long)hk * a.K;
        const T *vp = (const T *)a.v + b * a.vsb + t * a.vst + (long long)h * a.V;
        const long long gate = ((long long)b * a.L + t) * a.H + h;
        decay = a.decay[gate], beta = a.beta[gate];
        if (a.vecq) {                           // (K a multiple of 8: a lane's rows are there or not)
            load_raw<T, NR>(kp + min(r0, a.K - NR), kn);
            load_raw<T, NR>(qp + min(r0, a.K - NR), qn);
        } else {
#pragma unroll
            for (int i = 0; i < NR; ++i) kn[i] = kp[min(r0 + i, a.K - 1)], qn[i] = qp[min(r0 + i, a.K - 1)];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) vn[j] = vp[min(v0 + j, a.V - 1)];
    };
    if (n > 0) fetch(0);
    float S[NR][4];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const long long at = sbase + (long long)min(r0 + i, a.K - 1) * a.V;
        if (!a.state_in || idle) {
#pragma unroll
            for (int j = 0; j < 4; ++j) S[i][j] = 0.f;
        } else if (VEC4) load_n<float, 4>(a.state_in + at + min(v0, a.V - 4), S[i]);
        else {
#pragma unroll
            for (int j = 0; j < 4; ++j) S[i][j] = a.state_in[at + min(v0 + j, a.V - 1)];
        }
    }
    for (int t = 0; t < n; ++t) {
        const float alpha = expf(decay < DECAY_MIN ? DECAY_MIN : decay), be = beta;
        float v[4], k[NR], q[NR], x[11];        // sums: r^T k (4), r^T q (4), k.k, q.q, k.q
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)vn[j];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            k[i] = r0 + i < a.K ? (float)kn[i] : 0.f;
            q[i] = r0 + i < a.K ? (float)qn[i] : 0.f;
        }
        if (t + 1 < n) fetch(t + 1);
#pragma unroll
        for (int j = 0; j < 11; ++j) x[j] = 0.f;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            x[8] = fmaf(k[i], k[i], x[8]), x[9] = fmaf(q[i], q[i], x[9]), x[10] = fmaf(k[i], q[i], x[10]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = fmaf(k[i], S[i][j], x[j]);
                x[4 + j] = fmaf(q[i], S[i][j], x[4 + j]);
            }
        }
#pragma unroll
        for (int m = CL; m < 64; m <<= 1) {
#pragma unroll
            for (int j = 0; j < 11; ++j) x[j] += __shfl_xor(x[j], m);
        }
        if (NW > 1) {                           // (two buffers: a wave may be a token ahead of another)
            if (lane < CL) {
#pragma unroll
                for (int j = 0; j < 11; ++j) sums[t & 1][w][lane][j] = x[j];
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 11; ++j) {
                x[j] = 0.f;
#pragma unroll
                for (int p = 0; p < NW; ++p) x[j] += sums[t & 1][p][lane % CL][j];
            }
        }
        const float rk = a.norm ? 1.f / sqrtf(x[8] + a.eps) : 1.f, rq = a.norm ? 1.f / sqrtf(x[9] + a.eps) : 1.f;
        float u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = be * (v[j] - alpha * rk * x[j]);
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) S[i][j] = fmaf(rk * k[i], u[j], alpha * S[i][j]);
        if (w == 0 && lane < CL) {
            T *op = (T *)a.o + b * a.osb + t * a.ost + (long long)h * a.V;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (v0 + j < a.V) op[v0 + j] = (T)(a.scale * rq * (alpha * x[4 + j] + rk * x[10] * u[j]));
        }
    }
    for (int t = n; t < a.L; ++t) {         // tokens that the row does not have
        if (w == 0 && lane < CL) {
            T *op = (T *)a.o + b * a.osb + t * a.ost + (long long)h * a.V;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (v0 + j < a.V) op[v0 + j] = (T)0.f;
        }
    }
    if (!a.state_out || idle) return;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const long long at = sbase + (long long)(r0 + i) * a.V + v0;
        if (VEC4) {
            if (r0 + i < a.K && v0 < a.V) store_n<float, 4>(a.state_out + at, S[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (r0 + i < a.K && v0 + j < a.V) a.state_out[at + j] = S[i][j];
        }
    }
}

template <typename T, int VS, int NW> static void launch_vs(Args a, hipStream_t s)
{
    a.slabs = (int)ceil_div(a.V, VS);
    const dim3 grid((unsigned)((long long)a.B * a.H * a.slabs));
#define CAWN_TOKENS(KP)                                                                                                        \
    if (a.vec4) hipLaunchKernelGGL((delta_tokens<T, KP, VS, NW, true>), grid, dim3(64 * NW), 0, s, a);                           \
    else hipLaunchKernelGGL((delta_tokens<T, KP, VS, NW, false>), grid, dim3(64 * NW), 0, s, a);
    if (a.K <= 32) { CAWN_TOKENS(32) }
    else if (a.K <= 64) { CAWN_TOKENS(64) }
    else { CAWN_TOKENS(128) }
#undef CAWN_TOKENS
}

int launch_token(const Args &a, bool bf16_, hipStream_t s)
{
    // Four waves to 64 columns, whole lines; one wave to 16, which has no barrier in a token, where that would leave compute units without
    // work.  (One token, 128 rows of 32 heads of 128 x 128: one wave to 32 columns 149 us, two waves 140, two to 64 142, four to 64 128, eight
    // to 128 152, before loads were fetched ahead, which took four to 64 to 101.  Narrow against four waves: 16 tokens of 12 heads of 64
    // 19.3 us, 22.2; one token of 4 rows of 32 heads of 128 7.7 us, 6.1.)
    const bool narrow = (long long)a.B * a.H * ceil_div(a.V, 64) < 256;
    if ((long long)a.B * a.H * ceil_div(a.V, 16) > 0x7fffffffLL) return CAWN_EUNSUPPORTED;
    if (bf16_) narrow ? launch_vs<bf16, 16, 1>(a, s) : launch_vs<bf16, 64, 4>(a, s);
    else narrow ? launch_vs<float, 16, 1>(a, s) : launch_vs<float, 64, 4>(a, s);
    return launched();
}

} // namespace delta
} // namespace cawn
