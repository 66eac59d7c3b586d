// Gated delta rule by chunks: the states at the segments' begins (forward, S' = A S + b) or, for the gradient, behind their ends
// (S' = A^T S + b, from the last segment to the first).
//
// A workgroup takes 64 columns of a head's state.  Wave w owns the rows of row tiles w, w + 4 of them; it splits its own rows of A and
// its own tiles of the new state, and the waves pass each other the state's planes in LDS: one barrier a segment.
#include "cawn_delta_mfma.hpp"

namespace cawn {
namespace delta {

template <int KP, bool REV> __global__ __launch_bounds__(256) void delta_join(const Args a)
{
    constexpr int KS = KP / 32, KT = KP / 16, OWN = (KT + 3) / 4;
    extern __shared__ __attribute__((aligned(16))) char lds[];      // [2][4 column tiles][KS][3] pieces
    const int groups = (a.VT + 3) / 4, bh = blockIdx.x / groups, vg = blockIdx.x % groups;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, g = lane / 16, c = lane % 16;
    const size_t st = (size_t)KT * a.VT * 1024;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const float *begin = REV ? a.dstate_out : a.state_in;
    f32x4 S[OWN][4];
    auto put = [&](int buf) {
#pragma unroll
        for (int o = 0; o < OWN; ++o) {
            const int t = w + 4 * o;
            if (t >= KT) break;
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) {
                float r[4] = {S[o][ct][0], S[o][ct][1], S[o][ct][2], S[o][ct][3]};
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    bf16x4 h;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        h[e] = (bf16)r[e];
                        r[e] -= (float)h[e];
                    }
                    *reinterpret_cast<bf16x4 *>(lds + ((((buf * 4 + ct) * KS + t / 2) * 3 + p) * 64 + lane) * 16 + (t % 2) * 8) = h;
                }
            }
        }
    };
    const int links = a.segments - 1;
    auto seg_of = [&](int i) { return REV ? a.segments - 1 - i : i; };      // the i-th link runs over this segment
#pragma unroll
    for (int o = 0; o < OWN; ++o)
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) {
            S[o][ct] = zero;
            const int t = w + 4 * o, v = 16 * (4 * vg + ct) + c;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int f = 16 * t + 4 * g + r;
                if (begin && f < a.K && v < a.V) S[o][ct][r] = begin[((long long)bh * a.K + f) * a.V + v];
            }
        }
    put(0);
    for (int i = 0; i < links; ++i) {
        const int s = seg_of(i);
        const float *A = (const float *)a.seg_a + ((size_t)bh * a.segments + s) * KP * KP;
        const char *bt = a.seg_b + ((size_t)bh * a.segments + s) * st + lane * 16;
        char *to = a.seg_s + ((size_t)bh * a.segments + (REV ? s - 1 : s + 1)) * st + lane * 16;
        Frag<3> af[OWN][KS];
#pragma unroll
        for (int o = 0; o < OWN; ++o) {
            const int t = w + 4 * o;
            if (t >= KT) break;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int step = 32 * ks + 16 * (e / 4) + 4 * g + e % 4, row = 16 * t + c;
                    x[e] = REV ? A[step * KP + row] : A[row * KP + step];
                }
                split8<3>(x, af[o][ks]);
            }
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) {
                const int vt = 4 * vg + ct;
                S[o][ct] = vt < a.VT ? *reinterpret_cast<const f32x4 *>(bt + ((size_t)t * a.VT + vt) * 1024) : zero;
            }
        }
        __syncthreads();
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                Frag<3> f;
#pragma unroll
                for (int p = 0; p < 3; ++p) f.p[p] = *reinterpret_cast<const bf16x8 *>(lds + (((((i & 1) * 4 + ct) * KS + ks) * 3 + p) * 64 + lane) * 16);
#pragma unroll
                for (int o = 0; o < OWN; ++o)
                    if (w + 4 * o < KT) S[o][ct] = mma<3>(af[o][ks], f, S[o][ct]);
            }
#pragma unroll
        for (int o = 0; o < OWN; ++o)
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) {
                const int t = w + 4 * o, vt = 4 * vg + ct;
                if (t < KT && vt < a.VT) *reinterpret_cast<f32x4 *>(to + ((size_t)t * a.VT + vt) * 1024) = S[o][ct];
            }
        if (i + 1 < links) put((i + 1) & 1);
    }
}

template <int KP> static int join_kp(const Args &a, bool reverse, hipStream_t s)
{
    constexpr int bytes = 2 * 4 * (KP / 32) * 3 * 1024;
    const void *fn = reverse ? (const void *)delta_join<KP, true> : (const void *)delta_join<KP, false>;
    if (bytes > 60000 && hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return CAWN_ELAUNCH;
    const dim3 grid((unsigned)((long long)a.B * a.H * ceil_div(a.VT, 4)));
    if (reverse) hipLaunchKernelGGL((delta_join<KP, true>), grid, dim3(256), bytes, s, a);
    else hipLaunchKernelGGL((delta_join<KP, false>), grid, dim3(256), bytes, s, a);
    return launched();
}

int launch_join(const Args &a, bool reverse, hipStream_t s)
{
    return a.K <= 32 ? join_kp<32>(a, reverse, s) : a.K <= 64 ? join_kp<64>(a, reverse, s) : join_kp<128>(a, reverse, s);
}

} // namespace delta
} // namespace cawn
