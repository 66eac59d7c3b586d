// Gated delta rule by chunks: the states at the segments' begins (forward, S' = A S + b) or, for the gradient, behind their ends
// (S' = A^T S + b, from the last segment to the first).  The first of the chain, which is the caller's, is written down with the others: the pass
// over the segments takes all of them from here, because the workgroup that stores the caller's other end does not wait for the one
// that begins with this, and both may be one buffer.  A segment that the row does not reach is no link: the state passes it unchanged.
//
// A workgroup takes 16 columns of a head's state: the segments are a chain, and what counts is the time of one link.  Wave w owns row
// tiles w and w + 4; it splits its own rows of A (fetched a link ahead) and its own tiles of the new state, and the waves pass each other
// the state's planes in LDS: one barrier a link.  A link takes 1.0 to 1.2 us (4,096 tokens of 12 heads of 64 in fp32, 21 links: 22 us; 4 x 2,048 in bf16, 15
// links: 18 us), eight where it moves 13 MB (2 x 32,768 tokens of 32 heads of 128, 3 links: 25 us): the chain split, LDS, six products, sum.  Rows of A fetched two or four links ahead made the
// first call 2 us slower.
#include "cawn_delta_mfma.hpp"

namespace cawn {
namespace delta {

template <int KP, bool REV> __global__ __launch_bounds__(256) void delta_join(const Args a)
{
    constexpr int KS = KP / 32, KT = KP / 16, OWN = (KT + 3) / 4;
    __shared__ __attribute__((aligned(16))) char lds[2 * KS * 3 * 1024];
    const int bh = blockIdx.x / a.VT, vt = blockIdx.x % a.VT;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, g = lane / 16, c = lane % 16;
    const size_t st = (size_t)KT * a.VT * 1024;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const float *begin = REV ? a.dstate_out : a.state_in;
    // links first .. last - 1 belong to segments that hold chunks of the row
    const int links = a.segments - 1, live = ((row_length(a, bh / a.H) + CHUNK - 1) / CHUNK + a.seg_chunks - 1) / a.seg_chunks;
    const int first = REV ? min(a.segments - live, links) : 0, last = REV ? links : min(live, links);
    f32x4 S[OWN], bn[OWN];
    float an[OWN][KS][8];
    auto put = [&](int buf) {
#pragma unroll
        for (int o = 0; o < OWN; ++o) {
            const int t = w + 4 * o;
            if (t >= KT) break;
            bf16x4 h[3];
            split4<3>(S[o], h);
#pragma unroll
            for (int p = 0; p < 3; ++p) *reinterpret_cast<bf16x4 *>(lds + (((buf * KS + t / 2) * 3 + p) * 64 + lane) * 16 + (t % 2) * 8) = h[p];
        }
    };
    auto fetch = [&](int i) {                   // of the i-th link
        const int s = REV ? a.segments - 1 - i : i;
        const float *A = (const float *)a.seg_a + ((size_t)bh * a.segments + s) * KP * KP;
#pragma unroll
        for (int o = 0; o < OWN; ++o) {
            const int t = min(w + 4 * o, KT - 1), row = 16 * t + c;
            bn[o] = *reinterpret_cast<const f32x4 *>(a.seg_b + ((size_t)bh * a.segments + s) * st + ((size_t)t * a.VT + vt) * 1024 + lane * 16);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int step = 32 * ks + 16 * half + 4 * g;
                    if (REV) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) an[o][ks][4 * half + e] = A[(step + e) * KP + row];
                    } else {
                        const f32x4 x = *reinterpret_cast<const f32x4 *>(A + row * KP + step);
#pragma unroll
                        for (int e = 0; e < 4; ++e) an[o][ks][4 * half + e] = x[e];
                    }
                }
        }
    };
    auto leave = [&](int s) {                   // the state as segment s finds it
        char *to = a.seg_s + ((size_t)bh * a.segments + s) * st + ((size_t)w * a.VT + vt) * 1024 + lane * 16;
#pragma unroll
        for (int o = 0; o < OWN; ++o)
            if (w + 4 * o < KT) *reinterpret_cast<f32x4 *>(to + (size_t)(4 * o) * a.VT * 1024) = S[o];
    };
    if (first < last) fetch(first);
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        S[o] = zero;
        const int t = w + 4 * o, v = 16 * vt + c;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int f = 16 * t + 4 * g + r;
            if (begin && f < a.K && v < a.V) S[o][r] = begin[((long long)bh * a.K + f) * a.V + v];
        }
    }
    leave(REV ? links : 0);
    for (int i = 0; i < first; ++i) leave(links - 1 - i);
    put(first & 1);
    for (int i = first; i < last; ++i) {
        Frag<3> af[OWN][KS];
        f32x4 acc[OWN][KS];
#pragma unroll
        for (int o = 0; o < OWN; ++o)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                split8<3>(an[o][ks], af[o][ks]);
                acc[o][ks] = ks == 0 ? bn[o] : zero;
            }
        if (i + 1 < last) fetch(i + 1);
        __syncthreads();
        Frag<3> f[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int p = 0; p < 3; ++p) f[ks].p[p] = *reinterpret_cast<const bf16x8 *>(lds + ((((i & 1) * KS + ks) * 3 + p) * 64 + lane) * 16);
        // a chain of instructions for every 32 rows of the state, side by side
#pragma unroll
        for (int q = 2; q >= 0; --q)
#pragma unroll
            for (int p = 0; p <= q; ++p)
#pragma unroll
                for (int o = 0; o < OWN; ++o)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) acc[o][ks] = mfma(af[o][ks].p[p], f[ks].p[q - p], acc[o][ks]);
#pragma unroll
        for (int o = 0; o < OWN; ++o) {
            S[o] = acc[o][0];
#pragma unroll
            for (int ks = 1; ks < KS; ++ks) S[o] += acc[o][ks];
        }
        leave(REV ? links - 1 - i : i + 1);
        if (i + 1 < last) put((i + 1) & 1);
    }
    for (int i = last; i < links; ++i) leave(i + 1);
}

template <int KP> static int join_kp(const Args &a, bool reverse, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)a.B * a.H * a.VT));
    if (reverse) hipLaunchKernelGGL((delta_join<KP, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((delta_join<KP, false>), grid, dim3(256), 0, s, a);
    return launched();
}

int launch_join(const Args &a, bool reverse, hipStream_t s)
{
    return a.K <= 32 ? join_kp<32>(a, reverse, s) : a.K <= 64 ? join_kp<64>(a, reverse, s) : join_kp<128>(a, reverse, s);
}

} // namespace delta
} // namespace cawn
