// Gated delta rule by chunks: the recurrence over chunks, forward and (with other operands) backward.
//
//     X   = X0 + W S                  (64 x 16 a wave)
//     S'  = e^{G_C} S + K^T (c o X) (+ Y)
// Forward X is u: X0 = T beta V, W = -T beta e^G K, c = e^{G_C - G} / |k|.  Backward X is the gradient of beta (v - ...), S the state's.
//
// A wave owns 16 columns of the state, all rows of them, in registers in result layout; that is also the operand layout of the next
// product, so a chunk costs two products and two splittings into planes and no exchange between waves.  The four waves of a workgroup
// share W and K^T, which come as ready operands, straight into LDS, a chunk ahead.  The chunks of a row are a chain: what bounds this
// kernel is the chain's length times the latency of one link.
#include "cawn_delta_mfma.hpp"

namespace cawn {
namespace delta {

// NK: planes of K^T.  NBUF 2: the next chunk's operands arrive during this one's products; 1: where two sets would not fit the LDS.
template <int NK, int KP, int NBUF, bool REV> __global__ __launch_bounds__(256) void delta_states(const StateArgs a)
{
    constexpr int KS = KP / 32, KT = KP / 16, WF = 4 * KS * 3, KF = KT * 2 * NK, PIECES = WF + KF;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int vgroups = (a.VT + 3) / 4, blk = blockIdx.x, vg = blk % vgroups, bh = blk / vgroups, b = bh / a.H;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, c = lane % 16, g = lane / 16, vt = 4 * vg + w;
    const bool mine = vt < a.VT;
    const int len = a.lengths ? min(max(a.lengths[b], 0), a.L) : a.L, nb = (len + CHUNK - 1) / CHUNK;
    const int n0 = a.c0, n1 = min(a.c1, nb), count = n1 - n0;
    char *carry = a.carry + ((size_t)bh * KT * a.VT + vt) * 1024 + lane * 16;        // + kt VT KiB
    f32x4 S[KT];
    const int v = 16 * vt + c;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        S[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (!mine) continue;
        if (!a.first) S[t] = *reinterpret_cast<const f32x4 *>(carry + (size_t)t * a.VT * 1024);
        else if (a.begin && v < a.V) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int f = 16 * t + 4 * g + r;
                if (f < a.K) S[t][r] = a.begin[((long long)bh * a.K + f) * a.V + v];
            }
        }
    }
    const char *slots = a.ws + (size_t)bh * a.span * a.slot;
    auto fetch = [&](int n, int buf) {
        const char *src = slots + (size_t)(n - a.c0) * a.slot + lane * 16;
        char *dst = lds + buf * PIECES * 1024;
#pragma unroll
        for (int u = 0; u < (PIECES + 3) / 4; ++u) {
            const int i = 4 * u + w;
            if (i >= PIECES) break;
#if defined(__HIP_DEVICE_COMPILE__)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(src + (size_t)i * 1024), (__attribute__((address_space(3))) void *)(dst + i * 1024), 16, 0, 0);
#else
            (void)src, (void)dst;
#endif
        }
    };
    f32x4 x0[4], cf[4], y[REV ? KT : 1];
    float e = 0.f;
    auto rows_of = [&](int n) {
        const char *p = slots + (size_t)(n - a.c0) * a.slot;
        const Gates *G = reinterpret_cast<const Gates *>(p + a.gates_at);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (mine) x0[r] = *reinterpret_cast<const f32x4 *>(p + a.x_at + ((size_t)r * a.VT + vt) * 1024 + lane * 16);
            cf[r] = *reinterpret_cast<const f32x4 *>(G->c + 16 * r + 4 * g);
        }
        if (REV) {
#pragma unroll
            for (int t = 0; t < KT; ++t)
                if (mine) y[t] = *reinterpret_cast<const f32x4 *>(p + a.y_at + ((size_t)t * a.VT + vt) * 1024 + lane * 16);
        }
        e = G->eg[CHUNK - 1];
    };
    if (count > 0) {
        const int first = REV ? n1 - 1 : n0;
        if (NBUF == 2) fetch(first, 0);
        rows_of(first);
    }
    for (int it = 0; it < count; ++it) {
        const int n = REV ? n1 - 1 - it : n0 + it;
        if (NBUF == 1) {
            __syncthreads();
            fetch(n, 0);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();                        // everyone's pieces are there, and nobody reads the other buffer any more
        const int next = REV ? n - 1 : n + 1;
        if (NBUF == 2 && it + 1 < count) fetch(next, (it + 1) & 1);
        const bf16x8 *op = reinterpret_cast<const bf16x8 *>(lds + (NBUF == 2 ? it & 1 : 0) * PIECES * 1024) + lane;
        if (mine) {
            char *st = a.s_tiles + (size_t)bh * a.s_row + (size_t)(n - a.s_first) * a.s_chunk + (size_t)vt * 1024 + lane * 16;
#pragma unroll
            for (int t = 0; t < KT; ++t) *reinterpret_cast<f32x4 *>(st + (size_t)t * a.VT * 1024) = S[t];
        }
        f32x4 X[4], cn[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) X[r] = x0[r], cn[r] = cf[r];
        const float en = e;
        Frag<3> sf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) split_tiles<3>(S[2 * ks], S[2 * ks + 1], sf[ks]);
#pragma unroll
        for (int t = 0; t < KT; ++t) {
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = en * S[t][r] + (REV ? y[t][r] : 0.f);
        }
        if (it + 1 < count) rows_of(next);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                Frag<3> f;
#pragma unroll
                for (int p = 0; p < 3; ++p) f.p[p] = op[((r * KS + ks) * 3 + p) * 64];
                X[r] = mma<3>(f, sf[ks], X[r]);
            }
        if (mine) {
            char *xt = a.x_tiles + (size_t)bh * a.x_row + (size_t)(n - a.x_first) * a.x_chunk + (size_t)vt * 1024 + lane * 16;
#pragma unroll
            for (int r = 0; r < 4; ++r) *reinterpret_cast<f32x4 *>(xt + (size_t)r * a.VT * 1024) = X[r];
        }
        Frag<3> xf[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) split_tiles<3>(X[2 * ks] * cn[2 * ks], X[2 * ks + 1] * cn[2 * ks + 1], xf[ks]);
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                Frag<NK> f;
#pragma unroll
                for (int p = 0; p < NK; ++p) f.p[p] = op[(WF + (t * 2 + ks) * NK + p) * 64];
                S[t] = mma<3>(f, xf[ks], S[t]);
            }
    }
    if (!mine) return;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        *reinterpret_cast<f32x4 *>(carry + (size_t)t * a.VT * 1024) = S[t];
        if (a.keep_end && count > 0)
            *reinterpret_cast<f32x4 *>(a.s_tiles + (size_t)bh * a.s_row + (size_t)(n1 - a.s_first) * a.s_chunk + ((size_t)t * a.VT + vt) * 1024 + lane * 16) = S[t];
        if (a.last && a.end && v < a.V) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int f = 16 * t + 4 * g + r;
                if (f < a.K) a.end[((long long)bh * a.K + f) * a.V + v] = S[t][r];
            }
        }
    }
}

template <int NK, int KP, int NBUF> static int launch_kp(const StateArgs &a, bool reverse, hipStream_t s)
{
    constexpr int bytes = NBUF * (4 * (KP / 32) * 3 + (KP / 16) * 2 * NK) * 1024;
    const void *fn = reverse ? (const void *)delta_states<NK, KP, NBUF, true> : (const void *)delta_states<NK, KP, NBUF, false>;
    if (bytes > 65536 && hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return CAWN_ELAUNCH;
    const dim3 grid((unsigned)((long long)a.B * a.H * ((a.VT + 3) / 4)));
    if (reverse) hipLaunchKernelGGL((delta_states<NK, KP, NBUF, true>), grid, dim3(256), bytes, s, a);
    else hipLaunchKernelGGL((delta_states<NK, KP, NBUF, false>), grid, dim3(256), bytes, s, a);
    return launched();
}

int launch_states(const StateArgs &a, bool bf16_, bool reverse, hipStream_t s)
{
    if (a.K <= 32) return bf16_ ? launch_kp<1, 32, 2>(a, reverse, s) : launch_kp<3, 32, 2>(a, reverse, s);
    if (a.K <= 64) return bf16_ ? launch_kp<1, 64, 2>(a, reverse, s) : launch_kp<3, 64, 2>(a, reverse, s);
    return bf16_ ? launch_kp<1, 128, 2>(a, reverse, s) : launch_kp<3, 128, 1>(a, reverse, s);
}

} // namespace delta
} // namespace cawn
