// Gated delta rule by chunks, forward: what a chunk contributes by itself (ahead of the recurrence over chunks), and the output
// (behind it).  Every chunk of every head is a workgroup of its own in both.
#include <stddef.h>

#include "cawn_delta_mfma.hpp"

namespace cawn {
namespace delta {

// W = -T beta e^G K (negated: the recurrence adds), K^T and T beta V as operands and tiles of delta_states, gates.
// Wave w makes row tile w of W and of T beta V; of T it needs the steps up to its own rows only.
template <typename T, int NP, int KP> __global__ __launch_bounds__(256) void delta_prepare(const Args a)
{
    constexpr int KS = KP / 32, KT = KP / 16;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ Gates G;
    const int blk = blockIdx.x, n = a.c0 + blk % (a.c1 - a.c0), bh = blk / (a.c1 - a.c0), h = bh % a.H, b = bh / a.H;
    const int len = row_length(a, b), t0 = n * CHUNK, rows = min(CHUNK, len - t0);
    if (rows <= 0) return;
    const Sizes z(a.K, a.V, NP);
    char *slot = a.ws + ((size_t)bh * a.span + (n - a.c0)) * z.slot;
    const Tile<NP, CHUNK, KP> k{(bf16 *)lds};
    const Tile<NP, CHUNK, 64> v{(bf16 *)(lds + Tile<NP, CHUNK, KP>::BYTES)};
    float *M = (float *)(lds + Tile<NP, CHUNK, KP>::BYTES + Tile<NP, CHUNK, 64>::BYTES);
    const int w = threadIdx.x / 64, lane = threadIdx.x % 64, g = lane / 16, c = lane % 16;
    const T *vp = (const T *)a.v + b * a.vsb + t0 * a.vst + (long long)h * a.V;
    stage_rows<T, NP, KP>(k, (const T *)a.k + b * a.qsb + t0 * a.qst + (long long)(h / (a.H / a.Hk)) * a.K, a.qst, rows, a.K, a.vecq, G.rk, a.norm, a.eps);
    stage_rows<T, NP, 64>(v, vp, a.vst, rows, min(64, a.V), a.vecv, nullptr, false, 0.f);
    load_gates(a, G, b, h, t0, rows);
    __syncthreads();
    if (threadIdx.x < CHUNK) G.c[threadIdx.x] = G.ed[threadIdx.x] * G.rk[threadIdx.x];
    system_of<NP, KP>(k, G, M);
    __syncthreads();
    {
        float *out = (float *)(slot + (size_t)(z.wf + z.kf + z.ut) * 1024);
        for (int i = threadIdx.x; i < (int)(sizeof(Gates) / 4); i += 256) out[i] = ((const float *)&G)[i];
        bf16x8 *kt = reinterpret_cast<bf16x8 *>(slot + (size_t)z.wf * 1024) + lane;
        for (int u = w; u < KT * 2; u += 4) {
            const Frag<NP> f = k.tiled_down(32 * (u % 2), 16 * (u / 2), lane);
#pragma unroll
            for (int p = 0; p < NP; ++p) kt[(u * NP + p) * 64] = f.p[p];
        }
    }
    invert(M);
    // row tile w of T, columns scaled for either product
    Frag<3> tw[2], tv[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        float xw[8], xv[8];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int j0 = 32 * ks + 16 * half + 4 * g;
            const f32x4 t = *reinterpret_cast<const f32x4 *>(M + (16 * w + c) * TLD + j0);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                xv[4 * half + r] = t[r] * G.beta[j0 + r];
                xw[4 * half + r] = -(xv[4 * half + r] * G.rk[j0 + r] * G.eg[j0 + r]);
            }
        }
        split8<3>(xw, tw[ks]);
        split8<3>(xv, tv[ks]);
    }
    // W^T tile by tile: its result layout is the operand that delta_states reads
    bf16x8 *wf = reinterpret_cast<bf16x8 *>(slot) + lane;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        f32x4 acc[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            acc[half] = f32x4{0.f, 0.f, 0.f, 0.f};
            acc[half] = mma<3>(k.tiled_down(0, 32 * ks + 16 * half, lane), tw[0], acc[half]);
            if (w >= 2) acc[half] = mma<3>(k.tiled_down(32, 32 * ks + 16 * half, lane), tw[1], acc[half]);
        }
        Frag<3> f;
        split_tiles<3>(acc[0], acc[1], f);
#pragma unroll
        for (int p = 0; p < 3; ++p) wf[((w * KS + ks) * 3 + p) * 64] = f.p[p];
    }
    char *ub = slot + (size_t)(z.wf + z.kf) * 1024 + lane * 16;
    for (int v0 = 0; v0 < a.V; v0 += 64) {
        if (v0 > 0) {
            __syncthreads();
            stage_rows<T, NP, 64>(v, vp + v0, a.vst, rows, min(64, a.V - v0), a.vecv, nullptr, false, 0.f);
            __syncthreads();
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (v0 + 16 * q >= a.V) break;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            acc = mma<3>(tv[0], v.tiled_down(0, 16 * q, lane), acc);
            if (w >= 2) acc = mma<3>(tv[1], v.tiled_down(32, 16 * q, lane), acc);
            *reinterpret_cast<f32x4 *>(ub + ((size_t)w * a.VT + v0 / 16 + q) * 1024) = acc;
        }
    }
}

// O^T = scale / |q| (e^G S0^T Q^T + U^T P^T): wave w makes row tile w of P, for all, and then columns 16 w, 16 (w + 4), ... of O.
// A bf16 output takes two planes of S0, U and P (its own rounding is 2^-9; theirs stays below 2^-16).
template <typename T, int NP, int KP> __global__ __launch_bounds__(256) void delta_output(const Args a)
{
    constexpr int KS = KP / 32, KT = KP / 16, PO = NP == 1 ? 2 : 3;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ Gates G;
    const int blk = blockIdx.x, n = a.c0 + blk % (a.c1 - a.c0), bh = blk / (a.c1 - a.c0), h = bh % a.H, b = bh / a.H;
    const int len = row_length(a, b), t0 = n * CHUNK, rows = min(CHUNK, len - t0), all = min(CHUNK, a.L - t0);
    T *op = (T *)a.o + b * a.osb + t0 * a.ost + (long long)h * a.V;
    if (rows <= 0) {
        for (int i = threadIdx.x; i < all * a.V; i += 256) op[(long long)(i / a.V) * a.ost + i % a.V] = (T)0.f;
        return;
    }
    const Sizes z(a.K, a.V, NP);
    const char *slot = a.ws + ((size_t)bh * a.span + (n - a.c0)) * z.slot;
    const Tile<NP, CHUNK, KP> q{(bf16 *)lds}, k{(bf16 *)(lds + Tile<NP, CHUNK, KP>::BYTES)};
    bf16x8 *pf = reinterpret_cast<bf16x8 *>(lds + 2 * Tile<NP, CHUNK, KP>::BYTES);
    const int w = threadIdx.x / 64, lane = threadIdx.x % 64, g = lane / 16, c = lane % 16;
    {
        const float *in = (const float *)(slot + (size_t)(z.wf + z.kf + z.ut) * 1024);
        for (int i = threadIdx.x; i < (int)(sizeof(Gates) / 4); i += 256)
            if (i < (int)(offsetof(Gates, rq) / 4)) ((float *)&G)[i] = in[i];       // (rq: stage_rows, below)
    }
    const long long qat = b * a.qsb + t0 * a.qst + (long long)(h / (a.H / a.Hk)) * a.K;
    stage_rows<T, NP, KP>(q, (const T *)a.q + qat, a.qst, rows, a.K, a.vecq, G.rq, a.norm, a.eps);
    stage_rows<T, NP, KP>(k, (const T *)a.k + qat, a.qst, rows, a.K, a.vecq, nullptr, false, 0.f);
    __syncthreads();
    {
        f32x4 p[4];
#pragma unroll
        for (int jt = 0; jt < 4; ++jt) {
            p[jt] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (jt <= w) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) p[jt] = mma<3>(k.straight(16 * jt, 32 * ks, lane), q.straight(16 * w, 32 * ks, lane), p[jt]);
                const int i = 16 * w + c;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 16 * jt + 4 * g + r;
                    p[jt][r] = i >= j ? p[jt][r] * (G.rk[j] * decay_between(G, i, j)) : 0.f;
                }
            }
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            Frag<PO> f;
            split_tiles<PO>(p[2 * ks], p[2 * ks + 1], f);
#pragma unroll
            for (int e = 0; e < PO; ++e) pf[((w * 2 + ks) * PO + e) * 64 + lane] = f.p[e];
        }
    }
    __syncthreads();
    const char *s0 = a.s_tiles + bh * a.s_row + (n - a.s_first) * a.s_chunk + lane * 16, *u0 = a.u_tiles + bh * a.u_row + (n - a.u_first) * a.u_chunk + lane * 16;
    for (int vt = w; vt < a.VT; vt += 4) {
        Frag<PO> sf[KS], uf[2];
        {
            f32x4 S[KT], U[4];
#pragma unroll
            for (int t = 0; t < KT; ++t) S[t] = *reinterpret_cast<const f32x4 *>(s0 + ((size_t)t * a.VT + vt) * 1024);
#pragma unroll
            for (int r = 0; r < 4; ++r) U[r] = *reinterpret_cast<const f32x4 *>(u0 + ((size_t)r * a.VT + vt) * 1024);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) split_tiles<PO>(S[2 * ks], S[2 * ks + 1], sf[ks]);
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) split_tiles<PO>(U[2 * ks], U[2 * ks + 1], uf[ks]);
        }
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) acc = mma<PO>(sf[ks], q.tiled(16 * it, 32 * ks, lane), acc);
            const int i = 16 * it + c;
            acc *= G.eg[i];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                if (2 * ks > it) break;
                Frag<PO> f;
#pragma unroll
                for (int e = 0; e < PO; ++e) f.p[e] = pf[((it * 2 + ks) * PO + e) * 64 + lane];
                acc = mma<PO>(uf[ks], f, acc);
            }
            if (i >= all) continue;
            const float m = a.scale * G.rq[i];
            float x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = i < rows ? acc[r] * m : 0.f;
            T *dst = op + (long long)i * a.ost + 16 * vt + 4 * g;
            if (a.veco && 16 * vt + 4 * g + 4 <= a.V) store_n<T, 4>(dst, x);
            else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (16 * vt + 4 * g + r < a.V) dst[r] = (T)x[r];
            }
        }
    }
}

template <typename T, int NP, int KP> static int prepare_kp(const Args &a, hipStream_t s)
{
    constexpr int bytes = Tile<NP, CHUNK, KP>::BYTES + Tile<NP, CHUNK, 64>::BYTES + CHUNK * TLD * 4;
    if (bytes > 65536 - (int)sizeof(Gates) &&
        hipFuncSetAttribute((const void *)delta_prepare<T, NP, KP>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return CAWN_ELAUNCH;
    hipLaunchKernelGGL((delta_prepare<T, NP, KP>), dim3((unsigned)((long long)a.B * a.H * (a.c1 - a.c0))), dim3(256), bytes, s, a);
    return launched();
}

template <typename T, int NP, int KP> static int output_kp(const Args &a, hipStream_t s)
{
    constexpr int bytes = 2 * Tile<NP, CHUNK, KP>::BYTES + 8 * (NP == 1 ? 2 : 3) * 1024;
    if (bytes > 65536 - (int)sizeof(Gates) &&
        hipFuncSetAttribute((const void *)delta_output<T, NP, KP>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return CAWN_ELAUNCH;
    hipLaunchKernelGGL((delta_output<T, NP, KP>), dim3((unsigned)((long long)a.B * a.H * (a.c1 - a.c0))), dim3(256), bytes, s, a);
    return launched();
}

int launch_prepare(const Args &a, bool bf16_, hipStream_t s)
{
    if (a.K <= 32) return bf16_ ? prepare_kp<bf16, 1, 32>(a, s) : prepare_kp<float, 3, 32>(a, s);
    if (a.K <= 64) return bf16_ ? prepare_kp<bf16, 1, 64>(a, s) : prepare_kp<float, 3, 64>(a, s);
    return bf16_ ? prepare_kp<bf16, 1, 128>(a, s) : prepare_kp<float, 3, 128>(a, s);
}

int launch_output(const Args &a, bool bf16_, hipStream_t s)
{
    if (a.K <= 32) return bf16_ ? output_kp<bf16, 1, 32>(a, s) : output_kp<float, 3, 32>(a, s);
    if (a.K <= 64) return bf16_ ? output_kp<bf16, 1, 64>(a, s) : output_kp<float, 3, 64>(a, s);
    return bf16_ ? output_kp<bf16, 1, 128>(a, s) : output_kp<float, 3, 128>(a, s);
}

} // namespace delta
} // namespace cawn
