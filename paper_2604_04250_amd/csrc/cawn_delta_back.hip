// Gated delta rule by chunks, backward: the recurrence from the last chunk to the first, in segments like the forward.
//
// With dS the gradient of the state behind a chunk, dO that of its output, KD = diag(e^{G_C - G}) K:
//     dR  = T^T (scale P^T dO + KD dS)            the gradient of U through everything but T; dV = beta dR
//     dS0 = e^{G_C} dS + scale (e^G Q)^T dO - (beta e^G K)^T dR
// dS0 is A^T dS plus what the segment's own dO add, A the forward's: MODE 1 finds the latter from dS = 0 (all segments but the first at
// once), delta_join the gradients behind the segments' ends, MODE 0 runs through all segments and leaves dR and dS of every chunk to
// delta_gradients.  Waves, columns and operands as in the forward; P^T takes three planes, because dR carries fp32 gradients.
//
// Measured: 8 x 8,192 tokens of 12 heads of 64 in bf16: MODE 1 181 us, MODE 0 213 (1.0 GB), bound by instruction issue like the forward.
#include "cawn_delta_mfma.hpp"

namespace cawn {
namespace delta {

// P^T's operands and then T in one place: room for three workgroups a CU, which wait for T less than two do that have it early (8 x 8,192
// tokens of 12 heads of 64 in bf16: 221 and 190 us for the two passes, 281 and 245 with a place for each).
template <int NP, int KP, int NW> struct BackLds {
    static constexpr int KB = Tile<NP, CHUNK, KP>::BYTES, TO = 2 * KB, BYTES = TO + T_BYTES;       // k, q; P^T's operands, and then T
    static constexpr int HELD = 163840 / (BYTES + (int)sizeof(Gates)) * NW / 4, WAVES = HELD > 3 ? 3 : HELD;
};

template <typename T, int NP, int KP, int MODE, int NW> __global__ __launch_bounds__((64 * NW), (BackLds<NP, KP, NW>::WAVES)) void delta_back(const Args a)
{
    using L = BackLds<NP, KP, NW>;
    constexpr int KS = KP / 32, KT = KP / 16, NT = 64 * NW;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ Gates G;
    const Tile<NP, CHUNK, KP> k{(bf16 *)lds}, q{(bf16 *)(lds + L::KB)};
    const char *tl = lds + L::TO;
    bf16x8 *pf = reinterpret_cast<bf16x8 *>(lds + L::TO);
    const int rows_all = a.B * a.H, blk = blockIdx.x, bh = blk % rows_all, nseg = MODE == 0 ? a.segments : a.segments - 1;
    const int seg = blk / rows_all % nseg + (MODE == 0 ? 0 : 1), group = blk / rows_all / nseg, b = bh / a.H, h = bh % a.H;
    const int len = row_length(a, b), nb = (len + CHUNK - 1) / CHUNK;
    const int n0 = min(seg * a.seg_chunks, nb), n1 = min(n0 + a.seg_chunks, nb);
    if (MODE == 1 && n0 == n1) return;          // (as in delta_scan)
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    int tid = threadIdx.x, lane = tid % 64, g = lane / 16, c = lane % 16;
    const int ct = group * NW + w;
    const bool mine = ct < a.VT;
    int v = 16 * ct + c;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    f32x4 S[KT];                                // dS
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        S[t] = zero;
        if (MODE == 1 || !mine) continue;
        if (a.segments > 1) S[t] = *reinterpret_cast<const f32x4 *>(a.seg_s + (((size_t)bh * a.segments + seg) * KT * a.VT + (size_t)t * a.VT + ct) * 1024 + lane * 16);
        else if (a.dstate_out && v < a.V) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * t + 4 * g + r < a.K) S[t][r] = a.dstate_out[((long long)bh * a.K + 16 * t + 4 * g + r) * a.V + v];
        }
    }
    long long qst = a.qst, ost = a.ost;
    uint32_t l16 = 16 * lane;
    auto anew = [&]() {                         // (as in delta_scan)
        tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        lane = tid % 64, g = lane / 16, c = lane % 16, v = 16 * ct + c, l16 = 16 * lane;
    };
    RowsAhead<T, NP, KP, NT> ka, qa;
    constexpr int GN = (GATE_FLOATS + NT - 1) / NT;
    float ga[GN];
    auto ahead = [&](int n) {
        const int rows = min(CHUNK, len - n * CHUNK);
        const long long qat = b * a.qsb + (long long)n * CHUNK * qst + (long long)(h / (a.H / a.Hk)) * a.K;
        ka.load(tid, (const T *)a.k + qat, qst, rows, a.K, a.vecq);
        qa.load(tid, (const T *)a.q + qat, qst, rows, a.K, a.vecq);
        const float *gp = a.gates + ((long long)bh * a.chunks + n) * GATE_FLOATS;
#pragma unroll
        for (int e = 0; e < GN; ++e) ga[e] = gp[min(tid + e * NT, GATE_FLOATS - 1)];
    };
    auto keep = [&](int n) {                    // dS behind chunk n
        if (MODE == 1 || !mine) return;
        char *st = a.ds_tiles + ((size_t)bh * a.chunks + n) * KT * a.VT * 1024 + (size_t)ct * 1024;
#pragma unroll
        for (int t = 0; t < KT; ++t) *reinterpret_cast<f32x4 *>(st + (size_t)t * a.VT * 1024 + l16) = S[t];
    };
    if (n0 < n1) {
        ahead(n1 - 1);
        keep(n1 - 1);
    }
    for (int n = n1 - 1; n >= n0; --n) {
        const int rows = min(CHUNK, len - n * CHUNK);
        anew();
        asm volatile("" : "+s"(qst), "+s"(ost));
        if (n < n1 - 1) __syncthreads();
        ka.put_plain(tid, k, rows, a.K);
        qa.put_plain(tid, q, rows, a.K);
#pragma unroll
        for (int e = 0; e < GN; ++e)
            if (tid + e * NT < GATE_FLOATS) ((float *)&G)[tid + e * NT] = ga[e];
        __syncthreads();
        T da[4][4];
        if (mine) {
            const T *dp = (const T *)a.dO + b * a.osb + (long long)n * CHUNK * ost + (long long)h * a.V;
            if (rows == CHUNK && 16 * ct + 16 <= a.V && ost < (1 << 22)) {
                dp += 16 * ct;
                const uint32_t dlane = (4 * (uint32_t)g * (uint32_t)ost + c) * sizeof(T);
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) da[t][r] = *reinterpret_cast<const T *>((const char *)(dp + (16 * t + r) * ost) + dlane);
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) da[t][r] = dp[min(16 * t + 4 * g + r, rows - 1) * ost + min(v, a.V - 1)];
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * t + 4 * g + r >= rows || v >= a.V) da[t][r] = (T)0.f;
            }
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) da[t][r] = (T)0.f;
        }
        if (n > n0) ahead(n - 1);
        anew();
        // scale P, whose result layout is the operand of P^T, shared out: with four waves the first two take two operands, one of them small
        const int two = NW == 4 && w < 2, first = NW == 4 && w > 1 ? w + 1 : w;
        for (int u = 0; u < 1 + two; ++u) {
            const int id = first + u * (w == 0 ? 2 : 4);
            if (id > 5) break;
            anew();
            const int jt = id < 4 ? id / 2 : id - 2, is = id < 4 ? id % 2 : 1, j = 16 * jt + c;
            const float m = a.scale * G.rk[j];
            f32x4 p[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int it = 2 * is + half;
                p[half] = zero;
                if (it < jt) continue;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) p[half] = mma<3>(q.straight(16 * it, 32 * ks, lane), k.straight(16 * jt, 32 * ks, lane), p[half]);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * it + 4 * g + r;
                    p[half][r] = i >= j ? p[half][r] * (m * G.rq[i] * decay_between(G, i, j)) : 0.f;
                }
            }
            Frag<3> f;
            split_tiles<3>(p[0], p[1], f);
#pragma unroll
            for (int e = 0; e < 3; ++e) pf[(id * 3 + e) * 64 + lane] = f.p[e];
        }
        anew();
        f32x4 Z[4] = {zero, zero, zero, zero}, R[4] = {zero, zero, zero, zero};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            Frag<3> sf;
            Frag<NP> f[4];
            split_tiles<3>(S[2 * ks], S[2 * ks + 1], sf);
#pragma unroll
            for (int t = 0; t < 4; ++t) f[t] = k.tiled(16 * t, 32 * ks, lane);
            mma_each<3>(f, sf, Z);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) Z[t] *= *reinterpret_cast<const f32x4 *>(G.c + 16 * t + 4 * g);
        __syncthreads();                        // the operands of P^T
        anew();
        // both are upper triangular: row tiles 0 and 1 take both halves of the tokens, 2 and 3 the second
        {
            Frag<NP> df[2];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                if constexpr (sizeof(T) == 2) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) df[ks].p[0][e] = da[2 * ks + e / 4][e % 4];
                } else {
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = (float)da[2 * ks + e / 4][e % 4];
                    split8<NP>(y, df[ks]);
                }
            }
            Frag<3> f[4], f2[2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 3; ++e) f2[t].p[e] = pf[(upper(t, 0) * 3 + e) * 64 + lane];
            mma_each<3>(f2, df[0], Z);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 3; ++e) f[t].p[e] = pf[(upper(t, 1) * 3 + e) * 64 + lane];
            mma_each<3>(f, df[1], Z);
        }
        __syncthreads();                        // nobody reads them any more: T in their place
        anew();
        {
            const char *src = a.t_ops + ((size_t)bh * a.chunks + n) * T_BYTES;
#pragma unroll
            for (int u = 0; u < (T_BYTES / 1024 + NW - 1) / NW; ++u) {
                const int i = u * NW + w;
                if (i < T_BYTES / 1024) load_piece(src + (size_t)i * 1024 + l16, lds + L::TO + i * 1024);
            }
        }
        constexpr int AT = KT < 4 ? KT : 4;
        // meanwhile, the share of dO in the gradient of the state before the chunk
        {
            const float e = G.eg[CHUNK - 1];
#pragma unroll
            for (int t = 0; t < KT; ++t) S[t] *= e;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                Frag<3> of;
                f32x4 o[2];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int t = 2 * ks + half;
                    const f32x4 eg = *reinterpret_cast<const f32x4 *>(G.eg + 16 * t + 4 * g), rq = *reinterpret_cast<const f32x4 *>(G.rq + 16 * t + 4 * g);
#pragma unroll
                    for (int x = 0; x < 4; ++x) o[half][x] = (float)da[t][x] * (a.scale * eg[x] * rq[x]);
                }
                split_tiles<3>(o[0], o[1], of);
#pragma unroll
                for (int t0 = 0; t0 < KT; t0 += AT) {
                    Frag<NP> f[AT];
#pragma unroll
                    for (int t = 0; t < AT; ++t) f[t] = q.tiled_down(32 * ks, 16 * (t0 + t), lane);
                    mma_each<3>(f, of, S + t0);
                }
            }
        }
        Frag<3> zf[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) split_tiles<3>(Z[2 * ks], Z[2 * ks + 1], zf[ks]);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();                        // T
        anew();
        {
            Frag<3> f[4], f2[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) f2[t] = t_columns(tl, t, 0, lane);
            mma_each<3>(f2, zf[0], R);
#pragma unroll
            for (int t = 0; t < 4; ++t) f[t] = t_columns(tl, t, 1, lane);
            mma_each<3>(f, zf[1], R);
        }
        // (stores behind the wait for T, which would wait for them too)
        if (MODE == 0 && mine) {
            char *rt = a.dr_tiles + ((size_t)bh * a.chunks + n) * 4 * a.VT * 1024 + (size_t)ct * 1024;
#pragma unroll
            for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4 *>(rt + (size_t)t * a.VT * 1024 + l16) = R[t];
        }
        anew();
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            Frag<3> rf;
            f32x4 r[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) r[half] = -R[2 * ks + half] * *reinterpret_cast<const f32x4 *>(G.x + 16 * (2 * ks + half) + 4 * g);
            split_tiles<3>(r[0], r[1], rf);
#pragma unroll
            for (int t0 = 0; t0 < KT; t0 += AT) {
                Frag<NP> f[AT];
#pragma unroll
                for (int t = 0; t < AT; ++t) f[t] = k.tiled_down(32 * ks, 16 * (t0 + t), lane);
                mma_each<3>(f, rf, S + t0);
            }
        }
        if (n > n0) keep(n - 1);
    }
    if (!mine) return;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        if (MODE == 1) *reinterpret_cast<f32x4 *>(a.seg_b + (((size_t)bh * a.segments + seg) * KT * a.VT + (size_t)t * a.VT + ct) * 1024 + lane * 16) = S[t];
        else if (seg == 0 && a.dstate_in && v < a.V) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * t + 4 * g + r < a.K) a.dstate_in[((long long)bh * a.K + 16 * t + 4 * g + r) * a.V + v] = S[t][r];
        }
    }
}

template <typename T, int NP, int KP, int NW> static int back_nw(const Args &a, hipStream_t s)
{
    constexpr int bytes = BackLds<NP, KP, NW>::BYTES;
    static_assert(bytes + sizeof(Gates) <= 163840, "LDS");
    const long long wgs = (long long)a.B * a.H * ceil_div(a.VT, NW);
    if (bytes > 60000 && (hipFuncSetAttribute((const void *)delta_back<T, NP, KP, 0, NW>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess ||
                          hipFuncSetAttribute((const void *)delta_back<T, NP, KP, 1, NW>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess)) return CAWN_ELAUNCH;
    if (a.segments > 1) {
        hipLaunchKernelGGL((delta_back<T, NP, KP, 1, NW>), dim3((unsigned)(wgs * (a.segments - 1))), dim3(64 * NW), bytes, s, a);
        if (int r = launched()) return r;
        if (int r = launch_join(a, true, s)) return r;
    }
    hipLaunchKernelGGL((delta_back<T, NP, KP, 0, NW>), dim3((unsigned)(wgs * a.segments)), dim3(64 * NW), bytes, s, a);
    return launched();
}
template <typename T, int NP, int KP> static int back_kp(const Args &a, hipStream_t s)
{
    if constexpr (NP == 3 && KP == 128)         // (as in delta_scan)
        if (a.VT > 4) return back_nw<T, NP, KP, 8>(a, s);
    return back_nw<T, NP, KP, 4>(a, s);
}

int launch_back(const Args &a, bool bf16_, hipStream_t s)
{
    if (a.K <= 32) return bf16_ ? back_kp<bf16, 1, 32>(a, s) : back_kp<float, 3, 32>(a, s);
    if (a.K <= 64) return bf16_ ? back_kp<bf16, 1, 64>(a, s) : back_kp<float, 3, 64>(a, s);
    return bf16_ ? back_kp<bf16, 1, 128>(a, s) : back_kp<float, 3, 128>(a, s);
}

} // namespace delta
} // namespace cawn
