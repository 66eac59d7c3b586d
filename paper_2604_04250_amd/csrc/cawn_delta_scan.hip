// Gated delta rule by chunks, forward.
//
// The chunks of a row are a chain, and a chain is as slow as its links; so the row is cut into segments, each of them some chunks that
// a workgroup takes one after the other with the state in its registers:
//   delta_system  what a chunk is by itself: running sums of the decays, norms, T; all chunks at once
//   delta_scan    MODE 1, all segments at once (the last only for a backward, which takes A from here): what a segment makes of a state, S_end = A S_begin + b; A comes from running
//                 the recurrence on the columns of the identity with v = 0
//   delta_join    the states at the segments' begins, one product a segment
//   delta_scan    MODE 0, all segments at once: the outputs
// Nothing of a chunk goes through memory but its inputs and outputs (and, for a backward, the state before it and its u).  With enough
// rows and heads to fill the chip there is one segment, and MODE 0 is all.
//
// A wave owns 16 columns of the state, all rows of them, in result layout, which is the operand layout of the next product.  Per chunk:
//     X = beta (V - e^G K S),  U = T X,  O^T = scale (e^G S^T Q^T + U^T P^T),  S = e^{G_C} S + K^T (e^{G_C - G} U)
// with P made by all waves together and T fetched.  Four waves to 64 columns keep the state's columns in registers and share what the
// chunk's rows give; k, q and gates of the next chunk travel meanwhile.
//
// Measured, bf16, whole kernels: 8 x 8,192 tokens of 12 heads of 64 (a training step's forward): delta_system 124 us, MODE 1 183, join 16, MODE 0
// 287 (1.1 GB, of them 0.4 the checkpoint); 2 x 32,768 tokens of 32 heads of 128: 420, 949, 25 and 1,541 us.  What bounds MODE 0 and 1 is
// instruction issue: the matrix units are busy a fifth to two fifths of the time, vector instructions (splits into planes, factors)
// another third to two thirds, and between the barriers of a chunk the two to four waves of a SIMD do not always have the other kind to offer.
#include "cawn_delta_mfma.hpp"

namespace cawn {
namespace delta {

// What a chunk is by itself, every chunk a workgroup: gates, the norms' factors, and T = (I + diag(beta) N)^-1.  Bound by vector
// instructions (59 % of the time at K = 64, 70 % at 128) and by the chain of the inverse, four workgroups a CU.
template <typename T, int NP, int KP> __global__ __launch_bounds__(256) void delta_system(const Args a)
{
    constexpr int KS = KP / 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ Gates G;
    const int n = blockIdx.x % a.chunks, bh = blockIdx.x / a.chunks, b = bh / a.H, h = bh % a.H;
    const int rows = min(CHUNK, row_length(a, b) - n * CHUNK);
    if (rows <= 0) return;
    const Tile<NP, CHUNK, KP> k{(bf16 *)lds};
    float *M = (float *)(lds + Tile<NP, CHUNK, KP>::BYTES);
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, g = lane / 16, c = lane % 16;
    const long long qat = b * a.qsb + (long long)n * CHUNK * a.qst + (long long)(h / (a.H / a.Hk)) * a.K;
    RowsAhead<T, NP, KP, 256> ka, qa;
    ka.load(tid, (const T *)a.k + qat, a.qst, rows, a.K, a.vecq);
    if (a.norm) qa.load(tid, (const T *)a.q + qat, a.qst, rows, a.K, a.vecq);
    load_gates(a, G, b, h, n * CHUNK, rows);
    ka.put(tid, k, G.rk, rows, a.K, a.norm, a.eps);
    qa.factors(tid, G.rq, rows, a.K, a.norm, a.eps);
    __syncthreads();
    if (tid < CHUNK) {
        G.c[tid] = G.ed[tid] * G.rk[tid];
        G.x[tid] = tid < rows ? G.beta[tid] * G.eg[tid] * G.rk[tid] : 0.f;
    }
    {
        const int i = 16 * w + c;
        const float m = G.beta[i] * G.rk[i];
#pragma unroll
        for (int jt = 0; jt < 4; ++jt) {
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
            if (jt <= w) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) x = mma<3>(k.straight(16 * jt, 32 * ks, lane), k.straight(16 * w, 32 * ks, lane), x);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 16 * jt + 4 * g + r;
                    x[r] = i > j ? x[r] * (m * G.rk[j] * decay_between(G, i, j)) : 0.f;
                }
            }
            *reinterpret_cast<f32x4 *>(M + i * TLD + 16 * jt + 4 * g) = x;
        }
    }
    __syncthreads();
    const long long at = (long long)bh * a.chunks + n;
    for (int i = tid; i < (int)(sizeof(Gates) / 4); i += 256) a.gates[at * GATE_FLOATS + i] = ((const float *)&G)[i];
    invert(M, w, lane);
    char *out = a.t_ops + (size_t)at * T_BYTES + t_slot(g, c);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        if (2 * ks > w) break;
        float y[8];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const f32x4 e = *reinterpret_cast<const f32x4 *>(M + (16 * w + c) * TLD + 32 * ks + 16 * half + 4 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) y[4 * half + r] = e[r];
        }
        Frag<3> f;
        split8<3>(y, f);
#pragma unroll
        for (int e = 0; e < 3; ++e) *reinterpret_cast<bf16x8 *>(out + (lower(w, ks) * 3 + e) * 1024) = f.p[e];
    }
}

// The scan's LDS: k, q (MODE 0); T; P's operands.  P has a place of its own and is made ahead of the products with the state where that costs no
// workgroup of a CU; elsewhere it is made where T was, for one more barrier.  (In T's place and in its own, us: one workgroup a CU either way, 4,096 tokens
// of 8 heads of 128 in fp32 174 and 169; two, 2 x 32,768 of 32 heads of 128 in bf16 2,855 and 2,803; three and two, 8 x 8,192 of 12 heads of 64 in
// bf16, training, 1,477 and 1,572, but 4 x 16,384 of 8 heads, forward, 364 and 348; two and one, 4,096 of 12 heads of 64 in fp32 91 and 95.)
template <int NP, int KP, int MODE, int NW> struct ScanLds {
    static constexpr int KB = Tile<NP, CHUNK, KP>::BYTES, TO = MODE == 0 ? 2 * KB : KB;
    // waves a SIMD that the registers are budgeted for: as many workgroups as the LDS holds, but three waves (MODE 1 of K <= 64: four) at most
    static constexpr int MOST = MODE == 1 && KP < 128 ? 4 : 3;
    static constexpr int waves(int bytes) { return 163840 / (bytes + (int)sizeof(Gates)) * NW / 4 > MOST ? MOST : 163840 / (bytes + (int)sizeof(Gates)) * NW / 4; }
    static constexpr bool P_EARLY = MODE == 0 && waves(TO + 2 * T_BYTES) == waves(TO + T_BYTES);
    static constexpr int P = P_EARLY ? TO + T_BYTES : TO, BYTES = P + T_BYTES;
    static constexpr int WAVES = waves(BYTES);
};

template <typename T, int NP, int KP, int MODE, int NW> __global__ __launch_bounds__((64 * NW), (ScanLds<NP, KP, MODE, NW>::WAVES)) void delta_scan(const Args a)
{
    using L = ScanLds<NP, KP, MODE, NW>;
    constexpr int KS = KP / 32, KT = KP / 16, NT = 64 * NW;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ Gates G;
    const Tile<NP, CHUNK, KP> k{(bf16 *)lds}, q{(bf16 *)(lds + L::KB)};
    const char *tl = lds + L::TO;
    bf16x8 *pf = reinterpret_cast<bf16x8 *>(lds + L::P);
    const int rows_all = a.B * a.H, blk = blockIdx.x, bh = blk % rows_all, nseg = MODE == 0 || a.s_tiles ? a.segments : a.segments - 1;
    const int seg = blk / rows_all % nseg, group = blk / rows_all / nseg, b = bh / a.H, h = bh % a.H;
    const int len = row_length(a, b), nb = (len + CHUNK - 1) / CHUNK;
    const int n0 = min(seg * a.seg_chunks, nb), n1 = min(n0 + a.seg_chunks, nb);
    if (MODE == 1 && n0 == n1) return;          // (the join asks nothing of a segment that the row does not reach)
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    int tid = threadIdx.x, lane = tid % 64, g = lane / 16, c = lane % 16;
    // column tile: of v, and (MODE 1) beyond it of the identity
    const int ct = group * NW + w, at = ct - a.VT;
    const bool of_v = ct < a.VT, mine = of_v || (MODE == 1 && at < KT);
    int v = 16 * ct + c;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};

    f32x4 S[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        S[t] = zero;
        if (MODE == 1) {
            if (!of_v && at == t) {
#pragma unroll
                for (int r = 0; r < 4; ++r) S[t][r] = 4 * g + r == c ? 1.f : 0.f;
            }
        } else if (of_v && a.segments > 1) S[t] = *reinterpret_cast<const f32x4 *>(a.seg_s + (((size_t)bh * a.segments + seg) * KT * a.VT + (size_t)t * a.VT + ct) * 1024 + lane * 16);
        else if (of_v && a.state_in && v < a.V) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * t + 4 * g + r < a.K) S[t][r] = a.state_in[((long long)bh * a.K + 16 * t + 4 * g + r) * a.V + v];
        }
    }

    // Lane numbers anew, in every chunk and between its steps: left to itself the compiler forms all that follows from them (row
    // numbers, comparisons, addresses: hundreds of values) ahead of the loop, and keeps them.
    // The strides likewise: their multiples would fill the scalar registers.
    long long qst = a.qst, vst = a.vst, ost = a.ost;
    uint32_t l16 = 16 * lane;
    auto anew = [&]() {
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
        if (MODE == 0) qa.load(tid, (const T *)a.q + qat, qst, rows, a.K, a.vecq);
        const float *gp = a.gates + ((long long)bh * a.chunks + n) * GATE_FLOATS;
#pragma unroll
        for (int e = 0; e < GN; ++e) ga[e] = gp[min(tid + e * NT, GATE_FLOATS - 1)];
    };
    auto make_p = [&]() {
        // P's operands, transposed (the result layout is the operand's), shared out: with four waves the first two, whose rows are short, take two
        const int two = NW == 4 && w < 2, first = two ? 2 * w : NW == 4 ? w + 2 : w;
        for (int id = first; id < min(first + 1 + two, 6); ++id) {
            anew();
            const int it = id < 2 ? id : id / 2 + 1, js = id == 3 || id == 5, i = 16 * it + c;
            f32x4 pt[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int jt = 2 * js + half;
                pt[half] = zero;
                if (jt <= it) {
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) pt[half] = mma<3>(k.straight(16 * jt, 32 * ks, lane), q.straight(16 * it, 32 * ks, lane), pt[half]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int j = 16 * jt + 4 * g + r;
                        pt[half][r] = i >= j ? pt[half][r] * (G.rk[j] * decay_between(G, i, j)) : 0.f;
                    }
                }
            }
            Frag<3> f;
            split_tiles<3>(pt[0], pt[1], f);
#pragma unroll
            for (int e = 0; e < 3; ++e) pf[(id * 3 + e) * 64 + lane] = f.p[e];
        }
    };
    if (n0 < n1) ahead(n0);
    for (int n = n0; n < n1; ++n) {
        const int rows = min(CHUNK, len - n * CHUNK);
        anew();
        asm volatile("" : "+s"(qst), "+s"(vst), "+s"(ost));
        if (n > n0) __syncthreads();
        ka.put_plain(tid, k, rows, a.K);
        if (MODE == 0) qa.put_plain(tid, q, rows, a.K);
#pragma unroll
        for (int e = 0; e < GN; ++e)
            if (tid + e * NT < GATE_FLOATS) ((float *)&G)[tid + e * NT] = ga[e];
        __syncthreads();
        {
            // T comes straight into LDS (behind the barrier, which would wait for it)
            const char *src = a.t_ops + ((size_t)bh * a.chunks + n) * T_BYTES;
            char *dst = lds + L::TO;
#pragma unroll
            for (int u = 0; u < (T_BYTES / 1024 + NW - 1) / NW; ++u) {
                const int i = u * NW + w;
                if (i < T_BYTES / 1024) load_piece(src + (size_t)i * 1024 + l16, dst + i * 1024);
            }
        }
        // v is wanted last.  (What is not there is loaded from where something is, and dropped where it is used: a load behind a lane's
        // branch, or one whose value is converted at once, would be waited for here)
        T va[4][4];
        if (of_v) {
            const T *vp = (const T *)a.v + b * a.vsb + (long long)n * CHUNK * vst + (long long)h * a.V;
            if (rows == CHUNK && 16 * ct + 16 <= a.V && vst < (1 << 22)) {
                vp += 16 * ct;
                const uint32_t vlane = (4 * (uint32_t)g * (uint32_t)vst + c) * sizeof(T);         // a lane's place among the rows
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) va[t][r] = *reinterpret_cast<const T *>((const char *)(vp + (16 * t + r) * vst) + vlane);
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) va[t][r] = vp[min(16 * t + 4 * g + r, rows - 1) * vst + min(v, a.V - 1)];
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * t + 4 * g + r >= rows || v >= a.V) va[t][r] = (T)0.f;
            }
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) va[t][r] = (T)0.f;
        }
        if (n + 1 < n1) ahead(n + 1);
        anew();
        if (MODE == 0 && L::P_EARLY) make_p();
        // what hangs on the state before the chunk
        anew();
        f32x4 U[4];
        f32x4 O[MODE == 0 ? 4 : 1];
        {
            Frag<3> sf[KS];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) split_tiles<3>(S[2 * ks], S[2 * ks + 1], sf[ks]);
            f32x4 X[4] = {zero, zero, zero, zero};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                Frag<NP> f[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) f[t] = k.tiled(16 * t, 32 * ks, lane);
                mma_each<3>(f, sf[ks], X);
            }
            if (MODE == 0) {
#pragma unroll
                for (int t = 0; t < 4; ++t) O[t] = zero;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    Frag<NP> f[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) f[t] = q.tiled(16 * t, 32 * ks, lane);
                    mma_each<3>(sf[ks], f, O);
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) O[t] *= G.eg[16 * t + c];
            }
            Frag<3> xf[2];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const f32x4 xs = *reinterpret_cast<const f32x4 *>(G.x + 16 * t + 4 * g), be = *reinterpret_cast<const f32x4 *>(G.beta + 16 * t + 4 * g);
#pragma unroll
                for (int r = 0; r < 4; ++r) X[t][r] = fmaf(-xs[r], X[t][r], be[r] * (float)va[t][r]);
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) split_tiles<3>(X[2 * ks], X[2 * ks + 1], xf[ks]);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();                    // T
            anew();
            Frag<3> f[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                U[t] = zero;
                f[t] = t_rows(tl, t, 0, lane);
            }
            mma_each<3>(f, xf[0], U);
            Frag<3> f2[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) f2[t] = t_rows(tl, 2 + t, 1, lane);
            mma_each<3>(f2, xf[1], U + 2);
        }
        anew();
        if (MODE == 0) {
            // (stores behind the wait for T, which would wait for them too)
            if (a.s_tiles && mine) {
                char *st = a.s_tiles + bh * a.s_row + n * a.s_chunk + (size_t)ct * 1024;
#pragma unroll
                for (int t = 0; t < KT; ++t) *reinterpret_cast<f32x4 *>(st + (size_t)t * a.VT * 1024 + l16) = S[t];
            }
            if (a.u_tiles && mine) {
                char *ut = a.u_tiles + bh * a.u_row + n * a.u_chunk + (size_t)ct * 1024;
#pragma unroll
                for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4 *>(ut + (size_t)t * a.VT * 1024 + l16) = U[t];
            }
        }
        if (MODE == 0 && !L::P_EARLY) {
            __syncthreads();                    // nobody reads T any more
            make_p();
        }
        anew();
        {
            Frag<3> uf[2];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                f32x4 y[2];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int t = 2 * ks + half;
                    y[half] = U[t] * *reinterpret_cast<const f32x4 *>(G.c + 16 * t + 4 * g);
                }
                split_tiles<3>(y[0], y[1], uf[ks]);
            }
            const float e = G.eg[CHUNK - 1];
#pragma unroll
            for (int t = 0; t < KT; ++t) S[t] *= e;
            constexpr int AT = KT < 4 ? KT : 4;
#pragma unroll
            for (int t0 = 0; t0 < KT; t0 += AT)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    Frag<NP> f[AT];
#pragma unroll
                    for (int t = 0; t < AT; ++t) f[t] = k.tiled_down(32 * ks, 16 * (t0 + t), lane);
                    mma_each<3>(f, uf[ks], S + t0);
                }
        }
        if (MODE == 0) {
            if (!L::P_EARLY) __syncthreads();   // P's operands
            anew();
            Frag<3> uf[2];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) split_tiles<3>(U[2 * ks], U[2 * ks + 1], uf[ks]);
            const int all = min(CHUNK, a.L - n * CHUNK);
            // a lane's place among rows of o, in bytes
            const bool whole = rows == CHUNK && a.veco && 16 * ct + 16 <= a.V && ost < (1 << 22);
            const uint32_t olane = ((uint32_t)c * (uint32_t)ost + 4 * g) * sizeof(T);
            T *op = (T *)a.o + b * a.osb + (long long)n * CHUNK * ost + (long long)h * a.V + 16 * ct;
            {
                Frag<3> f[4], f2[2];
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 3; ++e) f[t].p[e] = pf[(lower(t, 0) * 3 + e) * 64 + lane];
                mma_each<3>(uf[0], f, O);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 3; ++e) f2[t].p[e] = pf[(lower(2 + t, 1) * 3 + e) * 64 + lane];
                mma_each<3>(uf[1], f2, O + 2);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int i = 16 * t + c;
                const float m = i < rows ? a.scale * G.rq[i] : 0.f;
                float y[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) y[r] = O[t][r] * m;
                if (rows < CHUNK && i >= rows) y[0] = y[1] = y[2] = y[3] = 0.f;         // (whatever the state holds)
                if (!mine) continue;
                T *dst = op + (long long)(16 * t) * ost;
                if (whole) store_n<T, 4>(reinterpret_cast<T *>((char *)dst + olane), y);
                else if (i < all) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * ct + 4 * g + r < a.V) dst[c * ost + 4 * g + r] = (T)y[r];
                }
            }
        }
    }
    if (MODE == 0) {
        // chunks of this segment that the row does not have
        const int last = min(seg == a.segments - 1 ? a.chunks : (seg + 1) * a.seg_chunks, a.chunks);
        for (int t = max(n1, seg * a.seg_chunks) * CHUNK + (int)threadIdx.x / 64; t < min(last * CHUNK, a.L); t += NW) {
            for (int vv = group * NW * 16 + lane; vv < min(a.V, (group + 1) * NW * 16); vv += 64) ((T *)a.o)[b * a.osb + (long long)t * a.ost + (long long)h * a.V + vv] = (T)0.f;
        }
    }
    if (!mine) return;
    if (MODE == 1) {
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            if (of_v) *reinterpret_cast<f32x4 *>(a.seg_b + (((size_t)bh * a.segments + seg) * KT * a.VT + (size_t)t * a.VT + ct) * 1024 + lane * 16) = S[t];
            else {
                float *A = (float *)a.seg_a + ((size_t)bh * a.segments + seg) * KP * KP + (size_t)(16 * t + 4 * g) * KP + 16 * at + c;
#pragma unroll
                for (int r = 0; r < 4; ++r) A[r * KP] = S[t][r];
            }
        }
        return;
    }
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        if (seg == a.segments - 1 && a.state_out && v < a.V) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * t + 4 * g + r < a.K) a.state_out[((long long)bh * a.K + 16 * t + 4 * g + r) * a.V + v] = S[t][r];
        }
    }
}

template <typename T, int NP, int KP, int MODE, int NW> static int launch(const Args &a, long long segments, long long tiles, hipStream_t s)
{
    constexpr int bytes = ScanLds<NP, KP, MODE, NW>::BYTES;
    static_assert(bytes + sizeof(Gates) <= 163840, "LDS");
    if (bytes > 60000 && hipFuncSetAttribute((const void *)delta_scan<T, NP, KP, MODE, NW>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return CAWN_ELAUNCH;
    hipLaunchKernelGGL((delta_scan<T, NP, KP, MODE, NW>), dim3((unsigned)((long long)a.B * a.H * segments * ceil_div(tiles, NW))), dim3(64 * NW), bytes, s, a);
    return launched();
}

template <typename T, int NP, int KP> static int scan_kp(const Args &a, hipStream_t s)
{
    if (a.segments > 1) {
        // Eight waves where they divide the columns; four where half of eight would have none, and at K = 128, where they have more registers (us for
        // eight and four: 8 x 8,192 tokens of 12 heads of 64 in bf16, training, 1,476 and 1,510; 8 x 4,096 of 8 heads of 64 x 128 283 and 257;
        // 8 x 4,096 of 16 heads of 32, training, 700 and 663; 2 x 32,768 of 32 heads of 128 3,094 and 2,790)
        const long long segments = a.s_tiles ? a.segments : a.segments - 1, tiles = a.VT + KP / 16;
        int r;
        if constexpr (KP == 128) r = launch<T, NP, KP, 1, 4>(a, segments, tiles, s);
        else r = ceil_div(tiles, 4) % 2 ? launch<T, NP, KP, 1, 4>(a, segments, tiles, s) : launch<T, NP, KP, 1, 8>(a, segments, tiles, s);
        if (r) return r;
        if (int r = launch_join(a, false, s)) return r;
    }
    // Where the LDS holds one workgroup of four waves a CU, eight waves take twice the columns, if there are as many (us for eight and four, 4,096
    // tokens of 8 heads in fp32: of 128 x 192 184 and 197, of 128 x 128 169 and 160).  Elsewhere four, where eight gain on long rows and lose on others
    // (bf16, heads of 128: 2 x 32,768 of 32 2,622 and 2,790, 4 x 16,384 of 8 747 and 775; 16 x 512 of 8 105 and 91, 16 x 4,096 of them, training, 2,332 and 2,253)
    if constexpr (NP == 3 && KP == 128)
        if (a.VT > 4) return launch<T, NP, KP, 0, 8>(a, a.segments, a.VT, s);
    return launch<T, NP, KP, 0, 4>(a, a.segments, a.VT, s);
}

template <typename T, int NP, int KP> static int system_kp(const Args &a, hipStream_t s)
{
    constexpr int bytes = Tile<NP, CHUNK, KP>::BYTES + CHUNK * TLD * 4;
    if (bytes > 60000 && hipFuncSetAttribute((const void *)delta_system<T, NP, KP>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return CAWN_ELAUNCH;
    const long long n = (long long)a.B * a.H * a.chunks;
    if (n == 0) return CAWN_OK;
    hipLaunchKernelGGL((delta_system<T, NP, KP>), dim3((unsigned)n), dim3(256), bytes, s, a);
    return launched();
}

int launch_system(const Args &a, bool bf16_, hipStream_t s)
{
    if (a.K <= 32) return bf16_ ? system_kp<bf16, 1, 32>(a, s) : system_kp<float, 3, 32>(a, s);
    if (a.K <= 64) return bf16_ ? system_kp<bf16, 1, 64>(a, s) : system_kp<float, 3, 64>(a, s);
    return bf16_ ? system_kp<bf16, 1, 128>(a, s) : system_kp<float, 3, 128>(a, s);
}

template <int NP, int KP> static int held(int VT, int *columns)
{
    const bool wide = NP == 3 && KP == 128 && VT > 4;           // as scan_kp has it
    *columns = wide ? 8 : 4;
    return wide ? ScanLds<NP, KP, 0, 8>::WAVES / 2 : ScanLds<NP, KP, 0, 4>::WAVES;
}

int scan_held(int K, int VT, bool bf16_, int *columns)
{
    if (K <= 32) return bf16_ ? held<1, 32>(VT, columns) : held<3, 32>(VT, columns);
    if (K <= 64) return bf16_ ? held<1, 64>(VT, columns) : held<3, 64>(VT, columns);
    return bf16_ ? held<1, 128>(VT, columns) : held<3, 128>(VT, columns);
}

int launch_scan(const Args &a, bool bf16_, hipStream_t s)
{
    if (a.K <= 32) return bf16_ ? scan_kp<bf16, 1, 32>(a, s) : scan_kp<float, 3, 32>(a, s);
    if (a.K <= 64) return bf16_ ? scan_kp<bf16, 1, 64>(a, s) : scan_kp<float, 3, 64>(a, s);
    return bf16_ ? scan_kp<bf16, 1, 128>(a, s) : scan_kp<float, 3, 128>(a, s);
}

} // namespace delta
} // namespace cawn
