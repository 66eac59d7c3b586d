// Gated delta rule by chunks, backward.
//
// With dS the gradient of the state behind a chunk, dO that of its output, and the forward's S0 and U from the checkpoint:
//     dR  = T^T (scale P^T dO + KD dS),  KD = diag(e^{G_C - G}) K      gradient of U through everything but T's inverse; dV = beta dR
//     dS0 = e^{G_C} dS + scale (e^G Q)^T dO - (beta e^G K)^T dR
//     Z   = scale (dO U^T) o D (lower),  M = -(beta dR U^T) o D (strictly lower)
//     dQ  = scale e^G dO S0^T + Z K
//     dK  = -beta e^G dR S0^T + M K + Z^T Q + M^T K + e^{G_C - G} U dS^T
//     dbeta_i = dR_i . U_i / beta_i
//     ddecay_t = sum_{i >= t} a_i + sum_{j < t} b_j + sum_{i >= t > j} (Z_ij q_i . k_j + M_ij k_i . k_j) + e^{G_C} <dS, S0>
//     a_i = q_i . (scale e^G dO S0^T)_i - k_i . (beta e^G dR S0^T)_i,   b_j = k_j . (e^{G_C - G} U dS^T)_j
// The last: a decay scales all that passes from before its token to it and behind it, from the chunk's begin or a token in it to its end or a
// token in it.  Every term holds the factors of the decays between its ends, the token's own among them, and the sum has its digits however little is
// left of what came before.  (The same sum is that of q.dq - v.dv over the tokens behind, and <dS, S_C>: there the terms do not shrink with the decay, cancel,
// and leave their rounding, 1e-2 of the gradient at a decay of -8 and nothing but rounding from -15 on.)
//
// dR and dS come from the recurrence (delta_back); here every chunk is a workgroup.
#include "cawn_delta_mfma.hpp"

namespace cawn {
namespace delta {

// Gradients of a chunk.  A workgroup takes all value heads of a key head, one after the other, and keeps dq and dk in registers: wave w
// and wave 4 + w rows 16 w .. of them, half of the columns each.  First everything that runs over the value columns, 32 at a time, with U, dR, S0 and dS in LDS as they come
// from their tiles (a tile's lane holds four rows of a column: a matrix is kept as its transpose, and read down); then, in the same
// LDS, Z and M with q and k.
// Measured: 8 x 8,192 tokens of 12 heads of 64 in bf16: 622 us for 1.5 GB (of them U, dR, S0 and dS 0.8), 2.4 TB/s.  Of a workgroup's time a third
// is the way of its first loads and last stores, the rest splits, products and barriers in turn: neither bandwidth nor the units are full.
// Eight waves of half the columns, not four of all: fp32, 5 x 777 tokens of 4 heads of 64 x 128 45 us, 53; this shape within 1 %.
constexpr int WLD = CHUNK + 4;          // (four rows apart begin in other banks)
template <typename T, int NP, int KP> struct GradLds {
    using MatU = Tile<3, 32, 64>;
    using MatR = Tile<3, 32, 64>;
    using MatS = Tile<3, 32, KP>;
    using MatD = Tile<3, 32, KP>;
    using MatO = Tile<NP, CHUNK, 32>;
    using MatQ = Tile<NP, CHUNK, KP>;
    using MatZ = Tile<3, CHUNK, CHUNK>;
    using MatM = Tile<3, CHUNK, CHUNK>;
    static_assert(MatZ::BYTES >= (CHUNK * WLD + CHUNK / 4 * CHUNK + 4 * CHUNK) * 4, "wl, its sums and the norms' in Z's place");
    static constexpr int FIRST = MatU::BYTES + MatR::BYTES + MatS::BYTES + MatD::BYTES + MatO::BYTES;
    static constexpr int SECOND = 2 * MatQ::BYTES + MatZ::BYTES + MatM::BYTES;
    static constexpr int BYTES = FIRST > SECOND ? FIRST : SECOND;
    // waves a SIMD: as many workgroups as the LDS holds, two at most.  (With SHARED one, which has registers for the sums over the heads:
    // 4 x 4,096 tokens of 12 heads of 64 on 4 of keys in bf16, whole backward and forward: 452 us, 479 with two.)
    static constexpr int HELD = 163840 / (BYTES + 4096), WAVES = HELD > 2 ? 4 : 2 * HELD;
};

// four rows of a column, N planes, into a transposed matrix
template <int N, int ROWS, int COLS> __device__ inline void put_column(const Tile<N, ROWS, COLS> &t, int col, int row0, f32x4 x)
{
    bf16x4 h[N];
    split4<N>(x, h);
#pragma unroll
    for (int p = 0; p < N; ++p) *reinterpret_cast<bf16x4 *>(t.p + p * Tile<N, ROWS, COLS>::PLANE + col * Tile<N, ROWS, COLS>::LD + row0) = h[p];
}

// four values of a row, from their planes
template <int N, int ROWS, int COLS> __device__ inline void row_of(const Tile<N, ROWS, COLS> &t, int row, int col, float (&x)[4])
{
    bf16x4 h[N];
#pragma unroll
    for (int p = 0; p < N; ++p) h[p] = *reinterpret_cast<const bf16x4 *>(t.p + p * Tile<N, ROWS, COLS>::PLANE + row * Tile<N, ROWS, COLS>::LD + col);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        x[r] = 0.f;
#pragma unroll
        for (int p = N - 1; p >= 0; --p) x[r] += (float)h[p][r];
    }
}

// sum over the 16 lanes of a result tile's row
__device__ inline float row_sum(float x)
{
#pragma unroll
    for (int m = 8; m > 0; m >>= 1) x += __shfl_xor(x, m);
    return x;
}

// SHARED: several value heads to a key head
template <typename T, int NP, int KP, bool SHARED> __global__ __launch_bounds__(512, (SHARED ? 2 : GradLds<T, NP, KP>::WAVES)) void delta_gradients(const Args a)
{
    using L = GradLds<T, NP, KP>;
    constexpr int KT = KP / 16, KH = KT / 2, OWN = (KT + 3) / 4, NT = 512;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ Gates G;
    __shared__ float reads[2][CHUNK], writes[2][CHUNK], udr[2][CHUNK], part[8];       // a, b, dR.U; shares of <dS, S0>
    const int blk = blockIdx.x, n = blk % a.chunks, bk = blk / a.chunks, hk = bk % a.Hk, b = bk / a.Hk, rep = a.H / a.Hk;
    const int len = row_length(a, b), t0 = n * CHUNK, rows = min(CHUNK, len - t0), all = min(CHUNK, a.L - t0);
    const long long qat = b * a.qsb + t0 * a.qst + (long long)hk * a.K;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), w = wave % 4, half = wave / 4;
    int tid = threadIdx.x, lane = tid % 64, g = lane / 16, c = lane % 16;
    auto anew = [&]() {                         // (as in delta_scan)
        tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        lane = tid % 64, g = lane / 16, c = lane % 16;
    };
    if (rows <= 0) {                            // tokens that the row does not have
        for (int i = threadIdx.x; i < all * a.K; i += NT) {
            const long long at = qat + (long long)(i / a.K) * a.qst + i % a.K;
            if (a.dq) ((T *)a.dq)[at] = (T)0.f;
            if (a.dk) ((T *)a.dk)[at] = (T)0.f;
        }
        for (int hh = 0; hh < rep; ++hh) {
            const int h = hk * rep + hh;
            if (a.dv)
                for (int i = threadIdx.x; i < all * a.V; i += NT) ((T *)a.dv)[b * a.vsb + (t0 + i / a.V) * a.vst + (long long)h * a.V + i % a.V] = (T)0.f;
            if ((int)threadIdx.x < all) {
                const long long at = ((long long)b * a.L + t0 + threadIdx.x) * a.H + h;
                if (a.ddecay) a.ddecay[at] = 0.f;
                if (a.dbeta) a.dbeta[at] = 0.f;
            }
        }
        return;
    }
    const Sizes z(a.K, a.V);
    const typename L::MatU ut{(bf16 *)lds};
    const typename L::MatR rt{(bf16 *)(lds + L::MatU::BYTES)};
    const typename L::MatS st{(bf16 *)(lds + L::MatU::BYTES + L::MatR::BYTES)};
    const typename L::MatD dt{(bf16 *)(lds + L::MatU::BYTES + L::MatR::BYTES + L::MatS::BYTES)};
    const typename L::MatO ot{(bf16 *)(lds + L::MatU::BYTES + L::MatR::BYTES + L::MatS::BYTES + L::MatD::BYTES)};
    const typename L::MatQ qm{(bf16 *)lds}, km{(bf16 *)(lds + L::MatQ::BYTES)};
    const typename L::MatZ zm{(bf16 *)(lds + 2 * L::MatQ::BYTES)};
    const typename L::MatM mm{(bf16 *)(lds + 2 * L::MatQ::BYTES + L::MatZ::BYTES)};
    // the wave's two column tiles of Z and M: 0 and 3, or 1 and 2
    auto own = [&](int e) { return half ? 1 + e : 3 * e; };
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    f32x4 dq[KH], dk[KH];
    if (SHARED) {
#pragma unroll
        for (int t = 0; t < KH; ++t) dq[t] = dk[t] = zero;
    }
    for (int hh = 0; hh < (SHARED ? rep : 1); ++hh) {
        const int h = hk * rep + hh, bh = b * a.H + h;
        const size_t at = (size_t)bh * a.chunks + n;
        const char *sp = a.s_tiles + bh * a.s_row + n * a.s_chunk, *up = a.u_tiles + bh * a.u_row + n * a.u_chunk;
        const char *rp = a.dr_tiles + at * z.ut * 1024, *dp = a.ds_tiles + at * z.st * 1024;
        __syncthreads();                        // the previous head's LDS
        anew();
        f32x4 A1[KH], A2[KH], A3[KH], zt[2], mt[2];
#pragma unroll
        for (int t = 0; t < KH; ++t) A1[t] = A2[t] = A3[t] = zero;
#pragma unroll
        for (int t = 0; t < 2; ++t) zt[t] = mt[t] = zero;
        float inner = 0.f;                      // <dS, S0>
        float su[4] = {0.f, 0.f, 0.f, 0.f};
        // A step's loads are all under way before the first is wanted: tiles, and (from where something is, and dropped below) dO.
        // Waves w and 4 + w: row tile w of U and dR; row tiles w, w + 4 of the states; a column tile each
        f32x4 tu, tr, ts[OWN], td[OWN];
        RowsAhead<T, NP, 32, NT> to;
        auto ahead = [&](int v0) {
            const int vt = min(v0 / 16 + half, a.VT - 1);
            tu = *reinterpret_cast<const f32x4 *>(up + ((size_t)w * a.VT + vt) * 1024 + lane * 16);
            tr = *reinterpret_cast<const f32x4 *>(rp + ((size_t)w * a.VT + vt) * 1024 + lane * 16);
#pragma unroll
            for (int o = 0; o < OWN; ++o) {
                const size_t at = ((size_t)min(w + 4 * o, KT - 1) * a.VT + vt) * 1024 + lane * 16;
                ts[o] = *reinterpret_cast<const f32x4 *>(sp + at);
                td[o] = *reinterpret_cast<const f32x4 *>(dp + at);
            }
            to.load(tid, (const T *)a.dO + b * a.osb + (long long)t0 * a.ost + (long long)h * a.V + v0, a.ost, rows, min(32, a.V - v0), a.veco);
        };
        // (the gates first: what is loaded before them would have to come before they do)
        constexpr int GN = (GATE_FLOATS + NT - 1) / NT;
        float ga[GN];
#pragma unroll
        for (int e = 0; e < GN; ++e) ga[e] = a.gates[at * GATE_FLOATS + min(tid + e * NT, GATE_FLOATS - 1)];
        ahead(0);
#pragma unroll
        for (int e = 0; e < GN; ++e)
            if (tid + e * NT < GATE_FLOATS) ((float *)&G)[tid + e * NT] = ga[e];
        for (int v0 = 0; v0 < a.V; v0 += 32) {
            __syncthreads();
            anew();
            {
                const int vt = v0 / 16 + half, v = 16 * vt + c;
                const bool there = vt < a.VT;
                const f32x4 u = there ? tu : zero, r = there ? tr : zero;
                put_column(ut, 16 * half + c, 16 * w + 4 * g, u);
                put_column(rt, 16 * half + c, 16 * w + 4 * g, r);
                T *dvp = (T *)a.dv + b * a.vsb + (long long)t0 * a.vst + (long long)h * a.V + v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 16 * w + 4 * g + e;
                    su[e] += u[e] * r[e];
                    const float dv = G.beta[i] * r[e];
                    if (a.dv && v < a.V && i < all) dvp[i * a.vst] = (T)(i < rows ? dv : 0.f);
                }
#pragma unroll
                for (int o = 0; o < OWN; ++o) {
                    const int t = w + 4 * o;
                    if (t >= KT) break;
                    const f32x4 s = there ? ts[o] : zero, d = there ? td[o] : zero;
                    put_column(st, 16 * half + c, 16 * t + 4 * g, s);
                    put_column(dt, 16 * half + c, 16 * t + 4 * g, d);
#pragma unroll
                    for (int x = 0; x < 4; ++x) inner += d[x] * s[x];
                }
            }
            to.put_plain(tid, ot, rows, min(32, a.V - v0));
            __syncthreads();
            anew();
            const Frag<NP> o = ot.straight(16 * w, 0, lane);
            const Frag<3> r = rt.straight_down(0, 16 * w, lane);
            // before their factors: Z^T and M^T, rows j and column i = c of row tile w; dO S0^T and the like, rows f and column i = c
            // (a tile at a time: there are four waves a SIMD to fill the pauses, but no registers)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (own(e) > w) continue;
                const Frag<3> uj[1] = {ut.straight_down(0, 16 * own(e), lane)};
                mma_each<3>(uj, o, zt + e);
                mma_each<3>(uj, r, mt + e);
                __builtin_amdgcn_sched_barrier(0);
            }
            anew();
#pragma unroll
            for (int t = 0; t < KH; ++t) {
                const Frag<3> f[1] = {st.straight_down(0, 16 * (half * KH + t), lane)};
                mma_each<3>(f, o, A1 + t);
                mma_each<3>(f, r, A2 + t);
                __builtin_amdgcn_sched_barrier(0);
            }
            const Frag<3> u = ut.straight_down(0, 16 * w, lane);
#pragma unroll
            for (int t = 0; t < KH; ++t) {
                const Frag<3> d[1] = {dt.straight_down(0, 16 * (half * KH + t), lane)};
                mma_each<3>(d, u, A3 + t);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (v0 + 32 < a.V) ahead(v0 + 32);
        }
        // the second half's
        RowsAhead<T, NP, KP, NT> qa, ka;
        qa.load(tid, (const T *)a.q + qat, a.qst, rows, a.K, a.vecq);
        ka.load(tid, (const T *)a.k + qat, a.qst, rows, a.K, a.vecq);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float t = row_sum(su[e]);
            if (c == 0) udr[half][16 * w + 4 * g + e] = t;
        }
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) inner += __shfl_xor(inner, m);
        if (lane == 0) part[wave] = inner;
        __syncthreads();                        // the LDS of the first half is free
        anew();
        qa.put_plain(tid, qm, rows, a.K);
        ka.put_plain(tid, km, rows, a.K);
        const int i = 16 * w + c;               // the lane's token from here on
        const float eg = G.eg[i], beta = G.beta[i], rk = G.rk[i], rq = G.rq[i], sq = a.scale * rq, bk = -beta * rk;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int j0 = 16 * own(e) + 4 * g;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = j0 + r;
                const float D = i >= j ? G.rk[j] * decay_between(G, i, j) : 0.f;
                zt[e][r] = i >= j ? zt[e][r] * (sq * D) : 0.f;
                mt[e][r] = i > j ? mt[e][r] * (bk * D) : 0.f;
            }
            put_column(zm, i, j0, zt[e]);                       // (here the column of the transpose is the row)
            put_column(mm, i, j0, mt[e]);
        }
        // y = r dx^ of the norm's x^ = r x:  yq = scale rq e^G A1 + Z k,  yk = rk (e^{G_C - G} A3 - beta e^G A2) + M k + Z^T q + M^T k
        const float f1 = sq * eg, f2 = bk * eg, f3 = rk * G.ed[i];
        __syncthreads();
        anew();
        // Z o Q K^T + M o K K^T, of which ddecay takes what lies below; a and b
        f32x4 wt[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (own(e) > w) continue;
            f32x4 qk = zero, kk = zero;
#pragma unroll
            for (int ks = 0; ks < KP / 32; ++ks) {
                const Frag<NP> kj = km.straight(16 * own(e), 32 * ks, lane);
                qk = mma<3>(kj, qm.straight(16 * w, 32 * ks, lane), qk);
                kk = mma<3>(kj, km.straight(16 * w, 32 * ks, lane), kk);
            }
            wt[e] = zt[e] * qk + mt[e] * kk;
        }
        {
            float sa = 0.f, sb = 0.f;
#pragma unroll
            for (int t = 0; t < KH; ++t) {
                float xq[4], xk[4];
                row_of(qm, 16 * w + c, 16 * (half * KH + t) + 4 * g, xq);
                row_of(km, 16 * w + c, 16 * (half * KH + t) + 4 * g, xk);
                A1[t] *= f1, A2[t] *= f2, A3[t] *= f3;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    sa = fmaf(xq[r], A1[t][r], sa);
                    sa = fmaf(xk[r], A2[t][r], sa);
                    sb = fmaf(xk[r], A3[t][r], sb);
                }
                A2[t] += A3[t];
            }
            sa += __shfl_xor(sa, 16), sb += __shfl_xor(sb, 16);
            sa += __shfl_xor(sa, 32), sb += __shfl_xor(sb, 32);
            if (g == 0) reads[half][16 * w + c] = sa, writes[half][16 * w + c] = sb;
        }
        anew();
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            constexpr int AT = KH < 4 ? KH : 4;
            const bool left = 2 * ks <= w, right = 2 * ks + 1 >= w;
            Frag<3> zf, zd, mf, md;
            if (left) zf = zm.straight(16 * w, 32 * ks, lane), mf = mm.straight(16 * w, 32 * ks, lane);
            if (right) zd = zm.straight_down(32 * ks, 16 * w, lane), md = mm.straight_down(32 * ks, 16 * w, lane);
#pragma unroll
            for (int t0 = 0; t0 < KH; t0 += AT) {
                Frag<NP> kf[AT], qf[AT];
#pragma unroll
                for (int t = 0; t < AT; ++t) kf[t] = km.straight_down(32 * ks, 16 * (half * KH + t0 + t), lane);
                if (left) {
                    mma_each<3>(kf, zf, A1 + t0);
                    mma_each<3>(kf, mf, A2 + t0);
                }
                if (right) {
#pragma unroll
                    for (int t = 0; t < AT; ++t) qf[t] = qm.straight_down(32 * ks, 16 * (half * KH + t0 + t), lane);
                    mma_each<3>(qf, zd, A2 + t0);
                    mma_each<3>(kf, md, A2 + t0);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < KH; ++t) {
            dq[t] = SHARED ? dq[t] + A1[t] : A1[t];
            dk[t] = SHARED ? dk[t] + A2[t] : A2[t];
        }
        __syncthreads();                        // nobody wants Z any more
        anew();
        // wl[j][i], and the sums of four rows j of it (rows beyond i, which are not written, are dropped below)
        float *wl = (float *)zm.p, *quads = wl + CHUNK * WLD;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (own(e) > w) continue;
            const int j0 = 16 * own(e) + 4 * g;
#pragma unroll
            for (int r = 0; r < 4; ++r) wl[(j0 + r) * WLD + 16 * w + c] = wt[e][r];
            quads[j0 / 4 * CHUNK + 16 * w + c] = (wt[e][0] + wt[e][1]) + (wt[e][2] + wt[e][3]);
        }
        __syncthreads();
        {
            // a wave takes eight tokens t, a lane one i: what passes from before t to i, or (i < t) from i to the chunk's end
            const int i = lane, first = 8 * wave;
            const float read = reads[0][i] + reads[1][i], write = writes[0][i] + writes[1][i];
            float before = 0.f, x[8];
            for (int j = 0; j < 2 * wave; ++j) before += quads[j * CHUNK + i];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = i >= rows ? 0.f : i >= first + e ? before + read : write;
                before += wl[(first + e) * WLD + i];
            }
            // eight sums over the lanes: halves of them change hands, so that a lane is left with one
#pragma unroll
            for (int m = 32, n = 4; n > 0; m >>= 1, n >>= 1) {
#pragma unroll
                for (int e = 0; e < n; ++e) {
                    const float give = i & m ? x[e] : x[e + n];
                    x[e] = (i & m ? x[e + n] : x[e]) + __shfl_xor(give, m);
                }
            }
            x[0] += __shfl_xor(x[0], 4);
            x[0] += __shfl_xor(x[0], 2);
            x[0] += __shfl_xor(x[0], 1);
            const int t = first + (lane >> 3);          // bits 5, 4, 3 of the lane: which half was kept
            const float whole = ((part[0] + part[1]) + (part[2] + part[3])) + ((part[4] + part[5]) + (part[6] + part[7]));
            const long long at = ((long long)b * a.L + t0 + t) * a.H + h;
            // (a complete forgetting hangs on nothing)
            if (a.ddecay && lane % 8 == 0 && t < all) a.ddecay[at] = t < rows && !(a.decay[at] < DECAY_MIN) ? fmaf(G.eg[CHUNK - 1], whole, x[0]) : 0.f;
        }
        if (a.dbeta && tid < all) a.dbeta[((long long)b * a.L + t0 + tid) * a.H + h] = tid < rows ? (udr[0][tid] + udr[1][tid]) / G.beta[tid] : 0.f;
    }
    // through the norm, and out: dx = r (dx^ - x^ (x^ . dx^)) = y - r^2 x (x . y)
    const int i = 16 * w + c, f0 = 16 * KH * half + 4 * g;
    float (*xdx)[2][CHUNK] = reinterpret_cast<float (*)[2][CHUNK]>((float *)zm.p + CHUNK * WLD + CHUNK / 4 * CHUNK);      // (behind wl and its sums)
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float s = 0.f;
#pragma unroll
        for (int t = 0; t < KH; ++t) {
            float x[4];
            row_of(which ? km : qm, i, f0 + 16 * t, x);
#pragma unroll
            for (int r = 0; r < 4; ++r) s = fmaf(x[r], which ? dk[t][r] : dq[t][r], s);
        }
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (g == 0) xdx[which][half][i] = s;
    }
    __syncthreads();
    if (i >= all) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (!(which ? a.dk : a.dq)) continue;
        T *out = (T *)(which ? a.dk : a.dq) + qat + (long long)i * a.qst + f0;
        const float f = which ? G.rk[i] : G.rq[i], s = a.norm ? -(xdx[which][0][i] + xdx[which][1][i]) * f * f : 0.f;
#pragma unroll
        for (int t = 0; t < KH; ++t) {
            float x[4], y[4];
            row_of(which ? km : qm, i, f0 + 16 * t, x);
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = i < rows ? fmaf(x[r], s, which ? dk[t][r] : dq[t][r]) : 0.f;
            if (a.vecd && f0 + 16 * t + 4 <= a.K) store_n<T, 4>(out + 16 * t, y);
            else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (f0 + 16 * t + r < a.K) out[16 * t + r] = (T)y[r];
            }
        }
    }
}

template <typename T, int NP, int KP, bool SHARED> static int gradients_of(const Args &a, hipStream_t s)
{
    constexpr int bytes = GradLds<T, NP, KP>::BYTES;
    static_assert(bytes + sizeof(Gates) + (6 * CHUNK + 8) * 4 <= 163840, "LDS");
    if (a.chunks == 0) return CAWN_OK;
    if (hipFuncSetAttribute((const void *)delta_gradients<T, NP, KP, SHARED>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return CAWN_ELAUNCH;
    hipLaunchKernelGGL((delta_gradients<T, NP, KP, SHARED>), dim3((unsigned)((long long)a.B * a.Hk * a.chunks)), dim3(512), bytes, s, a);
    return launched();
}
template <typename T, int NP, int KP> static int gradients_kp(const Args &a, hipStream_t s)
{
    return a.H > a.Hk ? gradients_of<T, NP, KP, true>(a, s) : gradients_of<T, NP, KP, false>(a, s);
}

int launch_gradients(const Args &a, bool bf16_, hipStream_t s)
{
    if (a.K <= 32) return bf16_ ? gradients_kp<bf16, 1, 32>(a, s) : gradients_kp<float, 3, 32>(a, s);
    if (a.K <= 64) return bf16_ ? gradients_kp<bf16, 1, 64>(a, s) : gradients_kp<float, 3, 64>(a, s);
    return bf16_ ? gradients_kp<bf16, 1, 128>(a, s) : gradients_kp<float, 3, 128>(a, s);
}

} // namespace delta
} // namespace cawn
