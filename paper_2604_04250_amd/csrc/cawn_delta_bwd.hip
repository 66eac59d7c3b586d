// Gated delta rule by chunks, backward.
//
// With dS the gradient of the state behind a chunk, dO that of its output, and the forward's S0 and U from the checkpoint:
//     dR  = T^T (scale P^T dO + KD dS),  KD = diag(e^{G_C - G}) K      gradient of U through everything but T's inverse; dV = beta dR
//     dS0 = e^{G_C} dS + scale (e^G Q)^T dO - (beta e^G K)^T dR
//     Z   = scale (dO U^T) o D (lower),  M = -(beta dR U^T) o D (strictly lower)
//     dQ  = scale e^G dO S0^T + Z K
//     dK  = -beta e^G dR S0^T + M K + Z^T Q + M^T K + e^{G_C - G} U dS^T
//     dbeta_i = dR_i . U_i / beta_i
//     ddecay_t = sum_{i >= t, in the chunk} (q_i . dq_i - v_i . dv_i) + <dS, S_C>
// The last line: a decay scales all that a later query reads and all that came before it; summed over the places where e^{G_i} stands
// (queries, keys that read, keys that write) the keys' two shares meet in dR.U and cancel, and what is left is the above.
//
// dR and dS come from the recurrence (delta_back); here every chunk is a workgroup.
#include <stddef.h>

#include "cawn_delta_mfma.hpp"

namespace cawn {
namespace delta {

// Gradients of a chunk.  A workgroup takes all value heads of a key head, one after the other, and keeps dq and dk in registers: wave w
// rows 16 w .. of them.  First everything that runs over the value columns, 32 at a time, with U, dR, S0 and dS in LDS as they come
// from their tiles (a tile's lane holds four rows of a column: a matrix is kept as its transpose, and read down); then, in the same
// LDS, Z and M with q and k.
// dq carries ddecay and takes full precision; dk of a bf16 call takes two planes (16 bits) of its operands.
template <typename T, int NP, int KP> struct GradLds {
    static constexpr int PK = NP == 1 ? 2 : 3;          // planes of what only dk needs
    using MatU = Tile<3, 32, 64>;
    using MatR = Tile<3, 32, 64>;
    using MatS = Tile<3, 32, KP>;
    using MatD = Tile<PK, 32, KP>;
    using MatO = Tile<NP, CHUNK, 32>;
    using MatQ = Tile<NP, CHUNK, KP>;
    using MatZ = Tile<3, CHUNK, CHUNK>;
    using MatM = Tile<PK, CHUNK, CHUNK>;
    static constexpr int FIRST = MatU::BYTES + MatR::BYTES + MatS::BYTES + MatD::BYTES + MatO::BYTES;
    static constexpr int SECOND = 2 * MatQ::BYTES + MatZ::BYTES + MatM::BYTES;
    static constexpr int BYTES = FIRST > SECOND ? FIRST : SECOND;
    static constexpr int HELD = 163840 / (BYTES + 4096), WAVES = HELD > 2 ? 2 : HELD;     // waves a SIMD: as many workgroups as the LDS holds, two at most
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
template <typename T, int NP, int KP, bool SHARED> __global__ __launch_bounds__(256, (GradLds<T, NP, KP>::WAVES)) void delta_gradients(const Args a)
{
    using L = GradLds<T, NP, KP>;
    constexpr int KT = KP / 16, PK = L::PK, OWN = (KT + 3) / 4;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ Gates G;
    __shared__ float qdq[CHUNK], vdv[CHUNK], udr[CHUNK], part[4];
    const int blk = blockIdx.x, n = blk % a.chunks, bk = blk / a.chunks, hk = bk % a.Hk, b = bk / a.Hk, rep = a.H / a.Hk;
    const int len = row_length(a, b), t0 = n * CHUNK, rows = min(CHUNK, len - t0), all = min(CHUNK, a.L - t0);
    const long long qat = b * a.qsb + t0 * a.qst + (long long)hk * a.K;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    int tid = threadIdx.x, lane = tid % 64, g = lane / 16, c = lane % 16;
    auto anew = [&]() {                         // (as in delta_scan)
        tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        lane = tid % 64, g = lane / 16, c = lane % 16;
    };
    if (rows <= 0) {                            // tokens that the row does not have
        for (int i = threadIdx.x; i < all * a.K; i += 256) {
            const long long at = qat + (long long)(i / a.K) * a.qst + i % a.K;
            if (a.dq) ((T *)a.dq)[at] = (T)0.f;
            if (a.dk) ((T *)a.dk)[at] = (T)0.f;
        }
        for (int hh = 0; hh < rep; ++hh) {
            const int h = hk * rep + hh;
            if (a.dv)
                for (int i = threadIdx.x; i < all * a.V; i += 256) ((T *)a.dv)[b * a.vsb + (t0 + i / a.V) * a.vst + (long long)h * a.V + i % a.V] = (T)0.f;
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
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    f32x4 dq[KT], dk[KT];
    if (SHARED) {
#pragma unroll
        for (int t = 0; t < KT; ++t) dq[t] = dk[t] = zero;
    }
    for (int hh = 0; hh < (SHARED ? rep : 1); ++hh) {
        const int h = hk * rep + hh, bh = b * a.H + h;
        const size_t at = (size_t)bh * a.chunks + n;
        const char *sp = a.s_tiles + bh * a.s_row + n * a.s_chunk, *up = a.u_tiles + bh * a.u_row + n * a.u_chunk;
        const char *rp = a.dr_tiles + at * z.ut * 1024, *dp = a.ds_tiles + at * z.st * 1024;
        __syncthreads();                        // the previous head's LDS
        anew();
        f32x4 A1[KT], A2[KT], A3[KT], zt[4], mt[4];
#pragma unroll
        for (int t = 0; t < KT; ++t) A1[t] = A2[t] = A3[t] = zero;
#pragma unroll
        for (int t = 0; t < 4; ++t) zt[t] = mt[t] = zero;
        float inner = 0.f;                      // <dS, S_C>
        float sv[4] = {0.f, 0.f, 0.f, 0.f}, su[4] = {0.f, 0.f, 0.f, 0.f};
        // A step's loads are all under way before the first is wanted: tiles, and (from where something is, and dropped below) v and dO.
        // Wave w: row tile w of U and dR; row tiles w, w + 4 of the states
        f32x4 tu[2], tr[2], ts[OWN][2], te[OWN][2], td[OWN][2];
        T tv[2][4];
        RowsAhead<T, NP, 32, 256> to;
        RowsAhead<T, NP, KP, 256> qa, ka;
        auto ahead = [&](int v0) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int vt = min(v0 / 16 + half, a.VT - 1), v = min(16 * vt + c, a.V - 1);
                tu[half] = *reinterpret_cast<const f32x4 *>(up + ((size_t)w * a.VT + vt) * 1024 + lane * 16);
                tr[half] = *reinterpret_cast<const f32x4 *>(rp + ((size_t)w * a.VT + vt) * 1024 + lane * 16);
#pragma unroll
                for (int o = 0; o < OWN; ++o) {
                    const size_t at = ((size_t)min(w + 4 * o, KT - 1) * a.VT + vt) * 1024 + lane * 16;
                    ts[o][half] = *reinterpret_cast<const f32x4 *>(sp + at);
                    te[o][half] = *reinterpret_cast<const f32x4 *>(sp + a.s_chunk + at);
                    td[o][half] = *reinterpret_cast<const f32x4 *>(dp + at);
                }
                const T *vp = (const T *)a.v + b * a.vsb + (long long)t0 * a.vst + (long long)h * a.V + v;
#pragma unroll
                for (int e = 0; e < 4; ++e) tv[half][e] = vp[min(16 * w + 4 * g + e, rows - 1) * a.vst];
            }
            to.load(tid, (const T *)a.dO + b * a.osb + (long long)t0 * a.ost + (long long)h * a.V + v0, a.ost, rows, min(32, a.V - v0), a.veco);
        };
        ahead(0);
        for (int i = tid; i < GATE_FLOATS; i += 256) ((float *)&G)[i] = a.gates[at * GATE_FLOATS + i];
        for (int v0 = 0; v0 < a.V; v0 += 32) {
            __syncthreads();
            anew();
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int vt = v0 / 16 + half, v = 16 * vt + c;
                const bool there = vt < a.VT;
                const f32x4 u = there ? tu[half] : zero, r = there ? tr[half] : zero;
                put_column(ut, 16 * half + c, 16 * w + 4 * g, u);
                put_column(rt, 16 * half + c, 16 * w + 4 * g, r);
                T *dvp = (T *)a.dv + b * a.vsb + (long long)t0 * a.vst + (long long)h * a.V + v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 16 * w + 4 * g + e;
                    su[e] += u[e] * r[e];
                    const float dv = G.beta[i] * r[e];
                    sv[e] += v < a.V && i < rows ? (float)tv[half][e] * dv : 0.f;
                    if (a.dv && v < a.V && i < all) dvp[i * a.vst] = (T)(i < rows ? dv : 0.f);
                }
#pragma unroll
                for (int o = 0; o < OWN; ++o) {
                    const int t = w + 4 * o;
                    if (t >= KT) break;
                    const f32x4 s = there ? ts[o][half] : zero, d = there ? td[o][half] : zero;
                    put_column(st, 16 * half + c, 16 * t + 4 * g, s);
                    put_column(dt, 16 * half + c, 16 * t + 4 * g, d);
#pragma unroll
                    for (int x = 0; x < 4; ++x) inner += d[x] * te[o][half][x];
                }
            }
            to.put_plain(tid, ot, rows, min(32, a.V - v0));
            __syncthreads();
            if (v0 + 32 < a.V) ahead(v0 + 32);
            else {                              // the second half's
                qa.load(tid, (const T *)a.q + qat, a.qst, rows, a.K, a.vecq);
                ka.load(tid, (const T *)a.k + qat, a.qst, rows, a.K, a.vecq);
            }
            anew();
            const Frag<NP> o = ot.straight(16 * w, 0, lane);
            const Frag<3> r = rt.straight_down(0, 16 * w, lane);
            Frag<PK> u;
            {
                const Frag<3> u3 = ut.straight_down(0, 16 * w, lane);
#pragma unroll
                for (int p = 0; p < PK; ++p) u.p[p] = u3.p[p];
            }
            // before their factors: Z^T and M^T, rows j and column i = c of row tile w; dO S0^T and the like, rows f and column i = c
#pragma unroll
            for (int j0 = 0; j0 < 4; j0 += 2) {         // (two at a time: registers)
                if (j0 > w) break;
                Frag<3> uj[2];
#pragma unroll
                for (int jt = 0; jt < 2; ++jt) uj[jt] = ut.straight_down(0, 16 * (j0 + jt), lane);
                mma_each<3>(uj, o, zt + j0);            // (one beyond row tile w: it is masked below)
                mma_each<PK>(uj, r, mt + j0);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int t0 = 0; t0 < KT; t0 += 2) {
                Frag<3> f[2];
                Frag<PK> d[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) f[t] = st.straight_down(0, 16 * (t0 + t), lane), d[t] = dt.straight_down(0, 16 * (t0 + t), lane);
                mma_each<3>(f, o, A1 + t0);
                mma_each<PK>(f, r, A2 + t0);
                mma_each<PK>(d, u, A3 + t0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float s = row_sum(sv[e]), t = row_sum(su[e]);
            if (c == 0) vdv[16 * w + 4 * g + e] = s, udr[16 * w + 4 * g + e] = t;
        }
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) inner += __shfl_xor(inner, m);
        if (lane == 0) part[w] = inner;
        __syncthreads();                        // the LDS of the first half is free
        anew();
        qa.put_plain(tid, qm, rows, a.K);
        ka.put_plain(tid, km, rows, a.K);
        const int i = 16 * w + c;               // the lane's token from here on
        const float eg = G.eg[i], beta = G.beta[i], rk = G.rk[i], rq = G.rq[i], sq = a.scale * rq, bk = -beta * rk;
#pragma unroll
        for (int jt = 0; jt < 4; ++jt) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = 16 * jt + 4 * g + r;
                const float D = i >= j ? G.rk[j] * decay_between(G, i, j) : 0.f;
                zt[jt][r] = i >= j ? zt[jt][r] * (sq * D) : 0.f;
                mt[jt][r] = i > j ? mt[jt][r] * (bk * D) : 0.f;
            }
            put_column(zm, i, 16 * jt + 4 * g, zt[jt]);         // (here the column of the transpose is the row)
            put_column(mm, i, 16 * jt + 4 * g, mt[jt]);
        }
        // y = r dx^ of the norm's x^ = r x:  yq = scale rq e^G A1 + Z k,  yk = rk (e^{G_C - G} A3 - beta e^G A2) + M k + Z^T q + M^T k
        const float f1 = sq * eg, f2 = bk * eg, f3 = rk * G.ed[i];
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            A1[t] *= f1;
            A2[t] = f3 * A3[t] + f2 * A2[t];
        }
        __syncthreads();
        anew();
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            constexpr int AT = KT < 4 ? KT : 4;
            const bool left = 2 * ks <= w, right = 2 * ks + 1 >= w;
            Frag<3> zf, zd;
            Frag<PK> mf, md;
            if (left) zf = zm.straight(16 * w, 32 * ks, lane), mf = mm.straight(16 * w, 32 * ks, lane);
            if (right) zd = zm.straight_down(32 * ks, 16 * w, lane), md = mm.straight_down(32 * ks, 16 * w, lane);
#pragma unroll
            for (int t0 = 0; t0 < KT; t0 += AT) {
                Frag<NP> kf[AT], qf[AT];
#pragma unroll
                for (int t = 0; t < AT; ++t) kf[t] = km.straight_down(32 * ks, 16 * (t0 + t), lane);
                if (left) {
                    mma_each<3>(kf, zf, A1 + t0);
                    mma_each<PK>(kf, mf, A2 + t0);
                }
                if (right) {
#pragma unroll
                    for (int t = 0; t < AT; ++t) qf[t] = qm.straight_down(32 * ks, 16 * (t0 + t), lane);
                    mma_each<PK>(qf, zd, A2 + t0);
                    mma_each<PK>(kf, md, A2 + t0);
                }
            }
        }
        anew();
        // q^ . dq^ of this head = q . yq
        {
            float s = 0.f;
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                float x[4];
                row_of(qm, 16 * w + c, 16 * t + 4 * g, x);
#pragma unroll
                for (int r = 0; r < 4; ++r) s = fmaf(x[r], A1[t][r], s);
                dq[t] = SHARED ? dq[t] + A1[t] : A1[t];
                dk[t] = SHARED ? dk[t] + A2[t] : A2[t];
            }
            s += __shfl_xor(s, 16);
            s += __shfl_xor(s, 32);
            if (g == 0) qdq[16 * w + c] = s;
        }
        __syncthreads();
        if (tid < CHUNK) {
            const int i = tid;
            float s = i < rows ? qdq[i] - vdv[i] : 0.f;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) {          // sum over the tokens behind
                const float o = __shfl_down(s, m);
                if (i + m < 64) s += o;
            }
            s += (part[0] + part[1]) + (part[2] + part[3]);
            if (i < all) {
                const long long at = ((long long)b * a.L + t0 + i) * a.H + h;
                // (a complete forgetting hangs on nothing; the sum would leave its rounding)
                if (a.ddecay) a.ddecay[at] = i < rows && !(a.decay[at] < DECAY_MIN) ? s : 0.f;
                if (a.dbeta) a.dbeta[at] = i < rows ? udr[i] / G.beta[i] : 0.f;
            }
        }
    }
    // through the norm, and out: dx = r (dx^ - x^ (x^ . dx^)) = y - r^2 x (x . y)
    const int i = 16 * w + c;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (!(which ? a.dk : a.dq)) continue;
        const typename L::MatQ &xm = which ? km : qm;
        T *out = (T *)(which ? a.dk : a.dq) + qat + (long long)i * a.qst + 4 * g;
        float x[KT][4], s = 0.f;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            row_of(xm, i, 16 * t + 4 * g, x[t]);
#pragma unroll
            for (int r = 0; r < 4; ++r) s = fmaf(x[t][r], which ? dk[t][r] : dq[t][r], s);
        }
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        const float f = which ? G.rk[i] : G.rq[i];
        s = a.norm ? -s * f * f : 0.f;
        if (i >= all) continue;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            float y[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = i < rows ? fmaf(x[t][r], s, which ? dk[t][r] : dq[t][r]) : 0.f;
            if (a.vecd && 16 * t + 4 * g + 4 <= a.K) store_n<T, 4>(out + 16 * t, y);
            else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (16 * t + 4 * g + r < a.K) out[16 * t + r] = (T)y[r];
            }
        }
    }
}

template <typename T, int NP, int KP, bool SHARED> static int gradients_of(const Args &a, hipStream_t s)
{
    constexpr int bytes = GradLds<T, NP, KP>::BYTES;
    static_assert(bytes + sizeof(Gates) + 1024 <= 163840, "LDS");
    if (a.chunks == 0) return CAWN_OK;
    if (hipFuncSetAttribute((const void *)delta_gradients<T, NP, KP, SHARED>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return CAWN_ELAUNCH;
    hipLaunchKernelGGL((delta_gradients<T, NP, KP, SHARED>), dim3((unsigned)((long long)a.B * a.Hk * a.chunks)), dim3(256), bytes, s, a);
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
