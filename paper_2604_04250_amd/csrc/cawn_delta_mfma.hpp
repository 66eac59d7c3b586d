// Gated delta rule by chunks: what the kernels share.
//
// A chunk of C = 64 tokens is treated at once.  With G the running sum of the decays, D_ij = exp(G_i - G_j) for i >= j,
// N = strictly lower part of D o K K^T, P = lower part of D o Q K^T, T = (I + diag(beta) N)^-1:
//     U   = T diag(beta) (V - diag(e^G) K S0)             the u of every token, S0 the state before the chunk
//     O   = scale (diag(e^G) Q S0 + P U)
//     S_C = e^{G_C} S0 + sum_j e^{G_C - G_j} k_j u_j^T
// (the norms' factors of q and k multiply rows and columns of these and are applied there, never rounded into q and k).
//
// Matrix products run on the bf16 matrix instruction (16 x 16 x 32).  A bf16 operand is exact; an fp32 one is cut into three bf16
// planes x = x0 + x1 + x2 of 8 bits each, 24 in all, and a product takes the pairs whose planes' numbers add up to less than 3: three
// instructions for exact x fp32, six for fp32 x fp32, with the error of an fp32 product.  (The fp32 matrix instruction has a 16th of the
// bf16 one's rate.)
//
// Layout of the instruction, g = lane / 16, c = lane % 16: operands hold row (column) c and eight steps of the contraction, 8g .. 8g+7;
// the result holds column c and rows 4g .. 4g+3.  Which eight steps a lane holds is free as long as both operands agree, so two result
// tiles (rows 4g .. 4g+3 of each) are one operand of the next product, without leaving their registers.  That order -- 4g .. 4g+3 of
// the first 16 steps, then of the second -- is called the tile order below; "straight" is 8g .. 8g+7.
#pragma once
#include "cawn_delta.hpp"

namespace cawn {
namespace delta {

typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v lds_short4v;

__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

template <int N> struct Frag { bf16x8 p[N]; };      // an operand's planes, the leading one first

// acc += a b, over the pairs of planes whose numbers add up to less than S
template <int S, int NA, int NB> __device__ inline f32x4 mma(const Frag<NA> &a, const Frag<NB> &b, f32x4 acc)
{
#pragma unroll
    for (int s = S - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int j = s - i;
            if (j >= 0 && j < NB) acc = mfma(a.p[i], b.p[j], acc);
        }
    return acc;
}

// N products with a factor in common, side by side: one instruction's result is the next one's operand, so a product by itself is a
// chain of waits
template <int S, int N, int NA, int NB> __device__ inline void mma_each(const Frag<NA> (&a)[N], const Frag<NB> &b, f32x4 *acc)
{
#pragma unroll
    for (int s = S - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int j = s - i;
            if (j < 0 || j >= NB) continue;
#pragma unroll
            for (int n = 0; n < N; ++n) acc[n] = mfma(a[n].p[i], b.p[j], acc[n]);
        }
}
template <int S, int N, int NA, int NB> __device__ inline void mma_each(const Frag<NA> &a, const Frag<NB> (&b)[N], f32x4 *acc)
{
#pragma unroll
    for (int s = S - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int j = s - i;
            if (j < 0 || j >= NB) continue;
#pragma unroll
            for (int n = 0; n < N; ++n) acc[n] = mfma(a.p[i], b[n].p[j], acc[n]);
        }
}

// Pairs at a time: one conversion makes two values of a plane
typedef float f32x2 __attribute__((ext_vector_type(2)));
template <int N, int W> __device__ inline void split_pairs(const float *x, bf16 (*f)[W])
{
    static_assert(W % 2 == 0, "");
#pragma unroll
    for (int e = 0; e < W; e += 2) {
        float lo = x[e], hi = x[e + 1];
#pragma unroll
        for (int p = 0; p < N; ++p) {
            const f32x2 r = {lo, hi};
            const bf16x2 h = __builtin_convertvector(r, bf16x2);
            if (p + 1 < N) {
                const uint32_t u = __builtin_bit_cast(uint32_t, h);
                lo -= __builtin_bit_cast(float, u << 16);
                hi -= __builtin_bit_cast(float, u & 0xffff0000u);
            }
            f[p][e] = h[0], f[p][e + 1] = h[1];
        }
    }
}

template <int N> __device__ inline void split8(const float (&x)[8], Frag<N> &f)
{
    bf16 y[N][8];
    split_pairs<N, 8>(x, y);
#pragma unroll
    for (int p = 0; p < N; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) f.p[p][e] = y[p][e];
}
// four values, plane by plane
template <int N> __device__ inline void split4(f32x4 x, bf16x4 (&f)[N])
{
    const float r[4] = {x[0], x[1], x[2], x[3]};
    bf16 y[N][4];
    split_pairs<N, 4>(r, y);
#pragma unroll
    for (int p = 0; p < N; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) f[p][e] = y[p][e];
}

// two result tiles as one operand in tile order
template <int N> __device__ inline void split_tiles(f32x4 lo, f32x4 hi, Frag<N> &f)
{
    const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    split8<N>(x, f);
}

// P and T are lower triangular: of their operands (row tile, 32 columns) row tiles 0 and 1 have one that is not zero, 2 and 3 two; of the
// transpose's tiles 0 and 1 two, 2 and 3 one
__device__ inline constexpr int lower(int t, int ks) { return t < 2 ? t : 2 + (t - 2) * 2 + ks; }
__device__ inline constexpr int upper(int t, int ks) { return t < 2 ? t * 2 + ks : 2 + t; }

// T, kept as operands in tile order, three planes each: rows 16 t .., steps 32 ks .. at lower(t, ks).  A lane's 16 bytes lie at slot 16 g + (c ^ 8 (g & 1)),
// so that the columns, read transposed, come from as many banks as 8 bytes out of 16 can.
constexpr int T_BYTES = 6 * 3 * 1024;
static_assert(T_BYTES == OPERAND_BYTES, "");
__device__ inline int t_slot(int g, int c) { return (16 * g + (c ^ (g & 1) * 8)) * 16; }
__device__ inline bf16x4 read_down(const bf16 *q)      // 16 lanes fetch 4 rows of 16 and receive them transposed
{
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)q));
}
__device__ inline Frag<3> t_rows(const char *T, int t, int ks, int lane)
{
    Frag<3> f;
#pragma unroll
    for (int p = 0; p < 3; ++p) f.p[p] = *reinterpret_cast<const bf16x8 *>(T + (lower(t, ks) * 3 + p) * 1024 + t_slot(lane / 16, lane % 16));
    return f;
}
// columns 16 t .. of T (rows of its transpose), steps 32 ks ..
__device__ inline Frag<3> t_columns(const char *T, int t, int ks, int lane)
{
    const bf16x4 none = {};
    const int i = lane % 16;
    Frag<3> f;
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        const char *at = T + p * 1024 + t_slot(i % 4, 4 * (lane / 16) + i / 4) + t % 2 * 8;
        const bf16x4 a = 2 * ks >= t ? read_down(reinterpret_cast<const bf16 *>(at + lower(2 * ks, t / 2) * 3 * 1024)) : none;
        const bf16x4 b = read_down(reinterpret_cast<const bf16 *>(at + lower(2 * ks + 1, t / 2) * 3 * 1024));
        f.p[p] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    return f;
}

// 1 KiB from memory straight into LDS, 16 bytes a lane; src the lane's, dst the wave's (the same in all lanes).  Waited for with vmcnt
__device__ inline void load_piece(const char *src, char *dst)
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src, (__attribute__((address_space(3))) void *)dst, 16, 0, 0);
#else
    (void)src, (void)dst;
#endif
}

// A matrix in LDS: N planes of ROWS x (COLS + 8) bf16.  (Eight more than COLS: rows begin on 16 bytes and not all in one bank.)
template <int N, int ROWS, int COLS> struct Tile {
    static constexpr int LD = COLS + 8, PLANE = ROWS * LD, BYTES = N * PLANE * 2;
    bf16 *p;
    // row r0 + c, steps k0 + 8g ..: the contraction runs along the row
    __device__ Frag<N> straight(int r0, int k0, int lane) const
    {
        Frag<N> f;
#pragma unroll
        for (int n = 0; n < N; ++n) f.p[n] = *reinterpret_cast<const bf16x8 *>(p + n * PLANE + (r0 + lane % 16) * LD + k0 + 8 * (lane / 16));
        return f;
    }
    // the same in tile order
    __device__ Frag<N> tiled(int r0, int k0, int lane) const
    {
        Frag<N> f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const bf16 *q = p + n * PLANE + (r0 + lane % 16) * LD + k0 + 4 * (lane / 16);
            const bf16x4 a = *reinterpret_cast<const bf16x4 *>(q), b = *reinterpret_cast<const bf16x4 *>(q + 16);
            f.p[n] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
        return f;
    }
    // column m0 + c, the contraction runs down the rows
    __device__ Frag<N> straight_down(int k0, int m0, int lane) const
    {
        Frag<N> f;
        const int i = lane % 16;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const bf16 *q = p + n * PLANE + (k0 + 8 * (lane / 16) + i / 4) * LD + m0 + 4 * (i % 4);
            f.p[n] = __builtin_shufflevector(read_down(q), read_down(q + 4 * LD), 0, 1, 2, 3, 4, 5, 6, 7);
        }
        return f;
    }
    __device__ Frag<N> tiled_down(int k0, int m0, int lane) const
    {
        Frag<N> f;
        const int i = lane % 16;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const bf16 *q = p + n * PLANE + (k0 + 4 * (lane / 16) + i / 4) * LD + m0 + 4 * (i % 4);
            f.p[n] = __builtin_shufflevector(read_down(q), read_down(q + 16 * LD), 0, 1, 2, 3, 4, 5, 6, 7);
        }
        return f;
    }
};

// `rows` (of 64) rows of `cols` elements into planes, zeros beyond, in two steps, so that a chunk's rows travel while the one before is
// treated: into registers, and from there into planes.  (Lanes beyond 64 rows' units do what others do too.)
template <typename T, int N, int COLS, int NT> struct RowsAhead {
    static constexpr int U = COLS / 8, ALL = CHUNK * U, UNITS = ALL < NT ? 1 : ALL / NT;
    static_assert(ALL < NT ? NT % ALL == 0 : ALL % NT == 0, "");
    Pack<T, 8> x[UNITS];
    // What is not there is loaded from where something is, and dropped in put(): a load behind a lane's branch would be waited for.
    // rows, cols >= 1; vec: cols a multiple of 16 bytes' elements, and every row aligned to 16 bytes
    __device__ void load(int tid, const T *base, long long stride, int rows, int cols, bool vec)
    {
        constexpr int W = 16 / sizeof(T), STEP = NT / U;        // rows from one unit of a lane to its next
        if (ALL < NT) tid %= ALL;
        const long long row = stride * (long long)sizeof(T);
        if (vec && rows == CHUNK && cols == COLS && row < (1 << 24)) {
            // all there: one offset a lane, the rest the same for all
            const uint32_t at = (uint32_t)(tid / U) * (uint32_t)row + (uint32_t)(tid % U) * (8 * sizeof(T));
#pragma unroll
            for (int e = 0; e < UNITS; ++e) {
                const char *src = (const char *)base + e * STEP * row;
#pragma unroll
                for (int p = 0; p < 8 / W; ++p) *reinterpret_cast<f32x4 *>(&x[e].v[p * W]) = *reinterpret_cast<const f32x4 *>(src + at + p * 16);
            }
            return;
        }
#pragma unroll
        for (int e = 0; e < UNITS; ++e) {
            const int u = tid + e * NT, r = min(u / U, rows - 1), c = u % U * 8;
            const T *src = base + r * stride;
            if (vec) {
#pragma unroll
                for (int p = 0; p < 8 / W; ++p) *reinterpret_cast<f32x4 *>(&x[e].v[p * W]) = *reinterpret_cast<const f32x4 *>(src + min(c + p * W, cols - W));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[e].v[i] = src[min(c + i, cols - 1)];
            }
            __builtin_amdgcn_sched_barrier(0);          // (one unit at a time: single values take a register each)
        }
    }
    __device__ void put_plain(int tid, const Tile<N, CHUNK, COLS> &t, int rows, int cols)
    {
        if (ALL < NT) tid %= ALL;
        if (rows < CHUNK || cols < COLS) {              // (the same for all lanes)
#pragma unroll
            for (int e = 0; e < UNITS; ++e) {
                const int u = tid + e * NT, r = u / U, c = u % U * 8;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (r >= rows || c + i >= cols) x[e].v[i] = (T)0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < UNITS; ++e) {
            const int u = tid + e * NT, r = u / U, c = u % U * 8;
            bf16 *dst = t.p + r * Tile<N, CHUNK, COLS>::LD + c;
            if constexpr (sizeof(T) == 2) *reinterpret_cast<Pack<T, 8> *>(dst) = x[e];
            else {
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = x[e].v[i];
                Frag<N> f;
                split8<N>(y, f);
#pragma unroll
                for (int n = 0; n < N; ++n) *reinterpret_cast<bf16x8 *>(dst + n * Tile<N, CHUNK, COLS>::PLANE) = f.p[n];
            }
        }
    }
    // ... and the rows' norm factors
    __device__ void put(int tid, const Tile<N, CHUNK, COLS> &t, float *norm, int rows, int cols, bool normed, float eps)
    {
        put_plain(tid, t, rows, cols);
        factors(tid, norm, rows, COLS, normed, eps);
    }
    // (cols: of which what lies beyond has not been zeroed yet)
    __device__ void factors(int tid, float *norm, int rows, int cols, bool normed, float eps)
    {
        if (ALL < NT) tid %= ALL;
#pragma unroll
        for (int e = 0; e < UNITS; ++e) {
            const int u = tid + e * NT, r = u / U;
            if (normed) {
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) s = u % U * 8 + i < cols ? fmaf((float)x[e].v[i], (float)x[e].v[i], s) : s;
#pragma unroll
                for (int m = U / 2; m > 0; m >>= 1) s += __shfl_xor(s, m);
                if (u % U == 0) norm[r] = r < rows ? 1.f / sqrtf(s + eps) : 1.f;
            } else if (u % U == 0) norm[r] = 1.f;
        }
    }
};

// Per token of a chunk; also what later kernels find in the workspace, in this order
struct Gates {
    float gh[CHUNK], gl[CHUNK];     // G / ln 2 in two parts: exact differences, whatever the sum
    float eg[CHUNK], ed[CHUNK];     // e^G, e^{G_C - G}
    float beta[CHUNK];
    float rk[CHUNK], rq[CHUNK];     // factors of the norms
    float c[CHUNK];                 // factor of a token's row in the update of the state
    float x[CHUNK];                 // factor of k S in X: beta e^G / |k|, 0 for tokens that are not there
};

static_assert(sizeof(Gates) == GATE_FLOATS * 4, "as the workspace keeps them");

constexpr float BETA_MIN = 8.673617379884035e-19f;      // 2^-60: betas nearer to 0 count as this, so that u / beta exists

// Wave 0 fills gh, gl, eg, ed, beta of the chunk that begins at token t0 of row b, head h; `n` of its tokens exist.
__device__ inline void load_gates(const Args &a, Gates &G, int b, int h, int t0, int n)
{
    if (threadIdx.x >= CHUNK) return;
    const int i = threadIdx.x;
    const long long at = ((long long)b * a.L + t0 + i) * a.H + h;
    float g = i < n ? a.decay[at] : 0.f, beta = i < n ? a.beta[at] : 1.f;
    if (g < DECAY_MIN) g = DECAY_MIN;
    if (fabsf(beta) < BETA_MIN) beta = copysignf(BETA_MIN, beta);
    double s = g;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const double o = __shfl_up(s, m);
        if (i >= m) s += o;
    }
    const double total = __shfl(s, 63);
    const double two = s * 1.4426950408889634;
    G.gh[i] = (float)two;
    G.gl[i] = (float)(two - (double)(float)two);
    G.eg[i] = expf((float)s);
    G.ed[i] = expf((float)(total - s));
    G.beta[i] = beta;
}

__device__ inline float decay_between(const Gates &G, int i, int j)
{
    return __builtin_amdgcn_exp2f((G.gh[i] - G.gh[j]) + (G.gl[i] - G.gl[j]));
}

// (I + L)^-1 in place: L strictly lower, 64 x 64 fp32 in LDS, zeros above.  Blocks of 16 by substitution, a column a lane; then
// [[A,0],[C,B]]^-1 = [[A^-1,0],[-B^-1 C A^-1, B^-1]] twice, on the fp32 matrix instruction (16 x 16 x 4: lane c + 16 g holds step g; the
// four steps of a call are taken as 4g + s, s = 0..3, so that a result is an operand of the next).  256 threads.
constexpr int TLD = CHUNK + 4;
__device__ inline f32x4 mul16(const float *A, f32x4 B, f32x4 acc, int lane)     // A 16 x 16 in LDS, B in result layout
{
    const f32x4 a = *reinterpret_cast<const f32x4 *>(A + (lane % 16) * TLD + 4 * (lane / 16));
#pragma unroll
    for (int s = 0; s < 4; ++s) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s], B[s], acc, 0, 0, 0);
    return acc;
}
__device__ inline f32x4 tile16(const float *A, int lane)        // in result layout
{
    f32x4 x;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = A[(4 * (lane / 16) + r) * TLD + lane % 16];
    return x;
}
__device__ inline void put16(float *A, f32x4 x, int lane, float sign)
{
#pragma unroll
    for (int r = 0; r < 4; ++r) A[(4 * (lane / 16) + r) * TLD + lane % 16] = sign * x[r];
}
__device__ inline void invert(float *T, int w, int lane)         // (waves beyond the fourth only wait with the others)
{
    const int c = lane % 16;
    float *D = T + (16 * w) * TLD + 16 * w;
    float x[16];
    if (w < 4) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = i == c ? 1.f : 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            // four rows at a time (all of them at once would take 136 registers)
            f32x4 L[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e <= q; ++e) L[i][e] = *reinterpret_cast<const f32x4 *>(D + (4 * q + i) * TLD + 4 * e);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < 4 * q; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[4 * q + i] = fmaf(-L[i][j / 4][j % 4], x[j], x[4 * q + i]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = j + 1; i < 4; ++i) x[4 * q + i] = fmaf(-L[i][q][j], x[4 * q + j], x[4 * q + i]);
        }
    }
    __syncthreads();
    if (w < 4 && lane < 16) {
#pragma unroll
        for (int i = 0; i < 16; ++i) D[i * TLD + c] = x[i];
    }
    __syncthreads();
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    if (w < 2) {
        float *A = T + 32 * w * TLD + 32 * w;
        const f32x4 m = mul16(A + 16 * TLD, tile16(A, lane), zero, lane);
        put16(A + 16 * TLD, mul16(A + 16 * TLD + 16, m, zero, lane), lane, -1.f);
    }
    __syncthreads();
    const int ct = w & 1, rt = w >> 1;
    f32x4 X[2] = {zero, zero}, out = zero;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int m = 0; m < 2; ++m)
            if (m >= ct && w < 4) X[kt] = mul16(T + (32 + 16 * kt) * TLD + 16 * m, tile16(T + 16 * m * TLD + 16 * ct, lane), X[kt], lane);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
        if (kt <= rt && w < 4) out = mul16(T + (32 + 16 * rt) * TLD + 32 + 16 * kt, X[kt], out, lane);
    __syncthreads();
    if (w < 4) put16(T + (32 + 16 * rt) * TLD + 16 * ct, out, lane, -1.f);
    __syncthreads();
}

} // namespace delta
} // namespace cawn
