// Selective state space scan: what its translation units share.
//
//     delta = softplus(dt + bias),  u = delta x,  S[t] = exp(delta A) S[t-1] + u B[t],  y = (C[t] . S[t] + D x) SiLU(z)
//
// A lane owns a channel, a wave 64 of them and up to 16 of their states: B and C, which the channels share, then come by scalar loads and are
// operands of the vector instructions as they stand.  More than 16 states are shared out over the waves of a workgroup.
#pragma once
#include "cawn_sums.hpp"

namespace cawn {
namespace select {

using namespace cawn::ops;

constexpr int TILE = 16;            // tokens treated at once; the states before each tile are kept for a backward
constexpr int TOKEN_MAX = 16;       // longest call that goes token by token
constexpr int N_MAX = 128;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

typedef float f32x16 __attribute__((ext_vector_type(16)));

struct Args {
    int B, L, D, N, G, cg;          // cg: channels of a group
    int softplus;
    long long xsb, xst, dsb, dst, bsb, bst, zsb, zst, ysb, yst;
    const void *x, *dt, *Bm, *Cm, *z;
    const float *A, *Dk, *bias, *state_in;
    const int32_t *lengths;
    void *y;
    float *state_out;
    // backward
    const void *dy;
    const float *dstate_out;
    void *dx, *ddt, *dB, *dC, *dz;
    float *dstate_in;
    // Geometry of the tiled form: states of a wave (4, 8 or 16) and waves that share a channel's (1, 2, 4, 8); columns of 64 channels in a group, of which a
    // workgroup takes `wide`, and workgroups for a group; Dp = 64 x columns; tiles of a full row, segments of them
    int NP, NB, cpg, wide, cbg;
    int Dp, tiles, segments, seg_tiles;
    // B and C in fp32, padded with zeros: [b][tile][g][NPT][2][16], NPT = NP NB
    float *bc;
    // states [b][..][Dp][NPT]: before each tile (or null); of a segment from zero, its sum of delta [b][segment][Dp], and at its begin (backward:
    // what reaches its end)
    float *ck, *seg_b, *seg_g, *seg_s;
    // backward: sums over the channels of a workgroup [b][tile][16][g][parts][2][NPT], over a segment's tokens [b][segment][Dp][NPT] and, of
    // D's and the bias's gradients, [b][segment][wave of a channel][2][Dp]
    float *part_bc, *part_a, *part_d;
    int parts;
};

__device__ inline int row_length(const Args &a, int b)
{
    const int n = a.lengths ? a.lengths[b] : a.L;
    return n < 0 ? 0 : n < a.L ? n : a.L;
}

// log(1 + e^v).  With u = 1 + e rounded, log(u) e / (u - 1) corrects the rounding of u (Goldberg 1991, theorem 4).  The hardware's exponential ends at
// 2^-126, this at 2^-149: the smallest delta still meets a rate of minus infinity.
__device__ inline float softplus_f(float v)
{
    const float x = -fabsf(v) * LOG2E;
    const bool low = x < -125.f;
    const float e = __builtin_amdgcn_exp2f(low ? x + 64.f : x) * (low ? 0x1p-64f : 1.f), u = 1.f + e;
    const float l = u == 1.f ? e : __builtin_amdgcn_logf(u) * LN2 * (e * __builtin_amdgcn_rcpf(u - 1.f));
    return fmaxf(v, 0.f) + (v != v ? v : l);
}
__device__ inline float sigmoid_f(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-z * LOG2E)); }

// A's value for exp2: finite where A is.
__device__ inline float rate(float A)
{
    const float r = A * LOG2E;
    return r < -3.4028235e38f && A >= -3.4028235e38f ? -3.4028235e38f : r;
}

__device__ float mul_zero(float a, float b) __asm("llvm.amdgcn.fmul.legacy");       // v_mul_legacy_f32: 0 times anything is 0

// exp(delta A).  The product is 0 where delta is, also times minus infinity: there nothing is forgotten, and tokens that are none change nothing.
__device__ inline float factor(float delta, float A) { return __builtin_amdgcn_exp2f(mul_zero(delta, A)); }

int launch_token(const Args &a, bool bf16, hipStream_t s);
int launch_forward(const Args &a, bool bf16, hipStream_t s);
int launch_join(const Args &a, bool reverse, hipStream_t s);
int launch_backward(const Args &a, bool bf16, hipStream_t s);       // behind it launch_bc
int launch_bc_sums(const Args &a, bool bf16, hipStream_t s);

// ---------------------------------------------------------------------------------------------- the tiled kernels' common parts
// Where a wave of the tiled form is.
struct Place {
    int b, g, seg, col, blk, lane, cb;      // col: column of the group; blk: which of the channel's states; cb: workgroup of the group
    bool there, on;                         // the column exists; the lane has a channel
    int ch;                                 // channel (the group's last for lanes without one)
    long long pad;                          // place among Dp channels
};

template <bool MULTI> __device__ inline Place place_of(const Args &a)
{
    Place p;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    p.lane = threadIdx.x % 64;
    int at = blockIdx.x;
    const int cb = at % (a.cbg * a.G);
    at /= a.cbg * a.G;
    p.seg = at % a.segments, p.b = at / a.segments;
    p.g = cb / a.cbg, p.cb = cb % a.cbg;
    p.col = MULTI ? p.cb : p.cb * a.wide + w, p.blk = MULTI ? w : 0;
    p.there = p.col < a.cpg;
    const int in = min(p.col, a.cpg - 1) * 64 + p.lane;
    p.on = p.there && in < a.cg;
    p.ch = p.g * a.cg + min(in, a.cg - 1);
    p.pad = (long long)(p.g * a.cpg + min(p.col, a.cpg - 1)) * 64 + p.lane;
    return p;
}

// NP adjacent floats of an internal buffer
template <int NP> __device__ inline void load_states(const float *p, float (&s)[NP])
{
#pragma unroll
    for (int i = 0; i < NP; i += 4) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(p + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i + j] = v[j];
    }
}
template <int NP> __device__ inline void store_states(float *p, const float (&s)[NP])
{
#pragma unroll
    for (int i = 0; i < NP; i += 4) *reinterpret_cast<f32x4 *>(p + i) = f32x4{s[i], s[i + 1], s[i + 2], s[i + 3]};
}

// ... of the caller's [D][N], states n0 .. n0 + NP - 1 of channel ch, those that there are (0 for the others)
template <int NP> __device__ inline void load_user(const float *p, const Args &a, long long ch, int n0, float (&s)[NP])
{
#pragma unroll
    for (int i = 0; i < NP; ++i) s[i] = n0 + i < a.N ? p[ch * a.N + n0 + i] : 0.f;
}
template <int NP> __device__ inline void store_user(float *p, const Args &a, long long ch, int n0, const float (&s)[NP])
{
#pragma unroll
    for (int i = 0; i < NP; ++i)
        if (n0 + i < a.N) p[ch * a.N + n0 + i] = s[i];
}

template <int NP> __device__ inline void load_rates(const Args &a, const Place &p, float (&A)[NP])
{
    load_user<NP>(a.A, a, p.ch, p.blk * NP, A);
#pragma unroll
    for (int i = 0; i < NP; ++i) A[i] = rate(A[i]);
}

// Values that are ready here.  (Sums that a branch alone uses are moved behind it by the compiler, with everything that they are made of.)
template <int N> __device__ inline void stay(float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

// The 16 values of B (which = 0) or C (1) of a tile and a state, the same for all lanes: scalar loads.
typedef const __attribute__((address_space(4))) f32x16 *ScalarTile;
__device__ inline f32x16 bc_tile(const float *tile, int n, int which) { return *(ScalarTile)(uintptr_t)(tile + (n * 2 + which) * TILE); }

} // namespace select
} // namespace cawn
