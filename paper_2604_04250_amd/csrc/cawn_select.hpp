// Selective state space scan: what its translation units share.
//
//     delta = softplus(dt + bias),  u = delta x,  S[t] = exp(delta A) S[t-1] + u B[t],  y = (C[t] . S[t] + D x) SiLU(z)
//
// A lane owns a channel, a wave 64 of them and up to 16 of their states: B and C, which the channels share, then come by scalar loads and are
// operands of the vector instructions as they stand.  More than 16 states are shared out over the waves of a workgroup.
#pragma once
#include <type_traits>

#include "cawn_sums.hpp"

namespace cawn {
namespace select {

using namespace cawn::ops;

constexpr int TILE = 16;            // tokens treated at once; the states before each tile are kept for a backward
constexpr int RUN = 8;              // tokens of which the passes without gradients keep what they have read
constexpr int TOKEN_MAX = 16;       // longest call that goes token by token
constexpr int N_MAX = 128;
constexpr int SEGMENTS_MAX = 256;   // of a row
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

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
    // Geometry of the tiled form: states of a wave (4, 8, 12 or 16) and waves that share a channel's (1, 2, 4, 8); columns of 64 channels in a group, of which a
    // workgroup takes `wide`, and workgroups for a group; Dp = 64 x columns; tiles of a full row, segments of them
    int NP, NB, cpg, wide, cbg;
    int Dp, tiles, segments, seg_tiles;
    // B and C in fp32, padded with zeros: [b][tile][g][NPT][2][16], NPT = NP NB
    float *bc;
    // states [b][..][Dp][NPT]: before each tile (or null); of a segment from zero, its sum of delta [b][segment][Dp], and at its begin (backward:
    // what reaches its end)
    float *ck, *seg_b, *seg_g, *seg_s;
    // backward: sums over the channels of a workgroup [b][tile][16][g][parts][2][NPT], and over a segment's tokens of the parameters' gradients
    // [b][segment], a row of Dp NPT for A, Dp for D, Dp for the bias
    float *part_bc, *part_a;
    int parts;
};

__device__ inline int row_length(const Args &a, int b)
{
    const int n = a.lengths ? a.lengths[b] : a.L;
    return n < 0 ? 0 : n < a.L ? n : a.L;
}

// log(1 + e^v) = max(v, 0) + log(1 + e^-|v|).  u = 1 + e rounds e away; what it lost, e - (u - 1), is added to log(u) (its factor 1 / u is left out: it
// is off from 1 by e, and what was lost is 2^-24 of u at most).  The exponential is the square of the half's: the hardware's ends at 2^-126, this at 2^-149,
// so that the smallest delta still meets a rate of minus infinity.
__device__ inline float softplus_f(float v)
{
    const float half = __builtin_amdgcn_exp2f(fabsf(v) * (-0.5f * LOG2E)), e = half * half, u = 1.f + e;
    return fmaxf(v, 0.f) + fmaf(__builtin_amdgcn_logf(u), LN2, e - (u - 1.f));
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

struct ParamSums {      // column of a row of part_a -> its place in the gradients of A, D and the bias
    float *dA, *dD, *db;
    int N, NPT, Dp, cpg, cg;
    __device__ float *operator()(long long c) const
    {
        const long long wide = (long long)Dp * NPT;
        const long long pad = c < wide ? c / NPT : (c - wide) % Dp, g = pad / 64 / cpg, in = pad - g * cpg * 64;
        if (in >= cg) return nullptr;
        if (c < wide) {
            const int n = (int)(c - pad * NPT);
            return dA && n < N ? dA + (g * cg + in) * N + n : nullptr;
        }
        float *out = c - wide < Dp ? dD : db;
        return out ? out + g * cg + in : nullptr;
    }
};

// Token by token: eight states a lane, half the waves, where they are more than the chip holds at once (128 rows of 4,096 channels of 16 states: four 17.9 us,
// eight 15.8, sixteen 20); lanes of a channel.
inline int token_states(const Args &a) { return a.N > 4 && (long long)a.B * a.D * a.N >= 1 << 21 ? 8 : 4; }
inline int token_lanes(const Args &a)
{
    int lanes = 1;
    while (lanes * token_states(a) < a.N) lanes *= 2;
    return lanes;
}

int launch_token(const Args &a, bool bf16, hipStream_t s);
int launch_forward(const Args &a, bool bf16, hipStream_t s);
int launch_join(const Args &a, bool reverse, hipStream_t s);
int launch_backward(const Args &a, bool bf16, hipStream_t s);       // behind it launch_bc
int launch_bc_sums(const Args &a, bool bf16, const ParamSums &sums, int accumulate, hipStream_t s);

// f(states of a wave, waves that share a channel's), as types
template <typename F> void by_states(const Args &a, F f)
{
    auto waves = [&](auto nb) {
        if (a.NP == 12) f(std::integral_constant<int, 12>(), nb);
        else f(std::integral_constant<int, 16>(), nb);
    };
    if (a.NB == 8) waves(std::integral_constant<int, 8>());
    else if (a.NB == 4) waves(std::integral_constant<int, 4>());
    else if (a.NB == 2) waves(std::integral_constant<int, 2>());
    else if (a.NP == 8) f(std::integral_constant<int, 8>(), std::integral_constant<int, 1>());
    else if (a.NP == 4) f(std::integral_constant<int, 4>(), std::integral_constant<int, 1>());
    else waves(std::integral_constant<int, 1>());
}

// ---------------------------------------------------------------------------------------------- the tiled kernels' common parts
// Where a wave of the tiled form is.
struct Place {
    int b, g, seg, col, blk, lane, cb;      // col: column of the group; blk: which of the channel's states; cb: workgroup of the group
    bool there, on;                         // the column exists; the lane has a channel
    int ch;                                 // channel (the group's last for lanes without one)
    long long base;                         // of the group, the same for all lanes; ch = base + in
    uint32_t in;
    template <typename T> __device__ uint32_t bytes() const { return in * (uint32_t)sizeof(T); }
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
    p.base = (long long)p.g * a.cg, p.in = min(in, a.cg - 1);
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

// ... of the caller's [D][N], states n0 .. n0 + NP - 1 of channel ch, those that there are (0 for the others); four at a time where N and the address allow it
template <int NP> __device__ inline void load_user(const float *p, const Args &a, long long ch, int n0, float (&s)[NP])
{
    if (a.N % 4 == 0 && ((uintptr_t)p & 15) == 0) {
#pragma unroll
        for (int i = 0; i < NP; i += 4) {
            const f32x4 v = n0 + i < a.N ? *reinterpret_cast<const f32x4 *>(p + ch * a.N + n0 + i) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i + j] = v[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < NP; ++i) s[i] = n0 + i < a.N ? p[ch * a.N + n0 + i] : 0.f;
    }
}
template <int NP> __device__ inline void store_user(float *p, const Args &a, long long ch, int n0, const float (&s)[NP])
{
    if (a.N % 4 == 0 && ((uintptr_t)p & 15) == 0) {
#pragma unroll
        for (int i = 0; i < NP; i += 4)
            if (n0 + i < a.N) *reinterpret_cast<f32x4 *>(p + ch * a.N + n0 + i) = f32x4{s[i], s[i + 1], s[i + 2], s[i + 3]};
    } else {
#pragma unroll
        for (int i = 0; i < NP; ++i)
            if (n0 + i < a.N) p[ch * a.N + n0 + i] = s[i];
    }
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

// W values of B (which = 0) or C (1) of a tile and a state, the same for all lanes: scalar loads.
template <int W> using Scalars = float __attribute__((ext_vector_type(W)));
template <int W> __device__ inline Scalars<W> bc_run(const float *tile, int n, int which)
{
    typedef const __attribute__((address_space(4))) Scalars<W> *At;
    return *(At)(uintptr_t)(tile + (n * 2 + which) * TILE);
}

// A stream's rows of W tokens from `row` on: the tokens' places are scalar, the lane's 32 bits of bytes, as buffer instructions take them.  (From pointers
// the compiler adds the lane's place first and walks along the tokens with vector instructions.)  The resource ends nowhere: the callers' bounds count.
__device__ inline __amdgpu_buffer_rsrc_t rows_at(const void *row) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(row), 0, -1, 0x00020000); }
// A value as it comes, in a register of its own (of values of 16 bits the compiler would put two in one, which costs instructions), and what it is.
template <typename T> __device__ inline uint32_t load_at(__amdgpu_buffer_rsrc_t r, uint32_t lane, uint32_t token)
{
    if constexpr (sizeof(T) == 2) return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, lane, token, 0);
    else return __builtin_amdgcn_raw_buffer_load_b32(r, lane, token, 0);
}
template <typename T> __device__ inline float value(uint32_t raw) { return __uint_as_float(sizeof(T) == 2 ? raw << 16 : raw); }
template <typename T> __device__ inline void store_at(__amdgpu_buffer_rsrc_t r, uint32_t lane, uint32_t token, float v)
{
    const T x = (T)v;
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, x), r, lane, token, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, x), r, lane, token, 0);
}

// W tokens of a stream, of which `left` are there (the last of them again for the others); step: of a token, in bytes
template <typename T, int W> __device__ inline void load_run(const T *row, uint32_t step, int left, uint32_t lane, uint32_t (&v)[W])
{
    const auto r = rows_at(row);
    uint32_t token = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        v[i] = load_at<T>(r, lane, token);
        token += i + 1 < left ? step : 0;
    }
}

// Nothing: values that a branch leaves alone would be kept from the round before.
template <int W> __device__ inline void no_run(uint32_t (&v)[W])
{
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = 0;
}

// ... of an output, from f(i)
template <typename T, int W, typename F> __device__ inline void store_run(T *row, uint32_t step, int left, uint32_t lane, F f)
{
    const auto r = rows_at(row);
    uint32_t token = 0;
#pragma unroll
    for (int i = 0; i < W; ++i, token += step)
        if (i < left) store_at<T>(r, lane, token, f(i));
}

} // namespace select
} // namespace cawn
