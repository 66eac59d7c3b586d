// Short causal convolution along the tokens with an activation, channels last, forward and backward.
//
// Forward: z[t] = bias + sum_i w[i] x[t-(k-1)+i], y = act(z).
// Backward: dz = dy act'(z) with z made again, dx[t] = sum_i w[k-1-i] dz[t+i], dw[i] = sum_t dz[t] x[t-(k-1)+i], db = sum_t dz[t].
//
// A thread takes four adjacent channels along a run of tokens; the k - 1 inputs before the run's first token are read again, and backward the k - 1 tokens behind
// its last.  Bound by memory: 8 x 8,192 tokens of 768 channels in bf16 forward 38 us (5.2 TB/s), backward 70 (4.3: also what it computes, z and two products a
// tap, two thirds of the issue slots), the sums of dw 5.  A step of 128 rows of 4,096 channels 5.6.  (Two channels a thread, both directions: 119 us, eight 151.)
// The row's state (the k - 1 inputs before its first token, in fp32) is read and replaced by the thread of the row's first run alone.
#include "cawn_rows.hpp"
#include "cawn_sums.hpp"

using namespace cawn::ops;

namespace {

constexpr int K_MAX = 4;
constexpr int U = 2;            // tokens at a time, the next ones on their way

struct ConvArgs {
    const void *x, *dy;
    const float *w, *bias, *state_in, *dstate_out;
    const int32_t *lengths;
    void *y, *dx;
    float *state_out, *dstate_in, *part;
    int B, L, C, act;
    long long xsb, xst, ysb, yst;
    int units;              // of VEC channels in a row
    int run;                // tokens of a run
    long long runs;         // of a row
    int ub, rb, ublocks;    // backward: units and runs of a workgroup, workgroups side by side
    long long rblocks;
};

__device__ inline int row_length(const ConvArgs &a, int b)
{
    const int n = a.lengths ? a.lengths[b] : a.L;
    return n < 0 ? 0 : n < a.L ? n : a.L;
}

__device__ inline float sigmoid_f(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

template <int K, int VEC> struct Taps {
    float w[K][VEC], b[VEC];
    __device__ Taps(const ConvArgs &a, int c)
    {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
#pragma unroll
            for (int i = 0; i < K; ++i) w[i][j] = a.w[(long long)(c + j) * K + i];
            b[j] = a.bias ? a.bias[c + j] : 0.f;
        }
    }
};

// VEC channels of row `at` of a state [B][K - 1][C]
template <int K, int VEC> __device__ inline void load_state(const ConvArgs &a, const float *p, long long b, int at, int c, float (&x)[VEC])
{
    p += (b * (K - 1) + at) * a.C + c;
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] = p[j];
}
template <int K, int VEC> __device__ inline void store_state(const ConvArgs &a, float *p, long long b, int at, int c, int skip, const float (&x)[VEC])
{
    p += (b * (K - 1) + at) * a.C + c;
#pragma unroll
    for (int j = 0; j < VEC; ++j)
        if (j >= skip) p[j] = x[j];
}

// Input `back` (1 .. K - 1) places before the row's first token
template <int K, int VEC> __device__ inline void before_row(const ConvArgs &a, int b, int back, int c, float (&x)[VEC])
{
    if (a.state_in) load_state<K, VEC>(a, a.state_in, b, K - 1 - back, c, x);
    else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[j] = 0.f;
    }
}

// U tokens' values from token t on, those below `end`; what is not there is the row's last again (a load behind a lane's branch would be waited for by
// itself) and is left out where it is used
template <typename T, int VEC> __device__ inline void fetch(const T *row, long long stride, int t, int end, Loose<T, VEC> (&v)[U])
{
#pragma unroll
    for (int i = 0; i < U; ++i) v[i] = *reinterpret_cast<const Loose<T, VEC> *>(row + min(t + i, end - 1) * stride);
}

template <typename T, int VEC> __device__ inline void widen(const Loose<T, VEC> &v, float (&x)[VEC])
{
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] = (float)v.v[j];
}

template <typename T, int K, int VEC, bool TAIL> __global__ __launch_bounds__(256) void conv_forward(const ConvArgs a)
{
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x, rest = id / a.units;
    const Unit<VEC, TAIL> u((int)(id - rest * a.units), a.C);
    const int c = u.c, skip = u.skip;
    const long long bl = rest / a.runs;
    if (bl >= a.B) return;
    const int b = (int)bl, t0 = (int)(rest - bl * a.runs) * a.run, end = min(a.L, t0 + a.run);
    const T *x = (const T *)a.x + b * a.xsb + c;
    T *y = (T *)a.y + b * a.ysb + c;
    // (what does not depend on the row's length first: a single token's call is a chain of two loads and a store)
    const Taps<K, VEC> p(a, c);
    float win[K - 1 + U][VEC];          // the inputs that U tokens see
    if (t0 == 0) {
#pragma unroll
        for (int i = 0; i < K - 1; ++i) before_row<K, VEC>(a, b, K - 1 - i, c, win[i]);
    }
    const int n = row_length(a, b), t1 = min(n, t0 + a.run);
    Loose<T, VEC> next[U];
    if (t0 < t1) {
        fetch<T, VEC>(x, a.xst, t0, t1, next);
        if (t0 > 0) {
#pragma unroll
            for (int i = 0; i < K - 1; ++i) read_n<T, VEC>(x + (t0 - (K - 1) + i) * a.xst, win[i]);
        }
    }
    if (t0 == 0 && K > 1 && a.state_out) {
        // the last K - 1 of what came before and the row's own; all is read before any is written
        float s[K > 1 ? K - 1 : 1][VEC];
#pragma unroll
        for (int i = 0; i < K - 1; ++i) {
            const int t = n - (K - 1) + i;
            if (t >= 0) read_n<T, VEC>(x + t * a.xst, s[i]);
            else before_row<K, VEC>(a, b, -t, c, s[i]);
        }
#pragma unroll
        for (int i = 0; i < K - 1; ++i) store_state<K, VEC>(a, a.state_out, b, i, c, skip, s[i]);
    }
    for (int t = t0; t < t1; t += U) {
#pragma unroll
        for (int i = 0; i < U; ++i) widen<T, VEC>(next[i], win[K - 1 + i]);
        if (t + U < t1) fetch<T, VEC>(x, a.xst, t + U, t1, next);
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (t + k >= t1) break;
            float z[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                z[j] = p.b[j];
#pragma unroll
                for (int i = 0; i < K; ++i) z[j] = fmaf(p.w[i][j], win[k + i][j], z[j]);
                if (a.act) z[j] *= sigmoid_f(z[j]);
            }
            write_n<T, VEC>(y + (t + k) * a.yst, z, skip);
        }
#pragma unroll
        for (int i = 0; i < K - 1; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) win[i][j] = win[U + i][j];
    }
    for (int t = max(t0, n); t < end; ++t) {
        const float z[VEC] = {};
        write_n<T, VEC>(y + t * a.yst, z, skip);
    }
}

// dz of token t of the row, from the inputs that it sees
template <int K, int VEC> __device__ inline void slope(const ConvArgs &a, const Taps<K, VEC> &p, const float (*win)[VEC], const float (&dy)[VEC], float (&dz)[VEC])
{
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        dz[j] = dy[j];
        if (a.act) {
            float z = p.b[j];
#pragma unroll
            for (int i = 0; i < K; ++i) z = fmaf(p.w[i][j], win[i][j], z);
            const float f = sigmoid_f(z);
            dz[j] *= f * fmaf(z, 1.f - f, 1.f);
        }
    }
}

template <typename T, int K, int VEC, bool TAIL> __global__ __launch_bounds__(256) void conv_backward(const ConvArgs a)
{
    __shared__ float sh[(K + 1) * VEC * 256];
    const int unit = threadIdx.x % a.ub, row = threadIdx.x / a.ub;
    const long long rblk = blockIdx.x / a.ublocks;
    const Unit<VEC, TAIL> u((int)(blockIdx.x - rblk * a.ublocks) * a.ub + unit, a.C);
    const int c = u.c, skip = u.skip;
    const Taps<K, VEC> p(a, c);
    float dw[K][VEC], db[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        db[j] = 0.f;
#pragma unroll
        for (int i = 0; i < K; ++i) dw[i][j] = 0.f;
    }
    const long long all = a.runs * a.B;
    for (long long rr = rblk * a.rb + row; u.in && row < a.rb && rr < all; rr += a.rblocks * a.rb) {
        const int b = (int)(rr / a.runs), n = row_length(a, b);
        const int t0 = (int)(rr - b * a.runs) * a.run, t1 = min(n, t0 + a.run), end = min(a.L, t0 + a.run);
        const T *x = (const T *)a.x + b * a.xsb + c, *dyp = (const T *)a.dy + b * a.ysb + c;
        T *dx = a.dx ? (T *)a.dx + b * a.xsb + c : nullptr;
        Loose<T, VEC> xn[U], dn[U];
        if (t0 < t1) fetch<T, VEC>(x, a.xst, t0, n, xn), fetch<T, VEC>(dyp, a.yst, t0, n, dn);
        float win[K - 1 + U][VEC], dzs[K - 1 + U][VEC];         // the inputs that U tokens see; their dz and the K - 1 before them
#pragma unroll
        for (int i = 0; i < K - 1; ++i) {
            const int t = t0 - (K - 1) + i;
#pragma unroll
            for (int j = 0; j < VEC; ++j) dzs[i][j] = win[i][j] = 0.f;
            if (t0 >= t1) continue;
            if (t >= 0) read_n<T, VEC>(x + t * a.xst, win[i]);
            else before_row<K, VEC>(a, b, -t, c, win[i]);
        }
        // up to K - 1 tokens behind the run: the gradients of its last inputs need their dz
        const bool first = K > 1 && t0 == 0 && a.dstate_in;             // the state's gradient too, which lies before the row
        const int stop = t0 < t1 || first ? t1 + K - 1 : t0;
        for (int t = t0; t < stop; t += U) {
            float dy[U][VEC];
#pragma unroll
            for (int i = 0; i < U; ++i) widen<T, VEC>(xn[i], win[K - 1 + i]), widen<T, VEC>(dn[i], dy[i]);
            if (t + U < min(stop, n)) fetch<T, VEC>(x, a.xst, t + U, n, xn), fetch<T, VEC>(dyp, a.yst, t + U, n, dn);
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (t + k < n && t + k < stop) slope<K, VEC>(a, p, &win[k], dy[k], dzs[K - 1 + k]);
                else {
#pragma unroll
                    for (int j = 0; j < VEC; ++j) dzs[K - 1 + k][j] = 0.f;
                }
                if (t + k < t1) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        db[j] += dzs[K - 1 + k][j];
#pragma unroll
                        for (int i = 0; i < K; ++i) dw[i][j] = fmaf(dzs[K - 1 + k][j], win[k + i][j], dw[i][j]);
                    }
                }
                const int at = t + k - (K - 1);         // its dz have all come
                if (at < t1 && (at >= t0 ? dx != nullptr : first)) {
                    float d[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        d[j] = 0.f;
#pragma unroll
                        for (int i = 0; i < K; ++i) d[j] = fmaf(p.w[K - 1 - i][j], dzs[k + i][j], d[j]);
                    }
                    const int left = at - (n - (K - 1));
                    if (K > 1 && a.dstate_out && left >= 0) {           // it is part of the state behind the row
                        float e[VEC];
                        load_state<K, VEC>(a, a.dstate_out, b, left, c, e);
#pragma unroll
                        for (int j = 0; j < VEC; ++j) d[j] += e[j];
                    }
                    if (at >= 0) write_n<T, VEC>(dx + at * a.xst, d, skip);
                    else store_state<K, VEC>(a, a.dstate_in, b, at + K - 1, c, skip, d);
                }
            }
#pragma unroll
            for (int i = 0; i < K - 1; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) win[i][j] = win[U + i][j], dzs[i][j] = dzs[U + i][j];
        }
        if (dx) {
            for (int t = max(t0, n); t < end; ++t) {
                const float z[VEC] = {};
                write_n<T, VEC>(dx + t * a.xst, z, skip);
            }
        }
    }
    if (!a.part) return;
    // [K + 1][C] a workgroup
    float sums[(K + 1) * VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
#pragma unroll
        for (int i = 0; i < K; ++i) sums[i * VEC + j] = dw[i][j];
        sums[K * VEC + j] = db[j];
    }
    over_runs<256>(sums, a.rb, a.ub, sh);
    if (row > 0 || !u.in) return;
#pragma unroll
    for (int i = 0; i <= K; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (j >= skip) a.part[(rblk * (K + 1) + i) * a.C + c + j] = sums[i * VEC + j];
}

// The gradient of the state before the row alone, where it takes the place of that behind the row, which the other workgroups read: what its first
// K - 1 tokens make of it, and what of it is still there behind the last.  Beyond STATE_BLOCKS workgroups they go round.
constexpr long long STATE_BLOCKS = 1 << 16;

template <typename T, int K, int VEC, bool TAIL> __global__ __launch_bounds__(256) void conv_state_backward(const ConvArgs a)
{
    for (long long id = (long long)blockIdx.x * 256 + threadIdx.x, all = (long long)a.B * a.units; id < all; id += (long long)gridDim.x * 256) {
        const long long b = id / a.units;
        const Unit<VEC, TAIL> u((int)(id - b * a.units), a.C);
        const int c = u.c, n = row_length(a, (int)b);
        const Taps<K, VEC> p(a, c);
        float d[K][VEC], dz[K][VEC], win[K][VEC];
#pragma unroll
        for (int i = 1; i < K; ++i) before_row<K, VEC>(a, (int)b, K - i, c, win[i]);
#pragma unroll
        for (int t = 0; t < K - 1; ++t) {
            float dy[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) dz[t][j] = 0.f;
            if (t >= n) continue;
#pragma unroll
            for (int i = 0; i + 1 < K; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) win[i][j] = win[i + 1][j];
            read_n<T, VEC>((const T *)a.x + b * a.xsb + t * a.xst + c, win[K - 1]);
            read_n<T, VEC>((const T *)a.dy + b * a.ysb + t * a.yst + c, dy);
            slope<K, VEC>(a, p, win, dy, dz[t]);
        }
        // (the sum in the order of the other kernel, whose bits these are)
#pragma unroll
        for (int s = 0; s < K - 1; ++s)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                d[s][j] = 0.f;
#pragma unroll
                for (int t = 0; t <= s; ++t) d[s][j] = fmaf(p.w[s - t][j], dz[t][j], d[s][j]);
                if (a.dstate_out && s >= n) d[s][j] += a.dstate_out[(b * (K - 1) + (s - n)) * a.C + c + j];
            }
#pragma unroll
        for (int i = 0; i < K - 1; ++i) store_state<K, VEC>(a, a.dstate_in, b, i, c, u.skip, d[i]);
    }
}

struct TapSums {        // column (i, c) of a part's [K + 1][C]
    float *dw, *db;
    int C, K;
    __device__ float *operator()(long long at) const
    {
        const int i = (int)(at / C), c = (int)(at - (long long)i * C);
        return i < K ? (dw ? dw + (long long)c * K + i : nullptr) : (db ? db + c : nullptr);
    }
};

// ---------------------------------------------------------------------------------------------- host
struct Plan {
    ConvArgs a;
    int vec, k;
    long long blocks;
};

int plan_of(const cawn_conv_desc *d, bool bwd, Plan *p)
{
    if (!d || d->B < 0 || d->L < 0 || d->C <= 0 || d->k <= 0 || d->act < 0 || d->act > 1 || (d->bf16 & ~1) || d->reserved) return CAWN_EINVAL;
    if (d->k > K_MAX || d->L > 1 << 30 || d->C > 1 << 30) return CAWN_EUNSUPPORTED;        // (places of tokens and channels, and of a run behind them, in 32 bits)
    ConvArgs &a = p->a;
    a = ConvArgs{};
    a.B = d->B, a.L = d->L, a.C = d->C, a.act = d->act, p->k = d->k;
    a.xst = d->x_stride_t ? d->x_stride_t : d->C, a.yst = d->y_stride_t ? d->y_stride_t : d->C;
    if (a.xst < a.C || a.yst < a.C) return CAWN_EINVAL;
    a.xsb = d->x_stride_b ? d->x_stride_b : a.xst * d->L, a.ysb = d->y_stride_b ? d->y_stride_b : a.yst * d->L;
    p->vec = a.C >= 4 ? 4 : 1;
    a.units = (int)ceil_div(a.C, p->vec);
    // Tokens of a run: a longer one reads fewer tokens twice, where as many threads are left as the chip holds; the shortest, where each waits for its loads
    // alone, for calls of few threads, whose partial sums are few too.  (Forward and backward, us: 8 x 8,192 tokens of 768 channels in bf16 with runs of 32 and
    // 64 112, 16 and 16 144; 8 x 4,096 with 32 and 32 58, 32 and 64 70; 2 x 512 with 16, 8 and 4 backward 23.6, 19.6, 16.8; 16 x 2,000 of 200 in fp32 with
    // 16 and 8 38, 46: the sums.)
    a.run = bwd ? 64 : 32;
    auto threads = [&] { return ceil_div(a.L, a.run) * a.B * a.units; };
    while (a.run > (bwd ? 16 : 8) && threads() < 1 << (bwd ? 17 : 18)) a.run /= 2;
    while (a.run > 4 && bwd && threads() < 1 << 15) a.run /= 2;
    a.runs = a.L > 0 ? ceil_div(a.L, a.run) : 1;
    const long long all = a.runs * a.B;
    if (all > (1LL << 40) / a.units) return CAWN_EUNSUPPORTED;
    if (!bwd) p->blocks = ceil_div(all * a.units, 256);
    else {
        a.ub = a.units < 32 ? a.units : 32;
        a.rb = 256 / a.ub;
        a.ublocks = (int)ceil_div(a.units, a.ub);
        const long long want = 2048 / a.ublocks > 1 ? 2048 / a.ublocks : 1, there = ceil_div(all, a.rb);
        a.rblocks = there < want ? there : want;
        if (a.rblocks < 1) a.rblocks = 1;
        p->blocks = a.rblocks * a.ublocks;
    }
    return launchable((double)p->blocks, 256) ? CAWN_OK : CAWN_EUNSUPPORTED;
}

size_t part_bytes(const Plan &p) { return (size_t)p.a.rblocks * (p.k + 1) * p.a.C * 4; }

template <typename T, int K, int VEC, bool TAIL> int launch(const Plan &p, bool bwd, hipStream_t s)
{
    if (!bwd) hipLaunchKernelGGL((conv_forward<T, K, VEC, TAIL>), dim3((unsigned)p.blocks), dim3(256), 0, s, p.a);
    else {
        ConvArgs a = p.a;
        const bool replaces = K > 1 && a.dstate_in && a.dstate_in == a.dstate_out;
        if (replaces) a.dstate_in = nullptr;
        if (a.dx || a.part || a.dstate_in) hipLaunchKernelGGL((conv_backward<T, K, VEC, TAIL>), dim3((unsigned)p.blocks), dim3(256), 0, s, a);
        const long long all = ceil_div((long long)a.B * a.units, 256), blocks = all < STATE_BLOCKS ? all : STATE_BLOCKS;
        if (replaces) hipLaunchKernelGGL((conv_state_backward<T, K, VEC, TAIL>), dim3((unsigned)blocks), dim3(256), 0, s, p.a);
    }
    return launched();
}

template <typename T, int VEC, bool TAIL> int launch_k(const Plan &p, bool bwd, hipStream_t s)
{
    switch (p.k) {
    case 1: return launch<T, 1, VEC, TAIL>(p, bwd, s);
    case 2: return launch<T, 2, VEC, TAIL>(p, bwd, s);
    case 3: return launch<T, 3, VEC, TAIL>(p, bwd, s);
    default: return launch<T, 4, VEC, TAIL>(p, bwd, s);
    }
}

template <typename T> int launch_vec(const Plan &p, bool bwd, hipStream_t s)
{
    if (p.vec == 1) return launch_k<T, 1, false>(p, bwd, s);        // fewer than four channels
    return p.a.C % 4 ? launch_k<T, 4, true>(p, bwd, s) : launch_k<T, 4, false>(p, bwd, s);
}

int run(const cawn_conv_desc *d, const Plan &p, bool bwd, hipStream_t s)
{
    return d->bf16 ? launch_vec<bf16>(p, bwd, s) : launch_vec<float>(p, bwd, s);
}

} // namespace

extern "C" {

size_t cawn_causal_conv_state_bytes(const cawn_conv_desc *d)
{
    Plan p;
    return plan_of(d, false, &p) != CAWN_OK ? 0 : (size_t)d->B * (d->k - 1) * d->C * 4;
}

size_t cawn_causal_conv_workspace_bytes(const cawn_conv_desc *d)
{
    Plan p;
    if (plan_of(d, true, &p) != CAWN_OK) return 0;
    return part_bytes(p) > 256 ? part_bytes(p) : 256;
}

int cawn_causal_conv_fwd(const cawn_conv_desc *d, const void *x, const float *w, const float *bias, const int32_t *lengths, const void *state_in, void *y, void *state_out,
                         void *stream)
{
    Plan p;
    if (int r = plan_of(d, false, &p)) return r;
    const size_t e = d->bf16 ? 2 : 4;
    if (!aligned_to(x, e) || !aligned_to(y, e) || !aligned_to(w, 4) || !aligned_to(bias, 4) || !aligned_to(lengths, 4) || !aligned_to(state_in, 4) || !aligned_to(state_out, 4))
        return CAWN_EINVAL;
    if (d->B == 0) return CAWN_OK;
    if (!w || (d->L > 0 && (!x || !y))) return CAWN_EINVAL;
    p.a.x = x, p.a.w = w, p.a.bias = bias, p.a.lengths = lengths, p.a.state_in = (const float *)state_in, p.a.y = y, p.a.state_out = (float *)state_out;
    return run(d, p, false, (hipStream_t)stream);
}

int cawn_causal_conv_bwd(const cawn_conv_desc *d, const void *x, const float *w, const float *bias, const int32_t *lengths, const void *state_in, const void *dy,
                         const void *dstate_out, void *dx, float *dw, float *dbias, void *dstate_in, void *workspace, size_t workspace_bytes, void *stream)
{
    Plan p;
    if (int r = plan_of(d, true, &p)) return r;
    const size_t e = d->bf16 ? 2 : 4;
    if (!aligned_to(x, e) || !aligned_to(dy, e) || !aligned_to(dx, e) || !aligned_to(w, 4) || !aligned_to(bias, 4) || !aligned_to(lengths, 4) || !aligned_to(state_in, 4) ||
        !aligned_to(dstate_out, 4) || !aligned_to(dstate_in, 4) || !aligned_to(dw, 4) || !aligned_to(dbias, 4)) return CAWN_EINVAL;
    hipStream_t s = (hipStream_t)stream;
    const bool grads = dw || dbias;
    const TapSums out{dw, dbias, d->C, d->k};
    if (d->B == 0) {
        if (grads && !d->accumulate_param_grads) launch_sums(nullptr, 0, (long long)d->C * (d->k + 1), out, 0, s);      // the sums over nothing
        return launched();
    }
    if (!w || (d->L > 0 && (!x || !dy))) return CAWN_EINVAL;
    if (grads && (!workspace || workspace_bytes < part_bytes(p) || !aligned_to(workspace, 256))) return CAWN_EWORKSPACE;
    p.a.x = x, p.a.w = w, p.a.bias = bias, p.a.lengths = lengths, p.a.state_in = (const float *)state_in, p.a.dy = dy, p.a.dstate_out = (const float *)dstate_out;
    p.a.dx = dx, p.a.dstate_in = (float *)dstate_in, p.a.part = grads ? (float *)workspace : nullptr;
    if (int r = run(d, p, true, s)) return r;
    if (grads) launch_sums(p.a.part, p.a.rblocks, (long long)d->C * (d->k + 1), out, d->accumulate_param_grads, s);
    return launched();
}

} // extern "C"
