// Gated delta rule: what its translation units share.
#pragma once
#include "cawn_ops.hpp"

namespace cawn {
namespace delta {

using namespace cawn::ops;

constexpr int CHUNK = 64;           // tokens treated at once by the chunked kernels
constexpr int TOKEN_MAX = 16;       // longest call that goes token by token
constexpr float DECAY_MIN = -104.f; // exp underflows to 0 below: a decay of minus infinity counts as this, so that sums of decays stay finite

struct Args {
    int B, L, H, Hk, K, V;
    int norm;
    float scale, eps;
    long long qsb, qst, vsb, vst, osb, ost;
    const void *q, *k, *v;
    const float *decay, *beta;
    const int32_t *lengths;
    const float *state_in;
    void *o;
    float *state_out;
    // backward
    const void *dO;
    const float *dstate_out;
    void *dq, *dk, *dv;
    float *ddecay, *dbeta, *dstate_in;
    // checkpoint and workspace
    float *ck_state;                // [B][H][chunks][K][V]: the state before each chunk
    float *ck_u;                    // [B][H][chunks][CHUNK][V]
    char *ws;
    int chunks, slabs;
    int vec4;                       // state rows may be read 16 bytes at a time
};

__device__ inline int row_length(const Args &a, int b)
{
    const int n = a.lengths ? a.lengths[b] : a.L;
    return n < 0 ? 0 : n < a.L ? n : a.L;
}

int launch_token(const Args &a, bool bf16, hipStream_t s);

} // namespace delta
} // namespace cawn
