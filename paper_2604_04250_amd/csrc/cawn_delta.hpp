// Gated delta rule: what its translation units share.
#pragma once
#include "cawn_ops.hpp"

namespace cawn {
namespace delta {

using namespace cawn::ops;

constexpr int CHUNK = 64;           // tokens treated at once by the chunked kernels
constexpr int TOKEN_MAX = 16;       // longest call that goes token by token
constexpr int OPERAND_BYTES = 18 * 1024;     // T as operands, three planes
constexpr int GATE_FLOATS = 9 * CHUNK;
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
    int chunks, slabs;              // chunks of a full row; (token form) slabs of a head's columns
    int vec4;                       // state rows may be read 16 bytes at a time
    int vecq, veco;                 // rows of q and k (16 bytes), of o (four values) and dO (16 bytes) may be taken several values at a time
    int vecd;                       // rows of dq, dk: four values
    // Chunked form.  Tiles of the state before each chunk and of u, kept for a backward (null: not wanted): those of
    // chunk n of head bh begin bh * row + n * chunk bytes behind
    int VT;                         // tiles of 16 value columns
    char *s_tiles, *u_tiles;
    size_t s_row, s_chunk, u_row, u_chunk;
    char *dr_tiles, *ds_tiles;      // backward: dR and dS of every chunk, in tiles
    // Segments of seg_chunks chunks; per head and chunk GATE_FLOATS gates; per head and segment the matrix A (KP x KP, row-major),
    // the offset b and the state at its begin (backward: its gradient behind its end), in tiles
    int segments, seg_chunks;
    float *gates;
    char *t_ops;                    // per head and chunk T
    char *seg_a, *seg_b, *seg_s;
};

// Sizes in the chunked form, in pieces of 1 KiB: a plane of a matrix operand (64 lanes x 8 bf16) or an fp32 tile (16 x 16, a lane's four
// rows together)
struct Sizes {
    int KP, VT, ut, st;             // padded K; tiles of V; pieces of a chunk's u, of a state
    __host__ __device__ Sizes(int K, int V)
    {
        KP = K <= 32 ? 32 : K <= 64 ? 64 : 128;
        VT = (V + 15) / 16;
        ut = 4 * VT;
        st = (KP / 16) * VT;
    }
};

__device__ inline int row_length(const Args &a, int b)
{
    const int n = a.lengths ? a.lengths[b] : a.L;
    return n < 0 ? 0 : n < a.L ? n : a.L;
}

int launch_token(const Args &a, bool bf16, hipStream_t s);
int launch_system(const Args &a, bool bf16, hipStream_t s);
int scan_held(int K, int VT, bool bf16, int *columns);                  // workgroups of the scan that a CU holds, and the column tiles of each
int launch_scan(const Args &a, bool bf16, hipStream_t s);               // forward, behind the gates
int launch_join(const Args &a, bool reverse, hipStream_t s);
int launch_back(const Args &a, bool bf16, hipStream_t s);               // backward: the recurrence
int launch_gradients(const Args &a, bool bf16, hipStream_t s);          // backward: every gradient but the state's

} // namespace delta
} // namespace cawn
