// Gated delta rule: what its translation units share.
#pragma once
#include "cawn_ops.hpp"

namespace cawn {
namespace delta {

using namespace cawn::ops;

constexpr int CHUNK = 64;           // tokens treated at once by the chunked kernels
constexpr int TOKEN_MAX = 16;       // longest call that goes token by token
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
    int chunks, slabs;
    int vec4;                       // state rows may be read 16 bytes at a time
    int vecq, vecv, veco;           // rows of q, k (dq, dk), of v (dv), of o (dO) may be: 16 bytes at a time
    // Chunked form.  The launches of a call treat the chunks c0 .. c1-1 of every row; the workspace holds `span` of them.
    int c0, c1, span, VT;           // VT: tiles of 16 value columns
    char *ws;
    // tiles of the state before each chunk, and of u: in the checkpoint or in the workspace.  Chunk n of head bh begins
    // bh * row + (n - first) * chunk bytes behind
    char *s_tiles, *u_tiles;
    size_t s_row, s_chunk, u_row, u_chunk;
    int s_first, u_first;
    // Segments of seg_chunks chunks; per head and chunk GATE_FLOATS gates; per head and segment the matrix A (KP x KP, row-major),
    // the offset b and the state at its begin, in tiles
    int segments, seg_chunks;
    float *gates;
    char *t_ops, *tt_ops;           // per head and chunk T's operands, and its transpose's (null: not wanted)
    char *seg_a, *seg_b, *seg_s;
};

// Sizes in the chunked form; everything is made of 1 KiB pieces: a matrix operand's plane (64 lanes x 8 bf16) or an fp32 tile
// (16 x 16, a lane's four rows together).
struct Sizes {
    int KP, VT, wf, kf, ut, st;     // padded K; tiles of V; pieces of W, of K^T, of a chunk's u, of a state
    size_t slot;                    // workspace of one chunk of one head, forward
    size_t bslot;                   // backward
    __host__ __device__ Sizes(int K, int V, int planes)
    {
        KP = K <= 32 ? 32 : K <= 64 ? 64 : 128;
        VT = (V + 15) / 16;
        wf = 4 * (KP / 32) * 3;
        kf = (KP / 16) * 2 * planes;
        ut = 4 * VT;
        st = (KP / 16) * VT;
        slot = (size_t)(wf + kf + ut + 2) * 1024;               // W, K^T, u, gates
        bslot = (size_t)(wf + kf + ut + 3 + 2 * st) * 1024;     // ... dR for u, Y and dS
    }
};

__device__ inline int row_length(const Args &a, int b)
{
    const int n = a.lengths ? a.lengths[b] : a.L;
    return n < 0 ? 0 : n < a.L ? n : a.L;
}

int launch_token(const Args &a, bool bf16, hipStream_t s);
int launch_system(const Args &a, bool bf16, hipStream_t s);
int launch_scan(const Args &a, bool bf16, hipStream_t s);               // forward, behind the gates
int launch_join(const Args &a, bool reverse, hipStream_t s);

int launch_adjoint(const Args &a, bool bf16, hipStream_t s);            // backward: Wd, K^T, dR0, Y, gates
int launch_gradients(const Args &a, bool bf16, hipStream_t s);          // backward: every gradient but the state's

// The recurrence over chunks, either direction: X += W S, S = e S + K^T (c X) (+ Y), with S stored ahead of every chunk.
struct StateArgs {
    int B, L, H, K, V, VT, chunks, c0, c1, span;
    const int32_t *lengths;
    char *ws;                       // a chunk's slot: W, K^T, X0, gates, (Y)
    size_t slot;
    size_t x_at, gates_at, y_at;    // in the slot
    char *s_tiles;                  // states ahead of the chunks
    size_t s_row, s_chunk;          // bytes from one head's to the next, from one chunk's to the next
    int s_first;                    // chunk of the first
    char *x_tiles;                  // X of the chunks, likewise
    size_t x_row, x_chunk;
    int x_first;
    char *carry;                    // [B H][st] tiles: from one launch to the next
    const float *begin;             // row-major state at the beginning (or null: zero), read when `first`
    float *end;                     // row-major state at the end, written when `last`
    int first, last, keep_end;      // keep_end: the state behind the last chunk goes to s_tiles too
};
int launch_states(const StateArgs &a, bool bf16, bool reverse, hipStream_t s);

} // namespace delta
} // namespace cawn
