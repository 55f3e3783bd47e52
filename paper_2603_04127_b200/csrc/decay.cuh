// Attention with a decay per head: what its kernels and its host side share.
//
// The forward pass and the three gradients are one operator on rows x, y (a wide) and z (c wide) of a sequence,
//     out_i = p_mul sum_j lambda^|i-j| (x_i . y_j) z_j + row_mul lambda^(distance of i to the boundary) x_i S,
// j running over i and what lies before it in the pass's direction, S the state at the boundary the pass enters by:
//     O : (Q, K, V)  forwards      S = sum_j lambda^(..) k_j v_j^T
//     dQ: (dO, V, K) forwards      S^T
//     dK: (V, dO, Q) backwards     R^T,  R = sum_i lambda^(..) scale q_i do_i^T, the gradient of the state
//     dV: (K, Q, dO) backwards     R
// It is evaluated in chunks: masked products inside a chunk, the state between chunks. In a chunk of L rows, row r lies r + 1 steps
// behind the boundary before it and L - 1 - r before the one after it, so a pass forwards reads the state by lambda^(r+1) and adds
// row r to it by lambda^(L-1-r), a pass backwards the other way round, and either multiplies the state by lambda^L: every
// power of lambda is one of 0 .. L, never a quotient, so that no decay is too strong.
#pragma once

#include "common.cuh"

#include <initializer_list>

namespace darkattn {

struct DecayPass {
    const void *X, *Y, *Z;      // [B, HX, N, a], [B, HY, N, a], [B, HY, N, c]
    void *O;                    // [B, HX, N, c]
    const float *S_in;          // state the pass enters by, [B, Hkv, d, dv]; null: zero
    float *S_out;               // state it leaves by; null: not wanted (always null where trans is set)
    const float *seg;           // states the pieces behind the first enter by, [B * Hkv, (nseg - 1) sub, d, dv]
    int a, c;
    int HX, HY;                 // heads of X and O, and of Y and Z: where HX > HY consecutive heads of X share one of Y, where
                                // HY > HX the sum runs over consecutive heads of Y
    int reverse;                // direction
    int trans;                  // S is [c, a] in memory
    float p_mul, row_mul, tok_mul;   // tok_mul: of a token's share of the state
    int whole;                  // (states of segments) the state reaches the caller
};

constexpr int kDecayPasses = 3;

struct DecayArgs {
    DecayPass pass[kDecayPasses];
    int npass;
    const float *log_decay;     // [Hkv]
    const int *lengths;         // [B] or null
    int B, Hkv, N;
    int nseg, cps;              // segments of a sequence, chunks of each
    int sub;                    // pieces that each of the first nseg - 1 segments is cut into where their states are summed
    int *status;
    int clear;                  // the call's first kernel: sets the status to zero
    int zero;                   // rows out behind a sequence's end are set to zero (else left as they were)
};

// Segments are counted in the order the pass takes the chunks: its k-th chunk is chunk k forwards, T - 1 - k backwards.
struct DecaySpan {
    int n, T;                   // tokens and chunks of this sequence
    int k0, k1;                 // chunks of this segment, in the pass's order
};
template <int C>
__device__ __forceinline__ DecaySpan decay_span(const DecayArgs &A, int b, int seg)
{
    DecaySpan s;
    s.n = A.N;
    if (A.lengths) s.n = min(max(A.lengths[b], 0), A.N);
    s.T = (s.n + C - 1) / C;
    s.k0 = min(seg * A.cps, s.T);
    s.k1 = min(s.k0 + A.cps, s.T);
    return s;
}
// Zeros for the rows behind the sequence's end that lie where this segment would be in a full one: `out` is the head's first row. (A kernel of its
// own, 48 blocks of a padded batch, started beside the call before on the few idle SMs: 16 heads of 5888 tokens, a quarter and a half of
// them there, gradients in 214 us instead of 102, for what full ones take 83.)
template <int C, typename T>
__device__ __forceinline__ void zero_behind(const DecayArgs &A, const DecaySpan &s, int seg, T *out, int width, int tid, int threads)
{
    if (!A.zero) return;
    const long long from = max((long long)s.n, (long long)seg * A.cps * C), to = seg == A.nseg - 1 ? A.N : min((long long)A.N, (long long)(seg + 1) * A.cps * C);
    unsigned char *at = reinterpret_cast<unsigned char *>(out + from * width);
    const int row = width * (int)sizeof(T);
    const long long bytes = (to - from) * row;
    if (row % 16 == 0) for (long long i = tid; i < bytes / 16; i += threads) reinterpret_cast<uint4 *>(at)[i] = make_uint4(0, 0, 0, 0);
    else for (long long i = tid; i < bytes / 2; i += threads) reinterpret_cast<unsigned short *>(at)[i] = 0;
}
// lambda^n, right to the last bit or so: the tables are a few numbers per block
__device__ __forceinline__ float decay_power(float g, int n) { return n == 0 ? 1.f : (float)exp((double)g * (double)n); }

struct darkattn_decay_layout {
    size_t status, seg[2], bytes;        // seg: states of the segments of a pass forwards, of one backwards
};

}  // namespace darkattn

struct darkattn_decay_plan_s {
    darkattn_decay_desc_t desc;
    int path;
    struct { int nseg, cps, sub; } fwd, bwd;
    darkattn::darkattn_decay_layout ws;
    size_t workspace_bytes;
};

namespace darkattn {

// Arrays of a call, on the host. What a call writes must not lie over anything else that it reads or writes: blocks take rows in any order.
struct Span {
    const void *p;
    size_t bytes;
};
inline bool clash(std::initializer_list<Span> out, std::initializer_list<Span> in)
{
    const auto meet = [](const Span &a, const Span &b) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
        return a.p && b.p && x < y + b.bytes && y < x + a.bytes;
    };
    for (const Span *o = out.begin(); o != out.end(); ++o) {
        for (const Span *p = out.begin(); p != o; ++p)
            if (meet(*o, *p)) return true;
        for (const Span &i : in)
            if (meet(*o, i)) return true;
    }
    return false;
}

// Heads whose chunks are one item of work each, and heads that sum over a group of G.
struct DecayLoad {
    long long heads, sums;
    int G;
};

// FP32 kernels, any shape
void decay_simt_split(darkattn_decay_plan_s *plan);
darkattn_status_t decay_simt_run(DecayArgs &A, DecayPass *state_pass, int nstate, int bf16, cudaStream_t st);
// The arguments of the kernels that sum the states of the pieces: segments of cps / sub chunks, all but the last summed.
inline DecayArgs decay_pieces(const DecayArgs &A, const DecayPass *pass, int npass)
{
    DecayArgs P = A;
    P.npass = npass;
    for (int i = 0; i < npass; ++i) P.pass[i] = pass[i];
    P.nseg = (A.nseg - 1) * A.sub + 1;
    P.cps = A.cps / A.sub;
    P.sub = 1;
    return P;
}
// Adds up the pieces' states in place: slot s then holds the state that piece s + 1 enters by. `by4`: a slot's numbers lie as
// [dv / 4][d][4] (what a warp with a row a lane reads and writes 16 bytes at a time is contiguous), else as [d][dv].
cudaError_t decay_scan_pieces(const DecayArgs &P, const DecayPass &p, int chunk, bool by4, cudaStream_t st);

// tcgen05 kernels, bf16
bool decay_tc_supported(const darkattn_decay_desc_t &ds);
void decay_tc_split(darkattn_decay_plan_s *plan);
darkattn_status_t decay_tc_run(DecayArgs &A, DecayPass *state_pass, int nstate, cudaStream_t st);

darkattn_status_t decay_step(const darkattn_decay_plan_s *plan, const void *q, const void *k, const void *v, const float *log_decay,
                             float *S, const int *slots, int n_slots, void *o, cudaStream_t st);

}  // namespace darkattn
