// Attention with a decay per head in FP32 arithmetic: any width up to 512, any length, fp32 or bf16 in memory.
//
// A block takes a segment of one head's chunks in the pass's order (64 rows a chunk) and TZ columns of the output; the state's
// columns stay in shared memory for the whole segment. Per chunk four products, 256 threads with 4 x 4 or 4 x 8 numbers each:
// scores X Y^T, X S, the state's update Y^T Z, and P Z.
#include "decay.cuh"

#include <float.h>

namespace darkattn {
namespace {

constexpr int C = 64, F = 64, kThreadsS = 256, kPad = 68;

template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <int TZ>
struct SimtSmem {
    static constexpr int XT = 0, YT = XT + F * kPad, Yr = YT + F * kPad, Z = Yr + C * F, PT = Z + C * TZ, pw = PT + C * kPad, S = pw + 72;
    static int bytes(int a) { return (S + (a + F - 1) / F * F * TZ) * 4; }
};

__device__ __forceinline__ int zcol(int tx, int v) { return v < 4 ? tx * 4 + v : 64 + tx * 4 + v - 4; }

// acc[4][RZ] += sum_k A[k][ty*4 ..] B[k][columns of tx]
template <int RZ, int K>
__device__ __forceinline__ void outer(float (&acc)[4][RZ], const float *A, int lda, const float *B, int ldb, int ty, int tx)
{
#pragma unroll 8
    for (int k = 0; k < K; ++k) {
        const float4 x = *reinterpret_cast<const float4 *>(A + k * lda + ty * 4);
        float y[RZ];
#pragma unroll
        for (int q = 0; q < RZ / 4; ++q) *reinterpret_cast<float4 *>(y + 4 * q) = *reinterpret_cast<const float4 *>(B + k * ldb + q * 64 + tx * 4);
#pragma unroll
        for (int v = 0; v < RZ; ++v) {
            acc[0][v] = fmaf(x.x, y[v], acc[0][v]);
            acc[1][v] = fmaf(x.y, y[v], acc[1][v]);
            acc[2][v] = fmaf(x.z, y[v], acc[2][v]);
            acc[3][v] = fmaf(x.w, y[v], acc[3][v]);
        }
    }
}

// MAIN: rows out; otherwise only the state of each of the first nseg - 1 segments, from zero, into pass.seg
template <typename T, int TZ, bool MAIN>
__global__ void __launch_bounds__(kThreadsS) decay_simt_kernel(const __grid_constant__ DecayArgs A, int ntz)
{
    constexpr int RZ = TZ / 16;
    using M = SimtSmem<TZ>;
    extern __shared__ __align__(16) float sm[];
    float *XT = sm + M::XT, *YT = sm + M::YT, *Yr = sm + M::Yr, *Zs = sm + M::Z, *PT = sm + M::PT, *pw = sm + M::pw, *S = sm + M::S;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    pdl_wait();

    if (MAIN && blockIdx.x == 0 && tid == 0) *A.status = 0;     // (nothing here waits: the call's status is known)
    const int nseg = MAIN ? A.nseg : A.nseg - 1;
    int id = blockIdx.x;
    const DecayPass &p = A.pass[id % A.npass]; id /= A.npass;
    const int zt = id % ntz; id /= ntz;
    const int seg = id % nseg, head = id / nseg;            // head: of X, or of the state
    const int z0 = zt * TZ;
    if (z0 >= p.c) return;
    const int HX = MAIN ? p.HX : A.Hkv;
    const int b = head / HX, hx = head % HX;
    const int hs = hx / (HX / A.Hkv);                        // state and decay
    const int G = p.HY > HX ? p.HY / HX : 1;                 // heads of Y that are summed over
    const int hy0 = p.HY > HX ? hx * G : hx / (HX / p.HY);
    const DecaySpan sp = decay_span<C>(A, b, seg);
    const int a = p.a, c = p.c, nf = (a + F - 1) / F;
    const bool last = sp.T == 0 ? seg == 0 : sp.k0 < sp.k1 && sp.k1 == sp.T;
    float *S_out = MAIN ? (p.S_out && last && hx % (HX / A.Hkv) == 0 ? p.S_out + (size_t)(b * A.Hkv + hs) * a * c : nullptr)
                        : const_cast<float *>(p.seg) + ((size_t)(b * A.Hkv + hs) * nseg + seg) * a * c;
    if (sp.k0 == sp.k1 && !(MAIN && last && S_out)) return;

    if (tid <= C) pw[tid] = decay_power(A.log_decay[hs], tid);
    const float *S_in = nullptr;
    if (MAIN) S_in = seg == 0 ? (p.S_in ? p.S_in + (size_t)(b * A.Hkv + hs) * a * c : nullptr) : p.seg + ((size_t)(b * A.Hkv + hs) * (nseg - 1) * A.sub + seg * A.sub - 1) * a * c;
    for (int i = tid; i < nf * F * TZ; i += kThreadsS) {
        const int f = i / TZ, z = z0 + i % TZ;
        S[i] = S_in && f < a && z < c ? (p.trans ? S_in[(size_t)z * a + f] : S_in[(size_t)f * c + z]) : 0.f;
    }
    const T *X = static_cast<const T *>(p.X) + (size_t)(b * p.HX + (MAIN ? hx : 0)) * A.N * a;
    T *O = static_cast<T *>(p.O) + (size_t)(b * p.HX + (MAIN ? hx : 0)) * A.N * c;

    for (int k = sp.k0; k < sp.k1; ++k) {
        const int t0 = (p.reverse ? sp.T - 1 - k : k) * C, L = min(C, sp.n - t0);
        float o[4][RZ];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int v = 0; v < RZ; ++v) o[u][v] = 0.f;
        for (int g = 0; g < G; ++g) {
            const T *Y = static_cast<const T *>(p.Y) + ((size_t)(b * p.HY + hy0 + g) * A.N + t0) * a;
            const T *Z = static_cast<const T *>(p.Z) + ((size_t)(b * p.HY + hy0 + g) * A.N + t0) * c;
            float sc[4][4] = {};
            __syncthreads();                                 // the tiles of the step before have been read, pw and S are there
            for (int i = tid; i < C * TZ; i += kThreadsS) {
                const int r = i / TZ, z = z0 + i % TZ;
                Zs[i] = r < L && z < c ? to_f(Z[(size_t)r * c + z]) : 0.f;
            }
            for (int fs = 0; fs < nf; ++fs) {
                if (fs) __syncthreads();
                for (int i = tid; i < C * F; i += kThreadsS) {
                    const int r = i / F, fl = i % F, f = fs * F + fl;
                    const bool in = r < L && f < a;
                    const float y = in ? to_f(Y[(size_t)r * a + f]) : 0.f;
                    if (MAIN) {
                        XT[fl * kPad + r] = in ? to_f(X[(size_t)(t0 + r) * a + f]) : 0.f;
                        YT[fl * kPad + r] = y;
                    }
                    Yr[r * F + fl] = in ? y * (pw[p.reverse ? r + 1 : L - 1 - r] * p.tok_mul) : 0.f;
                }
                __syncthreads();
                float d[4][RZ];
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int v = 0; v < RZ; ++v) d[u][v] = 0.f;
                if (MAIN) {
                    outer<4, F>(sc, XT, kPad, YT, kPad, ty, tx);
                    if (g == 0) outer<RZ, F>(o, XT, kPad, S + fs * F * TZ, TZ, ty, tx);
                }
                outer<RZ, C>(d, Yr, F, Zs, TZ, ty, tx);
                if (MAIN && g == 0) __syncthreads();         // the state before this chunk has been read
                const float keep = g == 0 ? pw[L] : 1.f;
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int v = 0; v < RZ; ++v) {
                        float &s = S[(fs * F + ty * 4 + u) * TZ + zcol(tx, v)];
                        s = keep * s + d[u][v];
                    }
            }
            if (!MAIN) continue;
            if (g == 0) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int r = ty * 4 + u;
                    const float m = r < L ? pw[p.reverse ? L - 1 - r : r + 1] * p.row_mul : 0.f;
#pragma unroll
                    for (int v = 0; v < RZ; ++v) o[u][v] *= m;
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int n = p.reverse ? tx * 4 + v - (ty * 4 + u) : ty * 4 + u - (tx * 4 + v);
                    PT[(tx * 4 + v) * kPad + ty * 4 + u] = n >= 0 ? sc[u][v] * (pw[n] * p.p_mul) : 0.f;
                }
            __syncthreads();
            outer<RZ, C>(o, PT, kPad, Zs, TZ, ty, tx);
        }
        if (MAIN) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int r = ty * 4 + u;
                if (r >= L) continue;
#pragma unroll
                for (int v = 0; v < RZ; ++v) {
                    const int z = z0 + zcol(tx, v);
                    if (z < c) O[(size_t)(t0 + r) * c + z] = from_f<T>(o[u][v]);
                }
            }
        }
    }
    if (S_out) {
        __syncthreads();
        for (int i = tid; i < a * TZ; i += kThreadsS) {
            const int f = i / TZ, z = z0 + i % TZ;
            if (z < c) S_out[(size_t)f * c + z] = S[i];
        }
    }
}

// One thread per element of the state, along the segments. Tokens of segment s: whole chunks, but for a pass backwards, whose first
// chunk may be a short one.
__global__ void __launch_bounds__(256) decay_scan_kernel(const __grid_constant__ DecayArgs A, const __grid_constant__ DecayPass p, int chunk, int by4)
{
    pdl_wait();
    __shared__ float power[2];
    const int size = p.a * p.c, i = blockIdx.x * 256 + threadIdx.x, hs = blockIdx.y % A.Hkv, b = blockIdx.y / A.Hkv;
    int n = A.N;
    if (A.lengths) n = min(max(A.lengths[b], 0), A.N);
    const int T = (n + chunk - 1) / chunk;
    if (threadIdx.x < 2) power[threadIdx.x] = decay_power(A.log_decay[hs], A.cps * chunk - (threadIdx.x && p.reverse ? T * chunk - n : 0));
    __syncthreads();
    if (i >= size) return;
    const float whole = power[0], first = power[1];
    const int from = by4 ? i / 4 % p.a * p.c + i / 4 / p.a * 4 + i % 4 : i;
    float s = p.S_in ? p.S_in[(size_t)blockIdx.y * size + from] : 0.f;
    float *at = const_cast<float *>(p.seg) + (size_t)blockIdx.y * (A.nseg - 1) * size + i;
    const int n_at = min(A.nseg - 1, (T + A.cps - 1) / A.cps - 1);      // pieces that another with a chunk follows
    constexpr int kAhead = 8;                                // loads on their way together (a piece at a time took 0.3 us each)
    for (int k0 = 0; k0 < n_at; k0 += kAhead) {
        float x[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) x[j] = k0 + j < n_at ? at[(size_t)(k0 + j) * size] : 0.f;
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (k0 + j < n_at) {
                s = (k0 + j == 0 ? first : whole) * s + x[j];
                at[(size_t)(k0 + j) * size] = s;
            }
    }
}

template <typename T, int TZ, bool MAIN>
cudaError_t launch(const DecayArgs &A, cudaStream_t st)
{
    int a = 0, c = 0, heads = 0;
    for (int i = 0; i < A.npass; ++i) {
        a = max(a, A.pass[i].a);
        c = max(c, A.pass[i].c);
        heads = max(heads, MAIN ? A.B * A.pass[i].HX : A.B * A.Hkv);
    }
    const int ntz = (c + TZ - 1) / TZ, nseg = MAIN ? A.nseg : A.nseg - 1;
    return launch_pdl(decay_simt_kernel<T, TZ, MAIN>, dim3((unsigned)((long long)A.npass * ntz * nseg * heads)), dim3(kThreadsS), SimtSmem<TZ>::bytes(a), st, A, ntz);
}

template <typename T, bool MAIN>
cudaError_t launch_t(const DecayArgs &A, cudaStream_t st)
{
    int a = 0, c = 0;
    for (int i = 0; i < A.npass; ++i) { a = max(a, A.pass[i].a); c = max(c, A.pass[i].c); }
    return a <= 128 && c > 64 ? launch<T, 128, MAIN>(A, st) : launch<T, 64, MAIN>(A, st);
}

}  // namespace

cudaError_t decay_scan_pieces(const DecayArgs &A, const DecayPass &p, int chunk, bool by4, cudaStream_t st)
{
    return launch_pdl(decay_scan_kernel, dim3((unsigned)((p.a * p.c + 255) / 256), (unsigned)(A.B * A.Hkv)), dim3(256), 0, st, A, p, chunk, (int)by4);
}

// passes of equal numbers of heads share a launch
static cudaError_t run_main(const DecayArgs &A, int bf16, cudaStream_t st)
{
    for (int i = 0; i < A.npass;) {
        DecayArgs B = A;
        int n = 0;
        while (i < A.npass && (n == 0 || A.pass[i].HX == B.pass[0].HX)) B.pass[n++] = A.pass[i++];
        B.npass = n;
        const cudaError_t e = bf16 ? launch_t<__nv_bfloat16, true>(B, st) : launch_t<float, true>(B, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

darkattn_status_t decay_simt_run(DecayArgs &A, DecayPass *state_pass, int nstate, int bf16, cudaStream_t st)
{
    if (A.nseg > 1) {
        const DecayArgs P = decay_pieces(A, state_pass, nstate);
        DARKATTN_CUDA_TRY((bf16 ? launch_t<__nv_bfloat16, false>(P, st) : launch_t<float, false>(P, st)), "decay_simt_kernel (states)");
        for (int i = 0; i < nstate; ++i) DARKATTN_CUDA_TRY(decay_scan_pieces(P, state_pass[i], C, false, st), "decay_scan_kernel");
    }
    DARKATTN_CUDA_TRY(run_main(A, bf16, st), "decay_simt_kernel");
    return DARKATTN_OK;
}

// Segments: as many as shorten the longest chain of chunks by more than the states' own pass and the sum over them cost. In units of a
// chunk's time; a chunk of the states' pass is one product of four.
static void pick(int T, long long units, long long state_units, int slots, int &nseg, int &cps, int &sub)
{
    double best = 1e30;
    sub = 1;
    for (int n = 1; n <= T && n <= 128; ++n) {
        const int per = (T + n - 1) / n, m = (T + per - 1) / per;
        double cost = (double)((units * m + slots - 1) / slots) * (per + 1);
        if (m > 1) cost += (double)((state_units * (m - 1) + slots - 1) / slots) * (0.5 * per + 1) + 2 + 0.1 * m;
        if (cost < best) { best = cost; nseg = m; cps = per; }
    }
}

void decay_simt_split(darkattn_decay_plan_s *plan)
{
    const darkattn_decay_desc_t &ds = plan->desc;
    const int T = (ds.N + C - 1) / C, w = ds.d > ds.dv ? ds.d : ds.dv;
    const int tz = w <= 128 && w > 64 ? 128 : 64;
    const long long zf = (ds.dv + tz - 1) / tz, zb = (w + tz - 1) / tz;
    const int slots = w <= 64 ? 296 : 148;
    pick(T, (long long)ds.B * ds.H * zf, (long long)ds.B * ds.H_kv * zf, slots, plan->fwd.nseg, plan->fwd.cps, plan->fwd.sub);
    pick(T, (long long)ds.B * (ds.H + 2 * ds.H) * zb, 2LL * ds.B * ds.H * zf, slots, plan->bwd.nseg, plan->bwd.cps, plan->bwd.sub);
}

}  // namespace darkattn
