// Attention with a decay per head in FP32 arithmetic: any width up to 512, any length, fp32 or bf16 in memory.
//
// A block takes a segment of one head's chunks in the pass's order (64 rows a chunk), per chunk four products: scores X Y^T, X S, the
// state's update Y^T Z, and P Z. Widths up to 128 have kernels of their own below; wider ones go by slices of 64 and tiles of 64 columns
// of the output, whose share of the state stays in shared memory for the whole segment.
#include "decay.cuh"

namespace darkattn {
namespace {

constexpr int C = 64, F = 64, kThreadsS = 256, kPad = 68;

template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// ---------------------------------------------------------------- widths up to 128
// The whole width of X, Y and Z at once: 256 threads, thread (ty, tx) holds R x R numbers of the state in registers (rows of ty, columns of tx)
// and 4 x R of the rows out. R = 4, 5, 6 or 8 for widths up to 64, 80, 96, 128. Products two numbers at a time (FFMA2: an FFMA was measured
// at 2.3 cycles a scheduler, an FFMA2, twice the work, at 2.0).
__device__ __forceinline__ int spot(int t, int v, int R) { return v < 4 ? t * 4 + v : 64 + t * (R - 4) + v - 4; }

// The R numbers of thread t's spots, from a row
template <int R>
__device__ __forceinline__ void take(float (&y)[8], const float *row, int t)
{
    *reinterpret_cast<float4 *>(y) = *reinterpret_cast<const float4 *>(row + t * 4);
    if (R == 5) y[4] = row[64 + t];
    if (R == 6) *reinterpret_cast<float2 *>(y + 4) = *reinterpret_cast<const float2 *>(row + 64 + t * 2);
    if (R == 8) *reinterpret_cast<float4 *>(y + 4) = *reinterpret_cast<const float4 *>(row + 64 + t * 4);
}
__device__ __forceinline__ unsigned long long pair(float a, float b)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void fma_pair(unsigned long long &acc, unsigned long long a, unsigned long long b)
{
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(a), "l"(b));
}
__device__ __forceinline__ float2 both(unsigned long long a)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a));
    return r;
}
// Numbers of one row by columns: pairs, and one alone where R is odd
template <int R> struct Row {
    unsigned long long p[R / 2];
    float last;
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < R / 2; ++i) p[i] = 0ull;
        last = 0.f;
    }
    __device__ __forceinline__ void scale(float f)
    {
        const unsigned long long f2 = pair(f, f);
#pragma unroll
        for (int i = 0; i < R / 2; ++i) asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(p[i]) : "l"(f2));
        last *= f;
    }
    __device__ __forceinline__ void add(float x, const unsigned long long (&y)[4], float ylast)
    {
        const unsigned long long x2 = pair(x, x);
#pragma unroll
        for (int i = 0; i < R / 2; ++i) fma_pair(p[i], x2, y[i]);
        if (R & 1) last = fmaf(x, ylast, last);
    }
    __device__ __forceinline__ float get(int v) const
    {
        if ((R & 1) && v == R - 1) return last;
        const float2 b = both(p[v / 2]);
        return v & 1 ? b.y : b.x;
    }
    // to thread t's spots of a row in shared memory
    __device__ __forceinline__ void put(float *row, int t) const
    {
        *reinterpret_cast<float4 *>(row + t * 4) = make_float4(get(0), get(1), get(2), get(3));
        if (R == 5) row[64 + t] = get(4);
        if (R == 6) *reinterpret_cast<float2 *>(row + 64 + t * 2) = make_float2(get(4), get(5));
        if (R == 8) *reinterpret_cast<float4 *>(row + 64 + t * 4) = make_float4(get(4), get(5), get(6), get(7));
    }
    __device__ __forceinline__ void set(int v, float x)
    {
        if ((R & 1) && v == R - 1) { last = x; return; }
        const float2 b = both(p[v / 2]);
        p[v / 2] = v & 1 ? pair(b.x, x) : pair(x, b.y);
    }
};
// acc[u] += sum over k < K of a_u[k] b[k][columns of tx]: a_u[k] the u-th number of ty in row k of A (RA of them)
template <int RA, int R, int RB>
__device__ __forceinline__ void products(Row<R> (&acc)[RA], const float *A, int lda, const float *B, int ldb, int K, int ty, int tx)
{
#pragma unroll 8
    for (int k = 0; k < K; ++k) {
        float x[8], y[8];
        take<RA>(x, A + k * lda, ty);
        take<RB>(y, B + k * ldb, tx);
        unsigned long long y2[4];
#pragma unroll
        for (int i = 0; i < R / 2; ++i) y2[i] = pair(y[2 * i], y[2 * i + 1]);
#pragma unroll
        for (int u = 0; u < RA; ++u) acc[u].add(x[u], y2, y[R - 1]);
    }
}

template <int R>
struct TileSmem {
    static constexpr int LW = R == 4 ? 64 : 64 + 16 * (R - 4);                       // widest row
    // P takes the place of Y transposed when the scores are there: so two blocks of 80 columns fit an SM
    static constexpr int XT = 0, YT = XT + LW * kPad, PT = YT, Yw = YT + LW * kPad, Z = Yw + C * LW, S = Z + C * LW, pw = S + LW * LW, total = (pw + 72) * 4;
    static_assert(total <= 232448, "shared memory of a block");
};

// four numbers of a row of `width`, zeros behind its end
template <typename T>
__device__ __forceinline__ float4 load4(const T *row, int f, int width, bool vec)
{
    float4 x = make_float4(0, 0, 0, 0);
    if (vec) {
        if (f < width) {
            if constexpr (sizeof(T) == 4) x = *reinterpret_cast<const float4 *>(row + f);
            else {
                const uint2 r = *reinterpret_cast<const uint2 *>(row + f);
                x = make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u), __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u));
            }
        }
        return x;
    }
    if (f < width) x.x = to_f(row[f]);
    if (f + 1 < width) x.y = to_f(row[f + 1]);
    if (f + 2 < width) x.z = to_f(row[f + 2]);
    if (f + 3 < width) x.w = to_f(row[f + 3]);
    return x;
}

__device__ __forceinline__ void store4(float *at, float a, float b, float c, float d) { *reinterpret_cast<float4 *>(at) = make_float4(a, b, c, d); }
__device__ __forceinline__ void store4(__nv_bfloat16 *at, float a, float b, float c, float d)
{
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b), y = __floats2bfloat162_rn(c, d);
    *reinterpret_cast<uint2 *>(at) = make_uint2(*reinterpret_cast<const unsigned *>(&x), *reinterpret_cast<const unsigned *>(&y));
}

// (Up to 80 columns two blocks fit an SM's shared memory, and have to fit its registers: with one, 4 x 24 heads of 2000 tokens, d 80, 422 us for 348.)
template <typename T, int R, bool MAIN>
__global__ void __launch_bounds__(kThreadsS, R <= 5 ? 2 : 1) decay_tile_kernel(const __grid_constant__ DecayArgs A)
{
    using M = TileSmem<R>;
    constexpr int LW = M::LW;
    extern __shared__ __align__(16) float sm[];
    float *XT = sm + M::XT, *YT = sm + M::YT, *Yw = sm + M::Yw, *Zs = sm + M::Z, *PT = sm + M::PT, *Ss = sm + M::S, *pw = sm + M::pw;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, warp = tid >> 5, lane = tid & 31;
    pdl_wait();
    if (MAIN && blockIdx.x == 0 && tid == 0) *A.status = 0;     // (nothing here waits: the call's status is known)

    const int nseg = MAIN ? A.nseg : A.nseg - 1;
    int id = blockIdx.x;
    const DecayPass &p = A.pass[id % A.npass]; id /= A.npass;
    const int seg = id % nseg, head = id / nseg, HX = MAIN ? p.HX : A.Hkv;
    if (head >= A.B * HX) return;
    const int b = head / HX, hx = head % HX, hs = hx / (HX / A.Hkv);
    const int G = p.HY > HX ? p.HY / HX : 1, hy0 = p.HY > HX ? hx * G : hx / (HX / p.HY);
    const DecaySpan sp = decay_span<C>(A, b, seg);
    const int a = p.a, c = p.c, reverse = p.reverse;
    const bool va = a % 4 == 0, vc = c % 4 == 0;
    const bool last = sp.T == 0 ? seg == 0 : sp.k0 < sp.k1 && sp.k1 == sp.T;
    const size_t state = (size_t)(b * A.Hkv + hs) * a * c;
    float *S_out = MAIN ? (p.S_out && last && hx % (HX / A.Hkv) == 0 ? p.S_out + state : nullptr)
                        : const_cast<float *>(p.seg) + ((size_t)(b * A.Hkv + hs) * nseg + seg) * a * c;
    T *O = static_cast<T *>(p.O) + (size_t)(b * p.HX + (MAIN ? hx : 0)) * A.N * c;
    if (MAIN) zero_behind<C>(A, sp, seg, O, c, tid, kThreadsS);
    if (sp.k0 == sp.k1 && !(MAIN && last && S_out)) return;
    if (tid <= C) pw[tid] = decay_power(A.log_decay[hs], tid);
    const float *S_in = nullptr;
    if (MAIN) S_in = seg == 0 ? (p.S_in ? p.S_in + state : nullptr) : p.seg + ((size_t)(b * A.Hkv + hs) * (nseg - 1) * A.sub + seg * A.sub - 1) * a * c;

    Row<R> s[R];                                             // rows spot(ty, u), columns spot(tx, v)
#pragma unroll
    for (int u = 0; u < R; ++u) {
        s[u].clear();
#pragma unroll
        for (int v = 0; v < R; ++v) {
            const int f = spot(ty, u, R), z = spot(tx, v, R);
            if (S_in && f < a && z < c) s[u].set(v, p.trans ? S_in[(size_t)z * a + f] : S_in[(size_t)f * c + z]);
        }
    }
    const auto put_state = [&]() {
#pragma unroll
        for (int u = 0; u < R; ++u) s[u].put(Ss + spot(ty, u, R) * LW, tx);
    };
    if (MAIN) put_state();
    const T *X = static_cast<const T *>(p.X) + (size_t)(b * p.HX + (MAIN ? hx : 0)) * A.N * a;

    // A warp brings 8 rows, 16 columns at a time: whole sectors, and two-way bank conflicts where it stores them transposed. All of a thread's loads are
    // on their way together (two rounds of them at a time: d 128, 16 heads of 2757 tokens 179 us for 156). The next item's, fetched before P Z: 164.
    constexpr int kLoads = LW / 16;
    const int lr = warp * 8 + (lane >> 2), lf = (lane & 3) * 4;
    float4 lx[kLoads], ly[kLoads], lz[kLoads];
    const auto fetch = [&](int k, int g) {
        const int t0 = (reverse ? sp.T - 1 - k : k) * C;
        const bool in = lr < min(C, sp.n - t0);
        const size_t at = (size_t)(b * p.HY + hy0 + g) * A.N + t0 + lr;
        const T *x = X + (size_t)(t0 + lr) * a, *y = static_cast<const T *>(p.Y) + at * a, *z = static_cast<const T *>(p.Z) + at * c;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            lx[j] = ly[j] = lz[j] = make_float4(0, 0, 0, 0);
            if (in) {
                ly[j] = load4(y, lf + 16 * j, a, va);
                lz[j] = load4(z, lf + 16 * j, c, vc);
                if (MAIN && g == 0) lx[j] = load4(x, lf + 16 * j, a, va);
            }
        }
    };

    // X S is left out where the state is zero: before a first chunk (12 heads of 100 tokens, d 128: 35.5 -> 29.8 us). Not where two blocks share an SM and
    // others of the grid do have a state: 2 x 12 heads of 1000 tokens, d 80, in 16 segments took 56 us for 51.
    for (int k = sp.k0; k < sp.k1; ++k) {
        const int t0 = (reverse ? sp.T - 1 - k : k) * C, L = min(C, sp.n - t0);
        Row<R> o[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) o[u].clear();
        const bool mine = warp * 8 < L;                      // the warp has rows (of short chunks few do: 9 tokens of 12 heads on 3, d 128, gradients 67 -> 58 us)
        for (int g = 0; g < G; ++g) {
            __syncthreads();                                 // the tiles of the step before have been read; pw and the state are there
            fetch(k, g);
            const float w = lr < L ? pw[reverse ? lr + 1 : L - 1 - lr] * p.tok_mul : 0.f;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int f = lf + 16 * j;
                const float4 x = lx[j], y = ly[j];
                *reinterpret_cast<float4 *>(Zs + lr * LW + f) = lz[j];
                if (MAIN) {
                    YT[f * kPad + lr] = y.x; YT[(f + 1) * kPad + lr] = y.y; YT[(f + 2) * kPad + lr] = y.z; YT[(f + 3) * kPad + lr] = y.w;
                    if (g == 0) { XT[f * kPad + lr] = x.x; XT[(f + 1) * kPad + lr] = x.y; XT[(f + 2) * kPad + lr] = x.z; XT[(f + 3) * kPad + lr] = x.w; }
                }
                *reinterpret_cast<float4 *>(Yw + lr * LW + f) = make_float4(y.x * w, y.y * w, y.z * w, y.w * w);
            }
            __syncthreads();
            if (MAIN) {
                Row<4> sc[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) sc[u].clear();
                if (mine) products<4, 4, 4>(sc, XT, kPad, YT, kPad, a, ty, tx);
                if (g == 0 && mine && (S_in || k > sp.k0 || (R <= 5 && nseg > 1))) {
                    products<4, R, R>(o, XT, kPad, Ss, LW, a, ty, tx);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int r = ty * 4 + u;
                        o[u].scale(r < L ? pw[reverse ? L - 1 - r : r + 1] * p.row_mul : 0.f);
                    }
                }
                __syncthreads();                             // Y transposed has been read
                const int n0 = reverse ? tx * 4 - ty * 4 : ty * 4 - tx * 4;      // distance of the 4 x 4 numbers' first
                float w[7];                                  // decays of distances n0 - 3 .. n0 + 3
#pragma unroll
                for (int i = 0; i < 7; ++i) w[i] = n0 + i - 3 >= 0 ? pw[n0 + i - 3] * p.p_mul : 0.f;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    float x[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) x[u] = n0 + (reverse ? v - u : u - v) >= 0 ? sc[u].get(v) * (reverse ? w[3 + v - u] : w[3 + u - v]) : 0.f;
                    *reinterpret_cast<float4 *>(PT + (tx * 4 + v) * kPad + ty * 4) = make_float4(x[0], x[1], x[2], x[3]);
                }
            }
            if (k + 1 < sp.k1 || S_out) {                    // somebody reads the state behind this chunk
                if (g == 0) {
                    const float keep = pw[L];
#pragma unroll
                    for (int u = 0; u < R; ++u) s[u].scale(keep);
                }
                products<R, R, R>(s, Yw, LW, Zs, LW, L, ty, tx);
            }
            if (!MAIN) continue;
            __syncthreads();                                 // P is there; the state before this chunk has been read
            // rows 8 warp .. 8 warp + 7 of P: zero behind (backwards: before) the diagonal
            const int from = reverse ? warp * 8 : 0, to = reverse ? L : mine ? min(warp * 8 + 8, L) : 0;
            products<4, R, R>(o, PT + from * kPad, kPad, Zs + from * LW, LW, to - from, ty, tx);
            if (g == G - 1) put_state();
        }
        if (MAIN) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int r = ty * 4 + u;
                if (r >= L) continue;
                T *at = O + (size_t)(t0 + r) * c;
                if (vc) {
                    if (tx * 4 < c) store4(at + tx * 4, o[u].get(0), o[u].get(1), o[u].get(2), o[u].get(3));
                    if (R == 8 && 64 + tx * 4 < c) store4(at + 64 + tx * 4, o[u].get(4), o[u].get(5), o[u].get(6), o[u].get(7));
                }
#pragma unroll
                for (int v = 0; v < R; ++v) {
                    const int z = spot(tx, v, R);
                    if (z < c && !(vc && (v < 4 || R == 8))) at[z] = from_f<T>(o[u].get(v));
                }
            }
        }
    }
    if (S_out) {
#pragma unroll
        for (int u = 0; u < R; ++u)
#pragma unroll
            for (int v = 0; v < R; ++v) {
                const int f = spot(ty, u, R), z = spot(tx, v, R);
                if (f < a && z < c) S_out[(size_t)f * c + z] = s[u].get(v);
            }
    }
}

// ---------------------------------------------------------------- wider
// What the tiles above are, by slices of 64 of X and Y and for 64 columns of Z; the scores are formed again for each 64 columns. Bound by the products and
// the barriers between them: 4 x 16 heads of 2048 tokens, 256 x 256, 2.4 ms (0.9 by their arithmetic alone).
struct SimtSmem {
    static constexpr int XT = 0, YT = XT + F * kPad, Yr = YT + F * kPad, Z = Yr + C * F, PT = Z + C * F, pw = PT + C * kPad, S = pw + 72;
    static int bytes(int a) { return (S + (a + F - 1) / F * F * F) * 4; }
};

// MAIN: rows out; otherwise only the state of each of the first nseg - 1 segments, from zero, into pass.seg
template <typename T, bool MAIN>
__global__ void __launch_bounds__(kThreadsS) decay_simt_kernel(const __grid_constant__ DecayArgs A, int ntz)
{
    using M = SimtSmem;
    extern __shared__ __align__(16) float sm[];
    float *XT = sm + M::XT, *YT = sm + M::YT, *Yr = sm + M::Yr, *Zs = sm + M::Z, *PT = sm + M::PT, *pw = sm + M::pw, *S = sm + M::S;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, warp = tid >> 5, lane = tid & 31, lr = warp * 8 + (lane >> 2), lf = (lane & 3) * 4;
    pdl_wait();

    if (MAIN && blockIdx.x == 0 && tid == 0) *A.status = 0;     // (nothing here waits: the call's status is known)
    const int nseg = MAIN ? A.nseg : A.nseg - 1;
    int id = blockIdx.x;
    const DecayPass &p = A.pass[id % A.npass]; id /= A.npass;
    const int zt = id % ntz; id /= ntz;
    const int seg = id % nseg, head = id / nseg;            // head: of X, or of the state
    const int z0 = zt * F;
    if (z0 >= p.c) return;
    const int HX = MAIN ? p.HX : A.Hkv;
    const int b = head / HX, hx = head % HX;
    const int hs = hx / (HX / A.Hkv);                        // state and decay
    const int G = p.HY > HX ? p.HY / HX : 1;                 // heads of Y that are summed over
    const int hy0 = p.HY > HX ? hx * G : hx / (HX / p.HY);
    const DecaySpan sp = decay_span<C>(A, b, seg);
    const int a = p.a, c = p.c, nf = (a + F - 1) / F;
    const bool va = a % 4 == 0, vc = c % 4 == 0;
    const bool last = sp.T == 0 ? seg == 0 : sp.k0 < sp.k1 && sp.k1 == sp.T;
    float *S_out = MAIN ? (p.S_out && last && hx % (HX / A.Hkv) == 0 ? p.S_out + (size_t)(b * A.Hkv + hs) * a * c : nullptr)
                        : const_cast<float *>(p.seg) + ((size_t)(b * A.Hkv + hs) * nseg + seg) * a * c;
    T *O = static_cast<T *>(p.O) + (size_t)(b * p.HX + (MAIN ? hx : 0)) * A.N * c;
    if (MAIN && zt == 0) zero_behind<C>(A, sp, seg, O, c, tid, kThreadsS);
    if (sp.k0 == sp.k1 && !(MAIN && last && S_out)) return;

    if (tid <= C) pw[tid] = decay_power(A.log_decay[hs], tid);
    const float *S_in = nullptr;
    if (MAIN) S_in = seg == 0 ? (p.S_in ? p.S_in + (size_t)(b * A.Hkv + hs) * a * c : nullptr) : p.seg + ((size_t)(b * A.Hkv + hs) * (nseg - 1) * A.sub + seg * A.sub - 1) * a * c;
    for (int i = tid; i < nf * F * F; i += kThreadsS) {
        const int f = i / F, z = z0 + i % F;
        S[i] = S_in && f < a && z < c ? (p.trans ? S_in[(size_t)z * a + f] : S_in[(size_t)f * c + z]) : 0.f;
    }
    const T *X = static_cast<const T *>(p.X) + (size_t)(b * p.HX + (MAIN ? hx : 0)) * A.N * a;

    for (int k = sp.k0; k < sp.k1; ++k) {
        const int t0 = (p.reverse ? sp.T - 1 - k : k) * C, L = min(C, sp.n - t0);
        const bool mine = warp * 8 < L;                      // the warp has rows
        Row<4> o[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) o[u].clear();
        for (int g = 0; g < G; ++g) {
            const size_t at = (size_t)(b * p.HY + hy0 + g) * A.N + t0 + lr;
            const T *X1 = X + (size_t)(t0 + lr) * a, *Y = static_cast<const T *>(p.Y) + at * a, *Z = static_cast<const T *>(p.Z) + at * c;
            Row<4> sc[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) sc[u].clear();
            for (int fs = 0; fs < nf; ++fs) {
                float4 lx[4], ly[4], lz[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    lx[j] = ly[j] = lz[j] = make_float4(0, 0, 0, 0);
                    if (lr < L) {
                        ly[j] = load4(Y, fs * F + lf + 16 * j, a, va);
                        if (MAIN) lx[j] = load4(X1, fs * F + lf + 16 * j, a, va);
                        if (fs == 0) lz[j] = load4(Z, z0 + lf + 16 * j, c, vc);
                    }
                }
                __syncthreads();                             // the tiles of the step before have been read; pw and S are there
                const float w = lr < L ? pw[p.reverse ? lr + 1 : L - 1 - lr] * p.tok_mul : 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int f = lf + 16 * j;
                    const float4 x = lx[j], y = ly[j];
                    if (fs == 0) *reinterpret_cast<float4 *>(Zs + lr * F + f) = lz[j];
                    if (MAIN) {
                        XT[f * kPad + lr] = x.x; XT[(f + 1) * kPad + lr] = x.y; XT[(f + 2) * kPad + lr] = x.z; XT[(f + 3) * kPad + lr] = x.w;
                        YT[f * kPad + lr] = y.x; YT[(f + 1) * kPad + lr] = y.y; YT[(f + 2) * kPad + lr] = y.z; YT[(f + 3) * kPad + lr] = y.w;
                    }
                    *reinterpret_cast<float4 *>(Yr + lr * F + f) = make_float4(y.x * w, y.y * w, y.z * w, y.w * w);
                }
                __syncthreads();
                if (MAIN && mine) {
                    products<4, 4, 4>(sc, XT, kPad, YT, kPad, F, ty, tx);
                    if (g == 0 && (S_in || k > sp.k0)) products<4, 4, 4>(o, XT, kPad, S + fs * F * F, F, F, ty, tx);
                }
                if (k + 1 == sp.k1 && !S_out) continue;      // nobody reads the state behind this chunk
                Row<4> d[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) d[u].clear();
                products<4, 4, 4>(d, Yr, F, Zs, F, L, ty, tx);
                if (MAIN && g == 0) __syncthreads();         // the state before this chunk has been read
                const float keep = g == 0 ? pw[L] : 1.f;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    float4 *at4 = reinterpret_cast<float4 *>(S + (fs * F + ty * 4 + u) * F + tx * 4);
                    const float4 s = *at4;
                    *at4 = make_float4(fmaf(keep, s.x, d[u].get(0)), fmaf(keep, s.y, d[u].get(1)), fmaf(keep, s.z, d[u].get(2)), fmaf(keep, s.w, d[u].get(3)));
                }
            }
            if (!MAIN) continue;
            if (g == 0) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int r = ty * 4 + u;
                    o[u].scale(r < L ? pw[p.reverse ? L - 1 - r : r + 1] * p.row_mul : 0.f);
                }
            }
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                float x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int n = p.reverse ? tx * 4 + v - (ty * 4 + u) : ty * 4 + u - (tx * 4 + v);
                    x[u] = n >= 0 ? sc[u].get(v) * (pw[n] * p.p_mul) : 0.f;
                }
                *reinterpret_cast<float4 *>(PT + (tx * 4 + v) * kPad + ty * 4) = make_float4(x[0], x[1], x[2], x[3]);
            }
            __syncthreads();
            const int from = p.reverse ? warp * 8 : 0, to = p.reverse ? L : mine ? min(warp * 8 + 8, L) : 0;
            products<4, 4, 4>(o, PT + from * kPad, kPad, Zs + from * F, F, to - from, ty, tx);
        }
        if (MAIN) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int r = ty * 4 + u;
                if (r >= L) continue;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int z = z0 + tx * 4 + v;
                    if (z < c) O[(size_t)(t0 + r) * c + z] = from_f<T>(o[u].get(v));
                }
            }
        }
    }
    if (S_out) {
        __syncthreads();
        for (int i = tid; i < a * F; i += kThreadsS) {
            const int f = i / F, z = z0 + i % F;
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

template <typename T, int R, bool MAIN>
cudaError_t launch_tile(const DecayArgs &A, cudaStream_t st)
{
    int heads = 0;
    for (int i = 0; i < A.npass; ++i) heads = max(heads, MAIN ? A.B * A.pass[i].HX : A.B * A.Hkv);
    const long long blocks = (long long)A.npass * (MAIN ? A.nseg : A.nseg - 1) * heads;
    // (Ordinary launches up to 148 blocks, so that none start early and go two to an SM: 12 heads of 700 tokens, d 64, 22.9 us for 19.4; at best 2 and 4 %
    // less, 128 and 140 heads in one segment.)
    return launch_pdl(decay_tile_kernel<T, R, MAIN>, dim3((unsigned)blocks), dim3(kThreadsS), TileSmem<R>::total, st, A);
}

template <typename T, bool MAIN>
cudaError_t launch_wide(const DecayArgs &A, cudaStream_t st)
{
    int a = 0, c = 0, heads = 0;
    for (int i = 0; i < A.npass; ++i) {
        a = max(a, A.pass[i].a);
        c = max(c, A.pass[i].c);
        heads = max(heads, MAIN ? A.B * A.pass[i].HX : A.B * A.Hkv);
    }
    const int ntz = (c + F - 1) / F, nseg = MAIN ? A.nseg : A.nseg - 1;
    return launch_pdl(decay_simt_kernel<T, MAIN>, dim3((unsigned)((long long)A.npass * ntz * nseg * heads)), dim3(kThreadsS), SimtSmem::bytes(a), st, A, ntz);
}

template <typename T, bool MAIN>
cudaError_t launch_t(const DecayArgs &A, cudaStream_t st)
{
    int a = 0, c = 0;
    for (int i = 0; i < A.npass; ++i) { a = max(a, A.pass[i].a); c = max(c, A.pass[i].c); }
    const int w = max(a, c);
    return w <= 64 ? launch_tile<T, 4, MAIN>(A, st) : w <= 80 ? launch_tile<T, 5, MAIN>(A, st) : w <= 96 ? launch_tile<T, 6, MAIN>(A, st)
           : w <= 128 ? launch_tile<T, 8, MAIN>(A, st) : launch_wide<T, MAIN>(A, st);
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

// Segments: the cheapest by an estimate in units of the time of a chunk by itself, fitted to fp32 on a B200: two blocks on an SM take 1.35 times as long, a
// chunk of the states alone 0.28, three kernels instead of one about one more.
static void pick(int T, DecayLoad rows, DecayLoad states, int per_sm, int &nseg, int &cps, int &sub)
{
    const auto phase = [&](const DecayLoad &x, long long pieces, int per, double one) {
        const double two = per_sm == 2 ? 1.35 : 1.0;
        const long long blocks = (x.heads + x.sums) * pieces;
        if (x.G > 1) {                                       // the heads that sum over a group take longest
            const double long_one = x.G * (blocks > 148 ? two : 1.0), shared = (double)(x.heads + x.sums * x.G) * pieces / (148 * per_sm) * two;
            return per * one * (long_one > shared ? long_one : shared);
        }
        const long long slots = 148LL * per_sm, rest = blocks % slots;
        return per * one * ((double)(blocks / slots) * two + (rest > 148 ? two : rest ? 1.0 : 0.0));
    };
    nseg = 1; cps = T; sub = 1;
    double best = phase(rows, 1, T, 1.0);
    for (int n = 2; n <= T && n <= 128; ++n) {
        const int per = (T + n - 1) / n, m = (T + per - 1) / per;
        const double cost = phase(rows, m, per, 1.0) + phase(states, m - 1, per, 0.28) + 1.0 + 0.01 * m;
        if (cost < best) { best = cost; nseg = m; cps = per; }
    }
}

void decay_simt_split(darkattn_decay_plan_s *plan)
{
    const darkattn_decay_desc_t &ds = plan->desc;
    const int T = (ds.N + C - 1) / C, w = ds.d > ds.dv ? ds.d : ds.dv;
    const long long zf = w <= 128 ? 1 : (ds.dv + 63) / 64, zb = w <= 128 ? 1 : (w + 63) / 64;      // tiles of the output's columns
    const int per_sm = w <= 80 ? 2 : 1;
    const long long q = (long long)ds.B * ds.H, k = (long long)ds.B * ds.H_kv;
    const int G = ds.H / ds.H_kv;
    pick(T, {q * zf, 0, 1}, {k * zf, 0, 1}, per_sm, plan->fwd.nseg, plan->fwd.cps, plan->fwd.sub);
    pick(T, {q * zb, 2 * k * zb, G}, {k * zf, k * zf, G}, per_sm, plan->bwd.nseg, plan->bwd.cps, plan->bwd.sub);
}

}  // namespace darkattn
