// One token of attention with a decay per head, the recurrent form: per key/value head
//     S <- lambda S + k v^T,   o_h = scale q_h^T S   for the query heads h that share it.
//
// Bound by the state, read and written once. A block takes CT columns of one head's state: its warps take rows in turn, every lane
// four columns of a row; the products with the queries are summed over a thread's rows in registers, over the block's in shared memory.
// The block's whole share of the state is on its way into shared memory before anything else happens (every thread copies what it will use
// itself, so nothing is waited for but a thread's own copies): 128 sequences of 16 heads, 128 x 128 (268 MB to and fro) 47.2 us, 5.7 TB/s, over pools by
// turns. On one pool, in part in L2, 43 to 45 at 64 columns a block, 46 at 32, 49 at 128; with loads into registers 52. 4 sequences: 3.2 us.
#include "decay.cuh"

namespace darkattn {
namespace {

constexpr int kWarps = 8;

template <typename T> __device__ __forceinline__ float ld_f(const T *p);
template <> __device__ __forceinline__ float ld_f<float>(const float *p) { return *p; }
template <> __device__ __forceinline__ float ld_f<__nv_bfloat16>(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st_f(float *p, float x) { *p = x; }
__device__ __forceinline__ void st_f(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }

// Any shape: CT columns a block; W columns a lane (4, or 1 where dv is no multiple of four); kBatch rows a thread holds at a time, in registers
template <typename T, int CT, int W, int kBatch>
__global__ void __launch_bounds__(kWarps * 32) decay_step_kernel(const T *__restrict__ q, const T *__restrict__ k, const T *__restrict__ v,
                                                                 const float *__restrict__ log_decay, float *S, const int *__restrict__ slots, int n_slots,
                                                                 T *o, int Hkv, int G, int d, int dv, float scale)
{
    constexpr int LPR = CT / W, RW = 32 / LPR;               // lanes of a row, rows of a warp at a time
    static_assert(LPR <= 32 && CT <= kWarps * 32, "a row fits a warp, a column has a thread");
    extern __shared__ float sm[];
    float *qs = sm, *ks = qs + G * d, *red = ks + d;         // red: [G][kWarps][CT]
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int h = blockIdx.y % Hkv, b = blockIdx.y / Hkv, col = blockIdx.x * CT + (lane % LPR) * W, row0 = warp * RW + lane / LPR;
    pdl_wait();
    int slot = b;
    if (slots) {
        slot = slots[b];
        if (slot < 0 || slot >= n_slots) return;             // a row of padding
        int taken = 0;
        for (int i = tid; i < b; i += kWarps * 32) taken |= slots[i] == slot;
        if (__syncthreads_or(taken)) return;                 // an earlier row has this slot
    }
    float *St = S + ((size_t)slot * Hkv + h) * d * dv;
    const bool in = col < dv;
    const float lam = expf(log_decay[h]);
    float vv[W], s[kBatch][W];
    auto load = [&](int r0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int r = r0 + i * kWarps * RW;
            if (r < d && in) {
                if (W == 4) *reinterpret_cast<float4 *>(s[i]) = __ldcs(reinterpret_cast<const float4 *>(St + (size_t)r * dv + col));
                else s[i][0] = St[(size_t)r * dv + col];
            } else {
#pragma unroll
                for (int w = 0; w < W; ++w) s[i][w] = 0.f;
            }
        }
    };
    load(row0);
    for (int i = tid; i < G * d; i += kWarps * 32) qs[i] = ld_f(q + ((size_t)b * Hkv + h) * G * d + i);
    for (int i = tid; i < d; i += kWarps * 32) ks[i] = ld_f(k + ((size_t)b * Hkv + h) * d + i);
#pragma unroll
    for (int w = 0; w < W; ++w) vv[w] = in ? ld_f(v + ((size_t)b * Hkv + h) * dv + col + w) : 0.f;
    __syncthreads();
    for (int r0 = row0; r0 < d + row0; r0 += kBatch * kWarps * RW) {     // (all lanes take every turn: they meet in the shuffles)
        if (r0 != row0) load(r0);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int r = r0 + i * kWarps * RW;
            if (r < d && in) {
                const float kr = ks[r];
#pragma unroll
                for (int w = 0; w < W; ++w) s[i][w] = fmaf(kr, vv[w], lam * s[i][w]);
                if (W == 4) __stcs(reinterpret_cast<float4 *>(St + (size_t)r * dv + col), *reinterpret_cast<float4 *>(s[i]));
                else St[(size_t)r * dv + col] = s[i][0];
            }
        }
        for (int g = 0; g < G; ++g) {
            float acc[W];
#pragma unroll
            for (int w = 0; w < W; ++w) acc[w] = 0.f;
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int r = r0 + i * kWarps * RW;
                const float qr = r < d ? qs[g * d + r] : 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) acc[w] = fmaf(qr, s[i][w], acc[w]);
            }
#pragma unroll
            for (int m = LPR; m < 32; m *= 2)
#pragma unroll
                for (int w = 0; w < W; ++w) acc[w] += __shfl_xor_sync(0xffffffffu, acc[w], m);
            if (lane < LPR) {
                float *at = red + (g * kWarps + warp) * CT + lane * W;
#pragma unroll
                for (int w = 0; w < W; ++w) at[w] = r0 == row0 ? acc[w] : at[w] + acc[w];
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < G * CT; i += kWarps * 32) {
        const int g = i / CT, z = i % CT, c = blockIdx.x * CT + z;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) sum += red[(g * kWarps + w) * CT + z];
        if (c < dv) st_f(o + (((size_t)b * Hkv + h) * G + g) * dv + c, scale * sum);
    }
}

// Waits until at most n groups of asynchronous copies are on their way.
__device__ __forceinline__ void copies_left(int n)
{
    if (n == 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
    else if (n == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else if (n == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

// ROWS rows of a thread, four of them in registers at a time
template <typename T, int CT, int ROWS>
__global__ void __launch_bounds__(kWarps * 32) decay_step_async_kernel(const T *__restrict__ q, const T *__restrict__ k, const T *__restrict__ v,
                                                                       const float *__restrict__ log_decay, float *S, const int *__restrict__ slots, int n_slots,
                                                                       T *o, int Hkv, int G, int d, int dv, float scale)
{
    constexpr int LPR = CT / 4, RW = 32 / LPR, kTurn = 4;    // lanes of a row, rows of a warp at a time, rows of a thread a turn
    static_assert(ROWS % kTurn == 0 && ROWS / kTurn <= 4, "groups of copies");
    extern __shared__ float4 sm4[];                          // [ROWS][kWarps * 32], then the queries, the key and the sums
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int h = blockIdx.y % Hkv, b = blockIdx.y / Hkv, col = blockIdx.x * CT + (lane % LPR) * 4, row0 = warp * RW + lane / LPR;
    float *qs = reinterpret_cast<float *>(sm4 + ROWS * kWarps * 32), *ks = qs + G * d, *red = ks + d;
    pdl_wait();
    int slot = b;
    if (slots) {
        slot = slots[b];
        if (slot < 0 || slot >= n_slots) return;             // a row of padding
    }
    float *St = S + ((size_t)slot * Hkv + h) * d * dv;
    const bool in = col < dv;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = row0 + i * kWarps * RW;
        if (r < d && in)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(sm4 + i * kWarps * 32 + tid)), "l"(St + (size_t)r * dv + col) : "memory");
        if (i % kTurn == kTurn - 1) asm volatile("cp.async.commit_group;" ::: "memory");
    }
    if (slots) {
        int taken = 0;
        for (int i = tid; i < b; i += kWarps * 32) taken |= slots[i] == slot;
        if (__syncthreads_or(taken)) {                       // an earlier row has this slot
            asm volatile("cp.async.wait_all;" ::: "memory");
            return;
        }
    }
    const float lam = expf(log_decay[h]);
    for (int i = tid; i < G * d; i += kWarps * 32) qs[i] = ld_f(q + ((size_t)b * Hkv + h) * G * d + i);
    for (int i = tid; i < d; i += kWarps * 32) ks[i] = ld_f(k + ((size_t)b * Hkv + h) * d + i);
    float vv[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) vv[w] = in ? ld_f(v + ((size_t)b * Hkv + h) * dv + col + w) : 0.f;
    __syncthreads();
#pragma unroll
    for (int i0 = 0; i0 < ROWS; i0 += kTurn) {
        copies_left((ROWS - i0) / kTurn - 1);
        float s[kTurn][4];
#pragma unroll
        for (int i = 0; i < kTurn; ++i) {
            const int r = row0 + (i0 + i) * kWarps * RW;
            float4 x = make_float4(0, 0, 0, 0);
            if (r < d && in) {
                x = sm4[(i0 + i) * kWarps * 32 + tid];
                const float kr = ks[r];
                x.x = fmaf(kr, vv[0], lam * x.x); x.y = fmaf(kr, vv[1], lam * x.y); x.z = fmaf(kr, vv[2], lam * x.z); x.w = fmaf(kr, vv[3], lam * x.w);
                __stcs(reinterpret_cast<float4 *>(St + (size_t)r * dv + col), x);
            }
            s[i][0] = x.x; s[i][1] = x.y; s[i][2] = x.z; s[i][3] = x.w;
        }
        for (int g = 0; g < G; ++g) {
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kTurn; ++i) {
                const int r = row0 + (i0 + i) * kWarps * RW;
                const float qr = r < d ? qs[g * d + r] : 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) acc[w] = fmaf(qr, s[i][w], acc[w]);
            }
#pragma unroll
            for (int m = LPR; m < 32; m *= 2)
#pragma unroll
                for (int w = 0; w < 4; ++w) acc[w] += __shfl_xor_sync(0xffffffffu, acc[w], m);
            if (lane < LPR) {
                float *at = red + (g * kWarps + warp) * CT + lane * 4;
#pragma unroll
                for (int w = 0; w < 4; ++w) at[w] = i0 == 0 ? acc[w] : at[w] + acc[w];
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < G * CT; i += kWarps * 32) {
        const int g = i / CT, z = i % CT, c = blockIdx.x * CT + z;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) sum += red[(g * kWarps + w) * CT + z];
        if (c < dv) st_f(o + (((size_t)b * Hkv + h) * G + g) * dv + c, scale * sum);
    }
}

template <typename T, int CT, int ROWS>
cudaError_t launch_async(const darkattn_decay_desc_t &ds, const void *q, const void *k, const void *v, const float *log_decay, float *S, const int *slots, int n_slots,
                         void *o, cudaStream_t st)
{
    const int G = ds.H / ds.H_kv, smem = ROWS * kWarps * 32 * 16 + 4 * (G * ds.d + ds.d + G * kWarps * CT);
    return launch_pdl(decay_step_async_kernel<T, CT, ROWS>, dim3((unsigned)((ds.dv + CT - 1) / CT), (unsigned)(ds.B * ds.H_kv)), dim3(kWarps * 32), smem, st,
                      static_cast<const T *>(q), static_cast<const T *>(k), static_cast<const T *>(v), log_decay, S, slots, n_slots, static_cast<T *>(o), ds.H_kv, G,
                      ds.d, ds.dv, ds.scale);
}

template <typename T, int CT, int W, int kBatch>
cudaError_t launch(const darkattn_decay_desc_t &ds, const void *q, const void *k, const void *v, const float *log_decay, float *S, const int *slots, int n_slots,
                   void *o, cudaStream_t st)
{
    const int G = ds.H / ds.H_kv, smem = 4 * (G * ds.d + ds.d + G * kWarps * CT);
    return launch_pdl(decay_step_kernel<T, CT, W, kBatch>, dim3((unsigned)((ds.dv + CT - 1) / CT), (unsigned)(ds.B * ds.H_kv)), dim3(kWarps * 32), smem, st,
                      static_cast<const T *>(q), static_cast<const T *>(k), static_cast<const T *>(v), log_decay, S, slots, n_slots, static_cast<T *>(o), ds.H_kv, G,
                      ds.d, ds.dv, ds.scale);
}

template <typename T>
cudaError_t launch_t(const darkattn_decay_desc_t &ds, const void *q, const void *k, const void *v, const float *log_decay, float *S, const int *slots, int n_slots,
                     void *o, cudaStream_t st)
{
    const int G = ds.H / ds.H_kv;
    if (ds.dv % 4 == 0 && ds.d <= 256 && G <= 32) {
#define GO(ct, rows) return launch_async<T, ct, rows>(ds, q, k, v, log_decay, S, slots, n_slots, o, st)
        if (ds.dv <= 32) {
            if (ds.d <= 128) GO(32, 4);
            GO(32, 8);
        }
        if (ds.d <= 64) GO(64, 4);
        if (ds.d <= 128) GO(64, 8);
        GO(64, 16);
#undef GO
    }
    return ds.dv % 4 ? launch<T, 32, 1, 16>(ds, q, k, v, log_decay, S, slots, n_slots, o, st) : launch<T, 32, 4, 16>(ds, q, k, v, log_decay, S, slots, n_slots, o, st);
}

}  // namespace

darkattn_status_t decay_step(const darkattn_decay_plan_s *plan, const void *q, const void *k, const void *v, const float *log_decay, float *S, const int *slots,
                             int n_slots, void *o, cudaStream_t st)
{
    const darkattn_decay_desc_t &ds = plan->desc;
    // shared memory of the narrowest block: the queries of a group and their sums
    if (4ll * ((ds.H / ds.H_kv) * (ds.d + kWarps * 32) + ds.d) > 200 * 1024) return DARKATTN_ERR_UNSUPPORTED;
    const size_t e = ds.dtype == DARKATTN_BF16 ? 2 : 4, B = (size_t)ds.B;
    if (clash({{o, B * ds.H * ds.dv * e}, {S, (size_t)n_slots * ds.H_kv * ds.d * ds.dv * 4}},
              {{q, B * ds.H * ds.d * e}, {k, B * ds.H_kv * ds.d * e}, {v, B * ds.H_kv * ds.dv * e}, {log_decay, (size_t)ds.H_kv * 4}, {slots, B * 4}})) return DARKATTN_ERR_INVALID_ARG;
    const cudaError_t rc = ds.dtype == DARKATTN_BF16 ? launch_t<__nv_bfloat16>(ds, q, k, v, log_decay, S, slots, n_slots, o, st)
                                                    : launch_t<float>(ds, q, k, v, log_decay, S, slots, n_slots, o, st);
    DARKATTN_CUDA_TRY(rc, "decay_step_kernel");
    return DARKATTN_OK;
}

}  // namespace darkattn
