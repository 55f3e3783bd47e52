// Running states kept in 8 bits: a row of `cols` numbers becomes as many codes and one scale,
//     scale = max |x| / top  (in 32 bits; top = 127 for signed integers, 448 for e4m3),   code = x / scale, rounded to nearest, ties to even.
// The quotient's rounding counts once: it is taken to 32 bits by rounding to odd (what its division left out sets the last bit), so that
// the rounding to the code's few bits sees on which side of a border the exact quotient lies.
//
// Bound by the traffic, 5 bytes an element; a warp takes four rows at a time, so that enough loads are on their way.
#include "common.cuh"

#include <cuda_fp8.h>
#include <float.h>

namespace darkattn {
namespace {

constexpr int kWarps = 8, kRows = 4;         // rows a warp takes at a time
constexpr int kBlockRows = kWarps * kRows;

__device__ __forceinline__ float quotient_odd(float x, float s)
{
    const float q = x / s, rest = fmaf(-q, s, x);
    const int bits = __float_as_int(q);
    if (rest == 0.f || (bits & 1) || q == 0.f) return q;
    return __int_as_float((rest > 0.f) == (q > 0.f) ? bits + 1 : bits - 1);      // (scales are positive)
}
template <bool E4M3>
__device__ __forceinline__ unsigned code(float x, float s)
{
    if (!(s > 0.f)) return 0;                // a row of zeros, or one that holds what is not finite
    const float q = quotient_odd(x, s);
    if (E4M3) return __nv_cvt_float_to_fp8(q, __NV_SATFINITE, __NV_E4M3);
    return (unsigned)(int)fminf(fmaxf(rintf(q), -127.f), 127.f) & 0xffu;
}
template <bool E4M3>
__device__ __forceinline__ float value(unsigned c)
{
    if (E4M3) return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)c, __NV_E4M3)));
    return (float)(signed char)c;
}
// top such that scale = max / top; NaN where the row holds what is not finite
template <bool E4M3>
__device__ __forceinline__ float scale_of(float amax, bool finite)
{
    return finite ? amax / (E4M3 ? 448.f : 127.f) : __int_as_float(0x7fc00000);
}
// Row of the cache that holds sequence b; -1 where it has none. `first`: only the first of several rows that name one slot counts.
__device__ __forceinline__ int slot_of(const int *slots, int n_slots, int b, bool first)
{
    if (!slots) return b;
    const int s = slots[b];
    if (s < 0 || s >= n_slots) return -1;
    if (!first) return s;
    int taken = 0;
    for (int i = threadIdx.x; i < b; i += kWarps * 32) taken |= slots[i] == s;
    return __syncthreads_or(taken) ? -1 : s;
}

// V: vectors of four a lane holds of each row (cols <= 128 V, a multiple of four); 0: any cols, the row read twice
template <bool E4M3, int V>
__global__ void __launch_bounds__(kWarps * 32) state_store_kernel(const float *__restrict__ S, const int *__restrict__ slots, int n_slots, int rows, int cols,
                                                                  unsigned char *codes, float *scales)
{
    const int b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r0 = blockIdx.x * kBlockRows + warp * kRows;
    pdl_wait();
    const int slot = slot_of(slots, n_slots, b, true);
    if (slot < 0) return;
    const float *src = S + (size_t)b * rows * cols;
    unsigned char *dst = codes + (size_t)slot * rows * cols;
    if constexpr (V > 0) {
        float4 x[kRows][V];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i * 32 + lane) * 4;
                x[r][i] = r0 + r < rows && c < cols ? __ldcs(reinterpret_cast<const float4 *>(src + (size_t)(r0 + r) * cols + c)) : make_float4(0, 0, 0, 0);
            }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            float amax = 0.f;
            bool finite = true;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float4 f = x[r][i];
                amax = fmaxf(fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y))), fmaxf(fabsf(f.z), fabsf(f.w)));
                finite = finite && fabsf(f.x) <= FLT_MAX && fabsf(f.y) <= FLT_MAX && fabsf(f.z) <= FLT_MAX && fabsf(f.w) <= FLT_MAX;
            }
            amax = __int_as_float(__reduce_max_sync(0xffffffffu, __float_as_int(amax)));      // (not negative: ordered like their bits)
            const float s = scale_of<E4M3>(amax, __all_sync(0xffffffffu, finite));
            if (r0 + r >= rows) continue;
            if (lane == 0) scales[(size_t)slot * rows + r0 + r] = s;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i * 32 + lane) * 4;
                const float4 f = x[r][i];
                if (c < cols)
                    *reinterpret_cast<unsigned *>(dst + (size_t)(r0 + r) * cols + c) =
                        code<E4M3>(f.x, s) | code<E4M3>(f.y, s) << 8 | code<E4M3>(f.z, s) << 16 | code<E4M3>(f.w, s) << 24;
            }
        }
    } else for (int r = r0; r < min(r0 + kRows, rows); ++r) {
        float amax = 0.f;
        bool finite = true;
        for (int c = lane; c < cols; c += 32) {
            const float f = fabsf(src[(size_t)r * cols + c]);
            amax = fmaxf(amax, f);
            finite = finite && f <= FLT_MAX;
        }
        amax = __int_as_float(__reduce_max_sync(0xffffffffu, __float_as_int(amax)));
        const float s = scale_of<E4M3>(amax, __all_sync(0xffffffffu, finite));
        if (lane == 0) scales[(size_t)slot * rows + r] = s;
        for (int c = lane; c < cols; c += 32) dst[(size_t)r * cols + c] = (unsigned char)code<E4M3>(src[(size_t)r * cols + c], s);
    }
}

template <bool E4M3, int V>
__global__ void __launch_bounds__(kWarps * 32) state_load_kernel(const unsigned char *__restrict__ codes, const float *__restrict__ scales,
                                                                 const int *__restrict__ slots, int n_slots, int rows, int cols, float *S)
{
    const int b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r0 = blockIdx.x * kBlockRows + warp * kRows;
    pdl_wait();
    const int slot = slot_of(slots, n_slots, b, false);
    if (slot < 0) return;
    const unsigned char *src = codes + (size_t)slot * rows * cols;
    float *dst = S + (size_t)b * rows * cols;
    if constexpr (V > 0) {
        unsigned x[kRows][V];
        float s[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            s[r] = r0 + r < rows ? scales[(size_t)slot * rows + r0 + r] : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i * 32 + lane) * 4;
                x[r][i] = r0 + r < rows && c < cols ? __ldcs(reinterpret_cast<const unsigned *>(src + (size_t)(r0 + r) * cols + c)) : 0u;
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i * 32 + lane) * 4;
                const unsigned w = x[r][i];
                if (r0 + r < rows && c < cols)
                    *reinterpret_cast<float4 *>(dst + (size_t)(r0 + r) * cols + c) =
                        make_float4(value<E4M3>(w & 0xff) * s[r], value<E4M3>(w >> 8 & 0xff) * s[r], value<E4M3>(w >> 16 & 0xff) * s[r], value<E4M3>(w >> 24) * s[r]);
            }
    } else for (int r = r0; r < min(r0 + kRows, rows); ++r) {
        const float s = scales[(size_t)slot * rows + r];
        for (int c = lane; c < cols; c += 32) dst[(size_t)r * cols + c] = value<E4M3>(src[(size_t)r * cols + c]) * s;
    }
}

template <int V>
cudaError_t store(const float *S, const int *slots, int n_slots, int B, int rows, int cols, int e4m3, unsigned char *codes, float *scales, cudaStream_t st)
{
    const dim3 grid((unsigned)((rows + kBlockRows - 1) / kBlockRows), (unsigned)B);
    return e4m3 ? launch_pdl(state_store_kernel<true, V>, grid, dim3(kWarps * 32), 0, st, S, slots, n_slots, rows, cols, codes, scales)
                : launch_pdl(state_store_kernel<false, V>, grid, dim3(kWarps * 32), 0, st, S, slots, n_slots, rows, cols, codes, scales);
}
template <int V>
cudaError_t load(const unsigned char *codes, const float *scales, const int *slots, int n_slots, int B, int rows, int cols, int e4m3, float *S, cudaStream_t st)
{
    const dim3 grid((unsigned)((rows + kBlockRows - 1) / kBlockRows), (unsigned)B);
    return e4m3 ? launch_pdl(state_load_kernel<true, V>, grid, dim3(kWarps * 32), 0, st, codes, scales, slots, n_slots, rows, cols, S)
                : launch_pdl(state_load_kernel<false, V>, grid, dim3(kWarps * 32), 0, st, codes, scales, slots, n_slots, rows, cols, S);
}

darkattn_status_t check(int B, int rows, int cols, int n_slots, int format, const void *S, const void *codes, const void *scales, const void *slots)
{
    const auto low = [](const void *p) { return reinterpret_cast<uintptr_t>(p) & 15u; };
    if (B < 1 || rows < 1 || cols < 1 || n_slots < 1 || (!slots && n_slots < B) || !S || !codes || !scales) return DARKATTN_ERR_INVALID_ARG;
    if (format != DARKATTN_STATE_I8 && format != DARKATTN_STATE_E4M3) return DARKATTN_ERR_INVALID_ARG;
    if (low(S) || low(codes) || low(scales) || (low(slots) & 3u)) return DARKATTN_ERR_INVALID_ARG;
    return B > 65535 ? DARKATTN_ERR_UNSUPPORTED : DARKATTN_OK;
}

}  // namespace
}  // namespace darkattn

using namespace darkattn;

extern "C" {

darkattn_status_t darkattn_state_store(int32_t B, int32_t rows, int32_t cols, const float *S, const int32_t *slots, int32_t n_slots, int32_t format, void *codes,
                                       float *scales, void *cuda_stream)
{
    if (darkattn_status_t rc = check(B, rows, cols, n_slots, format, S, codes, scales, slots)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    unsigned char *c = static_cast<unsigned char *>(codes);
    const cudaError_t e = cols % 4 || cols > 256 ? store<0>(S, slots, n_slots, B, rows, cols, format, c, scales, st)
                          : cols <= 128          ? store<1>(S, slots, n_slots, B, rows, cols, format, c, scales, st)
                                                 : store<2>(S, slots, n_slots, B, rows, cols, format, c, scales, st);
    DARKATTN_CUDA_TRY(e, "state_store_kernel");
    return DARKATTN_OK;
}

darkattn_status_t darkattn_state_load(int32_t B, int32_t rows, int32_t cols, const void *codes, const float *scales, const int32_t *slots, int32_t n_slots, int32_t format,
                                      float *S, void *cuda_stream)
{
    if (darkattn_status_t rc = check(B, rows, cols, n_slots, format, S, codes, scales, slots)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const unsigned char *c = static_cast<const unsigned char *>(codes);
    const cudaError_t e = cols % 4 || cols > 256 ? load<0>(c, scales, slots, n_slots, B, rows, cols, format, S, st)
                          : cols <= 128          ? load<1>(c, scales, slots, n_slots, B, rows, cols, format, S, st)
                                                 : load<2>(c, scales, slots, n_slots, B, rows, cols, format, S, st);
    DARKATTN_CUDA_TRY(e, "state_load_kernel");
    return DARKATTN_OK;
}

}  // extern "C"
