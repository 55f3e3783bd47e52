// Running states kept in 8 bits: a row of `cols` numbers becomes as many codes and one scale,
//     scale = max |x| / top  (in 32 bits; top = 127 for signed integers, 448 for e4m3),   code = x / scale, rounded to nearest, ties to even.
// The quotient's rounding counts once: it is taken to 32 bits by rounding to odd (what its division left out sets the last bit), so that
// the rounding to the code's few bits sees on which side of a border the exact quotient lies.
//
// Bound by the traffic, 5 bytes an element; a warp takes four rows at a time, so that enough loads are on their way.
#include "decay.cuh"

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
// Codes of four numbers, a byte each. Where the products with a little less and a little more than 1 / s (which bracket the quotients) round to
// the same codes, those are it; only next to a border (one element in some hundred thousand) the quotient is taken. Divisions for all
// took 38 us for 25 million numbers where their bytes take 20.
template <bool E4M3>
__device__ __forceinline__ unsigned codes4(float4 x, float s, float below, float above)
{
    unsigned a, b;
    if (E4M3) {
        const auto four = [&](float r) {
            return (unsigned)__nv_cvt_float2_to_fp8x2(make_float2(x.x * r, x.y * r), __NV_SATFINITE, __NV_E4M3) |
                   (unsigned)__nv_cvt_float2_to_fp8x2(make_float2(x.z * r, x.w * r), __NV_SATFINITE, __NV_E4M3) << 16;
        };
        a = four(below);
        b = four(above);
    } else {                                 // 1.5 2^23 added: rounded to an integer, in the last byte, by the one rounding of the sum
        const float big = 12582912.f;
        const auto four = [&](float r) {
            const unsigned p = __byte_perm(__float_as_uint(fmaf(x.x, r, big)), __float_as_uint(fmaf(x.y, r, big)), 0x0040);
            return __byte_perm(p, __byte_perm(__float_as_uint(fmaf(x.z, r, big)), __float_as_uint(fmaf(x.w, r, big)), 0x0040), 0x5410);
        };
        a = four(below);
        b = four(above);
    }
    if (a == b) return a;
    return code<E4M3>(x.x, s) | code<E4M3>(x.y, s) << 8 | code<E4M3>(x.z, s) << 16 | code<E4M3>(x.w, s) << 24;
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
__device__ __forceinline__ int magnitude(float x) { return __float_as_int(x) & 0x7fffffff; }
// Row of the cache that holds sequence b; -1 where it has none.
__device__ __forceinline__ int slot_of(const int *slots, int n_slots, int b)
{
    const int s = slots ? slots[b] : b;
    return s >= 0 && s < n_slots ? s : -1;
}
// Whether an earlier row names the slot (of several that do only the first counts)
__device__ __forceinline__ bool taken_before(const int *slots, int b, int slot)
{
    if (!slots) return false;
    int taken = 0;
    for (int i = threadIdx.x; i < b; i += kWarps * 32) taken |= slots[i] == slot;
    return __syncthreads_or(taken);
}

// V: vectors of four a lane holds of each row; L: lanes of a row (cols <= 4 L V, a multiple of four: with all 32 on rows of 64 numbers half of them
// had nothing to do, 12.4 us for what now takes 8.7). V = 0: any cols, the row read twice
template <bool E4M3, int V, int L>
__global__ void __launch_bounds__(kWarps * 32) state_store_kernel(const float *__restrict__ S, const int *__restrict__ slots, int n_slots, int rows, int cols,
                                                                  unsigned char *codes, float *scales)
{
    const int b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r0 = (blockIdx.x * kWarps + warp) * kRows * (32 / L) + lane / L;
    pdl_wait();
    const int slot = slot_of(slots, n_slots, b);
    if (slot < 0) return;
    const float *src = S + (size_t)b * rows * cols;
    unsigned char *dst = codes + (size_t)slot * rows * cols;
    if constexpr (V > 0) {
        float4 x[kRows][V];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i * L + lane % L) * 4;
                x[r][i] = r0 + r * (32 / L) < rows && c < cols ? __ldcs(reinterpret_cast<const float4 *>(src + (size_t)(r0 + r * (32 / L)) * cols + c)) : make_float4(0, 0, 0, 0);
            }
        if (taken_before(slots, b, slot)) return;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            int amax = 0;                                    // magnitudes are ordered like their bits, infinities and NaN behind all numbers
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float4 f = x[r][i];
                amax = max(max(amax, max(magnitude(f.x), magnitude(f.y))), max(magnitude(f.z), magnitude(f.w)));
            }
            if (L == 32) amax = __reduce_max_sync(0xffffffffu, amax);
            else {
#pragma unroll
                for (int m = L / 2; m; m /= 2) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, m));
            }
            const float s = scale_of<E4M3>(__int_as_float(amax), amax < 0x7f800000);
            if (r0 + r * (32 / L) >= rows) continue;
            if (lane % L == 0) scales[(size_t)slot * rows + r0 + r * (32 / L)] = s;
            // 1 / s to 2^-24 and a product to 2^-24 lie well inside of 2^-21; a scale without a plain reciprocal (0, NaN, far out) brackets nothing
            const bool plain = s > 1e-30f && s < 1e30f;
            const float inv = 1.f / s, below = plain ? inv * (1.f - 0x1p-21f) : 0.f, above = plain ? inv * (1.f + 0x1p-21f) : __int_as_float(0x7fc00000);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i * L + lane % L) * 4;
                if (c < cols) *reinterpret_cast<unsigned *>(dst + (size_t)(r0 + r * (32 / L)) * cols + c) = codes4<E4M3>(x[r][i], s, below, above);
            }
        }
    } else if (!taken_before(slots, b, slot)) for (int r = r0; r < min(r0 + kRows, rows); ++r) {
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

template <bool E4M3, int V, int L>
__global__ void __launch_bounds__(kWarps * 32) state_load_kernel(const unsigned char *__restrict__ codes, const float *__restrict__ scales,
                                                                 const int *__restrict__ slots, int n_slots, int rows, int cols, float *S)
{
    const int b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r0 = (blockIdx.x * kWarps + warp) * kRows * (32 / L) + lane / L;
    pdl_wait();
    const int slot = slot_of(slots, n_slots, b);
    if (slot < 0) return;
    const unsigned char *src = codes + (size_t)slot * rows * cols;
    float *dst = S + (size_t)b * rows * cols;
    if constexpr (V > 0) {
        unsigned x[kRows][V];
        float s[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            s[r] = r0 + r * (32 / L) < rows ? scales[(size_t)slot * rows + r0 + r * (32 / L)] : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i * L + lane % L) * 4;
                x[r][i] = r0 + r * (32 / L) < rows && c < cols ? __ldcs(reinterpret_cast<const unsigned *>(src + (size_t)(r0 + r * (32 / L)) * cols + c)) : 0u;
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i * L + lane % L) * 4;
                const unsigned w = x[r][i];
                if (r0 + r * (32 / L) < rows && c < cols)
                    *reinterpret_cast<float4 *>(dst + (size_t)(r0 + r * (32 / L)) * cols + c) =
                        make_float4(value<E4M3>(w & 0xff) * s[r], value<E4M3>(w >> 8 & 0xff) * s[r], value<E4M3>(w >> 16 & 0xff) * s[r], value<E4M3>(w >> 24) * s[r]);
            }
    } else for (int r = r0; r < min(r0 + kRows, rows); ++r) {
        const float s = scales[(size_t)slot * rows + r];
        for (int c = lane; c < cols; c += 32) dst[(size_t)r * cols + c] = value<E4M3>(src[(size_t)r * cols + c]) * s;
    }
}

template <int V, int L>
cudaError_t store(const float *S, const int *slots, int n_slots, int B, int rows, int cols, int e4m3, unsigned char *codes, float *scales, cudaStream_t st)
{
    const dim3 grid((unsigned)((rows + kBlockRows * (32 / L) - 1) / (kBlockRows * (32 / L))), (unsigned)B);
    return e4m3 ? launch_pdl(state_store_kernel<true, V, L>, grid, dim3(kWarps * 32), 0, st, S, slots, n_slots, rows, cols, codes, scales)
                : launch_pdl(state_store_kernel<false, V, L>, grid, dim3(kWarps * 32), 0, st, S, slots, n_slots, rows, cols, codes, scales);
}
template <int V, int L>
cudaError_t load(const unsigned char *codes, const float *scales, const int *slots, int n_slots, int B, int rows, int cols, int e4m3, float *S, cudaStream_t st)
{
    const dim3 grid((unsigned)((rows + kBlockRows * (32 / L) - 1) / (kBlockRows * (32 / L))), (unsigned)B);
    return e4m3 ? launch_pdl(state_load_kernel<true, V, L>, grid, dim3(kWarps * 32), 0, st, codes, scales, slots, n_slots, rows, cols, S)
                : launch_pdl(state_load_kernel<false, V, L>, grid, dim3(kWarps * 32), 0, st, codes, scales, slots, n_slots, rows, cols, S);
}

darkattn_status_t check(int B, int rows, int cols, int n_slots, int format, const void *S, const void *codes, const void *scales, const void *slots, bool store)
{
    const auto low = [](const void *p) { return reinterpret_cast<uintptr_t>(p) & 15u; };
    if (B < 1 || rows < 1 || cols < 1 || n_slots < 1 || (!slots && n_slots < B) || !S || !codes || !scales) return DARKATTN_ERR_INVALID_ARG;
    if (format != DARKATTN_STATE_I8 && format != DARKATTN_STATE_E4M3) return DARKATTN_ERR_INVALID_ARG;
    if (low(S) || low(codes) || low(scales) || (low(slots) & 3u)) return DARKATTN_ERR_INVALID_ARG;
    if (B > 65535 || rows > 1 << 30 || cols > 1 << 30) return DARKATTN_ERR_UNSUPPORTED;       // (a row's and a column's index in 32 bits, a block's step behind the end too)
    const size_t r = (size_t)rows, c = (size_t)cols;
    const Span state = {S, B * r * c * 4}, kept = {codes, n_slots * r * c}, scale = {scales, n_slots * r * 4}, at = {slots, (size_t)B * 4};
    return (store ? clash({kept, scale}, {state, at}) : clash({state}, {kept, scale, at})) ? DARKATTN_ERR_INVALID_ARG : DARKATTN_OK;
}

}  // namespace
}  // namespace darkattn

using namespace darkattn;

extern "C" {

darkattn_status_t darkattn_state_store(int32_t B, int32_t rows, int32_t cols, const float *S, const int32_t *slots, int32_t n_slots, int32_t format, void *codes,
                                       float *scales, void *cuda_stream)
{
    if (darkattn_status_t rc = check(B, rows, cols, n_slots, format, S, codes, scales, slots, true)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    unsigned char *c = static_cast<unsigned char *>(codes);
    const cudaError_t e = cols % 4 || cols > 256 ? store<0, 32>(S, slots, n_slots, B, rows, cols, format, c, scales, st)
                          : cols <= 32           ? store<1, 8>(S, slots, n_slots, B, rows, cols, format, c, scales, st)
                          : cols <= 64           ? store<1, 16>(S, slots, n_slots, B, rows, cols, format, c, scales, st)
                          : cols <= 128          ? store<1, 32>(S, slots, n_slots, B, rows, cols, format, c, scales, st)
                                                 : store<2, 32>(S, slots, n_slots, B, rows, cols, format, c, scales, st);
    DARKATTN_CUDA_TRY(e, "state_store_kernel");
    return DARKATTN_OK;
}

darkattn_status_t darkattn_state_load(int32_t B, int32_t rows, int32_t cols, const void *codes, const float *scales, const int32_t *slots, int32_t n_slots, int32_t format,
                                      float *S, void *cuda_stream)
{
    if (darkattn_status_t rc = check(B, rows, cols, n_slots, format, S, codes, scales, slots, false)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const unsigned char *c = static_cast<const unsigned char *>(codes);
    const cudaError_t e = cols % 4 || cols > 256 ? load<0, 32>(c, scales, slots, n_slots, B, rows, cols, format, S, st)
                          : cols <= 32           ? load<1, 8>(c, scales, slots, n_slots, B, rows, cols, format, S, st)
                          : cols <= 64           ? load<1, 16>(c, scales, slots, n_slots, B, rows, cols, format, S, st)
                          : cols <= 128          ? load<1, 32>(c, scales, slots, n_slots, B, rows, cols, format, S, st)
                                                 : load<2, 32>(c, scales, slots, n_slots, B, rows, cols, format, S, st);
    DARKATTN_CUDA_TRY(e, "state_load_kernel");
    return DARKATTN_OK;
}

}  // extern "C"
