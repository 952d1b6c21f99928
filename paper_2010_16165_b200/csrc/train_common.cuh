// What the training-step kernels share: 16- and 32-bit element types, activations, checks of device buffers.
#pragma once

#include "../../include/fupruner.h"
#include "fp_internal.h"

#include <cuda_fp16.h>

namespace fp_detail { fp_status set_error(fp_status st, const char* msg); }

namespace fp {
namespace train {

// Errors of one entry point: sets the message and returns the status.
inline fp_status err(fp_status st, const char* msg) { return fp_detail::set_error(st, msg); }

inline bool is_half(int dtype) { return dtype == FP_DTYPE_BF16 || dtype == FP_DTYPE_F16; }
inline int elem_bytes(int dtype) { return dtype == FP_DTYPE_F32 ? 4 : 2; }

// A kernel that gets a host pointer, or one of a GPU that this one cannot read, faults, and takes the context with it: so the
// driver is asked about every buffer of a call (allowed while a stream is captured).  It names the allocation that an address
// lies in, and a program's buffers lie in few, so the 800 addresses of a network's step cost a handful of questions.
class Buffers {
public:
    explicit Buffers(int dev) : dev_(dev) {}
    bool here(const void* p) {
        const uint64_t a = (uint64_t)(uintptr_t)p;
        for (int i = 0; i < n_; ++i)
            if (a - start_[i] < size_[i]) return true;
        uint64_t start = 0, size = 0;
        if (!ask(a, &start, &size)) return false;
        const int at = n_ < kKept ? n_++ : (next_ = (next_ + 1) % kKept);
        start_[at] = start; size_[at] = size;
        return true;
    }
    bool here_or_null(const void* p) { return !p || here(p); }

private:
    bool ask(uint64_t a, uint64_t* start, uint64_t* size) const;
    static constexpr int kKept = 8;
    uint64_t start_[kKept], size_[kKept];
    int dev_, n_ = 0, next_ = 0;
};

// A function of the CUDA driver by name, or nullptr.
void* driver_function(const char* name, std::atomic<void*>* known);

// ---- elements -------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float to_f32(uint16_t bits, int dtype) {
    return dtype == FP_DTYPE_BF16 ? __uint_as_float((uint32_t)bits << 16) : __half2float(__ushort_as_half(bits));
}
__device__ __forceinline__ uint16_t to_16(float v, int dtype) {
    return dtype == FP_DTYPE_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}
__device__ __forceinline__ uint32_t to_16x2(float lo, float hi, int dtype) {
    uint32_t r;
    if (dtype == FP_DTYPE_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float load1(const void* base, long long at, int dtype) {
    return dtype == FP_DTYPE_F32 ? static_cast<const float*>(base)[at] : to_f32(static_cast<const uint16_t*>(base)[at], dtype);
}
__device__ __forceinline__ void store1(void* base, long long at, int dtype, float v) {
    if (dtype == FP_DTYPE_F32) static_cast<float*>(base)[at] = v;
    else static_cast<uint16_t*>(base)[at] = to_16(v, dtype);
}
// Four neighbours; `at` is a multiple of four elements of a base aligned to four.
__device__ __forceinline__ void load4(const void* base, long long at, int dtype, float (&v)[4]) {
    if (dtype == FP_DTYPE_F32) {
        const float4 u = *reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
        v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
    } else {
        const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(base) + at);
        v[0] = to_f32((uint16_t)u.x, dtype); v[1] = to_f32((uint16_t)(u.x >> 16), dtype);
        v[2] = to_f32((uint16_t)u.y, dtype); v[3] = to_f32((uint16_t)(u.y >> 16), dtype);
    }
}
__device__ __forceinline__ void store4(void* base, long long at, int dtype, const float (&v)[4]) {
    if (dtype == FP_DTYPE_F32) *reinterpret_cast<float4*>(static_cast<float*>(base) + at) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + at) = make_uint2(to_16x2(v[0], v[1], dtype), to_16x2(v[2], v[3], dtype));
}

// ---- activations ----------------------------------------------------------------------------------------------------
// tanh(u) = 1 - 2 / (1 + e^2u), so z/2 (1 + tanh u) = z / (1 + e^-2u): one exponential, and no cancellation where the result is
// small.  e^-2u = inf gives z * 0, the limit.  Exponentials and reciprocals are the approximate ones (2 ulp): results are rounded to
// 16 bits, and the epilogue of a product has some 30 instructions an element before it, not the tensor cores, sets the pace.

constexpr float kSqrt2OverPi2 = 1.5957691216057308f;       // 2 sqrt(2 / pi)
constexpr float kInvSqrt2 = 0.70710678118654752f, kInvSqrt2Pi = 0.39894228040143268f;

__device__ __forceinline__ float inverse(float x) {        // beyond 2^126: 0
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Phi(z), with e = e^(-z^2 / 2) left for the density: Abramowitz and Stegun, formula 7.1.26, erfc(x) = (a1 t + .. + a5 t^5) e^(-x^2)
// with t = 1 / (1 + p x) for x >= 0, off by 1.5e-7 at most; below zero nothing cancels.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
    const float t = inverse(fmaf(0.3275911f * kInvSqrt2, fabsf(z), 1.0f));
    e = __expf(-0.5f * z * z);
    const float tail = 0.5f * e * t * fmaf(fmaf(fmaf(fmaf(1.061405429f, t, -1.453152027f), t, 1.421413741f), t, -0.284496736f), t, 0.254829592f);
    return z > 0.0f ? 1.0f - tail : tail;
}
__device__ __forceinline__ float act_of(float z, int act) {
    switch (act) {
        case FP_ACT_RELU: return z < 0.0f ? 0.0f : z;       // NaN stays
        case FP_ACT_GELU: { float e; return z * normal_cdf(z, e); }
        case FP_ACT_GELU_TANH: return z * inverse(1.0f + __expf(-kSqrt2OverPi2 * (z + 0.044715f * z * z * z)));
        case FP_ACT_SILU: return z * inverse(1.0f + __expf(-z));
        default: return z;
    }
}
__device__ __forceinline__ float act_grad(float z, int act) {
    switch (act) {
        case FP_ACT_RELU: return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
        case FP_ACT_GELU: {
            float e;
            const float p = normal_cdf(z, e);
            return fmaf(z * kInvSqrt2Pi, e, p);
        }
        case FP_ACT_GELU_TANH: {
            // d/dz z s(2u) = s + z s (1 - s) 2u',  2u' = 2 sqrt(2/pi) (1 + 3 0.044715 z^2)
            const float s = inverse(1.0f + __expf(-kSqrt2OverPi2 * (z + 0.044715f * z * z * z)));
            return s + z * s * (1.0f - s) * kSqrt2OverPi2 * (1.0f + fminf(0.134145f * z * z, 1e30f));   // (0 times inf for a finite z)
        }
        case FP_ACT_SILU: {
            const float s = inverse(1.0f + __expf(-z));
            return s * (1.0f + z * (1.0f - s));
        }
        default: return 1.0f;
    }
}
// Rows of values, the choice made once for all of them.
template <int ACT, int U, int C>
__device__ __forceinline__ void act_rows(float (&v)[U][C]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < C; ++i) v[u][i] = act_of(v[u][i], ACT);
}
template <int U, int C>
__device__ __forceinline__ void act_all(float (&v)[U][C], int act) {
    if (act == FP_ACT_RELU) act_rows<FP_ACT_RELU>(v);
    else if (act == FP_ACT_GELU) act_rows<FP_ACT_GELU>(v);
    else if (act == FP_ACT_GELU_TANH) act_rows<FP_ACT_GELU_TANH>(v);
    else if (act == FP_ACT_SILU) act_rows<FP_ACT_SILU>(v);
}
}  // namespace train
}  // namespace fp
