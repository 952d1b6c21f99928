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

// ---- two floats in a register pair ----------------------------------------------------------------------------------

typedef unsigned long long Two;
__device__ __forceinline__ Two two(float lo, float hi) { Two r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ Two twice(float x) { return two(x, x); }
__device__ __forceinline__ void split(Two x, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ Two mul2(Two a, Two b) { Two r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ Two add2(Two a, Two b) { Two r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) { Two r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
// 2^x and 1 / x of both (2 ulp; results below 2^-126 are 0)
__device__ __forceinline__ Two exp2_of2(Two x) {
    float a, b;
    split(x, a, b);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    return two(a, b);
}
__device__ __forceinline__ Two inverse2(Two x) {
    float a, b;
    split(x, a, b);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    return two(a, b);
}

// ---- activations ----------------------------------------------------------------------------------------------------
// Two values at a time, in packed instructions: the epilogue of a product and dz are instruction-bound where the activation takes 40 instructions a
// value (dz of 8192 x 16384 with gelu: 174 us one at a time, 143 two at a time, of which the memory needs 123).
// tanh(u) = 1 - 2 / (1 + e^2u), so z/2 (1 + tanh u) = z / (1 + e^-2u): one exponential, and no cancellation where the result is
// small.  e^-2u = inf gives z * 0, the limit.

constexpr float kLog2E_ = 1.4426950408889634f;
constexpr float kSqrt2OverPi2 = 1.5957691216057308f;       // 2 sqrt(2 / pi)
constexpr float kInvSqrt2 = 0.70710678118654752f, kInvSqrt2Pi = 0.39894228040143268f;

// Phi(z), with e = e^(-z^2 / 2) left for the density: Abramowitz and Stegun, formula 7.1.26, erfc(x) = (a1 t + .. + a5 t^5) e^(-x^2)
// with t = 1 / (1 + p x) for x >= 0, off by 1.5e-7 at most; half of it is the tail of Phi.
__device__ __forceinline__ Two normal_cdf2(Two z, Two& e) {
    float a, b;
    split(z, a, b);
    const Two t = inverse2(fma2(twice(0.3275911f * kInvSqrt2), two(fabsf(a), fabsf(b)), twice(1.0f)));
    e = exp2_of2(mul2(mul2(z, z), twice(-0.5f * kLog2E_)));
    Two q = fma2(twice(0.5f * 1.061405429f), t, twice(0.5f * -1.453152027f));
    q = fma2(q, t, twice(0.5f * 1.421413741f));
    q = fma2(q, t, twice(0.5f * -0.284496736f));
    q = fma2(q, t, twice(0.5f * 0.254829592f));
    float lo, hi;
    split(mul2(mul2(q, t), e), lo, hi);
    return two(a > 0.0f ? 1.0f - lo : lo, b > 0.0f ? 1.0f - hi : hi);
}
// 1 / (1 + e^-2u) of gelu_tanh, and z^2
__device__ __forceinline__ Two tanh_gate2(Two z, Two& zz) {
    zz = mul2(z, z);
    return inverse2(add2(exp2_of2(mul2(mul2(fma2(zz, twice(0.044715f), twice(1.0f)), z), twice(-kSqrt2OverPi2 * kLog2E_))), twice(1.0f)));
}
__device__ __forceinline__ Two gate2(Two z) { return inverse2(add2(exp2_of2(mul2(z, twice(-kLog2E_))), twice(1.0f))); }      // 1 / (1 + e^-z)

template <int ACT>
__device__ __forceinline__ Two act2(Two z) {
    if (ACT == FP_ACT_RELU) {
        float a, b;
        split(z, a, b);
        return two(a < 0.0f ? 0.0f : a, b < 0.0f ? 0.0f : b);       // NaN stays
    }
    Two x;
    if (ACT == FP_ACT_GELU) return mul2(z, normal_cdf2(z, x));
    if (ACT == FP_ACT_GELU_TANH) return mul2(z, tanh_gate2(z, x));
    if (ACT == FP_ACT_SILU) return mul2(z, gate2(z));
    return z;
}
template <int ACT>
__device__ __forceinline__ Two act_grad2(Two z) {
    if (ACT == FP_ACT_RELU) {
        float a, b;
        split(z, a, b);
        return two(a > 0.0f ? 1.0f : (a <= 0.0f ? 0.0f : a), b > 0.0f ? 1.0f : (b <= 0.0f ? 0.0f : b));
    }
    if (ACT == FP_ACT_GELU) {
        Two e;
        const Two p = normal_cdf2(z, e);
        return fma2(mul2(z, twice(kInvSqrt2Pi)), e, p);
    }
    if (ACT == FP_ACT_GELU_TANH) {
        // d/dz z s(2u) = s + z s (1 - s) 2u',  2u' = 2 sqrt(2/pi) (1 + 3 0.044715 z^2)
        Two zz;
        const Two s = tanh_gate2(z, zz);
        float a, b;
        split(mul2(zz, twice(0.134145f)), a, b);
        const Two du = mul2(add2(two(fminf(a, 1e30f), fminf(b, 1e30f)), twice(1.0f)), twice(kSqrt2OverPi2));      // (0 times inf for a finite z)
        return fma2(mul2(mul2(z, s), fma2(s, twice(-1.0f), twice(1.0f))), du, s);
    }
    if (ACT == FP_ACT_SILU) {
        const Two s = gate2(z);
        return mul2(s, fma2(z, fma2(s, twice(-1.0f), twice(1.0f)), twice(1.0f)));
    }
    return twice(1.0f);
}

// Rows of values, the choice made once for all of them.
template <int ACT, int U, int C>
__device__ __forceinline__ void act_rows(float (&v)[U][C]) {
    static_assert(U * C % 2 == 0, "in pairs");
#pragma unroll
    for (int i = 0; i < U * C; i += 2) split(act2<ACT>(two(v[i / C][i % C], v[(i + 1) / C][(i + 1) % C])), v[i / C][i % C], v[(i + 1) / C][(i + 1) % C]);
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
