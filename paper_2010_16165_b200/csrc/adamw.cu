// One AdamW step over many tensors (fp_adamw_step).
//
// Memory bound: every parameter, gradient and state is read and written once, 28 bytes an element in 32 bits, 10 with 16-bit
// parameters and 8-bit states.  The tensors' addresses travel in the launch's parameters (up to kMaxTensors of them), so a
// step over a whole network is one launch with nothing to copy beforehand and nothing to keep; a block finds its tensor
// by bisection over the tensors' first blocks.
#include "train_common.cuh"

#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>

namespace fp {
namespace {

using namespace train;

constexpr int kThreads = 256;
constexpr int kMaxTensors = 360;
constexpr int kUnit32 = 4096, kUnit8 = 4096;             // elements of a block of threads

struct Entry {
    void* p;
    const void* g;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    const uint8_t* mask;
    long long n;
    long long per_row;
    int unit0;                                           // first block of threads
    int aligned;                                         // whether four (32-bit states) or eight (8-bit) neighbours lie aligned everywhere
};
struct Step {
    float decay, b1, ob1, b2, ob2, inv_sqrt_c2, eps, rate, grad_scale;
    double lr, beta1, beta2, weight_decay;
    const float* d_lr;
    const float* d_grad_scale;
    const int64_t* d_step;
    long long step;
};
struct Table {
    Step s;
    int count;
    Entry e[kMaxTensors];
};
static_assert(sizeof(Table) <= 32764, "the launch's parameters");

// The step's scalars, from 64-bit arithmetic as the host does it.
__host__ __device__ inline void scalars(Step& s, double lr, long long t) {
    const double c1 = 1.0 - pow(s.beta1, (double)t), c2 = 1.0 - pow(s.beta2, (double)t);
    s.decay = (float)(1.0 - lr * s.weight_decay);
    s.inv_sqrt_c2 = (float)(1.0 / sqrt(c2));
    s.rate = (float)(lr / c1);
}

// Every operation rounded by itself, in this order, so that a state in 8 bits, whose rounding turns the last bit of a sum
// into a step of 1/16, does not depend on what the compiler contracts.
__device__ __forceinline__ void moments(const Step& s, float g, float& m, float& v, float& r) {
    g = __fmul_rn(g, s.grad_scale);
    m = __fadd_rn(__fmul_rn(m, s.b1), __fmul_rn(g, s.ob1));
    v = __fadd_rn(__fmul_rn(v, s.b2), __fmul_rn(__fmul_rn(g, s.ob2), g));
    r = __fsqrt_rn(v);
}
__device__ __forceinline__ float updated(const Step& s, float p, float m, float r) {
    return __fmaf_rn(-s.rate, __fdividef(m, __fmaf_rn(r, s.inv_sqrt_c2, s.eps)), p * s.decay);
}

__device__ __forceinline__ const Entry& find(const Table& t, int unit) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.e[mid].unit0 <= unit) lo = mid; else hi = mid - 1;
    }
    return t.e[lo];
}

__device__ __forceinline__ Step step_of(const Table& t) {
    Step s = t.s;
    if (t.s.d_lr || t.s.d_step || t.s.d_grad_scale) {
        __shared__ float got[4];
        if (threadIdx.x == 0) {
            if (s.d_lr || s.d_step) scalars(s, s.d_lr ? (double)*s.d_lr : s.lr, s.d_step ? (long long)*s.d_step : s.step);
            got[0] = s.decay; got[1] = s.inv_sqrt_c2; got[2] = s.rate; got[3] = s.d_grad_scale ? *s.d_grad_scale : s.grad_scale;
        }
        __syncthreads();
        s.decay = got[0]; s.inv_sqrt_c2 = got[1]; s.rate = got[2]; s.grad_scale = got[3];
    }
    return s;
}

template <int PT, int GT>
__global__ void __launch_bounds__(kThreads) adamw32_kernel(const __grid_constant__ Table t) {
    const Entry& e = find(t, (int)blockIdx.x);
    const Step s = step_of(t);
    const long long at0 = (long long)((int)blockIdx.x - e.unit0) * kUnit32;
    float* m_ = static_cast<float*>(e.m);
    float* v_ = static_cast<float*>(e.v);
#pragma unroll
    for (int u = 0; u < kUnit32 / (4 * kThreads); ++u) {
        const long long at = at0 + (u * kThreads + (int)threadIdx.x) * 4;
        const int count = (int)min(4ll, e.n - at);
        if (count <= 0) break;
        const bool whole = e.aligned && count == 4;
        uint32_t keep = 15;
        if (e.mask)
            for (int i = 0; i < count; ++i)
                if (!e.mask[(at + i) / e.per_row]) keep &= ~(1u << i);
        float p[4] = {0, 0, 0, 0}, g[4] = {0, 0, 0, 0}, m[4] = {0, 0, 0, 0}, v[4] = {0, 0, 0, 0};
        if (whole) {
            load4(e.p, at, PT, p); load4(e.g, at, GT, g); load4(m_, at, FP_DTYPE_F32, m); load4(v_, at, FP_DTYPE_F32, v);
        } else {
            for (int i = 0; i < count; ++i) { p[i] = load1(e.p, at + i, PT); g[i] = load1(e.g, at + i, GT); m[i] = m_[at + i]; v[i] = v_[at + i]; }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float r;
            moments(s, g[i], m[i], v[i], r);
            p[i] = updated(s, p[i], m[i], r);
            if (!(keep >> i & 1)) p[i] = m[i] = v[i] = 0.0f;
        }
        if (whole) {
            store4(e.p, at, PT, p); store4(m_, at, FP_DTYPE_F32, m); store4(v_, at, FP_DTYPE_F32, v);
        } else {
            for (int i = 0; i < count; ++i) { store1(e.p, at + i, PT, p[i]); m_[at + i] = m[i]; v_[at + i] = v[i]; }
        }
    }
}

// ---- 8-bit states ---------------------------------------------------------------------------------------------------
// A warp has a block of 256 elements, eight a lane; the block's largest values come from shuffles.

__device__ __forceinline__ float e4m3_value(uint32_t code) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)code));
    return __half2float(__ushort_as_half((uint16_t)h));
}
__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int PT, int GT>
__global__ void __launch_bounds__(kThreads) adamw8_kernel(const __grid_constant__ Table t) {
    const Entry& e = find(t, (int)blockIdx.x);
    const Step s = step_of(t);
    const int lane = threadIdx.x & 31;
    uint8_t* m_ = static_cast<uint8_t*>(e.m);
    uint8_t* v_ = static_cast<uint8_t*>(e.v);
    for (int u = threadIdx.x >> 5; u < kUnit8 / FP_ADAMW_BLOCK; u += kThreads / 32) {
        const long long block = (long long)((int)blockIdx.x - e.unit0) * (kUnit8 / FP_ADAMW_BLOCK) + u;
        if (block * FP_ADAMW_BLOCK >= e.n) break;
        const long long at = block * FP_ADAMW_BLOCK + lane * 8;
        const int count = (int)max(0ll, min(8ll, e.n - at));
        const bool whole = e.aligned && count == 8;
        uint32_t keep = 255;
        if (e.mask)
            for (int i = 0; i < count; ++i)
                if (!e.mask[(at + i) / e.per_row]) keep &= ~(1u << i);
        float p[8], g[8];
        uint32_t mc[8], vc[8];
        if (whole) {
            float a[4], b[4];
            load4(e.p, at, PT, a); load4(e.p, at + 4, PT, b);
            for (int i = 0; i < 4; ++i) { p[i] = a[i]; p[4 + i] = b[i]; }
            load4(e.g, at, GT, a); load4(e.g, at + 4, GT, b);
            for (int i = 0; i < 4; ++i) { g[i] = a[i]; g[4 + i] = b[i]; }
            const uint2 cm = *reinterpret_cast<const uint2*>(m_ + at), cv = *reinterpret_cast<const uint2*>(v_ + at);
            for (int i = 0; i < 4; ++i) {
                mc[i] = cm.x >> (8 * i) & 255; mc[4 + i] = cm.y >> (8 * i) & 255;
                vc[i] = cv.x >> (8 * i) & 255; vc[4 + i] = cv.y >> (8 * i) & 255;
            }
        } else {
            for (int i = 0; i < 8; ++i) {
                const bool in = i < count;
                p[i] = in ? load1(e.p, at + i, PT) : 0.0f; g[i] = in ? load1(e.g, at + i, GT) : 0.0f;
                mc[i] = in ? m_[at + i] : 0; vc[i] = in ? v_[at + i] : 0;
            }
        }
        const float ms = e.m_scale[block], vs = e.v_scale[block];
        float m[8], r[8], m_top = 0.0f, r_top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] = __fmul_rn(e4m3_value(mc[i]), ms);
            r[i] = __fmul_rn(e4m3_value(vc[i]), vs);
            float v = __fmul_rn(r[i], r[i]);
            moments(s, g[i], m[i], v, r[i]);
            p[i] = updated(s, p[i], m[i], r[i]);
            if (!(keep >> i & 1) || i >= count) p[i] = m[i] = r[i] = 0.0f;
            m_top = fmaxf(m_top, fabsf(m[i])); r_top = fmaxf(r_top, r[i]);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) { m_top = fmaxf(m_top, __shfl_xor_sync(~0u, m_top, d)); r_top = fmaxf(r_top, __shfl_xor_sync(~0u, r_top, d)); }
        float ms1 = __fmul_rn(m_top, 1.0f / 448.0f), vs1 = __fmul_rn(r_top, 1.0f / 448.0f);
        if (ms1 < 1.17549435e-38f) ms1 = 0.0f;
        if (vs1 < 1.17549435e-38f) vs1 = 0.0f;
        const float mi = ms1 > 0.0f ? __frcp_rn(ms1) : 0.0f, vi = vs1 > 0.0f ? __frcp_rn(vs1) : 0.0f;
        float q[8];
        uint2 cm, cv;
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = __fmul_rn(m[i], mi);
        cm.x = e4m3_pair(q[0], q[1]) | e4m3_pair(q[2], q[3]) << 16; cm.y = e4m3_pair(q[4], q[5]) | e4m3_pair(q[6], q[7]) << 16;
#pragma unroll
        for (int i = 0; i < 8; ++i) { q[i] = __fmul_rn(r[i], vi); if (r[i] > 0.0f) q[i] = fmaxf(q[i], 0.001953125f); }
        cv.x = e4m3_pair(q[0], q[1]) | e4m3_pair(q[2], q[3]) << 16; cv.y = e4m3_pair(q[4], q[5]) | e4m3_pair(q[6], q[7]) << 16;
        if (whole) {
            const float a[4] = {p[0], p[1], p[2], p[3]}, b[4] = {p[4], p[5], p[6], p[7]};
            store4(e.p, at, PT, a); store4(e.p, at + 4, PT, b);
            *reinterpret_cast<uint2*>(m_ + at) = cm;
            *reinterpret_cast<uint2*>(v_ + at) = cv;
        } else {
            for (int i = 0; i < count; ++i) {
                store1(e.p, at + i, PT, p[i]);
                m_[at + i] = (uint8_t)((i < 4 ? cm.x : cm.y) >> (8 * (i & 3)));
                v_[at + i] = (uint8_t)((i < 4 ? cv.x : cv.y) >> (8 * (i & 3)));
            }
        }
        if (lane == 0) { e.m_scale[block] = ms1; e.v_scale[block] = vs1; }
    }
}

typedef void (*Kernel)(const Table);
template <int PT>
Kernel kernel_for(int gt, int bits) {
    if (gt == FP_DTYPE_F32) return bits == 8 ? adamw8_kernel<PT, FP_DTYPE_F32> : adamw32_kernel<PT, FP_DTYPE_F32>;
    if (gt == FP_DTYPE_BF16) return bits == 8 ? adamw8_kernel<PT, FP_DTYPE_BF16> : adamw32_kernel<PT, FP_DTYPE_BF16>;
    return bits == 8 ? adamw8_kernel<PT, FP_DTYPE_F16> : adamw32_kernel<PT, FP_DTYPE_F16>;
}
Kernel kernel_of(int pt, int gt, int bits) {
    return pt == FP_DTYPE_F32 ? kernel_for<FP_DTYPE_F32>(gt, bits) : pt == FP_DTYPE_BF16 ? kernel_for<FP_DTYPE_BF16>(gt, bits)
                                                                                        : kernel_for<FP_DTYPE_F16>(gt, bits);
}
bool dtype_ok(int d) { return d == FP_DTYPE_F32 || is_half(d); }
bool multiple(const void* p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

cudaError_t flush(Table& t, unsigned units, Kernel k, cudaStream_t st) {
    if (!t.count) return cudaSuccess;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3(units);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    void* args[1] = {&t};
    const cudaError_t e = cudaLaunchKernelExC(&cfg, (const void*)k, args);
    t.count = 0;
    return e;
}

}  // namespace
}  // namespace fp

using namespace fp;
using namespace fp::train;

extern "C" fp_status fp_adamw_step(const fp_adamw_tensor* ts, int32_t count, const fp_adamw_hyper* h, void* stream) {
    if (count < 0 || (count > 0 && !ts) || !h) return err(FP_ERR_ARG, "fp_adamw_step: NULL argument or a negative count");
    if (!(h->beta1 >= 0.0 && h->beta1 < 1.0 && h->beta2 >= 0.0 && h->beta2 < 1.0 && h->eps >= 0.0) || !isfinite(h->eps) || !isfinite(h->lr) ||
        !isfinite(h->weight_decay) || (!h->d_step && h->step < 1) || isnan(h->grad_scale))
        return err(FP_ERR_ARG, "fp_adamw_step: bad hyper-parameters (0 <= beta < 1, eps >= 0, step >= 1)");
    if (((uintptr_t)h->d_lr & 3) || ((uintptr_t)h->d_grad_scale & 3) || ((uintptr_t)h->d_step & 7))
        return err(FP_ERR_ARG, "fp_adamw_step: a device scalar is not aligned to its type");
    for (int i = 0; i < count; ++i) {
        const fp_adamw_tensor& t = ts[i];
        if (t.n < 0 || t.reserved) return err(FP_ERR_ARG, "fp_adamw_step: a tensor with a negative size, or reserved set");
        if (t.n > (1ll << 40)) return err(FP_ERR_BOUNDS, "fp_adamw_step: a tensor beyond 2^40 elements");
        if (!dtype_ok(t.p_dtype) || !dtype_ok(t.g_dtype)) return err(FP_ERR_UNSUPPORTED, "fp_adamw_step: dtypes are FP_DTYPE_F32, _BF16 or _F16");
        if (t.state_bits != 32 && t.state_bits != 8) return err(FP_ERR_UNSUPPORTED, "fp_adamw_step: state_bits must be 32 or 8");
        if (t.n == 0) continue;
        if (!t.d_p || !t.d_g || !t.d_m || !t.d_v || (t.state_bits == 8 && (!t.d_m_scale || !t.d_v_scale)))
            return err(FP_ERR_ARG, "fp_adamw_step: NULL parameter, gradient, state or scale");
        if (t.d_mask && t.per_row < 1) return err(FP_ERR_ARG, "fp_adamw_step: per_row must be positive where there is a mask");
        if (!multiple(t.d_p, elem_bytes(t.p_dtype)) || !multiple(t.d_g, elem_bytes(t.g_dtype)) ||
            (t.state_bits == 32 && (!multiple(t.d_m, 4) || !multiple(t.d_v, 4))) ||
            (t.state_bits == 8 && (!multiple(t.d_m_scale, 4) || !multiple(t.d_v_scale, 4))))
            return err(FP_ERR_ARG, "fp_adamw_step: a buffer is not aligned to its elements");
    }
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return err(FP_ERR_CUDA, "fp_adamw_step: no current device"); }
    Buffers buf(dev);
    bool there = buf.here_or_null(h->d_lr) && buf.here_or_null(h->d_grad_scale) && buf.here_or_null(h->d_step);
    for (int i = 0; i < count && there; ++i) {
        const fp_adamw_tensor& t = ts[i];
        if (t.n == 0) continue;
        there = buf.here(t.d_p) && buf.here(t.d_g) && buf.here(t.d_m) && buf.here(t.d_v) && buf.here_or_null(t.d_mask) &&
                (t.state_bits == 32 || (buf.here(t.d_m_scale) && buf.here(t.d_v_scale)));
    }
    if (!there) return err(FP_ERR_ARG, "fp_adamw_step: a buffer is not memory of the current device");

    Table t;                                             // 32 KB of stack
    Step& s = t.s;
    memset(&s, 0, sizeof(s));
    s.lr = h->lr; s.beta1 = h->beta1; s.beta2 = h->beta2; s.weight_decay = h->weight_decay; s.step = h->step;
    s.d_lr = h->d_lr; s.d_grad_scale = h->d_grad_scale; s.d_step = reinterpret_cast<const int64_t*>(h->d_step);
    s.b1 = (float)h->beta1; s.ob1 = (float)(1.0 - h->beta1); s.b2 = (float)h->beta2; s.ob2 = (float)(1.0 - h->beta2);
    s.eps = (float)h->eps; s.grad_scale = (float)h->grad_scale;
    scalars(s, h->lr, h->d_step ? 1 : h->step);
    t.count = 0;
    static const int kinds[3] = {FP_DTYPE_F32, FP_DTYPE_BF16, FP_DTYPE_F16};
    cudaError_t e = cudaSuccess;
    for (int pt : kinds)                                 // a launch has one type of each
        for (int gt : kinds)
            for (int bits = 8; bits <= 32; bits += 24) {
                const Kernel k = kernel_of(pt, gt, bits);
                const long long unit = bits == 32 ? kUnit32 : kUnit8;
                long long units = 0;
                for (int i = 0; i < count; ++i) {
                    const fp_adamw_tensor& x = ts[i];
                    if (x.n == 0 || x.p_dtype != pt || x.g_dtype != gt || x.state_bits != bits) continue;
                    const long long mine = (x.n + unit - 1) / unit;
                    if (t.count == kMaxTensors || units + mine > 0x7fffffffll) {
                        if ((e = flush(t, (unsigned)units, k, (cudaStream_t)stream)) != cudaSuccess) goto done;
                        units = 0;
                    }
                    Entry& r = t.e[t.count++];
                    r.p = x.d_p; r.g = x.d_g; r.m = x.d_m; r.v = x.d_v; r.m_scale = x.d_m_scale; r.v_scale = x.d_v_scale;
                    r.mask = x.d_mask; r.n = x.n; r.per_row = x.per_row; r.unit0 = (int)units;
                    const int vec = bits == 32 ? 4 : 8;
                    r.aligned = multiple(x.d_p, std::min(16, vec * elem_bytes(pt))) && multiple(x.d_g, std::min(16, vec * elem_bytes(gt))) &&
                                multiple(x.d_m, bits == 32 ? 16 : 8) && multiple(x.d_v, bits == 32 ? 16 : 8);
                    units += mine;
                }
                if ((e = flush(t, (unsigned)units, k, (cudaStream_t)stream)) != cudaSuccess) goto done;
            }
done:
    if (e != cudaSuccess) { cudaGetLastError(); return err(FP_ERR_CUDA, cudaGetErrorString(e)); }
    return FP_OK;
}
