// One AdamW step over many tensors (fp_adamw_step).
//
// Memory bound: every parameter, gradient and state is read and written once, 28 bytes an element in 32 bits, 10 with 16-bit
// parameters and 8-bit states.  The tensors' addresses travel in the launch's parameters (up to kMaxTensors of them), so a
// step over a whole network is one launch with nothing to copy beforehand and nothing to keep; a block finds its tensor
// by bisection over the tensors' first blocks.
#include "train_common.cuh"
#include "tc_common.cuh"

#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>

namespace fp {
namespace {

using namespace train;

constexpr int kThreads = 256;
constexpr int kFewTensors = 64, kMaxTensors = 320;     // of a launch: its parameters are 6 or 31 KB, copied at every call (4 us for the larger)
constexpr int kUnit32 = 2048, kUnit8 = 4096;             // elements of a block of threads

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
    tc::FastDiv rows;                                    // division by per_row; rows.d 0: beyond 31 bits
    int aligned;                                         // whether four (32-bit states) or sixteen (8-bit) neighbours lie in aligned vectors everywhere
};
struct Step {
    float decay, b1, ob1, b2, ob2, inv_sqrt_c2, eps, rate, grad_scale, one;
    double lr, beta1, beta2, weight_decay;
    const float* d_lr;
    const float* d_grad_scale;
    const int64_t* d_step;
    long long step;
};
template <int N> struct Table {
    Step s;
    int count;
    Entry e[N];
};
static_assert(sizeof(Table<kMaxTensors>) <= 32764, "the launch's parameters");

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
// The quotient is approximate, off by 2^-22 of itself: less than p's own rounding in 32 bits wherever the step is below a fourth of p, and of
// the step's size otherwise; nothing of it goes into a state.
__device__ __forceinline__ float updated(const Step& s, float p, float m, float r) {
    return __fmaf_rn(-s.rate, __fdividef(m, __fmaf_rn(r, s.inv_sqrt_c2, s.eps)), p * s.decay);
}

// Which of the elements at .. at + count - 1 (count <= 16) a mask keeps.
__device__ __forceinline__ uint32_t kept(const Entry& e, long long at, int count) {
    if (!e.mask) return 0xffffu;
    long long row = e.rows.d ? (long long)tc::fdiv((uint32_t)at, e.rows) : at / e.per_row;
    const long long left = (row + 1) * e.per_row - at;   // elements of this row from here on
    uint32_t keep = e.mask[row] ? 0xffffu : 0u;
    if (left >= count) return keep;
    int from = (int)left;                                // where the next row begins
    keep &= (1u << from) - 1u;
#pragma unroll 1
    do {
        const uint32_t rest = 0xffffu << from;
        from += (int)min(16ll, e.per_row);
        keep = (keep & ~rest) | (e.mask[++row] ? rest & 0xffffu : 0u);
    } while (from < count);
    return keep;
}

template <int N>
__device__ __forceinline__ const Entry& find(const Table<N>& t, int unit) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.e[mid].unit0 <= unit) lo = mid; else hi = mid - 1;
    }
    return t.e[lo];
}

__device__ __forceinline__ Step step_of(const Step& from) {
    Step s = from;
    if (s.d_lr || s.d_step || s.d_grad_scale) {
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

// 28 bytes an element with 32-bit parameters: 128 bytes a thread are asked for before the first is used.
template <int PT, int GT, int N>
__global__ void __launch_bounds__(kThreads) adamw32_kernel(const __grid_constant__ Table<N> t) {
    const Entry& e = find(t, (int)blockIdx.x);
    const Step s = step_of(t.s);
    const long long at0 = (long long)((int)blockIdx.x - e.unit0) * kUnit32 + (int)threadIdx.x * 4;
    float* m_ = static_cast<float*>(e.m);
    float* v_ = static_cast<float*>(e.v);
    constexpr int U = kUnit32 / (4 * kThreads);
    if (e.aligned && at0 + (U - 1) * 4 * kThreads + 4 <= e.n) {
        float p[U][4], g[U][4], m[U][4], v[U][4];
        uint32_t keep[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long at = at0 + u * 4 * kThreads;
            keep[u] = kept(e, at, 4);
            if (keep[u] & 15u) {                         // (what is pruned need not be read)
                load4(e.p, at, PT, p[u]); load4(e.g, at, GT, g[u]); load4(m_, at, FP_DTYPE_F32, m[u]); load4(v_, at, FP_DTYPE_F32, v[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long at = at0 + u * 4 * kThreads;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float r;
                moments(s, g[u][i], m[u][i], v[u][i], r);
                p[u][i] = updated(s, p[u][i], m[u][i], r);
                if (!(keep[u] >> i & 1)) p[u][i] = m[u][i] = v[u][i] = 0.0f;
            }
            store4(e.p, at, PT, p[u]); store4(m_, at, FP_DTYPE_F32, m[u]); store4(v_, at, FP_DTYPE_F32, v[u]);
        }
        return;
    }
#pragma unroll 1
    for (int u = 0; u < U; ++u) {                        // a tensor's end, or one that is not aligned
        const long long at = at0 + u * 4 * kThreads;
        const int count = (int)max(0ll, min(4ll, e.n - at));
        if (count == 0) break;
        const uint32_t keep = kept(e, at, count);
#pragma unroll 1
        for (int i = 0; i < count; ++i) {
            float p = load1(e.p, at + i, PT), m = m_[at + i], v = v_[at + i], r;
            moments(s, load1(e.g, at + i, GT), m, v, r);
            p = updated(s, p, m, r);
            if (!(keep >> i & 1)) p = m = v = 0.0f;
            store1(e.p, at + i, PT, p); m_[at + i] = m; v_[at + i] = v;
        }
    }
}

// ---- 8-bit states ---------------------------------------------------------------------------------------------------
// Half a warp has a block of 256 elements, sixteen a lane; the block's largest values come from shuffles.  With 16-bit parameters an
// element is 10 bytes, for which the memory leaves 27 instructions, hence: two elements go through one packed instruction where there
// is one (each half rounded as by itself), what a block needs once is paid for by sixteen elements, and the root is the approximate
// one, off by 2^-22 of itself at most: with the exact one 157 M elements took 368 us instead of 318.

// (A packed product and sum were contracted in spite of their .rn; as a 1 + b with a 1 that comes from the host they are not.)
__device__ __forceinline__ Two e4m3_values(uint32_t codes) {       // of the two low bytes
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes));
    return two(__half2float(__ushort_as_half((uint16_t)h)), __half2float(__ushort_as_half((uint16_t)(h >> 16))));
}
__device__ __forceinline__ uint32_t e4m3_codes(Two x) {
    float lo, hi;
    split(x, lo, hi);
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float quotient(float a, float b) {      // off by 2 ulp; b >= 0, and not so large that 1 / b is subnormal where a / b matters
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(b));
    return a * r;
}

__device__ __forceinline__ float root(float x) {                    // below 2^-126: 0
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Sixteen elements of a type as they are in memory.
template <int DT> struct Sixteen {
    uint32_t w[DT == FP_DTYPE_F32 ? 16 : 8];
    __device__ __forceinline__ Two pair(int i) const {             // elements 2 i, 2 i + 1
        if (DT == FP_DTYPE_F32) return two(__uint_as_float(w[(2 * i) % (DT == FP_DTYPE_F32 ? 16 : 8)]), __uint_as_float(w[(2 * i + 1) % (DT == FP_DTYPE_F32 ? 16 : 8)]));
        if (DT == FP_DTYPE_BF16) return two(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
        return two(to_f32((uint16_t)w[i], DT), to_f32((uint16_t)(w[i] >> 16), DT));
    }
    __device__ __forceinline__ void put(int i, float lo, float hi) {
        if (DT == FP_DTYPE_F32) { w[(2 * i) % (DT == FP_DTYPE_F32 ? 16 : 8)] = __float_as_uint(lo); w[(2 * i + 1) % (DT == FP_DTYPE_F32 ? 16 : 8)] = __float_as_uint(hi); }
        else w[i] = to_16x2(lo, hi, DT);
    }
    static constexpr int kBytes = DT == FP_DTYPE_F32 ? 4 : 2;      // of an element, and so vectors of sixteen elements
    __device__ __forceinline__ void read(const void* x, long long at) {
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const char*>(x) + at * kBytes);
#pragma unroll
        for (int k = 0; k < kBytes; ++k) { const uint4 u = src[k]; w[4 * k] = u.x; w[4 * k + 1] = u.y; w[4 * k + 2] = u.z; w[4 * k + 3] = u.w; }
    }
    __device__ __forceinline__ void write(void* x, long long at) const {
        uint4* dst = reinterpret_cast<uint4*>(static_cast<char*>(x) + at * kBytes);
#pragma unroll
        for (int k = 0; k < kBytes; ++k) dst[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
    }
    __device__ __forceinline__ void read(const void* x, long long at, int count) {
#pragma unroll
        for (int i = 0; i < 8; ++i) put(i, 2 * i < count ? load1(x, at + 2 * i, DT) : 0.0f, 2 * i + 1 < count ? load1(x, at + 2 * i + 1, DT) : 0.0f);
    }
    __device__ __forceinline__ void write(void* x, long long at, int count) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float lo, hi;
            split(pair(i), lo, hi);
            if (2 * i < count) store1(x, at + 2 * i, DT, lo);
            if (2 * i + 1 < count) store1(x, at + 2 * i + 1, DT, hi);
        }
    }
};

__device__ __forceinline__ uint4 read_codes(const uint8_t* x, long long at, int count) {
    uint32_t w[4] = {};
#pragma unroll
    for (int i = 0; i < 16; ++i) if (i < count) w[i >> 2] |= (uint32_t)x[at + i] << (8 * (i & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void write_codes(uint8_t* x, long long at, int count, const uint32_t (&w)[4]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) if (i < count) x[at + i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
}

// The largest of the values of half a warp, none of them negative (so they compare as their bits do).
__device__ __forceinline__ float largest_of_half(float x) {
#pragma unroll
    for (int d = 8; d; d >>= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, d));
    return x;
}

template <int PT, int GT, int N>
__global__ void __launch_bounds__(kThreads, 4) adamw8_kernel(const __grid_constant__ Table<N> t) {
    const Entry& e = find(t, (int)blockIdx.x);
    const Step s = step_of(t.s);
    const int lane16 = threadIdx.x & 15;
    uint8_t* m_ = static_cast<uint8_t*>(e.m);
    uint8_t* v_ = static_cast<uint8_t*>(e.v);
    static_assert(kUnit8 == 16 * kThreads && FP_ADAMW_BLOCK == 256, "half a warp a block");
    const long long block = (long long)((int)blockIdx.x - e.unit0) * (kUnit8 / FP_ADAMW_BLOCK) + (threadIdx.x >> 4), at = block * FP_ADAMW_BLOCK + lane16 * 16;
    const int count = (int)max(0ll, min(16ll, e.n - at));
    const bool whole = e.aligned && count == 16;
    Sixteen<PT> p;
    Sixteen<GT> g;
    uint4 mc, vc;
    if (whole) {
        p.read(e.p, at); g.read(e.g, at);
        mc = *reinterpret_cast<const uint4*>(m_ + at); vc = *reinterpret_cast<const uint4*>(v_ + at);
    } else {
        p.read(e.p, at, count); g.read(e.g, at, count);
        mc = read_codes(m_, at, count); vc = read_codes(v_, at, count);
    }
    const bool there = block * FP_ADAMW_BLOCK < e.n;
    const float ms0 = there ? e.m_scale[block] : 0.0f, vs0 = there ? e.v_scale[block] : 0.0f;
    const uint32_t keep = count ? kept(e, at, count) & ((1u << count) - 1u) : 0u;
    const Two gs = twice(s.grad_scale), b1 = twice(s.b1), ob1 = twice(s.ob1), b2 = twice(s.b2), ob2 = twice(s.ob2), c2 = twice(s.inv_sqrt_c2),
              eps = twice(s.eps), decay = twice(s.decay), rate = twice(-s.rate), one = twice(s.one), ms = twice(ms0), vs = twice(vs0);
    const uint32_t mw[4] = {mc.x, mc.y, mc.z, mc.w}, vw[4] = {vc.x, vc.y, vc.z, vc.w};
    Two m[8], r[8];
    float m_top = 0.0f, r_top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // as moments() and updated(), two at a time
        const Two d = mul2(g.pair(i), gs);
        m[i] = mul2(e4m3_values(mw[i >> 1] >> (16 * (i & 1))), ms);
        r[i] = mul2(e4m3_values(vw[i >> 1] >> (16 * (i & 1))), vs);
        m[i] = fma2(mul2(m[i], b1), one, mul2(d, ob1));
        const Two v = fma2(mul2(mul2(r[i], r[i]), b2), one, mul2(mul2(d, ob2), d));
        float lo, hi, a, b, x, y, q0, q1;
        split(v, lo, hi);
        lo = root(lo); hi = root(hi);
        r[i] = two(lo, hi);
        split(fma2(r[i], c2, eps), a, b);
        split(m[i], x, y);
        split(fma2(rate, two(quotient(x, a), quotient(y, b)), mul2(p.pair(i), decay)), q0, q1);
        if (keep != 0xffffu) {                           // pruned, or behind the tensor's end
            const bool k0 = keep >> (2 * i) & 1u, k1 = keep >> (2 * i + 1) & 1u;
            q0 = k0 ? q0 : 0.0f; q1 = k1 ? q1 : 0.0f; x = k0 ? x : 0.0f; y = k1 ? y : 0.0f; lo = k0 ? lo : 0.0f; hi = k1 ? hi : 0.0f;
            m[i] = two(x, y); r[i] = two(lo, hi);
        }
        p.put(i, q0, q1);
        m_top = fmaxf(m_top, fmaxf(fabsf(x), fabsf(y)));
        r_top = fmaxf(r_top, fmaxf(lo, hi));
    }
    m_top = largest_of_half(m_top);
    r_top = largest_of_half(r_top);
    float ms1 = __fmul_rn(m_top, 1.0f / 448.0f), vs1 = __fmul_rn(r_top, 1.0f / 448.0f);
    if (ms1 < 1.17549435e-38f) ms1 = 0.0f;
    if (vs1 < 1.17549435e-38f) vs1 = 0.0f;
    const Two mi = twice(ms1 > 0.0f ? __frcp_rn(ms1) : 0.0f), vi = twice(vs1 > 0.0f ? __frcp_rn(vs1) : 0.0f);
    uint32_t cm[4], cv[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = e4m3_codes(mul2(m[i], mi));
        float lo, hi, x, y;
        split(r[i], lo, hi);
        split(mul2(r[i], vi), x, y);
        if (lo > 0.0f) x = fmaxf(x, 0.001953125f);       // 2^-9, the smallest positive code
        if (hi > 0.0f) y = fmaxf(y, 0.001953125f);
        const uint32_t b = e4m3_codes(two(x, y));
        cm[i >> 1] = i & 1 ? cm[i >> 1] | a << 16 : a;
        cv[i >> 1] = i & 1 ? cv[i >> 1] | b << 16 : b;
    }
    if (whole) {
        p.write(e.p, at);
        *reinterpret_cast<uint4*>(m_ + at) = make_uint4(cm[0], cm[1], cm[2], cm[3]);
        *reinterpret_cast<uint4*>(v_ + at) = make_uint4(cv[0], cv[1], cv[2], cv[3]);
    } else {
        p.write(e.p, at, count);
        write_codes(m_, at, count, cm);
        write_codes(v_, at, count, cv);
    }
    if (lane16 == 0 && there) { e.m_scale[block] = ms1; e.v_scale[block] = vs1; }
}

template <int PT, int GT, int N>
const void* kernel_for(int bits) { return bits == 8 ? (const void*)adamw8_kernel<PT, GT, N> : (const void*)adamw32_kernel<PT, GT, N>; }
template <int PT, int N>
const void* kernel_for(int gt, int bits) {
    return gt == FP_DTYPE_F32 ? kernel_for<PT, FP_DTYPE_F32, N>(bits) : gt == FP_DTYPE_BF16 ? kernel_for<PT, FP_DTYPE_BF16, N>(bits)
                                                                                        : kernel_for<PT, FP_DTYPE_F16, N>(bits);
}
template <int N>
const void* kernel_of(int pt, int gt, int bits) {
    return pt == FP_DTYPE_F32 ? kernel_for<FP_DTYPE_F32, N>(gt, bits) : pt == FP_DTYPE_BF16 ? kernel_for<FP_DTYPE_BF16, N>(gt, bits)
                                                                                        : kernel_for<FP_DTYPE_F16, N>(gt, bits);
}
bool dtype_ok(int d) { return d == FP_DTYPE_F32 || is_half(d); }
bool multiple(const void* p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// Whether something that a tensor's step writes is also something else of that tensor, or one of the step's device scalars.
inline bool written_twice(const fp_adamw_tensor& t, const fp_adamw_hyper& h, bool device_scalars) {
    const void *p = t.d_p, *m = t.d_m, *v = t.d_v, *g = t.d_g, *k = t.d_mask;        // (none of the first three is NULL)
    if (p == m || p == v || p == g || p == k || m == v || m == g || m == k || v == g || v == k) return true;
    if (t.state_bits == 32 && !device_scalars) return false;
    auto in = [&](const void* s) { return s == p || s == m || s == v; };
    const void *a = t.d_m_scale, *b = t.d_v_scale;
    const bool scales = t.state_bits == 8;
    if (scales && (in(a) || in(b) || a == b || a == g || a == k || b == g || b == k)) return true;
    for (const void* s : {(const void*)h.d_lr, (const void*)h.d_grad_scale, (const void*)h.d_step})
        if (s && (in(s) || (scales && (s == a || s == b)))) return true;
    return false;
}

struct Kind { int p, g, bits; };
inline bool is_of(const fp_adamw_tensor& x, const Kind& k) { return x.n > 0 && x.p_dtype == k.p && x.g_dtype == k.g && x.state_bits == k.bits; }

// The tensors of one kind among ts[0 .. count), in launches of up to N.
template <int N>
cudaError_t run_kind(const Step& s, const fp_adamw_tensor* ts, int count, const Kind& k, cudaStream_t st) {
    Table<N> t;                                          // at most 31 KB of stack
    t.s = s;
    t.count = 0;
    const long long unit = k.bits == 32 ? kUnit32 : kUnit8;
    long long units = 0;
    for (int i = 0; i <= count; ++i) {
        if (i < count && !is_of(ts[i], k)) continue;
        const long long mine = i < count ? (ts[i].n + unit - 1) / unit : 0;
        if (t.count && (i == count || t.count == N || units + mine > 0x7fffffffll)) {
            cudaLaunchConfig_t cfg;
            memset(&cfg, 0, sizeof(cfg));
            cfg.gridDim = dim3((unsigned)units);
            cfg.blockDim = dim3(kThreads);
            cfg.stream = st;
            void* args[1] = {&t};
            const cudaError_t e = cudaLaunchKernelExC(&cfg, kernel_of<N>(k.p, k.g, k.bits), args);
            if (e != cudaSuccess) return e;
            t.count = 0;
            units = 0;
        }
        if (i == count) break;
        const fp_adamw_tensor& x = ts[i];
        Entry& r = t.e[t.count++];
        r.p = x.d_p; r.g = x.d_g; r.m = x.d_m; r.v = x.d_v; r.m_scale = x.d_m_scale; r.v_scale = x.d_v_scale;
        r.mask = x.d_mask; r.n = x.n; r.per_row = x.per_row; r.unit0 = (int)units;
        memset(&r.rows, 0, sizeof(r.rows));
        if (x.d_mask && x.n < (1ll << 31) && x.per_row < (1ll << 31)) r.rows = tc::make_fastdiv((uint32_t)x.per_row);
        const int vec = k.bits == 32 ? 4 : 16;
        r.aligned = multiple(x.d_p, std::min(16, vec * elem_bytes(k.p))) && multiple(x.d_g, std::min(16, vec * elem_bytes(k.g))) &&
                    multiple(x.d_m, 16) && multiple(x.d_v, 16);
        units += mine;
    }
    return cudaSuccess;
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
    const bool device_scalars = h->d_lr || h->d_grad_scale || h->d_step;
    bool again = false;
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
        again = again || written_twice(t, *h, device_scalars);
    }
    if (again) return err(FP_ERR_ARG, "fp_adamw_step: an output is another buffer of its tensor, or a device scalar");
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

    Step s;
    memset(&s, 0, sizeof(s));
    s.lr = h->lr; s.beta1 = h->beta1; s.beta2 = h->beta2; s.weight_decay = h->weight_decay; s.step = h->step;
    s.d_lr = h->d_lr; s.d_grad_scale = h->d_grad_scale; s.d_step = reinterpret_cast<const int64_t*>(h->d_step);
    s.b1 = (float)h->beta1; s.ob1 = (float)(1.0 - h->beta1); s.b2 = (float)h->beta2; s.ob2 = (float)(1.0 - h->beta2);
    s.eps = (float)h->eps; s.grad_scale = (float)h->grad_scale; s.one = 1.0f;
    scalars(s, h->lr, h->d_step ? 1 : h->step);
    static const int dtypes[3] = {FP_DTYPE_F32, FP_DTYPE_BF16, FP_DTYPE_F16};
    int left = 0;                                        // tensors that no launch has had yet
    for (int i = 0; i < count; ++i) left += ts[i].n > 0;
    for (int pt : dtypes)                                // a launch has one type of each
        for (int gt : dtypes)
            for (int bits = 8; bits <= 32 && left > 0; bits += 24) {
                const Kind k = {pt, gt, bits};
                int mine = 0;
                for (int i = 0; i < count; ++i) mine += is_of(ts[i], k);
                if (!mine) continue;
                left -= mine;
                const cudaError_t e = mine <= kFewTensors ? run_kind<kFewTensors>(s, ts, count, k, (cudaStream_t)stream)
                                                          : run_kind<kMaxTensors>(s, ts, count, k, (cudaStream_t)stream);
                if (e != cudaSuccess) { cudaGetLastError(); return err(FP_ERR_CUDA, cudaGetErrorString(e)); }
            }
    return FP_OK;
}
