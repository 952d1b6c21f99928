// Softmax cross-entropy of every row and its gradient (fp_cross_entropy).
//
// With m the row's maximum, s = sum exp(x - m):  loss = log s + (m - x_y) - e mean(x - x_y),
// d loss / dx_j = exp(x_j - m) / s - e / C - (1 - e) [j = y].
//
// Memory bound: logits are read once and the gradient written once.  The gradient needs s, so a row has to be kept between the
// two.  Rows of up to 1024 16-byte units stay in the registers of 8, 32 or 256 threads; longer ones in the shared memory of blocks
// of 512, each thread's units in places that it alone reads, so that nothing waits for another thread's copies: up to nine units a thread, 72 KB, leave room for
// three blocks on an SM, and one row's copies run beside another's arithmetic (in registers two blocks fit: 8192 x 32000 logits of 16 bits 212 us).
// A row may be shared by 2, 4 or 8 blocks, a cluster, whose maxima and sums meet in shared memory.  Units lie at
// 16-byte boundaries of memory, whatever the row starts at: its first and last one may be partial.  Where the gradient's row lies
// otherwise than the logits', a warp passes it through shared memory and writes elements, neighbours by neighbouring lanes.  Rows of more than 110000 units are
// read twice.
// Two exponentials and some ten instructions an element are close to what the memory leaves time for, hence: the maximum of 16-bit logits is
// taken two at a time, an exponential's argument is one fused product and sum, what is missing of a partial unit counts as -inf instead
// of being asked for everywhere, and the label's own element is written a second time instead of every element being compared with it.
#include "train_common.cuh"
#include "tc_common.cuh"

#include <math.h>
#include <string.h>

namespace fp {
namespace {

using namespace train;

struct LossParams {
    const void* x;
    const void* labels;
    const float* row_grad;
    float* loss;
    void* dx;
    long long ld_x, ld_dx, ignore, rows;
    int C, label_bytes;
    float smoothing, scale;
    float unit, spread;                                  // of the smoothed mean: 2^-k with 2^k >= 4 C, and smoothing 2^k / C
};

// 2^x; results below 2^-126 are 0.
__device__ __forceinline__ float exp2_of(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
constexpr float kLog2E = 1.4426950408889634f;
__device__ __forceinline__ float exp_of(float d) { return exp2_of(d * kLog2E); }
// e^(x - m) as 2^(x log2e - c) `fix`: c = m log2e rounded, and 2^(c - m log2e), which a fused product and sum gives exactly, makes up for
// the rounding.  That is at most 1/2 for |m| < 1e7 (c below 2^24); of larger m (`far`) the rounding alone would take one factor to 0
// and the other to infinity, so the difference is taken first, whose own rounding is 2^-24 of it: exact where the exponential is not 0.
struct Below {
    float m, c, fix;
    bool far;
    __device__ __forceinline__ explicit Below(float m_) : m(m_) {
        far = !(fabsf(m) < 1e7f);
        c = m * kLog2E;
        fix = far ? 1.0f : exp2_of(-fmaf(m, kLog2E, -c));
    }
    __device__ __forceinline__ float near_value(float x) const { return exp2_of(fmaf(x, kLog2E, -c)); }     // without fix
    __device__ __forceinline__ Two near_values(Two x) const { return exp2_of2(fma2(x, twice(kLog2E), twice(-c))); }
    __device__ __forceinline__ float value(float x) const { return far ? exp_of(x - m) : near_value(x) * fix; }
};

// Maximum, sum of exponentials below it, and sum of `unit` (x - x_y) of a part of a row.  A part of -inf alone has m = -inf, s = 0.
struct Part { float m, s, t; };
__device__ __forceinline__ Part join(const Part& a, const Part& b) {
    Part r;
    r.m = fmaxf(a.m, b.m);
    r.t = a.t + b.t;
    r.s = (a.m == r.m ? a.s : a.s * exp_of(a.m - r.m)) + (b.m == r.m ? b.s : b.s * exp_of(b.m - r.m));
    return r;
}

// 16 bytes of a row.
template <int DT> struct Unit {
    static constexpr int E = DT == FP_DTYPE_F32 ? 4 : 8;
    __device__ __forceinline__ static float get(const uint4& u, int i) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        if (DT == FP_DTYPE_F32) return __uint_as_float(w[i]);
        if (DT == FP_DTYPE_BF16) return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
        return __half2float(__ushort_as_half((uint16_t)(w[i >> 1] >> (16 * (i & 1)))));
    }
    __device__ __forceinline__ static Two pair_at(const uint4& u, int i) { return two(get(u, i), get(u, i + 1)); }
    __device__ __forceinline__ static uint4 make(const float (&v)[8]) {
        if (DT == FP_DTYPE_F32) return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        return make_uint4(to_16x2(v[0], v[1], DT), to_16x2(v[2], v[3], DT), to_16x2(v[4], v[5], DT), to_16x2(v[6], v[7], DT));
    }
    __device__ __forceinline__ static uint4 nothing() {
        const float v[8] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY};
        return make(v);
    }
    __device__ __forceinline__ static uint4 load(const void* x, long long at) {
        return __ldcs(reinterpret_cast<const uint4*>(static_cast<const char*>(x) + at * (16 / E)));
    }
    __device__ __forceinline__ static void store(void* x, long long at, const uint4& u) {
        __stcs(reinterpret_cast<uint4*>(static_cast<char*>(x) + at * (16 / E)), u);
    }
    // the larger of two units, element by element (NaN gives way, as in fmaxf)
    __device__ __forceinline__ static uint4 larger(const uint4& a, const uint4& b) {
        if (DT == FP_DTYPE_F32) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = fmaxf(get(a, i), get(b, i));
            return make(v);
        }
        return make_uint4(pair(a.x, b.x), pair(a.y, b.y), pair(a.z, b.z), pair(a.w, b.w));
    }
    __device__ __forceinline__ static uint32_t pair(uint32_t a, uint32_t b) {
        uint32_t r;
        if (DT == FP_DTYPE_BF16) asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    // elements of memory from the last 16-byte boundary to this row's start
    __device__ __forceinline__ static int shift(const void* x, long long at) {
        return (int)((reinterpret_cast<uintptr_t>(x) + (uintptr_t)at * (16 / E)) & 15) / (16 / E);
    }
};

// What a thread has of its row in the first `used` of its units: the maximum first, then the sum below it.
template <int DT, int V>
__device__ __forceinline__ Part part_of(const uint4 (&u)[V], int used) {
    typedef Unit<DT> U;
    uint4 top = u[0];
#pragma unroll
    for (int k = 1; k < V; ++k) top = U::larger(top, u[k]);
    Part a = {-INFINITY, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < U::E; ++i) a.m = fmaxf(a.m, U::get(top, i));
    const Below e(a.m == -INFINITY ? 0.0f : a.m);        // (of -inf alone every exponential below is 0)
    if (e.far) {
#pragma unroll 1
        for (int i = 0; i < U::E; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < used) a.s += e.value(U::get(u[k], i));
    } else {
        Two s = twice(0.0f);
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k < used)
#pragma unroll
                for (int i = 0; i < U::E; i += 2) s = add2(s, e.near_values(U::pair_at(u[k], i)));
        float lo, hi;
        split(s, lo, hi);
        a.s = (lo + hi) * e.fix;
    }
    return a;
}

// G threads (of a warp, of a block, or of a cluster of `CL` blocks of 1024) join their parts; all get the result.  The order is that of the
// threads' numbers, whatever the rest of the launch does.
template <int G, int CL>
__device__ __forceinline__ Part join_all(Part a, Part* shared) {
#pragma unroll
    for (int d = 1; d < (G < 32 ? G : 32); d <<= 1) {
        Part b;
        b.m = __shfl_xor_sync(~0u, a.m, d); b.s = __shfl_xor_sync(~0u, a.s, d); b.t = __shfl_xor_sync(~0u, a.t, d);
        a = join(a, b);
    }
    if (G <= 32) return a;
    constexpr int W = G / 32;
    const int lane = threadIdx.x & 31;
    if (lane == 0) shared[threadIdx.x >> 5] = a;
    __syncthreads();
    a = shared[lane % W];
#pragma unroll
    for (int d = 1; d < W; d <<= 1) {
        Part b;
        b.m = __shfl_xor_sync(~0u, a.m, d); b.s = __shfl_xor_sync(~0u, a.s, d); b.t = __shfl_xor_sync(~0u, a.t, d);
        a = join(a, b);
    }
    if (CL == 1) return a;
    if (threadIdx.x == 0) shared[32] = a;
    tc::cluster_sync_all();
    Part all[CL];
#pragma unroll
    for (int c = 0; c < CL; ++c) {
        const uint32_t at = tc::cluster_addr(tc::smem_u32(&shared[32]), (uint32_t)c);
        asm volatile("ld.shared::cluster.f32 %0, [%3];\n\tld.shared::cluster.f32 %1, [%3+4];\n\tld.shared::cluster.f32 %2, [%3+8];" : "=f"(all[c].m), "=f"(all[c].s), "=f"(all[c].t) : "r"(at));
    }
    a = all[0];
#pragma unroll
    for (int c = 1; c < CL; ++c) a = join(a, all[c]);
    return a;
}

// `less`: what is taken from x `unit` to have `unit` (x - x_y), exactly but for one rounding and whatever the sizes.  (x itself summed loses what the row
// has in common, 1e4 2^-24 for logits near 1e4, and overflows where two classes are masked by the lowest value.)
struct Row { long long label; float g, label_x, less; bool ignored, bad; };
template <int DT>
__device__ __forceinline__ Row row_of(const LossParams& p, long long row) {
    Row r;
    r.label = p.label_bytes == 4 ? (long long)static_cast<const int32_t*>(p.labels)[row] : static_cast<const long long*>(p.labels)[row];
    r.ignored = r.label == p.ignore;
    r.bad = !r.ignored && (r.label < 0 || r.label >= p.C);
    r.label_x = r.ignored || r.bad ? 0.0f : load1(p.x, row * p.ld_x + r.label, DT);
    r.less = fabsf(r.label_x) < INFINITY ? -r.label_x * p.unit : 0.0f;      // (of a label's logit that is not finite, whatever makes it so is in the sum too)
    r.g = p.scale * (p.row_grad ? p.row_grad[row] : 1.0f);
    return r;
}
__device__ __forceinline__ float loss_of(const LossParams& p, const Row& r, const Part& a) {
    float l;
    if (p.smoothing == 0.0f) l = logf(a.s) - (r.label_x - a.m);
    else l = fmaf(2.0f, fmaf(-0.5f * p.spread, a.t, 0.5f * a.m - 0.5f * r.label_x), logf(a.s));        // (halves: the two may be as far apart as their type goes)
    return r.ignored ? 0.0f : r.bad ? NAN : l;
}

// The gradient's element from x, scale e^(x - m) - off: what is common to a row is in here.
struct Slope {
    Below e;
    float scale, near_scale, off;
    __device__ __forceinline__ Slope(const LossParams& p, const Row& r, const Part& a) : e(a.m) {
        scale = r.bad ? NAN : r.g / a.s;
        near_scale = scale * e.fix;
        off = r.g * (p.smoothing / (float)p.C);
    }
    __device__ __forceinline__ float near_value(float x) const { return fmaf(e.near_value(x), near_scale, -off); }
    __device__ __forceinline__ Two near_values(Two x) const { return fma2(e.near_values(x), twice(near_scale), twice(-off)); }
    __device__ __forceinline__ float operator()(float x) const { return e.far ? fmaf(exp_of(x - e.m), scale, -off) : near_value(x); }
};

// Rows in registers: V units a thread, G threads a row (G < 256: several rows a block of 256).
template <int DT, int G, int V>
__global__ void __launch_bounds__(256, 4) cross_entropy_kernel(const LossParams p) {
    typedef Unit<DT> U;
    constexpr int E = U::E, kStep = G;
    __shared__ Part shared[33];
    __shared__ uint4 staged[G < 32 ? 1 : 256];
    const long long row = (long long)blockIdx.x * (256 / G) + threadIdx.x / G;
    const bool there = row < p.rows;                     // (all threads of a row agree, and of a block of one row)
    const int t = (int)threadIdx.x % G, lane = threadIdx.x & 31;
    const long long at = row * p.ld_x, to = row * p.ld_dx;
    // unit n has elements n E - shift .. of the row; the first and the last may reach over its ends
    const int shift = U::shift(p.x, at), units = there ? (p.C + shift + E - 1) / E : 0, used = (units + kStep - 1) / kStep;
    uint4 u[V];
    auto partial = [&](int n) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < E && (unsigned)(n * E - shift + i) < (unsigned)p.C ? load1(p.x, at + n * E - shift + i, DT) : -INFINITY;
        return U::make(v);
    };
    auto full = [&](int n) { return n * E >= shift && n * E - shift + E <= p.C; };
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int n = t + k * kStep;
        if (n < units && full(n)) u[k] = U::load(p.x, at + (long long)n * E - shift);
        else u[k] = U::nothing();
    }
    Row r = {};
    if (there) {
        r = row_of<DT>(p, row);
        if (t == 0 && !full(0)) u[0] = partial(0);
        if (units > 1 && (units - 1) % kStep == t && !full(units - 1)) {
            const uint4 last = partial(units - 1);
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (t + k * kStep == units - 1) u[k] = last;
        }
    }
    Part a = part_of<DT, V>(u, used);
    if (p.smoothing != 0.0f)
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k < used)
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if ((unsigned)((t + k * kStep) * E - shift + i) < (unsigned)p.C) a.t += fmaf(U::get(u[k], i), p.unit, r.less);
    a = join_all<G, 1>(a, shared);
    if (there && p.loss && t == 0) p.loss[row] = loss_of(p, r, a);
    if (there && p.dx) {
        const Slope slope(p, r, a);
        const float own = slope(r.label_x) - r.g * (1.0f - p.smoothing);         // the label's element
        const bool labelled = !r.ignored && !r.bad;
        const bool alike = U::shift(p.dx, to) == shift;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (k >= used) break;
            const int n = t + k * kStep;
            float v[8] = {};
            if (slope.e.far) {
                if (!r.ignored)
#pragma unroll
                    for (int i = 0; i < E; ++i) v[i] = slope(U::get(u[k], i));
            } else if (!r.ignored) {
#pragma unroll
                for (int i = 0; i < E; i += 2) split(slope.near_values(U::pair_at(u[k], i)), v[i], v[i + 1]);
            }
            if (alike || G < 32) {
                if (alike && n < units && full(n)) U::store(p.dx, to + (long long)n * E - shift, U::make(v));
                else if (n < units)
#pragma unroll
                    for (int i = 0; i < E; ++i)
                        if ((unsigned)(n * E - shift + i) < (unsigned)p.C) store1(p.dx, to + n * E - shift + i, DT, v[i]);
            } else {
                uint4* mine = staged + (threadIdx.x & ~31u);
                mine[lane] = U::make(v);
                __syncwarp();
                const int j0 = (n - lane) * E - shift;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int j = j0 + 32 * i + lane;
                    if ((unsigned)j >= (unsigned)p.C) continue;
                    if (j == r.label && labelled) store1(p.dx, to + j, DT, own);
                    else if (DT == FP_DTYPE_F32) static_cast<float*>(p.dx)[to + j] = reinterpret_cast<const float*>(mine)[32 * i + lane];
                    else static_cast<uint16_t*>(p.dx)[to + j] = reinterpret_cast<const uint16_t*>(mine)[32 * i + lane];
                }
                __syncwarp();
            }
        }
        if ((alike || G < 32) && labelled && (int)((r.label + shift) / E) % kStep == t)      // the thread that has just written it
            store1(p.dx, to + r.label, DT, own);
    }
}

// Rows in shared memory: CL blocks of 512 threads.
template <int DT, int CL>
__global__ void __launch_bounds__(512, 3) cross_entropy_kept_kernel(const LossParams p) {
    typedef Unit<DT> U;
    constexpr int E = U::E, G = 512, kStep = G * CL;
    extern __shared__ uint4 kept[];                      // unit t + k kStep of the row at kept[k G + thread]
    __shared__ Part shared[33];
    const long long row = (long long)(blockIdx.x / CL);
    const int t = (int)(blockIdx.x % CL) * G + (int)threadIdx.x, lane = threadIdx.x & 31;
    const long long at = row * p.ld_x, to = row * p.ld_dx;
    const int shift = U::shift(p.x, at), units = (p.C + shift + E - 1) / E, used = (units + kStep - 1) / kStep;
    auto full = [&](int n) { return n * E >= shift && n * E - shift + E <= p.C; };
    uint4* const mine = kept + threadIdx.x;
    // this thread's units: k = 0 .. count - 1, of which lo .. hi - 1 are whole (only the row's first and last may not be)
    const int count = t < units ? (units - 1 - t) / kStep + 1 : 0;
    const int lo = t == 0 && !full(0) ? 1 : 0, hi = count > lo && !full(t + (count - 1) * kStep) ? count - 1 : max(count, lo);
    {
        const char* src = static_cast<const char*>(p.x) + (at - shift) * (16 / E) + (long long)(t + lo * kStep) * 16;
        uint32_t dst = tc::smem_u32(mine + lo * G);
#pragma unroll 4
        for (int k = lo; k < hi; ++k) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
            src += kStep * 16;
            dst += G * 16;
        }
    }
    auto partial = [&](int k) {
        const int n = t + k * kStep;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < E && (unsigned)(n * E - shift + i) < (unsigned)p.C ? load1(p.x, at + n * E - shift + i, DT) : -INFINITY;
        mine[k * G] = U::make(v);
    };
    if (lo) partial(0);
    if (hi < count) partial(hi);
    const Row r = row_of<DT>(p, row);
    asm volatile("cp.async.wait_all;" ::: "memory");
    Part a = {-INFINITY, 0.0f, 0.0f};
    {
        uint4 top = U::nothing();
#pragma unroll 4
        for (int k = 0; k < count; ++k) top = U::larger(top, mine[k * G]);
#pragma unroll
        for (int i = 0; i < E; ++i) a.m = fmaxf(a.m, U::get(top, i));
        const Below e(a.m == -INFINITY ? 0.0f : a.m);
        if (e.far) {
#pragma unroll 1
            for (int k = 0; k < count; ++k) {
                const uint4 u = mine[k * G];
#pragma unroll
                for (int i = 0; i < E; ++i) a.s += e.value(U::get(u, i));
            }
        } else {
            Two s = twice(0.0f);
#pragma unroll 4
            for (int k = 0; k < count; ++k) {
                const uint4 u = mine[k * G];
#pragma unroll
                for (int i = 0; i < E; i += 2) s = add2(s, e.near_values(U::pair_at(u, i)));
            }
            float lo, hi;
            split(s, lo, hi);
            a.s = (lo + hi) * e.fix;
        }
    }
    if (p.smoothing != 0.0f) {
        const Two unit = twice(p.unit), less = twice(r.less);
        Two s = twice(0.0f);
#pragma unroll 4
        for (int k = lo; k < hi; ++k) {
            const uint4 u = mine[k * G];
#pragma unroll
            for (int i = 0; i < E; i += 2) s = add2(s, fma2(U::pair_at(u, i), unit, less));
        }
        float even, odd;
        split(s, even, odd);
        a.t = even + odd;
        auto edge = [&](int k) {
            const uint4 u = mine[k * G];
#pragma unroll
            for (int i = 0; i < E; ++i)
                if ((unsigned)((t + k * kStep) * E - shift + i) < (unsigned)p.C) a.t += fmaf(U::get(u, i), p.unit, r.less);
        };
        if (lo) edge(0);
        if (hi < count) edge(hi);
    }
    a = join_all<G, CL>(a, shared);                      // (and all have read what dx may overwrite)
    if (p.loss && t == 0) p.loss[row] = loss_of(p, r, a);
    if (p.dx) {
        const Slope slope(p, r, a);
        const float own = slope(r.label_x) - r.g * (1.0f - p.smoothing);         // the label's element
        const bool labelled = !r.ignored && !r.bad, alike = U::shift(p.dx, to) == shift, plain = !r.ignored && !slope.e.far;
        auto gradient = [&](const uint4& u) {
            float v[8];
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = r.ignored ? 0.0f : slope(U::get(u, i));
            return U::make(v);
        };
        char* dst = static_cast<char*>(p.dx) + (to - shift) * (16 / E) + (long long)(t + lo * kStep) * 16;
        if (alike && plain) {
#pragma unroll 4
            for (int k = lo; k < hi; ++k) {
                const uint4 u = mine[k * G];
                float v[8];
#pragma unroll
                for (int i = 0; i < E; i += 2) split(slope.near_values(U::pair_at(u, i)), v[i], v[i + 1]);
                __stcs(reinterpret_cast<uint4*>(dst), U::make(v));
                dst += kStep * 16;
            }
        } else if (alike) {
#pragma unroll 1
            for (int k = lo; k < hi; ++k, dst += kStep * 16) __stcs(reinterpret_cast<uint4*>(dst), gradient(mine[k * G]));
        }
        if (alike) {
            auto edge = [&](int k) {
                const uint4 u = gradient(mine[k * G]);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int j = (t + k * kStep) * E - shift + i;
                    if ((unsigned)j < (unsigned)p.C) store1(p.dx, to + j, DT, U::get(u, i));
                }
            };
            if (lo) edge(0);
            if (hi < count) edge(hi);
            if (labelled && (int)((r.label + shift) / E) % kStep == t) store1(p.dx, to + r.label, DT, own);      // the thread that has just written it
        } else {                                         // through the units' own places
            for (int k = 0; k < used; ++k) {
                uint4* const warps = kept + k * G + (threadIdx.x & ~31u);
                if (k < count) warps[lane] = gradient(mine[k * G]);
                __syncwarp();
                const int j0 = (t - lane + k * kStep) * E - shift;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int j = j0 + 32 * i + lane;
                    if ((unsigned)j >= (unsigned)p.C) continue;
                    if (j == r.label && labelled) store1(p.dx, to + j, DT, own);
                    else if (DT == FP_DTYPE_F32) static_cast<float*>(p.dx)[to + j] = reinterpret_cast<const float*>(warps)[32 * i + lane];
                    else static_cast<uint16_t*>(p.dx)[to + j] = reinterpret_cast<const uint16_t*>(warps)[32 * i + lane];
                }
            }
        }
    }
    if (CL > 1) tc::cluster_sync_all();                  // no block leaves while another may still read its part
}

// Rows that do not fit: read twice, an element at a time, by CL blocks.
template <int DT, int CL>
__global__ void __launch_bounds__(1024) cross_entropy_twice_kernel(const LossParams p) {
    __shared__ Part shared[33];
    const long long row = (long long)(blockIdx.x / CL), step = 1024 * CL;
    const int t = (int)(blockIdx.x % CL) * 1024 + (int)threadIdx.x;
    const long long at = row * p.ld_x, to = row * p.ld_dx;
    const Row r = row_of<DT>(p, row);
    Part a = {-INFINITY, 0.0f, 0.0f};
    constexpr int U = 8;
#pragma unroll 1
    for (long long j = t; j < p.C; j += U * step) {
        float x[U], m = a.m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u] = j + u * step < p.C ? load1(p.x, at + j + u * step, DT) : -INFINITY;
            m = fmaxf(m, x[u]);
        }
        const float m0 = m == -INFINITY ? 0.0f : m;
        if (m > a.m) a.s *= exp_of(a.m - m);             // (0 from -inf)
        a.m = m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            a.s += exp_of(x[u] - m0);
            if (j + u * step < p.C) a.t += fmaf(x[u], p.unit, r.less);
        }
    }
    a = join_all<1024, CL>(a, shared);                   // (and all have read the label's logit: dx may be x)
    if (p.loss && t == 0) p.loss[row] = loss_of(p, r, a);
    if (p.dx) {
        const Slope slope(p, r, a);
#pragma unroll 1
        for (long long j = t; j < p.C; j += U * step) {
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = j + u * step < p.C ? load1(p.x, at + j + u * step, DT) : 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (j + u * step < p.C) store1(p.dx, to + j + u * step, DT, r.ignored ? 0.0f : slope(x[u]));
        }
        if (!r.ignored && !r.bad && r.label % step == t) store1(p.dx, to + r.label, DT, slope(r.label_x) - r.g * (1.0f - p.smoothing));
    }
    if (CL > 1) tc::cluster_sync_all();
}

typedef void (*Kernel)(const LossParams);
struct Choice { Kernel k; int threads, rows_a_block, cluster, smem; };

constexpr int kMostUnits = 27;                           // a thread's units in shared memory: 216 KB a block
constexpr int kOwnSmem = 1024;                           // at least what cross_entropy_kept_kernel has beside them
static_assert(33 * sizeof(Part) <= kOwnSmem && kMostUnits * 512 * 16 + kOwnSmem <= 232448, "a block's shared memory");
template <int DT>
Choice choose(long long C, long long rows) {
    const int sms = sm_count();
    const long long units = (C - 1) / Unit<DT>::E + 2;   // at the worst alignment
    if (units <= 8 * 4) return {cross_entropy_kernel<DT, 8, 4>, 256, 32, 1, 0};
    if (units <= 32 * 4) return {cross_entropy_kernel<DT, 32, 4>, 256, 8, 1, 0};
    // (A warp a row, eight units a lane, once there are rows enough for warps on every SM, or else a block a row: 20000 x 800 f32 26 against 87 us, 20000 x 1900 bf16
    // 38 against 101, 1190 x 800 f32 4.6 against 7.0; 148 x 800 f32 4.0 against 2.6, 600 x 1900 bf16 5.9 against 5.6.  In f32 they meet at fewer rows: 600 x 800 4.0 against 4.6.)
    if (units <= 32 * 8 && rows > 8 * sms) return {cross_entropy_kernel<DT, 32, 8>, 256, 8, 1, 0};
    if (units <= 256 * 4) return {cross_entropy_kernel<DT, 256, 4>, 256, 1, 1, 0};
    // as few blocks a row as leave three on an SM; more where there are few rows
    int cl = 1;
    while (cl < 8 && ((units + 512 * cl - 1) / (512 * cl) > 9 || (rows * cl * 2 <= sms && units > 512 * cl))) cl *= 2;
    const long long each = (units + 512 * cl - 1) / (512 * cl);
    if (each > kMostUnits) return {cross_entropy_twice_kernel<DT, 8>, 1024, 1, 8, 0};
    return {cl == 1 ? cross_entropy_kept_kernel<DT, 1> : cl == 2 ? cross_entropy_kept_kernel<DT, 2> : cl == 4 ? cross_entropy_kept_kernel<DT, 4>
                                                                                             : cross_entropy_kept_kernel<DT, 8>, 512, 1, cl, (int)each * 512 * 16};
}

}  // namespace
}  // namespace fp

using namespace fp;
using namespace fp::train;

extern "C" fp_status fp_cross_entropy(const fp_cross_entropy_args* a, void* stream) {
    if (!a) return err(FP_ERR_ARG, "fp_cross_entropy: NULL argument");
    if (a->rows < 0 || a->classes < 1) return err(FP_ERR_ARG, "fp_cross_entropy: bad sizes (rows >= 0, classes >= 1)");
    if (a->rows > (1ll << 30) || a->classes > (1ll << 30)) return err(FP_ERR_BOUNDS, "fp_cross_entropy: a size beyond 2^30");
    if (a->dtype != FP_DTYPE_F32 && !is_half(a->dtype)) return err(FP_ERR_UNSUPPORTED, "fp_cross_entropy: dtype must be FP_DTYPE_F32, _BF16 or _F16");
    if (a->label_bytes != 4 && a->label_bytes != 8) return err(FP_ERR_ARG, "fp_cross_entropy: label_bytes must be 4 or 8");
    if (!(a->label_smoothing >= 0.0f && a->label_smoothing <= 1.0f)) return err(FP_ERR_ARG, "fp_cross_entropy: label_smoothing must lie in [0, 1]");
    if (a->rows == 0) return FP_OK;
    if (!a->d_logits || !a->d_labels || (!a->d_loss && !a->d_dlogits)) return err(FP_ERR_ARG, "fp_cross_entropy: NULL logits or labels, or no output");
    if (a->rows > 1 && (a->ld_logits < a->classes || (a->d_dlogits && a->ld_dlogits < a->classes)))
        return err(FP_ERR_ARG, "fp_cross_entropy: a row stride is shorter than its row");
    if (a->d_logits == a->d_dlogits && a->rows > 1 && a->ld_logits != a->ld_dlogits)
        return err(FP_ERR_ARG, "fp_cross_entropy: a gradient in the logits' place needs their row stride");
    const int bytes = elem_bytes(a->dtype);
    if ((((uintptr_t)a->d_logits | (uintptr_t)a->d_dlogits) & (uintptr_t)(bytes - 1)) || ((uintptr_t)a->d_labels & (uintptr_t)(a->label_bytes - 1)) ||
        (((uintptr_t)a->d_loss | (uintptr_t)a->d_row_grad) & 3))
        return err(FP_ERR_ARG, "fp_cross_entropy: a buffer is not aligned to its elements");
    auto other = [](const void* out, const void* b) { return out && out == b; };
    if (other(a->d_loss, a->d_logits) || other(a->d_loss, a->d_dlogits) || other(a->d_loss, a->d_labels) || other(a->d_loss, a->d_row_grad) ||
        other(a->d_dlogits, a->d_labels) || other(a->d_dlogits, a->d_row_grad))
        return err(FP_ERR_ARG, "fp_cross_entropy: an output is an input (only dlogits may be the logits) or the other output");
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return err(FP_ERR_CUDA, "fp_cross_entropy: no current device"); }
    Buffers buf(dev);
    if (!buf.here(a->d_logits) || !buf.here(a->d_labels) || !buf.here_or_null(a->d_row_grad) || !buf.here_or_null(a->d_loss) ||
        !buf.here_or_null(a->d_dlogits))
        return err(FP_ERR_ARG, "fp_cross_entropy: a buffer is not memory of the current device");
    LossParams p;
    memset(&p, 0, sizeof(p));
    p.x = a->d_logits; p.labels = a->d_labels; p.row_grad = a->d_row_grad; p.loss = a->d_loss; p.dx = a->d_dlogits;
    p.ld_x = a->ld_logits; p.ld_dx = a->ld_dlogits; p.ignore = a->ignore_index; p.rows = a->rows; p.C = (int)a->classes; p.label_bytes = a->label_bytes;
    p.smoothing = a->label_smoothing; p.scale = a->grad_scale;
    double all = 4.0;
    while (all < 4.0 * (double)p.C) all *= 2.0;
    p.unit = (float)(1.0 / all); p.spread = (float)((double)p.smoothing * all / (double)p.C);
    const Choice c = a->dtype == FP_DTYPE_F32 ? choose<FP_DTYPE_F32>(p.C, p.rows) : a->dtype == FP_DTYPE_BF16 ? choose<FP_DTYPE_BF16>(p.C, p.rows)
                                                                                                        : choose<FP_DTYPE_F16>(p.C, p.rows);
    const long long blocks = (a->rows + c.rows_a_block - 1) / c.rows_a_block * c.cluster;
    if (blocks > 0x7fffffffll) return err(FP_ERR_BOUNDS, "fp_cross_entropy: too many rows of this length");
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)c.threads);
    cfg.dynamicSmemBytes = (size_t)c.smem;
    cfg.stream = (cudaStream_t)stream;
    // (A block has 48 KB without being asked for, of which the kernel's own shared memory is taken first.)
    if (c.smem > 48 * 1024 - kOwnSmem && cudaFuncSetAttribute((const void*)c.k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostUnits * 512 * 16) != cudaSuccess) {
        cudaGetLastError();
        return err(FP_ERR_CUDA, "fp_cross_entropy: no room for a row in shared memory");
    }
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)c.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = c.cluster > 1 ? 1 : 0;
    void* args[1] = {&p};
    const cudaError_t e = cudaLaunchKernelExC(&cfg, (const void*)c.k, args);
    if (e != cudaSuccess) { cudaGetLastError(); return err(FP_ERR_CUDA, cudaGetErrorString(e)); }
    return FP_OK;
}
