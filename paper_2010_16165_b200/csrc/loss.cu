// Softmax cross-entropy of every row and its gradient (fp_cross_entropy).
//
// With m the row's maximum, s = sum exp(x - m):  loss = log s - (1 - e) (x_y - m) - e (mean x - m),
// d loss / dx_j = exp(x_j - m) / s - e / C - (1 - e) [j = y].
//
// Memory bound: logits are read once and the gradient written once.  The gradient needs s, so a row has to be kept between the
// two: in registers.  A thread has up to kMaxVecs 16-byte vectors of its row, and a row is shared by as many threads as
// that takes: 8, 32 .. 1024, or 4 or 8 blocks of 1024 as a cluster (half a million logits of 16 bits) whose maxima and sums meet in shared memory.  Longer rows, and rows
// whose starts are not aligned to 16 bytes, are read twice by the same number of threads (the second time out of L2 where it
// holds them).
#include "train_common.cuh"
#include "tc_common.cuh"

#include <math.h>
#include <string.h>

#include <algorithm>

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
};

// Maximum, sum of exponentials below it, and plain sum of a part of a row.  A part of -inf alone has m = -inf, s = 0.
struct Part { float m, s, t; };
__device__ __forceinline__ Part join(const Part& a, const Part& b) {
    Part r;
    r.m = fmaxf(a.m, b.m);
    r.t = a.t + b.t;
    r.s = (a.m == r.m ? a.s : a.s * __expf(a.m - r.m)) + (b.m == r.m ? b.s : b.s * __expf(b.m - r.m));
    return r;
}

template <int DT> struct Elems { static constexpr int kPer = DT == FP_DTYPE_F32 ? 4 : 8; };      // elements of 16 bytes
template <int DT>
__device__ __forceinline__ float elem(const uint4& u, int i) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    if (DT == FP_DTYPE_F32) return __uint_as_float(w[i]);
    return to_f32((uint16_t)(w[i >> 1] >> (16 * (i & 1))), DT);
}
template <int DT>
__device__ __forceinline__ uint4 vec_of(const float* v) {
    if (DT == FP_DTYPE_F32) return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    return make_uint4(to_16x2(v[0], v[1], DT), to_16x2(v[2], v[3], DT), to_16x2(v[4], v[5], DT), to_16x2(v[6], v[7], DT));
}

// What a thread adds up of its row: the maximum of its elements first, then the sum below it.
template <int DT, int V>
__device__ __forceinline__ Part part_of(const uint4 (&u)[V], int vecs, int count_last) {
    constexpr int E = Elems<DT>::kPer;
    Part a = {-INFINITY, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (k < vecs)
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (k < vecs - 1 || i < count_last) a.m = fmaxf(a.m, elem<DT>(u[k], i));
    const float m = a.m == -INFINITY ? 0.0f : a.m;       // (of -inf alone every exponential below is 0)
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (k < vecs)
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (k < vecs - 1 || i < count_last) {
                    const float x = elem<DT>(u[k], i);
                    a.t += x;
                    a.s += __expf(x - m);
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
    Part r;
#pragma unroll 1
    for (int c = 0; c < CL; ++c) {
        const uint32_t at = tc::cluster_addr(tc::smem_u32(&shared[32]), (uint32_t)c);
        Part b;
        asm volatile("ld.shared::cluster.f32 %0, [%3];\n\tld.shared::cluster.f32 %1, [%3+4];\n\tld.shared::cluster.f32 %2, [%3+8];" : "=f"(b.m), "=f"(b.s), "=f"(b.t) : "r"(at));
        r = c ? join(r, b) : b;
    }
    return r;
}

struct Row { long long label; float g, label_x; bool ignored, bad; };
template <int DT>
__device__ __forceinline__ Row row_of(const LossParams& p, long long row) {
    Row r;
    r.label = p.label_bytes == 4 ? (long long)static_cast<const int32_t*>(p.labels)[row] : static_cast<const long long*>(p.labels)[row];
    r.ignored = r.label == p.ignore;
    r.bad = !r.ignored && (r.label < 0 || r.label >= p.C);
    r.label_x = r.ignored || r.bad ? 0.0f : load1(p.x, row * p.ld_x + r.label, DT);
    r.g = p.scale * (p.row_grad ? p.row_grad[row] : 1.0f);
    return r;
}
__device__ __forceinline__ float loss_of(const LossParams& p, const Row& r, const Part& a) {
    float l = logf(a.s) - (1.0f - p.smoothing) * (r.label_x - a.m);
    if (p.smoothing != 0.0f) l -= p.smoothing * (a.t / (float)p.C - a.m);
    return r.ignored ? 0.0f : r.bad ? NAN : l;
}

// Rows in registers: V vectors a thread, G threads a row (G < 256: several rows a block of 256), CL blocks.
template <int DT, int G, int V, int CL>
__global__ void __launch_bounds__(G < 256 ? 256 : G) cross_entropy_kernel(const LossParams p) {
    constexpr int E = Elems<DT>::kPer, B = G < 256 ? 256 : G;
    __shared__ Part shared[33];
    const long long row = CL > 1 ? (long long)(blockIdx.x / CL) : (long long)blockIdx.x * (B / G) + threadIdx.x / G;
    const bool there = row < p.rows;                     // (all threads of a row, and of a block of several warps a row, agree)
    const int t = (CL > 1 ? (int)(blockIdx.x % CL) * G : 0) + (int)threadIdx.x % G;
    const int all = (p.C + E - 1) / E, vecs = there && t < all ? (all - 1 - t) / (G * CL) + 1 : 0;
    const int last = t + (vecs - 1) * G * CL, count_last = vecs > 0 ? min(E, p.C - last * E) : 0;
    Row r = {};
    uint4 u[V];
    if (there) {
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const char*>(p.x) + row * p.ld_x * (16 / E));
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k < vecs - 1 || (k == vecs - 1 && count_last == E)) u[k] = __ldcs(src + t + k * G * CL);
            else if (k == vecs - 1) {                    // the row's end inside a vector
                float v[8] = {};
#pragma unroll
                for (int i = 0; i < E; ++i) if (i < count_last) v[i] = load1(p.x, row * p.ld_x + (long long)last * E + i, DT);
                u[k] = vec_of<DT>(v);
            }
        r = row_of<DT>(p, row);
    }
    const Part a = join_all<G, CL>(part_of<DT, V>(u, vecs, count_last), shared);
    if (there && p.loss && t == 0) p.loss[row] = loss_of(p, r, a);
    if (there && p.dx) {
        const float inv = 1.0f / a.s, off = p.smoothing / (float)p.C;
        uint4* dst = reinterpret_cast<uint4*>(static_cast<char*>(p.dx) + row * p.ld_dx * (16 / E));
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k < vecs) {
                float v[8];
                const long long j0 = (long long)(t + k * G * CL) * E;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    float d = __expf(elem<DT>(u[k], i) - a.m) * inv - off;
                    if (j0 + i == r.label) d -= 1.0f - p.smoothing;
                    v[i] = r.ignored ? 0.0f : r.bad ? NAN : d * r.g;
                }
                if (k < vecs - 1 || count_last == E) __stcs(dst + t + k * G * CL, vec_of<DT>(v));
                else
#pragma unroll
                    for (int i = 0; i < E; ++i) if (i < count_last) store1(p.dx, row * p.ld_dx + j0 + i, DT, v[i]);
            }
    }
    if (CL > 1) tc::cluster_sync_all();                  // no block leaves while another may still read its part
}

// Rows that do not fit, or do not start at 16-byte boundaries: read twice, an element at a time.
template <int DT, int CL>
__global__ void __launch_bounds__(1024) cross_entropy_twice_kernel(const LossParams p) {
    __shared__ Part shared[33];
    const long long row = (long long)(blockIdx.x / CL);
    const int t = (int)(blockIdx.x % CL) * 1024 + (int)threadIdx.x;
    const long long at = row * p.ld_x, to = row * p.ld_dx;
    const Row r = row_of<DT>(p, row);
    Part a = {-INFINITY, 0.0f, 0.0f};
    constexpr int U = 8;
#pragma unroll 1
    for (int j = t; j < p.C; j += U * 1024 * CL) {
        float x[U], m = a.m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u] = j + u * 1024 * CL < p.C ? load1(p.x, at + j + u * 1024 * CL, DT) : -INFINITY;
            m = fmaxf(m, x[u]);
        }
        const float m0 = m == -INFINITY ? 0.0f : m;
        if (m > a.m) a.s = a.m == -INFINITY ? 0.0f : a.s * __expf(a.m - m);
        a.m = m;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j + u * 1024 * CL < p.C) { a.t += x[u]; a.s += __expf(x[u] - m0); }
    }
    a = join_all<1024, CL>(a, shared);
    if (p.loss && t == 0) p.loss[row] = loss_of(p, r, a);
    if (p.dx) {
        const float inv = 1.0f / a.s, off = p.smoothing / (float)p.C;
        if (CL == 1) __syncthreads();                    // the label's logit has been read by all (dx may be x); a cluster has met above
#pragma unroll 1
        for (int j = t; j < p.C; j += U * 1024 * CL) {
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = j + u * 1024 * CL < p.C ? load1(p.x, at + j + u * 1024 * CL, DT) : 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = j + u * 1024 * CL;
                if (c >= p.C) break;
                float d = __expf(x[u] - a.m) * inv - off;
                if (c == r.label) d -= 1.0f - p.smoothing;
                store1(p.dx, to + c, DT, r.ignored ? 0.0f : r.bad ? NAN : d * r.g);
            }
        }
    }
    if (CL > 1) tc::cluster_sync_all();
}

typedef void (*Kernel)(const LossParams);
struct Choice { Kernel k; int threads, rows_a_block, cluster; };

constexpr int kMaxVecs = 8;
// The fewest threads that hold a row in kMaxVecs vectors each.
template <int DT>
Choice choose(long long C, long long rows, bool vectors) {
    const int sms = sm_count();
    const long long vecs = (C + Elems<DT>::kPer - 1) / Elems<DT>::kPer;
    if (vectors) {
        if (vecs <= 8 * 4) return {cross_entropy_kernel<DT, 8, 4, 1>, 256, 32, 1};
        if (vecs <= 32 * 8) return {cross_entropy_kernel<DT, 32, 8, 1>, 256, 8, 1};
        if (vecs <= 256 * 4) return {cross_entropy_kernel<DT, 256, 4, 1>, 256, 1, 1};
        if (vecs <= 512 * 8) return {cross_entropy_kernel<DT, 512, 8, 1>, 512, 1, 1};
        if (vecs <= 1024 * 8 && rows * 4 > sms) return {cross_entropy_kernel<DT, 1024, 8, 1>, 1024, 1, 1};
        if (vecs <= 1024 * 8 * 4) return {cross_entropy_kernel<DT, 1024, 8, 4>, 1024, 1, 4};
        if (vecs <= 1024 * 8 * 8) return {cross_entropy_kernel<DT, 1024, 8, 8>, 1024, 1, 8};
    }
    if (C > 16384 && rows * 8 <= 2 * sms) return {cross_entropy_twice_kernel<DT, 8>, 1024, 1, 8};
    return {cross_entropy_twice_kernel<DT, 1>, 1024, 1, 1};
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
    const bool vectors = (((uintptr_t)a->d_logits | (uintptr_t)a->d_dlogits) & 15) == 0 &&
                         (a->rows == 1 || (a->ld_logits * bytes % 16 == 0 && (!a->d_dlogits || a->ld_dlogits * bytes % 16 == 0)));
    const Choice c = a->dtype == FP_DTYPE_F32 ? choose<FP_DTYPE_F32>(p.C, p.rows, vectors) : a->dtype == FP_DTYPE_BF16 ? choose<FP_DTYPE_BF16>(p.C, p.rows, vectors)
                                                                                          : choose<FP_DTYPE_F16>(p.C, p.rows, vectors);
    const long long blocks = (a->rows + c.rows_a_block - 1) / c.rows_a_block * c.cluster;
    if (blocks > 0x7fffffffll) return err(FP_ERR_BOUNDS, "fp_cross_entropy: too many rows of this length");
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)c.threads);
    cfg.stream = (cudaStream_t)stream;
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
