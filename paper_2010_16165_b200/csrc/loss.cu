// Softmax cross-entropy of every row and its gradient (fp_cross_entropy).
//
// With m the row's maximum, s = sum exp(x - m):  loss = log s - (1 - e) (x_y - m) - e (mean x - m),
// d loss / dx_j = exp(x_j - m) / s - e / C - (1 - e) [j = y].
#include "train_common.cuh"

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
    long long ld_x, ld_dx, ignore;
    int C, dtype, label_bytes;
    float smoothing, scale;
};

// Running maximum, sum of exponentials below it, and plain sum of a part of a row.  A part of -inf alone has m = -inf, s = 0.
struct Part { float m, s, t; };
__device__ __forceinline__ Part join(const Part& a, const Part& b) {
    Part r;
    r.m = fmaxf(a.m, b.m);
    r.t = a.t + b.t;
    r.s = (a.m == r.m ? a.s : a.s * __expf(a.m - r.m)) + (b.m == r.m ? b.s : b.s * __expf(b.m - r.m));
    return r;
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) cross_entropy_kernel(const LossParams p) {
    __shared__ Part parts[32];
    const long long row = blockIdx.x;
    const long long label = p.label_bytes == 4 ? (long long)static_cast<const int32_t*>(p.labels)[row] : static_cast<const long long*>(p.labels)[row];
    const bool ignored = label == p.ignore, bad = !ignored && (label < 0 || label >= p.C);
    const long long at = row * p.ld_x, to = row * p.ld_dx;
    Part a = {-INFINITY, 0.0f, 0.0f};
    if (!ignored)
        for (int j = threadIdx.x; j < p.C; j += THREADS) {
            const float x = load1(p.x, at + j, p.dtype);
            a.t += x;
            if (x > a.m) { a.s = a.m == -INFINITY ? 0.0f : a.s * __expf(a.m - x); a.m = x; }
            if (x != -INFINITY) a.s += __expf(x - a.m);
        }
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        Part b;
        b.m = __shfl_xor_sync(~0u, a.m, d); b.s = __shfl_xor_sync(~0u, a.s, d); b.t = __shfl_xor_sync(~0u, a.t, d);
        a = join(a, b);
    }
    if ((threadIdx.x & 31) == 0) parts[threadIdx.x >> 5] = a;
    __syncthreads();
    a = parts[0];
    for (int w = 1; w < THREADS / 32; ++w) a = join(a, parts[w]);
    float label_x = 0.0f;
    if (!ignored && !bad) label_x = load1(p.x, at + label, p.dtype);
    if (p.loss && threadIdx.x == 0) {
        float l = logf(a.s) - (1.0f - p.smoothing) * (label_x - a.m);
        if (p.smoothing != 0.0f) l -= p.smoothing * (a.t / (float)p.C - a.m);
        p.loss[row] = ignored ? 0.0f : bad ? NAN : l;
    }
    if (!p.dx) return;
    __syncthreads();                                     // the label's logit has been read: dx may be x
    const float g = p.scale * (p.row_grad ? p.row_grad[row] : 1.0f), inv = 1.0f / a.s, off = p.smoothing / (float)p.C;
    for (int j = threadIdx.x; j < p.C; j += THREADS) {
        float d = __expf(load1(p.x, at + j, p.dtype) - a.m) * inv - off;
        if (j == label) d -= 1.0f - p.smoothing;
        store1(p.dx, to + j, p.dtype, ignored ? 0.0f : bad ? NAN : d * g);
    }
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
    if ((((uintptr_t)a->d_logits | (uintptr_t)a->d_dlogits) & (uintptr_t)(elem_bytes(a->dtype) - 1)) || ((uintptr_t)a->d_labels & (uintptr_t)(a->label_bytes - 1)) ||
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
    p.ld_x = a->ld_logits; p.ld_dx = a->ld_dlogits; p.ignore = a->ignore_index; p.C = (int)a->classes; p.dtype = a->dtype; p.label_bytes = a->label_bytes;
    p.smoothing = a->label_smoothing; p.scale = a->grad_scale;
    cross_entropy_kernel<256><<<(unsigned)a->rows, 256, 0, (cudaStream_t)stream>>>(p);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? FP_OK : err(FP_ERR_CUDA, cudaGetErrorString(e));
}
