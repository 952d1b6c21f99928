// Fully connected layers and their gradients (fp_linear_forward, fp_linear_backward).
//
// All three products are D(i, j) = sum_k A(i, k) B(j, k) on the tensor cores, which take either operand with k or with i (j)
// contiguous in memory, so that nothing is transposed beforehand:
//     y  = x w'    A = x  (rows m, k contiguous)     B = w  (rows n, k contiguous)
//     dx = dz w    A = dz (rows m, n contiguous)     B = w  read with its rows as the sum's index, its columns contiguous
//     dw = dz' x   A = dz and B = x, both with the sum's index m as rows
// Operands come by tensor-map copies (zeros outside the matrix, so ragged sizes need no other code); those need 16-byte
// aligned rows, and an operand that has none is copied into scratch first.
#include "train_common.cuh"
#include "tc_common.cuh"

#include <cuda.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <atomic>

namespace fp {
namespace {

using namespace tc;
using namespace train;

constexpr int kBlockK = 64;                              // elements of the sum a stage: 128 bytes, a swizzled row
constexpr int64_t kMaxSize = 1ll << 30;
constexpr int kMaxSmem = 232448, kAllSmem = kMaxSmem - 512;      // shared memory a block may have, and without what these kernels have statically

__device__ int g_linear_status;                          // raised by a bounded wait that ran out

// The tensor cores cut a sum's low bits at every step instead of rounding, always toward zero: after 1024 terms 32-bit sums are 1e-6 too small, after
// 16384 2e-5 (measured; with terms of random signs).  Results in 16 bits do not show it; where a result is written in 32 bits, a sum is
// taken in runs of at most kRun K blocks (where there is room for that many), which are added by rounded additions.
constexpr int kRun = 8;

// What is done with a finished sum.  Outputs are rows of n neighbours; n is j, or with few rows (linear_tile_kernel) i.
struct Epilogue {
    void* y;
    void* pre;
    const void* res;
    const void* bias;                                    // by n
    long long ld_y, ld_pre, ld_res;
    int y_type, pre_type, res_type, bias_type, act, res_first;
    int vec;                                             // 1: four neighbours of every buffer lie aligned
};
struct Problem {
    CUtensorMap a, b;                                    // boxes of 64 k x rows, or 64 rows x 64 k (…_mn)
    int I, J, kblocks;
    int tiles_i, tiles_j, tile0;                         // this problem's tiles are tile0 ..
    int a_mn, b_mn;
    Epilogue e;
};
struct DzParams {
    const uint16_t* dy;
    const uint16_t* pre;
    uint16_t* out[2];
    void* db;
    long long ld_dy, ld_pre, ld_out[2], M;
    int N, act, dtype, db_type, accumulate, splits;
};
struct TileParams {
    Problem prob[2];
    int n_prob, stages, tiles;
    int run;                                             // K blocks that an accumulator adds up before another one takes over (see kRun)
    int late;                                            // this launch's operands were there before the launch in front of it began: see after_the_last()
    uint32_t bf16;
    int* status;
    DzParams sums;                                       // linear_split_kernel: column sums of dy, by clusters behind the tiles'
    int sums_vec;
};

// Bounded wait by polling.  (A try_wait with a time hint sleeps in steps of 2.05 us here: products of some microseconds took whole
// multiples of that.)
__device__ __forceinline__ bool mbar_poll(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit_cycles = kWaitCycles) {
    if (mbar_test_wait(bar, parity)) return true;
    const long long t0 = clock64();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (mbar_test_wait(bar, parity)) return true;
        if (*abort_flag || clock64() - t0 > limit_cycles) return false;
    }
}
// Launches of these kernels overlap: each may begin while the one before it ends, prepares its barriers, and then waits here for
// that one's results.  It lets the next one begin after that wait, so when the next one runs, all that was complete before
// THIS launch is; a product that needs no more (the second of a call) is `late`: it waits only before it ends, so that whatever
// follows it still follows both.
// Tensor memory: an allocation blocks while other CTAs of the SM hold the columns, so a CTA that holds some must never wait for one that may be
// blocked.  Hence it is taken after the wait for the launch before, and before the next launch may begin; and the CTAs of a
// cluster, which wait for each other, take an SM's whole shared memory (kAllSmem), so that no other CTA with tensor memory, of this stream or of
// another, is on their SMs.
__device__ __forceinline__ void after_the_last(int late) {
    if (!late) asm volatile("griddepcontrol.wait;" ::: "memory");
}
__device__ __forceinline__ void let_the_next_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void before_the_end(int late) {
    if (late) asm volatile("griddepcontrol.wait;" ::: "memory");
}
// Cycles after which a wait for a whole sum has run out: a block of 64 terms takes some hundred.
__device__ __forceinline__ long long sum_limit(int kblocks) { return kWaitCycles + 4096ll * kblocks; }

// A copy whose fields are in registers.  (Read where they are needed, through the pointer to the chosen problem, they were loaded
// again for every few rows: 500 cycles a time.)
__device__ __forceinline__ Epilogue held(const Epilogue& from) {
    Epilogue e = from;
    asm volatile("" : "+l"(e.y), "+l"(e.pre), "+l"(e.res), "+l"(e.bias), "+l"(e.ld_y), "+l"(e.ld_pre), "+l"(e.ld_res));
    asm volatile("" : "+r"(e.y_type), "+r"(e.pre_type), "+r"(e.res_type), "+r"(e.bias_type), "+r"(e.act), "+r"(e.res_first), "+r"(e.vec));
    return e;
}
// A lane's C outputs of a row: neighbours n .. n + 3 where four neighbours lie aligned in every buffer (STRIDE 1), or else n, n + 32, ..., so that
// neighbouring lanes have neighbouring columns.  What exists of them and of U rows is asked once, types once for all of them:
// asked at every element, code that runs twice a launch was fetched for longer than it ran (829 x 2816 x 256 with an unaligned residual 44 us).
template <int C, int STRIDE>
__device__ __forceinline__ uint32_t columns_in(int n, int N) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < C; ++i) m |= n + STRIDE * i < N ? 1u << i : 0u;
    return m;
}
template <int C, int STRIDE>
__device__ __forceinline__ void bias_of(const Epilogue& e, int n, int N, float (&b)[C]) {
#pragma unroll
    for (int i = 0; i < C; ++i) b[i] = e.bias && n + STRIDE * i < N ? load1(e.bias, n + STRIDE * i, e.bias_type) : 0.0f;
}
// The residual of U rows `step` apart, `rows` of which exist.
template <int U, int C, int STRIDE>
__device__ __forceinline__ void fetch(const Epilogue& e, long long row, int step, int rows, int n, uint32_t in, float (&r)[U][C]) {
    if (!e.res) return;
    const int bytes = e.res_type == FP_DTYPE_F32 ? 4 : 2;
    const char* from = static_cast<const char*>(e.res) + (row * e.ld_res + n) * bytes;
    const long long hop = step * e.ld_res * bytes;
    if (STRIDE == 1 && C == 4 && in == 15u) {
#pragma unroll
        for (int u = 0; u < U; ++u, from += hop)
            if (u < rows) load4(from, 0, e.res_type, reinterpret_cast<float(&)[4]>(r[u]));
    } else if (bytes == 4) {
#pragma unroll
        for (int u = 0; u < U; ++u, from += hop)
#pragma unroll
            for (int i = 0; i < C; ++i) if (u < rows && (in >> i & 1u)) r[u][i] = reinterpret_cast<const float*>(from)[STRIDE * i];
    } else {
        uint16_t w[U][C];
#pragma unroll
        for (int u = 0; u < U; ++u, from += hop)
#pragma unroll
            for (int i = 0; i < C; ++i) w[u][i] = u < rows && (in >> i & 1u) ? reinterpret_cast<const uint16_t*>(from)[STRIDE * i] : (uint16_t)0;
        const bool bf16 = e.res_type == FP_DTYPE_BF16;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < C; ++i) r[u][i] = bf16 ? __uint_as_float((uint32_t)w[u][i] << 16) : __half2float(__ushort_as_half(w[u][i]));
    }
}
template <int U, int C, int STRIDE>
__device__ __forceinline__ void put(void* base, long long ld, int type, long long row, int step, int rows, int n, uint32_t in, const float (&v)[U][C]) {
    const int bytes = type == FP_DTYPE_F32 ? 4 : 2;
    char* to = static_cast<char*>(base) + (row * ld + n) * bytes;
    const long long hop = step * ld * bytes;
    if (STRIDE == 1 && C == 4 && in == 15u) {
#pragma unroll
        for (int u = 0; u < U; ++u, to += hop)
            if (u < rows) store4(to, 0, type, reinterpret_cast<const float(&)[4]>(v[u]));
    } else if (bytes == 4) {
#pragma unroll
        for (int u = 0; u < U; ++u, to += hop)
#pragma unroll
            for (int i = 0; i < C; ++i) if (u < rows && (in >> i & 1u)) reinterpret_cast<float*>(to)[STRIDE * i] = v[u][i];
    } else {
        const bool bf16 = type == FP_DTYPE_BF16;
#pragma unroll
        for (int u = 0; u < U; ++u, to += hop)
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const uint16_t h = bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v[u][i])) : __half_as_ushort(__float2half_rn(v[u][i]));
                if (u < rows && (in >> i & 1u)) reinterpret_cast<uint16_t*>(to)[STRIDE * i] = h;
            }
    }
}
// The outputs from their sums v, biases b and residuals r.  `e` is the caller's own copy: its fields stay in registers.
template <int U, int C, int STRIDE>
__device__ __forceinline__ void finish(const Epilogue& e, long long row, int step, int rows, int n, uint32_t in, float (&v)[U][C], const float (&b)[C], const float (&r)[U][C]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < C; ++i) {
            v[u][i] += b[i];
            if (e.res && e.res_first) v[u][i] += r[u][i];
        }
    if (e.pre) put<U, C, STRIDE>(e.pre, e.ld_pre, e.pre_type, row, step, rows, n, in, v);
    act_all(v, e.act);
    if (e.res && !e.res_first)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < C; ++i) v[u][i] += r[u][i];
    put<U, C, STRIDE>(e.y, e.ld_y, e.y_type, row, step, rows, n, in, v);
}
// Four words of a row of sums: neighbours, or every 32nd.
template <bool VEC>
__device__ __forceinline__ void lds4(uint32_t addr, float (&v)[4]) {
    if (VEC) asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(addr));
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v[i]) : "r"(addr + 128u * (uint32_t)i));
}
template <bool VEC>
__device__ __forceinline__ void lds4_cluster(uint32_t addr, float (&v)[4]) {
    if (VEC) asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(addr));
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[i]) : "r"(addr + 128u * (uint32_t)i));
}

// 128 columns of sums (n0 .. of the outputs), finished by a warp: rows r0, r0 + step, ... below `rows` of those at `base` (pitch words apart), which
// are rows row0 + r of the outputs; the sum's S parts are in the shared memory of CTAs first, first + every, ... of the cluster and are added in that order.  U rows
// at once: another CTA's memory answers after a thousand cycles, as the residual's does.
template <int S, int U, bool VEC>
__device__ __forceinline__ void finish_rows(const Epilogue& e, uint32_t base, int pitch, int r0, int step, int rows, long long row0, int n0, int N, uint32_t first,
                                            uint32_t every) {
    const int lane = threadIdx.x & 31, n = n0 + (VEC ? 4 * lane : lane);
    constexpr int STRIDE = VEC ? 1 : 32;
    if (n >= N) return;
    const uint32_t in = columns_in<4, STRIDE>(n, N);
    float bias[4];
    bias_of<4, STRIDE>(e, n, N, bias);
    auto sums = [&](int r, float (&v)[U][4]) {
        uint32_t at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) at[u] = base + (uint32_t)(min(r + u * step, rows - 1) * pitch + (VEC ? 4 : 1) * lane) * 4u;
        if (S > 1) {
            float part[U][S][4];
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int u = 0; u < U; ++u) lds4_cluster<VEC>(cluster_addr(at[u], first + every * (uint32_t)s), part[u][s]);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[u][i] = part[u][0][i];
#pragma unroll
                    for (int s = 1; s < S; ++s) v[u][i] += part[u][s][i];
                }
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) lds4<VEC>(at[u], v[u]);
        }
    };
    if (VEC && n + 4 <= N && !e.res && !e.pre && e.act == FP_ACT_NONE) {       // nothing but a bias: a gradient, or logits
        const int bytes = e.y_type == FP_DTYPE_F32 ? 4 : 2;
        char* to = static_cast<char*>(e.y) + ((row0 + r0) * e.ld_y + n) * bytes;
        const long long hop = step * e.ld_y * bytes;
#pragma unroll 1
        for (int r = r0; r < rows; r += U * step) {
            float v[U][4];
            sums(r, v);
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[u][i] += bias[i];
                if (r + u * step < rows) store4(to, 0, e.y_type, v[u]);
                to += hop;
            }
        }
        return;
    }
#pragma unroll 1
    for (int r = r0; r < rows; r += U * step) {
        float v[U][4], res[U][4];
        const int there = (rows - r + step - 1) / step;
        fetch<U, 4, STRIDE>(e, row0 + r, step, there, n, in, res);
        sums(r, v);
        finish<U, 4, STRIDE>(e, row0 + r, step, there, n, in, v, bias, res);
    }
}

// ---- few rows: 128 outputs x BN rows a cluster ----------------------------------------------------------------------
// With few rows (M <= 128) the weights take the 128 rows of the tensor core's tile and the activations its BN columns: a
// single token costs 16 columns instead of 128 rows, and the weights' bytes are all that counts.  S CTAs share a
// tile's sum, a range of K blocks each; their parts meet in shared memory, where every CTA finishes some rows (the terms in the
// CTAs' order: one order of sums for a size).  1 x 1000 x 2048: 4.4 us; 16 x 16384 x 4096: 25 us, 20.6 of them the weights at the copy rate.

constexpr int kTileThreads = 256;
struct TileCtrl {
    uint64_t full[16], empty[16], done;
    uint32_t tmem;
    int abort_flag;
};

template <int BN, int S>
__global__ void __launch_bounds__(kTileThreads) linear_tile_kernel(const __grid_constant__ TileParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ TileCtrl ctrl;
    constexpr uint32_t kStage = 128 * 128 + BN * 128;
    constexpr int kMost = 512 / BN < 16 ? 512 / BN : 16;             // accumulators at most
    const uint32_t cols = p.run ? (uint32_t)(kMost * BN) : BN < 32 ? 32u : (uint32_t)BN;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = S > 1 ? cluster_rank() : 0u;
    const Problem& q = p.prob[0];
    const int tile = (int)(blockIdx.x / (unsigned)S), i0 = tile * 128;
    const int kb0 = (int)((long long)q.kblocks * rank / S), kb1 = (int)((long long)q.kblocks * (rank + 1) / S);
    // accumulators of this CTA's part of the sum: one, or one every `run` K blocks
    const int run = p.run ? max(p.run, (kb1 - kb0 + kMost - 1) / kMost) : kb1 - kb0, sums = (kb1 - kb0 + run - 1) / run;
    volatile int* abort_flag = &ctrl.abort_flag;
    const uint32_t full0 = smem_u32(ctrl.full), empty0 = smem_u32(ctrl.empty), done = smem_u32(&ctrl.done);

    if (warp == 0) {
        if (lane == 0) {
            prefetch_map(&q.a);
            prefetch_map(&q.b);
            for (int s = 0; s < p.stages; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
            mbar_init(done, 1);
            ctrl.abort_flag = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            // While the launch before ends, the first weights come into L2 (which is where memory is one: what that launch still
            // writes of them is found there all the same).
            for (int kb = kb0; kb < min(kb1, kb0 + p.stages); ++kb) {
                if (q.a_mn) {
                    tma_prefetch_2d(&q.a, i0, kb * kBlockK);
                    tma_prefetch_2d(&q.a, i0 + 64, kb * kBlockK);
                } else {
                    tma_prefetch_2d(&q.a, kb * kBlockK, i0);
                }
            }
        }
    }
    after_the_last(p.late);
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctrl.tmem)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctrl.tmem;
    let_the_next_begin();
    bool ok = true;
    if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0;
        for (int kb = kb0; kb < kb1; ++kb) {
            if (kb - kb0 >= p.stages) ok = __all_sync(0xffffffffu, mbar_poll(empty0 + 8 * stage, phase ^ 1u, abort_flag));
            if (!ok) break;
            if (elect_one()) {
                const uint32_t bar = full0 + 8 * stage, a = base + (uint32_t)stage * kStage, b = a + 128 * 128;
                mbar_expect_tx(bar, kStage);
                const int k = kb * kBlockK;
                if (q.a_mn) {
                    tma_load_2d(a, &q.a, i0, k, bar);
                    tma_load_2d(a + 8192, &q.a, i0 + 64, k, bar);
                } else {
                    tma_load_2d(a, &q.a, k, i0, bar);
                }
                tma_load_2d(b, &q.b, k, 0, bar);
            }
            __syncwarp();
            if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
    } else if (warp == 1) {
        const uint32_t idesc = f16_idesc((int)p.bf16, q.a_mn, 0, 128, BN), a_step = q.a_mn ? 128u : 2u;
        int stage = 0;
        uint32_t phase = 0;
        uint32_t d = tmem;
        int left = run;                                  // K blocks until the next accumulator
        for (int kb = kb0; kb < kb1; ++kb) {
            ok = __all_sync(0xffffffffu, mbar_poll(full0 + 8 * stage, phase, abort_flag));
            if (!ok) break;
            tc_fence_after();
            bool begins = kb == kb0;
            if (left == 0) { left = run; d += BN; begins = true; }
            --left;
            const uint32_t a = base + (uint32_t)stage * kStage;
            const uint32_t al = sw128_lo(a, 8192), bl = sw128_lo(a + 128 * 128, 8192), leader = elect_one();
#pragma unroll
            for (int s = 0; s < 4; ++s) umma_sw128_if(leader, d, al + (uint32_t)s * a_step, bl + (uint32_t)s * 2u, idesc, !begins || s ? 1u : 0u);
            if (leader) {
                umma_commit(empty0 + 8 * stage);
                if (kb == kb1 - 1) umma_commit(done);
            }
            __syncwarp();
            if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
    }
    if (!ok && lane == 0) { atomicExch(&ctrl.abort_flag, 1); atomicExch(p.status, 1); }
    if (ok) {
        ok = __all_sync(0xffffffffu, mbar_poll(done, 0, abort_flag, sum_limit(kb1 - kb0)));
        if (!ok && lane == 0) { atomicExch(&ctrl.abort_flag, 1); atomicExch(p.status, 1); }
    }
    tc_fence_after();
    if (*abort_flag)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);         // copies in flight land before the memory is used again
    __syncthreads();                                             // every stage has been read: its memory takes the sums now

    // Sums in shared memory as rows of 128 outputs.  A pitch of 4 (mod 32) words keeps 16-byte accesses of neighbouring lanes in
    // different banks.
    constexpr int kPitch = 132;
    const Epilogue e = held(q.e);
    const int rows = q.J;
    {
        const int col = (warp & 3) * 32 + lane;
        const uint32_t taddr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
#pragma unroll
        for (int c = 0; c < BN / 16; ++c) {
            const int r = 8 * (2 * c + (warp >> 2));
            if (r >= rows) break;
            uint32_t v[8];
            tmem_ld8(taddr + (uint32_t)r, v);
            tmem_ld_wait();
#pragma unroll 1
            for (int x = 1; x < sums; ++x) {
                uint32_t u[8];
                tmem_ld8(taddr + (uint32_t)(x * BN + r), u);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(u[i]));
            }
            const uint32_t to = base + (uint32_t)(r * kPitch + col) * 4u;
#pragma unroll
            for (int i = 0; i < 8; ++i) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + (uint32_t)(i * kPitch) * 4u), "r"(v[i]) : "memory");
        }
    }
    tc_fence_before();
    if (S > 1) cluster_sync_all();
    else __syncthreads();
    // warp w of CTA r: every (8 S)th row from 8 r + w on
    constexpr int U = S >= 8 || BN < 32 ? 1 : S == 4 ? 2 : 4;
    if (e.vec) finish_rows<S, U, true>(e, base, kPitch, (int)rank * 8 + warp, 8 * S, rows, 0, i0, q.I, 0u, 1u);
    else finish_rows<S, U, false>(e, base, kPitch, (int)rank * 8 + warp, 8 * S, rows, 0, i0, q.I, 0u, 1u);
    __syncwarp();
    if (S > 1) cluster_sync_all();                        // no CTA leaves while another may still read its sums
    else __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
    }
    before_the_end(p.late);
}

// ---- 256 x 256 tiles by CTA pairs -----------------------------------------------------------------------------------
// Large products.  A 128 x 256 tile a CTA reads 48 KB of shared memory for 512 cycles of its tensor core, three quarters of what
// the memory gives, with the epilogue's share on top; a pair of CTAs with one 256 x 256 tile (cta_group::2) holds half of B
// each and reads 32 KB.  Pairs are persistent; accumulators of two tiles fill tensor memory, so that a tile is finished by eight
// warps while the next one is summed.  Warp 0 copies, warp 1 of the pair's first CTA issues the MMAs, warps 4-11 finish.
// With RUNS the accumulators hold runs of a tile's sum instead (see kRun): sixteen warps add them up in registers.
// What bounds it is L2: 32 KB a K block into every SM, 2.1 GB for 4096 x 8192 x 4096, in 190 us: 11.3 TB/s; the tensor pipe is active for 74-78 %.
// 8192 x 16384 x 4096 takes 810-880 us plain, by card (10 TB/s), 820-945 with gelu and a kept pre-activation (a library product 780-810).  Eight row tiles at a time over all column
// tiles keep what runs at once in L2: with 4, 6, 12, 16, 24 and 32 it took 5, 3, 1, 1, 5 and 11 % longer, with K ranges that begin
// at different places in different pairs 5 %.

constexpr uint32_t kPairStage = 2 * 128 * 128;           // bytes of a stage in each CTA: 128 rows of A, 128 of B
constexpr uint32_t kEpiPitch = 36;                       // words; 16-byte accesses of neighbouring lanes in different banks
constexpr uint32_t kEpiWarp = 32 * kEpiPitch * 4;
template <bool RUNS> struct PairShape {
    static constexpr int kWarps = RUNS ? 16 : 8, kThreads = 128 + 32 * kWarps, kStages = RUNS ? 4 : 5, kCols = 1024 / kWarps;      // warps that finish, and a warp's columns
    static_assert(kStages * (int)kPairStage + kWarps * (int)kEpiWarp + 1024 <= kAllSmem, "");
};
struct PairCtrl {
    uint64_t full[5], empty[5], sums_full[2], sums_empty[2];
    uint32_t tmem;
    int abort_flag;
};

struct Place { const Problem* q; int i0, j0; };
template <int BN>
__device__ __forceinline__ Place pair_place(const TileParams& p, int tile_all) {
    Place r;
    r.q = &p.prob[p.n_prob > 1 && tile_all >= p.prob[1].tile0 ? 1 : 0];
    const int tile = tile_all - r.q->tile0;
    const int group = tile / (8 * r.q->tiles_j), in_group = tile - group * 8 * r.q->tiles_j, rows_here = min(8, r.q->tiles_i - group * 8);
    r.i0 = (group * 8 + in_group % rows_here) * 256;
    r.j0 = (in_group / rows_here) * BN;
    return r;
}

// ROWS rows of an operand (from row0 on, 64 terms of the sum from k on) into this CTA's stage.
template <int ROWS>
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap& map, int mn, int row0, int k, uint32_t bar) {
    if (mn) {
        tma_load_2d_pair(dst, &map, row0, k, bar);
        if (ROWS > 64) tma_load_2d_pair(dst + 8192, &map, row0 + 64, k, bar);
    } else {
        tma_load_2d_pair(dst, &map, k, row0, bar);
    }
}

template <bool RUNS>
__global__ void __launch_bounds__(PairShape<RUNS>::kThreads, 1) linear_pair_kernel(const __grid_constant__ TileParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ PairCtrl ctrl;
    typedef PairShape<RUNS> Shape;
    constexpr int kStages = Shape::kStages, kCols = Shape::kCols;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int pair = (int)(blockIdx.x >> 1), pairs = (int)(gridDim.x >> 1);
    volatile int* abort_flag = &ctrl.abort_flag;
    const uint32_t full0 = smem_u32(ctrl.full), empty0 = smem_u32(ctrl.empty), sums_full = smem_u32(ctrl.sums_full), sums_empty = smem_u32(ctrl.sums_empty);

    if (warp == 0) {
        if (lane == 0) {
            for (int i = 0; i < p.n_prob; ++i) { prefetch_map(&p.prob[i].a); prefetch_map(&p.prob[i].b); }
            for (int s = 0; s < kStages; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
            for (int s = 0; s < 2; ++s) { mbar_init(sums_full + 8 * s, 1); mbar_init(sums_empty + 8 * s, 2 * Shape::kWarps); }
            ctrl.abort_flag = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
    }
    after_the_last(p.late);
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctrl.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    tc_fence_before();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = ctrl.tmem;
    let_the_next_begin();
    bool ok = true;
    if (warp == 0) {
        uint32_t stage = 0, phase = 0;
        bool again = false;                              // whether the ring has come round
        for (int t = pair; t < p.tiles && ok; t += pairs) {
            const Place w = pair_place<256>(p, t);
            const int i0 = w.i0 + 128 * (int)rank, j0 = w.j0 + 128 * (int)rank;
            for (int kb = 0; kb < w.q->kblocks; ++kb) {
                if (again) ok = __all_sync(0xffffffffu, mbar_poll(empty0 + 8 * stage, phase ^ 1u, abort_flag));
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t own = full0 + 8 * stage, bar = cluster_addr(own, 0), a = base + stage * kPairStage;
                    if (rank == 0) mbar_expect_tx(own, 2 * kPairStage);
                    load_rows<128>(a, w.q->a, w.q->a_mn, i0, kb * kBlockK, bar);
                    load_rows<128>(a + 128 * 128, w.q->b, w.q->b_mn, j0, kb * kBlockK, bar);
                }
                __syncwarp();
                if (++stage == kStages) { stage = 0; phase ^= 1u; again = true; }
            }
        }
    } else if (warp == 1 && rank == 0) {
        uint32_t stage = 0, phase = 0, n = 0;
        for (int t = pair; t < p.tiles && ok; t += pairs) {
            const Place w = pair_place<256>(p, t);
            const uint32_t idesc = f16_idesc((int)p.bf16, w.q->a_mn, w.q->b_mn, 256, 256);
            const uint32_t a_step = w.q->a_mn ? 128u : 2u, b_step = w.q->b_mn ? 128u : 2u;
            uint32_t d = tmem;
            int left = 0;                                // K blocks until the next accumulator
            for (int kb = 0; kb < w.q->kblocks; ++kb) {
                const bool begins = RUNS ? left == 0 : kb == 0;
                if (begins) {
                    left = p.run;
                    d = tmem + (n & 1) * 256u;
                    if (n >= 2) ok = __all_sync(0xffffffffu, mbar_poll(sums_empty + 8 * (n & 1), ((n >> 1) & 1u) ^ 1u, abort_flag));
                    if (!ok) break;
                }
                ok = __all_sync(0xffffffffu, mbar_poll(full0 + 8 * stage, phase, abort_flag));
                if (!ok) break;
                tc_fence_after();
                const uint32_t a = base + stage * kPairStage, al = sw128_lo(a, 8192), bl = sw128_lo(a + 128 * 128, 8192), leader = elect_one();
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    umma_sw128_pair_if(leader, d, al + (uint32_t)s * a_step, bl + (uint32_t)s * b_step, idesc, !begins || s ? 1u : 0u);
                const bool ends = kb == w.q->kblocks - 1 || (RUNS && --left == 0);
                if (leader) {
                    umma_commit_pair(empty0 + 8 * stage, 0);
                    if (ends) umma_commit_pair(sums_full + 8 * (n & 1), 0);
                }
                __syncwarp();
                if (ends) ++n;
                if (++stage == kStages) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp >= 4) {
        const int quarter = warp & 3, col_w = ((warp - 4) >> 2) * kCols;
        const uint32_t buf = base + kStages * kPairStage + (uint32_t)(warp - 4) * kEpiWarp, taddr = tmem + ((uint32_t)(32 * quarter) << 16) + (uint32_t)col_w;
        const uint32_t put = buf + (uint32_t)lane * (kEpiPitch * 4), get = buf + (uint32_t)(lane >> 3) * (kEpiPitch * 4) + (uint32_t)(lane & 7) * 16u;
        uint32_t n = 0;
        for (int t = pair; t < p.tiles && ok; t += pairs) {
            const Place w = pair_place<256>(p, t);
            const Epilogue e = held(w.q->e);
            float sum[2][RUNS ? 32 : 1];                 // with RUNS: this lane's columns col_w .., 32 and 32
            if (RUNS)
#pragma unroll
                for (int i = 0; i < 64; ++i) sum[i >> 5][RUNS ? i & 31 : 0] = 0.0f;
            if (RUNS) {
                for (int kb = 0; kb < w.q->kblocks; kb += p.run, ++n) {
                    ok = __all_sync(0xffffffffu, mbar_poll(sums_full + 8 * (n & 1), (n >> 1) & 1u, abort_flag, sum_limit(p.run)));
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t v[16];
                        tmem_ld16(taddr + (n & 1) * 256u + (uint32_t)(16 * c), v);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[c >> 1][RUNS ? 16 * (c & 1) + i : 0] += __uint_as_float(v[i]);
                    }
                    tc_fence_before();
                    if (lane == 0) mbar_arrive_cluster(cluster_addr(sums_empty + 8 * (n & 1), 0));
                }
            } else {
                ok = __all_sync(0xffffffffu, mbar_poll(sums_full + 8 * (n & 1), (n >> 1) & 1u, abort_flag, sum_limit(w.q->kblocks)));
                tc_fence_after();
            }
            if (!ok) break;
            const int row0 = w.i0 + 128 * (int)rank + 32 * quarter;
#pragma unroll 1
            for (int c = 0; c < kCols / 32; ++c) {
                uint32_t v[32];
                const int col0 = w.j0 + col_w + 32 * c;
                if (RUNS) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) { v[i] = __float_as_uint(sum[0][RUNS ? i : 0]); sum[0][RUNS ? i : 0] = sum[1][RUNS ? i : 0]; }
                } else {
                    tmem_ld32(taddr + (n & 1) * 256u + (uint32_t)(32 * c), v);
                    tmem_ld_wait();
                    if (c == kCols / 32 - 1) {           // the accumulator is free for the tile after the next
                        tc_fence_before();
                        if (lane == 0) mbar_arrive_cluster(cluster_addr(sums_empty + 8 * (n & 1), 0));
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(put + (uint32_t)i * 16u), "r"(v[4 * i]), "r"(v[4 * i + 1]), "r"(v[4 * i + 2]), "r"(v[4 * i + 3]) : "memory");
                __syncwarp();
                if (e.vec) {                             // four rows at a time, eight lanes a row
                    const int col = col0 + (lane & 7) * 4, rows = w.q->I - row0 - (lane >> 3);
                    if (col < w.q->J) {
                        const uint32_t in = columns_in<4, 1>(col, w.q->J);
                        float bias[4];
                        bias_of<4, 1>(e, col, w.q->J, bias);
                        constexpr int U = RUNS ? 1 : 4;
#pragma unroll 1
                        for (int r = 0; r < 8; r += U) {
                            float x[U][4], res[U][4];
                            const int there = (rows - 4 * r + 3) / 4;
                            fetch<U, 4, 1>(e, row0 + (lane >> 3) + 4 * r, 4, there, col, in, res);
#pragma unroll
                            for (int u = 0; u < U; ++u) lds4<true>(get + (uint32_t)(4 * (r + u)) * (kEpiPitch * 4), x[u]);
                            finish<U, 4, 1>(e, row0 + (lane >> 3) + 4 * r, 4, there, col, in, x, bias, res);
                        }
                    }
                } else if (col0 + lane < w.q->J) {       // a lane a column
                    const int col = col0 + lane;
                    float bias[1];
                    bias_of<1, 1>(e, col, w.q->J, bias);
                    constexpr int U = RUNS ? 8 : 16;
#pragma unroll 1
                    for (int r = 0; r < 32; r += U) {
                        float x[U][1], res[U][1];
                        fetch<U, 1, 1>(e, row0 + r, 1, w.q->I - row0 - r, col, 1u, res);
#pragma unroll
                        for (int u = 0; u < U; ++u) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x[u][0]) : "r"(buf + (uint32_t)((r + u) * kEpiPitch + lane) * 4u));
                        finish<U, 1, 1>(e, row0 + r, 1, w.q->I - row0 - r, col, 1u, x, bias, res);
                    }
                }
                __syncwarp();
            }
            if (!RUNS) ++n;
        }
    }
    if (!ok && lane == 0) { atomicExch(&ctrl.abort_flag, 1); atomicExch(p.status, 1); }
    if (*abort_flag)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);         // copies in flight land before the memory is given back
    tc_fence_before();
    cluster_sync_all();                                          // no CTA leaves while the other may still signal it
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    before_the_end(p.late);
}

// ---- dz and the bias's gradient -------------------------------------------------------------------------------------
// dz = dy * act'(pre), rounded into up to two places, and its column sums.  A cluster of CTAs has 128 columns; each CTA takes a
// range of rows, half a warp a row, eight columns a lane.  Column sums: a thread's rows, then the halves of warps, then the CTAs, each
// in order.  Memory bound: 6 bytes an element with an activation.
// Where there is nothing but column sums to take, a product's launch takes them along (linear_split_kernel).

template <int DT, int ACT, bool VEC, int HALVES>
__device__ __forceinline__ void dz_columns(const DzParams& p, int block, int share, float (*part)[128], float* sums) {
    const int lane = threadIdx.x & 15, half = threadIdx.x >> 4, n0 = block * 128;
    const long long m0 = p.M * share / p.splits, m1 = p.M * (share + 1) / p.splits;
    Two s[4] = {};                                       // (zeros)
    // columns of a thread: eight neighbours, or (rows that are not aligned) every sixteenth
    auto col = [&](int i) { return n0 + (VEC ? 8 * lane + i : lane + 16 * i); };
    auto load = [&](const uint16_t* base, long long row) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (VEC) { if (col(0) < p.N) u = __ldcs(reinterpret_cast<const uint4*>(base + row + col(0))); }
        else {
            uint32_t w[4] = {};
#pragma unroll
            for (int i = 0; i < 8; ++i) if (col(i) < p.N) w[i >> 1] |= (uint32_t)base[row + col(i)] << (16 * (i & 1));
            u = make_uint4(w[0], w[1], w[2], w[3]);
        }
        return u;
    };
    auto value = [](const uint4& u, int i) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        return to_f32((uint16_t)(w[i >> 1] >> (16 * (i & 1))), DT);
    };
    constexpr int kRows = VEC ? 4 : 2;                   // rows a thread has in flight
#pragma unroll 1
    for (long long m = m0 + half; m < m1; m += HALVES * kRows) {
        uint4 g[kRows], z[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if (m + HALVES * r < m1) {
                g[r] = load(p.dy, (m + HALVES * r) * p.ld_dy);
                if (ACT != FP_ACT_NONE) z[r] = load(p.pre, (m + HALVES * r) * p.ld_pre);
            }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (m + HALVES * r >= m1) break;
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                Two x = two(value(g[r], i), value(g[r], i + 1));
                if (ACT != FP_ACT_NONE) x = mul2(x, act_grad2<ACT>(two(value(z[r], i), value(z[r], i + 1))));
                s[i / 2] = add2(s[i / 2], x);
                split(x, d[i], d[i + 1]);
            }
            const uint4 u = make_uint4(to_16x2(d[0], d[1], DT), to_16x2(d[2], d[3], DT), to_16x2(d[4], d[5], DT), to_16x2(d[6], d[7], DT));
#pragma unroll
            for (int o = 0; o < 2; ++o)
                if (p.out[o]) {
                    uint16_t* to = p.out[o] + (m + HALVES * r) * p.ld_out[o];
                    if (VEC) { if (col(0) < p.N) *reinterpret_cast<uint4*>(to + col(0)) = u; }
                    else
#pragma unroll
                        for (int i = 0; i < 8; ++i) if (col(i) < p.N) to[col(i)] = to_16(d[i], DT);
                }
        }
    }
    if (!p.db) return;                                   // (the same for all CTAs of a cluster)
#pragma unroll
    for (int i = 0; i < 8; i += 2) split(s[i / 2], part[half][col(i) - n0], part[half][col(i + 1) - n0]);
    __syncthreads();
    float v = 0.0f;
    if (threadIdx.x < 128) {
#pragma unroll
        for (int w = 0; w < HALVES; ++w) v += part[w][threadIdx.x];
        sums[threadIdx.x] = v;
    }
    if (p.splits > 1) cluster_sync_all();
    if (share == 0 && threadIdx.x < 128) {
        float u[8];
#pragma unroll
        for (int c = 1; c < 8; ++c)
            if (c < p.splits) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(u[c]) : "r"(cluster_addr(smem_u32(&sums[threadIdx.x]), (uint32_t)c)));
#pragma unroll
        for (int c = 1; c < 8; ++c)
            if (c < p.splits) v += u[c];
        const int n = n0 + (int)threadIdx.x;
        if (n < p.N) store1(p.db, n, p.db_type, p.accumulate ? load1(p.db, n, p.db_type) + v : v);
    }
    if (p.splits > 1) cluster_sync_all();
}

// ---- 256 x BN tiles with the sum split over pairs -----------------------------------------------------------------------
// Products of fewer tiles than there are pairs: S pairs (a cluster of 2 S CTAs) share a tile's sum, as with few rows.
// An SM takes 64 bytes a cycle from L2, so tiles are what counts: 32 KB a K block for 512 cycles of the tensor cores at BN = 256, 24 KB (392
// cycles measured) for 256 cycles' work at BN = 128; 128 x 128 tiles of single CTAs need 32 KB for 256 cycles' work and ran at half the
// rate however they were spread.  Another CTA's sums come at 16 bytes a cycle, 4096 cycles for half a tile of 256 columns.

constexpr int kSplitThreads = 512;
template <int BN> struct SplitShape {
    static constexpr int kStages = BN == 256 ? 5 : 7, kPitch = BN + 4;     // words of a row of sums: 16-byte accesses of neighbouring lanes in different banks
    static constexpr uint32_t kStage = 128 * 128 + BN / 2 * 128;
    static_assert(kStages * (int)kStage + 1024 <= kAllSmem && 128 * kPitch * 4 <= kStages * (int)kStage, "the sums take the stages' memory");
};
struct SplitCtrl {
    uint64_t full[8], empty[8], done;
    uint32_t tmem;
    int abort_flag;
};

template <int BN, int S>
__global__ void __launch_bounds__(kSplitThreads, 1) linear_split_kernel(const __grid_constant__ TileParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ SplitCtrl ctrl;
    typedef SplitShape<BN> Shape;
    constexpr int kStages = Shape::kStages;
    constexpr uint32_t kStage = Shape::kStage;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank(), half = rank & 1u, first = rank & ~1u;      // this CTA's place in its pair, and the pair's first CTA
    const int split = (int)(rank >> 1);
    const int cluster = (int)(blockIdx.x / (unsigned)(2 * S));
    if (cluster >= p.tiles) {                            // columns of dy to be summed
        float (*part)[128] = reinterpret_cast<float (*)[128]>(smem_raw);
        float* sums = reinterpret_cast<float*>(smem_raw) + 32 * 128;
        after_the_last(p.late);
        let_the_next_begin();
        if (p.bf16 && p.sums_vec) dz_columns<FP_DTYPE_BF16, FP_ACT_NONE, true, 32>(p.sums, cluster - p.tiles, (int)rank, part, sums);
        else if (p.bf16) dz_columns<FP_DTYPE_BF16, FP_ACT_NONE, false, 32>(p.sums, cluster - p.tiles, (int)rank, part, sums);
        else if (p.sums_vec) dz_columns<FP_DTYPE_F16, FP_ACT_NONE, true, 32>(p.sums, cluster - p.tiles, (int)rank, part, sums);
        else dz_columns<FP_DTYPE_F16, FP_ACT_NONE, false, 32>(p.sums, cluster - p.tiles, (int)rank, part, sums);
        before_the_end(p.late);
        return;
    }
    const Place w = pair_place<BN>(p, cluster);
    const Problem& q = *w.q;
    const int i0 = w.i0 + 128 * (int)half;
    const int kb0 = (int)((long long)q.kblocks * split / S), kb1 = (int)((long long)q.kblocks * (split + 1) / S);
    // accumulators of this CTA's part of the sum: one, or one every `run` K blocks, as many as tensor memory holds
    const int run = p.run ? max(p.run, (kb1 - kb0 + 512 / BN - 1) / (512 / BN)) : kb1 - kb0, sums = (kb1 - kb0 + run - 1) / run;
    volatile int* abort_flag = &ctrl.abort_flag;
    const uint32_t full0 = smem_u32(ctrl.full), empty0 = smem_u32(ctrl.empty), done = smem_u32(&ctrl.done);

    if (warp == 0) {
        if (lane == 0) {
            prefetch_map(&q.a);
            prefetch_map(&q.b);
            for (int s = 0; s < kStages; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
            mbar_init(done, 1);
            ctrl.abort_flag = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
    }
    after_the_last(p.late);
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctrl.tmem)), "r"(p.run ? 512u : (uint32_t)BN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    tc_fence_before();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = ctrl.tmem;
    let_the_next_begin();
    bool ok = true;
    if (warp == 0) {
        uint32_t stage = 0, phase = 0;
        const int j0 = w.j0 + BN / 2 * (int)half;
        for (int kb = kb0; kb < kb1; ++kb) {
            if (kb - kb0 >= kStages) ok = __all_sync(0xffffffffu, mbar_poll(empty0 + 8 * stage, phase ^ 1u, abort_flag));
            if (!ok) break;
            if (elect_one()) {
                const uint32_t own = full0 + 8 * stage, bar = cluster_addr(own, first), a = base + stage * kStage;
                if (half == 0) mbar_expect_tx(own, 2 * kStage);
                load_rows<128>(a, q.a, q.a_mn, i0, kb * kBlockK, bar);
                load_rows<BN / 2>(a + 128 * 128, q.b, q.b_mn, j0, kb * kBlockK, bar);
            }
            __syncwarp();
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
    } else if (warp == 1 && half == 0) {
        uint32_t stage = 0, phase = 0;
        const uint32_t idesc = f16_idesc((int)p.bf16, q.a_mn, q.b_mn, 256, BN), a_step = q.a_mn ? 128u : 2u, b_step = q.b_mn ? 128u : 2u;
        uint32_t d = tmem;
        int left = run;                                  // K blocks until the next accumulator
        for (int kb = kb0; kb < kb1; ++kb) {
            ok = __all_sync(0xffffffffu, mbar_poll(full0 + 8 * stage, phase, abort_flag));
            if (!ok) break;
            tc_fence_after();
            bool begins = kb == kb0;
            if (left == 0) { left = run; d += BN; begins = true; }
            --left;
            const uint32_t a = base + stage * kStage, al = sw128_lo(a, 8192), bl = sw128_lo(a + 128 * 128, 8192), leader = elect_one();
#pragma unroll
            for (int s = 0; s < 4; ++s)
                umma_sw128_pair_if(leader, d, al + (uint32_t)s * a_step, bl + (uint32_t)s * b_step, idesc, !begins || s ? 1u : 0u);
            if (leader) {
                umma_commit_pair(empty0 + 8 * stage, first);
                if (kb == kb1 - 1) umma_commit_pair(done, first);
            }
            __syncwarp();
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
    }
    if (!ok && lane == 0) { atomicExch(&ctrl.abort_flag, 1); atomicExch(p.status, 1); }
    if (ok) {
        ok = __all_sync(0xffffffffu, mbar_poll(done, 0, abort_flag, sum_limit(kb1 - kb0)));
        if (!ok && lane == 0) { atomicExch(&ctrl.abort_flag, 1); atomicExch(p.status, 1); }
    }
    tc_fence_after();
    if (*abort_flag)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);         // copies in flight land before the memory is used again
    __syncthreads();                                             // every stage has been read: its memory takes the sums now
    {
        constexpr int kCols = BN / 4;                    // a warp's columns
        const uint32_t taddr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)((warp >> 2) * kCols);
        const uint32_t to = base + (uint32_t)(((warp & 3) * 32 + lane) * Shape::kPitch + (warp >> 2) * kCols) * 4u;
#pragma unroll
        for (int c = 0; c < kCols / 32; ++c) {
            uint32_t v[32];
            tmem_ld32(taddr + (uint32_t)(32 * c), v);
            tmem_ld_wait();
#pragma unroll 1
            for (int x = 1; x < sums; ++x) {
                uint32_t u[32];
                tmem_ld32(taddr + (uint32_t)(x * BN + 32 * c), u);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(u[i]));
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (uint32_t)(32 * c + 4 * i) * 4u), "r"(v[4 * i]), "r"(v[4 * i + 1]), "r"(v[4 * i + 2]), "r"(v[4 * i + 3]) : "memory");
        }
    }
    tc_fence_before();
    if (S > 1) cluster_sync_all();
    else __syncthreads();
    // Row r of this half of the tile is finished by warp r % 16 of pair (r / 16) % S.
    const Epilogue e = held(q.e);
    constexpr int U = S == 3 ? 3 : 8 / S < 4 ? 8 / S : 4;
#pragma unroll 1
    for (int c = 0; c < BN / 128; ++c) {
        const uint32_t from = base + 512u * (uint32_t)c;
        const int rows = min(128, q.I - i0), n0 = w.j0 + 128 * c;
        if (e.vec) finish_rows<S, U, true>(e, from, Shape::kPitch, split * 16 + warp, 16 * S, rows, i0, n0, q.J, half, 2u);
        else finish_rows<S, U, false>(e, from, Shape::kPitch, split * 16 + warp, 16 * S, rows, i0, n0, q.J, half, 2u);
    }
    __syncwarp();
    cluster_sync_all();                                          // no CTA leaves while another may still read its sums or signal it
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.run ? 512u : (uint32_t)BN) : "memory");
    }
    before_the_end(p.late);
}

// ---- operands that tensor-map copies cannot read --------------------------------------------------------------------

struct CopyJob {
    const uint16_t* src;
    uint16_t* dst;
    long long ld_src, ld_dst, rows;
    int cols, chunks;                                    // chunks of 512 elements a row
    long long warp0;
};
struct CopyParams { CopyJob job[2]; long long warps; };

// Rows of 16-bit elements of any alignment into rows that start at 16-byte boundaries.  A warp moves 512 elements, 64 bytes an
// instruction: whatever the alignment the lines are used whole.
__global__ void __launch_bounds__(256) copy_rows_kernel(const __grid_constant__ CopyParams p) {
    after_the_last(0);
    let_the_next_begin();
    const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (w >= p.warps) return;
    const CopyJob& j = p.job[w >= p.job[1].warp0 ? 1 : 0];
    const long long u = w - j.warp0, row = u / j.chunks;
    const int c0 = (int)(u - row * j.chunks) * 512 + (threadIdx.x & 31);
    const uint16_t* s = j.src + row * j.ld_src;
    uint16_t* d = j.dst + row * j.ld_dst;
    uint16_t v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = c0 + 32 * i < j.cols ? s[c0 + 32 * i] : (uint16_t)0;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (c0 + 32 * i < j.cols) d[c0 + 32 * i] = v[i];
}

// ---- dz by itself ----------------------------------------------------------------------------------------------------

template <int DT, int ACT, bool VEC, int HALVES>
__global__ void __launch_bounds__(16 * HALVES, HALVES == 16 ? 4 : 1) linear_dz_kernel(const DzParams p) {
    __shared__ float part[HALVES][128];
    __shared__ float sums[128];
    after_the_last(0);
    let_the_next_begin();
    dz_columns<DT, ACT, VEC, HALVES>(p, (int)(blockIdx.x / (unsigned)p.splits), (int)(blockIdx.x % (unsigned)p.splits), part, sums);
}

typedef void (*DzKernel)(const DzParams);
template <int DT, int ACT>
DzKernel dz_kernel(bool vec, bool narrow) {
    return vec ? (narrow ? linear_dz_kernel<DT, ACT, true, 64> : linear_dz_kernel<DT, ACT, true, 16>)
               : (narrow ? linear_dz_kernel<DT, ACT, false, 64> : linear_dz_kernel<DT, ACT, false, 16>);
}
template <int DT>
DzKernel dz_kernel(int act, bool vec, bool narrow) {
    return act == FP_ACT_RELU ? dz_kernel<DT, FP_ACT_RELU>(vec, narrow) : act == FP_ACT_GELU ? dz_kernel<DT, FP_ACT_GELU>(vec, narrow)
         : act == FP_ACT_GELU_TANH ? dz_kernel<DT, FP_ACT_GELU_TANH>(vec, narrow) : act == FP_ACT_SILU ? dz_kernel<DT, FP_ACT_SILU>(vec, narrow)
                                                                                                 : dz_kernel<DT, FP_ACT_NONE>(vec, narrow);
}

// ---- host -----------------------------------------------------------------------------------------------------------

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// A matrix of `rows` rows of `cols` contiguous 16-bit elements; boxes of 64 x box_rows.
bool make_map(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows, int dtype) {
    static std::atomic<void*> known;
    const EncodeTiled encode = (EncodeTiled)driver_function("cuTensorMapEncodeTiled", &known);
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? ld : (cols + 7) / 8 * 8) * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, one[2] = {1, 1};
    return encode(map, dtype == FP_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(base), dims,
                  strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool readable(const void* p, int64_t rows, int64_t ld) { return ((uintptr_t)p & 15) == 0 && (rows <= 1 || (ld & 7) == 0); }
bool aligned4(const void* p, int64_t ld, int dtype, int64_t rows) {
    return ((uintptr_t)p & (uintptr_t)(4 * elem_bytes(dtype) - 1)) == 0 && (rows <= 1 || (ld & 3) == 0);
}
size_t packed_bytes(int64_t rows, int64_t cols) { return ((size_t)rows * (size_t)((cols + 7) / 8 * 8) * 2 + 255) / 256 * 256; }

int* status_word(int dev) {
    static std::atomic<int*> known[64];
    if (dev < 0 || dev >= 64) return nullptr;
    int* p = known[dev].load(std::memory_order_acquire);
    if (!p) {
        if (cudaGetSymbolAddress((void**)&p, g_linear_status) != cudaSuccess) { cudaGetLastError(); return nullptr; }
        known[dev].store(p, std::memory_order_release);
    }
    return p;
}

// Shared memory that a kernel may have, asked for once on each device.
template <typename K>
cudaError_t allow_smem(K kernel, int bytes, std::atomic<unsigned long long>* done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = 1ull << (dev & 63);
    if (dev < 64 && (done->load(std::memory_order_acquire) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < 64) done->fetch_or(bit, std::memory_order_release);
    return e;
}

struct Operand { const void* p; int64_t rows, cols, ld; int mn; };   // mn: rows are the sum's index
struct Product { Operand a, b; int64_t I, J, Kc; int swap; Epilogue e; };

// Fills in a launch's problems for tiles of ti x tj, B in boxes of box_b rows.
fp_status lay_out(const Product* prod, int n, int ti, int tj, int box_b, int dtype, TileParams* p) {
    int64_t tiles = 0;
    for (int i = 0; i < n; ++i) {
        const Product& r = prod[i];
        Problem& q = p->prob[i];
        q.I = (int)r.I; q.J = (int)r.J; q.kblocks = (int)((r.Kc + kBlockK - 1) / kBlockK);
        q.tiles_i = (int)((r.I + ti - 1) / ti); q.tiles_j = (int)((r.J + tj - 1) / tj);
        q.tile0 = (int)tiles;
        tiles += (int64_t)q.tiles_i * q.tiles_j;
        if (tiles > (1 << 27)) return err(FP_ERR_BOUNDS, "fp_linear: more tiles than a launch takes");
        q.a_mn = r.a.mn; q.b_mn = r.b.mn; q.e = r.e;
        if (!make_map(&q.a, r.a.p, r.a.rows, r.a.cols, r.a.ld, r.a.mn ? 64 : 128, dtype) ||
            !make_map(&q.b, r.b.p, r.b.rows, r.b.cols, r.b.ld, r.b.mn ? 64 : box_b, dtype))
            return err(FP_ERR_CUDA, "fp_linear: an operand's tensor map was refused");
    }
    p->n_prob = n; p->tiles = (int)tiles;
    return FP_OK;
}

// A launch in clusters that may begin while the launch before it ends (see after_the_last).
template <typename K, typename P>
cudaError_t launch_clusters(K kernel, const P& p, long long blocks, int threads, int smem, int cluster, cudaStream_t st) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

// CTAs of linear_split_kernel that run at once in clusters of 2 S: a cluster lies within a group of SMs (B200: 148 in pairs, 132 in
// fours, 120 in eights), and one cluster too many takes as long as all others (1024 x 1024 x 1024 in 16 clusters of eight 19.8 us, of four 11).
int split_room(int S);

template <int BN, int S>
cudaError_t launch_tiles_of(const TileParams& p, int smem, cudaStream_t st) {
    static std::atomic<unsigned long long> done;
    const cudaError_t e = allow_smem(linear_tile_kernel<BN, S>, kAllSmem, &done);
    return e != cudaSuccess ? e : launch_clusters(linear_tile_kernel<BN, S>, p, p.tiles * S, kTileThreads, smem, S, st);
}
template <int BN>
cudaError_t launch_tiles(const TileParams& p, int splits, int smem, cudaStream_t st) {
    return splits == 1 ? launch_tiles_of<BN, 1>(p, smem, st) : splits == 2 ? launch_tiles_of<BN, 2>(p, smem, st)
         : splits == 4 ? launch_tiles_of<BN, 4>(p, smem, st) : launch_tiles_of<BN, 8>(p, smem, st);
}
template <int BN, int S>
cudaError_t launch_split_of(const TileParams& p, cudaStream_t st) {
    static std::atomic<unsigned long long> done;
    const cudaError_t e = allow_smem(linear_split_kernel<BN, S>, kAllSmem, &done);
    return e != cudaSuccess ? e : launch_clusters(linear_split_kernel<BN, S>, p, 2ll * (p.tiles + (p.sums.db ? (p.sums.N + 127) / 128 : 0)) * S, kSplitThreads, kAllSmem, 2 * S, st);
}
template <int BN>
cudaError_t launch_split(const TileParams& p, int S, cudaStream_t st) {
    return S == 1 ? launch_split_of<BN, 1>(p, st) : S == 2 ? launch_split_of<BN, 2>(p, st) : S == 3 ? launch_split_of<BN, 3>(p, st) : launch_split_of<BN, 4>(p, st);
}

constexpr int kMaxSplits = 4;
int split_room(int S) {
    static std::atomic<int> known[64][kMaxSplits + 1];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { cudaGetLastError(); dev = 0; }
    int n = known[dev][S].load(std::memory_order_acquire);
    if (n == 0) {
        cudaLaunchConfig_t cfg;
        memset(&cfg, 0, sizeof(cfg));
        cfg.gridDim = dim3((unsigned)(2 * S * 512));
        cfg.blockDim = dim3(kSplitThreads);
        cfg.dynamicSmemBytes = kAllSmem;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)(2 * S);
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        if (cudaFuncSetAttribute(linear_split_kernel<256, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAllSmem) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, linear_split_kernel<256, 2>, &cfg) != cudaSuccess || n <= 0) {
            cudaGetLastError();
            n = 1;
        }
        n = std::min(2 * S * n, sm_count());
        known[dev][S].store(n, std::memory_order_release);
    }
    return n;
}

fp_status launched(cudaError_t e) {
    if (e == cudaSuccess) return FP_OK;
    cudaGetLastError();
    return err(FP_ERR_CUDA, cudaGetErrorString(e));
}

// See kRun.
bool wide(const Product& r) { return r.e.y_type == FP_DTYPE_F32 && r.Kc > (int64_t)kRun * kBlockK; }
int64_t blocks_of(const Product& r) { return (r.Kc + kBlockK - 1) / kBlockK; }
int64_t tiles_of(const Product& r, int bn) { return ((r.I + 255) / 256) * ((r.J + bn - 1) / bn); }

// How linear_split_kernel takes a product that has `share` of the SMs: the tile's width and the pairs that share it by the cycles that they are
// expected to take: the K blocks, the exchange of sums, finishing, and 3000 for everything else; a launch of more CTAs than run at once takes
// as many rounds.  `extra`: clusters of the launch that sum columns.  (The 3000 only weigh a round against longer sums: with 1000 or 9000 twelve
// products from 200 x 300 x 1000 to 2048 x 2048 x 2048 took the same time to 1 %.)
struct SplitChoice { int bn, S; int64_t ctas; bool fits; double cycles; };
SplitChoice split_choice(const Product& r, int64_t share, int64_t extra) {
    const int64_t kblocks = blocks_of(r);
    SplitChoice best = {256, 1, 0, false, 0};
    for (int b = 256; b >= 128; b /= 2)
        for (int c = 1; c <= kMaxSplits && 2 * c <= std::max<int64_t>(kblocks, 2); ++c) {
            const int64_t ctas = 2 * c * (tiles_of(r, b) + extra), room = std::min<int64_t>(share, split_room(c));
            // (a 32-bit result whose runs would be longer than twice kRun: only where there is no other way)
            const double much = wide(r) && (kblocks + c - 1) / c > 2 * kRun * (512 / b) ? 1e6 * (b / 128) / c : 0;
            const double cost = much + (double)((ctas + room - 1) / room) *
                                (3000 + (double)((kblocks + c - 1) / c) * (b == 256 ? 522 : 392) + 32.0 * b * (c - 1) / c + 11.0 * b / c);
            if (best.cycles == 0 || cost < best.cycles) best = {b, c, ctas, ctas <= room, cost};
        }
    return best;
}

// What a K block costs in linear_pair_kernel, in split_choice's measure: as much as there where nothing but the copies into an SM bounds it, a third
// more with 32-bit results (8192 x 4096 x 4096: 249 and 329 us where the rule was fitted, 191-213 and 309-347 on other cards).  It is the ratio that counts: at
// these sizes all SMs copy at once, and a block takes about half a microsecond, twice that many cycles.
double pair_cycles(bool runs) { return runs ? 700 : 522; }

// Whether a call's products go in one launch of linear_pair_kernel, where every pair takes its tiles one after the other, or in one each.  The first
// saves a launch and a last round of idle pairs; two products of unlike sums take long together where a pair has one tile more of the
// longer sum (8192 x 1024 x 1024, 128 tiles of 16 K blocks and 16 of 128: 89 us in one launch, 53 in two).
bool together(const Product* prod, int n) {
    const int64_t pairs = sm_count() / 2, t0 = tiles_of(prod[0], 256), t1 = n > 1 ? tiles_of(prod[1], 256) : 0;
    if (prod[0].swap || t0 + t1 <= pairs) return false;
    if (n < 2) return true;
    int64_t longest = 0;
    for (int64_t p = 0; p < pairs; ++p) {
        const int64_t c0 = t0 > p ? (t0 - p - 1) / pairs + 1 : 0, c = t0 + t1 > p ? (t0 + t1 - p - 1) / pairs + 1 : 0;
        longest = std::max(longest, c0 * blocks_of(prod[0]) + (c - c0) * blocks_of(prod[1]));
    }
    double apart = 0;
    for (int i = 0; i < 2; ++i)
        apart += (i ? t1 : t0) > pairs ? 3000 + pair_cycles(wide(prod[i])) * (((i ? t1 : t0) + pairs - 1) / pairs * blocks_of(prod[i])) : split_choice(prod[i], sm_count(), 0).cycles;
    return 3000 + pair_cycles(wide(prod[0]) || wide(prod[1])) * longest <= apart;
}

// A call's products, one after the other, the second beside the first: the first has its share of the SMs by its work, the second what is
// left, or its share.  (All of them where the first is one of few rows, for linear_tile_kernel, or one takes linear_pair_kernel.)
int64_t share_of(const Product* prod, int n, int i, int64_t used) {
    const int sms = sm_count();
    if (n < 2 || prod[0].swap || tiles_of(prod[0], 256) + tiles_of(prod[1], 256) > sms / 2) return sms;
    const int64_t w0 = tiles_of(prod[0], 256) * blocks_of(prod[0]), w1 = tiles_of(prod[1], 256) * blocks_of(prod[1]);
    return std::max<int64_t>(i ? sms - used : 2, std::max<int64_t>(2, sms * (i ? w1 : w0) / (w0 + w1)));
}

// Whether a call's last product runs in linear_split_kernel with room for `extra` clusters that sum columns: beside the tiles, in one round
// (300 x 2048 x 1000, where they do not fit: 17.8 us with them, 13.3 with a launch in front).  With few rows the first product's CTAs are
// short, and need not leave room (64 x 512 x 512 8.8 -> 6.9 us, 64 x 2048 x 1024 14.0 -> 9.8, 64 x 1000 x 2048 14.0 -> 14.9).
bool room_for_sums(const Product* prod, int n, int64_t extra) {
    if (n == 0 || prod[n - 1].swap || tiles_of(prod[n - 1], 256) + extra > sm_count() / 2 || together(prod, n)) return false;
    const bool beside = n > 1 && !prod[0].swap && tiles_of(prod[0], 256) <= sm_count() / 2;
    const int64_t used = beside ? split_choice(prod[0], share_of(prod, n, 0, 0), 0).ctas : 0;
    const int64_t share = share_of(prod, n, n - 1, used);
    const SplitChoice with = split_choice(prod[n - 1], share, extra);
    // (6000 is a launch's time.  With 0 256 x 1000 x 2048 took 11.9 us instead of 10.4, 1000 x 1000 x 1000 15.8 instead of 13.6, 64 x 512 x 512 7.8 instead of 6.7;
    // with 20000 none of ten sizes changed.)
    return with.fits && with.cycles < split_choice(prod[n - 1], share, 0).cycles + 6000;
}

// The products of a call (two, or one); `late`: their operands were there before the launch in front of them began; `sums`: column sums that the
// last one takes along, or nullptr.
fp_status run_products(const Product* prod, int n, int dtype, int late, const DzParams* sums, int sums_vec, int* status, cudaStream_t st) {
    const int sms = sm_count();
    fp_status s;
    TileParams p;
    memset(&p, 0, sizeof(p));
    p.status = status; p.bf16 = dtype == FP_DTYPE_BF16;
    int64_t used = 0;                                    // CTAs of the first product
    auto pairs = [&](bool runs) -> cudaError_t {
        static std::atomic<unsigned long long> done[2];
        p.run = runs ? kRun : 0;
        cudaError_t e = runs ? allow_smem(linear_pair_kernel<true>, kAllSmem, &done[1]) : allow_smem(linear_pair_kernel<false>, kAllSmem, &done[0]);
        if (e != cudaSuccess) return e;
        return runs ? launch_clusters(linear_pair_kernel<true>, p, 2 * (sms / 2), PairShape<true>::kThreads, kAllSmem, 2, st)
                    : launch_clusters(linear_pair_kernel<false>, p, 2 * (sms / 2), PairShape<false>::kThreads, kAllSmem, 2, st);
    };
    if (together(prod, n)) {
        if ((s = lay_out(prod, n, 256, 256, 128, dtype, &p)) != FP_OK) return s;
        p.late = late;
        return launched(pairs(wide(prod[0]) || (n > 1 && wide(prod[1]))));
    }
    // one after the other, the second beside the first
    for (int i = 0; i < n; ++i) {
        p.late = late || i > 0;
        p.run = wide(prod[i]) ? kRun : 0;
        if (prod[i].swap) {
            const int bn = prod[i].J <= 16 ? 16 : prod[i].J <= 32 ? 32 : prod[i].J <= 64 ? 64 : 128;
            if ((s = lay_out(prod + i, 1, 128, bn, bn, dtype, &p)) != FP_OK) return s;
            const int kblocks = p.prob[0].kblocks;
            int splits = 1;
            const int most = p.run ? std::min(512 / bn, 16) : 1;       // accumulators
            while (splits < 8 && kblocks >= splits * 4 && (p.tiles * splits * 2 <= sms || (p.run && kblocks > 2 * kRun * most * splits))) splits *= 2;
            // (two CTAs on an SM share its 512 columns)
            const int stage = 128 * 128 + bn * 128, room = p.tiles * splits > sms && most * bn <= 256 ? kAllSmem / 2 - 2048 : kAllSmem - 1024;
            p.stages = std::min(std::min(room / stage, 16), (kblocks + splits - 1) / splits);
            const int smem = splits > 1 ? kAllSmem : std::max(p.stages * stage, bn * 132 * 4) + 1024;
            s = launched(bn == 16 ? launch_tiles<16>(p, splits, smem, st) : bn == 32 ? launch_tiles<32>(p, splits, smem, st)
                         : bn == 64 ? launch_tiles<64>(p, splits, smem, st) : launch_tiles<128>(p, splits, smem, st));
        } else if (tiles_of(prod[i], 256) > sms / 2) {
            if ((s = lay_out(prod + i, 1, 256, 256, 128, dtype, &p)) != FP_OK) return s;
            s = launched(pairs(wide(prod[i])));
        } else {
            const int64_t extra = sums && i == n - 1 ? (sums->N + 127) / 128 : 0;
            const SplitChoice c = split_choice(prod[i], share_of(prod, n, i, used), extra);
            if ((s = lay_out(prod + i, 1, 256, c.bn, c.bn / 2, dtype, &p)) != FP_OK) return s;
            used = c.ctas;
            if (extra) { p.sums = *sums; p.sums.splits = 2 * c.S; p.sums_vec = sums_vec; }
            s = launched(c.bn == 256 ? launch_split<256>(p, c.S, st) : launch_split<128>(p, c.S, st));
        }
        if (s != FP_OK) return s;
    }
    return FP_OK;
}

fp_status copy_rows(const CopyJob* jobs, int n, cudaStream_t st) {
    CopyParams p;
    memset(&p, 0, sizeof(p));
    p.job[1].warp0 = 1ll << 62;
    for (int i = 0; i < n; ++i) {
        p.job[i] = jobs[i];
        p.job[i].chunks = (jobs[i].cols + 511) / 512;
        p.job[i].warp0 = p.warps;
        p.warps += p.job[i].rows * p.job[i].chunks;
    }
    if ((p.warps + 7) / 8 > 0x7fffffffll) return err(FP_ERR_BOUNDS, "fp_linear: operand too large");
    return launched(launch_clusters(copy_rows_kernel, p, (p.warps + 7) / 8, 256, 0, 1, st));
}

// Takes an operand into scratch where it cannot be read in place.
const void* place(const void* src, int64_t rows, int64_t cols, int64_t* ld, char** work, CopyJob* jobs, int* n_jobs) {
    if (readable(src, rows, *ld)) return src;
    CopyJob& j = jobs[(*n_jobs)++];
    memset(&j, 0, sizeof(j));
    j.src = static_cast<const uint16_t*>(src);
    j.dst = reinterpret_cast<uint16_t*>(*work);
    j.rows = rows; j.cols = (int)cols; j.ld_src = *ld; j.ld_dst = (cols + 7) / 8 * 8;
    *ld = j.ld_dst;
    *work += packed_bytes(rows, cols);
    return j.dst;
}

bool sizes_ok(int64_t M, int64_t N, int64_t K) { return M >= 0 && N >= 1 && K >= 1; }
bool in_bounds(int64_t M, int64_t N, int64_t K) { return M <= kMaxSize && N <= kMaxSize && K <= kMaxSize; }
// Rows of `cols` elements: the stride must reach over a row and stay within what a tensor map can hold.
bool ld_ok(int64_t ld, int64_t cols, int64_t rows) { return rows <= 1 ? true : ld >= cols && ld <= (1ll << 38); }

fp_status check(const fp_linear_args* a) {
    if (!a) return err(FP_ERR_ARG, "fp_linear_forward: NULL argument");
    if (!sizes_ok(a->M, a->N, a->K)) return err(FP_ERR_ARG, "fp_linear_forward: bad sizes (M >= 0, N and K >= 1)");
    if (!in_bounds(a->M, a->N, a->K)) return err(FP_ERR_BOUNDS, "fp_linear_forward: a size beyond 2^30");
    if (!is_half(a->dtype)) return err(FP_ERR_UNSUPPORTED, "fp_linear_forward: dtype must be FP_DTYPE_BF16 or FP_DTYPE_F16");
    if ((a->y_dtype != a->dtype && a->y_dtype != FP_DTYPE_F32) || (a->d_bias && a->bias_dtype != a->dtype && a->bias_dtype != FP_DTYPE_F32))
        return err(FP_ERR_UNSUPPORTED, "fp_linear_forward: y and bias have dtype, or FP_DTYPE_F32");
    if (a->act < FP_ACT_NONE || a->act > FP_ACT_SILU || (a->res_first != 0 && a->res_first != 1) || a->reserved)
        return err(FP_ERR_ARG, "fp_linear_forward: bad activation, res_first or reserved");
    if (a->M == 0) return FP_OK;
    if (!a->d_x || !a->d_w || !a->d_y) return err(FP_ERR_ARG, "fp_linear_forward: NULL x, w or y");
    if (!ld_ok(a->ld_x, a->K, a->M) || !ld_ok(a->ld_w, a->K, a->N) || !ld_ok(a->ld_y, a->N, a->M) || (a->d_res && !ld_ok(a->ld_res, a->N, a->M)) ||
        (a->d_pre && !ld_ok(a->ld_pre, a->N, a->M)))
        return err(FP_ERR_ARG, "fp_linear_forward: a row stride is shorter than its row");
    const uintptr_t odd = (uintptr_t)a->d_x | (uintptr_t)a->d_w | (uintptr_t)a->d_res | (uintptr_t)a->d_pre;
    if ((odd & 1) || ((uintptr_t)a->d_y & (uintptr_t)(elem_bytes(a->y_dtype) - 1)) || ((uintptr_t)a->d_bias & (uintptr_t)(elem_bytes(a->bias_dtype) - 1)))
        return err(FP_ERR_ARG, "fp_linear_forward: a buffer is not aligned to its elements");
    if (a->d_y == a->d_x || a->d_y == a->d_w || a->d_y == a->d_bias || (a->d_pre && (a->d_pre == a->d_x || a->d_pre == a->d_w || a->d_pre == a->d_y || a->d_pre == a->d_res || a->d_pre == a->d_bias)) ||
        (a->d_res == a->d_y && (a->y_dtype != a->dtype || (a->M > 1 && a->ld_res != a->ld_y))))
        return err(FP_ERR_ARG, "fp_linear_forward: an output is an input (only y may be res, with its type and row stride) or another output");
    return FP_OK;
}

size_t forward_work(const fp_linear_args* a) {
    if (a->M == 0) return 0;
    return (readable(a->d_x, a->M, a->ld_x) ? 0 : packed_bytes(a->M, a->K)) + (readable(a->d_w, a->N, a->ld_w) ? 0 : packed_bytes(a->N, a->K));
}

fp_status check(const fp_linear_grad_args* a) {
    if (!a) return err(FP_ERR_ARG, "fp_linear_backward: NULL argument");
    if (!sizes_ok(a->M, a->N, a->K)) return err(FP_ERR_ARG, "fp_linear_backward: bad sizes (M >= 0, N and K >= 1)");
    if (!in_bounds(a->M, a->N, a->K)) return err(FP_ERR_BOUNDS, "fp_linear_backward: a size beyond 2^30");
    if (!is_half(a->dtype) || (a->dw_dtype != a->dtype && a->dw_dtype != FP_DTYPE_F32))
        return err(FP_ERR_UNSUPPORTED, "fp_linear_backward: dtype must be FP_DTYPE_BF16 or FP_DTYPE_F16, dw_dtype the same or FP_DTYPE_F32");
    if (a->act < FP_ACT_NONE || a->act > FP_ACT_SILU || (a->accumulate != 0 && a->accumulate != 1))
        return err(FP_ERR_ARG, "fp_linear_backward: bad activation or accumulate");
    if (!a->d_dw && !a->d_db && !(a->M == 0 || a->d_dx || a->d_dz)) return err(FP_ERR_ARG, "fp_linear_backward: no output is asked for");
    if (a->d_dw && !ld_ok(a->ld_dw, a->K, a->N)) return err(FP_ERR_ARG, "fp_linear_backward: a row stride is shorter than its row");
    const uintptr_t outs = (uintptr_t)a->d_dw | (uintptr_t)a->d_db;
    if (outs & (uintptr_t)(elem_bytes(a->dw_dtype) - 1)) return err(FP_ERR_ARG, "fp_linear_backward: a buffer is not aligned to its elements");
    if (a->M == 0) return FP_OK;
    if (!a->d_dy || (a->act != FP_ACT_NONE && !a->d_pre) || (a->d_dw && !a->d_x) || (a->d_dx && !a->d_w))
        return err(FP_ERR_ARG, "fp_linear_backward: NULL dy, pre (with an activation), x (for dw) or w (for dx)");
    if (!ld_ok(a->ld_dy, a->N, a->M) || (a->act != FP_ACT_NONE && !ld_ok(a->ld_pre, a->N, a->M)) || (a->d_dw && !ld_ok(a->ld_x, a->K, a->M)) ||
        (a->d_dx && (!ld_ok(a->ld_w, a->K, a->N) || !ld_ok(a->ld_dx, a->K, a->M))) || (a->d_dz && !ld_ok(a->ld_dz, a->N, a->M)))
        return err(FP_ERR_ARG, "fp_linear_backward: a row stride is shorter than its row");
    if (a->d_dz == a->d_dy && a->M > 1 && a->ld_dz != a->ld_dy) return err(FP_ERR_ARG, "fp_linear_backward: dz in dy's place needs dy's row stride");
    const uintptr_t odd = (uintptr_t)a->d_dy | (uintptr_t)a->d_pre | (uintptr_t)a->d_x | (uintptr_t)a->d_w | (uintptr_t)a->d_dx | (uintptr_t)a->d_dz;
    if (odd & 1) return err(FP_ERR_ARG, "fp_linear_backward: a buffer is not aligned to its elements");
    // (dz may be dy, and nothing else that is written anything else)
    const void* outs_of[4] = {a->d_dx, a->d_dw, a->d_db, a->d_dz};
    for (int i = 0; i < 4; ++i) {
        const void* o = outs_of[i];
        if (!o) continue;
        bool again = (o == a->d_dy && i != 3) || (a->act != FP_ACT_NONE && o == a->d_pre) || (a->d_dw && o == a->d_x) || (a->d_dx && o == a->d_w);
        for (int j = 0; j < i; ++j) again = again || o == outs_of[j];
        if (again) return err(FP_ERR_ARG, "fp_linear_backward: an output is an input (only dz may be dy) or another output");
    }
    return FP_OK;
}

// Where the products read dz: in d_dz, or without an activation in d_dy, if those can be read in place, or else in scratch.
enum DzPlace { kDzNowhere, kDzOut, kDzIn, kDzWork };
DzPlace dz_place(const fp_linear_grad_args* a) {
    if (!a->d_dx && !a->d_dw) return kDzNowhere;
    if (a->d_dz && readable(a->d_dz, a->M, a->ld_dz)) return kDzOut;
    return a->act == FP_ACT_NONE && readable(a->d_dy, a->M, a->ld_dy) ? kDzIn : kDzWork;
}
size_t backward_work(const fp_linear_grad_args* a) {
    if (a->M == 0) return 0;
    return (dz_place(a) == kDzWork ? packed_bytes(a->M, a->N) : 0) + (a->d_dw && !readable(a->d_x, a->M, a->ld_x) ? packed_bytes(a->M, a->K) : 0) +
           (a->d_dx && !readable(a->d_w, a->N, a->ld_w) ? packed_bytes(a->N, a->K) : 0);
}
// (Inputs are copied into scratch, and dz is written there, before anything else is read or written.)
fp_status check_work_apart(const void* work, size_t need, const void* const* others, int n) {
    for (int i = 0; i < n && need && work; ++i)
        if (work == others[i]) return err(FP_ERR_ARG, "fp_linear: the scratch is another buffer of the call");
    return FP_OK;
}
fp_status check_work(const void* work, size_t have, size_t need, Buffers& buf) {
    if (need == 0) return FP_OK;
    if (!work || have < need) return err(FP_ERR_BOUNDS, "fp_linear: the scratch is smaller than the workspace call says");
    if ((uintptr_t)work & 255) return err(FP_ERR_ARG, "fp_linear: the scratch is not aligned to 256 bytes");
    return buf.here(work) ? FP_OK : err(FP_ERR_ARG, "fp_linear: the scratch is not memory of the current device");
}

}  // namespace
}  // namespace fp

using namespace fp;
using namespace fp::train;

extern "C" fp_status fp_linear_workspace(const fp_linear_args* a, size_t* bytes) {
    if (!bytes) return err(FP_ERR_ARG, "fp_linear_workspace: NULL argument");
    const fp_status s = check(a);
    if (s == FP_OK) *bytes = forward_work(a);
    return s;
}

extern "C" fp_status fp_linear_backward_workspace(const fp_linear_grad_args* a, size_t* bytes) {
    if (!bytes) return err(FP_ERR_ARG, "fp_linear_backward_workspace: NULL argument");
    const fp_status s = check(a);
    if (s == FP_OK) *bytes = backward_work(a);
    return s;
}

extern "C" fp_status fp_linear_forward(const fp_linear_args* a, void* work, size_t work_bytes, void* stream) {
    fp_status s = check(a);
    if (s != FP_OK || a->M == 0) return s;
    const void* others[6] = {a->d_x, a->d_w, a->d_bias, a->d_res, a->d_y, a->d_pre};
    if ((s = check_work_apart(work, forward_work(a), others, 6)) != FP_OK) return s;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return err(FP_ERR_CUDA, "fp_linear_forward: no current device"); }
    Buffers buf(dev);
    if (!buf.here(a->d_x) || !buf.here(a->d_w) || !buf.here(a->d_y) || !buf.here_or_null(a->d_bias) ||
        !buf.here_or_null(a->d_res) || !buf.here_or_null(a->d_pre))
        return err(FP_ERR_ARG, "fp_linear_forward: a buffer is not memory of the current device");
    if ((s = check_work(work, work_bytes, forward_work(a), buf)) != FP_OK) return s;
    int* status = status_word(dev);
    if (!status) return err(FP_ERR_CUDA, "fp_linear_forward: no status word on this device");
    const cudaStream_t st = (cudaStream_t)stream;
    char* w = static_cast<char*>(work);
    CopyJob jobs[2];
    int n_jobs = 0;
    int64_t ld_x = a->ld_x, ld_w = a->ld_w;
    const void* x = place(a->d_x, a->M, a->K, &ld_x, &w, jobs, &n_jobs);
    const void* wt = place(a->d_w, a->N, a->K, &ld_w, &w, jobs, &n_jobs);
    if (n_jobs && (s = copy_rows(jobs, n_jobs, st)) != FP_OK) return s;
    Product p;
    memset(&p, 0, sizeof(p));
    const Operand ox = {x, a->M, a->K, ld_x, 0}, ow = {wt, a->N, a->K, ld_w, 0};
    p.swap = a->M <= 128;
    p.a = p.swap ? ow : ox; p.b = p.swap ? ox : ow;
    p.I = p.swap ? a->N : a->M; p.J = p.swap ? a->M : a->N; p.Kc = a->K;
    Epilogue& e = p.e;
    e.y = a->d_y; e.pre = a->d_pre; e.res = a->d_res; e.bias = a->d_bias;
    e.ld_y = a->ld_y; e.ld_pre = a->ld_pre; e.ld_res = a->ld_res;
    e.y_type = a->y_dtype; e.pre_type = e.res_type = a->dtype; e.bias_type = a->bias_dtype; e.act = a->act; e.res_first = a->res_first;
    e.vec = aligned4(a->d_y, a->ld_y, a->y_dtype, a->M) && (!a->d_pre || aligned4(a->d_pre, a->ld_pre, a->dtype, a->M)) &&
            (!a->d_res || aligned4(a->d_res, a->ld_res, a->dtype, a->M));
    return run_products(&p, 1, a->dtype, 0, nullptr, 0, status, st);
}

extern "C" fp_status fp_linear_backward(const fp_linear_grad_args* a, void* work, size_t work_bytes, void* stream) {
    fp_status s = check(a);
    if (s != FP_OK) return s;
    const void* others[8] = {a->d_dy, a->act != FP_ACT_NONE ? a->d_pre : nullptr, a->d_dw ? a->d_x : nullptr, a->d_dx ? a->d_w : nullptr,      // (what is not read may be anything)
                             a->d_dx, a->d_dw, a->d_db, a->d_dz};
    if ((s = check_work_apart(work, backward_work(a), others, 8)) != FP_OK) return s;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return err(FP_ERR_CUDA, "fp_linear_backward: no current device"); }
    Buffers buf(dev);
    if (!buf.here_or_null(a->d_dw) || !buf.here_or_null(a->d_db) ||
        (a->M > 0 && (!buf.here(a->d_dy) || (a->act != FP_ACT_NONE && !buf.here(a->d_pre)) || (a->d_dw && !buf.here(a->d_x)) ||
                      (a->d_dx && !buf.here(a->d_w)) || !buf.here_or_null(a->d_dx) || !buf.here_or_null(a->d_dz))))
        return err(FP_ERR_ARG, "fp_linear_backward: a buffer is not memory of the current device");
    const cudaStream_t st = (cudaStream_t)stream;
    const int dw_bytes = elem_bytes(a->dw_dtype);
    if (a->M == 0) {                                     // empty sums
        cudaError_t e = cudaSuccess;
        if (!a->accumulate && a->d_dw)
            e = cudaMemset2DAsync(a->d_dw, (size_t)std::max(a->N > 1 ? a->ld_dw : 0, a->K) * dw_bytes, 0, (size_t)a->K * dw_bytes, (size_t)a->N, st);
        if (e == cudaSuccess && !a->accumulate && a->d_db) e = cudaMemsetAsync(a->d_db, 0, (size_t)a->N * dw_bytes, st);
        if (e != cudaSuccess) { cudaGetLastError(); return err(FP_ERR_CUDA, cudaGetErrorString(e)); }
        return FP_OK;
    }
    if ((s = check_work(work, work_bytes, backward_work(a), buf)) != FP_OK) return s;
    int* status = status_word(dev);
    if (!status) return err(FP_ERR_CUDA, "fp_linear_backward: no status word on this device");
    char* w = static_cast<char*>(work);
    // dz: where the products read it, and what has to be written for that
    const void* dz = a->d_dy;
    int64_t ld_dz = a->ld_dy;
    DzParams d;
    memset(&d, 0, sizeof(d));
    const DzPlace at = dz_place(a);
    if (a->d_dz) { d.out[0] = static_cast<uint16_t*>(a->d_dz); d.ld_out[0] = a->ld_dz; }
    if (at == kDzOut) { dz = a->d_dz; ld_dz = a->ld_dz; }
    if (at == kDzWork) {
        d.out[1] = reinterpret_cast<uint16_t*>(w);
        d.ld_out[1] = (a->N + 7) / 8 * 8;
        w += packed_bytes(a->M, a->N);
        dz = d.out[1]; ld_dz = d.ld_out[1];
    }
    CopyJob jobs[2];
    int n_jobs = 0, n = 0;
    int64_t ld_x = a->ld_x, ld_w = a->ld_w;
    const void* x = a->d_dw ? place(a->d_x, a->M, a->K, &ld_x, &w, jobs, &n_jobs) : nullptr;
    const void* wt = a->d_dx ? place(a->d_w, a->N, a->K, &ld_w, &w, jobs, &n_jobs) : nullptr;
    Product p[2];
    memset(p, 0, sizeof(p));
    if (a->d_dx) {
        Product& r = p[n++];
        const Operand odz = {dz, a->M, a->N, ld_dz, 0}, ow = {wt, a->N, a->K, ld_w, 1};
        r.swap = a->M <= 128;
        r.a = r.swap ? ow : odz; r.b = r.swap ? odz : ow;
        r.I = r.swap ? a->K : a->M; r.J = r.swap ? a->M : a->K; r.Kc = a->N;
        r.e.y = a->d_dx; r.e.ld_y = a->ld_dx; r.e.y_type = a->dtype;
        r.e.vec = aligned4(a->d_dx, a->ld_dx, a->dtype, a->M);
    }
    if (a->d_dw) {
        Product& r = p[n++];
        r.swap = 0;
        r.a = {dz, a->M, a->N, ld_dz, 1}; r.b = {x, a->M, a->K, ld_x, 1};
        r.I = a->N; r.J = a->K; r.Kc = a->M;
        r.e.y = a->d_dw; r.e.ld_y = a->ld_dw; r.e.y_type = a->dw_dtype;
        if (a->accumulate) { r.e.res = a->d_dw; r.e.ld_res = a->ld_dw; r.e.res_type = a->dw_dtype; }
        r.e.vec = aligned4(a->d_dw, a->ld_dw, a->dw_dtype, a->N);
    }
    const bool writes = d.out[0] || d.out[1];
    int along = 0, vec = 0;                              // whether the last product's launch sums dy's columns too (256 x 1000 x 2048: 12.7 -> 10.7 us)
    if (writes || a->d_db) {
        d.dy = static_cast<const uint16_t*>(a->d_dy); d.pre = static_cast<const uint16_t*>(a->d_pre); d.db = a->d_db;
        d.ld_dy = a->ld_dy; d.ld_pre = a->ld_pre; d.M = a->M; d.N = (int)a->N; d.act = a->act; d.dtype = a->dtype; d.db_type = a->dw_dtype;
        d.accumulate = a->accumulate;
        vec = (a->N & 7) == 0 && readable(a->d_dy, a->M, a->ld_dy) && (a->act == FP_ACT_NONE || readable(a->d_pre, a->M, a->ld_pre)) &&
              (!a->d_dz || readable(a->d_dz, a->M, a->ld_dz));
        along = !writes && a->act == FP_ACT_NONE && room_for_sums(p, n, (a->N + 127) / 128);
    }
    if (writes || (a->d_db && !along)) {
        const int64_t blocks = (a->N + 127) / 128;
        d.splits = 1;
        while (d.splits < 8 && a->M > 32 * d.splits && blocks * d.splits < 8 * sm_count()) d.splits *= 2;
        // fewer CTAs than SMs, and many rows: they are large (4637 x 15 unaligned 37 -> 13-19 us, 32768 x 1024 with gelu 164 -> 68-85 with dz and db)
        const bool narrow = blocks * d.splits <= sm_count() && a->M > 64 * d.splits;
        const DzKernel k = a->dtype == FP_DTYPE_BF16 ? dz_kernel<FP_DTYPE_BF16>(a->act, vec, narrow) : dz_kernel<FP_DTYPE_F16>(a->act, vec, narrow);
        if ((s = launched(launch_clusters(k, d, blocks * d.splits, narrow ? 1024 : 256, 0, d.splits, st))) != FP_OK) return s;
    }
    if (n_jobs && (s = copy_rows(jobs, n_jobs, st)) != FP_OK) return s;
    if (!n) return FP_OK;
    // Where the launch in front of the products only sums dz's columns, they need not wait for it.
    const int late = a->d_db && !writes && !along && !n_jobs;
    return run_products(p, n, a->dtype, late, along ? &d : nullptr, vec, status, st);
}

extern "C" fp_status fp_linear_status(int32_t* out) {
    if (!out) return err(FP_ERR_ARG, "fp_linear_status: NULL argument");
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return err(FP_ERR_CUDA, "fp_linear_status: no current device"); }
    int* word = status_word(dev);
    int v = 0;
    if (!word || cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&v, word, sizeof(v), cudaMemcpyDeviceToHost) != cudaSuccess ||
        (v && cudaMemset(word, 0, sizeof(v)) != cudaSuccess)) {
        cudaGetLastError();
        return err(FP_ERR_CUDA, "fp_linear_status: the status word cannot be read");
    }
    *out = v ? FP_ERR_TIMEOUT : FP_OK;
    return FP_OK;
}
