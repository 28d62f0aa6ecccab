// Gradient of the softmax cross-entropy of an fp32 layer's outputs, dX = f D W, dW = f D^T X with D and f as in ce_grad.hip, everything in fp32 and the products on
// the fp64 matrix cores (gemm_f32.hip: both operands with the contracted dimension side by side, hence the transposed copies).  The three products of a piece of the
// outputs are what it costs: 1000 x 1024 -> 8000 in 940 us, of which the products 870 (57 TFLOP/s, where a large fp64 product reaches 67).
#include <algorithm>

#include "agzo_internal.h"

namespace agzo {

namespace {

// *scale = g / max(count, 1), count of the rows whose id is an output; one workgroup
__global__ __launch_bounds__(256) void ce32_scale_kernel(const int32_t* __restrict__ ids, int64_t M, int64_t V, const double* __restrict__ g, double* __restrict__ scale) {
    __shared__ int red[4];
    int n = 0;
    for (int64_t t = threadIdx.x; t < M; t += 256) n += ids[t] >= 0 && ids[t] < V;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
    __syncthreads();
    if (threadIdx.x == 0) *scale = (g ? *g : 1.0) / (double)max(red[0] + red[1] + red[2] + red[3], 1);
}

// 32 x 32 tiles of y [C][R] = x^T of x [R][ldx]; with ids, rows that are not counted as zeros (D is 0 there, and a value that is not finite would make NaNs of it)
__global__ __launch_bounds__(256) void ce32_flip_kernel(const float* __restrict__ x, int64_t ldx, int64_t R, int64_t C, float* __restrict__ y, const int32_t* __restrict__ ids, int64_t V) {
    __shared__ float tile[32][33];
    const int64_t down = (R + 31) / 32, r0 = blockIdx.x % down * 32, c0 = blockIdx.x / down * 32;
    const int j = threadIdx.x & 31;
    for (int i = threadIdx.x >> 5; i < 32; i += 8) {
        const bool there = r0 + i < R && c0 + j < C;
        tile[i][j] = there && (!ids || (ids[r0 + i] >= 0 && ids[r0 + i] < V)) ? x[(r0 + i) * ldx + c0 + j] : 0.f;
    }
    __syncthreads();
    for (int i = threadIdx.x >> 5; i < 32; i += 8)
        if (c0 + i < C && r0 + j < R) y[(c0 + i) * R + r0 + j] = tile[j][i];
}

// z [M][n], a piece's logits, the first of them output v0, becomes D, and dt [n][M] D^T
__global__ __launch_bounds__(256) void ce32_d_kernel(float* __restrict__ z, int64_t M, int64_t v0, int64_t n, int64_t V, const int32_t* __restrict__ ids, const float* __restrict__ lse,
                                                     float* __restrict__ dt) {
    __shared__ float tile[32][33];
    const int64_t across = (n + 31) / 32, c0 = blockIdx.x % across * 32, r0 = blockIdx.x / across * 32;
    const int j = threadIdx.x & 31;
    for (int i = threadIdx.x >> 5; i < 32; i += 8) {
        if (r0 + i >= M || c0 + j >= n) continue;
        const int64_t id = ids[r0 + i];
        float* at = z + (r0 + i) * n + c0 + j;
        const float p = expf(*at - lse[r0 + i]), d = id < 0 || id >= V ? 0.f : v0 + c0 + j == id ? p - 1.f : p;
        *at = tile[i][j] = d;
    }
    __syncthreads();
    for (int i = threadIdx.x >> 5; i < 32; i += 8)
        if (c0 + i < n && r0 + j < M) dt[(c0 + i) * M + r0 + j] = tile[j][i];
}

__global__ __launch_bounds__(256) void ce32_add_kernel(const float* __restrict__ part, float* __restrict__ sum, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) sum[i] += part[i];
}

// out [rows][ldo] = *scale in [rows][ldi]; in may be out
__global__ __launch_bounds__(256) void ce32_out_kernel(const float* in, int64_t ldi, int64_t rows, int64_t d, const double* __restrict__ scale, float* out, int64_t ldo) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * d; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / d, c = i - row * d;
        out[row * ldo + c] = (float)(*scale * (double)in[row * ldi + c]);
    }
}

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

struct Ce32Layout {
    int64_t piece;
    size_t scale, z, dt, xt, wt, sum, part, total;
};
Ce32Layout ce32_layout(int64_t M, int64_t V, int64_t d, bool want_dx, bool want_dw) {
    Ce32Layout l;
    // (64 million values of D: 256 MB)
    const int64_t most = std::max<int64_t>(256, (1LL << 26) / std::max(M, d));
    l.piece = (V + (V + most - 1) / most - 1) / ((V + most - 1) / most);
    size_t o = 0;
    auto take = [&](size_t values) { const size_t at = o; o += up256(values * 4); return at; };
    l.scale = take(2);
    l.z = take((size_t)M * l.piece);
    l.dt = take((size_t)l.piece * M);
    l.xt = take(want_dw ? (size_t)d * M : 0);
    l.wt = take(want_dx ? (size_t)d * l.piece : 0);
    l.sum = take(want_dx ? (size_t)M * d : 0);
    l.part = take(want_dx && l.piece < V ? (size_t)M * d : 0);
    l.total = o;
    return l;
}

hipError_t flip(const float* x, int64_t ldx, int64_t R, int64_t C, float* y, const int32_t* ids, int64_t V, hipStream_t st) {
    hipLaunchKernelGGL(ce32_flip_kernel, dim3((unsigned)((R + 31) / 32 * ((C + 31) / 32))), dim3(256), 0, st, x, ldx, R, C, y, ids, V);
    return hipGetLastError();
}
hipError_t product(const float* x, int64_t ldx, const float* w, int64_t ldw, int64_t M, int64_t N, int64_t K, float* y, int64_t ldy, hipStream_t st) {
    F32FwdArgs a{};
    a.X = x; a.ldx = ldx; a.W = w; a.ldw = ldw; a.M = M; a.N = N; a.K = K; a.Y = y; a.ldy = ldy; a.r = 1;
    return launch_forward_f32_many(&a, 1, st);
}
// workgroups for so many values.  (A launch of 2^32 threads and more is cut off without a word: from 2^31 values on they go round)
unsigned ce32_blocks(int64_t values) { return (unsigned)std::min<int64_t>((values + 255) / 256, 1 << 23); }
hipError_t store(const float* in, int64_t ldi, int64_t rows, int64_t d, const double* scale, float* out, int64_t ldo, hipStream_t st) {
    hipLaunchKernelGGL(ce32_out_kernel, dim3(ce32_blocks(rows * d)), dim3(256), 0, st, in, ldi, rows, d, scale, out, ldo);
    return hipGetLastError();
}

}  // namespace

size_t ce_grad_f32_workspace_bytes(int64_t M, int64_t V, int64_t d, bool want_dx, bool want_dw) { return ce32_layout(M, V, d, want_dx, want_dw).total; }

hipError_t launch_ce_grad_f32(const CeGradF32Args& a, void* workspace, hipStream_t st) {
    const Ce32Layout l = ce32_layout(a.M, a.V, a.d, a.dX != nullptr, a.dW != nullptr);
    char* ws = static_cast<char*>(workspace);
    auto at = [&](size_t off) { return reinterpret_cast<float*>(ws + off); };
    double* scale = reinterpret_cast<double*>(ws + l.scale);
    float *z = at(l.z), *dt = at(l.dt), *xt = at(l.xt), *wt = at(l.wt), *sum = at(l.sum), *part = at(l.part);
#define CE_TRY(expr)                            \
    do {                                        \
        const hipError_t e__ = (expr);          \
        if (e__ != hipSuccess) return e__;      \
    } while (0)
    hipLaunchKernelGGL(ce32_scale_kernel, dim3(1), dim3(256), 0, st, a.ids, a.M, a.V, a.g, scale);
    CE_TRY(hipGetLastError());
    if (a.dW) CE_TRY(flip(a.X, a.ldx, a.M, a.d, xt, a.ids, a.V, st));
    for (int64_t v0 = 0; v0 < a.V; v0 += l.piece) {
        const int64_t n = std::min(l.piece, a.V - v0);
        const float* W = a.W + v0 * a.ldw;
        CE_TRY(product(a.X, a.ldx, W, a.ldw, a.M, n, a.d, z, n, st));
        hipLaunchKernelGGL(ce32_d_kernel, dim3((unsigned)((n + 31) / 32 * ((a.M + 31) / 32))), dim3(256), 0, st, z, a.M, v0, n, a.V, a.ids, a.lse, dt);
        CE_TRY(hipGetLastError());
        if (a.dW) {
            float* dW = a.dW + v0 * a.lddw;
            CE_TRY(product(dt, a.M, xt, a.M, n, a.d, a.M, dW, a.lddw, st));
            CE_TRY(store(dW, a.lddw, n, a.d, scale, dW, a.lddw, st));
        }
        if (!a.dX) continue;
        CE_TRY(flip(W, a.ldw, n, a.d, wt, nullptr, 0, st));
        CE_TRY(product(z, n, wt, n, a.M, a.d, n, v0 ? part : sum, a.d, st));
        if (v0) {
            hipLaunchKernelGGL(ce32_add_kernel, dim3(ce32_blocks(a.M * a.d)), dim3(256), 0, st, part, sum, a.M * a.d);
            CE_TRY(hipGetLastError());
        }
    }
#undef CE_TRY
    return a.dX ? store(sum, a.d, a.M, a.d, scale, a.dX, a.lddx, st) : hipSuccess;
}

}  // namespace agzo
