// Gradient of the softmax cross-entropy of a layer's outputs Y = X W^T [M][V], whose mean over the counted rows is the loss of loss.hip:
//     D_tv = exp(y_tv - lse_t) - [v = id_t]   (0 in rows that are not counted),     dX = f D W,     dW = f D^T X,     f = g / count.
// The logits are made once more, for a piece of the outputs at a time, and only D of that piece is stored, as bf16, in both orders
// (without f, whose rounding all of its values would share: with it in D the gradients of 8192 tokens of 131072 outputs were off by 0.0032 of their norm): the
// products contract over outputs and over tokens, and the forward's kernels want the contracted dimension side by side.  So W's piece and X are
// transposed too.  The products are those of gemm_bf16_aligned.hip where a 256 x 256 tile fits: D leaves the logits' product in both orders, and dX is
// summed over the pieces in fp32, in shares of a piece where its tiles alone would not fill the chip.  Other shapes go through fp32 logits and
// the forward's kernels, their dX and all of the gradient of few tokens through those of ce_few.hip, which copy nothing transposed.
// This file: everything around the products.
#include "gemm_bf16_common.h"

namespace agzo {

namespace {

// What a piece's products need, in one launch (by itself each of these is a launch of some 5 us and next to no work): its blocks are
//   one, for the first piece: *scale = g / max(count, 1), count of the rows whose id is an output; rowf: 1 for these, 0 for the others
//   tiles of 64 x 64 of y [C][ldy] = x^T of x [R][ldx], for X (first piece) and for the piece of W; columns R .. ldy of y are zeros (rows C and on are not written), and
//     with ids those of the rows that are not counted: D is 0 there, and a value that is not finite would make NaNs of it
//   256 values each of the columns from .. to of rows of ld values <- 0, for D and D^T, whose products end before them
struct CeFlip { const bf16_t* x; int64_t ldx, R, C; bf16_t* y; int64_t ldy; int64_t blocks; };
struct CeZero { bf16_t* y; int64_t rows, ld, from, to; int64_t blocks; };
struct CePrepare {
    const int32_t* ids; int64_t M, V; const double* g; float *rowf, *scale; int64_t count_blocks;
    CeFlip X, W;
    CeZero D, Dt;
};
__device__ __forceinline__ void ce_count(const CePrepare& a) {
    __shared__ int red[4];
    int n = 0;
    for (int64_t t0 = threadIdx.x; t0 < a.M; t0 += 256 * 8) {
        int32_t id[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) id[u] = a.ids[min(t0 + 256 * u, a.M - 1)];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (t0 + 256 * u < a.M) {
                const bool counted = id[u] >= 0 && id[u] < a.V;
                n += counted;
                a.rowf[t0 + 256 * u] = counted ? 1.f : 0.f;
            }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
    __syncthreads();
    if (threadIdx.x == 0) *a.scale = (float)((a.g ? *a.g : 1.0) / (double)max(red[0] + red[1] + red[2] + red[3], 1));
}
__device__ __forceinline__ void ce_flip(const CeFlip& a, const int32_t* ids, int64_t V, int64_t block) {
    __shared__ bf16_t tile[64][66];
    const int64_t across = (a.ldy + 63) / 64, r0 = block % across * 64, c0 = block / across * 64;
    const int t = threadIdx.x;
    for (int i = t; i < 64 * 8; i += 256) {
        const int r = i >> 3, c = (i & 7) * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        const bool counted = !ids || (r0 + r < a.R && ids[r0 + r] >= 0 && ids[r0 + r] < V);
        if (counted && r0 + r < a.R && c0 + c < a.C) v = *reinterpret_cast<const uint4*>(a.x + (r0 + r) * a.ldx + c0 + c);      // (C is a multiple of 8)
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) *reinterpret_cast<uint32_t*>(&tile[r][c + 2 * k]) = w[k];
    }
    __syncthreads();
    for (int i = t; i < 64 * 8; i += 256) {
        const int c = i >> 3, r = (i & 7) * 8;
        if (c0 + c >= a.C || r0 + r >= a.ldy) continue;
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = (uint32_t)tile[r + 2 * k][c] | (uint32_t)tile[r + 2 * k + 1][c] << 16;
        *reinterpret_cast<uint4*>(a.y + (c0 + c) * a.ldy + r0 + r) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
__device__ __forceinline__ void ce_zero(const CeZero& a, int64_t block) {
    const int64_t i = block * 256 + threadIdx.x, w = a.to - a.from;
    if (i >= a.rows * w) return;
    const int64_t row = i / w;
    a.y[row * a.ld + a.from + (i - row * w)] = 0;
}
__global__ __launch_bounds__(256) void ce_prepare_kernel(const CePrepare a) {
    int64_t b = blockIdx.x;
    if (b < a.count_blocks) return ce_count(a);
    b -= a.count_blocks;
    if (b < a.X.blocks) return ce_flip(a.X, a.ids, a.V, b);
    b -= a.X.blocks;
    if (b < a.W.blocks) return ce_flip(a.W, nullptr, 0, b);
    b -= a.W.blocks;
    if (b < a.D.blocks) return ce_zero(a.D, b);
    ce_zero(a.Dt, b - a.D.blocks);
}

// D and D^T of a piece, from its logits z [M][ldz]: outputs v0 .. v0 + n; D [M][ldd] zero from column n on, D^T [n][ldt] zero from column M on
__global__ __launch_bounds__(256) void ce_softmax_grad_kernel(const float* __restrict__ z, int64_t ldz, int64_t M, int64_t v0, int64_t n,
                                                              const int32_t* __restrict__ ids, const float* __restrict__ lse, const float* __restrict__ rowf,
                                                              bf16_t* __restrict__ d, int64_t ldd, bf16_t* __restrict__ dt, int64_t ldt) {
    __shared__ bf16_t tile[64][66];
    const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
    const int t = threadIdx.x;
    for (int i = t; i < 64 * 32; i += 256) {
        const int r = i >> 5, c = (i & 31) * 2;
        const int64_t row = r0 + r;
        float v[2] = {0.f, 0.f};
        if (row < M && rowf[row] != 0.f) {
            const float l = lse[row];
            const int id = ids[row];
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (c0 + c + u < n) {
                    const float p = __builtin_amdgcn_exp2f((z[row * ldz + c0 + c + u] - l) * 1.44269504088896341f);
                    v[u] = v0 + c0 + c + u == id ? p - 1.f : p;
                }
        }
        const uint32_t w = pack_bf16x2(v[0], v[1]);
        *reinterpret_cast<uint32_t*>(&tile[r][c]) = w;
        if (row < M && c0 + c < ldd) *reinterpret_cast<uint32_t*>(d + row * ldd + c0 + c) = w;
    }
    __syncthreads();
    for (int i = t; i < 64 * 8; i += 256) {
        const int c = i >> 3, r = (i & 7) * 8;
        if (c0 + c >= n || r0 + r >= ldt) continue;
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = (uint32_t)tile[r + 2 * k][c] | (uint32_t)tile[r + 2 * k + 1][c] << 16;
        *reinterpret_cast<uint4*>(dt + (c0 + c) * ldt + r0 + r) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// dX or dW: the shares' sums [shares][M][d] added in order, times *scale, as bf16
__global__ __launch_bounds__(256) void ce_join_kernel(const float* __restrict__ sums, int shares, int64_t M, int64_t d, const float* __restrict__ scale, bf16_t* __restrict__ out, int64_t ldo) {
    for (int64_t i = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * 4; i < M * d; i += (int64_t)gridDim.x * blockDim.x * 4) {
        float4 s = *reinterpret_cast<const float4*>(sums + i);
        for (int k = 1; k < shares; k += 8) {
            float4 o[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) o[u] = *reinterpret_cast<const float4*>(sums + min(k + u, shares - 1) * M * d + i);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (k + u < shares) { s.x += o[u].x; s.y += o[u].y; s.z += o[u].z; s.w += o[u].w; }
        }
        const int64_t row = i / d;
        const float f = *scale;
        *reinterpret_cast<uint2*>(out + row * ldo + (i - row * d)) = make_uint2(pack_bf16x2(s.x * f, s.y * f), pack_bf16x2(s.z * f, s.w * f));
    }
}
hipError_t join(const float* sums, int shares, int64_t M, int64_t d, const float* scale, bf16_t* out, int64_t ldo, hipStream_t st) {
    const int wide = M * d <= 1 << 18 ? 64 : 256;      // (few values: a wave a workgroup, for the sake of their number)
    // (a launch of 2^32 threads and more is cut off without a word: from 2^33 values on workgroups go round)
    const int64_t blocks = std::min<int64_t>((M * d / 4 + wide - 1) / wide, 1 << 23);
    hipLaunchKernelGGL(ce_join_kernel, dim3((unsigned)blocks), dim3(wide), 0, st, sums, shares, M, d, scale, out, ldo);
    return hipGetLastError();
}

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int64_t up64(int64_t x) { return (x + 63) / 64 * 64; }

// Outputs of a piece: some 2^27 values of D (and of W transposed), which is 256 MB each, and pieces of about the same size
int64_t ce_piece(int64_t M, int64_t V, int64_t d) {
    const int64_t most = std::max<int64_t>(1024, (1LL << 27) / std::max(M, d) / 256 * 256);
    const int64_t pieces = (V + most - 1) / most;
    return ((V + pieces - 1) / pieces + 255) / 256 * 256;
}

struct CeLayout {
    int64_t piece, width, kt;       // outputs of a piece; outputs and tokens as far as zeros go
    bool few;                       // the kernels of ce_few.hip, all outputs at once
    bool few_w;                     // and for dW
    bool tiles_z, tiles_x;          // 256 x 256 tiles fit the logits of a piece, the sums of dX
    int shares, shares_w;           // of dX's outputs, of dW's tokens
    size_t rowf, scale, z, d, dt, wt, xt, sum, wsum, total;
};
// D's columns of n outputs (D^T's of n tokens): their shares' slices
int64_t ce_width(int64_t n, int shares) { return shares == 1 ? std::max<int64_t>(up64(n), 2 * BK) : std::max<int64_t>((up64(n) / 64 + shares - 1) / shares, 2) * 64 * shares; }

// whether the tiles store dW themselves, of n outputs; else it goes through fp32 sums, which shares of the tokens or a kernel for any shape leave
bool ce_dw_stored(const CeLayout& l, int64_t n, int64_t d) { return gemm_bf16_grad_fits(n, d, l.kt) && l.shares_w == 1; }

CeLayout ce_layout(int64_t M, int64_t V, int64_t d, bool want_dx, bool want_dw) {
    CeLayout l;
    l.few = ce_few_fits(M, V);
    l.few_w = M <= 128;
    l.piece = l.few ? V : std::min(ce_piece(M, V, d), V);
    l.tiles_z = gemm_bf16_grad_fits(M, l.piece, d);
    l.tiles_x = gemm_bf16_grad_fits(M, d, 2 * BK);
    l.shares = !want_dx ? 1 : l.tiles_x ? gemm_bf16_sum_shares(M, d, up64(l.piece) / 64) : ce_few_dx_shares(M, l.piece, d);
    l.shares_w = l.few_w || !want_dw || !gemm_bf16_grad_fits(l.piece, d, M) ? 1 : gemm_bf16_sum_shares(l.piece, d, up64(M) / 64);
    l.width = ce_width(l.piece, l.tiles_x ? l.shares : 1);
    l.kt = M <= 32 ? 32 : M <= 64 ? 64 : ce_width(M, l.shares_w);
    const int64_t last = V - (V - 1) / l.piece * l.piece, logits = l.few ? 0 : !l.tiles_z ? l.piece : gemm_bf16_grad_fits(M, last, d) ? 0 : last;
    const int64_t sums_w = !want_dw || l.few_w ? 0 : !ce_dw_stored(l, l.piece, d) ? l.piece : !ce_dw_stored(l, last, d) ? last : 0;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += up256(bytes); return at; };
    l.rowf = take((size_t)M * 4);
    l.scale = take(4);
    l.z = take((size_t)M * logits * 4);
    l.d = take((size_t)M * l.width * 2);
    l.dt = take(want_dw || !l.few ? (size_t)l.piece * l.kt * 2 : 0);
    l.wt = take(want_dx && l.tiles_x ? (size_t)d * l.width * 2 : 0);
    l.sum = take(want_dx ? (size_t)l.shares * M * d * 4 : 0);
    l.wsum = take((size_t)l.shares_w * sums_w * d * 4);
    l.xt = take(want_dw && !l.few_w ? (size_t)d * l.kt * 2 : 0);
    l.total = o;
    return l;
}

CeFlip flip(const bf16_t* x, int64_t ldx, int64_t R, int64_t C, bf16_t* y, int64_t ldy) { return CeFlip{x, ldx, R, C, y, ldy, (ldy + 63) / 64 * ((C + 63) / 64)}; }
CeZero zero_columns(bf16_t* y, int64_t rows, int64_t ld, int64_t from, int64_t to) { return CeZero{y, rows, ld, from, to, from < to ? (rows * (to - from) + 255) / 256 : 0}; }
hipError_t prepare(const CePrepare& a, hipStream_t st) {
    const int64_t blocks = a.count_blocks + a.X.blocks + a.W.blocks + a.D.blocks + a.Dt.blocks;
    if (blocks == 0) return hipSuccess;
    if (blocks > 0x7FFFFFFFLL) return hipErrorInvalidValue;
    hipLaunchKernelGGL(ce_prepare_kernel, dim3((unsigned)blocks), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t product(const bf16_t* x, int64_t ldx, const bf16_t* w, int64_t ldw, int64_t M, int64_t N, int64_t K, float* y, int64_t ldy, hipStream_t st) {
    GemmBf16Args a;
    a.X = x; a.ldx = ldx; a.W = w; a.ldw = ldw; a.M = M; a.N = N; a.K = K; a.Y = y; a.y_dtype = AGZO_F32; a.ldy = ldy;
    a.P = nullptr; a.r = 1; a.eps_signed = 0.f; a.seed = 0;
    a.loss.kind = AGZO_LOSS_NONE; a.loss.target_dtype = 0; a.loss.target = nullptr; a.loss.ldt = 0; a.loss.partials = nullptr;
    return launch_gemm_bf16(a, st);
}

}  // namespace

size_t ce_grad_workspace_bytes(int64_t M, int64_t V, int64_t d, bool want_dx, bool want_dw) { return ce_layout(M, V, d, want_dx, want_dw).total; }

hipError_t launch_ce_grad(const CeGradArgs& a, void* workspace, hipStream_t st) {
    const CeLayout l = ce_layout(a.M, a.V, a.d, a.dX != nullptr, a.dW != nullptr);
    char* ws = static_cast<char*>(workspace);
    float *rowf = reinterpret_cast<float*>(ws + l.rowf), *scale = reinterpret_cast<float*>(ws + l.scale), *z = reinterpret_cast<float*>(ws + l.z);
    bf16_t *D = reinterpret_cast<bf16_t*>(ws + l.d), *Dt = reinterpret_cast<bf16_t*>(ws + l.dt), *Wt = reinterpret_cast<bf16_t*>(ws + l.wt), *Xt = reinterpret_cast<bf16_t*>(ws + l.xt);
    float *sum = reinterpret_cast<float*>(ws + l.sum), *wsum = reinterpret_cast<float*>(ws + l.wsum);
#define CE_TRY(expr)                            \
    do {                                        \
        const hipError_t e__ = (expr);          \
        if (e__ != hipSuccess) return e__;      \
    } while (0)
    if (l.few) {
        CE_TRY(launch_ce_few_d(a.X, a.ldx, a.W, a.ldw, a.M, a.V, a.d, a.ids, a.lse, a.g, scale, D, l.width, a.dW ? Dt : nullptr, l.kt, st));
    }
    for (int64_t v0 = 0; v0 < a.V; v0 += l.piece) {
        const int64_t n = std::min(l.piece, a.V - v0), width = ce_width(n, l.tiles_x ? l.shares : 1);
        const bf16_t* W = a.W + v0 * a.ldw;
        const bool tiles_z = !l.few && gemm_bf16_grad_fits(a.M, n, a.d);
        if (!l.few || (a.dW && !l.few_w)) {
            CePrepare p{a.ids, a.M, a.V, a.g, rowf, scale, !l.few && v0 == 0, {}, {}, {}, {}};
            if (v0 == 0 && a.dW && !l.few_w) p.X = flip(a.X, a.ldx, a.M, a.d, Xt, l.kt);
            if (a.dX && l.tiles_x) p.W = flip(W, a.ldw, n, a.d, Wt, width);
            if (tiles_z && a.dX) p.D = zero_columns(D, a.M, width, n, width);
            if (tiles_z && a.dW) p.Dt = zero_columns(Dt, n, l.kt, a.M, l.kt);
            CE_TRY(prepare(p, st));
        }
        if (l.few) {
            // (D is there)
        } else if (tiles_z) {
            CE_TRY(launch_gemm_bf16_softmax_grad(a.X, a.ldx, W, a.ldw, a.M, n, a.d, v0, a.ids, a.lse, rowf, D, width, Dt, l.kt, st));
        } else {
            CE_TRY(product(a.X, a.ldx, W, a.ldw, a.M, n, a.d, z, n, st));
            hipLaunchKernelGGL(ce_softmax_grad_kernel, dim3((unsigned)(width / 64), (unsigned)(l.kt / 64)), dim3(256), 0, st, z, n, a.M, v0, n, a.ids, a.lse, rowf, D, width, Dt, l.kt);
            CE_TRY(hipGetLastError());
        }
        bf16_t* dW = a.dW ? a.dW + v0 * a.lddw : nullptr;
        const bool few_x = a.dX && !l.tiles_x, few_w = a.dW && l.few_w;
        if (few_x || few_w)
            CE_TRY(launch_ce_few_grad(CeFewGrad{a.M, n, a.d, D, width, W, a.ldw, l.shares, v0 > 0, few_x ? sum : nullptr,
                                                Dt, l.kt, a.X, a.ldx, a.ids, a.V, scale, few_w ? dW : nullptr, a.lddw}, st));
        if (a.dW && !l.few_w) {
            if (ce_dw_stored(l, n, a.d)) {
                CE_TRY(launch_gemm_bf16_scaled(Dt, l.kt, Xt, l.kt, n, a.d, l.kt, scale, dW, a.lddw, st));
            } else {
                const bool fits = gemm_bf16_grad_fits(n, a.d, l.kt / l.shares_w);
                if (fits) CE_TRY(launch_gemm_bf16_sum(Dt, l.kt, Xt, l.kt, n, a.d, l.kt / l.shares_w, l.shares_w, wsum, false, st));
                else CE_TRY(product(Dt, l.kt, Xt, l.kt, n, a.d, l.kt, wsum, a.d, st));
                CE_TRY(join(wsum, fits ? l.shares_w : 1, n, a.d, scale, dW, a.lddw, st));
            }
        }
        if (!a.dX || !l.tiles_x) continue;
        CE_TRY(launch_gemm_bf16_sum(D, width, Wt, width, a.M, a.d, width / l.shares, l.shares, sum, v0 > 0, st));
    }
#undef CE_TRY
    return a.dX ? join(sum, l.shares, a.M, a.d, scale, a.dX, a.lddx, st) : hipSuccess;
}

}  // namespace agzo
