// Norms of queries and keys for each head with the rotation by the token's position, and the gradient, for the attention of packed
// batches (glue_packed.hip).  A head's D values x, gain w, s = 1 / sqrt(mean x^2 + eps):
//     n = w * x * s;     y_i = n_i cos - n_{i + D/2} sin,  y_{i + D/2} = n_{i + D/2} cos + n_i sin,   angle = position * theta^(-2i/D)
// and back, from dy:  dn = the rotation by the opposite angle;  dw = sum over tokens and heads of dn * x s;  with u = dn * w:
//     dx = s (u - x s * mean(u * x s))
// One pass over memory each, bound by HBM.  D / 8 lanes share a head (16-byte accesses); a pair's two values are D / 16 lanes apart.
// The angles of a token serve all of its heads, so a workgroup makes them once, in LDS, from a product and a remainder in fp64: an
// fp32 product is off by position * 2^-24, 0.01 at positions of 10^5.
#include "agzo_internal.h"

namespace agzo {

namespace {

constexpr int NR_WG = 256;

__device__ __forceinline__ void nr_unpack8(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 nr_pack8(const float (&f)[8]) {
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// cosines and sines of `count` tokens from `first` on, [token][D / 2]
template <int D>
__device__ __forceinline__ void make_angles(float2* cs, const int32_t* __restrict__ positions, int64_t first, int count, double log2_theta) {
    for (int i = threadIdx.x; i < count * (D / 2); i += NR_WG) {
        const int t = i / (D / 2), p = i % (D / 2);
        // turns of the circle, without the whole ones
        const double turns = (double)positions[first + t] * (exp2(-2.0 * p / D * log2_theta) * 0.15915494309189533577);
        float sn, c;
        sincospif(2.f * (float)(turns - rint(turns)), &sn, &c);
        cs[i] = make_float2(c, sn);
    }
}

// tokens [tok0, tok0 + count) of one of the two tensors
template <int D>
__device__ __forceinline__ void norm_rope_tokens(const NormRopeSide& a, const float2* cs, int64_t tok0, int count, float eps) {
    constexpr int LANES = D / 8;
    const int grp = threadIdx.x / LANES, j = threadIdx.x % LANES;
    float gain[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) gain[i] = a.gain ? a.gain[8 * j + i] : 1.f;
    const bool first = j < LANES / 2;
    for (int item = grp; item < count * a.heads; item += NR_WG / LANES) {
        const int t = item / a.heads, h = item - t * a.heads;
        float f[8], o[8];
        nr_unpack8(*reinterpret_cast<const uint4*>(a.x + (tok0 + t) * a.ldx + h * D + 8 * j), f);
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(f[i], f[i], ss);
#pragma unroll
        for (int off = LANES / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
        const float scale = rsqrtf(ss * (1.f / D) + eps);
        const float2* ang = cs + t * (D / 2) + 8 * (j % (LANES / 2));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float mine = f[i] * scale * gain[i], other = __shfl_xor(mine, LANES / 2);
            o[i] = fmaf(mine, ang[i].x, first ? -other * ang[i].y : other * ang[i].y);
        }
        *reinterpret_cast<uint4*>(a.y + (tok0 + t) * a.ldy + h * D + 8 * j) = nr_pack8(o);
    }
}

template <int D>
__global__ __launch_bounds__(NR_WG) void norm_rope_kernel(NormRopeSide q, NormRopeSide k, const int32_t* __restrict__ positions, int64_t n, int per_wg,
                                                          float eps, double log2_theta) {
    extern __shared__ float2 nr_angles[];
    const int64_t tok0 = (int64_t)blockIdx.x * per_wg;
    const int count = (int)min((int64_t)per_wg, n - tok0);
    make_angles<D>(nr_angles, positions, tok0, count, log2_theta);
    __syncthreads();
    norm_rope_tokens<D>(q, nr_angles, tok0, count, eps);
    norm_rope_tokens<D>(k, nr_angles, tok0, count, eps);
}

// ... and back; dgain += this thread's share of the gain's gradient
template <int D>
__device__ __forceinline__ void norm_rope_grad_tokens(const NormRopeSide& a, const float2* cs, int64_t tok0, int count, float eps, float (&dgain)[8]) {
    constexpr int LANES = D / 8;
    const int grp = threadIdx.x / LANES, j = threadIdx.x % LANES;
    float gain[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) gain[i] = a.gain ? a.gain[8 * j + i] : 1.f;
    const bool first = j < LANES / 2;
    for (int item = grp; item < count * a.heads; item += NR_WG / LANES) {
        const int t = item / a.heads, h = item - t * a.heads;
        float f[8], d[8];
        nr_unpack8(*reinterpret_cast<const uint4*>(a.x + (tok0 + t) * a.ldx + h * D + 8 * j), f);
        nr_unpack8(*reinterpret_cast<const uint4*>(a.dy + (tok0 + t) * a.lddy + h * D + 8 * j), d);
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(f[i], f[i], ss);
        const float2* ang = cs + t * (D / 2) + 8 * (j % (LANES / 2));
        float ux = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float other = __shfl_xor(d[i], LANES / 2);
            d[i] = fmaf(d[i], ang[i].x, first ? other * ang[i].y : -other * ang[i].y);
            ux = fmaf(d[i] * gain[i], f[i], ux);
        }
#pragma unroll
        for (int off = LANES / 2; off > 0; off >>= 1) { ss += __shfl_xor(ss, off); ux += __shfl_xor(ux, off); }
        const float scale = rsqrtf(ss * (1.f / D) + eps), back = ux * (1.f / D) * scale * scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dgain[i] = fmaf(d[i], f[i] * scale, dgain[i]);
            f[i] = scale * (d[i] * gain[i] - f[i] * back);
        }
        *reinterpret_cast<uint4*>(a.y + (tok0 + t) * a.ldy + h * D + 8 * j) = nr_pack8(f);
    }
}

// sums over a workgroup's groups of lanes, in a fixed order, to partial [2][D]
template <int D>
__device__ __forceinline__ void dgain_store(const float (&dgain)[8], float* red, float* __restrict__ to) {
    constexpr int LANES = D / 8, GROUPS = NR_WG / LANES;
    const int grp = threadIdx.x / LANES, j = threadIdx.x % LANES;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) red[grp * D + 8 * j + i] = dgain[i];
    __syncthreads();
    for (int c = threadIdx.x; c < D; c += NR_WG) {
        float s = 0.f;
        for (int g = 0; g < GROUPS; ++g) s += red[g * D + c];
        to[c] = s;
    }
}

template <int D>
__global__ __launch_bounds__(NR_WG) void norm_rope_grad_kernel(NormRopeSide q, NormRopeSide k, const int32_t* __restrict__ positions, int64_t n, int per_wg,
                                                               float eps, double log2_theta, float* __restrict__ partial) {
    extern __shared__ float2 nr_angles[];
    float dq[8] = {}, dk[8] = {};
    for (int64_t tok0 = (int64_t)blockIdx.x * per_wg; tok0 < n; tok0 += (int64_t)gridDim.x * per_wg) {
        const int count = (int)min((int64_t)per_wg, n - tok0);
        make_angles<D>(nr_angles, positions, tok0, count, log2_theta);
        __syncthreads();
        norm_rope_grad_tokens<D>(q, nr_angles, tok0, count, eps, dq);
        norm_rope_grad_tokens<D>(k, nr_angles, tok0, count, eps, dk);
        __syncthreads();
    }
    if (!partial) return;
    float* red = reinterpret_cast<float*>(nr_angles);
    dgain_store<D>(dq, red, partial + (int64_t)blockIdx.x * 2 * D);
    dgain_store<D>(dk, red, partial + (int64_t)blockIdx.x * 2 * D + D);
}

// dgain of q and k: the workgroups' sums, 16 columns a workgroup, 64 threads a column that have eight loads in flight each, in fp64 and a fixed order.  (1024
// sums of 256 columns: 20.7 us with 16 threads a column and a load after the other)
__global__ __launch_bounds__(1024) void norm_rope_dgain_kernel(const float* __restrict__ partial, int parts, int D, float* __restrict__ dq, float* __restrict__ dk) {
    __shared__ double red[64][17];
    const int c = threadIdx.x % 16, r = threadIdx.x / 16, col = blockIdx.x * 16 + c;
    double s = 0.0;
    for (int p = r; p < parts; p += 64 * 8) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = partial[(int64_t)min(p + 64 * u, parts - 1) * 2 * D + col];
#pragma unroll
        for (int u = 0; u < 8; ++u) s += p + 64 * u < parts ? (double)v[u] : 0.0;
    }
    red[r][c] = s;
    __syncthreads();
    if (r != 0) return;
    for (int i = 1; i < 64; ++i) s += red[i][c];
    float* to = col < D ? dq : dk;
    if (to) to[col < D ? col : col - D] = (float)s;
}

// (few tokens: a workgroup each, for it is latency that counts; more share a workgroup and with it the first loads' latency)
int norm_rope_tokens_per_wg(int64_t n) { return n >= 2048 ? 4 : 1; }
constexpr int kNormRopeGradBlocks = 1024;      // four workgroups to a compute unit
constexpr int64_t kNormRopeTokens = 1 << 25;   // of a launch: one of 2^32 threads and more is cut off without a word

int norm_rope_grad_blocks(int64_t n) {
    const int per = norm_rope_tokens_per_wg(n);
    return (int)std::min<int64_t>((n + per - 1) / per, kNormRopeGradBlocks);
}

}  // namespace

size_t norm_rope_workspace_bytes(int64_t n, int head_dim) { return (size_t)norm_rope_grad_blocks(n) * 2 * head_dim * sizeof(float); }

hipError_t launch_norm_rope(const NormRopeSide& q, const NormRopeSide& k, const int32_t* positions, int64_t n, int head_dim, float eps, float theta, hipStream_t st) {
    if (n == 0) return hipSuccess;
    const int per = norm_rope_tokens_per_wg(n);
    const size_t smem = (size_t)per * head_dim / 2 * sizeof(float2);
    const double l2 = log2((double)theta);
    auto from = [](NormRopeSide a, int64_t t) { a.x += t * a.ldx; a.y += t * a.ldy; return a; };
    for (int64_t t = 0; t < n; t += kNormRopeTokens) {
        const int64_t some = std::min(n - t, kNormRopeTokens);
        const dim3 blocks((unsigned)((some + per - 1) / per));
        if (head_dim == 128) hipLaunchKernelGGL(norm_rope_kernel<128>, blocks, dim3(NR_WG), smem, st, from(q, t), from(k, t), positions + t, some, per, eps, l2);
        else if (head_dim == 64) hipLaunchKernelGGL(norm_rope_kernel<64>, blocks, dim3(NR_WG), smem, st, from(q, t), from(k, t), positions + t, some, per, eps, l2);
        else return hipErrorInvalidValue;
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_norm_rope_grad(const NormRopeSide& q, const NormRopeSide& k, const int32_t* positions, int64_t n, int head_dim, float eps, float theta,
                                 float* dq_gain, float* dk_gain, void* workspace, hipStream_t st) {
    if (head_dim != 128 && head_dim != 64) return hipErrorInvalidValue;
    const int per = norm_rope_tokens_per_wg(n), blocks = n ? norm_rope_grad_blocks(n) : 0;
    const double l2 = log2((double)theta);
    float* partial = dq_gain || dk_gain ? static_cast<float*>(workspace) : nullptr;
    // (the angles, and after them the groups' sums: 256 threads of eight)
    const size_t smem = std::max((size_t)per * head_dim / 2 * sizeof(float2), (size_t)NR_WG * 8 * sizeof(float));
    if (blocks > 0) {
        if (head_dim == 128) hipLaunchKernelGGL(norm_rope_grad_kernel<128>, dim3(blocks), dim3(NR_WG), smem, st, q, k, positions, n, per, eps, l2, partial);
        else hipLaunchKernelGGL(norm_rope_grad_kernel<64>, dim3(blocks), dim3(NR_WG), smem, st, q, k, positions, n, per, eps, l2, partial);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!dq_gain && !dk_gain) return hipSuccess;
    hipLaunchKernelGGL(norm_rope_dgain_kernel, dim3(2 * head_dim / 16), dim3(1024), 0, st, partial, blocks, head_dim, dq_gain, dk_gain);
    return hipGetLastError();
}

}  // namespace agzo
